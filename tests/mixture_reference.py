"""Codebook lookups, routing and moving rows to experts in plain form on the CPU: integers as they have to be, numbers
in 64 bits."""
import torch


def sort_rows(group_of, groups):
    """order, sorted, place and offsets of the positions by their group."""
    flat = group_of.reshape(-1).long().cpu()
    key = torch.where((flat < 0) | (flat >= groups), groups, flat)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel())
    place[key == groups] = -1
    offsets = torch.searchsorted(key[order], torch.arange(groups + 1))
    return order, key[order], place, offsets


def embedding_grad(dy, index, entries, scale):
    """The gradient, and the sums of magnitudes and the numbers of rows that its errors are measured by."""
    index = index.long().cpu()
    keep = (index >= 0) & (index < entries)
    zero = torch.zeros(entries, dy.shape[1], dtype=torch.float64)
    d = dy.double().cpu()[keep]
    total, size = zero.index_add(0, index[keep], d), zero.index_add(0, index[keep], d.abs())
    return total * scale, size * abs(scale), torch.bincount(index[keep], minlength=entries)


def route(logits, k, normalise):
    """Experts and weights of each row, one choice after the other."""
    l = logits.double().cpu()
    rows, experts = l.shape
    expert, weight = torch.full((rows, k), -1), torch.zeros(rows, k, dtype=torch.float64)
    for r in range(rows):
        # undefined ones first, then the largest, the lowest expert of equals
        ranked = sorted((not torch.isnan(v), -v.item() if not torch.isnan(v) else 0.0, e) for e, v in enumerate(l[r])
                        if v != -torch.inf)
        chosen = [e for _, _, e in ranked[:k]]
        if not chosen:
            continue
        expert[r, :len(chosen)] = torch.tensor(chosen)
        of = l[r, chosen] if normalise else l[r]
        p = torch.exp(l[r, chosen] - l[r, chosen[0]]) / torch.exp(of - l[r, chosen[0]]).sum()
        weight[r, :len(chosen)] = p
    return expert, weight


def route_grad(dweight, logits, expert, normalise):
    """The gradient of sum(dweight * weight) by automatic differentiation of the softmax."""
    l = logits.double().cpu().clone().requires_grad_()
    loss = torch.zeros((), dtype=torch.float64)
    for r in range(l.shape[0]):
        at = [(j, e) for j, e in enumerate(expert[r].tolist()) if e >= 0]
        if not at:
            continue
        chosen = torch.tensor([e for _, e in at])
        p = torch.softmax(l[r, chosen], 0) if normalise else torch.softmax(l[r], 0)[chosen]
        loss = loss + (p * dweight[r, [j for j, _ in at]].double().cpu()).sum()
    if not loss.requires_grad:
        return torch.zeros_like(l)
    return torch.autograd.grad(loss, l)[0]


def gathered(rows, place, k):
    """Rows at the places of each row's choices, [rows][k][dim], zero where there is none."""
    at = place.long().cpu().view(-1, k)
    v = rows.double().cpu()[at.clamp(min=0)]
    return torch.where((at < 0).unsqueeze(2), 0.0, v)
