"""A codebook's codes are its own: forward and backward are of the same codes, whatever becomes of the tensor that they
came from, and codes that are refused leave it as it was. Against float64 with the bounds of the lookup's own tests."""
import pytest
import torch

from mixture_reference import embedding_grad
from paper_2609_05255_amd import gsraster as gs
from paper_2609_05255_amd.decoder import Codebook
from rows_reference import UNIT, assert_close, sum_bound

pytestmark = pytest.mark.gpu

N, ENTRIES, DIM, SCALE = 3000, 50, 24, 1.5


def make_codes(seed, n=N):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-1, ENTRIES, (n,), generator=g, device="cuda").int()


def gradient_of(seed, n=N):
    return torch.randn(n, DIM, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").half()


def check(book, codes, x, grad, dx):
    """x and the table's gradient are those of `codes`."""
    table, i = book.half.double(), codes.long()
    want = torch.where((i >= 0)[:, None], table[i.clamp(min=0)] * SCALE, 0.0)
    assert_close("embeddings", x, want, 2.0 ** -24 * want.abs(), torch.float16)
    want, size, rows = embedding_grad(dx, codes, ENTRIES, SCALE)
    # (fp32 sums of binary16 values, and one product with the scale)
    assert_close("gradient", grad, want, sum_bound(int(rows.max())) * size + 2 * UNIT[torch.float32] * want.abs(),
                 torch.float32)


def step(book, dx, stream=None):
    x = book.forward(stream)
    return x, book.backward(dx, stream)


@pytest.mark.parametrize("n", [1, 77, N, 20_000])
def test_the_callers_codes_may_change(n):
    codes, dx = make_codes(1, n), gradient_of(2, n)
    book = Codebook(codes, ENTRIES, DIM, SCALE)
    kept = codes.clone()
    codes.copy_(make_codes(3, n))   # the caller's tensor serves another purpose
    check(book, kept, *step(book, dx), dx)
    book.set_codes(codes)
    new = codes.clone()
    codes.fill_(-1)
    check(book, new, *step(book, dx), dx)


def test_codes_written_in_the_book():
    """The book's own codes written in place, as any tensor is: the next forward sorts them again."""
    book, dx = Codebook(make_codes(1), ENTRIES, DIM, SCALE), gradient_of(2)
    for seed in (4, 5):
        new = make_codes(seed)
        book.codes.copy_(new)
        check(book, new, *step(book, dx), dx)
    book.codes[7:400] = 3
    new = book.codes.clone()
    check(book, new, *step(book, dx), dx)
    # without a change nothing is sorted
    book.order.offsets.fill_(0)
    book.forward()
    assert not book.order.offsets.any()


def test_codes_cannot_be_replaced_unsorted():
    book = Codebook(make_codes(1), ENTRIES, DIM, SCALE)
    with pytest.raises(AttributeError):
        book.codes = make_codes(2)


@pytest.mark.parametrize("shape", [(N, 1), (1, N), (30, N // 30)])
def test_codes_of_any_shape(shape):
    new, dx = make_codes(6), gradient_of(2)
    book = Codebook(make_codes(1).view(shape), ENTRIES, DIM, SCALE)
    book.set_codes(new.view(shape))
    check(book, new, *step(book, dx), dx)
    assert book.codes.shape == (N,)


@pytest.mark.parametrize("bad", [lambda c: c[:-1], lambda c: torch.cat([c, c[:1]]), lambda c: c.long(), lambda c: c.cpu(),
                                 lambda c: torch.stack([c, c], 1)[:, 0], lambda c: c.float()])
def test_refused_codes_change_nothing(bad):
    old, dx = make_codes(1), gradient_of(2)
    book = Codebook(old, ENTRIES, DIM, SCALE)
    with pytest.raises(ValueError):
        book.set_codes(bad(make_codes(7)))
    assert torch.equal(book.codes, old)
    check(book, old, *step(book, dx), dx)


def test_on_another_stream():
    """Codes given on a stream that has them last, and let go of at once."""
    book, dx, s = Codebook(make_codes(1, 20_000), ENTRIES, DIM, SCALE), gradient_of(2, 20_000), torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (s, s.cuda_stream):
        for seed in range(10, 14):
            new = make_codes(seed, 20_000)
            torch.cuda.current_stream().synchronize()
            book.set_codes(new, handle)
            want = make_codes(seed, 20_000)
            del new
            torch.full((20_000,), 1, dtype=torch.int32, device="cuda")
            out = step(book, dx, handle)
            torch.cuda.synchronize()
            check(book, want, *out, dx)


def test_under_inference_mode():
    codes, dx = make_codes(1), gradient_of(2)
    with torch.inference_mode():
        book = Codebook(codes, ENTRIES, DIM, SCALE)
        book.set_codes(make_codes(8))
        check(book, make_codes(8), *step(book, dx), dx)


def test_captured():
    """New codes each step, captured and replayed with eager work between."""
    given, dx, s = make_codes(1), gradient_of(2), torch.cuda.Stream()
    book = Codebook(given, ENTRIES, DIM, SCALE)

    def run():
        book.set_codes(given)
        return step(book, dx)

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        x, grad = run()
    for seed in (21, 22, 23, 24):
        with torch.cuda.stream(s):
            given.copy_(make_codes(seed))
            graph.replay()
        s.synchronize()
        check(book, make_codes(seed), x, grad, dx)
        torch.randn(1000, device="cuda").sum().item()


def test_captured_and_not_yet_run():
    """A capture sorts nothing: forwards beside it are of the codes as they are."""
    book, dx, s = Codebook(make_codes(1), ENTRIES, DIM, SCALE), gradient_of(2), torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(book, dx)
        given, other = make_codes(31), make_codes(32)
        book.codes.copy_(given)   # not sorted yet
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        x, grad = step(book, dx)
    check(book, given, *step(book, dx), dx)
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
        book.set_codes(other)
    check(book, given, *step(book, dx), dx)
    with torch.cuda.stream(s):
        graph.replay()
    s.synchronize()
    check(book, given, x, grad, dx)
