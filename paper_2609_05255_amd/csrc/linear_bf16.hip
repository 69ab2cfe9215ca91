// The linear operators' kernels for bf16 elements.
#include "narrow.h"

namespace gsr {
template struct LinearOps<bf16>;
template struct NarrowOps<bf16>;
}
