// The linear operators' kernels for bf16 elements.
#include "gemm.h"

namespace gsr {
template struct LinearOps<bf16>;
}
