// The linear operators' kernels for f16 elements.
#include "gemm.h"

namespace gsr {
template struct LinearOps<f16>;
}
