// The linear operators' kernels for f32 elements.
#include "gemm.h"

namespace gsr {
template struct LinearOps<float>;
}
