// The linear operators' kernels for f16 elements.
#include "narrow.h"

namespace gsr {
template struct LinearOps<f16>;
template struct NarrowOps<f16>;
}
