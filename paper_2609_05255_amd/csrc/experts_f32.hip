// The kernels of a mixture's layers for f32 elements.
#include "experts.h"

namespace gsr {
template struct MixtureOps<float>;
}
