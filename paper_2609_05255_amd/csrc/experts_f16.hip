// The kernels of a mixture's layers for f16 elements.
#include "experts.h"

namespace gsr {
template struct MixtureOps<f16>;
}
