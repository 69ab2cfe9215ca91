// The kernels of a mixture's layers for bf16 elements.
#include "experts.h"

namespace gsr {
template struct MixtureOps<bf16>;
}
