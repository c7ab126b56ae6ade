#include "routed_launch.h"

namespace gemm_gfx950 {
ROUTED_TYPES(, __bf16)
}
