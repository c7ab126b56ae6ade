#include "routed_launch.h"

namespace gemm_gfx950 {
ROUTED_FORMS(, __bf16, __bf16)
}
