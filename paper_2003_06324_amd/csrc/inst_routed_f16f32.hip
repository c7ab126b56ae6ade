#include "routed_launch.h"

namespace gemm_gfx950 {
ROUTED_FORMS(, _Float16, float)
}
