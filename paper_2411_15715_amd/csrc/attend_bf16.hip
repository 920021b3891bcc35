// Attention over a bf16 cache: the kernels' instances (a file for each type, so that they are compiled side by side).
#include "attend_device.h"

namespace si {

hipError_t launch_attend_bf16(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch<SI_KV_BF16, 64>(g, stream);
    case 96: return launch<SI_KV_BF16, 96>(g, stream);
    case 128: return launch<SI_KV_BF16, 128>(g, stream);
    case 192: return launch<SI_KV_BF16, 192>(g, stream);
    default: return launch<SI_KV_BF16, 256>(g, stream);
  }
}

}  // namespace si
