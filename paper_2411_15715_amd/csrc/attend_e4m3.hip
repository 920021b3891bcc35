// Attention over an e4m3 cache: the kernels' instances (a file for each type, so that they are compiled side by side).
#include "attend_device.h"

namespace si {

hipError_t launch_attend_e4m3(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch<SI_KV_E4M3, 64>(g, stream);
    case 128: return launch<SI_KV_E4M3, 128>(g, stream);
    case 192: return launch<SI_KV_E4M3, 192>(g, stream);
    default: return launch<SI_KV_E4M3, 256>(g, stream);
  }
}

}  // namespace si
