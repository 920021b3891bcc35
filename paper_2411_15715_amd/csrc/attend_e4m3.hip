// Attention over an e4m3 cache: the kernels' instances (a file for each type, so that they are compiled side by side).
#include "attend_device.h"

namespace si {

hipError_t launch_attend_e4m3(const AttendArgs& g, int nt, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch_rows<SI_KV_E4M3, 64, 4>(g, nt, stream);
    case 128: return launch_rows<SI_KV_E4M3, 128, 4>(g, nt, stream);
    case 192: return launch_rows<SI_KV_E4M3, 192, 2>(g, nt, stream);
    default: return launch_rows<SI_KV_E4M3, 256, 2>(g, nt, stream);
  }
}

}  // namespace si
