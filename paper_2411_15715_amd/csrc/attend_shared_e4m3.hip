// Attention over shared pages of an e4m3 cache: the kernels' instances.
#include "attend_device.h"

namespace si {

hipError_t launch_attend_pieces_e4m3(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch<SI_KV_E4M3, 64, ATTEND_PIECES>(g, stream);
    case 128: return launch<SI_KV_E4M3, 128, ATTEND_PIECES>(g, stream);
    case 192: return launch<SI_KV_E4M3, 192, ATTEND_PIECES>(g, stream);
    default: return launch<SI_KV_E4M3, 256, ATTEND_PIECES>(g, stream);
  }
}

}  // namespace si
