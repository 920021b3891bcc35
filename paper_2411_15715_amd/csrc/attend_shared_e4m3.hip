// Attention over shared pages of an e4m3 cache: the kernels' instances.
#include <algorithm>

#include "attend_wide.h"

namespace si {

hipError_t launch_attend_pieces_e4m3(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch_pieces<SI_KV_E4M3, 64>(g, stream);
    case 128: return launch_pieces<SI_KV_E4M3, 128>(g, stream);
    case 192: return launch_pieces<SI_KV_E4M3, 192>(g, stream);
    default: return launch_pieces<SI_KV_E4M3, 256>(g, stream);
  }
}

}  // namespace si
