// Attention over shared pages of a bf16 cache: the kernels' instances.
#include <algorithm>

#include "attend_wide.h"

namespace si {

hipError_t launch_attend_pieces_bf16(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch_pieces<SI_KV_BF16, 64>(g, stream);
    case 96: return launch_pieces<SI_KV_BF16, 96>(g, stream);
    case 128: return launch_pieces<SI_KV_BF16, 128>(g, stream);
    case 192: return launch_pieces<SI_KV_BF16, 192>(g, stream);
    default: return launch_pieces<SI_KV_BF16, 256>(g, stream);
  }
}

}  // namespace si
