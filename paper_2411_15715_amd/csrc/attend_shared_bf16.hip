// Attention over shared pages of a bf16 cache: the kernels' instances.
#include "attend_device.h"

namespace si {

hipError_t launch_attend_pieces_bf16(const AttendArgs& g, hipStream_t stream) {
  switch (g.c.head_dim) {
    case 64: return launch<SI_KV_BF16, 64, ATTEND_PIECES>(g, stream);
    case 96: return launch<SI_KV_BF16, 96, ATTEND_PIECES>(g, stream);
    case 128: return launch<SI_KV_BF16, 128, ATTEND_PIECES>(g, stream);
    case 192: return launch<SI_KV_BF16, 192, ATTEND_PIECES>(g, stream);
    default: return launch<SI_KV_BF16, 256, ATTEND_PIECES>(g, stream);
  }
}

}  // namespace si
