// Attention over shared pages of a bf16 cache: the kernels' instances.
#include "attend_device.h"

namespace si {
namespace {

template <int D> hipError_t both(const AttendArgs& shared, const AttendArgs& own, hipStream_t stream) {
  const hipError_t e = launch<SI_KV_BF16, D, ATTEND_SHARED>(shared, stream);
  return e != hipSuccess ? e : launch<SI_KV_BF16, D, ATTEND_OWN>(own, stream);
}

}  // namespace

hipError_t launch_attend_shared_bf16(const AttendArgs& shared, const AttendArgs& own, hipStream_t stream) {
  switch (shared.c.head_dim) {
    case 64: return both<64>(shared, own, stream);
    case 96: return both<96>(shared, own, stream);
    case 128: return both<128>(shared, own, stream);
    case 192: return both<192>(shared, own, stream);
    default: return both<256>(shared, own, stream);
  }
}

}  // namespace si
