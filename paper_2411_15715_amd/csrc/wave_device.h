// Sums over the lanes of a wave, and its accesses to LDS (hipcc only).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace si {

// LDS of a wave: its accesses are in order, only the compiler has to keep it
__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ uint64_t composite(uint32_t hi, uint32_t lo) { return (uint64_t)hi << 32 | lo; }

// Steps over the lanes of a wave in registers (by way of LDS each waits some hundred cycles).  MASK: rows of 16 lanes that take part, 0 elsewhere
template <int CTRL, int MASK = 0xf> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, MASK, 0xf, false); }
template <int CTRL, int MASK = 0xf> __device__ __forceinline__ uint64_t moved(uint64_t v) {
  return composite(moved<CTRL, MASK>((uint32_t)(v >> 32)), moved<CTRL, MASK>((uint32_t)v));
}
template <int CTRL> __device__ __forceinline__ double moved(double v) { return __longlong_as_double((long long)moved<CTRL>((uint64_t)__double_as_longlong(v))); }
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane) { return composite(of_lane((uint32_t)(v >> 32), lane), of_lane((uint32_t)v, lane)); }
__device__ __forceinline__ double of_lane(double v, int lane) { return __longlong_as_double((long long)of_lane((uint64_t)__double_as_longlong(v), lane)); }
constexpr int SHIFT = 0x110, TURN = 0x120, FROM_ROW = 0x142, FROM_HALF = 0x143;  // SHIFT, TURN + n: from the lane n before, in rows of 16

// of the lanes up to this one
template <class T> __device__ __forceinline__ T scan_row(T v) {  // of 16
  v += moved<SHIFT + 1>(v);
  v += moved<SHIFT + 2>(v);
  v += moved<SHIFT + 4>(v);
  return v + moved<SHIFT + 8>(v);
}
template <class T> __device__ __forceinline__ T scan_wave(T v) {
  v = scan_row(v);
  v += moved<FROM_ROW, 0xa>(v);
  return v + moved<FROM_HALF, 0xc>(v);
}
template <class T> __device__ __forceinline__ T total_row(T v) {
  v += moved<TURN + 1>(v);
  v += moved<TURN + 2>(v);
  v += moved<TURN + 4>(v);
  return v + moved<TURN + 8>(v);
}
// the same in all lanes (of doubles, whose sums depend on their order, those of the lanes of one row after the other)
template <class T> __device__ __forceinline__ T wave_total(T v) {
  v = total_row(v);
  return (of_lane(v, 0) + of_lane(v, 16)) + (of_lane(v, 32) + of_lane(v, 48));
}

}  // namespace si
