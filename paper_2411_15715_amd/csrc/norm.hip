// Residual step between two blocks of a Transformer layer: r' = a r + b gate * N1(y), out = N2(r'), one pass over the rows.
// A row lives in the registers of the threads that share it (8 consecutive elements a slot, up to 4 slots a thread), so r, y and gate
// are read once and r' and out written once whatever the norms are; the second moment of N_mean is taken about the mean, in a
// second sweep over the registers, as a difference of sums would cancel where the mean is large.
#include "si_internal.h"
#include "si_error.h"
#include "scheinfer_attention.h"

#include <algorithm>
#include <cmath>

namespace si {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));  // rows of an odd width start at any element: the vector loads of this GPU take
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));  // any address, and an unaligned one costs less than eight loads of an element
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int WAVE = 64;
constexpr int SLOT = 8;  // elements of a thread that are next to each other

struct Raw { u32x4 v[2]; };  // 8 elements as loaded (bf16: in v[0])

__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// elements at .. at + 7 of a row of d, zeros beyond it.  No conversion here, so that all loads of a thread are on their way together
__device__ __forceinline__ Raw load_raw(const void* base, int64_t at, int left, int type) {
  Raw x{};
  if (type == SI_BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (left >= SLOT) {
      x.v[0] = *reinterpret_cast<const u32x4_a2*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) x.v[0][i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    }
  } else {
    const uint32_t* p = static_cast<const uint32_t*>(base) + at;
    if (left >= SLOT) {
      x.v[0] = *reinterpret_cast<const u32x4_a4*>(p);
      x.v[1] = *reinterpret_cast<const u32x4_a4*>(p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) x.v[i / 4][i % 4] = p[i];
    }
  }
  return x;
}

__device__ __forceinline__ void widen(const Raw& x, int type, float (&f)[SLOT]) {
  if (type == SI_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(x.v[0][i] << 16); f[2 * i + 1] = __uint_as_float(x.v[0][i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < SLOT; ++i) f[i] = __uint_as_float(x.v[i / 4][i % 4]);
  }
}

__device__ __forceinline__ void store8(void* base, int64_t at, int left, int type, const float (&f)[SLOT]) {
  if (type == SI_BF16) {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    if (left >= SLOT) {
      *reinterpret_cast<u32x4_a2*>(p) = u32x4{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) p[i] = bf16_bits(f[i]);
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (left >= SLOT) {
      *reinterpret_cast<u32x4_a4*>(p) = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4*>(&f[0]));
      *reinterpret_cast<u32x4_a4*>(p + 4) = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4*>(&f[4]));
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) p[i] = f[i];
    }
  }
}

// Sum over the threads of a row: P < 64 neighbouring lanes of a wave, or (P == 0) all waves of the block.  `slot` is a pair of floats per
// wave that no sum of this row or the one before uses: one barrier a sum.
template <int P> __device__ __forceinline__ float row_sum(float v, float* slot) {
#pragma unroll
  for (int m = (P ? P : WAVE) / 2; m > 0; m /= 2) v += __shfl_xor(v, m);
  if constexpr (P == 0) {
    const int waves = blockDim.x / WAVE;
    if (waves > 1) {
      if (threadIdx.x % WAVE == 0) slot[threadIdx.x / WAVE] = v;
      __syncthreads();
      v = 0.f;
      for (int w = 0; w < waves; ++w) v += slot[w];
    }
  }
  return v;
}

constexpr int MAX_WAVES = 16;
struct NormLds { float sum[2][4][MAX_WAVES]; };

template <int P, int N>
__device__ __forceinline__ void normalise(float (&x)[N][SLOT], int kind, int d, int tid, int threads, float eps, const Raw (&w)[N], const Raw (&b)[N],
                                          bool has_w, bool has_b, int w_type, float* s0, float* s1) {
  float t = 0.f;
  if (kind == SI_NORM_MEAN) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < SLOT; ++i) t += x[n][i];
    const float mu = row_sum<P>(t, s0) / (float)d;
    t = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int left = d - SLOT * (tid + n * threads);
#pragma unroll
      for (int i = 0; i < SLOT; ++i) x[n][i] = i < left ? x[n][i] - mu : 0.f;
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < SLOT; ++i) t = fmaf(x[n][i], x[n][i], t);
  const float rs = rsqrtf(row_sum<P>(t, s1) / (float)d + eps);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float f[SLOT], g[SLOT];
    widen(w[n], w_type, f);
    widen(b[n], w_type, g);
#pragma unroll
    for (int i = 0; i < SLOT; ++i) {
      float v = x[n][i] * rs;
      if (has_w) v *= f[i];
      if (has_b) v += g[i];
      x[n][i] = v;
    }
  }
}

// P > 0: P neighbouring lanes share a row (d <= 8 P); P == 0: the block does, N slots a thread.
template <int P, int N> __global__ __launch_bounds__(P ? 256 : 1024) void k_norm(si_norm_t a) {
  __shared__ NormLds s;
  const int threads = P ? P : (int)blockDim.x, tid = P ? (int)threadIdx.x % P : (int)threadIdx.x;
  const int per_block = P ? (int)blockDim.x / P : 1, d = a.d;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * per_block + (P ? threadIdx.x / P : 0); row < a.rows; row += (int64_t)gridDim.x * per_block, turn ^= 1) {
    Raw y[N], r[N], g[N], w1[N], b1[N], w2[N], b2[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = SLOT * (tid + n * threads), left = d - at;
      y[n] = r[n] = g[n] = w1[n] = b1[n] = w2[n] = b2[n] = Raw{};
      if (left > 0) {
        if (a.y) y[n] = load_raw(a.y, row * a.y_stride + at, left, a.y_type);
        if (a.r) r[n] = load_raw(a.r, row * a.r_stride + at, left, a.r_type);
        if (a.y && a.gate) g[n] = load_raw(a.gate, row * a.gate_stride + at, left, a.gate_type);
        if (a.post && a.w_post) w1[n] = load_raw(a.w_post, at, left, a.w_type);
        if (a.post && a.b_post) b1[n] = load_raw(a.b_post, at, left, a.w_type);
        if (a.pre && a.w_pre) w2[n] = load_raw(a.w_pre, at, left, a.w_type);
        if (a.pre && a.b_pre) b2[n] = load_raw(a.b_pre, at, left, a.w_type);
      }
    }
    float x[N][SLOT];
    if (a.y) {
#pragma unroll
      for (int n = 0; n < N; ++n) widen(y[n], a.y_type, x[n]);
      if (a.post) normalise<P, N>(x, a.post, d, tid, threads, a.eps, w1, b1, a.w_post, a.b_post, a.w_type, s.sum[turn][0], s.sum[turn][1]);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float f[SLOT];
        widen(g[n], a.gate_type, f);
#pragma unroll
        for (int i = 0; i < SLOT; ++i) x[n][i] = a.y_scale * (a.gate ? x[n][i] * f[i] : x[n][i]);
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float f[SLOT];
      widen(r[n], a.r_type, f);
#pragma unroll
      for (int i = 0; i < SLOT; ++i) {
        if (!a.y) x[n][i] = a.res_scale * f[i];
        else if (a.r) x[n][i] = fmaf(a.res_scale, f[i], x[n][i]);
      }
      // (b_post moves the elements beyond the row's end away from 0: they are in the sums of N2)
      const int at = SLOT * (tid + n * threads), left = d - at;
#pragma unroll
      for (int i = 0; i < SLOT; ++i) x[n][i] = i < left ? x[n][i] : 0.f;
      if (a.r_out && left > 0) store8(a.r_out, row * a.r_out_stride + at, left, a.r_out_type, x[n]);
    }
    if (a.out) {
      if (a.pre) normalise<P, N>(x, a.pre, d, tid, threads, a.eps, w2, b2, a.w_pre, a.b_pre, a.w_type, s.sum[turn][2], s.sum[turn][3]);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int at = SLOT * (tid + n * threads), left = d - at;
        if (left > 0) store8(a.out, row * a.out_stride + at, left, a.out_type, x[n]);
      }
    }
  }
}

template <int P, int N> hipError_t launch(const si_norm_t& a, int threads, int per_block, hipStream_t stream) {
  const int64_t blocks = ((int64_t)a.rows + per_block - 1) / per_block;
  hipLaunchKernelGGL((k_norm<P, N>), dim3((unsigned)std::min<int64_t>(blocks, 65536)), dim3(threads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_norm(const si_norm_t& a, hipStream_t stream) {
  const int slots = (a.d + SLOT - 1) / SLOT;
  if (slots <= 8) return launch<8, 1>(a, 256, 32, stream);
  if (slots <= 16) return launch<16, 1>(a, 256, 16, stream);
  if (slots <= 32) return launch<32, 1>(a, 256, 8, stream);
  if (slots <= 64) return launch<64, 1>(a, 256, 4, stream);
  auto threads = [&](int n) { return (slots + WAVE * n - 1) / (WAVE * n) * WAVE; };
  const int n = slots <= 512 ? 1 : slots <= 2048 ? 2 : 4;
  if (n == 1) return launch<0, 1>(a, threads(1), 1, stream);
  if (n == 2) return launch<0, 2>(a, threads(2), 1, stream);
  return launch<0, 4>(a, threads(4), 1, stream);
}

bool type_ok(int t) { return t == SI_F32 || t == SI_BF16; }
bool misaligned(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == SI_BF16 ? 1 : 3)) != 0; }

}  // namespace
}  // namespace si

extern "C" int si_norm(const si_norm_t* a, void* stream) {
  using namespace si;
  if (!a) return set_error(SI_EINVAL, "si_norm: descriptor is NULL");
  if (!a->r && !a->y) return set_error(SI_EINVAL, "si_norm: neither r nor y");
  if (!a->r_out && !a->out) return set_error(SI_EINVAL, "si_norm: neither r_out nor out");
  if (a->rows < 0 || a->d < 1 || a->d > SI_NORM_MAX_D) return set_error(SI_EINVAL, "si_norm: bad rows=%d or d=%d (1 .. %d)", a->rows, a->d, SI_NORM_MAX_D);
  if (!std::isfinite(a->eps) || a->eps < 0.f) return set_error(SI_EINVAL, "si_norm: eps has to be finite and not negative");
  for (int k : {a->post, a->pre})
    if (k != SI_NORM_NONE && k != SI_NORM_RMS && k != SI_NORM_MEAN) return set_error(SI_EINVAL, "si_norm: unknown norm %d", k);
  if (a->post != SI_NORM_NONE && !a->y) return set_error(SI_EINVAL, "si_norm: post normalises y, which is NULL");
  const struct { const char* name; const void* p; int type; int64_t stride; bool output; } ops[] = {
      {"r", a->r, a->r_type, a->r_stride, false}, {"y", a->y, a->y_type, a->y_stride, false}, {"gate", a->gate, a->gate_type, a->gate_stride, false},
      {"w_post", a->w_post, a->w_type, 0, false}, {"b_post", a->b_post, a->w_type, 0, false}, {"w_pre", a->w_pre, a->w_type, 0, false},
      {"b_pre", a->b_pre, a->w_type, 0, false}, {"r_out", a->r_out, a->r_out_type, a->r_out_stride, true}, {"out", a->out, a->out_type, a->out_stride, true}};
  for (const auto& o : ops) {
    if (!o.p) continue;
    if (!type_ok(o.type)) return set_error(SI_EINVAL, "si_norm: unknown type %d of %s", o.type, o.name);
    if (misaligned(o.p, o.type)) return set_error(SI_EINVAL, "si_norm: %s is not aligned to its type", o.name);
    if (o.stride < (o.output ? a->d : 0)) return set_error(SI_EINVAL, "si_norm: stride %lld of %s", (long long)o.stride, o.name);
  }
  if (a->rows == 0) return SI_OK;
  const hipError_t e = launch_norm(*a, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "norm launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
