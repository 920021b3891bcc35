// Residual step between two blocks of a Transformer layer: r' = a r + b gate * N1(y), out = N2(r'), one pass over the rows.
// A row lives in the registers of the threads that share it (8 consecutive elements a slot, up to 4 slots a thread), so r, y and gate
// are read once and r' and out written once whatever the norms are; the second moment of N_mean is taken about the mean, in a
// second sweep over the registers, as a difference of sums would cancel where the mean is large.
// Bound by memory: 4096 rows of 6144 (bf16 r, fp32 y, 252 MB) 45.3 us, 5.6 TB/s, above the 5.1 TB/s of a 1 GiB copy, as more of it is read than written; 1931 rows
// of 2049 with both norms and a gate, where a row starts at any element, 14.3 us for 11 at that rate.  One row of 4096: 2.6 us in the kernel.
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

// 8 elements as loaded.  ANY: of a type that the kernel is told at run time
constexpr int ANY = -1;
template <int TYPE> struct Raw { u32x4 v[TYPE == SI_BF16 ? 1 : 2]; };

__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// Elements of a slot.  The last slot of a row whose width is not a multiple of 8 takes the row's last 8 elements: `dup` of them are also in the
// slot before, come out the same there, and are left out of the sums.  (Eight guarded loads of one element each took a row of
// 2049 through seven trips to memory one after the other.)  Rows of fewer than 8 elements are loaded one by one.
struct Slot {
  int at, left, dup;
  bool in;
  __device__ __forceinline__ Slot(int slot, int d) {
    at = SLOT * slot;
    in = at < d;
    dup = 0;
    if (in && at + SLOT > d && d >= SLOT) {
      dup = at + SLOT - d;
      at = d - SLOT;
    }
    left = d - at;
  }
  // sum over the elements of f(element), those of the slot before and those beyond the row's end left out
  template <class F> __device__ __forceinline__ float sum(const F& f) const {
    float t = 0.f;
    if (in) {
      if (dup > 0 || left < SLOT) {
#pragma unroll
        for (int i = 0; i < SLOT; ++i) t = f(i, t, i >= dup && i < left);
      } else {
#pragma unroll
        for (int i = 0; i < SLOT; ++i) t = f(i, t, true);
      }
    }
    return t;
  }
};

// No conversion here, so that all loads of a thread are on their way together.  (What is not loaded stays as it is and is not looked at.)
template <bool SHORT, int TYPE> __device__ __forceinline__ Raw<TYPE> load_raw(const void* base, int64_t at, int left, int type = TYPE) {
  Raw<TYPE> x;
  if constexpr (SHORT) x = Raw<TYPE>{};
  if (TYPE == SI_BF16 || (TYPE == ANY && type == SI_BF16)) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (!SHORT || left >= SLOT) {
      x.v[0] = *reinterpret_cast<const u32x4_a2*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) x.v[0][i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    }
  } else if constexpr (TYPE != SI_BF16) {
    const uint32_t* p = static_cast<const uint32_t*>(base) + at;
    if (!SHORT || left >= SLOT) {
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

template <int TYPE> __device__ __forceinline__ void widen(const Raw<TYPE>& x, float (&f)[SLOT], int type = TYPE) {
  if (TYPE == SI_BF16 || (TYPE == ANY && type == SI_BF16)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(x.v[0][i] << 16); f[2 * i + 1] = __uint_as_float(x.v[0][i] & 0xffff0000u); }
  } else if constexpr (TYPE != SI_BF16) {
#pragma unroll
    for (int i = 0; i < SLOT; ++i) f[i] = __uint_as_float(x.v[i / 4][i % 4]);
  }
}

template <bool SHORT> __device__ __forceinline__ void store8(void* base, int64_t at, int left, int type, const float (&f)[SLOT]) {
  if (type == SI_BF16) {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    if (!SHORT || left >= SLOT) {
      *reinterpret_cast<u32x4_a2*>(p) = u32x4{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) p[i] = bf16_bits(f[i]);
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (!SHORT || left >= SLOT) {
      *reinterpret_cast<u32x4_a4*>(p) = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4*>(&f[0]));
      *reinterpret_cast<u32x4_a4*>(p + 4) = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4*>(&f[4]));
    } else {
#pragma unroll
      for (int i = 0; i < SLOT; ++i)
        if (i < left) p[i] = f[i];
    }
  }
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}
// sum over P neighbouring lanes, the same in all of them, without LDS: lanes 1 and 2 apart, mirrored halves and rows of 16, then rows swapped
template <int P> __device__ __forceinline__ float lanes_sum(float v) {
  v = dpp_add<0xB1>(v);
  v = dpp_add<0x4E>(v);
  v = dpp_add<0x141>(v);
  if constexpr (P >= 16) v = dpp_add<0x140>(v);
  if constexpr (P >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (P >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Sum over the threads of a row: P neighbouring lanes of a wave, or (P == 0) all waves of the block, up to 16.  `slot` is a float per
// wave that no other sum uses: one barrier a sum.
template <int P> __device__ __forceinline__ float row_sum(float v, float* slot) {
  if constexpr (P != 0) return lanes_sum<P>(v);
  v = lanes_sum<WAVE>(v);
  if (threadIdx.x % WAVE == 0) slot[threadIdx.x / WAVE] = v;
  __syncthreads();
  const unsigned i = threadIdx.x % 16;
  return lanes_sum<16>(i < blockDim.x / WAVE ? slot[i] : 0.f);
}

constexpr int MAX_WAVES = 16;
struct NormLds { float sum[4][MAX_WAVES]; };

// A norm's weight and bias of the thread's elements: asked for before the sums, used after them
template <int P, int N> struct Affine {
  Raw<ANY> w[N], b[N];
  const void *w_at, *b_at;
  int type;
  __device__ __forceinline__ Affine(const void* w0, const void* b0, int t, int d, int tid, int threads) : w_at(w0), b_at(b0), type(t) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const Slot k(tid + n * threads, d);
      if (k.in && w_at) w[n] = load_raw<P == 8, ANY>(w_at, k.at, k.left, type);
      if (k.in && b_at) b[n] = load_raw<P == 8, ANY>(b_at, k.at, k.left, type);
    }
  }
};

// mean (0 for SI_NORM_RMS) and 1 / sqrt(second moment about it + eps) of a row
struct Moments { float mu, rs; };
template <int P, int N>
__device__ __forceinline__ Moments moments(const float (&x)[N][SLOT], int kind, int d, int tid, int threads, float eps, float* s0, float* s1) {
  Moments m{0.f, 1.f};
  float t = 0.f;
  if (kind == SI_NORM_MEAN) {
#pragma unroll
    for (int n = 0; n < N; ++n) t += Slot(tid + n * threads, d).sum([&](int i, float v, bool counts) { return v + (counts ? x[n][i] : 0.f); });
    m.mu = row_sum<P>(t, s0) / (float)d;
    t = 0.f;
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
    t += Slot(tid + n * threads, d).sum([&](int i, float v, bool counts) {
      const float z = counts ? x[n][i] - m.mu : 0.f;
      return fmaf(z, z, v);
    });
  m.rs = rsqrtf(row_sum<P>(t, s1) / (float)d + eps);
  return m;
}
template <int P, int N> __device__ __forceinline__ void normalise(float (&x)[N][SLOT], const Moments& m, const Affine<P, N>& a) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float w[SLOT], b[SLOT];
    widen(a.w[n], w, a.type);
    widen(a.b[n], b, a.type);
#pragma unroll
    for (int i = 0; i < SLOT; ++i) {
      float v = (x[n][i] - m.mu) * m.rs;
      if (a.w_at) v *= w[i];
      if (a.b_at) v += b[i];
      x[n][i] = v;
    }
  }
}

// P > 0: P neighbouring lanes share a row (d <= 8 P); P == 0: the block does, N slots a thread.  R, Y: types of r and y.  FULL: with N1 or a
// gate, whose operands take registers of their own.
template <int P, int N, int T, int R, int Y, bool FULL> __global__ __launch_bounds__(T) void k_norm(si_norm_t a, int row0) {
  __shared__ NormLds s;
  const int threads = P ? P : (int)blockDim.x, tid = P ? (int)threadIdx.x % P : (int)threadIdx.x;
  const int per_block = P ? (int)blockDim.x / P : 1, d = a.d;
  const int64_t row = row0 + (int64_t)blockIdx.x * per_block + (P ? threadIdx.x / P : 0);
  if (row >= a.rows) return;
  Raw<Y> y[N];
  Raw<R> r[N];
  Raw<ANY> g[FULL ? N : 1];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const Slot k(tid + n * threads, d);
    if (k.in && a.y) y[n] = load_raw<P == 8, Y>(a.y, row * a.y_stride + k.at, k.left);
    if (k.in && a.r) r[n] = load_raw<P == 8, R>(a.r, row * a.r_stride + k.at, k.left);
    if constexpr (FULL) {
      if (k.in && a.y && a.gate) g[n] = load_raw<P == 8, ANY>(a.gate, row * a.gate_stride + k.at, k.left, a.gate_type);
    }
  }
  float x[N][SLOT];
  if constexpr (FULL) {
    const Affine<P, N> post(a.post ? a.w_post : nullptr, a.post ? a.b_post : nullptr, a.w_type, d, tid, threads);
#pragma unroll
    for (int n = 0; n < N; ++n) widen(y[n], x[n]);
    if (a.post) normalise<P, N>(x, moments<P, N>(x, a.post, d, tid, threads, a.eps, s.sum[0], s.sum[1]), post);
  }
  const Affine<P, N> pre(a.pre ? a.w_pre : nullptr, a.pre ? a.b_pre : nullptr, a.w_type, d, tid, threads);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float f[SLOT], v[SLOT];
    widen(r[n], f);
    if constexpr (!FULL) widen(y[n], x[n]);
    if constexpr (FULL) widen(g[n], v, a.gate_type);
#pragma unroll
    for (int i = 0; i < SLOT; ++i) {
      if (FULL && a.gate) x[n][i] *= v[i];
      // (what is not there is 0 here; 0 times a scale that is not finite must not come in)
      float t = a.y ? a.y_scale * x[n][i] : 0.f;
      if (a.r) t = a.y ? fmaf(a.res_scale, f[i], t) : a.res_scale * f[i];
      x[n][i] = t;
    }
  }
  Moments m{0.f, 1.f};
  const bool normed = a.out && a.pre;
  if (normed) m = moments<P, N>(x, a.pre, d, tid, threads, a.eps, s.sum[2], s.sum[3]);
  // where an output is an input, what two threads read has to be read by both before either stores it (the sums have a barrier)
  else if (P == 0 && d % SLOT != 0) __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const Slot k(tid + n * threads, d);
    if (a.r_out && k.in) store8<P == 8>(a.r_out, row * a.r_out_stride + k.at, k.left, a.r_out_type, x[n]);
  }
  if (a.out) {
    if (normed) normalise<P, N>(x, m, pre);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const Slot k(tid + n * threads, d);
      if (k.in) store8<P == 8>(a.out, row * a.out_stride + k.at, k.left, a.out_type, x[n]);
    }
  }
}

struct Shape { int threads, per_block; };

template <int P, int N, int T> hipError_t launch(const si_norm_t& a, const Shape& h, hipStream_t stream) {
  const bool full = a.post != SI_NORM_NONE || (a.gate && a.y), r16 = a.r_type == SI_BF16, y16 = a.y_type == SI_BF16;
  auto go = [&](auto kernel) {
    const int64_t most = (int64_t)h.per_block * (0xffffffffu / h.threads);  // (a launch has fewer than 2^32 threads)
    for (int64_t row0 = 0; row0 < a.rows; row0 += most) {
      const int64_t rows = std::min<int64_t>(a.rows - row0, most);
      hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + h.per_block - 1) / h.per_block)), dim3(h.threads), 0, stream, a, (int)row0);
    }
  };
  if (full) {
    if (r16 && y16) go(k_norm<P, N, T, SI_BF16, SI_BF16, true>);
    else if (r16) go(k_norm<P, N, T, SI_BF16, SI_F32, true>);
    else if (y16) go(k_norm<P, N, T, SI_F32, SI_BF16, true>);
    else go(k_norm<P, N, T, SI_F32, SI_F32, true>);
  } else {
    if (r16 && y16) go(k_norm<P, N, T, SI_BF16, SI_BF16, false>);
    else if (r16) go(k_norm<P, N, T, SI_BF16, SI_F32, false>);
    else if (y16) go(k_norm<P, N, T, SI_F32, SI_BF16, false>);
    else go(k_norm<P, N, T, SI_F32, SI_F32, false>);
  }
  return hipGetLastError();
}

hipError_t launch_norm(const si_norm_t& a, hipStream_t stream) {
  const int slots = (a.d + SLOT - 1) / SLOT;
  if (slots <= 8) return launch<8, 1, 256>(a, {256, 32}, stream);
  if (slots <= 16) return launch<16, 1, 256>(a, {256, 16}, stream);
  if (slots <= 32) return launch<32, 1, 256>(a, {256, 8}, stream);
  if (slots <= 64) return launch<64, 1, 256>(a, {256, 4}, stream);
  auto shape = [&](int n) { return Shape{(slots + WAVE * n - 1) / (WAVE * n) * WAVE, 1}; };
  // One slot a thread: more threads hold fewer registers each, and more rows are in flight.  Beyond 12 waves a row's barriers leave too little
  // beside it.  25 M elements, bf16 r and fp32 y, us with one slot and with two:
  //   2048 columns 44.5, 45.5 (with N1 45.9, 50.5);  6144 44.7, 46.4 (50.5, 58.5);  6656 47.8, 46.9 (68.9, 58.4);  8192 46.5, 45.9 (63.9, 55.8)
  if (slots <= 768) return launch<0, 1, 768>(a, shape(1), stream);
  if (slots <= 1024) return launch<0, 2, 512>(a, shape(2), stream);
  if (slots <= 2048) return launch<0, 4, 512>(a, shape(4), stream);
  return launch<0, 4, 1024>(a, shape(4), stream);
}

bool type_ok(int t) { return t == SI_F32 || t == SI_BF16; }
bool misaligned(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == SI_BF16 ? 1 : 3)) != 0; }

}  // namespace
}  // namespace si

extern "C" int si_norm(const si_norm_t* a, void* stream) {
  using namespace si;
  if (!a) return set_error(SI_EINVAL, "si_norm: descriptor is NULL");
  if (a->rows < 0 || a->d < 1 || a->d > SI_NORM_MAX_D) return set_error(SI_EINVAL, "si_norm: bad rows=%d or d=%d (1 .. %d)", a->rows, a->d, SI_NORM_MAX_D);
  if (!std::isfinite(a->eps) || a->eps < 0.f) return set_error(SI_EINVAL, "si_norm: eps has to be finite and not negative");
  for (int k : {a->post, a->pre})
    if (k != SI_NORM_NONE && k != SI_NORM_RMS && k != SI_NORM_MEAN) return set_error(SI_EINVAL, "si_norm: unknown norm %d", k);
  if (a->rows == 0) return SI_OK;  // (an empty tensor's address may be NULL)
  if (!a->r && !a->y) return set_error(SI_EINVAL, "si_norm: neither r nor y");
  if (!a->r_out && !a->out) return set_error(SI_EINVAL, "si_norm: neither r_out nor out");
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
    // (an output in an input's place: with another type or stride, elements that other threads have still to read would be written)
    for (const auto& in : ops)
      if (o.output && !in.output && in.p == o.p && (in.type != o.type || (in.stride != o.stride && a->rows > 1)))
        return set_error(SI_EINVAL, "si_norm: %s is at the address of %s, with another type or stride", o.name, in.name);
  }
  const hipError_t e = launch_norm(*a, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "norm launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
