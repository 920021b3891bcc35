// Attention of a few new tokens over the paged cache: the kernel (hipcc only; instantiated by attend_bf16.hip and attend_e4m3.hip).
//
// The rows of a block are the query heads that share a kv head, for all new tokens: up to 128 of them.  Per cache block of
// B tokens a wave forms S^T = K Q^T (matrix instructions with K as the left operand) and O^T += V^T P^T.  The cache holds K and V in the
// operand order of these instructions, so that 16 bytes a lane and 1 KB in a run are an operand as they come: of up to 16 rows a block from memory
// straight into the registers that multiply, of more by way of a ring in LDS, which the waves share.  The tokens of a K block are placed so that
// the scores a lane receives are those of the tokens whose weights it has to hold for the second product: no score or weight passes
// through LDS or between lanes, only the maximum of a row does.  Running maximum m and sum l (base 2) per row; the waves of a block and the parts of a
// sequence are joined by
//   m = max m_i,  l = sum l_i 2^(m_i - m),  o = sum o_i 2^(m_i - m)
// in the order of the parts, so that the result does not depend on who does it.
// Bound by memory with up to 32 rows of bf16 (131071 positions 85.6 us, 6.3 TB/s; 64 sequences of 1 .. 8000 173 us, 6.2) and one row of e4m3 (32 x 8000 positions
// 87 us, 6.0); with more rows by the waits for LDS and for each other, vector and matrix instructions of two waves a SIMD (96 rows over 16 x 8000 164 us, half
// of the waves' time waiting).
//
// Who does what: the cache blocks of all sequences, one after the other, are cut into G equal slices, and each block of a kv head takes one:
// the end of a sequence, some whole ones, the beginning of another, or a piece from the middle of a long one.  Every compute unit has the
// same to read, however the lengths are spread, and a block leaves at most two unfinished sums.  (64 sequences of 1 .. 8000 positions, measured
// when the choice was made: a block for each sequence 192 us, for each equal part of the longest 178, slices 173.)
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv_layout.h"

namespace si {

constexpr int ATTEND_WAVES = 4;         // of a block
constexpr int ATTEND_THREADS = 64 * ATTEND_WAVES;
constexpr int ATTEND_COUNTERS = 16384;  // sequences times units (kv head, row group) whose parts the last block may join
constexpr int attend_wide_dim(int type) { return type == SI_KV_E4M3 ? 64 : 128; }  // longest heads of which a wave may have 32 rows

struct AttendArgs {
  si_cache_t c;
  si_attend_t a;
  int layer;
  int rows;       // rows of a unit in all: n_new * heads per kv head
  int groups;     // row groups: blocks that share a kv head
  int block_rows; // rows of a block: 16, 32, 64 or 128
  int slices;     // G
  int whole;      // a slice for each sequence instead (short ones: nothing to even out, nothing to join)
  int part_rows;  // rows of a unit that the scratch has room for: min(rows, block_rows)
  int last_joins; // the block that finishes last joins the parts of a sequence; else the join kernel does
  float scale2;   // scale * log2(e)
  uint32_t* count;  // [ATTEND_COUNTERS], of (sequence, unit); 0 between calls
  int2* parted;     // [n][unit] first slice of a sequence and number of them
  float* part;      // [unit][slice][2][part_rows][D + 2]: o, then m, l of each row; first the sum of a sequence that began before the slice
};

hipError_t launch_attend_bf16(const AttendArgs& g, hipStream_t stream);
hipError_t launch_attend_e4m3(const AttendArgs& g, hipStream_t stream);

#if defined(__HIPCC__)
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ bf16x8 operand(const u32x4& v) { return __builtin_bit_cast(bf16x8, v); }
// eight e4m3 codes as bf16 (exact)
__device__ __forceinline__ bf16x8 operand8(uint32_t lo, uint32_t hi) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return operand(r);
}

// over the lanes of a wave that hold the same row (16 apart)
__device__ __forceinline__ float max_of_row(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_row(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 2^x for x <= 0, or an infinity
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// What scores are taken less of: their maximum m, or the largest finite number where that is infinite (infinity less itself would be NaN; this way the
// weights' sum is infinite, as it should be, and the output NaN), or 0 where every weight is 0
__device__ __forceinline__ float finite_base(float m) { return m == -INFINITY ? 0.f : fminf(m, 3.402823466e38f); }
// factor of what was summed with maximum m where it is now m_new: 1 where they are alike, infinite ones too
__device__ __forceinline__ float rescale(float m, float m_new, float base) { return m == m_new ? 1.f : pow2(m - base); }

// Values that other blocks (on other dies, with caches of their own) read within the launch: device-scope accesses go to memory
__device__ __forceinline__ void put2(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Which kv head and row group a block has (blockIdx.x): the last rows, which see most, first, and the heads side by side, on the dies in turn (a prompt of
// 4096 tokens, 32 heads on 8: last rows last, head by head 456 us, this way 276; 8 of 700 138 and 123)
struct Unit { int kv, group; };
__device__ __forceinline__ Unit unit_of(const AttendArgs& g) {
  const int group = blockIdx.x / g.c.n_kv_heads;
  return Unit{(int)blockIdx.x - group * g.c.n_kv_heads, g.groups - 1 - group};
}

// What the new tokens t0 .. t1 of a sequence see, in positions and in blocks of B
struct Span {
  int seq, len, window, first;  // first: where the sight of token 0 ends
  int lo, hi, lo_all, hi_all;   // seen by some of them: [lo, hi), by all of them [lo_all, hi_all)
  int fb, nb;                   // first block and number of them
  int why;
  __device__ __forceinline__ Span(const AttendArgs& g, int seq_i, int t0, int t1, int B) {
    // (scalar loads: nothing in this launch writes the lists)
    typedef const int32_t __attribute__((address_space(4))) constant_t;
    const si_cache_t& c = g.c;
    seq = g.a.seqs ? ((constant_t*)(uintptr_t)g.a.seqs)[seq_i] : seq_i;
    len = 0;
    why = SI_CACHE_BAD_SEQ;
    if (seq >= 0 && seq < c.n_seqs) {
      const int most = c.max_pages * c.page_tokens;
      len = ((constant_t*)(uintptr_t)c.lens)[seq];
      why = len < 0 || len > most ? SI_CACHE_BAD_LEN : 0;
      len = len < 0 ? 0 : min(len, most);
    }
    window = g.a.window < len ? g.a.window : 0;
    first = len - g.a.n_new + 1;
    hi = max(0, first + t1);
    hi_all = max(0, first + t0);
    lo = window ? max(0, first + t0 - window) : 0;
    lo_all = window ? max(0, first + t1 - window) : 0;
    fb = lo / B;
    nb = hi > lo ? (hi + B - 1) / B - fb : 0;
  }
};

// what has been summed over some positions, for 4 elements of a row
struct Sum {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  __device__ __forceinline__ void add(const f32x4& o2, float m2, float l2) {
    const float m_new = fmaxf(m, m2), base = finite_base(m_new), f = rescale(m, m_new, base), h = rescale(m2, m_new, base);
    m = m_new;
    l = l * f + l2 * h;
    o = o * f + o2 * h;
  }
};

__device__ __forceinline__ void write_row(const AttendArgs& g, int seq_i, int kv, int row, int dim, const Sum& s, float scale_v) {
  const int per = g.a.n_heads / g.c.n_kv_heads, j = row / per, head = kv * per + row % per;
  const int64_t r = (int64_t)seq_i * g.a.n_new + j;
  const float inv = s.l == 0.f ? 0.f : scale_v / s.l;
  *reinterpret_cast<u32x2_a2*>(static_cast<uint16_t*>(g.a.out) + r * g.a.out_stride + (int64_t)head * g.c.head_dim + dim) =
      u32x2{bf16_pair(s.o[0] * inv, s.o[1] * inv), bf16_pair(s.o[2] * inv, s.o[3] * inv)};
  if (dim == 0 && g.a.lse) g.a.lse[r * g.a.n_heads + head] = s.l == 0.f ? -INFINITY : (s.m + log2f(s.l)) * 0.69314718055994531f;
}

// s_waitcnt vmcnt(n) alone, n < 64
template <int N> __device__ __forceinline__ void wait_vmcnt() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 0xf) | (((N >> 4) & 3) << 14)); }

// TILES waves of a block have 16 NT rows each and go through the same cache blocks; 4 / TILES streams of them take these in turn.  Alone
// (TILES == 1) a wave loads K and V into its registers, past the caches (131071 positions 86 us, without the hint 97 .. 101).  Several read them from LDS,
// into which the block loads each cache block once, without a detour through registers: S stages of a block for each stream.  (Each
// wave loading for itself, TILES requests for every line at the caches: 24 rows over 16 x 8000 positions 108 us, this way 97.)
// In blocks of 128 rows a wave has 32, in smaller ones 16: two waves with the same cache block hide each other's waits (before the weights had two
// operands, 20 rows of e4m3 over 29 windows of 9000 positions, 32 a wave and a ring for each wave: 113 us, 16: 91).
template <int TYPE, int D, int NT, int TILES> struct Attend {
  static constexpr int ROWS = 16 * NT, BLOCK_ROWS = ROWS * TILES;              // of a wave, of a block
  static constexpr bool RING = TILES > 1;                                     // K and V come by way of LDS
  static constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8, B = 4 * E, J = E / 4;  // J score tiles of 16 tokens
  static constexpr int NL = D / 16;                                           // loads of 16 bytes of K, and of V, a lane and block
  static constexpr int H = E / 8;                                             // operands of 8 elements in 16 bytes
  static constexpr int WAVES = ATTEND_WAVES, THREADS = ATTEND_THREADS;
  static constexpr int PAD = D + 4;                                           // (rows of 16 banks more: the four groups of lanes write side by side)

  // A stage of the ring holds a block for each stream, K and V.  (Two blocks a compute unit, but for 32 rows with heads of 192 and 256; stages of K and of
  // V in turn are twice the barriers: 20 rows of e4m3 over 29 windows of 9000 positions 99 us, this way 91.)
  static constexpr int STREAMS = WAVES / TILES, BLOCK_BYTES = 128 * D, STAGE = STREAMS * BLOCK_BYTES;
  static constexpr int S = STAGE > 27000 ? 2 : STAGE > 20000 ? 3 : 4;
  static constexpr int PIECES = STAGE / 1024 / WAVES;  // loads of a stage by each wave
  // Two waves share a SIMD, with 256 registers each; said to the compiler, it also keeps the accumulators out of the registers that only
  // matrix instructions reach (copies to and fro were a fifth of the loop).  With heads of 192 and 256 a wave of up to 16 rows a block has a SIMD for itself: K
  // and V on their way do not fit half the registers (192: 64 x 4000 positions 132 us spilling, 121 alone; e4m3 300 and 65).  Blocks of 64
  // rows have them in the ring (40 rows over 16 x 8000 positions, 192: 90 us in two, 107 alone, e4m3 77 and 85; 256: 111 and 130, 91 and 102);
  // of those of 32 a unit's LDS holds one.
  static constexpr int WAVES_PER_SIMD = D < 192 || TILES == 4 ? 2 : 1;
  // Heads of 256 of e4m3 without the ring: K and V of two blocks, sums and weights fill the 256 registers that vector instructions reach.  The next K is
  // asked for after the products with V instead of before, and q and the sums are held where only matrix instructions reach them (64 x 4000
  // positions 86 us; else registers are spilled in the loop, and a reload waits for all loads in flight: 223).
  static constexpr bool LEAN = !RING && TYPE == SI_KV_E4M3 && D == 256;

  struct Shared {
    union {
      struct {
        float o[WAVES][ROWS][PAD];
        float m[WAVES][ROWS], l[WAVES][ROWS];
      };
      char ring[RING ? S * STAGE : 16];
    };
    int64_t scan[WAVES];
    int64_t begin;  // of the block's slice, from the first block of its first sequence
    int first;      // that sequence
    uint32_t arrived[2];
    int again;      // RING: some wave's sums are not finite
  };

  // words of 16 bytes of V of this lane (E tokens from t0 on) that lie in [lo, hi)
  static __device__ __forceinline__ u32x4 token_mask(int t0, int lo, int hi) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int e = 0; e < E / 4; ++e) {
        const int t = t0 + i * (E / 4) + e;
        if (t >= lo && t < hi) w[i] |= (E == 8 ? 0xffffu : 0xffu) << (e * (E == 8 ? 16 : 8));
      }
    }
    return w;
  }
  // what is not finite becomes 0
  static __device__ __forceinline__ u32x4 finite_only(const u32x4& v) {
    u32x4 r = v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < E / 4; ++e) {
        const uint32_t all = E == 8 ? 0xffffu << (16 * e) : 0xffu << (8 * e), top = E == 8 ? 0x7f80u << (16 * e) : 0x7fu << (8 * e);
        if ((v[i] & top) == top) r[i] &= ~all;
      }
    return r;
  }
  static __device__ __forceinline__ u32x4 load16(const char* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
  // 1 KB from the lanes' addresses to LDS, on its way until waited for
  static __device__ __forceinline__ void load_lds(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)from, (void __attribute__((address_space(3)))*)to, 16, 0, 2 /* nt */);
  }
  // until no more than the `younger` stages asked for last are on their way
  template <int N> static __device__ __forceinline__ void wait_stage(int younger) {
    if constexpr (N == 0) wait_vmcnt<0>();
    else if (younger >= N) wait_vmcnt<N * PIECES>();
    else wait_stage<N - 1>(younger);
  }
  static __device__ __forceinline__ uint32_t lds_at(const char* p) { return (uint32_t)(uintptr_t)(const char __attribute__((address_space(3)))*)p; }
  // N times 16 bytes of LDS, 256 apart, asked for together.  (Left to the compiler: 40 rows with heads of 192 over 16 x 8000 positions 93 us, this way 90;
  // heads of 64 and 128 alike.)
  template <int N, int OFFSET> static __device__ __forceinline__ void read_lds(uint32_t at, u32x4* v) {
    if constexpr (N == 4)
      asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]) : "v"(at), "i"(OFFSET), "i"(OFFSET + 256), "i"(OFFSET + 512), "i"(OFFSET + 768) : "memory");
    else
      asm volatile("ds_read_b128 %0, %2 offset:%3\n\tds_read_b128 %1, %2 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(v[0]), "=&v"(v[1]) : "v"(at), "i"(OFFSET), "i"(OFFSET + 256) : "memory");
  }
  // the operands of K and of V from the I-th on, in turn to `use(i, operand)`
  template <int I, class F> static __device__ __forceinline__ void each_k(uint32_t at, F use) {
    constexpr int N = J;
    u32x4 v[N];
    read_lds<N, I / J * (4 * B * 16)>(at, v);
#pragma unroll
    for (int k = 0; k < N; ++k) use(I + k, v[k]);
    if constexpr (I + N < NL) each_k<I + N>(at, use);
  }
  template <int I, class F> static __device__ __forceinline__ void each_v(uint32_t at, F use) {
    constexpr int N = NL - I >= 4 ? 4 : 2;
    u32x4 v[N];
    read_lds<N, I * 256>(at, v);
#pragma unroll
    for (int k = 0; k < N; ++k) use(I + k, v[k]);
    if constexpr (I + N < NL) each_v<I + N>(at, use);
  }
  static __device__ __forceinline__ bf16x8 part_of(const u32x4& v, int h) { return E == 8 ? operand(v) : operand8(v[2 * h], v[2 * h + 1]); }

  // sum over the block, and the sum of the threads before this one
  static __device__ __forceinline__ int64_t scan(int64_t v, int64_t& before, Shared& s) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) s.scan[wave] = x;
    __syncthreads();
    int64_t total = 0;
    before = x - v;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += s.scan[w];
      total += s.scan[w];
    }
    return total;
  }

  static __device__ void run(const AttendArgs& g, Shared& s) {
    const int block_row0 = unit_of(g).group * BLOCK_ROWS, row_end = min(g.rows, block_row0 + BLOCK_ROWS);
    if (RING && threadIdx.x == 0) s.again = 0;
    const int n = g.a.n, slice = blockIdx.y, per = g.a.n_heads / g.c.n_kv_heads, t0 = block_row0 / per, t1 = (row_end - 1) / per;
    // The slice: blocks [begin, begin + left) from the first of sequence `i` on.  A sequence of no blocks counts as one, so that somebody
    // writes its rows.
    auto blocks_of = [&](int k) { return (int64_t)max(1, Span(g, k, t0, t1, B).nb); };
    const int mine = (n + THREADS - 1) / THREADS, k0 = min(n, (int)threadIdx.x * mine), k1 = min(n, k0 + mine);  // sequences that a thread counts
    int64_t total, before = 0, counted = 0;
    int i = g.whole ? slice : 0;
    Span sp(g, i, t0, t1, B);
    if (n == 1 || g.whole) {
      total = max(1, sp.nb);
    } else {
      for (int k = k0; k < k1; ++k) counted += blocks_of(k);
      total = scan(counted, before, s);
    }
    const int64_t G = min<int64_t>(g.slices, total);  // (no slice without a block)
    // (quotients by way of double: exact, as the dividends stay below 2^53, n below 2^16, blocks below 2^27, slices below 2^10)
    auto quotient = [](int64_t x, int64_t y) { return (int64_t)((double)x / (double)y); };
    auto slice_end = [&](int w) { return quotient((w + 1) * total, G); };
    auto slice_of = [&](int64_t block) { return (int)quotient((block + 1) * G - 1, total); };  // the one whose end is the first beyond the block
    int64_t begin = 0, left = total;
    if (g.slices > 1 && !g.whole) {
      begin = slice_end(slice - 1);
      left = slice < G ? slice_end(slice) - begin : 0;
    }
    if (n > 1 && !g.whole) {
      if (before <= begin && begin < before + counted)
        for (int k = k0; k < k1; ++k) {
          const int64_t nb = blocks_of(k);
          if (begin < before + nb) { s.first = k; s.begin = begin - before; break; }
          before += nb;
        }
      __syncthreads();
      i = __builtin_amdgcn_readfirstlane(s.first);
      begin = __builtin_amdgcn_readfirstlane((int)s.begin);
    }
    // unfinished sums of the slice, at its begin and at its end: sequence (-1: none), its first slice and their number
    int un_seq[2] = {-1, -1}, un_first[2] = {0, 0}, un_parts[2] = {1, 1};
    for (; left > 0; ++i) {
      if (n > 1 && !g.whole) sp = Span(g, i, t0, t1, B);
      const int nb = max(1, sp.nb), off = (int)begin, take = (int)min<int64_t>(nb - off, left), where_to = take == nb ? -1 : off > 0 ? 0 : 1;
      if (sp.why && off == 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(g.c.status, sp.why);
      part(g, s, sp, i, block_row0, row_end, sp.fb + off, sp.nb > 0 ? sp.fb + off + take : sp.fb, where_to);
      if (g.slices > 1 && !g.whole) {
        const int64_t first_block = slice_end(slice) - left - off;
        const int first = where_to < 0 ? slice : slice_of(first_block), parts = where_to < 0 ? 1 : slice_of(first_block + nb - 1) - first + 1;
        if (where_to == 0) { un_seq[0] = i; un_first[0] = first; un_parts[0] = parts; }
        if (where_to == 1) { un_seq[1] = i; un_first[1] = first; un_parts[1] = parts; }
        if (off == 0 && !g.last_joins && threadIdx.x == 0) g.parted[(int64_t)i * gridDim.x + blockIdx.x] = make_int2(first, parts);
      }
      begin = 0;
      left -= take;
    }
    if (g.last_joins && max(un_seq[0], un_seq[1]) >= 0) {
      // The parts of a sequence: the last block to arrive joins them.  Its own sums have reached memory before it is counted
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (threadIdx.x < 2) {
        const int seq_i = threadIdx.x == 0 ? un_seq[0] : un_seq[1];  // (an index that the compiler knows: no private memory)
        s.arrived[threadIdx.x] = seq_i < 0 ? 0 : __hip_atomic_fetch_add(g.count + seq_i * gridDim.x + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (un_seq[k] >= 0 && s.arrived[k] == (uint32_t)un_parts[k] - 1) {
          if (threadIdx.x == 0) __hip_atomic_store(g.count + un_seq[k] * gridDim.x + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          join(g, un_seq[k], un_first[k], un_parts[k], block_row0, row_end);
        }
    }
  }

  // Blocks [b0, b1) of sequence seq_i; where_to: -1: they are all of it, 0 / 1: the unfinished sum at the slice's begin / end
  static __device__ __forceinline__ void part(const AttendArgs& g, Shared& s, const Span& sp, int seq_i, int block_row0, int row_end, int b0, int b1, int where_to) {
    const si_cache_t& c = g.c;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), grp = lane / 16, col = lane % 16;
    const int kv = unit_of(g).kv, per = g.a.n_heads / c.n_kv_heads, n_new = g.a.n_new;
    // the block has the rows [block_row0, row_end), this wave ROWS of them from row0 on; STREAMS waves take the cache blocks in turn
    const int stream = wave / TILES, row0 = block_row0 + wave % TILES * ROWS;
    const int window = sp.window, first = sp.first, lo = sp.lo, hi = sp.hi, lo_all = sp.lo_all, hi_all = sp.hi_all;

    // this lane's rows of q, as right operands; token of a row, or -1
    int tok[NT];
    u32x4 q[NT][D / 32];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const int row = row0 + 16 * u + col;
      tok[u] = row < row_end ? row / per : -1;
      const uint16_t* p = static_cast<const uint16_t*>(g.a.q) + ((int64_t)seq_i * n_new + row / per) * g.a.q_stride + (int64_t)(kv * per + row % per) * D;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        // operand x of K covers, in this lane, elements 32 x + 8 grp of a head (bf16), or half x % 2 of the 16 from 64 (x / 2) + 16 grp on
        const int dim = E == 8 ? 32 * x + 8 * grp : 64 * (x / 2) + 16 * grp + 8 * (x % 2);
        q[u][x] = tok[u] >= 0 ? u32x4(*reinterpret_cast<const u32x4_a2*>(p + dim)) : u32x4{0, 0, 0, 0};
      }
    }
    if constexpr (LEAN) {
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) asm volatile("" : "+a"(q[u][x]));
    }
    const float sc = g.scale2 * (TYPE == SI_KV_E4M3 && c.scale_k ? c.scale_k[kv] : 1.f);
    const float scale_v = TYPE == SI_KV_E4M3 && c.scale_v ? c.scale_v[kv] : 1.f;

    f32x4 o[NT][NL];
    float m[NT], l[NT];

    // Where a block of the stream lies: entry of the table and place in the page.  The page's number comes by a scalar load, which the loads of K
    // and V in flight have nothing to do with (a vector load in their midst is waited for along with all of them); nothing in this
    // launch writes the table.
    const int32_t* table = c.table + (int64_t)max(sp.seq, 0) * c.max_pages;  // (read where nb > 0 only)
    const int per_page = c.page_tokens / B, last_entry = (b1 - 1) / per_page;
    struct Place { int entry, at; };
    auto page_of = [&](const Place& w) {
      typedef const int32_t __attribute__((address_space(4))) constant_t;
      const int page = ((constant_t*)(uintptr_t)table)[min(w.entry, last_entry)];
      return page >= 0 && page < c.n_pages ? page : -1;
    };
    auto step = [&](Place w, int by) {
      w.at += by;
      while (w.at >= per_page) { w.at -= per_page; ++w.entry; }
      return w;
    };
    constexpr int BYTES = TYPE == SI_KV_E4M3 ? 1 : 2;
    const int64_t page_bytes = kv_page_elems(c) * BYTES;
    const char* k_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 0, kv) * BYTES;
    const char* v_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 1, kv) * BYTES;
    const int k_lane = grp * (B * 16) + col * 16, v_lane = grp * (D * 16) + col * 16;
    const char *k_lds = nullptr, *v_lds = nullptr;  // RING: the block in work
    u32x4 kf[RING ? 1 : NL], vf[RING ? 1 : NL];
    auto load_k = [&](int page, int at) {
      const char* p = k_base + (uint32_t)max(page, 0) * page_bytes + at * (64 * D);
#pragma unroll
      for (int i = 0; i < NL; ++i) kf[i] = load16(p + k_lane + i / J * (4 * B * 16) + i % J * 256);
    };
    auto load_v = [&](int page, int at) {
      const char* p = v_base + (uint32_t)max(page, 0) * page_bytes + at * (64 * D);
#pragma unroll
      for (int i = 0; i < NL; ++i) vf[i] = load16(p + v_lane + i * 256);
    };
    // operands of K and of V, in turn to `use(i, operand)`
    auto k_to = [&](auto use) {
      if constexpr (RING) {
        each_k<0>(lds_at(k_lds) + k_lane, use);
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i) use(i, kf[i]);
      }
    };
    auto v_to = [&](auto use) {
      if constexpr (RING) {
        each_v<0>(lds_at(v_lds) + v_lane, use);
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i) use(i, vf[i]);
      }
    };

    // scores of a block: tile j, element i of this lane is token grp * E + 4 j + i
    f32x4 x[NT][J];
    auto scores = [&] {
      if constexpr (LEAN) {
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int i = 0; i < NL; ++i) asm volatile("" : "+a"(o[u][i]));
      }
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int j = 0; j < J; ++j) x[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      k_to([&](int i, const u32x4& k) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const bf16x8 k8 = part_of(k, h);
#pragma unroll
          for (int u = 0; u < NT; ++u) x[u][i % J] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, operand(q[u][i / J * H + h]), x[u][i % J], 0, 0, 0);
        }
      });
    };
    // weights of the block, and what has been summed brought to its maximum; EDGE: some rows may not see some of its tokens.
    // A weight is the sum of two operands, its rounding to bf16 and that of what the rounding left: 2^-16 of it is lost.  (One operand loses
    // 2^-8 of it, an error relative to sum p |v|, which shows where values cancel.)
    u32x4 p[NT][H], p_rest[NT][H];
    auto weights = [&](auto EDGE, int t0) {
      int mine = t0 + grp * E;  // first token of this lane
      if constexpr (EDGE) asm volatile("" : "+v"(mine));  // (or the tokens of each element are formed before the loop and held through it)
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        float top = -INFINITY;
        const int see_hi = tok[u] >= 0 ? max(0, first + tok[u]) : 0, see_lo = window ? max(0, first + tok[u] - window) : 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = x[u][j][i] * sc;
            if constexpr (EDGE) {
              const int pos = mine + 4 * j + i;
              v = pos >= see_lo && pos < see_hi ? v : -INFINITY;
            }
            x[u][j][i] = v;
            top = fmaxf(top, v);
          }
        const float m_new = fmaxf(m[u], max_of_row(top)), base = finite_base(m_new);
        if (__any(m_new > m[u])) {
          const float f = rescale(m[u], m_new, base);
          l[u] *= f;
#pragma unroll
          for (int i = 0; i < NL; ++i) o[u][i] *= f;
          m[u] = m_new;
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int j = 2 * h + w / 2, i = 2 * (w % 2);
            const float a = pow2(x[u][j][i] - base), e = pow2(x[u][j][i + 1] - base);
            l[u] += a + e;
            uint32_t pair = bf16_pair(a, e);
            asm("" : "+v"(pair));  // (or the first of the pair is rounded once more by itself)
            p[u][h][w] = pair;
            p_rest[u][h][w] = bf16_pair(a - __uint_as_float(pair << 16), e - __uint_as_float(pair & 0xffff0000u));
          }
      }
    };
    auto products = [&](auto EDGE, const u32x4& keep) {
      v_to([&](int i, u32x4 v) {
        if constexpr (EDGE) v &= keep;
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const bf16x8 v8 = part_of(v, h);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            o[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, operand(p_rest[u][h]), o[u][i], 0, 0, 0);
            o[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, operand(p[u][h]), o[u][i], 0, 0, 0);
          }
        }
      });
    };
    // the same where some rows may not see some tokens: what no row sees may be anything (weight 0 times infinity would be NaN)
    auto products_at_edge = [&](int t0) {
      int mine = t0 + grp * E;
      asm volatile("" : "+v"(mine));
      products(std::true_type{}, token_mask(mine, lo, hi));
    };
    auto weigh = [&](int t0) {  // after the scores; the main path and that of the edges
      if (t0 < lo_all || t0 + B > hi_all) {
        weights(std::true_type{}, t0);
        products_at_edge(t0);
      } else {
        weights(std::false_type{}, t0);
        products(std::false_type{}, u32x4{});
      }
    };
    // Blocks with values that are not finite: a product for each of the new tokens, with what it sees alone, and none of such a value with the
    // rest of a weight (which is 0, or of the other sign: infinity times the weight has to stay infinity)
    auto weigh_one_by_one = [&](int t0) {
      weights(std::true_type{}, t0);
      int mine = t0 + grp * E;
      asm volatile("" : "+v"(mine));
#pragma unroll 1
      for (int j = row0 / per; j <= (min(row_end, row0 + ROWS) - 1) / per; ++j) {
        const u32x4 seen = token_mask(mine, window ? max(0, first + j - window) : 0, max(0, first + j));
        v_to([&](int i, u32x4 v) {
          v &= seen;
          const u32x4 v_finite = finite_only(v);
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            f32x4 r = o[u][i];
#pragma unroll
            for (int h = 0; h < H; ++h) {
              r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part_of(v_finite, h), operand(p_rest[u][h]), r, 0, 0, 0);
              r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part_of(v, h), operand(p[u][h]), r, 0, 0, 0);
            }
            if (tok[u] == j) o[u][i] = r;
          }
        });
      }
    };
    auto clear = [&] {
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        m[u] = -INFINITY;
        l[u] = 0.f;
#pragma unroll
        for (int i = 0; i < NL; ++i) o[u][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    // (rows that the call has; what is not finite stays so through every later step, so the end is soon enough to look)
    auto sums_not_finite = [&] {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < NT; ++u)
        if (tok[u] >= 0)
#pragma unroll
          for (int i = 0; i < NL; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = fmaf(o[u][i][e], 0.f, t[e]);
      return (bool)__any(t[0] + t[1] + t[2] + t[3] != 0.f);
    };

    clear();
    bool bad_page = false;
    if constexpr (RING) {
      const int turns = (b1 - b0 + STREAMS - 1) / STREAMS;
      uint32_t missing = 0;  // bit turn * STREAMS + stream, modulo 32: the block's page is not there
      Place front{b0 / per_page, b0 % per_page};
      // (S stages at most hold 4 x 2 bits)
      auto issue = [&](int turn) {
#pragma unroll
        for (int st = 0; st < STREAMS; ++st) {
          const int page = page_of(front);
          const uint32_t bit = 1u << ((turn * STREAMS + st) % 32);
          missing = page < 0 ? missing | bit : missing & ~bit;
          const int64_t at = (uint32_t)max(page, 0) * page_bytes + front.at * (64 * D);
          char* to = s.ring + turn % S * STAGE + st * BLOCK_BYTES;
#pragma unroll
          for (int q4 = 0; q4 < PIECES / STREAMS; ++q4) {
            const int piece = WAVES * q4 + wave;  // of the block: K, then V
            load_lds((piece < D / 16 ? k_base + at + piece * 1024 : v_base + at + (piece - D / 16) * 1024) + lane * 16, to + piece * 1024);
          }
          if (b0 + turn * STREAMS + st < b1 - 1) front = step(front, 1);  // (beyond the last block: that one again)
        }
      };
      for (int turn = 0; turn < min(S - 1, turns); ++turn) issue(turn);
      for (int turn = 0; turn < turns; ++turn) {
        wait_stage<S - 2>(turns - 1 - turn);
        // everybody's loads of this stage have arrived, and what was read of the one before has been used
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int b = b0 + turn * STREAMS + stream;
        const bool here = !(missing >> ((turn * STREAMS + stream) % 32) & 1);
        if (turn + S - 1 < turns) issue(turn + S - 1);
        if (b < b1 && row0 < row_end) {
          bad_page |= !here;
          k_lds = s.ring + turn % S * STAGE + stream * BLOCK_BYTES;
          v_lds = k_lds + 64 * D;
          if (here) {
            scores();
            weigh(b * B);
          }
        }
      }
      if (turns > 0) {
        if (sums_not_finite() && lane == 0) s.again = 1;
        __syncthreads();  // (the ring's memory is used anew)
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(s.again), 0)) {  // once more, as below
          clear();
          front = Place{b0 / per_page, b0 % per_page};
#pragma unroll 1
          for (int turn = 0; turn < turns; ++turn) {
            __syncthreads();
            if (turn == 0 && threadIdx.x == 0) s.again = 0;
            issue(turn);
            wait_vmcnt<0>();
            __syncthreads();
            const int b = b0 + turn * STREAMS + stream;
            if (b < b1 && row0 < row_end && !(missing >> ((turn * STREAMS + stream) % 32) & 1)) {
              k_lds = s.ring + turn % S * STAGE + stream * BLOCK_BYTES;
              v_lds = k_lds + 64 * D;
              scores();
              weigh_one_by_one(b * B);
            }
          }
          __syncthreads();
        }
      }
    } else {
      // K of the next block is asked for when the scores of this one are formed, V when it has been multiplied: 8 to 16 KB of a wave are
      // always on their way (heads of 128).  The last block has no next: written out, so that the loop's loads stand under no condition.
      int b = b0 + stream;
      if (b < b1) {
        const Place here{b / per_page, b % per_page};
        Place next = step(here, STREAMS);
        int page = page_of(here), next_page = page_of(next);
        load_k(page, here.at);
        load_v(page, here.at);
        for (; b + STREAMS < b1; b += STREAMS) {
          const Place after = step(next, STREAMS);
          const int after_page = page_of(after);
          scores();
          if constexpr (!LEAN) load_k(next_page, next.at);
          if (page >= 0) weigh(b * B);  // (a block whose page is not there is passed over)
          if constexpr (LEAN) load_k(next_page, next.at);
          load_v(next_page, next.at);
          bad_page |= page < 0;
          page = next_page;
          next_page = after_page;
          next = after;
        }
        bad_page |= page < 0;
        if (page >= 0) {
          scores();
          weights(std::true_type{}, b * B);
          products_at_edge(b * B);
        }
      }
      // A value that is not finite spoils the sums of rows that do not see it, and its products with the rests of the weights those of rows that do:
      // once more, with an eye on each value.  Rows that see finite values only come out as they would without the others.
      if (__builtin_expect(sums_not_finite(), 0)) {
        clear();
#pragma unroll 1
        for (b = b0 + stream; b < b1; b += STREAMS) {
          const Place here{b / per_page, b % per_page};
          const int page = page_of(here);
          if (page < 0) continue;
          load_k(page, here.at);
          load_v(page, here.at);
          scores();
          weigh_one_by_one(b * B);
        }
      }
    }
    if (bad_page && lane == 0) atomicOr(c.status, SI_CACHE_BAD_PAGE);

    // the streams of the block
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      l[u] = sum_of_row(l[u]);
      if (grp == 0) { s.m[wave][16 * u + col] = m[u]; s.l[wave][16 * u + col] = l[u]; }
#pragma unroll
      for (int i = 0; i < NL; ++i) *reinterpret_cast<f32x4*>(&s.o[wave][16 * u + col][16 * i + 4 * grp]) = o[u][i];
    }
    __syncthreads();
    const int items = (row_end - block_row0) * (D / 4);
    float* sums = g.part + (((int64_t)blockIdx.x * g.slices + blockIdx.y) * 2 + max(where_to, 0)) * (g.part_rows * (D + 2));
    for (int i = threadIdx.x; i < items; i += THREADS) {
      const int r = i / (D / 4), dim = i % (D / 4) * 4;
      Sum sum;
      for (int w = r / ROWS; w < WAVES; w += TILES) sum.add(*reinterpret_cast<const f32x4*>(&s.o[w][r % ROWS][dim]), s.m[w][r % ROWS], s.l[w][r % ROWS]);
      float* to = sums + r * (D + 2);
      if (where_to < 0) {
        write_row(g, seq_i, kv, block_row0 + r, dim, sum, scale_v);
      } else if (g.last_joins) {
        put2(to + dim, sum.o[0], sum.o[1]);
        put2(to + dim + 2, sum.o[2], sum.o[3]);
        if (dim == 0) put2(to + D, sum.m, sum.l);
      } else {
        *reinterpret_cast<float2*>(to + dim) = make_float2(sum.o[0], sum.o[1]);
        *reinterpret_cast<float2*>(to + dim + 2) = make_float2(sum.o[2], sum.o[3]);
        if (dim == 0) *reinterpret_cast<float2*>(to + D) = make_float2(sum.m, sum.l);
      }
    }
    __syncthreads();
  }

  static __device__ __forceinline__ void join(const AttendArgs& g, int seq_i, int first, int parts, int block_row0, int row_end) {
    const int kv = unit_of(g).kv, part_floats = g.part_rows * (D + 2);
    const float* sums = g.part + ((int64_t)blockIdx.x * g.slices + first) * 2 * part_floats;
    for (int i = threadIdx.x; i < (row_end - block_row0) * (D / 4); i += THREADS) {
      const int r = i / (D / 4), dim = i % (D / 4) * 4;
      Sum sum;
      constexpr int AHEAD = 8;  // (a trip to memory is about a microsecond)
      for (int p0 = 0; p0 < parts; p0 += AHEAD) {
        float2 v[AHEAD][3];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int q = min(p0 + k, parts - 1);  // (all but the first hold the sequence from before)
          const float* from = sums + (int64_t)(2 * q + (q == 0 ? 1 : 0)) * part_floats + r * (D + 2);
          v[k][0] = get2(from + dim);
          v[k][1] = get2(from + dim + 2);
          v[k][2] = get2(from + D);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
          if (p0 + k < parts) sum.add(f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y}, v[k][2].x, v[k][2].y);
      }
      write_row(g, seq_i, kv, block_row0 + r, dim, sum, TYPE == SI_KV_E4M3 && g.c.scale_v ? g.c.scale_v[kv] : 1.f);
    }
  }
};

template <int TYPE, int D, int NT, int TILES>
__global__ __launch_bounds__((Attend<TYPE, D, NT, TILES>::THREADS), (Attend<TYPE, D, NT, TILES>::WAVES_PER_SIMD)) void k_attend(AttendArgs g) {
  __shared__ typename Attend<TYPE, D, NT, TILES>::Shared s;
  Attend<TYPE, D, NT, TILES>::run(g, s);
}

// Joins the parts of a sequence: a block has one row, and its threads a share of the parts of 4 elements each.
template <int D> __global__ __launch_bounds__(256) void k_join(AttendArgs g) {
  constexpr int LANES = D / 4, SHARES = 256 / LANES;
  __shared__ f32x4 s_o[SHARES][LANES];
  __shared__ float s_m[SHARES][LANES], s_l[SHARES][LANES];
  const int kv = unit_of(g).kv, seq_i = blockIdx.y, row = unit_of(g).group * g.block_rows + blockIdx.z;
  typedef const int32_t __attribute__((address_space(4))) constant_t;
  const constant_t* parted = (const constant_t*)(uintptr_t)(g.parted + (int64_t)seq_i * gridDim.x + blockIdx.x);
  const int first = parted[0], parts = parted[1];
  if (row >= g.rows || parts == 1) return;  // (one part is written already)
  const int lane = threadIdx.x % LANES, share = threadIdx.x / LANES, part_floats = g.part_rows * (D + 2);
  const float* from = g.part + ((int64_t)blockIdx.x * g.slices + first) * 2 * part_floats + blockIdx.z * (D + 2);
  Sum sum;
  if (share < SHARES) {
    constexpr int AHEAD = 4;
    for (int p0 = share; p0 < parts; p0 += AHEAD * SHARES) {
      float2 v[AHEAD][3];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int q = min(p0 + k * SHARES, parts - 1);
        const float* p = from + (int64_t)(2 * q + (q == 0 ? 1 : 0)) * part_floats;
        v[k][0] = *reinterpret_cast<const float2*>(p + 4 * lane);
        v[k][1] = *reinterpret_cast<const float2*>(p + 4 * lane + 2);
        v[k][2] = *reinterpret_cast<const float2*>(p + D);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (p0 + k * SHARES < parts) sum.add(f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y}, v[k][2].x, v[k][2].y);
    }
    s_o[share][lane] = sum.o; s_m[share][lane] = sum.m; s_l[share][lane] = sum.l;
  }
  __syncthreads();
  if (share > 0) return;
  for (int k = 1; k < min(SHARES, parts); ++k) sum.add(s_o[k][lane], s_m[k][lane], s_l[k][lane]);
  write_row(g, seq_i, kv, row, 4 * lane, sum, g.c.type == SI_KV_E4M3 && g.c.scale_v ? g.c.scale_v[kv] : 1.f);
}

template <int TYPE, int D> hipError_t launch(const AttendArgs& g, hipStream_t stream) {
  // (heads first: blocks go to the dies in turn, and all heads of a slice have the same to do)
  const dim3 grid(g.c.n_kv_heads * g.groups, g.slices);
  if (g.block_rows == 16) hipLaunchKernelGGL((k_attend<TYPE, D, 1, 1>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  else if (g.block_rows == 32) hipLaunchKernelGGL((k_attend<TYPE, D, 1, 2>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  else if (g.block_rows == 64) hipLaunchKernelGGL((k_attend<TYPE, D, 1, 4>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  else if constexpr (D <= attend_wide_dim(TYPE)) hipLaunchKernelGGL((k_attend<TYPE, D, 2, 4>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  if (g.slices > 1 && !g.whole && !g.last_joins) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_join<D>, dim3(grid.x, g.a.n, g.part_rows), dim3(256), 0, stream, g);
  }
  return hipGetLastError();
}

}  // namespace
#endif

}  // namespace si
