// Attention over positions that several sequences share: the kernel (hipcc only; instantiated by attend_shared_bf16.hip and attend_shared_e4m3.hip).
//
// A block has up to 128 rows of a kv head, of all sequences of a group, and goes through a slice of the group's cache blocks, which come to LDS once for all
// of them; a wave has 32 rows.  Matrix instructions of 32 x 32 x 16, K and V^T on the left as the cache holds them: the order of the slots in a K
// block puts the scores of a lane where the second product wants its weights for these too (lane l / 32 = h has, of 32 slots, 8 g + 4 h + i for
// g, i < 4: the tokens of the chunks h and 2 + h of V).  All rows see all positions but for a window, so that there is no mask in the loop.  Of at most 32 or 64
// rows the waves take the cache blocks in turn.
// Beside each such block runs one with sequences' own tokens (attend_device.h), which is bound by memory where this one is by instructions.
// Measured: 64 sequences with 8000 shared and up to 500 own tokens, 4 rows each, heads of 128: 37 us (si_attend 143: it reads 1.1 GB, in part from the
// caches, where this reads 112 MB); 45 windows of e4m3 over 6 prompts, 18 rows each, 89 us.  Compute units are busy 27 and 62 us of these, matrix
// instructions a fifth of that.  A wave's products of a cache block take 768 cycles and its vector instructions some 1000, one after the other: in 16 turns 12
// us of the 37; what takes the rest is not known.  Two tiles of V at a time, which could overlap them, need more registers than there are (50 us a call
// become 56).  Of e4m3 every wave of a block converts the codes for itself, and slices, which are equal in cache blocks, are not in time: of a
// piece of up to 32 rows the four waves take the blocks in turn.
#pragma once
#include "attend_device.h"

namespace si {
#if defined(__HIPCC__)
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int WIDE_ROWS = 128;  // of a block

template <int TYPE, int D> struct Wide {
  static constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8, B = 4 * E, J = E / 8;  // J score tiles of 32 tokens
  static constexpr int WAVES = ATTEND_WAVES, THREADS = ATTEND_THREADS, ROWS = 32, PAD = D + 4;
  static constexpr int BLOCK_BYTES = 128 * D, LOADS = BLOCK_BYTES / 1024 / WAVES;  // LOADS of a wave, a cache block
  static constexpr float LAG = D < 192 ? 8.f : 0.f;
  static constexpr int S = 4;                                                      // cache blocks in the ring
  using Helper = Attend<TYPE, D, 1, 1>;

  struct Shared {
    union {
      struct {
        float o[WAVES][ROWS][PAD];
        float m[WAVES][ROWS], l[WAVES][ROWS];
      };
      char ring[S * BLOCK_BYTES];
    };
    int again;
  };

  static __device__ __forceinline__ u32x4 lds16(const char* p) { return *reinterpret_cast<const u32x4*>(p); }
  // token of element 4 g + i of score tile T, from the block's first
  static __device__ __forceinline__ int token_of(int T, int g, int i, int h) {
    return E == 8 ? 8 * (2 * (g % 2) + h) + 4 * (g / 2) + i : 16 * (2 * (g % 2) + h) + 4 * (2 * T + g / 2) + i;
  }
  static __device__ __forceinline__ float max_of_row(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  static __device__ __forceinline__ float sum_of_row(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  static __device__ __forceinline__ bf16x8 part_of(const u32x4& v, int half) { return E == 8 ? operand(v) : operand8(v[2 * half], v[2 * half + 1]); }
  template <int N> static __device__ __forceinline__ void wait_blocks(int younger) {  // until no more than so many of the blocks asked for last are on their way
    if constexpr (N == 0) wait_vmcnt<0>();
    else if (younger >= N) wait_vmcnt<N * LOADS>();
    else wait_blocks<N - 1>(younger);
  }

  static __device__ __forceinline__ void run(const AttendArgs& g, Shared& s, int slice) {
    if (threadIdx.x == 0) s.again = 0;
    const SliceStart start = slice_start(g.shared, slice);
    for (int i = start.piece, off = start.off, left = start.left; left > 0; ++i) {
      const Piece p = piece_of(g.shared, i);
      const int nb = max(1, p.nb), take = min(nb - off, left);
      part(g, s, p, slice, p.fb + off, p.nb > 0 ? p.fb + off + take : p.fb, take == nb ? -1 : off > 0 ? 0 : 1);
      off = 0;
      left -= take;
    }
  }

  // Blocks [b0, b1) of a piece; where_to: -1: they are all of it, 0 / 1: the unfinished sum at the slice's begin / end
  static __device__ __forceinline__ void part(const AttendArgs& g, Shared& s, const Piece& pc, int slice, int b0, int b1, int where_to) {
    const si_cache_t& c = g.c;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 32, col = lane % 32;
    const int kv = blockIdx.x, per = g.a.n_heads / c.n_kv_heads, n_new = g.a.n_new, window = g.a.window;
    const int tiles = pc.rows > 64 ? 4 : pc.rows > 32 ? 2 : 1, streams = WAVES / tiles, stream = wave / tiles, row0 = wave % tiles * ROWS;
    const bool here = row0 < pc.rows;

    // this lane's row of q, as right operands; a negative scale goes with its signs, and the smallest number there is stands for 0 (a product with what a
    // window hides, -infinity, has to stay it; scores of up to 10^38 are as good as 0 this way)
    const int row = row0 + col;
    const float sc_all = g.scale2 * (TYPE == SI_KV_E4M3 && c.scale_k ? c.scale_k[kv] : 1.f), sc = sc_all == 0.f ? 1.4e-45f : fabsf(sc_all);
    const int tok = row < pc.rows ? (pc.first + row) / per : -1;
    u32x4 q[D / 16];
    {
      const uint16_t* p = static_cast<const uint16_t*>(g.a.q) + (int64_t)((pc.first + row) / per) * g.a.q_stride + (int64_t)(kv * per + (pc.first + row) % per) * D;
      const uint32_t signs = sc_all < 0.f ? 0x80008000u : 0u;
#pragma unroll
      for (int w = 0; w < D / 16; ++w) {
        const int dim = E == 8 ? 16 * w + 8 * h : 32 * (w / 2) + 16 * h + 8 * (w % 2);
        q[w] = tok >= 0 ? u32x4(*reinterpret_cast<const u32x4_a2*>(p + dim)) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) q[w][i] ^= signs;
      }
    }
    auto sees_from = [&](int t) {  // (members of a group have a place in the table)
      const int e = t / n_new, sq = g.a.seqs ? g.a.seqs[e] : e;
      return max(0, min(c.lens[sq], c.max_pages * c.page_tokens) - n_new + 1 + t % n_new - window);
    };
    const int see_lo = window && tok >= 0 ? sees_from(tok) : 0;

    f32x16 o[D / 32], x[J];
    float m, l;

    const int32_t* table = c.table + (int64_t)pc.seq * c.max_pages;
    const int per_page = c.page_tokens / B;
    constexpr int BYTES = TYPE == SI_KV_E4M3 ? 1 : 2;
    const int64_t page_bytes = kv_page_elems(c) * BYTES;
    const char* k_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 0, kv) * BYTES;
    const char* v_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 1, kv) * BYTES;
    int entry = b0 / per_page, at_page = b0 % per_page, asked = 0;  // of the next block that is asked for
    auto issue = [&] {
      // (the plan has seen that the pages are in the pool; a table that changed since leads nowhere else)
      const int page = min(max(((constant_t*)(uintptr_t)table)[entry], 0), c.n_pages - 1);
      const int64_t at = (uint32_t)page * page_bytes + at_page * (64 * D);
      char* to = s.ring + asked % S * BLOCK_BYTES;
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const int piece = WAVES * k + wave;  // of the block: K, then V
        Helper::load_lds((piece < D / 16 ? k_base + at + piece * 1024 : v_base + at + (piece - D / 16) * 1024) + lane * 16, to + piece * 1024);
      }
      ++asked;
      if (++at_page == per_page) { at_page = 0; ++entry; }
    };

    // Scores of a block, its weights, and its products with V; CAREFUL: values that are not finite (attend_device.h), EDGE: a window begins in it
    auto block = [&](auto EDGE, auto CAREFUL, const char* at, int t0) {
      const char *k_lds = at + (h * B + col) * 16, *v_lds = at + 64 * D + (h * D + col) * 16;
#pragma unroll
      for (int T = 0; T < J; ++T)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[T][i] = 0.f;
      // operands of K four at a time, the next four on their way meanwhile (left to itself the compiler asks for all of K and V at once and spills the sums)
      constexpr int KS = D / 16, AT_ONCE = KS % 4 == 0 && E == 8 && D < 192 ? 4 : 2;
      auto k_at = [&](int i) { return k_lds + (2 * (i / J) * B + 32 * (i % J)) * 16; };  // operand i: of score tile i % J
      u32x4 kf[2][AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) kf[0][i] = lds16(k_at(i));
#pragma unroll
      for (int i0 = 0; i0 < KS; i0 += AT_ONCE) {
        if (i0 + AT_ONCE < KS)
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) kf[(i0 / AT_ONCE + 1) % 2][i] = lds16(k_at(i0 + AT_ONCE + i));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
          for (int half = 0; half < J; ++half)
            x[(i0 + i) % J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part_of(kf[i0 / AT_ONCE % 2][i], half), operand(q[J * ((i0 + i) / J) + half]), x[(i0 + i) % J], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      auto v_at = [&](int n, int u) { return v_lds + (2 * u * D + 32 * n) * 16; };
      u32x4 vf[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) vf[0][u] = lds16(v_at(0, u));
      __builtin_amdgcn_sched_barrier(0);
      float top = -INFINITY;
#pragma unroll
      for (int T = 0; T < J; ++T)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if constexpr (EDGE) x[T][i] = t0 + token_of(T, i / 4, i % 4, h) >= see_lo ? x[T][i] : -INFINITY;
          top = fmaxf(top, x[T][i]);
        }
      // m is the largest score or up to LAG below it: weights of up to 2^LAG are as exact, and the sums need a new scale a few times at the slice's begin (of
      // 32 rows one has a new largest score nearly every turn).  64 x 8000 / 32000 shared tokens 50.6 / 112 us without, 49.6 / 106 with; heads of 256, where
      // registers are short, 128 and 137, so there m is the largest.
      const float m_new = fmaxf(m, max_of_row(top) * sc), base_new = finite_base(m_new);
      if (__any(m_new > (LAG > 0.f ? m + LAG : m))) {
        const float f = rescale(m, m_new, base_new);
        l *= f;
#pragma unroll
        for (int n = 0; n < D / 32; ++n) o[n] *= f;
        m = m_new;
      }
      const float base = LAG > 0.f ? finite_base(m) : base_new;
      u32x4 p[2][J], rest[2][J];
#pragma unroll
      for (int T = 0; T < J; ++T)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int i = 8 * (w / 2) + 4 * u + 2 * (w % 2);
            const float a = pow2(fmaf(x[T][i], sc, -base)), e = pow2(fmaf(x[T][i + 1], sc, -base));
            l += a + e;
            uint32_t pair = bf16_pair(a, e);
            asm("" : "+v"(pair));  // (or the first of the pair is rounded once more by itself)
            p[u][T][w] = pair;
            rest[u][T][w] = bf16_pair(a - __uint_as_float(pair << 16), e - __uint_as_float(pair & 0xffff0000u));
          }
      auto products = [&](auto MASKED, int from, bool mine) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
          if (n + 1 < D / 32)
#pragma unroll
            for (int u = 0; u < 2; ++u) vf[(n + 1) % 2][u] = lds16(v_at(n + 1, u));
          __builtin_amdgcn_sched_barrier(0);
          f32x16 r = o[n];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            u32x4 v = vf[n % 2][u];
            if constexpr (MASKED) v &= Helper::token_mask(t0 + (2 * u + h) * E, from, 0x7fffffff);
            const u32x4 v_rest = CAREFUL ? Helper::finite_only(v) : v;
#pragma unroll
            for (int T = 0; T < J; ++T) {
              r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part_of(v_rest, T), operand(rest[u][T]), r, 0, 0, 0);
              r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part_of(v, T), operand(p[u][T]), r, 0, 0, 0);
            }
          }
          if (!MASKED || mine) o[n] = r;
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if constexpr (CAREFUL && EDGE) {
        // a product for each token's rows, with what these see alone
#pragma unroll 1
        for (int t = (pc.first + row0) / per; t <= (pc.first + min(pc.rows, row0 + ROWS) - 1) / per; ++t) {
#pragma unroll
          for (int u = 0; u < 2; ++u) vf[0][u] = lds16(v_at(0, u));
          products(std::true_type{}, sees_from(t), tok == t);
        }
      } else if constexpr (EDGE) {
        products(std::true_type{}, pc.lo, true);  // (what no row sees may be anything)
      } else {
        products(std::false_type{}, 0, true);
      }
    };
    auto clear = [&] {
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
    };
    clear();

    const int turns = (b1 - b0 + streams - 1) / streams, ahead = S / streams - 1, count = b1 - b0;
    auto issue_turn = [&] {  // the blocks of the next turn that is not asked for yet
      for (int k = 0; k < streams; ++k)
        if (asked < count) issue();
    };
    auto barrier = [&] {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    for (int turn = 0; turn < min(ahead, turns); ++turn) issue_turn();
    for (int turn = 0; turn < turns; ++turn) {
      if (ahead == 0) {
        if (turn > 0) barrier();  // (everybody is done with what the ring held)
        issue_turn();
      }
      wait_blocks<S - 1>(asked - min(count, (turn + 1) * streams));
      barrier();  // everybody's loads of this turn have arrived, and what was read of the one before has been used
      if (ahead > 0) issue_turn();
      const int k = turn * streams + stream, t0 = (b0 + k) * B;
      if (k < count && here) {
        if (t0 < pc.lo_all) block(std::true_type{}, std::false_type{}, s.ring + k % S * BLOCK_BYTES, t0);
        else block(std::false_type{}, std::false_type{}, s.ring + k % S * BLOCK_BYTES, t0);
      }
    }
    if (turns > 0) {
      float t = 0.f;  // (what is not finite stays so through every later step, so the end is soon enough to look)
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) t = fmaf(o[n][i], 0.f, t);
      if (__any(tok >= 0 && t != 0.f) && lane == 0) s.again = 1;
      __syncthreads();  // (the ring's memory is used anew)
      if (__builtin_expect(__builtin_amdgcn_readfirstlane(s.again), 0)) {
        clear();
        asked = 0;
        entry = b0 / per_page;
        at_page = b0 % per_page;
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
          __syncthreads();
          if (k == 0 && threadIdx.x == 0) s.again = 0;
          issue();
          wait_vmcnt<0>();
          __syncthreads();
          const int t0 = (b0 + k) * B;
          if (k % streams == stream && here) {
            if (window) block(std::true_type{}, std::true_type{}, s.ring + k % S * BLOCK_BYTES, t0);
            else block(std::false_type{}, std::true_type{}, s.ring + k % S * BLOCK_BYTES, t0);
          }
        }
        __syncthreads();
      }
    }

    l = sum_of_row(l);
    float* sums = g.shared.part + (((int64_t)blockIdx.x * g.shared.slices + slice) * 2 + max(where_to, 0)) * (WIDE_ROWS * PAD);
    if (tiles == WAVES) {  // a wave has all of its rows
      if (tok >= 0) {
        float* to = where_to < 0 ? piece_sum(g, false, kv, pc.first + row) : sums + row * PAD;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int k = 0; k < 4; ++k) *reinterpret_cast<f32x4*>(to + 32 * n + 8 * k + 4 * h) = f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]};
        if (h == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m, l);
      }
      __syncthreads();
      return;
    }
    // the streams of the block
    if (h == 0) { s.m[wave][col] = m; s.l[wave][col] = l; }
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f32x4*>(&s.o[wave][col][32 * n + 8 * k + 4 * h]) = f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]};
    __syncthreads();
    const int items = pc.rows * (D / 4);
    for (int i = threadIdx.x; i < items; i += THREADS) {
      const int r = i / (D / 4), dim = i % (D / 4) * 4;
      Sum sum;
      for (int w = r / ROWS; w < WAVES; w += tiles) sum.add(*reinterpret_cast<const f32x4*>(&s.o[w][r % ROWS][dim]), s.m[w][r % ROWS], s.l[w][r % ROWS]);
      float* to = where_to < 0 ? piece_sum(g, false, kv, pc.first + r) : sums + r * PAD;
      *reinterpret_cast<f32x4*>(to + dim) = sum.o;
      if (dim == 0) *reinterpret_cast<float2*>(to + D) = make_float2(sum.m, sum.l);
    }
    __syncthreads();
  }
};

template <int TYPE, int D, int NT, int TILES> __global__ __launch_bounds__(ATTEND_THREADS, (D < 192 ? 2 : 1)) void k_attend_pieces(AttendArgs g) {
  using Own = Attend<TYPE, D, NT, TILES, ATTEND_PIECES>;
  __shared__ union {
    typename Wide<TYPE, D>::Shared shared;
    typename Own::Shared own;
  } s;
  // (all of one kind first: neighbouring blocks go to neighbouring compute units, and in turns one kind would have every other unit to itself)
  if ((int)blockIdx.y < g.shared.slices) Wide<TYPE, D>::run(g, s.shared, blockIdx.y);
  else Own::run_own_pieces(g, s.own);
}

// Joins what a row has over shared positions and over its own, each in parts or whole: D / 4 threads a row.
template <int D> __global__ __launch_bounds__(256) void k_join_pieces(AttendArgs g) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES;
  const int per = g.a.n_heads / g.c.n_kv_heads, of_entry = g.a.n_new * per, all = g.a.n * of_entry;
  const int kv = blockIdx.x, row = blockIdx.y * ROWS + threadIdx.x / LANES, dim = threadIdx.x % LANES * 4;
  if (threadIdx.x / LANES >= ROWS || row >= all) return;
  const int entry = row / of_entry;
  const int2 group = g.group[entry];
  Sum sum;
  auto add = [&](const PieceList& list, bool own, int piece, int at) {  // row `at` of the piece
    const int2 parted = list.parted[piece];
    if (parted.y == 1) {
      const float* from = piece_sum(g, own, kv, row);
      const float2 ml = *reinterpret_cast<const float2*>(from + D);
      sum.add(*reinterpret_cast<const f32x4*>(from + dim), ml.x, ml.y);
      return;
    }
    const int64_t part_floats = (int64_t)list.part_rows * list.stride;
    const float* from = list.part + ((int64_t)kv * list.slices + parted.x) * 2 * part_floats + (int64_t)at * list.stride;
    constexpr int AHEAD = 8;
    for (int p0 = 0; p0 < parted.y; p0 += AHEAD) {
      float2 v[AHEAD][3];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int q = min(p0 + k, parted.y - 1);  // (all but the first hold the piece from before)
        const float* p = from + (2 * q + (q == 0 ? 1 : 0)) * part_floats;
        v[k][0] = *reinterpret_cast<const float2*>(p + dim);
        v[k][1] = *reinterpret_cast<const float2*>(p + dim + 2);
        v[k][2] = *reinterpret_cast<const float2*>(p + D);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (p0 + k < parted.y) sum.add(f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y}, v[k][2].x, v[k][2].y);
    }
  };
  if (group.x >= 0) {
    const int at = row - group.y * of_entry;
    add(g.shared, false, group.x + at / WIDE_ROWS, at % WIDE_ROWS);
  }
  const int at = row - entry * of_entry;
  add(g.own, true, entry * g.chunks + at / g.block_rows, at % g.block_rows);
  write_row(g, entry, kv, at, dim, sum, g.c.type == SI_KV_E4M3 && g.c.scale_v ? g.c.scale_v[kv] : 1.f);
}

template <int TYPE, int D> hipError_t launch_pieces(const AttendArgs& g, hipStream_t stream) {
  const dim3 grid(g.c.n_kv_heads, g.shared.slices + g.own.slices);
  if (g.block_rows == 16) hipLaunchKernelGGL((k_attend_pieces<TYPE, D, 1, 1>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  else if (g.block_rows == 32) hipLaunchKernelGGL((k_attend_pieces<TYPE, D, 1, 2>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  else hipLaunchKernelGGL((k_attend_pieces<TYPE, D, 1, 4>), grid, dim3(ATTEND_THREADS), 0, stream, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = 256 / (D / 4);
  hipLaunchKernelGGL(k_join_pieces<D>, dim3(grid.x, (unsigned)((g.a.n * g.a.n_new * (g.a.n_heads / g.c.n_kv_heads) + rows - 1) / rows)), dim3(256), 0, stream, g);
  return hipGetLastError();
}

}  // namespace
#endif
}  // namespace si
