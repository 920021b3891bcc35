// The next token of a row of logits (scheinfer_sample.h has the formulas).
//
// A block takes a chunk of a row and leaves its maximum, where the row needs it the sum of e^((l - max) / T) in 64 bits, and for top_k the maxima of
// runs of 32 elements.  One block a row does the rest, from the caches.  What can be left is cut down before anything is put in order: with
// n runs or more the top k lie at or above the k-th largest of the runs' maxima, a token of less than (1 - top_p) S / vocab cannot be needed for a share
// of top_p, and min_p is a lowest logit.  Few tokens beyond that bound (2048) are sorted in LDS.  Of many, the border is looked for in bins (border()).
// Weights are integers (2^62 / vocab or more for the largest), so that sums in any order are the same and a token never depends on scheduling.
//
// Up to 256 chunks and the rest are one launch, in which the block of a row that finishes last goes on; more have a launch of their own, whose blocks need
// half the registers.
// Measured in the kernels: one row of 32000 bf16, top_k 50 and top_p 0.95, 17 us, one dependent step after another (chunks 4, bound 4, pass over the
// row 3, order and draw 5); 256 x 131072 fp32, top_p 0.9, 38 + 73 us: 134 MB once at 3.5 TB/s and then twice at some 8 from the caches, bound by vector
// instructions, 25 for a weight in 64 bits, which a token's border needs (an error of 1e-7 of the sum would move one draw in a hundred here), and 10
// for a place in a bin; 61 rows of 100003 with limits of their own 12 + 70 us, a compute unit a row.
#include "si_internal.h"
#include "si_error.h"
#include "scheinfer_attention.h"
#include "scheinfer_sample.h"
#include "route_device.h"
#include "wave_device.h"

#include <algorithm>
#include <cmath>

namespace si {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int EACH = 8;                    // neighbouring elements of a thread
constexpr int ROUND = THREADS * EACH;      // elements that a block takes at once
constexpr int MAX_ROUNDS = SI_SAMPLE_MAX_VOCAB / ROUND;
constexpr int RUNS = THREADS / 4;          // of a round, 4 threads each
constexpr int WIDE = 4;                    // rounds of a chunk at most
constexpr int BINS = 2048, LIST = 2048;    // two a thread

struct Args {
  si_sample_t a;
  int rounds;      // of a row
  int chunks;      // of a row: 1 to WIDE rounds each
  int per;         // rounds of a chunk
  int shift;       // a weight of 1 is 2^shift
  uint32_t* count; // [rows] chunks done; 0 between calls
  double* sum;     // [rows][chunks]
  float* top;      // [rows][chunks]
  uint32_t* n;     // [rows][chunks] elements above -infinity
  float* runs;     // [rows][rounds * RUNS]
};

struct SumsShared {  // of a block that has chunks only: two on a compute unit
  double pow2[256];                   // 2^(i / 256)
  double wave_d[WAVES];
  uint32_t wave_k[WAVES];
  uint32_t counter;
};
struct Shared : SumsShared {
  union {
    uint64_t hist[BINS];
    uint64_t list[LIST];
  };
  uint64_t part[MAX_ROUNDS * WAVES];  // sums of runs of 512 elements
  uint64_t wave_a[WAVES], wave_b[WAVES];
  float queue[WAVES][64 * EACH];
  uint64_t late[WAVES][128];
  uint64_t found[3];
  uint32_t seen, last;
};

// what other blocks read within the launch goes past the caches of this die
template <class T> __device__ __forceinline__ void put(T* p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T> __device__ __forceinline__ T get(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
// order-preserving, of numbers
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = __float_as_uint(l + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
// of the largest that a token can have whose key is `key` or less: the key before 0 belongs to -0, which no token has
__device__ __forceinline__ float value_to(uint32_t key) { return value_of(key == 0x7fffffffu ? key - 1 : key); }
constexpr float LOWEST = -3.402823466e38f;    // the lowest finite number
constexpr uint32_t LOWEST_KEY = 0x00800000u;  // its key: below it -infinity

__device__ __forceinline__ float a_little_below(double v) {
  const float f = (float)v;
  return f - fabsf(f) * 1e-6f - 1e-30f;
}
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }  // (the same in all lanes)

__device__ __forceinline__ uint32_t lanes_before(unsigned long long who) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u)); }

// Elements of a thread one after the other: eight series at once do not fit the registers of 16 waves
__device__ __forceinline__ void one_by_one() { __builtin_amdgcn_sched_barrier(0); }

// sum over the block; before: of the threads before this one
template <class T> __device__ __forceinline__ T scan(T v, T& before, uint64_t (&waves)[WAVES]) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const T x = scan_wave(v);
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  const T own = (T)waves[lane % WAVES], y = scan_row(own);
  before = x - v + of_lane((T)(y - own), wave);
  return of_lane(y, WAVES - 1);
}
__device__ __forceinline__ double block_sum(double v, SumsShared& s) {
  v = wave_total(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) s.wave_d[threadIdx.x / 64] = v;
  __syncthreads();
  return of_lane(total_row(s.wave_d[threadIdx.x % WAVES]), 0);
}
__device__ __forceinline__ float block_max(float v, SumsShared& s) {  // of numbers
  const uint32_t key = wave_max(key_of(v));
  __syncthreads();
  if (threadIdx.x % 64 == 0) s.wave_k[threadIdx.x / 64] = key;
  __syncthreads();
  return uniform(value_of(wave_max(s.wave_k[threadIdx.x % WAVES])));
}

template <int TYPE, class S> struct Row {
  const Args& g;
  S& s;
  const char* logits;
  int vocab, row, tid;
  float top;        // the row's largest (in the first pass the chunk's)
  double rate;      // 256 log2(e) / T

  // 2^shift e^((l - top) / T) = 2^(shift + n / 256) 2^(f / 256) with n the integer next to 256 log2(e) (l - top) / T and |f| <= 1/2: a table of 256 and four
  // terms of the series, some 2^-52 of the value off.  Where the largest is infinite, it alone has a weight; what is -infinity or far below has
  // 2^-976 (the larger of NaN and a number is the number).  Adding 1.5 2^52 rounds to an integer and leaves it in the low bits; the power of two goes
  // to the exponent's bits (conversions and ldexp of doubles are slow: 134 MB of logits 57 us with them).
  __device__ __forceinline__ double weight(float l, int shift) const {
    if (top == INFINITY) return l == INFINITY ? ldexp(1.0, shift) : 0.0;
    constexpr double ROUND_IT = 0x1.8p52, C = 0.0027076061740622863;  // (ln 2 / 256)
    const double y = fmax(((double)l - (double)top) * rate, -250000.0), up = y + ROUND_IT, f = y - (up - ROUND_IT);
    const int n = (int)__double_as_longlong(up);
    const long long e = __double_as_longlong(s.pow2[n & 255] * fma(f, fma(f, fma(f, fma(f, C * C * C * C / 24, C * C * C / 6), C * C / 2), C), 1.0));
    return __longlong_as_double(e + ((long long)((n >> 8) + shift) << 52));
  }
  // the same as an integer, what is below 1 cut off
  __device__ __forceinline__ uint64_t whole(float l) const {
    const uint64_t v = (uint64_t)__double_as_longlong(weight(l, g.shift));
    const int exponent = (int)(v >> 52) - 1023;  // (at most 62, as the weights are)
    return exponent < 0 ? 0 : ((v & 0xfffffffffffffull) | 1ull << 52) << 10 >> (62 - exponent);
  }

  // EACH elements of a round, on their way; beyond the row's end -infinity
  struct Raw { u32x4 v[TYPE == SI_BF16 ? 1 : 2]; };
  __device__ __forceinline__ Raw fetch(int at) const {
    Raw r;
    if (at + EACH <= vocab) {
      if constexpr (TYPE == SI_BF16) {
        r.v[0] = *reinterpret_cast<const u32x4_a2*>(logits + (int64_t)at * 2);
      } else {
        r.v[0] = *reinterpret_cast<const u32x4_a4*>(logits + (int64_t)at * 4);
        r.v[1] = *reinterpret_cast<const u32x4_a4*>(logits + (int64_t)at * 4 + 16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if constexpr (TYPE == SI_BF16) {
          const uint32_t x = at + i < vocab ? reinterpret_cast<const uint16_t*>(logits)[at + i] : 0xff80u;
          r.v[0][i / 2] = i % 2 ? r.v[0][i / 2] | x << 16 : x;
        } else {
          r.v[i / 4][i % 4] = at + i < vocab ? reinterpret_cast<const uint32_t*>(logits)[at + i] : 0xff800000u;
        }
      }
    }
    return r;
  }
  // As they are: NaN, which counts as -infinity, is in no comparison and has a weight of 0; 0 is added to what becomes a key (-0 counts as 0)
  __device__ __forceinline__ void widen(const Raw& r, float (&l)[EACH]) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if constexpr (TYPE == SI_BF16) l[i] = __uint_as_float(i % 2 ? r.v[0][i / 2] & 0xffff0000u : r.v[0][i / 2] << 16);
      else l[i] = __uint_as_float(r.v[i / 4][i % 4]);
    }
  }
  // f(first element, its EACH elements, round) for the rounds [r0, r1), the next round on its way meanwhile (two rounds ahead: the same time)
  template <class F> __device__ __forceinline__ void each(int r0, int r1, F f) const {
    Raw next = fetch(r0 * ROUND + tid * EACH);
    for (int r = r0; r < r1; ++r) {
      const int at = r * ROUND + tid * EACH;
      float l[EACH];
      widen(next, l);
      if (r + 1 < r1) next = fetch(at + ROUND);
      if (!f(at, l, r)) break;
    }
  }

  // those of a round's elements for which in(logit) holds, into the list as (key, ~index); s.counter counts beyond LIST too.  (One addition a wave: with one for
  // each of its elements a pass that lists 1442 of 100003 took 14 us.)
  template <class F> __device__ __forceinline__ void listed(const float (&l)[EACH], int at, F in) const {
    unsigned long long who[EACH];
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      who[i] = __ballot(in(l[i]));
      n += __popcll(who[i]);
    }
    if (n == 0) return;
    uint32_t to = 0;
    if (tid % 64 == 0) to = atomicAdd(&s.counter, n);
    to = __builtin_amdgcn_readfirstlane(to);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint32_t mine = to + lanes_before(who[i]);
      if (in(l[i]) && mine < LIST) s.list[mine] = composite(key_of(l[i]), ~(uint32_t)(at + i));
      to += __popcll(who[i]);
    }
  }

  // The lowest key of [lo, hi] for which `is` holds, where it holds for hi and for all above one that it holds for: 64 keys at a time, by any one wave
  template <class F> __device__ __forceinline__ uint32_t lowest_key(uint32_t lo, uint32_t hi, F is) const {
#pragma unroll 1
    while (lo < hi) {
      const uint32_t step = (hi - lo) / 64 + 1;
      const uint64_t at = lo + (uint64_t)(tid % 64) * step;
      const unsigned long long who = __ballot(at >= hi || is((uint32_t)at));
      const uint32_t n = who ? __builtin_ctzll(who) : 64;  // probes for which it does not hold
      hi = (uint32_t)min((uint64_t)hi, lo + (uint64_t)n * step);
      if (n > 0) lo += (n - 1) * step + 1;
    }
    return lo;
  }

  // What a token adds where the row is gone through in ascending index
  enum { SAME, WEIGHT };  // 1 with this key; of what is left, its weight
  struct Left {
    uint32_t key, index;  // the last that is left
  };
  __device__ __forceinline__ bool is_left(float last, uint32_t index, float l, int i) const { return l > last || (l == last && (uint32_t)i <= index); }
  __device__ __forceinline__ uint64_t adds(int what, const Left& left, float l, int i) const {
    const float last = value_of(left.key);
    return what == SAME ? l == last : is_left(last, left.index, l, i) ? whole(l) : 0;
  }
  // The sum over s.part of the rounds [r0, r1)
  __device__ __forceinline__ uint64_t add_parts(int r0, int r1) const {
    __syncthreads();
    const int parts = (r1 - r0) * WAVES;
    uint64_t before;
    return scan((2 * tid < parts ? s.part[2 * tid] : 0) + (2 * tid + 1 < parts ? s.part[2 * tid + 1] : 0), before, s.wave_a);
  }
  // Numbers of tokens with left's key over runs of 512 tokens of the rounds [r0, r1), into s.part; returns the number of all
  __device__ __forceinline__ uint64_t count_same(int r0, int r1, const Left& left) const {
    __syncthreads();
    const float same = value_of(left.key);
    each(r0, r1, [&](int, const float (&l)[EACH], int r) {
      uint32_t n = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) n += __popcll(__ballot(l[i] == same));
      if (tid % 64 == 0) s.part[(r - r0) * WAVES + tid / 64] = n;
      return true;
    });
    return add_parts(r0, r1);
  }
  // Sums of weights over runs of 512 tokens of the rounds [r0, r1), into s.part; returns their sum and the number of tokens.  in(logit, index): whether it counts;
  // other(logits, first index): looked at besides.  What counts goes through a queue of its wave, so that weights are formed by 64 lanes that have one
  // each.  (By the lanes that found them, a third of 131072 or not: 50 vector instructions an element, this way 25.  Rounds
  // of few by themselves: of a row in which 328 of 100003 count the pass 17.5 us, together 11.6; all by way of the runs' atomics: where 56000 do 44 us, this way 36.)
  struct Sum { uint64_t w, n; };
  template <class F, class G> __device__ __forceinline__ Sum add_weights(int r0, int r1, F in, G other) const {
    const int lane = tid % 64, wave = tid / 64, parts = (r1 - r0) * WAVES;
    __syncthreads();
    for (int i = tid; i < parts; i += THREADS) s.part[i] = 0;
    __syncthreads();
    // What 64 or more of a round bring is summed at once; of fewer, logits wait with their runs until they are 64.  A wave alone adds to the sums of its runs
    float* queue = s.queue[wave];
    uint64_t* late = s.late[wave];
    uint32_t n_late = 0, all = 0;
    auto add_late = [&](uint32_t many) {  // the first 64, or as many as there are
      wave_lds();
      if ((uint32_t)lane < many) {
        const uint64_t e = late[lane];
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.part[(e >> 32) * WAVES + wave]), (unsigned long long)whole(__uint_as_float((uint32_t)e)));
      }
      const uint64_t next = late[lane + 64];
      wave_lds();
      late[lane] = next;
      n_late -= many;
      wave_lds();
    };
    each(r0, r1, [&](int at, const float (&l)[EACH], int r) {
      other(l, at);
      unsigned long long who[EACH];
      uint32_t n = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        who[i] = __ballot(in(l[i], at + i));
        n += __popcll(who[i]);
      }
      if (n == 0) return true;
      all += n;
      uint32_t to = 0;
      if (n >= 64) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          if (in(l[i], at + i)) queue[to + lanes_before(who[i])] = l[i];
          to += __popcll(who[i]);
        }
        wave_lds();
        uint64_t sum = 0;
        for (uint32_t k = lane; k - lane < n; k += 128) {  // (two series at a time; -infinity weighs nothing)
          const float a = k < n ? queue[k] : -INFINITY, b = k + 64 < n ? queue[k + 64] : -INFINITY;
          sum += whole(a) + whole(b);
        }
        wave_lds();
        sum = wave_total(sum);
        if (lane == 0) s.part[(r - r0) * WAVES + wave] = sum;
        return true;
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (in(l[i], at + i)) late[n_late + to + lanes_before(who[i])] = composite((uint32_t)(r - r0), __float_as_uint(l[i]));
        to += __popcll(who[i]);
      }
      n_late += n;
      if (n_late >= 64) add_late(64);
      return true;
    });
    if (n_late > 0) add_late(n_late);
    __syncthreads();
    uint32_t unused;
    const uint32_t total = scan(lane == 0 ? all : 0u, unused, s.wave_b);
    return Sum{add_parts(r0, r1), total};
  }
  __device__ __forceinline__ Sum add_left(int r0, int r1, const Left& left) const {
    const float last = value_of(left.key);
    return add_weights(r0, r1, [&](float l, int i) { return is_left(last, left.index, l, i); }, [](const float (&)[EACH], int) {});
  }
  // The first token at which the sum is above `target` (below the sum of all), with s.part of the same
  __device__ __forceinline__ int locate(int r0, int r1, int what, const Left& left, uint64_t target) const {
    const int parts = (r1 - r0) * WAVES, lane = tid % 64;
    const uint64_t p0 = 2 * tid < parts ? s.part[2 * tid] : 0, p1 = 2 * tid + 1 < parts ? s.part[2 * tid + 1] : 0;
    uint64_t before;
    scan(p0 + p1, before, s.wave_a);
    if (before <= target && target < before + p0 + p1) {
      const bool second = target >= before + p0;
      s.found[0] = 2 * tid + second;
      s.found[1] = target - before - (second ? p0 : 0);
    }
    __syncthreads();
    const int run = (int)s.found[0];
    uint64_t rest = s.found[1];
    if (tid < 64) {
      float l[EACH];
      const int at = r0 * ROUND + run * 64 * EACH + lane * EACH;
      widen(fetch(at), l);
      uint64_t sum = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) { sum += adds(what, left, l[i], at + i); one_by_one(); }
      uint64_t x = scan_wave(sum) - sum;
      if (x <= rest && rest < x + sum) {
        int token = -1;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          x += adds(what, left, l[i], at + i);
          if (token < 0 && x > rest) token = at + i;
          one_by_one();
        }
        s.found[2] = token;
      }
    }
    __syncthreads();
    return (int)s.found[2];
  }
  __device__ __forceinline__ float logit(int i) const {
    float v;
    if constexpr (TYPE == SI_BF16) v = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(logits)[i] << 16);
    else v = reinterpret_cast<const float*>(logits)[i];
    return v;
  }

  // the list's first n entries in descending order (n <= LIST); every thread's part is in LDS before and after
  __device__ __forceinline__ void sort(int n) const {
    __syncthreads();
    if (n <= 64) {  // one a lane of one wave
      if (tid < 64) {
        uint64_t v = tid < n ? s.list[tid] : 0;
#pragma unroll
        for (int k = 2; k <= 64; k *= 2)
#pragma unroll
          for (int j = k / 2; j > 0; j /= 2) {
            const uint64_t o = __shfl_xor(v, j);
            v = ((tid & j) == 0) == ((tid & k) == 0) ? max(v, o) : min(v, o);
          }
        s.list[tid] = v;
      }
      __syncthreads();
      return;
    }
    int size = 128;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += THREADS) s.list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        if (j >= 64 && k > 128) __syncthreads();  // (to 32, and in all of the first 128, what a wave takes is what it left)
        else wave_lds();
        if (2 * tid < size) {
          const int i = 2 * tid - tid % j, o = i + j;  // (of 2 j neighbours, those of the first half)
          const uint64_t a = s.list[i], b = s.list[o];
          const bool down = (i & k) == 0;
          if ((a < b) == down) { s.list[i] = b; s.list[o] = a; }
        }
      }
    __syncthreads();
  }

  // elements of lo or more into the list; returns their number, or some number above LIST
  __device__ __forceinline__ int collect(float lo) const {
    __syncthreads();
    if (tid == 0) s.counter = 0;
    __syncthreads();
    each(0, g.rounds, [&](int at, const float (&l)[EACH], int) {
      listed(l, at, [&](float v) { return v >= lo; });
      // (a wave may see a count of the round that others are in: it only goes on for nothing)
      return __hip_atomic_load(&s.counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) <= LIST;
    });
    __syncthreads();
    return (int)s.counter;
  }

  // The last token left, how many they are with it and the sum of their weights; summed: s.part holds the sums of what is left
  struct Border { uint32_t key, index; uint64_t n, w; bool summed; };

  // Border of the first token at which the number (by_n) or the sum of those up to it reaches `need`, among keys of [lo, hi] (none is above hi); where none
  // does, of the last that adds to it.  A pass puts numbers or rough sums of the range into bins; the next takes what is above the bin in which they reach `need`
  // exactly, and lists what is in it.  Where that shows another bin, or the list is full, once more with what is left of the range.  Bins are equal
  // parts of the logits' range at first, where a lower end is known, and of the keys' then: keys are dense next to 0, where a range that holds it would leave
  // few bins for the rest.  Rough sums are some 1e-6 of the range off, and 0 where its end is far above what is left: a row whose border they
  // miss once more would be gone through bin by bin.  So from the third turn on the bins have exact sums: 11 bits of the key are found a turn, whatever the
  // values are.  (131072 logits of 999.95 to 1000.05 and one of 1023, top_p 0.99999: 4464 us with rough sums in every turn, 255 this way; an ordinary row 72.  One in 20
  // batches of 256 x 131072 at top_p 0.9 has a row that takes a second turn, for the next bin: 152 us, 170 with exact sums there, else 110.)
  __device__ __forceinline__ Border border(uint32_t lo, uint32_t hi, bool by_n, uint64_t need) const {
    uint64_t done = 0;  // number or sum above hi
    // The border is at or above `least_key`, and so many tokens are; lo is above it while the range is a bin that may not have the border
    uint32_t least_key = lo;
    uint64_t n_least = 0;
    bool counted = false;
    const float rate32 = (float)fmin(rate / 256, 1e30), range = value_of(hi) - value_of(lo);
    bool by_value = lo > LOWEST_KEY && range > 1e-30f && range < 1e30f;
    const float scale = (BINS - 1) / range;
    const uint32_t highest = hi;
    for (int turn = 0;; ++turn, by_value = false) {
      const bool exact = turn > 1;
      const uint32_t width = hi - lo;
      const int drop = max(0, 32 - __clz((int)width) - 11);  // (at most BINS bins of 2^drop keys)
      const float of = value_of(hi);
      const float from = value_of(lo), to = value_to(hi);
      __syncthreads();
      for (int i = tid; i < BINS; i += THREADS) s.hist[i] = 0;
      if (tid == 0) { s.counter = 0; s.seen = 0; s.found[0] = 0; }
      __syncthreads();
      uint32_t n_range = 0;
      // (a rough sum: 2^31 of the weight of `of`, in fp32)
      enum { NUMBERS, ROUGH, EXACT };
      auto put_all = [&](auto values, auto what) {
        each(0, g.rounds, [&](int, const float (&l)[EACH], int) {
          uint32_t bin[EACH], rough[EACH];
#pragma unroll
          for (int i = 0; i < EACH; ++i) {  // (of what is out of range: anything)
            const float below = of - l[i];
            bin[i] = values ? min((uint32_t)(below * scale), BINS - 1u) : (hi - key_of(l[i])) >> drop;
            rough[i] = what != ROUGH ? 1u : !values && l[i] == of ? 1u << 31 : (uint32_t)__builtin_amdgcn_exp2f(fmaf(below, -rate32, 31.f));
          }
#pragma unroll
          for (int i = 0; i < EACH; ++i) {
            const bool in = l[i] >= from && l[i] <= to;
            n_range += __popcll(__ballot(in));
            if (in) atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[bin[i]]), (unsigned long long)(what == EXACT ? whole(l[i]) : rough[i]));
            if constexpr (what == EXACT) one_by_one();
          }
          return true;
        });
      };
      constexpr std::integral_constant<int, NUMBERS> numbers{};
      constexpr std::integral_constant<int, ROUGH> rough_sums{};
      if (by_value) by_n ? put_all(std::true_type{}, numbers) : put_all(std::true_type{}, rough_sums);
      else if (by_n) put_all(std::false_type{}, numbers);
      else exact ? put_all(std::false_type{}, std::integral_constant<int, EXACT>{}) : put_all(std::false_type{}, rough_sums);
      if (tid % 64 == 0) atomicAdd(&s.seen, n_range);
      __syncthreads();
      n_range = s.seen;
      if (!counted) n_least = n_range;  // (the first range is all from its lower end on)
      counted = true;
      const uint64_t h0 = s.hist[2 * tid], h1 = s.hist[2 * tid + 1];
      uint64_t x;
      const uint64_t in_range = scan(h0 + h1, x, s.wave_a);
      if ((exact || by_n) && done + in_range < need) {  // the border is not in this range
        if (lo > least_key) {                 // but below it
          done += in_range;
          hi = lo - 1;
          lo = least_key;
          continue;
        }
        need = done + in_range;  // or nowhere (fewer tokens, or what is left weighs less than the smallest integers): the last that adds to the sum
        if (in_range == 0) {
          hi = highest;
          done = 0;
          continue;
        }
      }
      const uint64_t goal = by_n || exact ? need - done : (uint64_t)fmin(fmax((double)(need - done) / weight(of, g.shift) * 0x1p31, 1.0), 1e18);
      // (the last bin that begins below the goal and is not empty: the goal's, or the last of all)
      if (h1 > 0 && x + h0 < goal) atomicMax(reinterpret_cast<unsigned long long*>(&s.found[0]), (unsigned long long)(2 * tid + 2));
      else if (h0 > 0 && x < goal) atomicMax(reinterpret_cast<unsigned long long*>(&s.found[0]), (unsigned long long)(2 * tid + 1));
      __syncthreads();
      const uint32_t bin = max((int)s.found[0] - 1, 0);  // (weights that are all roughly 0: the first)
      // The bin, or a range that has all of it: what follows is right for any range
      uint32_t top_of = hi - (bin << drop), low_of = max(lo, top_of - ((1u << drop) - 1));
      if (by_value) {
        top_of = bin == 0 ? hi : min(hi, key_of(of - ((float)bin - 0.01f) / scale));
        low_of = bin == BINS - 1 ? lo : min(top_of, max(lo, key_of(of - ((float)bin + 1.01f) / scale)));
      }
      if (by_n && !by_value) {
        if (tid == (int)bin / 2) {
          s.found[1] = x + (bin % 2 ? h0 : 0);
          s.found[2] = bin % 2 ? h1 : h0;
        }
        __syncthreads();
        if (s.found[2] > LIST && low_of < top_of) {  // more than can be listed
          lo = low_of;
          hi = top_of;
          done += s.found[1];
          continue;
        }
      }
      const float bin_to = value_to(top_of), bin_from = value_of(low_of);
      const Sum above = add_weights(0, g.rounds, [&](float l, int) { return l > bin_to; }, [&](const float (&l)[EACH], int at) { listed(l, at, [&](float v) { return v >= bin_from && v <= bin_to; }); });
      const int inside = (int)s.counter;
      const uint64_t n_above = above.n, w_above = above.w, reached = by_n ? n_above : w_above;
      if (reached >= need && top_of < hi) {  // the border is above this bin
        lo = least_key = top_of + 1;
        n_least = n_above;
        continue;
      }
      const bool more = n_least > n_above + inside;  // below low_of
      if (inside > LIST && low_of < top_of) {
        lo = low_of;
        hi = top_of;
        done = reached;
        continue;
      }
      if (inside > LIST) {  // more tokens of one logit than the list holds: as many as are needed, from the lowest index
        const uint64_t each_w = whole(value_of(top_of)), most = inside;
        const uint64_t k = by_n ? min(need - reached, most) : each_w == 0 ? most : min((need - reached + each_w - 1) / each_w, most);
        if (more && (by_n ? reached + most : reached + most * each_w) < need) {
          lo = least_key;
          hi = low_of - 1;
          done = by_n ? reached + most : reached + most * each_w;
          continue;
        }
        const Left same{top_of, 0};
        count_same(0, g.rounds, same);
        const int at = locate(0, g.rounds, SAME, same, k - 1);
        return Border{top_of, (uint32_t)at, n_above + k, w_above + k * each_w, false};
      }
      sort(inside);
      uint64_t e[2], w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        e[i] = 2 * tid + i < inside ? s.list[2 * tid + i] : 0;
        w[i] = 2 * tid + i < inside ? whole(value_of((uint32_t)(e[i] >> 32))) : 0;
      }
      uint64_t before;
      const uint64_t listed_w = scan(w[0] + w[1], before, s.wave_a), all = by_n ? n_above + inside : w_above + listed_w;
      if (all < need && more) {  // the border is below this bin
        lo = least_key;
        hi = low_of - 1;
        done = all;
        continue;
      }
      const uint64_t last = min(need, all);
      before += w_above;
      if (tid == 0) s.found[0] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint64_t at = n_above + 2 * tid + i + 1;
        if (2 * tid + i < inside && (by_n ? at <= last : before < last || 2 * tid + i == 0))  // left
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.part[~(uint32_t)e[i] / (64 * EACH)]), (unsigned long long)w[i]);
        if (2 * tid + i < inside && (by_n ? at == last : (before < last || 2 * tid + i == 0) && (before + w[i] >= last || 2 * tid + i + 1 == inside))) {
          s.found[0] = e[i];
          s.found[1] = at;
          s.found[2] = before + w[i];
        }
        before += w[i];
      }
      __syncthreads();
      return Border{(uint32_t)(s.found[0] >> 32), ~(uint32_t)s.found[0], s.found[1], s.found[2], true};
    }
  }

  __device__ __forceinline__ void write(int token, double prob, int kept) const {
    if (tid != 0) return;
    g.a.token[row] = token;
    if (g.a.prob) g.a.prob[row] = (float)prob;
    if (g.a.kept) g.a.kept[row] = kept;
  }
};

// What a row is asked for
struct Wishes {
  float t;
  int k;               // 0: no limit
  bool greedy, by_p, by_m;
  double p, least;
  bool summed, all_left;
  __device__ __forceinline__ Wishes(const si_sample_t& a, int row) {
    t = a.temperature ? a.temperature[row] : 1.f;
    greedy = !(t > 0.f);
    k = a.top_k && a.top_k[row] > 0 && a.top_k[row] < a.vocab ? a.top_k[row] : 0;
    const float p_given = a.top_p ? a.top_p[row] : 1.f, m_given = a.min_p ? a.min_p[row] : 0.f;
    by_p = p_given < 1.f;
    by_m = m_given > 0.f;
    p = fmaxf(p_given, 0.f);
    least = fminf(m_given, 1.f);
    all_left = !greedy && k == 0 && !by_p && !by_m;
    summed = !greedy && k == 0 && (by_p || !by_m);  // the sum over the whole row is needed
  }
};
template <int TYPE, class S> __device__ __forceinline__ Row<TYPE, S> row_of(const Args& g, S& s, int row, const Wishes& w) {
  if (threadIdx.x < 256) s.pow2[threadIdx.x] = exp2(threadIdx.x / 256.0);
  return Row<TYPE, S>{g, s, static_cast<const char*>(g.a.logits) + (int64_t)row * g.a.stride * (TYPE == SI_BF16 ? 2 : 4), g.a.vocab, row, (int)threadIdx.x, 0.f,
                   w.greedy ? 0.0 : 369.3299304675746 / (double)w.t};
}

// A chunk of g.per rounds: its maximum, number of tokens, sum, and the maxima of its runs.  A wave goes on by itself, with a maximum of its own
// to which it brings its sum; the waves are joined at the end.
template <int TYPE, class S> __device__ __forceinline__ void sums_of_chunk(Row<TYPE, S>& R, const Wishes& w, int chunk) {
  const Args& g = R.g;
  S& s = R.s;
  const int tid = threadIdx.x, lane = tid % 64, r0 = chunk * g.per, r1 = min(r0 + g.per, g.rounds);
  uint32_t n = 0;
  double sum = 0.0;
  R.top = -INFINITY;
  if (tid == 0) s.counter = 0;
  __syncthreads();  // (and the table is there)
  R.each(r0, r1, [&](int, const float (&l)[EACH], int r) {
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      most = fmaxf(most, l[i]);
      n += __popcll(__ballot(l[i] >= LOWEST));  // (a ballot of > -INFINITY is compiled to one of != here, which NaN passes)
    }
    if (w.k > 0) {
      float run = fmaxf(most, __shfl_xor(most, 1));
      run = fmaxf(run, __shfl_xor(run, 2));
      if (lane % 4 == 0) put(g.runs + ((int64_t)R.row * g.rounds + r) * RUNS + tid / 4, run);
    }
    most = uniform(value_of(wave_max(key_of(most))));
    if (most > R.top) {
      const float before = R.top;
      R.top = most;
      if (w.summed && sum > 0.0) sum *= R.weight(before, 0);
    }
    if (w.summed && R.top > -INFINITY) {
#pragma unroll
      for (int i = 0; i < EACH; ++i) { sum += R.weight(l[i], 0); one_by_one(); }
    }
    return true;
  });
  const float mine = R.top;
  R.top = block_max(mine, s);
  if (w.summed) sum = block_sum(mine > -INFINITY ? sum * R.weight(mine, 0) : 0.0, s);
  if (lane == 0) atomicAdd(&s.counter, n);
  __syncthreads();
  if (tid == 0) {
    const int64_t at = (int64_t)R.row * g.chunks + chunk;
    put(g.top + at, R.top);
    put(g.n + at, s.counter);
    put(g.sum + at, sum);
  }
}

// Many rows: a launch for the chunks alone, two blocks a compute unit
template <int TYPE> __global__ __launch_bounds__(THREADS, 8) void k_sample_sums(Args g) {
  __shared__ SumsShared s;
  const int row = blockIdx.x / g.chunks;
  const Wishes w(g.a, row);
  auto R = row_of<TYPE>(g, s, row, w);
  sums_of_chunk(R, w, blockIdx.x % g.chunks);
}

// ALONE: the chunks too, and the block of a row that finishes last goes on; else a block a row
template <int TYPE, bool ALONE> __global__ __launch_bounds__(THREADS) void k_sample(Args g) {
  __shared__ Shared s;
  const int row = ALONE ? blockIdx.x / g.chunks : blockIdx.x, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const si_sample_t& a = g.a;
  const Wishes w(a, row);
  auto R = row_of<TYPE>(g, s, row, w);
  if constexpr (ALONE) {
    sums_of_chunk(R, w, blockIdx.x % g.chunks);
    // all of this block's values have reached memory before it is counted
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
      s.last = __hip_atomic_fetch_add(g.count + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)g.chunks - 1;
      if (s.last) put(g.count + row, 0u);
    }
    __syncthreads();
    if (!s.last) return;
  }
  const float t = w.t;
  const int k = w.k;
  const bool greedy = w.greedy, by_p = w.by_p, by_m = w.by_m, summed = w.summed, all_left = w.all_left;
  const double p = w.p, least = w.least;

  // The row's largest, its number of tokens, and its sum
  const int64_t first = (int64_t)row * g.chunks;
  const float chunk_top = tid < g.chunks ? get(g.top + first + tid) : -INFINITY;
  const float top = block_max(chunk_top, s);
  uint32_t before;
  const uint32_t n_all = scan(tid < g.chunks ? get(g.n + first + tid) : 0u, before, s.wave_a);
  if (n_all == 0) { R.write(-1, 0.0, 0); return; }
  R.top = top;
  const uint32_t top_key = key_of(top);
  const float u = a.u[row];
  const double one = ldexp(1.0, g.shift);
  // How the row is gone through in the end, and with which target
  int r0 = 0, r1 = g.rounds, what = R.WEIGHT;
  typename Row<TYPE, Shared>::Left left{LOWEST_KEY, 0xffffffffu};
  double sum = 0.0, rest = 0.0;
  int kept = (int)n_all;
  uint64_t w_all = 0;
  bool added = false, recount = false;  // s.part has the sums of what is left; kept is to be counted anew
  auto drawn = [&](uint64_t all) { return !(u > 0.f) ? 0 : u >= 1.f ? all - 1 : min((uint64_t)((double)u * (double)all), all - 1); };
  if (greedy) {
    // in the first chunk that has it
    const unsigned long long has = __ballot(chunk_top == top);
    __syncthreads();
    if (lane == 0) s.wave_a[wave] = has ? wave * 64 + __builtin_ctzll(has) : ~0ull;
    __syncthreads();
#pragma unroll 1
    for (int w = WAVES - 1; w >= 0; --w) r0 = s.wave_a[w] != ~0ull ? (int)s.wave_a[w] : r0;
    r0 *= g.per;
    r1 = min(r0 + g.per, g.rounds);
    what = R.SAME;
    left.key = top_key;
    kept = 1;
  }
  if (summed) {
    const double share = tid < g.chunks ? get(g.sum + first + tid) * R.weight(chunk_top, 0) : 0.0;
    sum = block_sum(share, s);
    if (all_left) {
      // the chunk in which u falls
      double x = share;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
      }
      __syncthreads();
      if (lane == 63) s.wave_d[wave] = x;
      if (tid == 0) s.found[0] = 0;
      __syncthreads();
      double base = 0.0;
      for (int w = 0; w < wave; ++w) base += s.wave_d[w];
      const double begin = base + x - share, target = !(u > 0.f) ? 0.0 : u >= 1.f ? sum : (double)u * sum;
      // (the last that begins at or before the target and is not empty: sums of doubles may leave a gap between two)
      if (share > 0.0 && begin <= target) atomicMax(reinterpret_cast<unsigned long long*>(&s.found[0]), (unsigned long long)tid);
      __syncthreads();
      r0 = (int)s.found[0];
      if (tid == r0) s.wave_d[0] = target - begin;
      __syncthreads();
      r0 *= g.per;
      r1 = min(r0 + g.per, g.rounds);
      rest = fmax(s.wave_d[0], 0.0);
    }
  }
  if (!greedy && !all_left) {
  // What can be left lies at or above `bound`
  float bound = LOWEST;
  if (k > 0) {
    // the k-th largest of the runs' maxima, by 22 leading bits of its key (a little below it)
    const int runs = g.rounds * RUNS;
    uint32_t lo = 0;
    if (k <= runs) {
      uint32_t need = k;
      for (int level = 0; level < 2; ++level) {
        __syncthreads();
        for (int i = tid; i < BINS; i += THREADS) s.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < runs; i += THREADS) {
          const uint32_t key = key_of(get(g.runs + (int64_t)row * runs + i));
          if (level == 0) atomicAdd(reinterpret_cast<uint32_t*>(&s.hist[2047 - (key >> 21)]), 1u);
          else if ((key >> 21) == (lo >> 21)) atomicAdd(reinterpret_cast<uint32_t*>(&s.hist[2047 - ((key >> 10) & 2047)]), 1u);
        }
        __syncthreads();
        const uint32_t n0 = (uint32_t)s.hist[2 * tid], n1 = (uint32_t)s.hist[2 * tid + 1];
        uint32_t x;
        scan(n0 + n1, x, s.wave_a);
        if (x < need && need <= x + n0 + n1) {
          const bool second = need > x + n0;
          s.found[0] = 2047 - (2 * tid + second);
          s.found[1] = need - x - (second ? n0 : 0);
        }
        __syncthreads();
        lo |= (uint32_t)s.found[0] << (level == 0 ? 21 : 10);
        need = (uint32_t)s.found[1];
      }
      bound = fmaxf(bound, value_of(lo));
    }
  } else if (by_p) {
    const double c = (1.0 - p) * (1.0 - 1e-6) * sum / a.vocab;
    if (c > 0.0 && c < 1.0 && top < INFINITY) bound = fmaxf(bound, a_little_below((double)top + log(c) * (double)t));
  }
  bound = fminf(bound, top);
  uint32_t bound_key = max(key_of(bound), LOWEST_KEY);
  // Weights rise with the logits, so min_p is a lowest key.  (With both top_k and top_p the sum of all k is needed, those below min_p too.)
  if (by_m) {
    __syncthreads();
    if (tid < 64) {
      const uint32_t key = R.lowest_key(LOWEST_KEY, top_key, [&](uint32_t key) { return R.weight(value_of(key), 0) >= least; });
      if (tid == 0) s.found[0] = key;
    }
    __syncthreads();
  }
  const uint32_t m_key = by_m ? (uint32_t)s.found[0] : LOWEST_KEY;
  if (!(k > 0 && by_p)) bound_key = max(bound_key, m_key);

  // Few: in order, all at once
  const int few = k > LIST ? LIST + 1 : R.collect(value_of(bound_key));
  if (few <= LIST) {
    if (by_p || (k > 0 && few > k)) R.sort(few);
    uint64_t e[2], w[2];
    bool fine[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e[i] = 2 * tid + i < few ? s.list[2 * tid + i] : 0;
      fine[i] = 2 * tid + i < few && (k == 0 || 2 * tid + i < k);
      w[i] = fine[i] ? R.whole(value_of((uint32_t)(e[i] >> 32))) : 0;
      fine[i] = fine[i] && (uint32_t)(e[i] >> 32) >= m_key;
    }
    uint64_t x;
    const uint64_t all = scan(w[0] + w[1], x, s.wave_a);
    if (by_p) {
      const double whole_sum = k > 0 ? (double)all : sum * one;
      const double goal = p * whole_sum;
      // (left while the sum before it has not reached the goal)
      fine[0] = fine[0] && (2 * tid == 0 || (double)x < goal);
      fine[1] = fine[1] && (double)(x + w[0]) < goal;
    }
    uint32_t unused;
    kept = (int)scan((uint32_t)fine[0] + fine[1], unused, s.wave_b);
    if (kept <= 64) {  // in order of the index, at once
      __syncthreads();
      if (tid == 0) s.counter = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (fine[i]) s.list[atomicAdd(&s.counter, 1u)] = e[i] << 32 | e[i] >> 32;
      R.sort(kept);
      const uint64_t mine = tid < kept ? s.list[tid] : 0, weight = tid < kept ? R.whole(value_of((uint32_t)mine)) : 0;
      const uint64_t total = scan(weight, x, s.wave_a), target = drawn(total);
      if (x <= target && target < x + weight) {
        s.found[0] = mine;
        s.found[1] = weight;
      }
      __syncthreads();
      R.write((int)~(uint32_t)(s.found[0] >> 32), (double)s.found[1] / (double)total, kept);
      return;
    }
    // into the sums of their runs
    for (int i = tid; i < g.rounds * WAVES; i += THREADS) s.part[i] = 0;
    __syncthreads();
    uint64_t last = ~0ull;  // of those that are left
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (fine[i]) {
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.part[~(uint32_t)e[i] / (64 * EACH)]), (unsigned long long)w[i]);
        last = min(last, e[i]);
      }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) last = min(last, (uint64_t)__shfl_xor(last, d));
    if (tid == 0) s.found[0] = ~0ull;
    __syncthreads();
    if (lane == 0) atomicMin(reinterpret_cast<unsigned long long*>(&s.found[0]), (unsigned long long)last);
    w_all = R.add_parts(0, g.rounds);
    left.key = (uint32_t)(s.found[0] >> 32);
    left.index = ~(uint32_t)s.found[0];
    added = true;
  } else {
  // Many: the border by number, then by sum
  w_all = (uint64_t)(sum * one);
  for (int by_n = 1; by_n >= 0; --by_n) {
    if (by_n ? k == 0 : !by_p) continue;
    const auto b = R.border(bound_key, top_key, by_n, by_n ? (uint64_t)k : max((uint64_t)1, (uint64_t)ceil(p * (double)w_all)));
    left.key = b.key;
    left.index = b.index;
    kept = (int)b.n;
    w_all = b.w;
    added = b.summed;
  }
  if (m_key > left.key) {
    left.key = m_key;
    left.index = 0xffffffffu;
    added = false;
  }
  recount = !added;
  }
  }
  uint64_t total = w_all;
  if (greedy) {
    total = R.count_same(r0, r1, left);
  } else if (!added) {
    const auto sums = R.add_left(r0, r1, left);
    total = sums.w;
    if (recount) kept = (int)sums.n;
  }
  uint64_t target = greedy ? 0 : drawn(total);
  if (all_left) {
    if (total > 0) {
      target = u >= 1.f ? total - 1 : min((uint64_t)(rest * one), total - 1);
    } else {  // (a chunk of weights that are all below the smallest integer)
      r0 = 0;
      r1 = g.rounds;
      total = R.add_left(r0, r1, left).w;
      target = drawn(total);
    }
  }
  const int at = R.locate(r0, r1, what, left, target);
  const double mine = R.weight(R.logit(at), 0);
  R.write(at, greedy ? 1.0 : all_left ? mine / sum : mine * one / (double)total, kept);
}

bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int check(const si_sample_t* a, const char* who) {
  if (!a) return set_error(SI_EINVAL, "%s: descriptor is NULL", who);
  if (a->type != SI_F32 && a->type != SI_BF16) return set_error(SI_EINVAL, "%s: unknown type %d", who, a->type);
  if (a->rows < 0 || a->rows > SI_SAMPLE_MAX_ROWS || a->vocab < 1 || a->vocab > SI_SAMPLE_MAX_VOCAB) return set_error(SI_EINVAL, "%s: rows %d, vocab %d", who, a->rows, a->vocab);
  if ((int64_t)a->rows * ((a->vocab + ROUND - 1) / ROUND) >= (1 << 22)) return set_error(SI_EINVAL, "%s: too many rows in one call (%d of %d)", who, a->rows, a->vocab);
  return SI_OK;
}

// Places in the scratch; returns its size
int64_t lay_out(const si_sample_t& a, Args* g) {
  const int64_t rounds = (a.vocab + ROUND - 1) / ROUND, n = a.rows * rounds;
  char* p = static_cast<char*>(a.scratch);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    char* q = p + at;
    at += (bytes + 15) / 16 * 16;
    return q;
  };
  // (the counters first, for any number of rows: they stay where they are, and 0, in calls of other sizes)
  uint32_t* count = reinterpret_cast<uint32_t*>(take(4ll * SI_SAMPLE_MAX_ROWS));
  double* sum = reinterpret_cast<double*>(take(8 * n));
  float* top = reinterpret_cast<float*>(take(4 * n));
  uint32_t* each = reinterpret_cast<uint32_t*>(take(4 * n));
  float* runs = reinterpret_cast<float*>(take(4 * n * RUNS));
  if (g) {
    g->rounds = (int)rounds;
    g->count = count;
    g->sum = sum;
    g->top = top;
    g->n = each;
    g->runs = runs;
  }
  return at;
}

}  // namespace
}  // namespace si

extern "C" int64_t si_sample_scratch_bytes(const si_sample_t* a) {
  using namespace si;
  if (int rc = check(a, "si_sample_scratch_bytes")) return rc;
  return lay_out(*a, nullptr);
}

extern "C" int si_sample(const si_sample_t* a, void* stream) {
  using namespace si;
  const char* who = "si_sample";
  if (int rc = check(a, who)) return rc;
  if (a->rows == 0) return SI_OK;  // (an empty tensor's address may be NULL)
  if (!a->logits || !a->u || !a->token || !a->scratch) return set_error(SI_EINVAL, "%s: logits, u, token or scratch is NULL", who);
  if (misaligned(a->logits, a->type == SI_F32 ? 4 : 2) || misaligned(a->temperature, 4) || misaligned(a->top_k, 4) || misaligned(a->top_p, 4) || misaligned(a->min_p, 4) ||
      misaligned(a->u, 4) || misaligned(a->token, 4) || misaligned(a->prob, 4) || misaligned(a->kept, 4) || misaligned(a->scratch, 16))
    return set_error(SI_EINVAL, "%s: a pointer is not aligned to its element (scratch: to 16 bytes)", who);
  if (a->stride < a->vocab && a->stride != 0) return set_error(SI_EINVAL, "%s: stride %lld of rows of %d", who, (long long)a->stride, a->vocab);
  Args g{};
  g.a = *a;
  const int64_t bytes = lay_out(*a, &g);
  if (a->scratch_bytes < bytes) return set_error(SI_EINVAL, "%s: %lld bytes of scratch needed", who, (long long)bytes);
  int log2 = 0;
  while ((1 << log2) < a->vocab) ++log2;
  g.shift = 62 - log2;
  // One launch for no more chunks than compute units (its blocks have registers for the row's end: one a unit).  Else chunks that fill the chip twice.
  // Rows of 100003 fp32 with top_p 0.9 in one launch and in two: 8 rows 69 and 74 us, 32 rows 98 and 74; 256 x 131072: 1116 and 120.
  const int64_t all = (int64_t)a->rows * g.rounds;
  const bool alone = all <= 256;
  g.per = alone ? 1 : (int)std::min<int64_t>(WIDE, (all + 511) / 512);
  g.chunks = (g.rounds + g.per - 1) / g.per;
  const dim3 chunks((unsigned)(a->rows * g.chunks)), rows((unsigned)a->rows), block(THREADS);
  const hipStream_t st = (hipStream_t)stream;
  if (!alone) {
    if (a->type == SI_BF16) hipLaunchKernelGGL(k_sample_sums<SI_BF16>, chunks, block, 0, st, g);
    else hipLaunchKernelGGL(k_sample_sums<SI_F32>, chunks, block, 0, st, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(SI_EHIP, "sample launch failed: %s", hipGetErrorString(e));
  }
  if (a->type == SI_BF16) {
    if (alone) hipLaunchKernelGGL((k_sample<SI_BF16, true>), chunks, block, 0, st, g);
    else hipLaunchKernelGGL((k_sample<SI_BF16, false>), rows, block, 0, st, g);
  } else {
    if (alone) hipLaunchKernelGGL((k_sample<SI_F32, true>), chunks, block, 0, st, g);
    else hipLaunchKernelGGL((k_sample<SI_F32, false>), rows, block, 0, st, g);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(SI_EHIP, "sample launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
