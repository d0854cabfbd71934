// Beam search over recurrent states: the best continuations over beams and vocabulary, and the states behind them.
//
// Selection.  A continuation of beam b by token v weighs s = score_b + (x_bv - log sum exp x_b), in 64 bits; the best n_out of a
// request's width x vocab continuations are wanted.  Inside a beam they are ordered like the logits themselves, so each part of a row gives its best n_out
// by 64-bit keys (logit, then lower token) while it sums exponentials, all from one pass over the row, and the few that are left meet with their beams' sums.
// Split: a request is a cluster of CL thread blocks; the rows of its beams that count (not ended, with a finite score) are cut into segments, alike for all rows, which
// the blocks take in order.  A block goes once through a segment, two rounds of 64 bytes per thread loaded at a time, for nothing but each thread's largest
// logit and sum of exponentials and the largest of each of its chunks of entries.  Sums are kept by segment and added up in their order, so that equal rows have equal sums
// whichever blocks they fell to.  A lower bound on the segment's n_out-th best entry comes from the maxima of groups of threads (there are at least
// n_out groups); the few chunks that reach it are read again, from L2 as a rule, an entry per lane, and entries from the bound on, a few dozen, go to shared
// memory.  Where too many tie, or an entry is no number, the segment is gone through once more and its n_out best keys are found bit by bit.  The first
// block ranks what all of them have left.  Nothing depends on the order of arrival.
// Bound: reading, and an exponential per entry on 16 lanes of special functions per SM, alike: 64 requests x 8 beams x 131,072 entries in bf16 take 37.6 us (bytes 21,
// exponentials 15; of a block's 57,000 cycles the stream takes 31,000, the ends of its two segments 11,500, joining and ranking 11,500); one request of 4 x 32,000 7.0 us, a chain of
// latencies.  Tried and slower: lists of the best
// kept while reading, ranked per segment (92), entries above a running bound written out by warps on their own (53).  Logits that fool the bound: all
// equal 228 us, rising with the token 1010 us (64 x 8 x 131,072); nine tenths masked with -1e10 or less, behind the others or among them, 37.4 us as with -infinity, but
// 38 us where one request of 4 x 32,000 has its good tokens side by side.
//
// Reordering.  The lowest new beam of each continued one keeps its slot; the others get the slots of beams that nobody continues, and only these are copied: sources
// stay as they are and every destination is a slot that nobody reads, so nothing has to wait for anything and there is no second buffer.  Bound: bytes.  16 requests
// x 4 beams, two forks each of 48 MB: 409 us, 7.9 TB/s where every byte is read and written once per fork (two forks of one beam read it from L2).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "decay_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512, NW = NT / 32;
constexpr int WORDS = 16;            // 32-bit words of a row that a thread holds at a time
constexpr int MAXW = kBeamMaxWidth, MAXN = kBeamMaxOut;  // beams per request, continuations wanted
constexpr int MAXS = 16;             // segments of a row
constexpr int CHUNKS = 16;           // parts of a thread's entries of a segment
constexpr int kMostHits = 4 * MAXN + 128;  // of a segment
constexpr float kNone = -__builtin_huge_valf(), kLog2e = 1.44269504f;
template <typename T>
constexpr float kLowest = sizeof(T) == 2 ? -3.38953139e38f : -3.40282347e38f;  // the type's lowest finite value

// 32 bits that order like the value
__device__ __forceinline__ uint32_t order32(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (one zero)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value32(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ uint64_t order64(double x) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double value64(uint64_t o) { return __longlong_as_double(static_cast<long long>(o >> 63 ? o & 0x7FFFFFFFFFFFFFFFull : ~o)); }
// larger logit first, then lower token; 0 is below every key
__device__ __forceinline__ uint64_t key_of(float x, int token) { return static_cast<uint64_t>(order32(x)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(token)); }
__device__ __forceinline__ int token_of(uint64_t key) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(key)); }
__device__ __forceinline__ float logit_of(uint64_t key) { return value32(static_cast<uint32_t>(key >> 32)); }

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __int_as_float(0x7f800000); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t dadd2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
struct Entry {
  uint64_t total;  // order64 of s
  uint64_t key;
  int beam, pad;
};
__device__ __forceinline__ bool ahead(const Entry &a, const Entry &b) {
  return a.total != b.total ? a.total > b.total : a.beam != b.beam ? a.beam < b.beam : a.key > b.key;
}

struct SelectSmem {
  double reference[MAXW * MAXS], sum[MAXW * MAXS];  // of each segment (those of this block): the sum of exponentials is e^reference times sum
  double lse[MAXW];
  float score[MAXW];
  int ended[MAXW];
  int counts[MAXW];  // the beams whose rows count
  float warp_top[MAXW][NW], warp_sum[MAXW][NW];  // the warps' shares of each of this block's segments
  uint32_t best_of[NT], bound;  // 16 or 32 bits of order of each thread's largest value
  int n_chosen[MAXW], n_hits[MAXW], odd[MAXW];  // of each of this block's segments
  int n_above, n_entries, n_left, n_rows;
  unsigned long long any_bit, all_bits;
  uint16_t chunk[CHUNKS][NT];   // the largest entry of each thread's chunks, 16 bits of order32
  uint16_t chosen[kMostHits];   // chunks that are read again: number * NT + thread
};
// behind it: uint64_t hit[segments of this block][a.budget], then in the first block Entry entry[all of them]

// A thread's part of a round: where entries of a row are, and how they come from memory
template <typename T, bool VEC>
struct Round {
  static constexpr bool PACKED = VEC && sizeof(T) == 2;
  static constexpr int EPT = PACKED ? 2 * WORDS : WORDS, SIZE = NT * EPT;  // entries per thread, and per block
  static constexpr int VW = VEC ? 16 / static_cast<int>(sizeof(T)) : 1;     // entries per load
  static __device__ __forceinline__ int index(int e, int thread) { return (e / VW * NT + thread) * VW + e % VW; }
  static __device__ __forceinline__ int index(int e) { return index(e, static_cast<int>(threadIdx.x)); }
  static __device__ __forceinline__ uint32_t bits(T x) {
    if constexpr (sizeof(T) == 2)
      return static_cast<uint32_t>(__bfloat16_as_ushort(x)) << 16;
    else
      return __float_as_uint(x);
  }
  // the first `len` entries from `row` on, at most SIZE; -infinity behind them
  static __device__ __forceinline__ void load(const T *row, int len, uint32_t (&w)[WORDS]) {
    constexpr uint32_t kPad = PACKED ? 0xFF80FF80u : 0xFF800000u;
    const T *const mine = row + static_cast<int>(threadIdx.x) * VW;
    if (len >= SIZE) {
#pragma unroll
      for (int l = 0; l < EPT / VW; ++l) {
        if constexpr (VEC) {
          const uint4 v = *reinterpret_cast<const uint4 *>(mine + l * NT * VW);
          w[4 * l] = v.x, w[4 * l + 1] = v.y, w[4 * l + 2] = v.z, w[4 * l + 3] = v.w;
        } else {
          w[l] = bits(mine[l * NT]);
        }
      }
      return;
    }
#pragma unroll
    for (int l = 0; l < EPT / VW; ++l) {
      const int left = len - (l * NT + static_cast<int>(threadIdx.x)) * VW;
      if constexpr (!VEC) {
        w[l] = left > 0 ? bits(mine[l * NT]) : kPad;
      } else if (left >= VW) {
        const uint4 v = *reinterpret_cast<const uint4 *>(mine + l * NT * VW);
        w[4 * l] = v.x, w[4 * l + 1] = v.y, w[4 * l + 2] = v.z, w[4 * l + 3] = v.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[4 * l + j] = kPad;
          if constexpr (PACKED) {
            if (2 * j < left) w[4 * l + j] = 0xFF800000u | bits(mine[l * NT * VW + 2 * j]) >> 16;
            if (2 * j + 1 < left) w[4 * l + j] = (w[4 * l + j] & 0xFFFFu) | bits(mine[l * NT * VW + 2 * j + 1]);
          } else {
            if (j < left) w[4 * l + j] = bits(mine[l * NT * VW + j]);
          }
        }
      }
    }
  }
  static __device__ __forceinline__ float get(const uint32_t (&w)[WORDS], int e) {
    if constexpr (PACKED)
      return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    else
      return __uint_as_float(w[e]);
  }
  static __device__ __forceinline__ float max(const uint32_t (&w)[WORDS]) {
    if constexpr (PACKED) {
      uint32_t m = w[0];
#pragma unroll
      for (int i = 1; i < WORDS; ++i) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i]));
      return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    } else {
      float m = __uint_as_float(w[0]);
#pragma unroll
      for (int i = 1; i < WORDS; ++i) m = fmaxf(m, __uint_as_float(w[i]));
      return m;
    }
  }
  // what is not a finite number becomes -infinity
  static __device__ __forceinline__ void clean(uint32_t (&w)[WORDS]) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (PACKED) {
        const float lo = get(w, 2 * i), hi = get(w, 2 * i + 1);
        w[i] = __byte_perm(__float_as_uint(finite(lo) ? lo : kNone), __float_as_uint(finite(hi) ? hi : kNone), 0x7632);
      } else {
        w[i] = finite(get(w, i)) ? w[i] : 0xFF800000u;
      }
    }
  }
  // Sum of e^(x - m).  The difference comes first, so that m's own term is 1 and no other one is larger however large m is: one multiply-add, x log2 e - c with c
  // a rounded m log2 e, is off by half a step of c, which from |m| of 2e9 on is more than an exponent has room for.
  static __device__ __forceinline__ float sum(const uint32_t (&w)[WORDS], float m) {
    const uint64_t r = dpack2(m, m), l = dpack2(kLog2e, kLog2e);
    uint64_t s[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < EPT; e += 2) {
      const float2 y = dunpack2(dmul2(dsub2(dpack2(get(w, e), get(w, e + 1)), r), l));
      s[e / 2 % 2] = dadd2(s[e / 2 % 2], dpack2(ex2(y.x), ex2(y.y)));
    }
    const float2 t = dunpack2(dadd2(s[0], s[1]));
    return t.x + t.y;
  }
};

// One more round's part of a thread's sum.  Sums of exponentials are relative to e^m, m the largest logit of what they are over.
template <typename Rd>
__device__ __forceinline__ float add_sum(const uint32_t (&w)[WORDS], float &m, float &s) {
  const float mr = Rd::max(w), mn = fmaxf(m, mr);
  const float part = Rd::sum(w, mn == kNone ? 0.f : mn), more = fmaf(s, ex2((m - mn) * kLog2e), part);
  s = m == kNone ? part : more;
  m = mn;
  return mr;
}
// A segment's sum of the threads': each warp leaves its share, and a warp adds them up at the end.
__device__ __forceinline__ void share_sum(SelectSmem &sm, int local, float m, float x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (threadIdx.x % 32 == 0) {
    sm.warp_top[local][threadIdx.x / 32] = m;
    sm.warp_sum[local][threadIdx.x / 32] = x;
  }
}
__device__ __forceinline__ double warp_max(double x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x = fmax(x, __shfl_xor_sync(0xffffffffu, x, d));
  return x;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}
// (factors between sums are good to 2^-22, as the exponentials themselves)
__device__ __forceinline__ void join_sums(const SelectSmem &sm, int local, double *to_reference, double *to_sum) {
  const int lane = threadIdx.x % 32;
  const float m = lane < NW ? sm.warp_top[local][lane] : kNone, top = warp_max(m);
  float x = lane < NW && m > kNone ? sm.warp_sum[local][lane] * ex2((m - top) * kLog2e) : 0.f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (lane == 0) {
    *to_reference = top;
    *to_sum = x;
  }
}

// A segment with a NaN or an infinity, or in which more entries were above the bound than there is room for (many that tie): once more, without what is no
// number, and its N best keys bit by bit from the top.  Called by the whole block; returns how many there are.
template <typename Rd, typename T>
__device__ __noinline__ int rescan(SelectSmem &sm, const T *row, int len, int from, int local, uint64_t *hit, int N) {
  const int tid = threadIdx.x;
  float m = kNone;
  for (int base = 0; base < len; base += Rd::SIZE) {
    uint32_t w[WORDS];
    Rd::load(row + base, len - base, w);
    Rd::clean(w);
    m = fmaxf(m, Rd::max(w));
  }
  m = warp_max(m);
  float s = 0.f;
  for (int base = 0; base < len; base += Rd::SIZE) {
    uint32_t w[WORDS];
    Rd::load(row + base, len - base, w);
    Rd::clean(w);
#pragma unroll
    for (int e = 0; e < Rd::EPT; ++e) s += ex2((Rd::get(w, e) - (m == kNone ? 0.f : m)) * kLog2e);
  }
  share_sum(sm, local, m, s);
  // The N best of the rounds so far are in `hit`, `least` of them the last; each round's better ones join them.
  int have = 0;
  uint64_t least = 0;
  for (int base = 0; base < len; base += Rd::SIZE) {
    uint32_t w[WORDS];
    Rd::load(row + base, len - base, w);
    Rd::clean(w);
    const int at = from + base;
    const uint64_t old = tid < have ? hit[tid] : 0;
    auto at_least = [&](uint64_t t) {  // how many keys there are from t on, this round's and the old ones
      const float v = value32(static_cast<uint32_t>(t >> 32));
      const uint32_t low = static_cast<uint32_t>(t), last = 0xFFFFFFFFu - static_cast<uint32_t>(at);
      int c = old >= t;
#pragma unroll
      for (int i = 0; i < WORDS; ++i) asm volatile("" : "+r"(w[i]));  // (nothing is kept from one bit to the next)
      if (low == 0) {
#pragma unroll
        for (int e = 0; e < Rd::EPT; ++e) c += Rd::get(w, e) >= v;
      } else {
#pragma unroll
        for (int e = 0; e < Rd::EPT; ++e) c += Rd::get(w, e) > v || (Rd::get(w, e) == v && last - Rd::index(e) >= low);
      }
      c = __reduce_add_sync(0xffffffffu, c);
      __syncthreads();
      if (tid == 0) sm.n_above = 0;
      __syncthreads();
      if (tid % 32 == 0 && c) atomicAdd(&sm.n_above, c);
      __syncthreads();
      return sm.n_above;
    };
    if (have == N && at_least(least + 1) < N) continue;
    uint64_t t = static_cast<uint64_t>(order32(kLowest<T>)) << 32;  // all of them
    if (at_least(t) > N) {
      // bit by bit from the top, those that differ between keys
      if (tid == 0) sm.any_bit = 0, sm.all_bits = ~0ull;
      __syncthreads();
      uint64_t any = old, all = old ? old : ~0ull;
#pragma unroll
      for (int e = 0; e < Rd::EPT; ++e) {
        const float x = Rd::get(w, e);
        const uint64_t key = key_of(x, at + Rd::index(e));
        if (x > kNone) any |= key, all &= key;
      }
      atomicOr(&sm.any_bit, any);
      atomicAnd(&sm.all_bits, all);
      __syncthreads();
      t = sm.all_bits;
      for (uint64_t bits = sm.any_bit ^ sm.all_bits; bits;) {
        const uint64_t bit = 1ull << (63 - __clzll(static_cast<long long>(bits)));
        if (at_least((t & ~(bit - 1)) | bit) >= N) t |= bit;
        bits ^= bit;
      }
    }
    __syncthreads();
    if (tid == 0) sm.n_left = 0;
    __syncthreads();
    if (old >= t) hit[atomicAdd(&sm.n_left, 1)] = old;
#pragma unroll
    for (int e = 0; e < Rd::EPT; ++e) {
      const float x = Rd::get(w, e);
      const uint64_t key = key_of(x, at + Rd::index(e));
      if (x > kNone && key >= t) hit[atomicAdd(&sm.n_left, 1)] = key;  // (N of them at most)
    }
    __syncthreads();
    have = sm.n_left;
    least = t;
    __syncthreads();
  }
  __syncthreads();
  if (tid == 0) sm.n_left = 0;
  return have;
}

// A lower bound on the N-th largest of many values, of which each thread has left its largest in `best_of` (0: none): the threads are G >= N groups, every G-th
// one together so that neighbours are apart, and the N-th largest of the groups' maxima is at most that.  By the whole block; `bound` is set behind the
// next barrier.
template <int G>
__device__ __forceinline__ void nth_of_groups(const uint32_t *best_of, int N, uint32_t *bound) {
  constexpr int PER = G / 32;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint32_t x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    x[i] = best_of[lane + 32 * i];
#pragma unroll
    for (int j = 1; j < NT / G; ++j) x[i] = max(x[i], best_of[lane + 32 * i + G * j]);
  }
#pragma unroll
  for (int i = 0; i < G / NW; ++i) {  // this warp's share of them: is it the one?
    const int g = warp * (G / NW) + i;
    uint32_t v = x[0];
#pragma unroll
    for (int j = 1; j < PER; ++j) v = g / 32 == j ? x[j] : v;
    v = __shfl_sync(0xffffffffu, v, g % 32);
    int above = 0, from = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      above += __popc(__ballot_sync(0xffffffffu, x[j] > v));
      from += __popc(__ballot_sync(0xffffffffu, x[j] >= v));
    }
    if (above < N && from >= N && lane == 0) *bound = v;
  }
}
__device__ __forceinline__ void find_bound(SelectSmem &sm, int N) {
  static_assert(MAXN <= 128, "a group for every n_out");
  if (N <= 32)
    nth_of_groups<64>(sm.best_of, N, &sm.bound);  // (with many values, 64 ln 2 = 44 of them are above it where N = 32, 18 where N = 16)
  else
    nth_of_groups<128>(sm.best_of, N, &sm.bound);
}

template <typename T, bool VEC, int CL>
__global__ void __launch_bounds__(NT, 2) beam_select_kernel(const __grid_constant__ DascBeamSelectArgs a) {
  using Rd = Round<T, VEC>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SelectSmem &sm = *reinterpret_cast<SelectSmem *>(smem_raw);
  uint64_t *const hit = reinterpret_cast<uint64_t *>(smem_raw + sizeof(SelectSmem));
  Entry *const entry = reinterpret_cast<Entry *>(hit + (a.per_block * a.budget + 1) / 2 * 2);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x % CL;
  const int W = a.width, N = a.n_out;
  stream_order_begin();

  if (tid < 32) {
    const float score = tid < W ? a.scores[static_cast<int64_t>(r) * W + tid] : kNone;
    // 0: its row counts, 1: it has ended, 2: it has no continuation
    const int ended = !finite(score) ? 2 : a.ended && a.ended[static_cast<int64_t>(r) * W + tid] != 0 ? 1 : 0;
    const uint32_t rows = __ballot_sync(0xffffffffu, ended == 0);
    const int place = __popc(rows & ((1u << tid) - 1u));
    sm.score[tid] = score;
    sm.ended[tid] = ended;
    if (ended == 0) sm.counts[place] = tid;
    if (tid == 0) sm.n_rows = __popc(rows);
  }
  if (tid < MAXW) sm.n_chosen[tid] = sm.n_hits[tid] = sm.odd[tid] = 0;
  if (tid == 0) sm.n_entries = sm.n_left = 0;
  __syncthreads();
  cg::cluster_group cluster = cg::this_cluster();
  auto there = cluster.barrier_arrive();  // (the first block is: waited for before anything is written to it)

  // the segments of the rows that count, shared out over the cluster's blocks
  const int items = sm.n_rows * a.segments, per_block = max((items + CL - 1) / CL, 1);
  const int first = min(rank * per_block, items), last = min(first + per_block, items);
  const int each = (a.segment_len + Rd::SIZE * CHUNKS - 1) / (Rd::SIZE * CHUNKS);  // rounds per chunk
  auto row_of = [&](int item) {
    return static_cast<const T *>(a.logits) + (static_cast<int64_t>(r) * W + sm.counts[item / a.segments]) * a.stride + item % a.segments * a.segment_len;
  };
  for (int item = first; item < last; ++item) {
    const int from = item % a.segments * a.segment_len, len = min(a.segment_len, a.vocab - from);
    const T *const row = row_of(item);
    // One pass over the segment: this thread's largest logit and its sum of exponentials, and the largest of each chunk of its entries.
    float m = kNone, s = 0.f, top = kNone;
    int chunks = 0, left = each;
    auto leave = [&](float x) {
      top = fmaxf(top, x);
      if (--left == 0) {
        sm.chunk[chunks++][tid] = static_cast<uint16_t>(order32(top) >> 16);
        left = each;
        top = kNone;
      }
    };
    for (int base = 0; base < len; base += 2 * Rd::SIZE) {  // two rounds' loads at a time
      uint32_t w[2][WORDS];
      Rd::load(row + base, len - base, w[0]);
      if (base + Rd::SIZE < len) Rd::load(row + base + Rd::SIZE, len - base - Rd::SIZE, w[1]);
      leave(add_sum<Rd>(w[0], m, s));
      if (base + Rd::SIZE < len) leave(add_sum<Rd>(w[1], m, s));
    }
    if (left != each) sm.chunk[chunks++][tid] = static_cast<uint16_t>(order32(top) >> 16);
    sm.best_of[tid] = order32(m) >> 16;
    const float high = warp_max(m);
    share_sum(sm, item - first, high, m == kNone ? 0.f : s * ex2((m - high) * kLog2e));
    // a NaN or an infinity, looked at as bits: a sum of ex2 is taken to be at least 0 by the assembler, and `!(s >= 0)` for never true
    const bool odd = __syncthreads_or(__float_as_uint(s) >= 0x7F800000u);
    find_bound(sm, N);
    if (tid == 0) sm.odd[item - first] = odd;
    __syncthreads();
    const uint32_t t = max(sm.bound, order32(kLowest<T>) >> 16);
    if (odd) continue;
    // The few chunks that may hold one of the best (each has an entry from the bound on) are shared out over the warps and read again, an entry
    // per lane.  Each warp with those of its own threads, us: 64 requests x 4 beams x 131,072 fp32 entries 32.4 instead of 30.3, one of 4 x 32,000 with many
    // good neighbours 8.2 instead of 7.3, 64 x 32 x 32,768 (eight short segments per block) 59 instead of 63.  All segments' at the end: 31.4, 8.0, 67.
#pragma unroll 4
    for (int c = 0; c < chunks; ++c) {
      const bool chosen = sm.chunk[c][tid] >= t;
      const uint32_t who = __ballot_sync(0xffffffffu, chosen);
      if (!who) continue;
      int to = lane == 0 ? atomicAdd(&sm.n_chosen[item - first], __popc(who)) : 0;
      to = __shfl_sync(0xffffffffu, to, 0) + __popc(who & ((1u << lane) - 1u));
      if (chosen && to < a.budget) sm.chosen[to] = static_cast<uint16_t>(c * NT + tid);
    }
    __syncthreads();
    const int n = sm.n_chosen[item - first];
    if (n > a.budget) continue;  // (all of it once more, see rescan)
    const float bound = value32(t << 16);
    for (int j = warp; j < n; j += NW) {
      const int c = sm.chosen[j] / NT, thread = sm.chosen[j] % NT;
      for (int i = lane; i < each * Rd::EPT; i += 32) {
        const int at = (c * each + i / Rd::EPT) * Rd::SIZE + Rd::index(i % Rd::EPT, thread);
        const float x = at < len ? __uint_as_float(Rd::bits(row[at])) : kNone;
        if (x >= bound) {
          const int to = atomicAdd(&sm.n_hits[item - first], 1);
          if (to < a.budget) hit[(item - first) * a.budget + to] = key_of(x, from + at);
        }
      }
    }
  }
  __syncthreads();
  for (int item = first; item < last; ++item) {
    const bool again = sm.odd[item - first] || sm.n_chosen[item - first] > a.budget || sm.n_hits[item - first] > a.budget;  // (the same for the whole block)
    if (!again) continue;
    const int from = item % a.segments * a.segment_len;
    const int n = rescan<Rd>(sm, row_of(item), min(a.segment_len, a.vocab - from), from, item - first, hit + (item - first) * a.budget, N);
    if (tid == 0) sm.n_hits[item - first] = n;
    __syncthreads();
  }

  // The first block takes the hits and sums of all of them.
  cluster.barrier_wait(std::move(there));
  {
    SelectSmem &to = *cluster.map_shared_rank(&sm, 0);
    Entry *const entries = cluster.map_shared_rank(entry, 0);
    for (int item = first + warp; item < last; item += NW) {
      const int local = item - first, n = sm.n_hits[local];
      int at = 0;
      if (lane == 0 && n > 0) at = atomicAdd(&to.n_entries, n);
      join_sums(sm, local, &to.reference[item], &to.sum[item]);
      at = __shfl_sync(0xffffffffu, at, 0);
      for (int i = lane; i < n; i += 32) {
        entries[at + i].key = hit[local * a.budget + i];
        entries[at + i].beam = sm.counts[item / a.segments];
      }
    }
    if (rank == 0 && tid < W && sm.ended[tid] == 1) {
      const int at = atomicAdd(&sm.n_entries, 1);
      entry[at].key = key_of(0.f, a.end_token);
      entry[at].beam = tid;
    }
  }
  cluster.sync();
  if (rank != 0) return;
  for (int row = warp; row < sm.n_rows; row += NW) {
    const int item = row * a.segments + lane;
    const double ref = lane < a.segments ? sm.reference[item] : -INFINITY, top = warp_max(ref);
    const double x = warp_sum(ref > -INFINITY ? sm.sum[item] * ex2(static_cast<float>(ref - top) * kLog2e) : 0.0);
    if (lane == 0) sm.lse[sm.counts[row]] = top + log(x);
  }
  __syncthreads();
  int total = sm.n_entries;
  uint64_t mine = 0;  // this thread's best total
  for (int i = tid; i < total; i += NT) {
    const int b = entry[i].beam;
    const double score = sm.score[b];
    entry[i].total = order64(sm.ended[b] ? score : score + (static_cast<double>(logit_of(entry[i].key)) - sm.lse[b]));
    mine = max(mine, entry[i].total);
  }
  __syncthreads();
  // Those that may be among the N best by 32 bits of their totals; where there are few, all.
  uint16_t *const kept = sm.chunk[0];  // (indexes of at most MAXW * budget of them)
  if (total > NT / 8) {
    sm.best_of[tid] = static_cast<uint32_t>(mine >> 32);
    __syncthreads();
    find_bound(sm, N);
    __syncthreads();
    const uint32_t t = sm.bound;
    for (int i = tid; i < total; i += NT)
      if (static_cast<uint32_t>(entry[i].total >> 32) >= t) kept[atomicAdd(&sm.n_left, 1)] = static_cast<uint16_t>(i);
    __syncthreads();
    total = sm.n_left;
  } else {
    for (int i = tid; i < total; i += NT) kept[i] = static_cast<uint16_t>(i);
    __syncthreads();
  }
  const int64_t out = static_cast<int64_t>(r) * N;
  for (int i0 = 0; i0 < total; i0 += NT / 8) {  // eight lanes count how many are ahead of each
    const int i = i0 + tid / 8;
    const Entry e = entry[kept[min(i, total - 1)]];
    int place = 0;
    for (int j = tid % 8; j < total; j += 8) place += ahead(entry[kept[j]], e);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) place += __shfl_xor_sync(0xffffffffu, place, d);
    if (i < total && tid % 8 == 0 && place < N) {
      const int token = token_of(e.key);
      a.out_scores[out + place] = static_cast<float>(value64(e.total));
      a.out_parent[out + place] = e.beam;
      a.out_token[out + place] = token;
      if (a.out_ended) a.out_ended[out + place] = sm.ended[e.beam] == 1 || token == a.end_token;
    }
  }
  for (int i = total + tid; i < N; i += NT) {
    a.out_scores[out + i] = kNone;
    a.out_parent[out + i] = a.out_token[out + i] = -1;
    if (a.out_ended) a.out_ended[out + i] = 1;
  }
}

template <typename T, bool VEC, int CL>
int select(DascBeamSelectArgs a, void *stream) {
  // Segments of a row, the same for all rows: whole rounds as far as possible.  A segment's end costs its block about as much as another round.
  using Rd = Round<T, VEC>;
  constexpr size_t kEntries = 40 * 1024;  // bytes of entries that leave room for two blocks per SM
  int64_t least = INT64_MAX;
  for (int n = 1; n <= MAXS; ++n) {
    const int64_t len = ((a.vocab + n - 1) / n + 7) / 8 * 8, per_block = (static_cast<int64_t>(a.width) * n + CL - 1) / CL;
    const int64_t cost = per_block * ((len + Rd::SIZE - 1) / Rd::SIZE + 1);
    if (cost < least && (n == 1 || (per_block <= MAXW && a.width * n * (2 * a.n_out + 64) * sizeof(Entry) <= kEntries))) {
      least = cost;
      a.segment_len = static_cast<int32_t>(len);
    }
  }
  a.segments = (a.vocab + a.segment_len - 1) / a.segment_len;
  a.per_block = (a.width * a.segments + CL - 1) / CL;
  // hits per segment: about 1.1 n_out are to be expected, more where good tokens are neighbours
  a.budget = std::max(2 * a.n_out + 64, std::min(4 * a.n_out + 128, static_cast<int>(kEntries / sizeof(Entry)) / (a.width * a.segments)));
  // hits of this block's segments; entries of all segments, a beam that has ended has none but its own
  const size_t smem = sizeof(SelectSmem) + static_cast<size_t>(a.per_block * a.budget + 1) / 2 * 16 +
                      static_cast<size_t>(a.width * a.segments) * a.budget * sizeof(Entry);
  auto kernel = beam_select_kernel<T, VEC, CL>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return static_cast<int>(e);
  }
  return static_cast<int>(launch_clusters(kernel, dim3(static_cast<unsigned>(a.n_req) * CL), dim3(NT), CL, smem, stream, a));
}

template <typename T>
int select_type(const DascBeamSelectArgs &a, void *stream) {
  const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.stride * static_cast<int64_t>(sizeof(T)) % 16 == 0;
  const auto with = [&](auto cl) {
    constexpr int CL = decltype(cl)::value;
    return vec ? select<T, true, CL>(a, stream) : select<T, false, CL>(a, stream);
  };
  // As many blocks per request as still fit the GPU at once, two per SM (not every GPC holds a whole number of clusters of 4 or 8).  4 beams over 65,536 entries
  // in bf16, us with 8 / 4 / 2 / 1 blocks: 1 request 9.4 / 10.1 / 14.3 / 22.7, 37 requests 17.5 / 14.4 / 15.0 / 23.4, 64 requests 22.8 / 14.6 / 21.2 / 30.1, 148 requests
  // 45.6 / 31.1 / 22.5 / 25.6, 296 requests 90 / 58 / 45 / 42.
  constexpr int kPlaces = 2 * 148, kClustered = kPlaces * 7 / 8;
  if (a.n_req * int64_t{8} <= kClustered) return with(std::integral_constant<int, 8>{});
  if (a.n_req * int64_t{4} <= kClustered) return with(std::integral_constant<int, 4>{});
  if (a.n_req * int64_t{2} <= kPlaces) return with(std::integral_constant<int, 2>{});
  return with(std::integral_constant<int, 1>{});
}

// ---- reordering --------------------------------------------------------------------------------------------------------------

// A thread block copies one tile of 16 KB of every fork of its request.  More of them per block are slower: two forks in each of 16 requests over 24 layers of 32 heads
// (both from one beam) with 1 / 2 / 4 / 8 tiles 350 / 361 / 420 / 485 us, one request with one fork 13.9 / 13.4 / 14.2 / 14.6.
constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyTile = kCopyThreads * kCopyUnroll;  // vectors of 16 bytes

// this block's vectors of a tile that ends at `end`
__device__ __forceinline__ void copy_tile(const uint4 *src, uint4 *dst, uint32_t begin, uint32_t end) {
  const uint32_t base = begin + threadIdx.x;
  uint4 v[kCopyUnroll];
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u)
    if (base + u * kCopyThreads < end)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(v[u].x), "=r"(v[u].y), "=r"(v[u].z), "=r"(v[u].w)
                   : "l"(src + base + u * kCopyThreads));
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u)
    if (base + u * kCopyThreads < end)
      asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(dst + base + u * kCopyThreads), "r"(v[u].x), "r"(v[u].y),
                   "r"(v[u].z), "r"(v[u].w)
                   : "memory");
}

__global__ void __launch_bounds__(kCopyThreads) beam_reorder_kernel(const __grid_constant__ DascBeamReorderArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t g = blockIdx.x / a.pieces;
  const uint32_t piece = static_cast<uint32_t>(blockIdx.x % a.pieces);
  stream_order_begin();
  // every warp for itself: lane i is new beam i, and old beam i
  const bool in = lane < a.width;
  const int64_t at = g * a.width + lane;
  const int slot = in ? a.req_idx[at] : -1;
  int parent = in ? a.parent[at] : -1;
  if (parent >= a.width) parent = -1;
  const bool has = parent >= 0;
  const uint32_t same = __match_any_sync(0xffffffffu, parent);
  const bool keeps = has && __ffs(same) - 1 == lane;
  const uint32_t continued = __reduce_or_sync(0xffffffffu, has ? 1u << parent : 0u);
  const uint32_t beams = a.width == 32 ? 0xffffffffu : (1u << a.width) - 1u;
  uint32_t free = beams & ~continued;
  const uint32_t others = __ballot_sync(0xffffffffu, in && !keeps);
  for (int i = __popc(others & ((1u << lane) - 1u)); i > 0; --i) free &= free - 1;  // (as many free slots as others)
  const int of = __shfl_sync(0xffffffffu, slot, has ? parent : 0);
  const int src = has ? of : -1;
  const int given = __shfl_sync(0xffffffffu, slot, free ? __ffs(free) - 1 : 0);
  const int dst = keeps ? src : given;
  if (piece == 0 && threadIdx.x < a.width) {
    a.new_idx[at] = dst;
    if (a.src_idx) a.src_idx[at] = src;
  }
  uint32_t forks = __ballot_sync(0xffffffffu, in && has && !keeps && src >= 0 && dst >= 0);
  const uint32_t state_pieces = static_cast<uint32_t>(a.n_layers_in_call) * a.layer_pieces;
  for (; forks; forks &= forks - 1) {
    const int i = __ffs(forks) - 1;
    const int64_t s = __shfl_sync(0xffffffffu, src, i), d = __shfl_sync(0xffffffffu, dst, i);
    if (piece < state_pieces) {
      const int64_t layer = (a.layer_begin + static_cast<int64_t>(piece / a.layer_pieces)) * a.layer_stride;
      const uint32_t begin = piece % a.layer_pieces * kCopyTile;
      copy_tile(reinterpret_cast<const uint4 *>(a.state + s * a.req_stride + layer), reinterpret_cast<uint4 *>(a.state + d * a.req_stride + layer), begin,
                a.layer_vecs);
    } else if (a.conv_vecs) {
      copy_tile(reinterpret_cast<const uint4 *>(static_cast<const char *>(a.conv) + s * a.conv_stride),
                reinterpret_cast<uint4 *>(static_cast<char *>(a.conv) + d * a.conv_stride), (piece - state_pieces) * kCopyTile, a.conv_vecs);
    }
  }
}

}  // namespace

int dasc_launch_beam_select(const DascBeamSelectArgs &a, void *stream) {
  return a.bf16 ? select_type<__nv_bfloat16>(a, stream) : select_type<float>(a, stream);
}

int dasc_launch_beam_reorder(DascBeamReorderArgs a, void *stream) {
  const int64_t layer_vecs = a.state ? a.layer_vecs : 0, conv_pieces = (a.conv_vecs + kCopyTile - 1) / kCopyTile;
  a.layer_pieces = static_cast<uint32_t>((layer_vecs + kCopyTile - 1) / kCopyTile);
  const int64_t pieces = std::max(int64_t{1}, static_cast<int64_t>(a.n_layers_in_call) * a.layer_pieces + conv_pieces);
  if (pieces * a.n_req > 2147483647LL) return static_cast<int>(cudaErrorInvalidConfiguration);
  a.pieces = static_cast<uint32_t>(pieces);
  return static_cast<int>(launch_blocks(beam_reorder_kernel, dim3(static_cast<unsigned>(pieces * a.n_req)), dim3(kCopyThreads), 0, stream, a));
}
