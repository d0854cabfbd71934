// Beam search over recurrent states: the best continuations over beams and vocabulary, and the states behind them.
//
// Selection.  A continuation of beam b by token v weighs s = score_b + (x_bv - log sum exp x_b), in 64 bits; the best n_out of a
// request's width x vocab continuations are wanted.  Inside a beam they are ordered like the logits themselves, so each part of a row gives its best n_out
// by 64-bit keys (logit, then lower token) while it sums exponentials, all from one pass over the row, and the few that are left meet with their beams' sums.
// Split: a request is a cluster of CL thread blocks; the rows of its beams are cut into segments, alike for all rows, which the blocks take in
// order.  A block goes through a segment in rounds of 64 bytes per thread, the next round's loads in flight.  Sums are kept by segment and added up in
// their order, so that equal rows have equal sums whichever blocks they fell to.  A lower bound on the segment's n_out-th best entry comes from the
// maxima of groups of threads (there are at least n_out groups); the entries above it, a few dozen as a rule, go to shared memory and are ranked
// there by counting at the segment's end.  Where too many tie or the bound is poor, a round's n_out-th key is found by bisection.  The first block
// ranks what all of them have left.  Nothing depends on the order of arrival.
//
// Reordering.  The lowest new beam of each continued one keeps its slot; the others get the slots of beams that nobody continues, and only these are copied: sources
// stay as they are and every destination is a slot that nobody reads, so nothing has to wait for anything and there is no second buffer.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "decay_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512, NW = NT / 32;
constexpr int WORDS = 16;            // 32-bit words of a row that a thread holds at a time
constexpr int CAP = 512;             // entries above the bound that are collected before they are ranked
constexpr int MAXW = kBeamMaxWidth, MAXN = kBeamMaxOut;  // beams per request, continuations wanted
constexpr int MAXS = 16;             // segments of a row
constexpr int GROUPS = 64;           // of NT / 64 threads, whose maxima bound the n_out-th best entry; at least MAXN
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
  uint64_t cand[CAP + MAXN];
  float top[MAXW * MAXS];     // of each segment (those of this block): the largest logit, and the sum of exponentials relative to it
  double sum[MAXW * MAXS];
  float group_max[GROUPS], bound, warp_top[NW], warp_sum[NW];
  int n_cand, n_above, n_entries;
  float score[MAXW];
  int ended[MAXW], count[MAXW];
  double lse[MAXW];
};
// behind it: uint64_t list[beams per block][n_out], best first; then a round's words where they are searched for the n_out-th key, and at the end
// in the first block Entry entry[lists of all blocks][n_out]

// A thread's part of a round: where entries of a row are, and how they come from memory
template <typename T, bool VEC>
struct Round {
  static constexpr bool PACKED = VEC && sizeof(T) == 2;
  static constexpr int EPT = PACKED ? 2 * WORDS : WORDS, SIZE = NT * EPT;  // entries per thread, and per block
  static constexpr int VW = VEC ? 16 / static_cast<int>(sizeof(T)) : 1;     // entries per load
  static __device__ __forceinline__ int index(int e) { return (e / VW * NT + static_cast<int>(threadIdx.x)) * VW + e % VW; }
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
  // sum of e^(x - ref); differences first, since a product with log2 e ahead of them would be off by the same amount in all of a row's terms
  static __device__ __forceinline__ float sum(const uint32_t (&w)[WORDS], float ref) {
    const uint64_t r = dpack2(ref, ref), l = dpack2(kLog2e, kLog2e);
    uint64_t s[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < EPT; e += 2) {
      const float2 y = dunpack2(dmul2(dsub2(dpack2(get(w, e), get(w, e + 1)), r), l));
      s[e / 2 % 2] = dadd2(s[e / 2 % 2], dpack2(ex2(y.x), ex2(y.y)));
    }
    const float2 t = dunpack2(dadd2(s[0], s[1]));
    return t.x + t.y;
  }
  // which entries are at least `bound` (one of the type's values): bit place(e) for entry e
  static __device__ __forceinline__ uint32_t at_least(const uint32_t (&w)[WORDS], float bound) {
    uint32_t hits = 0;
    if constexpr (PACKED) {
      const uint32_t b = __byte_perm(__float_as_uint(bound), 0, 0x3232);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        uint32_t yes;
        asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(yes) : "r"(w[i]), "r"(b));
        hits |= yes & 0x00010001u << i;
      }
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) hits |= __uint_as_float(w[i]) >= bound ? 1u << i : 0u;
    }
    return hits;
  }
  static __device__ __forceinline__ int entry(int place) { return PACKED ? 2 * (place % WORDS) + place / WORDS : place; }
  // entry e, which differs from thread to thread
  static __device__ __forceinline__ float pick(const uint32_t (&w)[WORDS], int e) {
    uint32_t x = w[0];
#pragma unroll
    for (int i = 1; i < WORDS; ++i) x = (PACKED ? e / 2 : e) == i ? w[i] : x;
    return __uint_as_float(!PACKED || e & 1 ? (PACKED ? x & 0xFFFF0000u : x) : x << 16);
  }
};

// The `n` keys that have been collected join the `have` ones of a list, of which the N best stay, best first; eight lanes count how many are
// ahead of each.  Called by the whole block behind a barrier, and ends with one; returns how many the list has now.
__device__ __noinline__ int join_list(SelectSmem &sm, uint64_t *best, int n, int have, int N) {
  const int tid = threadIdx.x, total = n + have;
  if (tid < have) sm.cand[n + tid] = best[tid];
  __syncthreads();
  for (int i0 = 0; i0 < total; i0 += NT / 8) {
    const int i = i0 + tid / 8;
    const uint64_t k = i < total ? sm.cand[i] : 0;
    int place = 0;
    for (int j = tid % 8; j < total; j += 8) place += sm.cand[j] > k;
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) place += __shfl_xor_sync(0xffffffffu, place, d);
    if (i < total && tid % 8 == 0 && place < N) best[place] = k;
  }
  if (tid == 0) sm.n_cand = 0;
  __syncthreads();
  return min(total, N);
}

// A warp's share of a segment's sum, relative to its own largest logit.
__device__ __forceinline__ void share_sum(SelectSmem &sm, float m, float s) {
  const float top = warp_max(m);
  float x = s * ex2((m - (top == kNone ? 0.f : top)) * kLog2e);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (threadIdx.x % 32 == 0) {
    sm.warp_top[threadIdx.x / 32] = top;
    sm.warp_sum[threadIdx.x / 32] = x;
  }
}
// one more round's part of a thread's sum
template <typename Rd>
__device__ __forceinline__ float add_sum(const uint32_t (&w)[WORDS], float &m, float &s) {
  const float mr = Rd::max(w), mn = fmaxf(m, mr), ref = mn == kNone ? 0.f : mn;
  s = fmaf(s, ex2((m - ref) * kLog2e), Rd::sum(w, ref));
  m = mn;
  return mr;
}

// A segment with a NaN or an infinity, or in which more entries were above the bound than there is room for (many that tie, or a poor bound): once more, a round at
// a time, each with the keys above the N-th best so far, of which at most N are collected.  `words`: a round's words in shared memory.  Called by the
// whole block behind a barrier; leaves the warps' sums and returns how many the list has.
template <typename Rd, typename T>
__device__ __noinline__ int rescan(SelectSmem &sm, uint32_t *words, const T *row, int len, int from, uint64_t *best, int have, int N) {
  const int tid = threadIdx.x;
  auto value = [&](int e) {
    if constexpr (Rd::PACKED) {
      const uint32_t x = words[e / 2 * NT + tid];
      return __uint_as_float(e & 1 ? x & 0xFFFF0000u : x << 16);
    } else {
      return __uint_as_float(words[e * NT + tid]);
    }
  };
  float m = kNone, s = 0.f;
  for (int base = 0; base < len; base += Rd::SIZE) {
    uint32_t w[WORDS];
    Rd::load(row + base, len - base, w);
    Rd::clean(w);
    add_sum<Rd>(w, m, s);
#pragma unroll
    for (int i = 0; i < WORDS; ++i) words[i * NT + tid] = w[i];  // (each thread reads its own)
    const int at = from + base;
    auto at_least = [&](uint64_t t) {  // how many keys there are from t on
      int c = 0;
#pragma unroll 4
      for (int e = 0; e < Rd::EPT; ++e) {
        const float x = value(e);
        c += x > kNone && key_of(x, at + Rd::index(e)) >= t;
      }
      c = __reduce_add_sync(0xffffffffu, c);
      __syncthreads();
      if (tid == 0) sm.n_above = 0;
      __syncthreads();
      if (tid % 32 == 0 && c) atomicAdd(&sm.n_above, c);
      __syncthreads();
      return sm.n_above;
    };
    uint64_t t = have == N ? best[N - 1] + 1 : 1;
    int n = at_least(t);
    if (n == 0) continue;
    if (n > CAP) {  // the N-th largest key, bit by bit from the top
      t = 0;
      for (int bit = 63; bit >= 0; --bit)
        if (at_least(t | 1ull << bit) >= N) t |= 1ull << bit;
    }
    __syncthreads();
    if (tid == 0) sm.n_cand = 0;
    __syncthreads();
    for (int e = 0; e < Rd::EPT; ++e) {
      const float x = value(e);
      const uint64_t key = key_of(x, at + Rd::index(e));
      if (x > kNone && key >= t) sm.cand[atomicAdd(&sm.n_cand, 1)] = key;  // (at most CAP of them, or N)
    }
    __syncthreads();
    n = sm.n_cand;
    __syncthreads();
    have = join_list(sm, best, n, have, N);
  }
  share_sum(sm, m, s);
  __syncthreads();
  if (tid == 0) sm.n_cand = 0;
  __syncthreads();
  return have;
}

template <typename T, bool VEC, int CL>
__global__ void __launch_bounds__(NT, 2) beam_select_kernel(const __grid_constant__ DascBeamSelectArgs a) {
  using Rd = Round<T, VEC>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SelectSmem &sm = *reinterpret_cast<SelectSmem *>(smem_raw);
  uint64_t *const list = reinterpret_cast<uint64_t *>(smem_raw + sizeof(SelectSmem));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x % CL;
  const int W = a.width, N = a.n_out;
  stream_order_begin();

  if (tid < W) {
    const float score = a.scores[static_cast<int64_t>(r) * W + tid];
    sm.score[tid] = score;
    // 0: its row counts, 1: it has ended, 2: it has no continuation
    sm.ended[tid] = !finite(score) ? 2 : a.ended && a.ended[static_cast<int64_t>(r) * W + tid] != 0 ? 1 : 0;
    sm.count[tid] = 0;
  }
  if (tid == 0) sm.n_cand = sm.n_entries = 0;
  __syncthreads();

  const int first = min(rank * a.per_block, W * a.segments), last = min(first + a.per_block, W * a.segments), first_beam = first / a.segments;
  // where this block is: a segment of a beam's row, and how many of its entries are left; rows that do not count are passed over
  struct Place {
    const T *row;
    int item, beam, segment, left;
  };
  auto open = [&](Place &p) {
    p.left = min(a.segment_len, a.vocab - p.segment * a.segment_len);
    p.row = static_cast<const T *>(a.logits) + (static_cast<int64_t>(r) * W + p.beam) * a.stride + p.segment * a.segment_len;
  };
  auto skip = [&](Place &p) {
    while (p.item < last && sm.ended[p.beam]) {
      p.item += a.segments - p.segment;
      p.segment = 0;
      ++p.beam;
    }
    if (p.item < last) open(p);
  };
  auto advance = [&](Place &p) {
    p.row += Rd::SIZE;
    p.left -= Rd::SIZE;
    if (p.left <= 0) {
      ++p.item;
      if (++p.segment == a.segments) {
        p.segment = 0;
        ++p.beam;
      }
      skip(p);
    }
  };
  Place next{nullptr, first, first_beam, first - first_beam * a.segments, 0};
  skip(next);
  uint32_t w[WORDS], ahead_w[WORDS];
  if (next.item < last) Rd::load(next.row, next.left, ahead_w);
  float m = kNone, s = 0.f;  // this thread's largest logit of the segment, and sum of exponentials relative to it
  int round = 0;
  volatile float *const group_max = sm.group_max, *const shared_bound = &sm.bound;
  while (next.item < last) {
    const Place at = next;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = ahead_w[i];
    advance(next);
    if (next.item < last) Rd::load(next.row, next.left, ahead_w);

    const float mr = add_sum<Rd>(w, m, s);
    uint64_t *const best = list + (at.beam - first_beam) * N;
    const int have = sm.count[at.beam];
    uint64_t floor = 0;
    float bound;
    if (have == N) {
      floor = best[N - 1];
      bound = logit_of(floor);
    } else {
      // At any time once all groups of threads have left the largest entry they have seen of this segment, the N-th largest of those is at most
      // the segment's N-th best entry.  Found to 16 bits of order32; all warps look for it in the first round, then one of them now and then.
      float g = m;
#pragma unroll
      for (int d = 1; d < NT / GROUPS; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
      if (lane % (NT / GROUPS) == 0) group_max[tid / (NT / GROUPS)] = g;
      if (round == 0) __syncthreads();
      if (round == 0 || ((round & (round - 1)) == 0 && warp == round % NW)) {
        const uint32_t x = order32(group_max[lane]), y = order32(group_max[lane + 32]);
        uint32_t t = 0;
        for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1) {
          const uint32_t trial = t | bit;
          if (__popc(__ballot_sync(0xffffffffu, x >= trial)) + __popc(__ballot_sync(0xffffffffu, y >= trial)) >= N) t = trial;
        }
        *shared_bound = fmaxf(t == 0 ? kNone : value32(t), kLowest<T>);  // (the same from all warps of the first round, or larger from a later one)
        __syncwarp();
      }
      bound = *shared_bound;
    }
    if (mr >= bound) {
      for (uint32_t hits = Rd::at_least(w, bound); hits; hits &= hits - 1) {
        const int e = Rd::entry(__ffs(hits) - 1);
        const uint64_t key = key_of(Rd::pick(w, e), at.segment * a.segment_len + round * Rd::SIZE + Rd::index(e));
        if (key > floor) {
          const int to = atomicAdd(&sm.n_cand, 1);
          if (to < CAP) sm.cand[to] = key;
        }
      }
    }
    ++round;
    if (next.item != at.item) {  // the segment's end
      share_sum(sm, m, s);
      // a NaN or an infinity, looked at as bits: a sum of ex2 is taken to be at least 0 by the assembler, and `!(s >= 0)` for never true
      const bool odd = __syncthreads_or(__float_as_uint(s) >= 0x7F800000u);
      const int n = sm.n_cand;
      int now;
      if (odd || n > CAP) {
        const int from = at.segment * a.segment_len;
        __syncthreads();
        now = rescan<Rd>(sm, reinterpret_cast<uint32_t *>(list + a.block_beams * N), at.row - (round - 1) * Rd::SIZE, min(a.segment_len, a.vocab - from), from,
                         best, have, N);
      } else {
        now = join_list(sm, best, n, have, N);
      }
      if (warp == 0) {
        const float its = lane < NW ? sm.warp_top[lane] : kNone, top = warp_max(its);
        double x = its > kNone ? sm.warp_sum[lane] * exp(static_cast<double>(its) - top) : 0.0;
#pragma unroll
        for (int d = NW / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (lane == 0) {
          sm.top[at.item] = top;
          sm.sum[at.item] = x;
          sm.count[at.beam] = now;
        }
      }
      m = kNone;
      s = 0.f;
      round = 0;
      __syncthreads();
    }
  }

  // The first block takes the lists and sums of all of them.
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  Entry *const entry = reinterpret_cast<Entry *>(list + a.block_beams * N);
  if (rank == 0) {
    if (tid < W && sm.ended[tid] == 0) {
      float top = kNone;
      for (int i = tid * a.segments; i < (tid + 1) * a.segments; ++i) top = fmaxf(top, cluster.map_shared_rank(sm.top, i / a.per_block)[i]);
      double x = 0.0;
      if (top > kNone)
        for (int i = tid * a.segments; i < (tid + 1) * a.segments; ++i) {
          const float t = cluster.map_shared_rank(sm.top, i / a.per_block)[i];
          if (t > kNone) x += cluster.map_shared_rank(sm.sum, i / a.per_block)[i] * exp(static_cast<double>(t) - top);
        }
      sm.lse[tid] = static_cast<double>(top) + log(x);
    }
    __syncthreads();
    for (int i = tid; i < CL * a.block_beams * N; i += NT) {
      const int c = i / (a.block_beams * N), j = i % (a.block_beams * N), its_first = c * a.per_block / a.segments, b = its_first + j / N;
      if (c * a.per_block < W * a.segments && b * a.segments < min((c + 1) * a.per_block, W * a.segments) && j % N < cluster.map_shared_rank(sm.count, c)[b]) {
        Entry e;
        e.key = cluster.map_shared_rank(list, c)[j];
        e.total = order64(static_cast<double>(sm.score[b]) + (static_cast<double>(logit_of(e.key)) - sm.lse[b]));
        e.beam = b;
        entry[atomicAdd(&sm.n_entries, 1)] = e;
      }
    }
    if (tid < W && sm.ended[tid] == 1) {
      Entry e;
      e.key = key_of(0.f, a.end_token);
      e.total = order64(sm.score[tid]);
      e.beam = tid;
      entry[atomicAdd(&sm.n_entries, 1)] = e;
    }
  }
  cluster.sync();  // (no block ends while the first one still reads it)
  if (rank != 0) return;
  const int total = sm.n_entries;
  const int64_t out = static_cast<int64_t>(r) * N;
  for (int i0 = 0; i0 < total; i0 += NT / 8) {
    const int i = i0 + tid / 8;
    const Entry e = entry[min(i, total - 1)];
    int place = 0;
    for (int j = tid % 8; j < total; j += 8) place += ahead(entry[j], e);
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
  int64_t least = INT64_MAX;
  for (int n = 1; n <= MAXS; ++n) {
    const int64_t len = ((a.vocab + n - 1) / n + 7) / 8 * 8, cost = (static_cast<int64_t>(a.width) * n + CL - 1) / CL * ((len + Rd::SIZE - 1) / Rd::SIZE + 1);
    if (cost < least) {
      least = cost;
      a.segment_len = static_cast<int32_t>(len);
    }
  }
  a.segments = (a.vocab + a.segment_len - 1) / a.segment_len;
  a.per_block = (a.width * a.segments + CL - 1) / CL;
  a.block_beams = std::min(a.width, (a.per_block + a.segments - 2) / a.segments + 1);
  // lists of this block's beams; entries of all lists and of the beams that have ended (a beam that is in several blocks has not)
  const size_t smem = sizeof(SelectSmem) + static_cast<size_t>(a.block_beams) * sizeof(uint64_t) * a.n_out +
                      std::max(static_cast<size_t>(a.width + CL) * sizeof(Entry) * a.n_out, NT * WORDS * sizeof(uint32_t));
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
  constexpr int kPlaces = 2 * 148;
  constexpr int kClustered = kPlaces * 7 / 8;  // (not every GPC holds a whole number of clusters of 4 or 8)
  if (a.n_req * int64_t{8} <= kClustered) return with(std::integral_constant<int, 8>{});
  if (a.n_req * int64_t{4} <= kClustered) return with(std::integral_constant<int, 4>{});
  if (a.n_req * int64_t{2} <= kPlaces) return with(std::integral_constant<int, 2>{});
  return with(std::integral_constant<int, 1>{});
}

// ---- reordering --------------------------------------------------------------------------------------------------------------

constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyTile = kCopyThreads * kCopyUnroll;  // vectors of 16 bytes per round of a block

__device__ __forceinline__ void copy_range(const uint4 *src, uint4 *dst, uint32_t begin, uint32_t end) {
  for (uint32_t base = begin + threadIdx.x; base < end; base += kCopyTile) {
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
      const uint32_t begin = piece % a.layer_pieces * a.piece_vecs;
      copy_range(reinterpret_cast<const uint4 *>(a.state + s * a.req_stride + layer), reinterpret_cast<uint4 *>(a.state + d * a.req_stride + layer), begin,
                 min(begin + a.piece_vecs, a.layer_vecs));
    } else if (a.conv_vecs) {
      const uint32_t begin = (piece - state_pieces) * a.piece_vecs;
      copy_range(reinterpret_cast<const uint4 *>(static_cast<const char *>(a.conv) + s * a.conv_stride),
                 reinterpret_cast<uint4 *>(static_cast<char *>(a.conv) + d * a.conv_stride), begin, min(begin + a.piece_vecs, a.conv_vecs));
    }
  }
}

}  // namespace

int dasc_launch_beam_select(const DascBeamSelectArgs &a, void *stream) {
  return a.bf16 ? select_type<__nv_bfloat16>(a, stream) : select_type<float>(a, stream);
}

int dasc_launch_beam_reorder(DascBeamReorderArgs a, void *stream) {
  // Pieces of a request's states: small ones where there is little to copy, so that all SMs have some
  const int64_t layer_vecs = a.state ? a.layer_vecs : 0, all = a.n_layers_in_call * layer_vecs + a.conv_vecs;
  const int64_t rounds = std::max(int64_t{1}, std::min(int64_t{8}, a.n_req * all / (int64_t{kCopyTile} * 148 * 32)));
  a.piece_vecs = static_cast<uint32_t>(rounds * kCopyTile);
  a.layer_pieces = static_cast<uint32_t>((layer_vecs + a.piece_vecs - 1) / a.piece_vecs);
  const int64_t conv_pieces = (a.conv_vecs + a.piece_vecs - 1) / a.piece_vecs;
  const int64_t pieces = std::max(int64_t{1}, static_cast<int64_t>(a.n_layers_in_call) * a.layer_pieces + conv_pieces);
  if (pieces * a.n_req > 2147483647LL) return static_cast<int>(cudaErrorInvalidConfiguration);
  a.pieces = static_cast<uint32_t>(pieces);
  return static_cast<int>(launch_blocks(beam_reorder_kernel, dim3(static_cast<unsigned>(pieces * a.n_req)), dim3(kCopyThreads), 0, stream, a));
}
