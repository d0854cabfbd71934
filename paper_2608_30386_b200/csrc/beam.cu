// Beam search over recurrent states: the best continuations over beams and vocabulary, and the states behind them.
//
// Selection.  A continuation of beam b by token v weighs s = score_b + (x_bv - log sum exp x_b), in 64 bits; the best n_out of a
// request's width x vocab continuations are wanted.  Inside a beam they are ordered like the logits themselves, so each part of a row gives its best n_out
// by 64-bit keys (logit, then lower token) while it sums exponentials, all from one pass over the row, and the few that are left meet with their beams' sums.
// Split: a request is a cluster of CL thread blocks; the rows of its beams are cut into segments, alike for all rows, which the blocks take in
// order, a slice of at most NT * EPT entries in registers at a time.  Sums are kept by segment and added up in their order, so that equal rows have
// equal sums whichever blocks they fell to.  A lower bound on the slice's n_out-th best entry comes from the maxima of groups of threads (there are at least
// n_out groups); the entries above it, a few dozen as a rule, go to shared memory and are ranked there by counting.  Where more of them tie or the
// bound is poor, the n_out-th key is found by bisection.  Nothing depends on the order of arrival.
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
constexpr int EPT = 32;              // entries of a slice per thread
constexpr int SLICE = NT * EPT;
constexpr int CAP = 512;             // entries above the bound that are ranked at once
constexpr int MAXW = kBeamMaxWidth, MAXN = kBeamMaxOut;  // beams per request, continuations wanted
constexpr int MAXS = 16, MAXCL = 8;  // segments of a row, thread blocks of a request
constexpr float kNone = -__builtin_huge_valf();

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
// larger logit first, then lower token
__device__ __forceinline__ uint64_t key_of(float x, int token) { return static_cast<uint64_t>(order32(x)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(token)); }
__device__ __forceinline__ int token_of(uint64_t key) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(key)); }

__device__ __forceinline__ float clean(float x) { return fabsf(x) < __int_as_float(0x7f800000) ? x : kNone; }

struct Pick {
  uint64_t total;  // order64 of s; 0: none
  uint64_t key;
  int beam, pad;
};

struct SelectSmem {
  uint64_t cand[CAP + MAXN];
  uint64_t list[MAXW][MAXN];  // this block's best of each beam, best first
  int count[MAXW];
  float top[MAXW * MAXS];     // of each segment (those of this block): the largest logit, and the sum of exponentials relative to it
  double sum[MAXW * MAXS];
  float group_max[NW * 4], warp_sum[NW];
  int n_cand, n_above;
  float score[MAXW];
  int ended[MAXW];
  double lse[MAXW];
  Pick pick[MAXN];            // this block's best over its beams
  int n_pick;
  Pick all[MAXCL * MAXN];     // first block: every block's
  int n_all[MAXCL];
};

// The best entry over the lanes: largest total; among equal ones the lower beam, the larger key.  Lanes without one have total 0.
__device__ __forceinline__ int best_lane(uint64_t total, int beam, uint64_t key) {
  const uint32_t hi = static_cast<uint32_t>(total >> 32), lo = static_cast<uint32_t>(total);
  uint32_t m = __ballot_sync(0xffffffffu, hi == __reduce_max_sync(0xffffffffu, hi));
  auto narrow = [&](uint32_t x) {  // of the lanes in m, those with the largest x
    const uint32_t in = m >> (threadIdx.x & 31) & 1u;
    const uint32_t best = __reduce_max_sync(0xffffffffu, in ? x : 0u);
    m = __ballot_sync(0xffffffffu, in && x == best);
  };
  if (m & (m - 1)) narrow(lo);
  if (m & (m - 1)) narrow(MAXW - static_cast<uint32_t>(beam));
  if (m & (m - 1)) narrow(static_cast<uint32_t>(key >> 32));
  if (m & (m - 1)) narrow(static_cast<uint32_t>(key));
  return __ffs(m) - 1;
}

// entries of a row, four or eight per load where rows are aligned
template <typename T, bool VEC>
struct Slice {
  static constexpr int VW = VEC ? 16 / static_cast<int>(sizeof(T)) : 1, LOADS = EPT / VW;
  static __device__ __forceinline__ int index(int e) { return (e / VW * NT + static_cast<int>(threadIdx.x)) * VW + e % VW; }
  // entries `from` .. `from + len - 1` of the row; kNone behind them and where there is no finite number
  static __device__ __forceinline__ void load(const T *row, int from, int len, float (&x)[EPT]) {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      const int i = (l * NT + static_cast<int>(threadIdx.x)) * VW;
      if constexpr (!VEC) {
        float y = kNone;
        if (i < len) {
          if constexpr (sizeof(T) == 2)
            y = __bfloat162float(row[from + i]);
          else
            y = row[from + i];
        }
        x[l] = y;
      } else if (i + VW <= len) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + from + i);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (sizeof(T) == 2) {
            x[l * VW + 2 * j] = __uint_as_float(w[j] << 16);
            x[l * VW + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
          } else {
            x[l * VW + j] = __uint_as_float(w[j]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < VW; ++j) {
          float y = kNone;
          if (i + j < len) {
            if constexpr (sizeof(T) == 2)
              y = __bfloat162float(row[from + i + j]);
            else
              y = row[from + i + j];
          }
          x[l * VW + j] = y;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) x[e] = clean(x[e]);
  }
};

template <typename T, bool VEC, int CL>
__global__ void __launch_bounds__(NT) beam_select_kernel(const __grid_constant__ DascBeamSelectArgs a) {
  using Sl = Slice<T, VEC>;
  __shared__ SelectSmem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x % CL;
  const int W = a.width, N = a.n_out;
  stream_order_begin();

  if (tid < W) {
    sm.score[tid] = a.scores[static_cast<int64_t>(r) * W + tid];
    sm.ended[tid] = a.ended ? a.ended[static_cast<int64_t>(r) * W + tid] != 0 : 0;
    sm.count[tid] = 0;
  }
  __syncthreads();

  const int groups = N <= NW ? 1 : N <= 2 * NW ? 2 : 4;  // per warp
  const int first = rank * a.per_block, last = min(first + a.per_block, W * a.segments);
  for (int step = 0; step < (last - first) * a.seg_slices; ++step) {
    const int item = first + step / a.seg_slices, b = item / a.segments;
    const bool opens = step % a.seg_slices == 0;
    const float seg_top = opens ? kNone : sm.top[item];
    const int from = (item % a.segments * a.seg_slices + step % a.seg_slices) * a.slice_len, len = min(a.slice_len, a.vocab - from);
    if (len <= 0 || sm.ended[b] || !(fabsf(sm.score[b]) < __int_as_float(0x7f800000))) continue;  // (the same for the whole block)
    float x[EPT];
    Sl::load(static_cast<const T *>(a.logits) + (static_cast<int64_t>(r) * W + b) * a.stride, from, len, x);
    float m = x[0];
#pragma unroll
    for (int e = 1; e < EPT; ++e) m = fmaxf(m, x[e]);
    float g = m;
    for (int d = 1; d < 32 / groups; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
    if (lane % (32 / groups) == 0) sm.group_max[warp * groups + lane / (32 / groups)] = g;
    if (tid == 0) sm.n_cand = 0;
    __syncthreads();
    float top = kNone, bound = -kNone;
    for (int i = lane; i < NW * groups; i += 32) {
      top = fmaxf(top, sm.group_max[i]);
      bound = fminf(bound, sm.group_max[i]);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, d));
    }
    const int have = sm.count[b];
    if (have == N) bound = fmaxf(bound, value32(static_cast<uint32_t>(sm.list[b][N - 1] >> 32) + 1));  // (slices come in order: equal ones lose)
    if (top > kNone) {
      // sum of exponentials relative to the segment's largest logit so far
      const float ref = fmaxf(top, seg_top);
      float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
      for (int e = 0; e < EPT; e += 4) {
        s0 += exp2f((x[e] - ref) * 1.44269504f);
        s1 += exp2f((x[e + 1] - ref) * 1.44269504f);
        s2 += exp2f((x[e + 2] - ref) * 1.44269504f);
        s3 += exp2f((x[e + 3] - ref) * 1.44269504f);
      }
      float s = (s0 + s1) + (s2 + s3);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      if (lane == 0) sm.warp_sum[warp] = s;
      if (m >= bound) {
#pragma unroll
        for (int e = 0; e < EPT; ++e)
          if (x[e] >= bound && x[e] > kNone) {
            const int at = atomicAdd(&sm.n_cand, 1);
            if (at < CAP) sm.cand[at] = key_of(x[e], from + Sl::index(e));
          }
      }
    }
    __syncthreads();
    if (!(top > kNone)) {  // (the same for the whole block: no logit of this slice counts)
      if (opens && tid == 0) sm.top[item] = kNone;
      __syncthreads();
      continue;
    }
    int n = sm.n_cand;
    if (n > CAP) {
      // The N-th largest key, bit by bit from the top.
      uint64_t t = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = t | 1ull << bit;
        int c = 0;
#pragma unroll
        for (int e = 0; e < EPT; ++e) c += x[e] > kNone && key_of(x[e], from + Sl::index(e)) >= trial;
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (tid == 0) sm.n_above = 0;
        __syncthreads();
        if (lane == 0 && c) atomicAdd(&sm.n_above, c);
        __syncthreads();
        if (sm.n_above >= N) t = trial;
      }
      if (tid == 0) sm.n_cand = 0;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < EPT; ++e)
        if (x[e] > kNone && key_of(x[e], from + Sl::index(e)) >= t) {
          const int at = atomicAdd(&sm.n_cand, 1);
          if (at < CAP) sm.cand[at] = key_of(x[e], from + Sl::index(e));
        }
      __syncthreads();
      n = min(sm.n_cand, CAP);
    }
    if (tid < have) sm.cand[n + tid] = sm.list[b][tid];
    if (tid == 0) {
      const float ref = fmaxf(top, seg_top);
      double s = 0.0;
      for (int i = 0; i < NW; ++i) s += sm.warp_sum[i];
      sm.sum[item] = seg_top > kNone ? sm.sum[item] * exp(static_cast<double>(seg_top) - ref) + s : s;
    }
    __syncthreads();
    const int total = n + have;
    for (int i = tid; i < total; i += NT) {
      const uint64_t k = sm.cand[i];
      int place = 0;
      for (int j = 0; j < total; ++j) place += sm.cand[j] > k;
      if (place < N) sm.list[b][place] = k;
    }
    if (tid == 0) {
      sm.count[b] = min(total, N);
      sm.top[item] = fmaxf(top, seg_top);
    }
    __syncthreads();
  }

  // every row's sum, from all blocks
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  if (tid < W) {
    float top = kNone;
    double s = 0.0;
    if (!sm.ended[tid] && fabsf(sm.score[tid]) < __int_as_float(0x7f800000)) {
      for (int i = tid * a.segments; i < (tid + 1) * a.segments; ++i) top = fmaxf(top, cluster.map_shared_rank(sm.top, i / a.per_block)[i]);
      if (top > kNone)
        for (int i = tid * a.segments; i < (tid + 1) * a.segments; ++i) {
          const float t = cluster.map_shared_rank(sm.top, i / a.per_block)[i];
          if (t > kNone) s += cluster.map_shared_rank(sm.sum, i / a.per_block)[i] * exp(static_cast<double>(t) - top);
        }
    }
    sm.lse[tid] = static_cast<double>(top) + log(s);
  }
  __syncthreads();
  // this block's best: lane b holds the best of beam b that is left
  if (warp == 0) {
    int at = 0, n = 0;
    uint64_t key = 0, total = 0;
    const bool mine = lane < W;
    const bool over = mine && sm.ended[lane];
    const bool counts = mine && fabsf(sm.score[lane]) < __int_as_float(0x7f800000);
    auto head = [&]() {
      total = key = 0;
      if (!counts) return;
      if (over) {
        if (rank == 0 && at == 0) {
          total = order64(sm.score[lane]);
          key = key_of(0.f, a.end_token);
        }
      } else if (at < sm.count[lane]) {
        key = sm.list[lane][at];
        total = order64(static_cast<double>(sm.score[lane]) + (static_cast<double>(value32(static_cast<uint32_t>(key >> 32))) - sm.lse[lane]));
      }
    };
    head();
    for (; n < N; ++n) {
      const int l = best_lane(total, lane, key);
      if (__shfl_sync(0xffffffffu, total, l) == 0) break;
      if (lane == l) {
        sm.pick[n].total = total;
        sm.pick[n].key = key;
        sm.pick[n].beam = lane;
        ++at;
        head();
      }
    }
    if (lane == 0) sm.n_pick = n;
  }
  cluster.sync();
  if (rank == 0) {
    if (tid < CL) sm.n_all[tid] = *cluster.map_shared_rank(&sm.n_pick, tid);
    __syncthreads();
    for (int i = tid; i < CL * N; i += NT) {
      const int c = i / N, j = i % N;
      if (j < sm.n_all[c]) sm.all[i] = cluster.map_shared_rank(sm.pick, c)[j];
    }
  }
  cluster.sync();  // (no block ends while the first one still reads it)
  if (rank == 0 && warp == 0) {
    int at = 0;
    Pick p{};
    auto head = [&]() {
      p.total = 0;
      p.beam = 0;
      if (lane < CL && at < sm.n_all[lane % MAXCL]) p = sm.all[lane * N + at];
    };
    head();
    const int64_t out = static_cast<int64_t>(r) * N;
    for (int n = 0; n < N; ++n) {
      const int l = best_lane(p.total, p.beam, p.key);
      const bool none = __shfl_sync(0xffffffffu, p.total, l) == 0;
      if (lane == l) {
        const int token = none ? -1 : token_of(p.key);
        a.out_scores[out + n] = none ? kNone : static_cast<float>(value64(p.total));
        a.out_parent[out + n] = none ? -1 : p.beam;
        a.out_token[out + n] = token;
        if (a.out_ended) a.out_ended[out + n] = none || sm.ended[p.beam] || token == a.end_token;
        if (!none) {
          ++at;
          head();
        }
      }
    }
  }
}

template <typename T, bool VEC, int CL>
int select(DascBeamSelectArgs a, void *stream) {
  // segments of a row: as many as fill whole rounds of the cluster's blocks
  const int need = (a.vocab + SLICE - 1) / SLICE;
  a.seg_slices = (need + MAXS - 1) / MAXS;
  const int least = (need + a.seg_slices - 1) / a.seg_slices, rounds = (a.width * least + CL - 1) / CL;
  a.segments = std::min(MAXS, std::max(least, rounds * CL / a.width));
  const int slices = a.segments * a.seg_slices;
  a.slice_len = ((a.vocab + slices - 1) / slices + 7) / 8 * 8;
  a.segments = (a.vocab + a.slice_len * a.seg_slices - 1) / (a.slice_len * a.seg_slices);
  a.per_block = (a.width * a.segments + CL - 1) / CL;
  return static_cast<int>(launch_clusters(beam_select_kernel<T, VEC, CL>, dim3(static_cast<unsigned>(a.n_req) * CL), dim3(NT), CL, 0, stream, a));
}

template <typename T>
int select_type(const DascBeamSelectArgs &a, void *stream) {
  const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.stride * static_cast<int64_t>(sizeof(T)) % 16 == 0;
  const auto with = [&](auto cl) {
    constexpr int CL = decltype(cl)::value;
    return vec ? select<T, true, CL>(a, stream) : select<T, false, CL>(a, stream);
  };
  constexpr int kPlaces = 2 * 148;
  if (a.n_req * int64_t{8} <= kPlaces) return with(std::integral_constant<int, 8>{});
  if (a.n_req * int64_t{4} <= kPlaces) return with(std::integral_constant<int, 4>{});
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
