// Verification of drafted tokens: which of them stand, and the next token by inverse transform sampling, from given random
// numbers.  All comparisons and sums are in 64 bits: a running sum over a vocabulary in 32 bits would move the border between
// two tokens by more than many of them weigh.
//
// Split: a request is one cluster of CL thread blocks, each of which owns a contiguous part of the row, and in it each warp a
// contiguous run of tiles.  One pass sums the weights per tile and per warp; the warps' sums meet through distributed shared memory in
// a fixed order, every block finds the one warp whose part holds the threshold, that warp finds the tile among its sums and reads
// this one tile again.  One launch, no workspace, nothing depends on the order of arrival.
// Bound: one pass over a row of the target, and one of the drafter where a token does not stand; in small calls the chain of loads to
// the first token that does not stand, two cluster barriers and the last tile.  64 requests of 8 drafts over 131,072 entries in fp32: 23 us,
// their bytes take 10.2 at 6567 GB/s; 37 of 5 over 50,257 in bf16, odd rows: 9.2 us; one: 6.7 us (calls one behind the other).  Not faster: the warp's part of the row
// prefetched into L2 ahead of its loads (27 us).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "decay_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512, NW = NT / 32;
constexpr int TILE = 128;  // entries of a row that a warp takes at once: four per lane
constexpr int SUMS = 64;   // sums that a warp keeps: one per tile, or per few tiles of a very long row

template <typename T>
__device__ __forceinline__ float prob(T x) {
  if constexpr (sizeof(T) == 2)
    return __bfloat162float(x);
  else
    return x;
}
// A probability that is none (negative, infinite, NaN) counts as nothing.
__device__ __forceinline__ float clean(float x) {
  x = fmaxf(x, 0.f);
  return x < __int_as_float(0x7f800000) ? x : 0.f;
}

// four entries of a row, from entry i on; 0 behind the end
template <typename T, bool VEC>
__device__ __forceinline__ void load4(const T *row, int i, int vocab, float (&x)[4]) {
  if (VEC && i + 4 <= vocab) {
    if constexpr (sizeof(T) == 4) {
      const float4 v = *reinterpret_cast<const float4 *>(row + i);
      x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2 *>(row + i);
      x[0] = __uint_as_float(v.x << 16), x[1] = __uint_as_float(v.x & 0xFFFF0000u);
      x[2] = __uint_as_float(v.y << 16), x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = i + j < vocab ? prob<T>(row[i + j]) : 0.f;
  }
}

template <typename T, bool VEC, int CL>
__global__ void __launch_bounds__(NT, 2) verify_draft_kernel(const __grid_constant__ DascVerifyArgs a) {
  __shared__ double warp_sum[NW], tile_sum[NW][SUMS], s_before, s_threshold;
  __shared__ int s_count, s_winner;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / CL, rank = blockIdx.x % CL;
  stream_order_begin();

  const int64_t d0 = a.cu_drafts[r];
  const float u_next = a.u_next[r];  // (on its way before it is needed)
  const int n = a.tokens ? min(max(static_cast<int>(a.cu_drafts[r + 1] - d0), 0), a.max_drafts) : 0;
  const T *const target = static_cast<const T *>(a.target) + (d0 + r) * a.target_stride;
  const T *const draft = a.draft ? static_cast<const T *>(a.draft) + d0 * a.draft_stride : nullptr;
  // every block of the cluster looks for itself which tokens stand: two probabilities each
  if (warp == 0) {
    int count = 0;
    for (int j0 = 0; j0 < n; j0 += 32) {
      const int j = j0 + lane;
      bool stands = false;
      if (j < n) {
        const int x = a.tokens[d0 + j];
        if (x >= 0 && x < a.vocab) {
          const double p = prob<T>(target[j * a.target_stride + x]), q = draft ? prob<T>(draft[j * a.draft_stride + x]) : 1.f;
          stands = static_cast<double>(a.u_accept[d0 + j]) * q < p;
        }
      }
      const uint32_t no = ~__ballot_sync(0xffffffffu, stands);
      count = j0 + (no ? __ffs(no) - 1 : 32);
      if (no) break;
    }
    if (lane == 0) s_count = min(count, n);
  }
  __syncthreads();
  const int count = s_count;
  const bool all = count == n;
  const T *const prow = target + count * a.target_stride;
  const T *qrow = !all && draft ? draft + count * a.draft_stride : nullptr;
  int taken = !all && !draft ? a.tokens[d0 + count] : -1;  // a deterministic drafter's token: its probability is 1

  if (rank == 0) {
    int32_t *const out = a.out + r * a.out_stride;
    for (int j = tid; j <= a.max_drafts; j += NT)
      if (j != count) out[j] = j < count ? a.tokens[d0 + j] : -1;
    if (tid == 0) a.n_kept[r] = count + 1;
  }

  const int tiles = (a.vocab + TILE - 1) / TILE, per_warp = (tiles + CL * NW - 1) / (CL * NW);
  const int gw = rank * NW + warp, group = (per_warp + SUMS - 1) / SUMS;  // tiles per sum
  const int first = min(gw * per_warp, tiles), last = min(first + per_warp, tiles);
  // max(p - q, 0), exact in 64 bits
  auto weights = [&](int tile, double (&w)[4]) {
    const int i = tile * TILE + lane * 4;
    float p[4], q[4];
    load4<T, VEC>(prow, i, a.vocab, p);
    if (qrow) load4<T, VEC>(qrow, i, a.vocab, q);
    const bool other = qrow || taken >= 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p[j] = clean(p[j]);
      w[j] = p[j];
      if (other) w[j] -= static_cast<double>(fminf(p[j], qrow ? clean(q[j]) : (i + j == taken ? 1.f : 0.f)));
    }
  };

  cg::cluster_group cluster = cg::this_cluster();
  constexpr int PER = (CL * NW + 31) / 32;
  for (int attempt = 0; attempt < 2; ++attempt) {
    // Four sums at a time: their loads are in flight together, and the lanes' parts fold into one another, so that lanes 8 j .. 8 j + 7
    // end with sum j (six exchanges for four sums, not twenty).
    double sum = 0.0;
    for (int i = 0; first + i * group < last; i += 4) {
      double x[4] = {0.0, 0.0, 0.0, 0.0};
      for (int u = 0; u < group; ++u) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = first + (i + j) * group + u;
          if (t < last) {
            double w[4];
            weights(t, w);
            x[j] += (w[0] + w[1]) + (w[2] + w[3]);
          }
        }
      }
      const bool up = lane & 16, up2 = lane & 8;
      double y0 = up ? x[2] : x[0], y1 = up ? x[3] : x[1];
      y0 += __shfl_xor_sync(0xffffffffu, up ? x[0] : x[2], 16);
      y1 += __shfl_xor_sync(0xffffffffu, up ? x[1] : x[3], 16);
      double z = up2 ? y1 : y0;
      z += __shfl_xor_sync(0xffffffffu, up2 ? y0 : y1, 8);
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
      if (lane % 8 == 0) tile_sum[warp][i + lane / 8] = z;
      sum += z;
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
    if (lane == 0) warp_sum[warp] = sum;
    cluster.sync();
    double x[PER];  // lane l of the first warp: the sums of warps PER l ... of the cluster
#pragma unroll
    for (int j = 0; j < PER; ++j) x[j] = 0.0;
    if (warp == 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int i = lane * PER + j;
        if (i < CL * NW) x[j] = cluster.map_shared_rank(warp_sum, i / NW)[i % NW];
      }
    }
    cluster.sync();  // (no block changes its sums, or ends, while another still reads them)
    if (warp == 0) {
      double incl = 0.0;
#pragma unroll
      for (int j = 0; j < PER; ++j) incl += x[j];
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      const double total = __shfl_sync(0xffffffffu, incl, 31);
      double run = __shfl_up_sync(0xffffffffu, incl, 1);
      if (lane == 0) run = 0.0;
      // the first warp whose part of the row takes the running sum over the threshold (the last one with any weight, should
      // a random number not be below 1)
      const double threshold = fmax(static_cast<double>(u_next) * total, 0.0);
      int here = -1, some = -1;
      double before = 0.0, before_some = 0.0;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const double next = run + x[j];
        if (x[j] > 0.0) {
          some = lane * PER + j;
          before_some = run;
          if (here < 0 && next > threshold) {
            here = some;
            before = run;
          }
        }
        run = next;
      }
      uint32_t m = __ballot_sync(0xffffffffu, here >= 0);
      int l = m ? __ffs(m) - 1 : 0;
      if (!m) {
        m = __ballot_sync(0xffffffffu, some >= 0);
        l = m ? 31 - __clz(m) : 0;
        here = some;
        before = before_some;
      }
      if (lane == l) {
        s_winner = total > 0.0 ? here : -1;
        s_before = before;
        s_threshold = threshold;
      }
    }
    __syncthreads();
    if (s_winner >= 0 || (!qrow && taken < 0)) break;
    qrow = nullptr;  // the drafter leaves nothing: the target's own row
    taken = -1;
    __syncthreads();
  }
  const int winner = s_winner;
  if (winner < 0) {
    if (rank == 0 && tid == 0) a.out[r * a.out_stride + count] = -1;
    return;
  }
  if (gw != winner) return;
  double before = s_before;
  const double threshold = s_threshold;
  // the first of this warp's sums that takes it over, or the last one that is not zero
  int at = -1;
  double at_before = before;
  for (int i = 0; first + i * group < last; ++i) {
    const double x = tile_sum[warp][i];
    if (x > 0.0) {
      at = i;
      at_before = before;
      if (before + x > threshold) break;
    }
    before += x;
  }
  // and the first of its entries (sums in another order may stay a last bit below: then the last entry with any weight)
  before = at_before;
  int token = -1, last_some = -1;
  const int begin = first + at * group;
  for (int t = begin; t < min(begin + group, last) && token < 0; ++t) {
    double w[4];
    weights(t, w);
    double incl = (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    const double excl = __shfl_up_sync(0xffffffffu, incl, 1);
    double x = before + (lane > 0 ? excl : 0.0);
    int here = -1, any = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x += w[j];
      if (w[j] > 0.0) {
        any = j;
        if (here < 0 && x > threshold) here = j;
      }
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, here >= 0), some = __ballot_sync(0xffffffffu, any >= 0);
    if (hit) {
      const int l = __ffs(hit) - 1;
      token = t * TILE + l * 4 + __shfl_sync(0xffffffffu, here, l);
    } else if (some) {
      const int l = 31 - __clz(some);
      last_some = t * TILE + l * 4 + __shfl_sync(0xffffffffu, any, l);
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) a.out[r * a.out_stride + count] = token >= 0 ? token : last_some;
}

template <typename T, bool VEC, int CL>
int launch(const DascVerifyArgs &a, void *stream) {
  return static_cast<int>(launch_clusters(verify_draft_kernel<T, VEC, CL>, dim3(static_cast<unsigned>(a.n_req) * CL), dim3(NT), CL, 0, stream, a));
}

template <typename T>
int launch_type(const DascVerifyArgs &a, void *stream) {
  // four entries per load where every row starts on their boundary
  auto even = [](const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0 && stride % 4 == 0; };
  const bool vec = even(a.target, a.target_stride) && (!a.draft || even(a.draft, a.draft_stride));
  // As many blocks per request as still fit the GPU at once, two per SM (not every GPC holds a whole number of clusters of 4 or 8).
  // Measured over 131072 entries, 4 drafts each, every call from a cold L2 (unlike the figures at the top), in us with 8 / 4 / 2 / 1 blocks: 32 requests 21 / 27 / 41 / 70, 37 requests 31 / 29 / 41 / 70, 64 requests
  // 35 / 31 / 43 / 72, 148 requests 74 / 68 / 53 / 78, 296 requests 129 / 109 / 90 / 87.
  const auto with = [&](auto cl) {
    constexpr int CL = decltype(cl)::value;
    return vec ? launch<T, true, CL>(a, stream) : launch<T, false, CL>(a, stream);
  };
  constexpr int kPlaces = 2 * 148, kClustered = kPlaces * 7 / 8;
  if (a.n_req * int64_t{8} <= kClustered) return with(std::integral_constant<int, 8>{});
  if (a.n_req * int64_t{4} <= kClustered) return with(std::integral_constant<int, 4>{});
  if (a.n_req * int64_t{2} <= kPlaces) return with(std::integral_constant<int, 2>{});
  return with(std::integral_constant<int, 1>{});
}

}  // namespace

int dasc_launch_verify_draft(const DascVerifyArgs &a, void *stream) {
  return a.bf16 ? launch_type<__nv_bfloat16>(a, stream) : launch_type<float>(a, stream);
}
