// The gated delta rule in serving, in fp32 on the CUDA cores: one token per request (decoding), and a few drafted tokens.
//     S <- Diag(a_t) S,   u_t = beta_t (v_t - S^T k_t),   S <- S + k_t u_t^T,   o_t = q_scale S^T q_t
// a_t is a vector over the key channels (KDA) or one number (GDN).
//
// One token: with r = S^T (a k) and y = S^T (a q) in one pass over the state, u = beta (v - r), o = q_scale (y + (k . q) u),
// and the new state is a S + k u^T on its way to memory.  The old state stays in registers, so beams that continue the same state read it once.
//
// Several tokens go through the state together.  P_t is the product of a group's decays up to token t, D_ts of those behind s up to t:
//     u_t = beta_t (v_t - S^T (P_t k_t) - sum_{s < t} (k_t . D_ts k_s) u_s)
//     o_t = q_scale (S^T (P_t q_t) + sum_{s <= t} (q_t . D_ts k_s) u_s),      S <- P_n S + sum_s (D_ns k_s) u_s^T
// so that the sums over the state's rows of all tokens are independent of one another, and only sums over at most TB values per column are a chain.
// Decays multiply, they are not differences of sums: exp(-inf) is a zero like any other.
//
// Split: columns of the state do not interact, so a thread block owns NCOL columns of one (request, layer, head) state, all of it in
// registers: a thread holds ROWS rows of four columns; sums over rows meet in shared memory in a fixed order.
#include <cuda_runtime.h>

#include "decay_common.cuh"

namespace {

constexpr int TB = 8;  // tokens per group

template <typename T>
__device__ __forceinline__ float to_float(T x) {
  if constexpr (sizeof(T) == 2)
    return __bfloat162float(x);
  else
    return x;
}
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  if constexpr (sizeof(T) == 2)
    return __float2bfloat16_rn(x);
  else
    return x;
}
__device__ __forceinline__ void cp_async16(void *smem, const void *gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(smem))), "l"(gmem) : "memory");
}
__device__ __forceinline__ void cp_async4(void *smem, const void *gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(smem))), "l"(gmem) : "memory");
}

// e^g as a rounded factor and what that is short of: a decay rounded to fp32 is off by up to half an ulp, the same every time where it is
// constant, 6e-4 of a state that lasts 10^4 tokens.
__device__ __forceinline__ void decay_factor(float g, float &hi, float &lo) {
  const float d = expm1f(g), a1 = 1.f + d;
  const bool slow = g > -0.7f;
  hi = slow ? a1 : expf(g);
  lo = slow ? d - (a1 - 1.f) : 0.f;
}

// 128 x 128 values are held by 256 threads, all else by 128: at most 64 registers of state per thread
template <int DK, int NCOL>
constexpr int kThreads = DK * NCOL > 128 * 64 ? 256 : 128;

struct Unit {
  int part, h, hk, lc, r;
};
__device__ __forceinline__ Unit unit_of(const DascDeltaArgs &a, int ncol) {
  const int parts = a.d_v / ncol, unit = blockIdx.x / parts;
  Unit u;
  u.part = blockIdx.x % parts;
  u.h = unit % a.H_v;
  u.lc = unit / a.H_v % a.n_layers_in_call;
  u.r = unit / (a.H_v * a.n_layers_in_call);
  u.hk = u.h / (a.H_v / a.H_k);
  return u;
}

template <int DK, int NCOL>
struct StepSmem {
  static constexpr int RG = kThreads<DK, NCOL> / (NCOL / 4);
  // each value twice: operands of the packed instructions
  alignas(16) uint64_t ak[DK], aq[DK], k[DK], hi[DK], lo[DK];
  alignas(16) float part[2][RG][NCOL];
  alignas(16) float v[NCOL], u[NCOL];
  float kq[4];
};

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
__global__ void __launch_bounds__((kThreads<DK, NCOL>)) delta_step_kernel(const __grid_constant__ DascDeltaArgs a) {
  constexpr int NT = kThreads<DK, NCOL>, LPR = NCOL / 4, RG = NT / LPR, ROWS = DK / RG;
  __shared__ StepSmem<DK, NCOL> sm;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, cg = tid % LPR, rg = tid / LPR;
  const Unit un = unit_of(a, NCOL);
  stream_order_begin();

  int r = un.r;
  int from = a.req_idx[r];
  uint32_t children = 1;  // which of the beams from `r` on this block advances
  if (a.src_idx) {
    // of the beams that continue one state the first one's block takes them all
    const int first = r - r % a.beam_width;
    const bool in = lane < a.beam_width;
    const int src = in ? a.src_idx[first + lane] : -1, dst = in ? a.req_idx[first + lane] : -1;
    from = __shfl_sync(0xffffffffu, src, r - first);
    children = __ballot_sync(0xffffffffu, src == from && dst >= 0);
    if (from < 0 || !(children & 1u << (r - first)) || children & ((1u << (r - first)) - 1u)) return;
    r = first;
  }
  if (from < 0) return;
  const int layer = a.layer_begin + un.lc;
  const int64_t in_state = layer * a.layer_stride + static_cast<int64_t>(un.h) * DK * a.d_v + un.part * NCOL + static_cast<int64_t>(rg) * ROWS * a.d_v + cg * 4;
  const float *const st = a.state + from * a.req_stride + in_state;

  uint64_t S[ROWS][2];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float4 x = *reinterpret_cast<const float4 *>(st + static_cast<int64_t>(i) * a.d_v);
    S[i][0] = dpack2(x.x, x.y);
    S[i][1] = dpack2(x.z, x.w);
  }
  for (; children; children &= children - 1) {
    const int beam = r + __ffs(children) - 1;
    const int64_t tok = static_cast<int64_t>(un.lc) * a.n_req + beam;
    const IO *const gq = static_cast<const IO *>(a.q) + (tok * a.H_k + un.hk) * DK;
    const IO *const gk = static_cast<const IO *>(a.k) + (tok * a.H_k + un.hk) * DK;
    const IO *const gv = static_cast<const IO *>(a.v) + (tok * a.H_v + un.h) * a.d_v + un.part * NCOL;
    const float *const gg = a.g + (tok * a.H_v + un.h) * (KDA ? DK : 1);
    const float beta = a.beta[tok * a.H_v + un.h];
    const int64_t slot = a.req_idx[beam];
    float kq = 0.f;
    if (tid < DK) {
      const float k = to_float<IO>(gk[tid]), q = to_float<IO>(gq[tid]) * a.q_scale;
      float hi, lo;
      decay_factor(gg[KDA ? tid : 0], hi, lo);
      const float ak = hi * k, aq = hi * q;
      sm.ak[tid] = dpack2(ak, ak);
      sm.aq[tid] = dpack2(aq, aq);
      sm.k[tid] = dpack2(k, k);
      sm.hi[tid] = dpack2(hi, hi);
      sm.lo[tid] = dpack2(lo, lo);
      kq = k * q;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) kq += __shfl_xor_sync(0xffffffffu, kq, d);
      if (lane == 0) sm.kq[warp] = kq;
    }
    for (int i = tid; i < NCOL; i += NT) sm.v[i] = to_float<IO>(gv[i]);
    __syncthreads();
    uint64_t x0 = 0, x1 = 0, y0 = 0, y1 = 0;
#pragma unroll
    for (int i = 0; i < ROWS; i += 2) {
      const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.ak[rg * ROWS + i]);
      const ulonglong2 qq = *reinterpret_cast<const ulonglong2 *>(&sm.aq[rg * ROWS + i]);
      x0 = dfma2(S[i][0], kk.x, x0);
      x1 = dfma2(S[i][1], kk.x, x1);
      y0 = dfma2(S[i][0], qq.x, y0);
      y1 = dfma2(S[i][1], qq.x, y1);
      x0 = dfma2(S[i + 1][0], kk.y, x0);
      x1 = dfma2(S[i + 1][1], kk.y, x1);
      y0 = dfma2(S[i + 1][0], qq.y, y0);
      y1 = dfma2(S[i + 1][1], qq.y, y1);
    }
    *reinterpret_cast<ulonglong2 *>(&sm.part[0][rg][cg * 4]) = make_ulonglong2(x0, x1);
    *reinterpret_cast<ulonglong2 *>(&sm.part[1][rg][cg * 4]) = make_ulonglong2(y0, y1);
    __syncthreads();
    if (tid < NCOL) {
      float x = 0.f, y = 0.f, dot = 0.f;
#pragma unroll
      for (int j = 0; j < RG; ++j) {
        x += sm.part[0][j][tid];
        y += sm.part[1][j][tid];
      }
#pragma unroll
      for (int j = 0; j < DK / 32; ++j) dot += sm.kq[j];
      const float u = beta * (sm.v[tid] - x);
      sm.u[tid] = u;
      static_cast<OT *>(a.o)[(tok * a.H_v + un.h) * a.d_v + un.part * NCOL + tid] = from_float<OT>(fmaf(dot, u, y));
    }
    __syncthreads();
    const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(&sm.u[cg * 4]);
    float *const to = a.state + slot * a.req_stride + in_state;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const uint64_t hi = sm.hi[rg * ROWS + i], lo = sm.lo[rg * ROWS + i], k = sm.k[rg * ROWS + i];
      const float2 x = dunpack2(dfma2(S[i][0], hi, dfma2(S[i][0], lo, dmul2(k, u.x))));
      const float2 y = dunpack2(dfma2(S[i][1], hi, dfma2(S[i][1], lo, dmul2(k, u.y))));
      *reinterpret_cast<float4 *>(to + static_cast<int64_t>(i) * a.d_v) = make_float4(x.x, x.y, y.x, y.y);
    }
    if (children & (children - 1)) __syncthreads();
  }
}

template <int DK, int NCOL, bool KDA, typename IO>
struct DraftSmem {
  static constexpr int RG = kThreads<DK, NCOL> / (NCOL / 4), GN = KDA ? DK : 4;
  // each value twice: operands of the packed instructions
  alignas(16) uint64_t pk[TB][DK], pq[TB][DK], dk[TB][DK], hi[DK], lo[DK];
  alignas(16) float part[2][TB][RG][NCOL];
  alignas(16) float u[TB][NCOL];
  alignas(16) float alpha[TB][KDA ? DK : 1];
  float kk[TB][TB], qk[TB][TB];  // k_t . D_ts k_s, q_scale q_t . D_ts k_s
  // the group as it comes from memory
  alignas(16) IO raw_q[TB][DK], raw_k[TB][DK], raw_v[TB][NCOL];
  alignas(16) float raw_g[TB][GN], raw_beta[TB];
};

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
__global__ void __launch_bounds__((kThreads<DK, NCOL>), (kThreads<DK, NCOL> == 256 ? 2 : 3)) delta_draft_kernel(const __grid_constant__ DascDeltaArgs a) {
  constexpr int NT = kThreads<DK, NCOL>, LPR = NCOL / 4, RG = NT / LPR, ROWS = DK / RG;
  using Sm = DraftSmem<DK, NCOL, KDA, IO>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, cg = tid % LPR, rg = tid / LPR;
  const Unit un = unit_of(a, NCOL);
  stream_order_wait();

  const int r = un.r, req = a.req_idx[r];
  if (req < 0) return;
  const int32_t begin = a.cu_seqlens[r];
  int n = max(a.cu_seqlens[r + 1] - begin, 0);
  if (a.seq_used) n = min(n, max(a.seq_used[r], 0));
  const bool zero = a.from_zero && a.from_zero[r] != 0, write = !a.score;
  if (n == 0 && !(write && zero)) return;

  const int64_t tok0 = static_cast<int64_t>(un.lc) * a.total_tokens + begin;
  float *const st = a.state + req * a.req_stride + (a.layer_begin + un.lc) * a.layer_stride + static_cast<int64_t>(un.h) * DK * a.d_v + un.part * NCOL +
                    static_cast<int64_t>(rg) * ROWS * a.d_v + cg * 4;
  const IO *const gq = static_cast<const IO *>(a.q) + (tok0 * a.H_k + un.hk) * DK;
  const IO *const gk = static_cast<const IO *>(a.k) + (tok0 * a.H_k + un.hk) * DK;
  const IO *const gv = static_cast<const IO *>(a.v) + (tok0 * a.H_v + un.h) * a.d_v + un.part * NCOL;
  const float *const gg = a.g + (tok0 * a.H_v + un.h) * (KDA ? DK : 1);
  const float *const gb = a.beta + tok0 * a.H_v + un.h;
  OT *const go = static_cast<OT *>(a.o) + (tok0 * a.H_v + un.h) * a.d_v + un.part * NCOL;
  const int64_t qk_stride = static_cast<int64_t>(a.H_k) * DK, v_stride = static_cast<int64_t>(a.H_v) * a.d_v;

  uint64_t S[ROWS][2];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!zero) x = *reinterpret_cast<const float4 *>(st + static_cast<int64_t>(i) * a.d_v);
    S[i][0] = dpack2(x.x, x.y);
    S[i][1] = dpack2(x.z, x.w);
  }
  auto stage = [&](int t0) {
    const int cnt = min(TB, n - t0);
    constexpr int QV = DK * sizeof(IO) / 16, VV = NCOL * sizeof(IO) / 16, GV = DK / 4;
    for (int i = tid; i < cnt * QV; i += NT) {
      const int t = i / QV, j = i % QV * (16 / sizeof(IO));
      cp_async16(&sm.raw_k[t][j], gk + (t0 + t) * qk_stride + j);
      if (a.o) cp_async16(&sm.raw_q[t][j], gq + (t0 + t) * qk_stride + j);
    }
    for (int i = tid; i < cnt * VV; i += NT) {
      const int t = i / VV, j = i % VV * (16 / sizeof(IO));
      cp_async16(&sm.raw_v[t][j], gv + (t0 + t) * v_stride + j);
    }
    if constexpr (KDA) {
      for (int i = tid; i < cnt * GV; i += NT) cp_async16(&sm.raw_g[i / GV][i % GV * 4], gg + static_cast<int64_t>(t0 + i / GV) * a.H_v * DK + i % GV * 4);
    } else {
      if (tid < cnt) cp_async4(&sm.raw_g[tid][0], gg + static_cast<int64_t>(t0 + tid) * a.H_v);
    }
    if (tid < cnt) cp_async4(&sm.raw_beta[tid], gb + static_cast<int64_t>(t0 + tid) * a.H_v);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  for (int t0 = 0; t0 < n; t0 += TB) {
    const int cnt = min(TB, n - t0);
    const bool update = write || t0 + TB < n;
    stage(t0);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int i = tid; i < cnt * (KDA ? DK : 1); i += NT) {
      if constexpr (KDA)
        sm.alpha[i / DK][i % DK] = expf(sm.raw_g[i / DK][i % DK]);
      else
        sm.alpha[i][0] = expf(sm.raw_g[i][0]);
    }
    __syncthreads();
    // keys and queries behind the group's start, and keys decayed to its end
    if (tid < DK) {
      float p = 1.f, sum = 0.f;
      for (int t = 0; t < cnt; ++t) {
        p *= sm.alpha[t][KDA ? tid : 0];
        sum += sm.raw_g[t][KDA ? tid : 0];
        const float k = p * to_float<IO>(sm.raw_k[t][tid]);
        sm.pk[t][tid] = dpack2(k, k);
        if (a.o) {
          const float q = p * to_float<IO>(sm.raw_q[t][tid]) * a.q_scale;
          sm.pq[t][tid] = dpack2(q, q);
        }
      }
      if (update) {
        float d = 1.f, hi, lo;
        for (int t = cnt - 1; t >= 0; --t) {
          const float k = d * to_float<IO>(sm.raw_k[t][tid]);
          sm.dk[t][tid] = dpack2(k, k);
          d *= sm.alpha[t][KDA ? tid : 0];
        }
        decay_factor(sum, hi, lo);
        sm.hi[tid] = dpack2(hi, hi);
        sm.lo[tid] = dpack2(lo, lo);
      }
    }
    // products between tokens: a warp has one or more tokens t
    constexpr int PER = DK / 32;
    for (int t = warp; t < cnt; t += NT / 32) {
      float k[PER], q[PER], d[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        k[j] = to_float<IO>(sm.raw_k[t][lane * PER + j]);
        q[j] = a.o ? to_float<IO>(sm.raw_q[t][lane * PER + j]) : 0.f;
        d[j] = 1.f;
      }
      for (int s = t; s >= 0; --s) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const float e = d[j] * to_float<IO>(sm.raw_k[s][lane * PER + j]);
          x = fmaf(k[j], e, x);
          y = fmaf(q[j], e, y);
          d[j] *= sm.alpha[s][KDA ? lane * PER + j : 0];
        }
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) {
          x += __shfl_xor_sync(0xffffffffu, x, w);
          y += __shfl_xor_sync(0xffffffffu, y, w);
        }
        if (lane == 0) {
          sm.kk[t][s] = x;
          sm.qk[t][s] = y * a.q_scale;
        }
      }
    }
    __syncthreads();
    for (int t = 0; t < cnt; ++t) {
      uint64_t x0 = 0, x1 = 0, y0 = 0, y1 = 0;
#pragma unroll
      for (int i = 0; i < ROWS; i += 2) {
        const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.pk[t][rg * ROWS + i]);
        x0 = dfma2(S[i][0], kk.x, x0);
        x1 = dfma2(S[i][1], kk.x, x1);
        x0 = dfma2(S[i + 1][0], kk.y, x0);
        x1 = dfma2(S[i + 1][1], kk.y, x1);
      }
      *reinterpret_cast<ulonglong2 *>(&sm.part[0][t][rg][cg * 4]) = make_ulonglong2(x0, x1);
      if (a.o) {
#pragma unroll
        for (int i = 0; i < ROWS; i += 2) {
          const ulonglong2 qq = *reinterpret_cast<const ulonglong2 *>(&sm.pq[t][rg * ROWS + i]);
          y0 = dfma2(S[i][0], qq.x, y0);
          y1 = dfma2(S[i][1], qq.x, y1);
          y0 = dfma2(S[i + 1][0], qq.y, y0);
          y1 = dfma2(S[i + 1][1], qq.y, y1);
        }
        *reinterpret_cast<ulonglong2 *>(&sm.part[1][t][rg][cg * 4]) = make_ulonglong2(y0, y1);
      }
    }
    __syncthreads();
    if (tid < NCOL) {
      float u[TB];
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        if (t < cnt) {
          float x = 0.f, y = 0.f;
#pragma unroll
          for (int j = 0; j < RG; ++j) {
            x += sm.part[0][t][j][tid];
            if (a.o) y += sm.part[1][t][j][tid];
          }
#pragma unroll
          for (int s = 0; s < t; ++s) x = fmaf(sm.kk[t][s], u[s], x);
          u[t] = sm.raw_beta[t] * (to_float<IO>(sm.raw_v[t][tid]) - x);
          sm.u[t][tid] = u[t];
          if (a.o) {
#pragma unroll
            for (int s = 0; s <= t; ++s) y = fmaf(sm.qk[t][s], u[s], y);
            go[(t0 + t) * v_stride + tid] = from_float<OT>(y);
          }
        }
      }
    }
    __syncthreads();
    if (update) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const uint64_t hi = sm.hi[rg * ROWS + i], lo = sm.lo[rg * ROWS + i];
        S[i][0] = dfma2(S[i][0], hi, dmul2(S[i][0], lo));
        S[i][1] = dfma2(S[i][1], hi, dmul2(S[i][1], lo));
      }
      for (int t = 0; t < cnt; ++t) {
        const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(&sm.u[t][cg * 4]);
#pragma unroll
        for (int i = 0; i < ROWS; i += 2) {
          const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.dk[t][rg * ROWS + i]);
          S[i][0] = dfma2(kk.x, u.x, S[i][0]);
          S[i][1] = dfma2(kk.x, u.y, S[i][1]);
          S[i + 1][0] = dfma2(kk.y, u.x, S[i + 1][0]);
          S[i + 1][1] = dfma2(kk.y, u.y, S[i + 1][1]);
        }
      }
    }
    __syncthreads();
  }
  stream_order_release();
  if (write) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float2 x = dunpack2(S[i][0]), y = dunpack2(S[i][1]);
      *reinterpret_cast<float4 *>(st + static_cast<int64_t>(i) * a.d_v) = make_float4(x.x, x.y, y.x, y.y);
    }
  }
}

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
int launch(const DascDeltaArgs &a, void *stream) {
  const int64_t blocks = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v * (a.d_v / NCOL);
  if (blocks > 2147483647LL) return static_cast<int>(cudaErrorInvalidConfiguration);
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads<DK, NCOL>);
  if (!a.cu_seqlens) return static_cast<int>(launch_blocks(delta_step_kernel<DK, NCOL, KDA, IO, OT>, grid, block, 0, stream, a));
  constexpr size_t smem = sizeof(DraftSmem<DK, NCOL, KDA, IO>);
  auto kernel = delta_draft_kernel<DK, NCOL, KDA, IO, OT>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return static_cast<int>(e);
  }
  return static_cast<int>(launch_blocks(kernel, grid, block, smem, stream, a));
}

template <int DK, bool KDA, typename IO, typename OT>
int launch_cols(const DascDeltaArgs &a, void *stream) {
  const int64_t units = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v;
  if (a.d_v % 64 == 0 && units * (a.d_v / 64) >= 2 * 148) return launch<DK, 64, KDA, IO, OT>(a, stream);
  return launch<DK, 32, KDA, IO, OT>(a, stream);
}

template <int DK, bool KDA>
int launch_types(const DascDeltaArgs &a, void *stream) {
  if (a.io_bf16)
    return a.o_bf16 ? launch_cols<DK, KDA, __nv_bfloat16, __nv_bfloat16>(a, stream) : launch_cols<DK, KDA, __nv_bfloat16, float>(a, stream);
  return a.o_bf16 ? launch_cols<DK, KDA, float, __nv_bfloat16>(a, stream) : launch_cols<DK, KDA, float, float>(a, stream);
}
template <int DK>
int launch_kind(const DascDeltaArgs &a, void *stream) {
  return a.kda ? launch_types<DK, true>(a, stream) : launch_types<DK, false>(a, stream);
}

}  // namespace

int dasc_launch_delta(const DascDeltaArgs &a, void *stream) {
  if (a.d_v % 32 != 0) return -1;
  switch (a.d_k) {
    case 128: return launch_kind<128>(a, stream);
    case 64: return launch_kind<64>(a, stream);
    case 32: return launch_kind<32>(a, stream);
  }
  return -1;
}
