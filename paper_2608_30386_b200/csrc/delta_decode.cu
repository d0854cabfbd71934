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

#include <algorithm>

#include "decay_common.cuh"

namespace {

constexpr int TB = 8;              // tokens per group

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

// Several tokens: the products with the state are 16 x DK x NCOL (eight keys, eight queries) and DK x 8 x NCOL, on the tensor cores in three products of tf32 parts
// (a value is its rounding to 11 bits and what that is short of, good to 2^-22 together): sums over rows end in one thread's registers, and eight tokens
// cost what one does.  A warp has 16 columns of the state and all of its rows.  Row k of a block of eight rows is operand row k / 2, or k / 2 + 4 where k is odd, and column
// n of the 16 is column n / 2 of the first tile or, where n is odd, of the second, so that what a thread holds of the state as an operand of the first
// product is what it gets from the second: rows 2 m and 2 m + 1 of every block and columns 2 n and 2 n + 1, m = lane % 4, n = lane / 4.
template <int DK, int NCOL>
struct DraftShape {
  static constexpr int WARPS = NCOL / 16, NT = NCOL > 32 ? WARPS * 32 : 128, BLOCKS = DK / 8;  // (a narrow part has two warps that only prepare)
};

template <int DK, int NCOL, bool KDA, typename IO>
struct DraftSmem {
  static constexpr int GN = KDA ? DK : 4, BLOCKS = DK / 8;
  // operands as the lanes take them, the rounded parts and what they are short of; a block's 32 lanes and 64 bytes that spread the writes over the banks
  alignas(16) float4 key_query[2][BLOCKS][36];  // P_t k_t and q_scale P_t q_t of token t = lane / 4: rows 2 m (key, query), 2 m + 1 (key, query)
  alignas(16) float4 last[BLOCKS][36];          // D_ns k_s: row lane / 4, tokens m and m + 4 rounded, and what they are short of
  alignas(16) float hi[DK], lo[DK];             // the group's decay
  alignas(16) float v[TB][NCOL], u[TB][NCOL];
  alignas(16) float alpha[TB][KDA ? DK : 1];
  alignas(16) float kk[TB][TB], qk[TB][TB];     // k_t . D_ts k_s for s < t, q_scale q_t . D_ts k_s for s <= t, 0 for later s
  float beta[TB];
  // the next group as it comes from memory
  alignas(16) IO raw_q[TB][DK], raw_k[TB][DK], raw_v[TB][NCOL];
  alignas(16) float raw_g[TB][GN], raw_beta[TB];
};

__device__ __forceinline__ float to_tf32(float x) {
  uint32_t y;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(y) : "f"(x));
  return __uint_as_float(y);
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const float4 &a, float b0, float b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(__float_as_uint(a.x)), "r"(__float_as_uint(a.y)), "r"(__float_as_uint(a.z)), "r"(__float_as_uint(a.w)), "r"(__float_as_uint(b0)),
        "r"(__float_as_uint(b1)));
}

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
__global__ void __launch_bounds__((DraftShape<DK, NCOL>::NT), (512 / DraftShape<DK, NCOL>::NT)) delta_draft_kernel(const __grid_constant__ DascDeltaArgs a) {
  using Sh = DraftShape<DK, NCOL>;
  using Sm = DraftSmem<DK, NCOL, KDA, IO>;
  constexpr int NT = Sh::NT, BLOCKS = Sh::BLOCKS;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, m = lane % 4, nn = lane / 4;
  // A block takes every gridDim.x-th part of a state; what the next one needs is on its way while one is worked on.
  const int parts = a.d_v / NCOL, jobs = static_cast<int>(static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v * parts);  // (below 2^31: launch)
  struct Job {
    int r, lc, h, part, req, begin, n;
    bool zero;
  };
  auto look_up = [&](int64_t job) {
    Job x{0, 0, 0, 0, -1, 0, 0, false};
    if (job < jobs) {
      const int i = static_cast<int>(job);
      x.part = i % parts;
      x.h = i / parts % a.H_v;
      x.lc = i / (parts * a.H_v) % a.n_layers_in_call;
      x.r = i / (parts * a.H_v) / a.n_layers_in_call;
      x.req = a.req_idx[x.r];
      x.begin = a.cu_seqlens[x.r];
      x.n = max(a.cu_seqlens[x.r + 1] - x.begin, 0);
      if (a.seq_used) x.n = min(x.n, max(a.seq_used[x.r], 0));
      if (x.req < 0) x.n = 0;
      x.zero = a.from_zero && a.from_zero[x.r] != 0;
    }
    return x;
  };
  auto state_of = [&](const Job &x) {
    return a.state + x.req * a.req_stride + (a.layer_begin + x.lc) * a.layer_stride + static_cast<int64_t>(x.h) * DK * a.d_v + x.part * NCOL;
  };
  const bool write = !a.score;
  const int64_t qk_stride = static_cast<int64_t>(a.H_k) * DK, v_stride = static_cast<int64_t>(a.H_v) * a.d_v;
  stream_order_wait();

  auto stage = [&](const Job &x, int t0) {  // a group's rows as they are, 16 bytes per copy
    const int cnt = min(TB, x.n - t0), hk = x.h / (a.H_v / a.H_k);
    const int64_t tok = static_cast<int64_t>(x.lc) * a.total_tokens + x.begin + t0;
    const IO *const gq = static_cast<const IO *>(a.q) + (tok * a.H_k + hk) * DK;
    const IO *const gk = static_cast<const IO *>(a.k) + (tok * a.H_k + hk) * DK;
    const IO *const gv = static_cast<const IO *>(a.v) + (tok * a.H_v + x.h) * a.d_v + x.part * NCOL;
    const float *const gg = a.g + (tok * a.H_v + x.h) * (KDA ? DK : 1);
    const float *const gb = a.beta + tok * a.H_v + x.h;
    constexpr int QV = DK * sizeof(IO) / 16, VV = NCOL * sizeof(IO) / 16, GV = DK / 4;
    for (int i = tid; i < cnt * QV; i += NT) {
      const int t = i / QV, j = i % QV * (16 / sizeof(IO));
      cp_async16(&sm.raw_k[t][j], gk + t * qk_stride + j);
      if (a.o) cp_async16(&sm.raw_q[t][j], gq + t * qk_stride + j);
    }
    for (int i = tid; i < cnt * VV; i += NT) {
      const int t = i / VV, j = i % VV * (16 / sizeof(IO));
      cp_async16(&sm.raw_v[t][j], gv + t * v_stride + j);
    }
    if constexpr (KDA) {
      for (int i = tid; i < cnt * GV; i += NT) cp_async16(&sm.raw_g[i / GV][i % GV * 4], gg + static_cast<int64_t>(i / GV) * a.H_v * DK + i % GV * 4);
    } else {
      if (tid < cnt) cp_async4(&sm.raw_g[tid][0], gg + static_cast<int64_t>(tid) * a.H_v);
    }
    if (tid < cnt) cp_async4(&sm.raw_beta[tid], gb + static_cast<int64_t>(tid) * a.H_v);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  Job now = look_up(blockIdx.x);
  stage(now, 0);
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
  const Job next = look_up(job + gridDim.x);
  const int n = now.n;
  const bool holds = warp < Sh::WARPS;
  float *const st = state_of(now) + static_cast<int64_t>(2 * m) * a.d_v + warp * 16 + 2 * nn;
  OT *const go = static_cast<OT *>(a.o) + ((static_cast<int64_t>(now.lc) * a.total_tokens + now.begin) * a.H_v + now.h) * a.d_v + now.part * NCOL;
  uint64_t S[BLOCKS][2];  // rows 8 b + 2 m and the one behind it; columns 2 nn, 2 nn + 1
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    float2 x = make_float2(0.f, 0.f), y = x;
    if (holds && !now.zero && n > 0) {
      x = *reinterpret_cast<const float2 *>(st + static_cast<int64_t>(8 * b) * a.d_v);
      y = *reinterpret_cast<const float2 *>(st + static_cast<int64_t>(8 * b + 1) * a.d_v);
    }
    S[b][0] = dpack2(x.x, y.x);
    S[b][1] = dpack2(x.y, y.y);
  }

  for (int t0 = 0; t0 < n; t0 += TB) {
    const int cnt = min(TB, n - t0);
    const bool update = write || t0 + TB < n;
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int i = tid; i < cnt * (KDA ? DK : 1); i += NT) {
      if constexpr (KDA)
        sm.alpha[i / DK][i % DK] = expf(sm.raw_g[i / DK][i % DK]);
      else
        sm.alpha[i][0] = expf(sm.raw_g[i][0]);
    }
    for (int i = tid; i < cnt * NCOL; i += NT) sm.v[i / NCOL][i % NCOL] = to_float<IO>(sm.raw_v[i / NCOL][i % NCOL]);
    if (tid < cnt) sm.beta[tid] = sm.raw_beta[tid];
    __syncthreads();
    // keys and queries behind the group's start, and keys decayed to its end: a thread per channel and kind
    for (int i = tid; i < 3 * DK; i += NT) {
      const int c = i % DK, what = i / DK, b = c / 8;
      if (what < 2) {
        const IO(*const raw)[DK] = what ? sm.raw_q : sm.raw_k;
        float p = what ? a.q_scale : 1.f;
        float *const to = reinterpret_cast<float *>(&sm.key_query[0][b][c % 8 / 2]) + c % 2 * 2 + what, *const short_of = to + BLOCKS * 36 * 4;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          float x = 0.f;
          if (t < cnt && (what == 0 || a.o)) {
            p *= sm.alpha[t][KDA ? c : 0];
            x = p * to_float<IO>(raw[t][c]);
          }
          const float hi = to_tf32(x);
          to[t * 16] = hi;
          short_of[t * 16] = x - hi;
        }
      } else if (update) {
        float d = 1.f, sum = 0.f, hi, lo;
        float *const to = reinterpret_cast<float *>(&sm.last[b][c % 8 * 4]);
#pragma unroll
        for (int t = TB - 1; t >= 0; --t) {
          float x = 0.f;
          if (t < cnt) {
            x = d * to_float<IO>(sm.raw_k[t][c]);
            d *= sm.alpha[t][KDA ? c : 0];
            sum += sm.raw_g[t][KDA ? c : 0];
          }
          hi = to_tf32(x);
          to[t % 4 * 4 + t / 4] = hi;
          to[t % 4 * 4 + t / 4 + 2] = x - hi;
        }
        decay_factor(sum, hi, lo);
        sm.hi[c] = hi;
        sm.lo[c] = lo;
      }
    }
    // Products between tokens: a warp has one token t or more; its lanes' parts of the 16 sums fold into one another.
    constexpr int PER = DK / 32;
    for (int t = warp; t < TB; t += NT / 32) {
      float x[2 * TB], k[PER], q[PER], d[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        k[j] = t < cnt ? to_float<IO>(sm.raw_k[t][lane * PER + j]) : 0.f;
        q[j] = t < cnt && a.o ? to_float<IO>(sm.raw_q[t][lane * PER + j]) * a.q_scale : 0.f;
        d[j] = 1.f;
      }
#pragma unroll
      for (int s = TB - 1; s >= 0; --s) {
        x[s] = x[TB + s] = 0.f;
        if (s <= t && t < cnt) {
#pragma unroll
          for (int j = 0; j < PER; ++j) {
            const float e = d[j] * to_float<IO>(sm.raw_k[s][lane * PER + j]);
            x[s] = fmaf(k[j], e, x[s]);
            x[TB + s] = fmaf(q[j], e, x[TB + s]);
            d[j] *= sm.alpha[s][KDA ? lane * PER + j : 0];
          }
        }
      }
#pragma unroll
      for (int w = TB; w > 0; w >>= 1) {
        const bool up = lane & w;
#pragma unroll
        for (int j = 0; j < w; ++j) {
          const float mine = up ? x[j + w] : x[j];
          x[j] = mine + __shfl_xor_sync(0xffffffffu, up ? x[j] : x[j + w], w);
        }
      }
      x[0] += __shfl_xor_sync(0xffffffffu, x[0], 16);
      if (lane < 2 * TB) (lane < TB ? sm.kk : sm.qk)[t][lane % TB] = lane == t ? 0.f : x[0];
    }
    __syncthreads();
    if (t0 + TB < n)
      stage(now, t0 + TB);
    else
      stage(next, 0);
    if (t0 == 0 && tid == NT - 1 && next.n > 0 && !next.zero) {  // and its rows of the state come as far as L2
      if (parts == 1) {
        bulk_prefetch(state_of(next), DK * NCOL * 4);
      } else {
#pragma unroll 1
        for (int i = 0; i < DK; ++i) asm volatile("prefetch.global.L2 [%0];" ::"l"(state_of(next) + static_cast<int64_t>(i) * a.d_v));
      }
    }

    if (!holds) continue;
    // S^T (P_t k_t) and S^T (P_t q_t) of token t = nn, columns 4 m .. 4 m + 3
    float big[2][4] = {}, one[2][4] = {}, two[2][4] = {};
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const float4 hi = sm.key_query[0][b][lane], lo = sm.key_query[1][b][lane];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 x = dunpack2(S[b][j]);
        const float x0 = to_tf32(x.x), x1 = to_tf32(x.y);
        mma_tf32(big[j], hi, x0, x1);
        mma_tf32(one[j], lo, x0, x1);
        mma_tf32(two[j], hi, x.x - x0, x.y - x1);
      }
    }
    float x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = i % 2, at = i / 2;
      x[i] = (one[j][at] + two[j][at]) + big[j][at];
      y[i] = (one[j][at + 2] + two[j][at + 2]) + big[j][at + 2];
    }
    // u_t, one token after the other, and outputs as the u_s come by
    const int c = warp * 16 + 4 * m;
    const bool valid = nn < cnt;
    const float beta = valid ? sm.beta[nn] : 0.f;
    const float4 v = valid ? *reinterpret_cast<const float4 *>(&sm.v[nn][c]) : make_float4(0.f, 0.f, 0.f, 0.f);
    x[0] = beta * (v.x - x[0]), x[1] = beta * (v.y - x[1]), x[2] = beta * (v.z - x[2]), x[3] = beta * (v.w - x[3]);
    float kk[TB], qk[TB];
    *reinterpret_cast<float4 *>(kk) = *reinterpret_cast<const float4 *>(&sm.kk[nn][0]);
    *reinterpret_cast<float4 *>(kk + 4) = *reinterpret_cast<const float4 *>(&sm.kk[nn][4]);
    *reinterpret_cast<float4 *>(qk) = *reinterpret_cast<const float4 *>(&sm.qk[nn][0]);
    *reinterpret_cast<float4 *>(qk + 4) = *reinterpret_cast<const float4 *>(&sm.qk[nn][4]);
#pragma unroll
    for (int s = 0; s < TB; ++s)
      if (s < cnt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = __shfl_sync(0xffffffffu, x[i], s * 4 + m);
          if (nn > s) x[i] = fmaf(-beta * kk[s], u, x[i]);
          if (nn >= s) y[i] = fmaf(qk[s], u, y[i]);
        }
      }
    if (a.o && valid) {
      OT *const to = go + (t0 + nn) * v_stride + c;
      if constexpr (sizeof(OT) == 2) {
        __nv_bfloat162 p[2] = {__floats2bfloat162_rn(y[0], y[1]), __floats2bfloat162_rn(y[2], y[3])};
        *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(p);
      } else {
        *reinterpret_cast<float4 *>(to) = make_float4(y[0], y[1], y[2], y[3]);
      }
    }
    if (update) {
      *reinterpret_cast<float4 *>(&sm.u[nn][c]) = valid ? make_float4(x[0], x[1], x[2], x[3]) : make_float4(0.f, 0.f, 0.f, 0.f);
      __syncwarp();
      const float2 ua = *reinterpret_cast<const float2 *>(&sm.u[m][warp * 16 + 2 * nn]), ub = *reinterpret_cast<const float2 *>(&sm.u[m + 4][warp * 16 + 2 * nn]);
      const float4 hi = make_float4(to_tf32(ua.x), to_tf32(ua.y), to_tf32(ub.x), to_tf32(ub.y));
      const float4 lo = make_float4(ua.x - hi.x, ua.y - hi.y, ub.x - hi.z, ub.y - hi.w);
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        const float4 k = sm.last[b][lane];
        float d[4] = {}, e[4] = {};
        mma_tf32(e, hi, k.z, k.w);
        mma_tf32(e, lo, k.x, k.y);
        mma_tf32(d, hi, k.x, k.y);
        const float2 ph = *reinterpret_cast<const float2 *>(&sm.hi[8 * b + 2 * m]), pl = *reinterpret_cast<const float2 *>(&sm.lo[8 * b + 2 * m]);
        const uint64_t h2 = dpack2(ph.x, ph.y), l2 = dpack2(pl.x, pl.y);
#pragma unroll
        for (int j = 0; j < 2; ++j)  // (the tensor cores' own sums start from zero: they would cut the state's last bit off)
          S[b][j] = dfma2(S[b][j], h2, dfma2(S[b][j], l2, dpack2(e[2 * j] + d[2 * j], e[2 * j + 1] + d[2 * j + 1])));
      }
    }
  }
  if (n == 0) stage(next, 0);
  if (holds && write && (n > 0 || (now.zero && now.req >= 0))) {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const float2 x = dunpack2(S[b][0]), y = dunpack2(S[b][1]);
      *reinterpret_cast<float2 *>(st + static_cast<int64_t>(8 * b) * a.d_v) = make_float2(x.x, y.x);
      *reinterpret_cast<float2 *>(st + static_cast<int64_t>(8 * b + 1) * a.d_v) = make_float2(x.y, y.y);
    }
  }
  now = next;
  }
}

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
int launch(const DascDeltaArgs &a, void *stream) {
  const int64_t blocks = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v * (a.d_v / NCOL);
  if (blocks > 2147483647LL) return static_cast<int>(cudaErrorInvalidConfiguration);
  const dim3 grid(static_cast<unsigned>(blocks));
  if constexpr (NCOL < 128)
    if (!a.cu_seqlens) return static_cast<int>(launch_blocks(delta_step_kernel<DK, NCOL, KDA, IO, OT>, grid, dim3(kThreads<DK, NCOL>), 0, stream, a));
  constexpr size_t smem = sizeof(DraftSmem<DK, NCOL, KDA, IO>);
  auto kernel = delta_draft_kernel<DK, NCOL, KDA, IO, OT>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return static_cast<int>(e);
  }
  constexpr int NT = DraftShape<DK, NCOL>::NT;
  const dim3 some(static_cast<unsigned>(std::min<int64_t>(blocks, 148 * (512 / NT))));  // as many as fit the GPU at once
  return static_cast<int>(launch_blocks(kernel, some, dim3(NT), smem, stream, a));
}

template <int DK, bool KDA, typename IO, typename OT>
int launch_cols(const DascDeltaArgs &a, void *stream) {
  const int64_t units = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v;
  if (a.cu_seqlens && a.d_v % 128 == 0 && units * (a.d_v / 128) >= 2 * 148) return launch<DK, 128, KDA, IO, OT>(a, stream);
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
