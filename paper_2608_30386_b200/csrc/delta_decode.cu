// The gated delta rule in serving: one token per request (decoding), and a few drafted tokens.
//     S <- Diag(a_t) S,   u_t = beta_t (v_t - S^T k_t),   S <- S + k_t u_t^T,   o_t = q_scale S^T q_t
// a_t is a vector over the key channels (KDA) or one number (GDN).
//
// One token, in fp32 on the CUDA cores: with r = S^T (a k) and y = S^T (a q) in one pass over the state, u = beta (v - r), o = q_scale (y + (k . q) u),
// and the new state is a S + k u^T on its way to memory.  The old state stays in registers, so beams that continue the same state read it once.
// Bound: bytes of the state (128 KB read and written per 128 x 128 head).  256 requests x 32 heads: 165 us over inputs that change from call to call (161 back to back over
// the same ones), the measured copy rate of 6462 GB/s; 32 x 8 beams, 5.25 of 8 states read on average: 148 us, 94 % (the blocks of beams that share a source have up to eight
// times the work of others); one request: 2.4 to 3.2 us.
//
// Several tokens go through the state together, in groups of TB.  P_t is the product of a group's decays up to token t, D_ts of those behind s up to t:
//     u_t = beta_t (v_t - S^T (P_t k_t) - sum_{s < t} (k_t . D_ts k_s) u_s)
//     o_t = q_scale (S^T (P_t q_t) + sum_{s <= t} (q_t . D_ts k_s) u_s),      S <- P_n S + sum_s (D_ns k_s) u_s^T
// so that the sums over the state's rows of all tokens are independent of one another, and only sums over at most TB values per column are a chain.
// All in fp32 on the CUDA cores: per token and value of the state three multiply-adds (key, query, update), 9 us of them where five tokens of 64 requests x 32 heads are
// scored.  Bound: those take 51 us scored and 66 us advanced (their bytes 23 and 42).  Instructions of two blocks of 256 threads per SM, each with its state in 64 registers
// of a thread, which issue in half of the cycles and overlap little of a block's steps: without the sums over rows it is 34 us, without the preparation of operands
// 40, without reading states 43, with reading alone 25.  Tried and slower: the products on the tensor cores in three tf32 parts (53 and 83: splitting values costs what
// the products gain, and eight tokens cost what one does), states in shared memory ahead of their use (57 / 88), preparation and products in warps of their
// own with a block per SM (73 / 115: the preparation is a chain of latencies), states read twice instead of held, with four blocks per SM (50 / 104).
//
// Split: columns of the state do not interact, so a thread block owns NCOL columns of one (request, layer, head) state.
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

// Of a block for single tokens: at most 64 registers of state per thread.  Where parts are 64 columns wide four blocks per SM: with the registers that the compiler
// would take where decays go by channel it is three, and 256 requests x 32 heads take 174 us instead of 161, 128 pairs of beams of one state 147 instead of 133; five
// blocks take 162 and 128, and 256 requests of d_k = d_v = 64 58 instead of 67.  Where they are 32 wide (few states, or a d_v that is no multiple of 64) five blocks
// instead of four: 5 requests x 32 heads 5.7 us instead of 6.7, 9 requests 9.1 instead of 9.5, 256 of d_v = 32 48 instead of 52, of d_v = 96 141 instead of 161; six
// 5.9, 8.9, 46 and 132.  (All back to back, layer after layer from memory.)
constexpr int kStepThreads = 128;

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
  static constexpr int RG = kStepThreads / (NCOL / 4);
  // each value twice: operands of the packed instructions
  alignas(16) uint64_t ak[DK], aq[DK], k[DK], hi[DK], lo[DK];
  alignas(16) float part[2][RG][NCOL];
  alignas(16) float v[NCOL], u[NCOL];
  float kq[4];
};

template <int DK, int NCOL, bool KDA, typename IO, typename OT>
__global__ void __launch_bounds__(kStepThreads, NCOL == 64 ? 4 : 5) delta_step_kernel(const __grid_constant__ DascDeltaArgs a) {
  constexpr int NT = kStepThreads, LPR = NCOL / 4, RG = NT / LPR, ROWS = DK / RG;
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

// Several tokens: a warp has 16 columns of the state and all of its rows, a lane four columns of rows 4 g .. 4 g + 3 of every 32, g = lane / 4.  They are held in
// pairs of rows: a 16-byte load brings four rows of a key to eight packed multiply-adds.  In pairs of columns it would be two rows, each value twice, to four of
// them, and these loads the bound (60 / 73 us).
template <int DK, int NCOL>
struct DraftShape {
  static constexpr int WARPS = NCOL / 16, NT = NCOL > 32 ? WARPS * 32 : 128, STEPS = DK / 32;  // (a narrow part has two warps that only prepare)
};

// What a group of tokens brings to a state's NCOL columns, and the rows it is made from.
template <int DK, int NCOL>
struct Operands {
  alignas(16) float k[TB][DK], q[TB][DK];    // P_t k_t, q_scale P_t q_t
  alignas(16) float last[TB][DK];            // D_ns k_s
  alignas(16) float hi[DK], lo[DK];          // the group's decay
  alignas(16) float v[TB][NCOL], u[TB][NCOL];
  // of s, then of t, first the even ones: -beta_t k_t . D_ts k_s where s < t, q_scale q_t . D_ts k_s where s <= t, else 0
  alignas(16) float kk[TB][TB], qk[TB][TB];
  float beta[TB];
};
template <int DK, int NCOL, bool KDA, typename IO>
struct RawRows {  // as they come from memory
  alignas(16) IO q[TB][DK], k[TB][DK], v[TB][NCOL];
  alignas(16) float g[TB][KDA ? DK : 4], beta[TB];
};
template <int DK, int NCOL, bool KDA, typename IO>
struct DraftSmem {
  Operands<DK, NCOL> op;
  RawRows<DK, NCOL, KDA, IO> raw;
};

// A block takes every gridDim.x-th part of a state; what the next one needs is on its way while one is worked on.
struct Job {
  int part, h, lc, r;  // counted up in this order
  int req, begin, n;
  bool zero;
};
template <int DK, int NCOL>
struct JobWalk {
  const DascDeltaArgs &a;
  const int dv, parts;
  const Job stride;
  __device__ __forceinline__ explicit JobWalk(const DascDeltaArgs &args)
      : a(args), dv(NCOL == 128 ? 128 : args.d_v), parts(dv / NCOL), stride(digits(static_cast<int>(gridDim.x))) {}  // (128 columns at once: only where that is all)
  __device__ __forceinline__ Job digits(int i) const {
    return Job{i % parts, i / parts % a.H_v, i / (parts * a.H_v) % a.n_layers_in_call, i / (parts * a.H_v) / a.n_layers_in_call, -1, 0, 0, false};
  }
  __device__ __forceinline__ void look_up(Job &x) const {
    x.req = -1;
    x.n = 0;
    if (x.r < a.n_req) {
      x.req = a.req_idx[x.r];
      x.begin = a.cu_seqlens[x.r];
      x.n = max(a.cu_seqlens[x.r + 1] - x.begin, 0);
      if (a.seq_used) x.n = min(x.n, max(a.seq_used[x.r], 0));
      if (x.req < 0) x.n = 0;
      x.zero = a.from_zero && a.from_zero[x.r] != 0;
    }
  }
  __device__ __forceinline__ Job first() const {
    Job x = digits(static_cast<int>(blockIdx.x));
    look_up(x);
    return x;
  }
  __device__ __forceinline__ Job after(const Job &x) const {  // gridDim.x behind x
    Job y = x;
    y.part += stride.part;
    bool carry = y.part >= parts;
    y.part -= carry ? parts : 0;
    y.h += stride.h + carry;
    carry = y.h >= a.H_v;
    y.h -= carry ? a.H_v : 0;
    y.lc += stride.lc + carry;
    carry = y.lc >= a.n_layers_in_call;
    y.lc -= carry ? a.n_layers_in_call : 0;
    y.r += stride.r + carry;
    look_up(y);
    return y;
  }
  __device__ __forceinline__ float *state_of(const Job &x) const {
    return a.state + x.req * a.req_stride + (a.layer_begin + x.lc) * a.layer_stride + (static_cast<int64_t>(x.h) * DK * dv + x.part * NCOL);
  }
};

// The rows of `cnt` tokens of a job from token t0 on, as they are, 16 bytes per copy, by the block's NT threads (offsets between eight
// tokens are below 2^31: the caller has looked).
template <int DK, int NCOL, bool KDA, typename IO, int NT>
__device__ __forceinline__ void copy_rows(RawRows<DK, NCOL, KDA, IO> &raw, const DascDeltaArgs &a, const Job &x, int cnt, int t0) {
  const int tid = threadIdx.x, dv = NCOL == 128 ? 128 : a.d_v, group = a.H_v / a.H_k, v_stride = a.H_v * dv;
  if (cnt > 0) {
    const int64_t tok = static_cast<int64_t>(x.lc) * a.total_tokens + (x.begin + t0), row = tok * a.H_v + x.h;
    const int64_t key = (tok * a.H_k + x.h / group) * DK;
    constexpr int VE = 16 / sizeof(IO), QV = DK / VE, VV = NCOL / VE, GV = DK / 4;
    const int qk_stride = a.H_k * DK;
    const IO *const gk = static_cast<const IO *>(a.k) + key, *const gq = static_cast<const IO *>(a.q) + key;
#pragma unroll
    for (int i = tid; i < TB * QV * 2; i += NT) {
      const int t = i / QV % TB, j = i % QV * VE;
      const bool query = i >= TB * QV;
      if (t < cnt && !(query && !a.o)) cp_async16(query ? &raw.q[t][j] : &raw.k[t][j], (query ? gq : gk) + t * qk_stride + j);
    }
    const IO *const gv = static_cast<const IO *>(a.v) + row * dv + x.part * NCOL;
#pragma unroll
    for (int i = tid; i < TB * VV; i += NT)
      if (i / VV < cnt) cp_async16(&raw.v[i / VV][i % VV * VE], gv + i / VV * v_stride + i % VV * VE);
    const float *const gg = a.g + row * (KDA ? DK : 1);
    if constexpr (KDA) {
#pragma unroll
      for (int i = tid; i < TB * GV; i += NT)
        if (i / GV < cnt) cp_async16(&raw.g[i / GV][i % GV * 4], gg + i / GV * (a.H_v * DK) + i % GV * 4);
    } else {
      if (tid < cnt) cp_async4(&raw.g[tid][0], gg + tid * a.H_v);
    }
    if (tid >= NT - 32 && tid - (NT - 32) < cnt) cp_async4(&raw.beta[tid - (NT - 32)], a.beta + row + (tid - (NT - 32)) * a.H_v);
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}

// The group's `cnt` tokens as operands, by the block's NT threads.
template <int DK, int NCOL, bool KDA, typename IO, int NT>
__device__ __forceinline__ void prepare(Operands<DK, NCOL> &op, const RawRows<DK, NCOL, KDA, IO> &raw, int cnt, bool update, bool want, float q_scale) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  // Products between tokens.  A warp has one token t or more; its lanes' parts of the 16 sums fold into one another.
  constexpr int PER = DK / 32;
  for (int i = tid; i < cnt * NCOL; i += NT) op.v[i / NCOL][i % NCOL] = to_float<IO>(raw.v[i / NCOL][i % NCOL]);
  if (tid < cnt) op.beta[tid] = raw.beta[tid];
  for (int t = warp; t < TB; t += NT / 32) {
    if (t >= cnt) {
      if (lane < 2 * TB) (lane < TB ? op.kk : op.qk)[lane % TB][t % 2 * 4 + t / 2] = 0.f;
      continue;
    }
    float x[2 * TB], k[PER], q[PER], G[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      k[j] = to_float<IO>(raw.k[t][lane * PER + j]);
      q[j] = want ? to_float<IO>(raw.q[t][lane * PER + j]) * q_scale : 0.f;
      G[j] = 0.f;
    }
#pragma unroll
    for (int s = TB - 1; s >= 0; --s) {
      x[s] = x[TB + s] = 0.f;
      if (s <= t) {
        float d = __expf(G[0]);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const float e = (KDA ? __expf(G[j]) : d) * to_float<IO>(raw.k[s][lane * PER + j]);
          x[s] = fmaf(k[j], e, x[s]);
          x[TB + s] = fmaf(q[j], e, x[TB + s]);
          G[j] += raw.g[s][KDA ? lane * PER + j : 0];
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
    if (lane < 2 * TB) (lane < TB ? op.kk : op.qk)[lane % TB][t % 2 * 4 + t / 2] = lane >= TB ? x[0] : lane == t ? 0.f : -raw.beta[t] * x[0];
  }
  // Keys and queries behind the group's start, and keys decayed to its end, a thread per channel and kind.  Decays of several tokens
  // are exponentials of sums of their logarithms, always over the tokens between two points (-infinity is like any other number there).  A factor e^G is good to
  // (2 + 1.2 |G|) 2^-23 of itself, the documented bound of __expf, and the sum's rounding, 2^-24 |G|: together never worse than 2^-22 of an undecayed one.  Only the decay
  // of the state itself, the same token after token, is better than that (decay_factor).
  const int kinds = (want ? 2 : 1) + update;
  for (int i = tid; i < kinds * DK; i += NT) {
    const int c = i % DK, what = i / DK;
    float G = 0.f;
    if (what < kinds - update) {
      const IO(*const rows)[DK] = what ? raw.q : raw.k;
      float(*const to)[DK] = what ? op.q : op.k;
      const float scale = what ? q_scale : 1.f;
#pragma unroll
      for (int t = 0; t < TB; ++t)
        if (t < cnt) {
          G += raw.g[t][KDA ? c : 0];
          to[t][c] = __expf(G) * (to_float<IO>(rows[t][c]) * scale);
        }
    } else {
#pragma unroll
      for (int t = TB - 1; t >= 0; --t)
        if (t < cnt) {
          op.last[t][c] = __expf(G) * to_float<IO>(raw.k[t][c]);
          G += raw.g[t][KDA ? c : 0];
        }
      decay_factor(G, op.hi[c], op.lo[c]);
    }
  }
}

// A warp's 16 columns of a group, the lane's first of them `col` of the block's.  Outputs go to `o`, v_stride apart, where `want`.
template <int DK, int NCOL, typename OT>
__device__ __forceinline__ void run_group(Operands<DK, NCOL> &op, uint64_t (&S)[DK / 32][2][4], int cnt, int col, bool update, bool want, OT *o, int64_t v_stride) {
  const int lane = threadIdx.x % 32, g = lane / 4;
  // S^T (P_t k_t) and S^T (P_t q_t), two tokens at a time: a lane's sums over its rows, four columns each, then folded into one another, so that lane g
  // ends with column col + g % 4 of the first token (g < 4) or the second
  const int odd = g / 4, c = col + g % 4;
  auto products = [&](const float *row, const float *other) {
    uint64_t x[2][4] = {};
#pragma unroll
    for (int i = 0; i < DK / 32; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>((j ? other : row) + 32 * i + 4 * g);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[j][c] = dfma2(S[i][1][c], k.y, dfma2(S[i][0][c], k.x, x[j][c]));
      }
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 a = dunpack2(x[j / 4][j % 4]);
      f[j] = a.x + a.y;
    }
#pragma unroll
    for (int w = 4; w > 0; w >>= 1) {
      const bool up = g & w;
#pragma unroll
      for (int j = 0; j < w; ++j) {
        const float mine = up ? f[j + w] : f[j];
        f[j] = mine + __shfl_xor_sync(0xffffffffu, up ? f[j] : f[j + w], w * 4);
      }
    }
    return f[0];
  };
  float x[TB / 2], y[TB / 2];
#pragma unroll
  for (int p = 0; p < TB / 2; ++p)
    if (2 * p < cnt) {  // (of a token behind the last one there is anything, and nothing reads it)
      const bool alone = want && 2 * p + 1 == cnt;  // the last token's key and query at once
      const float z = products(op.k[2 * p], alone ? op.q[2 * p] : op.k[2 * p + 1]);
      x[p] = op.beta[2 * p + odd] * (op.v[2 * p + odd][c] - z);
      if (alone)
        y[p] = __shfl_down_sync(0xffffffffu, z, 16);
      else if (want)
        y[p] = products(op.q[2 * p], op.q[2 * p + 1]);
    }
  // u_t, one token after the other, and what it brings to the later ones
#pragma unroll
  for (int t = 0; t < TB; ++t)
    if (t < cnt) {
      const float u = __shfl_sync(0xffffffffu, x[t / 2], lane % 16 + t % 2 * 16);
      if (odd == t % 2) op.u[t][c] = u;
      const float4 k4 = *reinterpret_cast<const float4 *>(&op.kk[t][4 * odd]), q4 = *reinterpret_cast<const float4 *>(&op.qk[t][4 * odd]);
      const float kk[4] = {k4.x, k4.y, k4.z, k4.w}, qk[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
      for (int p = t / 2; p < TB / 2; ++p)
        if (p > t / 2 || odd >= t % 2) {
          if (p > t / 2 || t % 2 == 0) x[p] = fmaf(kk[p], u, x[p]);
          y[p] = fmaf(qk[p], u, y[p]);
        }
    }
  if (want) {
#pragma unroll
    for (int p = 0; p < TB / 2; ++p)
      if (2 * p + odd < cnt) o[(2 * p + odd) * v_stride + c] = from_float<OT>(y[p]);
  }
  if (!update) return;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < DK / 32; ++i) {
    const ulonglong2 hi = *reinterpret_cast<const ulonglong2 *>(&op.hi[32 * i + 4 * g]), lo = *reinterpret_cast<const ulonglong2 *>(&op.lo[32 * i + 4 * g]);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      S[i][0][c] = dfma2(S[i][0][c], hi.x, dmul2(S[i][0][c], lo.x));
      S[i][1][c] = dfma2(S[i][1][c], hi.y, dmul2(S[i][1][c], lo.y));
    }
  }
#pragma unroll 2
  for (int t = 0; t < cnt; ++t) {
    const float4 w = *reinterpret_cast<const float4 *>(&op.u[t][col]);
    const uint64_t ww[4] = {dpack2(w.x, w.x), dpack2(w.y, w.y), dpack2(w.z, w.z), dpack2(w.w, w.w)};
#pragma unroll
    for (int i = 0; i < DK / 32; ++i) {
      const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>(&op.last[t][32 * i + 4 * g]);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        S[i][0][c] = dfma2(k.x, ww[c], S[i][0][c]);
        S[i][1][c] = dfma2(k.y, ww[c], S[i][1][c]);
      }
    }
  }
}

// A thread block goes from state to state; a group's rows are on their way, and the next state in L2, while the ones before are worked on.
template <int DK, int NCOL, bool KDA, typename IO, typename OT>
__global__ void __launch_bounds__((DraftShape<DK, NCOL>::NT), (512 / DraftShape<DK, NCOL>::NT)) delta_draft_kernel(const __grid_constant__ DascDeltaArgs a) {
  using Sh = DraftShape<DK, NCOL>;
  using Sm = DraftSmem<DK, NCOL, KDA, IO>;
  constexpr int NT = Sh::NT, STEPS = Sh::STEPS;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, col = warp * 16 + lane % 4 * 4, row = lane / 4 * 4;
  const JobWalk<DK, NCOL> walk(a);
  const int dv = walk.dv, v_stride = a.H_v * dv;
  const bool write = !a.score, holds = warp < Sh::WARPS;
  auto stage = [&](const Job &x, int t0) { copy_rows<DK, NCOL, KDA, IO, NT>(sm.raw, a, x, min(TB, x.n - t0), t0); };
  stream_order_wait();

  Job now = walk.first();
  stage(now, 0);
  while (now.r < a.n_req) {
    const Job next = walk.after(now);
    const int n = now.n;
    float *const st = walk.state_of(now) + row * dv + col;
    OT *const go = static_cast<OT *>(a.o) + ((static_cast<int64_t>(now.lc) * a.total_tokens + now.begin) * a.H_v + now.h) * dv + now.part * NCOL;
    uint64_t S[STEPS][2][4];  // rows row + 32 i + 2 j and the one behind it
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (holds && !now.zero && n > 0) {
          x = *reinterpret_cast<const float4 *>(st + (32 * i + 2 * j) * dv);
          y = *reinterpret_cast<const float4 *>(st + (32 * i + 2 * j + 1) * dv);
        }
        S[i][j][0] = dpack2(x.x, y.x);
        S[i][j][1] = dpack2(x.y, y.y);
        S[i][j][2] = dpack2(x.z, y.z);
        S[i][j][3] = dpack2(x.w, y.w);
      }
    for (int t0 = 0; t0 < n; t0 += TB) {
      const int cnt = min(TB, n - t0);
      const bool update = write || t0 + TB < n;
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
      prepare<DK, NCOL, KDA, IO, NT>(sm.op, sm.raw, cnt, update, a.o != nullptr, a.q_scale);
      __syncthreads();
      if (t0 + TB < n) {
        stage(now, t0 + TB);
      } else {
        stage(next, 0);
        if (next.n > 0 && !next.zero) {
          if (NCOL == 128) {
            if (tid == 0) bulk_prefetch(walk.state_of(next), DK * NCOL * 4);
          } else {
            for (int i = tid; i < DK; i += NT) asm volatile("prefetch.global.L2 [%0];" ::"l"(walk.state_of(next) + i * dv));
          }
        }
      }
      if (holds) run_group<DK, NCOL>(sm.op, S, cnt, col, update, a.o != nullptr, go + static_cast<int64_t>(t0) * v_stride, v_stride);
    }
    if (n == 0) stage(next, 0);
    if (holds && write && (n > 0 || (now.zero && now.req >= 0))) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 x = dunpack2(S[i][j][0]), y = dunpack2(S[i][j][1]), z = dunpack2(S[i][j][2]), w = dunpack2(S[i][j][3]);
          *reinterpret_cast<float4 *>(st + (32 * i + 2 * j) * dv) = make_float4(x.x, y.x, z.x, w.x);
          *reinterpret_cast<float4 *>(st + (32 * i + 2 * j + 1) * dv) = make_float4(x.y, y.y, z.y, w.y);
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
    if (!a.cu_seqlens) return static_cast<int>(launch_blocks(delta_step_kernel<DK, NCOL, KDA, IO, OT>, grid, dim3(kStepThreads), 0, stream, a));
  constexpr size_t smem = sizeof(DraftSmem<DK, NCOL, KDA, IO>);
  static_assert(smem <= 48 * 1024, "what a kernel has without asking for more");
  auto kernel = delta_draft_kernel<DK, NCOL, KDA, IO, OT>;
  constexpr int NT = DraftShape<DK, NCOL>::NT;
  const dim3 some(static_cast<unsigned>(std::min<int64_t>(blocks, 148 * (512 / NT))));  // as many as fit the GPU at once
  return static_cast<int>(launch_blocks(kernel, some, dim3(NT), smem, stream, a));
}

template <int DK, bool KDA, typename IO, typename OT>
int launch_cols(const DascDeltaArgs &a, void *stream) {
  // Drafts: wide parts, since what is prepared for a group serves all of its columns.  5 tokens of 1 / 8 / 32 requests of 32 heads with d_v = 128, scored, in us with parts
  // of 32 / 64 / 128 columns: 9.1 / 8.3 / 6.2, 21.1 / 11.8 / 8.2, 73.6 / 37.9 / 27.7; advanced, 16 requests: 43.5 / 24.4 / 19.0.  Parts of 128 columns have d_v as a
  // constant; larger multiples of 128 go in parts of 64, and what is no multiple of 64 in parts of 32, which do not hold all of their values in registers (up to 232
  // bytes are spilled): 64 requests of d_v = 32 / 64 / 96 / 128 / 256 take 40 / 39 / 110 / 50 / 140 us scored and 45 / 47 / 121 / 66 / 171 advanced.
  if (a.cu_seqlens) {
    if (a.d_v == 128) return launch<DK, 128, KDA, IO, OT>(a, stream);
    return a.d_v % 64 == 0 ? launch<DK, 64, KDA, IO, OT>(a, stream) : launch<DK, 32, KDA, IO, OT>(a, stream);
  }
  // Single tokens: narrow parts until wide ones fill the GPU's places once.  KDA requests of 32 heads, layer after layer from memory, in us with parts of 32 / 64 columns:
  // 2 4.4 / 4.6, 4 5.4 / 6.1, 6 6.6 / 6.9, 8 8.4 / 7.7, 9 9.0 / 8.1, 10 9.7 / 9.6, 16 14.0 / 13.6, 36 28.1 / 26.4, 64 47.9 / 44.1; one layer that stays in L2: 4 4.2 / 5.0,
  // 8 5.9 / 5.8, 10 6.5 / 6.8, 12 7.7 / 7.5, 16 9.1 / 8.8, 36 21.8 / 18.7.  (The crossing is between 7 and 11 requests, the rule's between 9 and 10.)
  const int64_t units = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v;
  if (a.d_v % 64 == 0 && units * (a.d_v / 64) >= 4 * 148) return launch<DK, 64, KDA, IO, OT>(a, stream);
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
