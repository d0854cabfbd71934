// Linear attention with a decay per head in fp32 on the CUDA cores:
//     S <- exp(g_t) S + k_t v_t^T,   o_t = q_scale S^T q_t.
// One token per request (decoding) is this recurrence with the state on its way from and to memory; a few tokens (drafts)
// and the shapes and types the chunked kernel does not take run through the same registers.
//
// Several tokens go through the state together.  With P_t the product of the group's decays up to token t and D_ts of those behind s up to t,
//     o_t = P_t S^T q_t + sum_{s <= t} D_ts (q_t . k_s) v_s,   then S <- P_n S + sum_s (D_ns k_s) v_s^T:
// one multiplication per value of the state and token for the outputs and one for the state, where the recurrence has three, and
// none for the state after the last group of a call that does not keep it.
//
// Split: columns of the state do not interact, so a thread block owns NCOL columns of one (request, layer, head) state, all
// of it in registers: a thread holds ROWS rows of four columns.  The read-out sums over rows, which are spread over
// RG groups of threads: partial sums meet in shared memory once per group of TB tokens, in a fixed order.  Decays multiply, they are not
// differences of sums: exp(-inf) is a zero like any other.
// Bound: bytes of the state (128 KB read and written per 128 x 128 head and call).  A token of 256 requests x 32 heads: 163 us, 101 % of the
// measured copy rate of 6567 GB/s.  Few tokens are bound by the latency of a block's steps (loads, decays, products of queries and keys,
// outputs), of which two blocks per SM hide one: 5 tokens of 64 requests x 32 heads scored in 45 us (22 us of bytes), advanced in 55 us (41).
// With 128 rows and columns two blocks per SM leave 128 registers, of which groups of tokens spill 11 to 15 (44 to 60 bytes).
#include <cuda_runtime.h>

#include "decay_common.cuh"

namespace {

constexpr int TB = 8;    // tokens per group
// How many states on the next to be fetched into L2 is: a wave of blocks (two per SM).  It took 5 tokens of 64 requests x
// 32 heads, scored, from 51 to 48 us (45 since), and advanced from 61 to 55.
constexpr int kAhead = 2 * 148;

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

// 128 x 128 values are held by 256 threads, all else by 128: at most 64 registers of state per thread
template <int DK, int NCOL>
constexpr int kThreads = DK * NCOL > 128 * 64 ? 256 : 128;

template <int DK, int NCOL, bool STEP, typename IO>
struct Smem {
  static constexpr int NT = kThreads<DK, NCOL>;
  static constexpr int N = STEP ? 1 : TB;
  static constexpr int RG = NT / (NCOL / 4);
  alignas(16) uint64_t kk[N][DK], qq[N][DK];  // each value twice: operands of the packed instructions
  alignas(16) float v[N][NCOL];
  alignas(16) float part[N][RG][NCOL];
  float alpha[N], alpha_lo[N];  // a single token's decay
  float upto[N];                // P_t
  float qk[N][N];               // D_ts q_scale q_t . k_s
  // the next group, as it comes from memory
  alignas(16) IO raw_q[STEP ? 1 : N][STEP ? 8 : DK], raw_k[STEP ? 1 : N][STEP ? 8 : DK], raw_v[STEP ? 1 : N][STEP ? 8 : NCOL];
  alignas(16) float raw_g[N];
};

template <int DK, int NCOL, bool STEP, typename IO, typename OT>
__global__ void __launch_bounds__((kThreads<DK, NCOL>), (kThreads<DK, NCOL> == 256 ? 2 : 3)) decay_seq_kernel(const __grid_constant__ DascDecayArgs a) {
  constexpr int NT = kThreads<DK, NCOL>, LPR = NCOL / 4, RG = NT / LPR, ROWS = DK / RG;
  using Sm = Smem<DK, NCOL, STEP, IO>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, cg = tid % LPR, rg = tid / LPR;
  const int parts = a.d_v / NCOL;
  const int part = blockIdx.x % parts, unit = blockIdx.x / parts;
  const int h = unit % a.H_v, lc = unit / a.H_v % a.n_layers_in_call, r = unit / (a.H_v * a.n_layers_in_call);
  const int hk = h / (a.H_v / a.H_k);
  if (STEP)
    stream_order_begin();
  else
    stream_order_wait();

  if (!STEP && a.workspace && blockIdx.x == 0)  // nothing here can time out
    for (int i = tid; i < kDecayStatusWords; i += NT) static_cast<uint32_t *>(a.workspace)[i] = 0;
  const int req = a.req_idx[r];
  if (req < 0) return;
  const DecayRange range = decay_range(a, r);
  const int n = range.n;
  const bool merge = a.mode == DASC_DECAY_SCRATCH_MERGE_LOCAL;
  const int layer = a.layer_begin + lc;
  const bool zero = merge || (a.from_zero && a.from_zero[r] != 0);
  const bool write = a.mode != DASC_DECAY_SCORE && !(merge && a.row_keep[layer * a.rows_per_layer + static_cast<int64_t>(h) * DK]);
  if (!STEP && ((n == 0 && !(write && zero)) || (!write && !a.o))) return;

  const int64_t tok0 = static_cast<int64_t>(lc) * a.total_tokens + range.begin;
  float *const st = a.state + req * a.req_stride + layer * a.layer_stride + static_cast<int64_t>(h) * DK * a.d_v + part * NCOL +
                    static_cast<int64_t>(rg) * ROWS * a.d_v + cg * 4;
  const IO *const gq = static_cast<const IO *>(a.q) + (tok0 * a.H_k + hk) * DK;
  const IO *const gk = static_cast<const IO *>(a.k) + (tok0 * a.H_k + hk) * DK;
  const IO *const gv = static_cast<const IO *>(a.v) + (tok0 * a.H_v + h) * a.d_v + part * NCOL;
  const float *const gg = a.g_per_head ? a.g + lc * a.H_v + h : a.g + tok0 * a.H_v + h;
  OT *const go = static_cast<OT *>(a.o) + (tok0 * a.H_v + h) * a.d_v + part * NCOL;
  const int64_t qk_stride = static_cast<int64_t>(a.H_k) * DK, v_stride = static_cast<int64_t>(a.H_v) * a.d_v;
  const int64_t g_stride = a.g_per_head ? 0 : a.H_v;

  uint64_t S[ROWS][2];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!zero) x = *reinterpret_cast<const float4 *>(st + static_cast<int64_t>(i) * a.d_v);
    S[i][0] = dpack2(x.x, x.y);
    S[i][1] = dpack2(x.z, x.w);
  }

  auto stage = [&](int t0) {  // raw rows of a group, 16 bytes per copy
    const int cnt = min(TB, n - t0);
    constexpr int QV = DK * sizeof(IO) / 16, VV = NCOL * sizeof(IO) / 16;
    for (int i = tid; i < cnt * QV; i += NT) {
      const int t = i / QV, j = i % QV * (16 / sizeof(IO));
      cp_async16(&sm.raw_k[t][j], gk + (t0 + t) * qk_stride + j);
      if (a.o) cp_async16(&sm.raw_q[t][j], gq + (t0 + t) * qk_stride + j);
    }
    for (int i = tid; i < cnt * VV; i += NT) {
      const int t = i / VV, j = i % VV * (16 / sizeof(IO));
      cp_async16(&sm.raw_v[t][j], gv + (t0 + t) * v_stride + j);
    }
    if (tid < cnt) cp_async4(&sm.raw_g[tid], gg + (t0 + tid) * g_stride);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // A decay rounded to fp32 is off by up to half an ulp, the same every time where the decay is constant: 6e-4 of a state that lasts 10^4
  // tokens.  So what it is short of is carried along (1 + d, d good to its own last bits).
  auto decay = [&](float g, float &hi, float &lo) {
    const float d = expm1f(g), a1 = 1.f + d;
    const bool slow = g > -0.7f;
    hi = slow ? a1 : expf(g);
    lo = slow ? d - (a1 - 1.f) : 0.f;
  };
  auto token = [&]() {  // a single one
    const uint64_t aa = dpack2(sm.alpha[0], sm.alpha[0]), ll = dpack2(sm.alpha_lo[0], sm.alpha_lo[0]);
    const auto step = [&](uint64_t &s, uint64_t kv) { s = dfma2(s, aa, dfma2(s, ll, kv)); };
    const ulonglong2 vv = *reinterpret_cast<const ulonglong2 *>(&sm.v[0][cg * 4]);
    uint64_t o0 = 0, o1 = 0;
#pragma unroll
    for (int i = 0; i < ROWS; i += 2) {
      const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.kk[0][rg * ROWS + i]);
      step(S[i][0], dmul2(kk.x, vv.x));
      step(S[i][1], dmul2(kk.x, vv.y));
      step(S[i + 1][0], dmul2(kk.y, vv.x));
      step(S[i + 1][1], dmul2(kk.y, vv.y));
      if (STEP || a.o) {
        const ulonglong2 qq = *reinterpret_cast<const ulonglong2 *>(&sm.qq[0][rg * ROWS + i]);
        o0 = dfma2(S[i][0], qq.x, o0);
        o1 = dfma2(S[i][1], qq.x, o1);
        o0 = dfma2(S[i + 1][0], qq.y, o0);
        o1 = dfma2(S[i + 1][1], qq.y, o1);
      }
    }
    if (STEP || a.o) *reinterpret_cast<ulonglong2 *>(&sm.part[0][rg][cg * 4]) = make_ulonglong2(o0, o1);
  };
  auto store_state = [&]() {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float2 x = dunpack2(S[i][0]), y = dunpack2(S[i][1]);
      *reinterpret_cast<float4 *>(st + static_cast<int64_t>(i) * a.d_v) = make_float4(x.x, x.y, y.x, y.y);
    }
  };
  auto outputs = [&](int t0, int cnt) {
#pragma unroll 2
    for (int i = tid; i < cnt * NCOL; i += NT) {
      const int t = i / NCOL, c = i % NCOL;
      float x = 0.f;
#pragma unroll
      for (int j = 0; j < RG; ++j) x += sm.part[t][j][c];
      if (!STEP && n > 1) {
        x *= sm.upto[t];
#pragma unroll
        for (int s = 0; s < TB; ++s)
          if (s <= t) x = fmaf(sm.qk[t][s % Sm::N], sm.v[s % Sm::N][c], x);
      }
      go[(t0 + t) * v_stride + c] = from_float<OT>(x);
    }
  };

  if constexpr (STEP) {
    for (int i = tid; i < DK; i += NT) {
      const float k = to_float<IO>(gk[i]), q = to_float<IO>(gq[i]) * a.q_scale;
      sm.kk[0][i] = dpack2(k, k);
      sm.qq[0][i] = dpack2(q, q);
    }
    for (int i = tid; i < NCOL; i += NT) sm.v[0][i] = to_float<IO>(gv[i]);
    if (tid == 0) decay(*gg, sm.alpha[0], sm.alpha_lo[0]);
    __syncthreads();
    token();
    store_state();
    __syncthreads();
    outputs(0, 1);
  } else {
    if (n > 0) stage(0);
    // the state of a unit that a block of the next wave works on starts on its way into L2
    const int64_t ahead = static_cast<int64_t>(unit) + kAhead / parts;
    if (tid == NT - 1 && part == 0 && !merge && ahead < static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v) {
      const int at = static_cast<int>(ahead), ah = at % a.H_v, al = at / a.H_v % a.n_layers_in_call, ar = at / (a.H_v * a.n_layers_in_call);
      const int other = a.req_idx[ar];
      if (other >= 0 && !(a.from_zero && a.from_zero[ar] != 0))
        bulk_prefetch(a.state + other * a.req_stride + (a.layer_begin + al) * a.layer_stride + static_cast<int64_t>(ah) * DK * a.d_v, DK * a.d_v * 4);
    }
    for (int t0 = 0; t0 < n; t0 += TB) {
      const int cnt = min(TB, n - t0);
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
      const bool update = write || t0 + TB < n || n == 1;  // (a single token's output comes from the new state)
      // every warp for itself: lane t < cnt holds token t's decay, the other lanes 1
      const float g = lane < cnt ? sm.raw_g[lane] : 0.f;
      float alpha, lo;
      decay(g, alpha, lo);
      if (tid == 0) {
        sm.alpha[0] = alpha;
        sm.alpha_lo[0] = lo;
      }
      float upto = alpha, behind = __shfl_down_sync(0xffffffffu, alpha, 1);  // products of the decays up to a token, and behind it
#pragma unroll
      for (int d = 1; d < TB; d <<= 1) {
        const float x = __shfl_up_sync(0xffffffffu, upto, d), y = __shfl_down_sync(0xffffffffu, behind, d);
        if (lane >= d) upto *= x;
        behind *= y;  // (lanes from cnt on: 1)
      }
      if (tid < TB) sm.upto[tid] = upto;
      // The whole group's decay of the state, with what a rounded factor is short of.  The sum G of the logarithms is off by an ulp
      // or so, which costs what it is multiplied with a relative G 2^-23, and leaves e^G of it.
      float all_hi = g, all_lo;
#pragma unroll
      for (int d = 1; d < TB; d <<= 1) all_hi += __shfl_xor_sync(0xffffffffu, all_hi, d);
      decay(__shfl_sync(0xffffffffu, all_hi, 0), all_hi, all_lo);
      for (int i = tid; i < cnt * DK; i += NT) {
        const int t = i / DK, c = i % DK;
        const float d = __shfl_sync(0xffffffffu, behind, t);  // (t is the same in all of a warp)
        if (update) {
          const float k = to_float<IO>(sm.raw_k[t][c]) * d;
          sm.kk[t][c] = dpack2(k, k);
        }
        if (a.o) {
          const float q = to_float<IO>(sm.raw_q[t][c]) * a.q_scale;
          sm.qq[t][c] = dpack2(q, q);
        }
      }
      for (int i = tid; i < cnt * NCOL; i += NT) sm.v[i / NCOL][i % NCOL] = to_float<IO>(sm.raw_v[i / NCOL][i % NCOL]);
      if (a.o && n > 1) {
        // D_ts q_t . k_s: a warp has one or two tokens t; its lanes' parts of the 8 or 16 sums fold into one another
        constexpr int PER = DK / 32, OWN = TB / (NT / 32), V = OWN * TB;
        struct alignas(sizeof(IO) * PER) Part {
          IO x[PER];
        };
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = 0.f;
        Part q[OWN];
#pragma unroll
        for (int o = 0; o < OWN; ++o) q[o] = *reinterpret_cast<const Part *>(&sm.raw_q[OWN * warp + o][lane * PER]);
#pragma unroll
        for (int s = 0; s < TB; ++s) {
          const Part k = *reinterpret_cast<const Part *>(&sm.raw_k[s][lane * PER]);
#pragma unroll
          for (int o = 0; o < OWN; ++o)
#pragma unroll
            for (int j = 0; j < PER; ++j) x[o * TB + s] = fmaf(to_float<IO>(q[o].x[j]), to_float<IO>(k.x[j]), x[o * TB + s]);
        }
#pragma unroll
        for (int w = V / 2; w > 0; w >>= 1) {
          const int other = w * 32 / V;
          const bool up = lane & other;
#pragma unroll
          for (int j = 0; j < w; ++j) {
            const float mine = up ? x[j + w] : x[j];
            x[j] = mine + __shfl_xor_sync(0xffffffffu, up ? x[j] : x[j + w], other);
          }
        }
#pragma unroll
        for (int d = 16 / V; d > 0; d >>= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], d);
        const int at = lane / (32 / V), t = OWN * warp + at / TB, s = at % TB;
        float d = 1.f;
#pragma unroll
        for (int u = 1; u < TB; ++u) {
          const float y = __shfl_sync(0xffffffffu, alpha, u);
          if (u > s && u <= t) d *= y;
        }
        if (s <= t && lane % (32 / V) == 0) sm.qk[t][s] = x[0] * a.q_scale * d;
      }
      __syncthreads();
      if (t0 + TB < n) stage(t0 + TB);
      if (n == 1) {
        token();
      } else {
        if (a.o) {
#pragma unroll 2
          for (int t = 0; t < cnt; ++t) {
            uint64_t o0 = 0, o1 = 0;
#pragma unroll
            for (int i = 0; i < ROWS; i += 2) {
              const ulonglong2 qq = *reinterpret_cast<const ulonglong2 *>(&sm.qq[t][rg * ROWS + i]);
              o0 = dfma2(S[i][0], qq.x, o0);
              o1 = dfma2(S[i][1], qq.x, o1);
              o0 = dfma2(S[i + 1][0], qq.y, o0);
              o1 = dfma2(S[i + 1][1], qq.y, o1);
            }
            *reinterpret_cast<ulonglong2 *>(&sm.part[t][rg][cg * 4]) = make_ulonglong2(o0, o1);
          }
        }
        if (update) {
          const uint64_t hi = dpack2(all_hi, all_hi), ll = dpack2(all_lo, all_lo);
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            S[i][0] = dfma2(S[i][0], hi, dmul2(S[i][0], ll));
            S[i][1] = dfma2(S[i][1], hi, dmul2(S[i][1], ll));
          }
#pragma unroll 2
          for (int t = 0; t < cnt; ++t) {
            const ulonglong2 vv = *reinterpret_cast<const ulonglong2 *>(&sm.v[t][cg * 4]);
#pragma unroll
            for (int i = 0; i < ROWS; i += 2) {
              const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.kk[t][rg * ROWS + i]);
              S[i][0] = dfma2(kk.x, vv.x, S[i][0]);
              S[i][1] = dfma2(kk.x, vv.y, S[i][1]);
              S[i + 1][0] = dfma2(kk.y, vv.x, S[i + 1][0]);
              S[i + 1][1] = dfma2(kk.y, vv.y, S[i + 1][1]);
            }
          }
        }
      }
      if (a.o) {
        __syncthreads();
        outputs(t0, cnt);  // (the next group's partial sums come behind two barriers)
      }
    }
    stream_order_release();
    if (write) store_state();
  }
}

template <int DK, int NCOL, bool STEP, typename IO, typename OT>
int launch(const DascDecayArgs &a, void *stream) {
  const int64_t blocks = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v * (a.d_v / NCOL);
  if (blocks > 2147483647LL) return static_cast<int>(cudaErrorInvalidConfiguration);
  constexpr int NT = kThreads<DK, NCOL>;
  constexpr size_t smem = sizeof(Smem<DK, NCOL, STEP, IO>);
  auto kernel = decay_seq_kernel<DK, NCOL, STEP, IO, OT>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return static_cast<int>(e);
  }
  return static_cast<int>(launch_blocks(kernel, dim3(static_cast<unsigned>(blocks)), dim3(NT), smem, stream, a));
}

template <int DK, int NCOL, typename IO, typename OT>
int launch_form(const DascDecayArgs &a, void *stream) {
  return a.cu_seqlens ? launch<DK, NCOL, false, IO, OT>(a, stream) : launch<DK, NCOL, true, IO, OT>(a, stream);
}

template <int DK, typename IO, typename OT>
int launch_cols(const DascDecayArgs &a, void *stream) {
  const int64_t units = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v;
  // The widest part of the columns that still gives every SM a block or two.  Measured for 64 tokens of one request, in us with parts of
  // 32 / 64 / 128 columns: 37 heads 29 / 35 / 43, 148 heads 59 / 45 / 45, 296 heads 94 / 80 / 68, 2048 heads 565 / 414 / 381.
  if (a.d_v % 128 == 0 && units * (a.d_v / 128) >= 2 * 148) {
    if (a.cu_seqlens) return launch<DK, 128, false, IO, OT>(a, stream);
    if constexpr (DK <= 64) return launch<DK, 128, true, IO, OT>(a, stream);  // (d_k = 128: 163 us with parts of 64 columns, 172 with 128, 256 requests of 32 heads)
  }
  if (a.d_v % 64 == 0 && units * (a.d_v / 64) >= 2 * 148) return launch_form<DK, 64, IO, OT>(a, stream);
  return launch_form<DK, 32, IO, OT>(a, stream);
}

template <int DK>
int launch_types(const DascDecayArgs &a, void *stream) {
  if (a.io_bf16)
    return a.o_bf16 ? launch_cols<DK, __nv_bfloat16, __nv_bfloat16>(a, stream) : launch_cols<DK, __nv_bfloat16, float>(a, stream);
  return a.o_bf16 ? launch_cols<DK, float, __nv_bfloat16>(a, stream) : launch_cols<DK, float, float>(a, stream);
}

}  // namespace

int dasc_launch_decay_seq(const DascDecayArgs &a, void *stream) {
  if (a.d_v % 32 != 0) return -1;
  switch (a.d_k) {
    case 128: return launch_types<128>(a, stream);
    case 64: return launch_types<64>(a, stream);
    case 32: return launch_types<32>(a, stream);
  }
  return -1;
}
