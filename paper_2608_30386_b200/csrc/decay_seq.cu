// Linear attention with a decay per head, token by token in fp32 on the CUDA cores:
//     S <- exp(g_t) S + k_t v_t^T,   o_t = q_scale S^T q_t.
// One token per request (decoding) is this recurrence with the state on its way from and to memory; a few tokens (drafts)
// and the shapes and types the chunked kernel does not take run through the same registers.
//
// Split: columns of the state do not interact, so a thread block owns NCOL columns of one (request, layer, head) state, all
// of it in registers: a thread holds ROWS rows of four columns.  The read-out sums over rows, which are spread over
// RG groups of threads: partial sums meet in shared memory once per group of TB tokens, in a fixed order.
// Bound: bytes of the state (128 KB read and written per 128 x 128 head and call).
#include <cuda_runtime.h>

#include <type_traits>

#include "decay_common.cuh"

namespace {

constexpr int NT = 128;  // threads per block
constexpr int TB = 8;    // tokens per group
constexpr int kFew = 16;  // tokens over which decays may be rounded

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

template <int DK, int NCOL, bool STEP, typename IO>
struct Smem {
  static constexpr int N = STEP ? 1 : TB;
  static constexpr int RG = NT / (NCOL / 4);
  alignas(16) uint64_t kk[N][DK], qq[N][DK];  // each value twice: operands of the packed instructions
  alignas(16) float v[N][NCOL];
  alignas(16) float part[N][RG][NCOL];
  float alpha[N], alpha_lo[N];
  // the next group, as it comes from memory
  alignas(16) IO raw_q[STEP ? 1 : N][STEP ? 8 : DK], raw_k[STEP ? 1 : N][STEP ? 8 : DK], raw_v[STEP ? 1 : N][STEP ? 8 : NCOL];
  alignas(16) float raw_g[N];
};

template <int DK, int NCOL, bool STEP, typename IO, typename OT>
__global__ void __launch_bounds__(NT, 3) decay_seq_kernel(const __grid_constant__ DascDecayArgs a) {
  constexpr int LPR = NCOL / 4, RG = NT / LPR, ROWS = DK / RG;
  using Sm = Smem<DK, NCOL, STEP, IO>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, cg = tid % LPR, rg = tid / LPR;
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
  // tokens.  So beyond a few tokens what alpha is short of is carried along (1 + d, d good to its own last bits).
  auto token = [&](int t, auto whole) {
    const float al = sm.alpha[t], lo = sm.alpha_lo[t];
    const uint64_t aa = dpack2(al, al), ll = dpack2(lo, lo);
    const auto step = [&](uint64_t &s, uint64_t kv) {
      if constexpr (decltype(whole)::value) kv = dfma2(s, ll, kv);
      s = dfma2(s, aa, kv);
    };
    const ulonglong2 vv = *reinterpret_cast<const ulonglong2 *>(&sm.v[t][cg * 4]);
    uint64_t o0 = 0, o1 = 0;
#pragma unroll
    for (int i = 0; i < ROWS; i += 2) {
      const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(&sm.kk[t][rg * ROWS + i]);
      step(S[i][0], dmul2(kk.x, vv.x));
      step(S[i][1], dmul2(kk.x, vv.y));
      step(S[i + 1][0], dmul2(kk.y, vv.x));
      step(S[i + 1][1], dmul2(kk.y, vv.y));
      if (STEP || a.o) {
        const ulonglong2 qq = *reinterpret_cast<const ulonglong2 *>(&sm.qq[t][rg * ROWS + i]);
        o0 = dfma2(S[i][0], qq.x, o0);
        o1 = dfma2(S[i][1], qq.x, o1);
        o0 = dfma2(S[i + 1][0], qq.y, o0);
        o1 = dfma2(S[i + 1][1], qq.y, o1);
      }
    }
    if (STEP || a.o) *reinterpret_cast<ulonglong2 *>(&sm.part[t][rg][cg * 4]) = make_ulonglong2(o0, o1);
  };
  auto store_state = [&]() {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float2 x = dunpack2(S[i][0]), y = dunpack2(S[i][1]);
      *reinterpret_cast<float4 *>(st + static_cast<int64_t>(i) * a.d_v) = make_float4(x.x, x.y, y.x, y.y);
    }
  };
  auto outputs = [&](int t0, int cnt) {
    for (int i = tid; i < cnt * NCOL; i += NT) {
      const int t = i / NCOL, c = i % NCOL;
      float x = 0.f;
#pragma unroll
      for (int j = 0; j < RG; ++j) x += sm.part[t][j][c];
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
    if (tid == 0) sm.alpha[0] = expf(*gg);
    __syncthreads();
    token(0, std::false_type{});
    store_state();
    __syncthreads();
    outputs(0, 1);
  } else {
    if (n > 0) stage(0);
    for (int t0 = 0; t0 < n; t0 += TB) {
      const int cnt = min(TB, n - t0);
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
      for (int i = tid; i < cnt * DK; i += NT) {
        const int t = i / DK, c = i % DK;
        const float k = to_float<IO>(sm.raw_k[t][c]);
        sm.kk[t][c] = dpack2(k, k);
        if (a.o) {
          const float q = to_float<IO>(sm.raw_q[t][c]) * a.q_scale;
          sm.qq[t][c] = dpack2(q, q);
        }
      }
      for (int i = tid; i < cnt * NCOL; i += NT) sm.v[i / NCOL][i % NCOL] = to_float<IO>(sm.raw_v[i / NCOL][i % NCOL]);
      if (tid < cnt) {
        const float g = sm.raw_g[tid], d = expm1f(g), a1 = 1.f + d;
        const bool slow = n > kFew && g > -0.7f;
        sm.alpha[tid] = slow ? a1 : expf(g);
        sm.alpha_lo[tid] = slow ? d - (a1 - 1.f) : 0.f;
      }
      __syncthreads();
      if (t0 + TB < n) stage(t0 + TB);
      if (n > kFew)
        for (int t = 0; t < cnt; ++t) token(t, std::true_type{});
      else
        for (int t = 0; t < cnt; ++t) token(t, std::false_type{});
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
  // the widest part of the columns that still gives every SM a block or two
  if constexpr (DK <= 64)  // (128 x 128 values do not fit the registers of 128 threads beside what a token needs)
    if (a.d_v % 128 == 0 && units * (a.d_v / 128) >= 2 * 148) return launch_form<DK, 128, IO, OT>(a, stream);
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
