// Linear attention with a decay per head, chunked form on the tensor cores, for d_k = d_v = 128 and bf16 streams.
//
// With G_t the sum of the log-decays of a chunk up to its token t (log2 units here), S_0 the state at its start:
//   O   = q_scale (diag(e^G) Q S_0 + P V),   P_ti = e^{G_t - G_i} q_t . k_i for i <= t, else 0
//   S_C = e^{G_C} S_0 + Kw^T V,               Kw_i = e^{G_C - G_i} k_i
// Products, C = 64 tokens, everything transposed so that d_v is the M index (the accumulators' 128 lanes):
//   QK   Q K^T               -> P before its weights    smem x smem, M = 64
//   QS   S_0^T Q^T           -> outputs from the state   tmem x smem
//   PV   V^T P^T             -> outputs inside the chunk  tmem x smem   (only the rows a slice of i can reach)
//   KV   V^T Kw              -> what the chunk adds        tmem x smem   (Kw in three parts)
// V, K and Q are exact in bf16: Q and K are used as they land, V^T goes to tensor memory (the tensor core's reads of shared memory are
// what bounds the products: 128 x 64 x 16 takes 49 cycles with both operands there, 33 with one of them in tensor memory).
// A value in n parts of bf16 (x rounded, the rest rounded, ...) is good to 2^-8n.  What the fp32 state is summed from stays at fp32's
// precision: Kw is in three parts (in pairs the state of 256 tokens is off by 2.4e-6, in three parts by 3e-7).  On the way to the outputs P and
// S_0 are pairs, for bf16 outputs too: these are then off by their own rounding (0.0017) and nothing else, where one part takes them to
// 0.0023, 1.4 times as far, in 5 to 11 % less time.
//
// One thread block per SM walks over (request, layer, head) units, or over segments of long ones; roles of its warps:
//   0       looks up the units (and clears the states of those without tokens); TMA: tiles of K, Q, V, three chunks ahead
//   1, 3    issue the products: KV; QK, QS and PV (issue alone, at 60 to 100 cycles a product, filled one warp's time)
//   2       announces the chunks to all others: sums of log-decays (as pairs of fp32), weights, where its unit's state is
//   4 - 7   P: out of tensor memory, weighted, into its operand tiles
//   8 - 11  outputs
//   12 - 15 Kw
//   16 - 23 the state, in fp32 registers: a thread has 64 key channels of one column; V^T, which is
//           looked at there for values that are none
// The only chain from chunk to chunk is S <- e^{G_C} S + (KV), 64 packed multiply-adds per thread, and its bf16 parts on the way
// to QS; KV itself does not depend on the state.
// Bound: with every SM at work, power (the SM clock settles at 1.45 to 1.6 of 1.965 GHz), so fewer products and instructions count, not idle
// cycles; and the roles' code as a whole, which runs at an instruction per cycle and scheduler up to 32 KB and at a third of that
// beyond (unrolled to 142 KB, its warps waited for instructions 5.5 times as long as they issued them, at 61 KB 1.1 times); and what a unit
// costs beside its chunks, chiefly the exchange of the state between its last product and the next unit's first: 14.2 us for a unit of four
// chunks in a batch, where a chunk of a long request takes 2.5.
// Measured, 32 heads, bf16 outputs: 64 requests of 256 tokens x 4 layers 784 us (the bytes take 410 us at 6567 GB/s), 64 requests of 1 to
// 1023 tokens 386 us, one of 32,768 tokens 528 us.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "decay_common.cuh"
#include "tcgen05_util.cuh"

namespace {

using namespace tc5;

constexpr int C = 64, D = 128;
constexpr int kSms = 148;
constexpr int NS = 3, NS_V = 2;  // stages of K and Q; of V
constexpr int KSPLIT = 3, OSPLIT = 2;  // parts of Kw; of P and of the state on the way to the outputs
constexpr int RING = 4;  // chunks whose weights are kept, and units that are looked up ahead
constexpr int WARP_TMA = 0, WARP_MMA = 1, WARP_DECAY = 2, WARP_P = 4, WARP_O = 8, WARP_K = 12, WARP_S = 16, NWARP = 24;
// Registers of a thread, by groups of four warps: what the launch gives each (65,536 over all threads, in steps of 8), and how the roles
// share it out.
constexpr int REGS = 80, REGS_0 = 56, REGS_P = 72, REGS_O = 72, REGS_K = 72, REGS_S = 104;
static_assert(NWARP * 32 * REGS <= 65536 && REGS_0 + REGS_P + REGS_O + REGS_K + 2 * REGS_S <= NWARP / 4 * REGS);
constexpr int NT = NWARP * 32;
constexpr int kMaxSorted = 512;  // entries (requests x segments) that are taken longest first
constexpr uint32_t kMaxPolls = 1u << 22, kPollNs = 1000;  // a poll sleeps for up to that long: the warps that wait leave the issue slots to the others
constexpr uint32_t kStatusWords = kDecayStatusWords / 2;  // per launch: one word per thread block

constexpr uint32_t TILE = C * D * 2;  // 64 tokens x 128 channels: two blocks of [64 rows][128 bytes]
constexpr uint32_t BLOCK = TILE / 2;
constexpr uint32_t OFF_K = 0, OFF_Q = OFF_K + NS * TILE, OFF_V = OFF_Q + NS * TILE;
constexpr uint32_t OFF_KW = OFF_V + NS_V * TILE;  // [KSPLIT]
constexpr uint32_t OFF_PH = OFF_KW + KSPLIT * TILE, OFF_PL = OFF_PH + C * C * 2;
constexpr uint32_t OFF_O = OFF_PL + C * C * 2;  // [4 warps][64 tokens][32 columns] bf16 on their way out
constexpr uint32_t OFF_MISC = OFF_O + TILE;

constexpr uint32_t COL_D = 0, COL_SH = 128, COL_SL = 192, COL_P = 256, COL_OI = 320, COL_OT = 384, COL_V = 448;  // (V^T twice, by chunk parity)

struct alignas(16) Chunk {
  int32_t rows;          // its tokens; negative: there are no more chunks
  int32_t first, last;   // of its unit
  float all, all_lo;     // e^{G_C}, and what it is short of it
  float log;             // G_C
  const float *src;      // first: the unit's state; null: zero
  float *dst, *decay;    // last: where its new state goes, and (a segment's) its decay; null: nowhere
  int64_t out;           // its first output, in elements
  // weights (read in pairs)
  float ghi[C], glo[C];  // G_t = ghi + glo, ghi a multiple of 2^-6: differences of ghi are exact
  float w[C];            // e^{G_C - G_i} (behind the last token 1: those keys are left out where Kw is made)
  float eg[C];           // q_scale e^{G_t}
  // P's weights outside its diagonal blocks of 16 x 16 are products: with B the last token before t's block, e^{G_t - G_B} times
  // e^{G_B - G_i}, neither above 1
  float row[C];          // q_scale e^{G_t - G_B}
  float col[3][3 * 16];  // e^{G_B - G_i}, B = 15, 31, 47
  int32_t has_bad[8];    // V's columns of 16 hold values that are none:
  int32_t bad[D];        // the first token with one, per column (C: no such token)
};
// The states and tokens of one unit, or of one segment of it.
struct alignas(16) Item {
  int64_t state;   // offset of its state in floats
  int64_t tok0;    // its first token in the streams of the call
  int32_t unit, seg;
  int32_t n;       // tokens; negative: there are no more items
  int32_t head, k_head, lc;
  int32_t from;    // 0: starts from zero, 1: from its state, 2: from the joined state of its segment
  int32_t write;   // its state is written back
};

struct Misc {
  Item items[RING];
  uint64_t full_k[NS], full_q[NS], full_v[NS_V], empty_k[NS], empty_q[NS], empty_v[NS_V];
  uint64_t dec_full[RING], dec_empty[RING], item_full[RING], item_empty[RING];
  uint64_t bar_p, bar_s, bar_o[2], bar_d;        // tensor core: QK, QS, PV (by chunk parity), KV of a chunk have completed
  uint64_t bar_kw;                               // and the first half of KV
  uint64_t v_ready[2], k_ready[2], p_ready, s_ready;  // V^T (by chunk parity), the halves of Kw, P, the state are in place
  uint64_t o_free, d_free;                       // accumulators have been read
  uint64_t s_whole;                              // the state's warps are all through with a unit
  uint64_t drain[2];
  uint32_t tmem_base;
  volatile uint32_t abort_flag;
  Chunk ch[RING];
  uint16_t order[kMaxSorted];
};
constexpr uint32_t SMEM_BYTES = OFF_MISC + sizeof(Misc);
static_assert(SMEM_BYTES <= 227 * 1024);
static_assert(kMaxSorted * 4 <= TILE);

struct Split {
  int32_t nseg, seg_chunks;  // segments of a request, chunks of a segment (the last one takes what is left)
  int32_t phase;             // 0: requests are not split; 1: states of all segments but the last, from zero; 2: everything, from the joined states
  float *seg_state;          // [unit][nseg][D][D]
  float *seg_decay;          // [unit][nseg]
  uint32_t *status;          // [kStatusWords] of this launch
};

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void arrive_warp(uint64_t *bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}
// Bounded wait; once one has run out, no wait of this thread block lasts longer than one poll.  Written as the smallest loop there is: it is
// inlined at some thirty places, and the roles' code together has to stay within reach of the instruction caches.
__device__ __forceinline__ void wait_bar(uint64_t *bar, uint32_t parity, Misc *m) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b32 n, f;\n\t"
      "mov.b32 n, 0;\n"
      "POLL:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%0], %1, %4;\n\t"
      "@p bra DONE;\n\t"
      "ld.volatile.shared.b32 f, [%2];\n\t"
      "add.u32 n, n, 1;\n\t"
      "setp.ne.b32 q, n, %3;\n\t"
      "setp.eq.and.b32 p, f, 0, q;\n\t"
      "@p bra POLL;\n\t"
      "st.volatile.shared.b32 [%2], 1;\n"
      "DONE:\n\t}" ::"r"(smem_u32(bar)),
      "r"(parity), "r"(smem_u32(const_cast<uint32_t *>(&m->abort_flag))), "n"(kMaxPolls), "r"(kPollNs)
      : "memory");
}
__device__ __forceinline__ int uni(int x) { return __shfl_sync(0xffffffffu, x, 0); }

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// (x, y) rounded to bf16; what is left of them stays in xy
__device__ __forceinline__ uint32_t take_bf16x2(uint64_t &xy) {
  const float2 v = dunpack2(xy);
  const uint32_t b = bf16x2(v.x, v.y);
  xy = dsub2(xy, dpack2(bf_lo(b), bf_hi(b)));
  return b;
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t &r0, uint32_t &r1, uint32_t &r2, uint32_t &r3, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Which of N buffers, and the phase of its barriers, chunk by chunk.
template <int N>
struct Ring {
  uint32_t i = 0, ph = 0;
  __device__ __forceinline__ void step() {
    if (++i == N) {
      i = 0;
      ph ^= 1u;
    }
  }
};

__device__ __forceinline__ int chunks_of(int n) { return (n + C - 1) / C; }
// Segments that a request of `chunks` chunks really has.
__device__ __forceinline__ int segments_of(const Split &sp, int chunks) {
  return sp.nseg == 1 ? 1 : min(sp.nseg, max((chunks + sp.seg_chunks - 1) / sp.seg_chunks, 1));
}
// Chunks of entry `e` = (request, segment) that this launch runs.
__device__ __forceinline__ int entry_chunks(const DascDecayArgs &a, const Split &sp, int e) {
  const int r = e / sp.nseg, s = e - r * sp.nseg;
  if (a.req_idx[r] < 0) return 0;
  const int chunks = chunks_of(decay_range(a, r).n), segs = segments_of(sp, chunks);
  if (s >= segs || (sp.phase == 1 && s == segs - 1)) return 0;
  return s == segs - 1 ? chunks - s * sp.seg_chunks : sp.seg_chunks;
}

// This thread block's k-th item: every gridDim.x-th, there and back, so that each block gets long and short ones.  False: nothing to do
// there; x.n < 0: there is no such item.
__device__ __forceinline__ bool item_at(const DascDecayArgs &a, const Split &sp, const Misc *m, bool sorted, uint32_t k, Item &x) {
  const uint32_t per_entry = static_cast<uint32_t>(a.n_layers_in_call) * a.H_v, total = per_entry * a.n_req * sp.nseg;
  const uint64_t idx64 = static_cast<uint64_t>(k) * gridDim.x + ((k & 1) ? gridDim.x - 1u - blockIdx.x : blockIdx.x);
  x.n = -1;
  if (idx64 >= total) return true;
  const uint32_t idx = static_cast<uint32_t>(idx64);
  int e = static_cast<int>(idx / per_entry);
  const int rest = static_cast<int>(idx - e * per_entry);
  if (sorted) e = m->order[e];
  const int r = e / sp.nseg, s = e - r * sp.nseg;
  const int req = a.req_idx[r];
  if (req < 0) return false;
  const DecayRange range = decay_range(a, r);
  const int chunks = chunks_of(range.n), segs = segments_of(sp, chunks);
  const bool last = s == segs - 1;
  if (s >= segs || (sp.phase == 1 && last)) return false;
  x.lc = rest / a.H_v;
  x.head = rest - x.lc * a.H_v;
  x.k_head = x.head / (a.H_v / a.H_k);
  const int layer = a.layer_begin + x.lc;
  const bool merge = a.mode == DASC_DECAY_SCRATCH_MERGE_LOCAL;
  const bool write = a.mode != DASC_DECAY_SCORE && !(merge && a.row_keep[layer * a.rows_per_layer + x.head * D]);
  const bool zero = merge || (a.from_zero && a.from_zero[r] != 0);
  if ((!write && !a.o) || (chunks == 0 && !(write && zero))) return false;
  x.from = sp.phase == 1 ? 0 : sp.phase == 2 && segs > 1 ? 2 : zero ? 0 : 1;
  x.write = last && write;
  x.seg = s;
  x.unit = (r * a.n_layers_in_call + x.lc) * a.H_v + x.head;
  x.tok0 = static_cast<int64_t>(x.lc) * a.total_tokens + range.begin + static_cast<int64_t>(s) * sp.seg_chunks * C;
  x.n = last ? range.n - s * sp.seg_chunks * C : sp.seg_chunks * C;
  x.state = req * a.req_stride + layer * a.layer_stride + static_cast<int64_t>(x.head) * (D * D);
  return true;
}

// Where an item's state is read.
__device__ __forceinline__ const float *state_of(const DascDecayArgs &a, const Split &sp, const Item &x) {
  return x.from == 2 ? sp.seg_state + (static_cast<int64_t>(x.unit) * sp.nseg + x.seg) * (D * D) : a.state + x.state;
}

template <bool WITH_O, typename OT>
__global__ void __launch_bounds__(NT, 1) decay_chunked_kernel(const __grid_constant__ DascDecayArgs a, const __grid_constant__ Split sp,
                                                             const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                                                             const __grid_constant__ CUtensorMap tmap_v) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  Misc *const m = reinterpret_cast<Misc *>(smem + OFF_MISC);
  const int tid = threadIdx.x, warp = uni(tid >> 5), lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&m->full_k[i], 1);
      mbar_init(&m->full_q[i], 1);
      mbar_init(&m->empty_k[i], WITH_O ? 5 : 4);  // Kw's warps; QK
      mbar_init(&m->empty_q[i], 1);
    }
    for (int i = 0; i < NS_V; ++i) {
      mbar_init(&m->full_v[i], 1);
      mbar_init(&m->empty_v[i], 8);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&m->bar_o[i], 1);
      mbar_init(&m->v_ready[i], 8);
      mbar_init(&m->k_ready[i], 4);
    }
    mbar_init(&m->bar_kw, 1);
    for (int i = 0; i < RING; ++i) {
      mbar_init(&m->dec_full[i], 1);
      mbar_init(&m->dec_empty[i], WITH_O ? 22 : 13);
      mbar_init(&m->item_full[i], 1);
      mbar_init(&m->item_empty[i], 1);
    }
    mbar_init(&m->bar_p, 1);
    mbar_init(&m->bar_s, 1);
    mbar_init(&m->bar_d, 1);
    mbar_init(&m->p_ready, 4);
    mbar_init(&m->s_ready, 8);
    mbar_init(&m->o_free, 4);
    mbar_init(&m->d_free, 8);
    mbar_init(&m->s_whole, 8);
    mbar_init(&m->drain[0], 1);
    mbar_init(&m->drain[1], 1);
    m->abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == WARP_MMA) {
    tmem_alloc(&m->tmem_base, 512);
    tmem_relinquish();
  }
  stream_order_wait();
  // the segments' states are not to be had where a wait of their launch has run out
  const bool failed = sp.phase == 2 && __syncthreads_or(tid < static_cast<int>(kStatusWords) && sp.status[kStatusWords + tid] != 0);
  const int entries = a.n_req * sp.nseg;
  const bool sorted = entries > 1 && entries <= kMaxSorted;
  if (sorted) {  // longest first, ties in their order
    int32_t *const key = reinterpret_cast<int32_t *>(smem);
    for (int e = tid; e < (entries + 3) / 4 * 4; e += NT) key[e] = e < entries ? entry_chunks(a, sp, e) : -1;
    __syncthreads();
    for (int e = tid; e < entries; e += NT) {
      const int own = key[e];
      int rank = 0;
#pragma unroll 1
      for (int j = 0; j < entries; j += 4) {
        const int4 o = *reinterpret_cast<const int4 *>(key + j);
        rank += (o.x > own || (o.x == own && j < e)) + (o.y > own || (o.y == own && j + 1 < e)) + (o.z > own || (o.z == own && j + 2 < e)) +
                (o.w > own || (o.w == own && j + 3 < e));
      }
      m->order[rank] = static_cast<uint16_t>(e);
    }
    fence_smem_to_async();  // (tiles land where the keys were)
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = static_cast<uint32_t>(uni(static_cast<int>(m->tmem_base)));

  const auto phase2 = [](int i) { return static_cast<uint32_t>(i) >> 1 & 1u; };  // of what there are two of, by chunk parity
  const auto slot = [](int i) { return static_cast<uint32_t>(i) % RING; };
  const auto slot_phase = [](int i) { return static_cast<uint32_t>(i) / RING & 1u; };
  // Chunk n, once it has been announced; false: there are no more, or a wait has run out.
  const auto there = [&](int n) {
    wait_bar(&m->dec_full[slot(n)], slot_phase(n), m);
    return m->abort_flag == 0 && m->ch[slot(n)].rows >= 0;
  };
  // All roles count chunks, n: buffers and barrier phases go by it.

  if (failed) {
    if (tid == 0) m->abort_flag = 1;
  } else if (warp < WARP_P) {
    regs_down<REGS_0>();
    if (warp == WARP_TMA) {
      // The next item is looked up, and its state brought into L2, behind the first loads of this one.
      bool ask = true;
      uint32_t k = 0;
      int it = 0, n = 0, c = 0, chunks = 0;
      Ring<NS> kq;
      Item x, next;
#pragma unroll 1
      for (;;) {
        if (ask) {
          ask = false;
#pragma unroll 1
          for (;;) {
            while (!item_at(a, sp, m, sorted, k++, next)) {
            }
            if (next.n != 0) break;
            float4 *const st = reinterpret_cast<float4 *>(a.state + next.state);  // no tokens: its new state is zero
#pragma unroll 1
            for (int i = lane; i < D * D / 4; i += 32) st[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
          if (it >= RING) wait_bar(&m->item_empty[it % RING], (static_cast<uint32_t>(it) / RING & 1u) ^ 1u, m);
          if (lane == 0) m->items[it % RING] = next;
          if (next.n > 0 && next.from != 0 && lane < 4) bulk_prefetch(state_of(a, sp, next) + lane * (D * D / 4), D * D);
          arrive_warp(&m->item_full[it % RING], lane);
          ++it;
        }
        if (c == chunks) {
          x = next;
          if (x.n < 0) break;
          chunks = chunks_of(x.n);
          c = 0;
          ask = true;
        }
        const int32_t z = static_cast<int32_t>(x.tok0 + c * C);
#pragma unroll 1
        for (int t = 0; t < (WITH_O ? 3 : 2); ++t) {  // V, K, Q
          const uint32_t st = t == 0 ? n & 1u : kq.i, ph = t == 0 ? phase2(n) : kq.ph;
          uint64_t *const full = (t == 0 ? m->full_v : t == 1 ? m->full_k : m->full_q) + st;
          if (n >= (t == 0 ? NS_V : NS)) wait_bar((t == 0 ? m->empty_v : t == 1 ? m->empty_k : m->empty_q) + st, ph ^ 1u, m);
          if (lane == 0) {
            const CUtensorMap *const map = t == 0 ? &tmap_v : t == 1 ? &tmap_k : &tmap_q;
            const uint32_t to = sbase + (t == 0 ? OFF_V : t == 1 ? OFF_K : OFF_Q) + st * TILE;
            const int head = t == 0 ? x.head : x.k_head;
            mbar_expect_tx(full, TILE);
            tma_load_3d(to, map, 0, head, z, full);
            tma_load_3d(to + BLOCK, map, 64, head, z, full);
          }
          if (uni(m->abort_flag)) break;
        }
        if (uni(m->abort_flag)) break;
        kq.step();
        ++c;
        ++n;
      }
      // Copies in flight land before the block ends, whoever has given up waiting for them.  After a time-out, which tiles have been
      // asked for is not known any more: a barrier that is not in use lets the bound on the polls run out.
      const bool sure = uni(m->abort_flag) == 0;
      const auto land = [&](uint64_t *bar, uint32_t phase) {
#pragma unroll 1
        for (uint32_t p = 0; p < (sure ? kMaxPolls : kMaxPolls >> 8) && !mbar_try_wait(bar, phase); ++p) {
        }
      };
#pragma unroll 1
      for (int i = max(n - NS, 0); i < (sure ? n : n + 1); ++i) {
        const uint32_t st = static_cast<uint32_t>(i) % NS, ph = static_cast<uint32_t>(i) / NS & 1u;
        if (i >= n - NS_V) land(&m->full_v[i & 1], phase2(i));
        land(&m->full_k[st], ph);
        if (WITH_O) land(&m->full_q[st], ph);
      }
    } else if (warp == WARP_DECAY) {
      int n = 0;
#pragma unroll 1
      for (int it = 0;; ++it) {
        wait_bar(&m->item_full[it % RING], static_cast<uint32_t>(it) / RING & 1u, m);
        if (uni(m->abort_flag)) break;
        const Item x = m->items[it % RING];
        arrive_warp(&m->item_empty[it % RING], lane);
        const float *g = (a.g_per_head ? a.g + x.lc * a.H_v + x.head : a.g + (x.tok0 + 2 * lane) * a.H_v + x.head);
        const int64_t stride = a.g_per_head ? 0 : a.H_v;
        const int chunks = x.n < 0 ? 1 : chunks_of(x.n);
        float next[2];
        next[0] = 2 * lane < x.n ? g[0] : 0.f;
        next[1] = 2 * lane + 1 < x.n ? g[stride] : 0.f;
#pragma unroll 1
        for (int c = 0; c < chunks; ++c, ++n) {
          const int left = x.n - c * C;
          float cur[2] = {next[0], next[1]};
          g += C * stride;
          if (C + 2 * lane < left) next[0] = g[0];
          if (C + 2 * lane + 1 < left) next[1] = g[stride];
          if (n >= RING) wait_bar(&m->dec_empty[slot(n)], slot_phase(n) ^ 1u, m);
          Chunk &w = m->ch[slot(n)];
          if (lane == 0) {
            w.rows = x.n < 0 ? -1 : min(left, C);
            w.first = c == 0;
            w.last = c == chunks - 1;
            w.src = x.from != 0 ? state_of(a, sp, x) : nullptr;
            const int64_t at = static_cast<int64_t>(x.unit) * sp.nseg + x.seg;
            w.dst = sp.phase == 1 ? sp.seg_state + (at + 1) * (D * D) : x.write ? a.state + x.state : nullptr;
            w.decay = sp.phase == 1 ? sp.seg_decay + at : nullptr;
            w.out = ((x.tok0 + c * C) * a.H_v + x.head) * D;
          }
          // Log-decays in log2 units as pairs: hi a multiple of 2^-6, so that sums of 64 and their differences are exact (at -1400,
          // 2020 in log2 units, a token forgets everything, and is clamped there), lo the rest, at most 2^-7 each.
          float hi[2], lo[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            constexpr float L = 1.4426950408889634f, L_LO = static_cast<float>(1.4426950408889634 - static_cast<double>(L));
            const float y = 2 * lane + j < left ? (cur[j] < -1400.f ? -1400.f : cur[j]) : 0.f;
            const float p = y * L;
            hi[j] = rintf(p * 64.f) * (1.f / 64.f);
            lo[j] = (p - hi[j]) + fmaf(y, L, -p) + y * L_LO;
          }
          float sum_hi = hi[0] + hi[1], sum_lo = lo[0] + lo[1];
#pragma unroll 1
          for (int d = 1; d < 32; d <<= 1) {
            const float y = __shfl_up_sync(0xffffffffu, sum_hi, d), z = __shfl_up_sync(0xffffffffu, sum_lo, d);
            if (lane >= d) {
              sum_hi += y;
              sum_lo += z;
            }
          }
          // sums up to this lane's tokens: gh + gl
          const float2 gh = make_float2(sum_hi - hi[1], sum_hi), gl = make_float2(sum_lo - lo[1], sum_lo);
          const auto below = [&](float *at, float h, float l) {  // e^{h + l - G}
            reinterpret_cast<float2 *>(at)[lane] = make_float2(ex2f((h - gh.x) + (l - gl.x)), ex2f((h - gh.y) + (l - gl.y)));
          };
          const auto above = [&](float *at, float h, float l) {  // q_scale e^{G - h - l}
            reinterpret_cast<float2 *>(at)[lane] =
                make_float2(a.q_scale * ex2f((gh.x - h) + (gl.x - l)), a.q_scale * ex2f((gh.y - h) + (gl.y - l)));
          };
          const float all_hi = __shfl_sync(0xffffffffu, sum_hi, 31), all_lo = __shfl_sync(0xffffffffu, sum_lo, 31);
          below(w.w, all_hi, all_lo);
          if (lane == 0) {
            // The state is multiplied by e^{G_C} once per chunk: half an ulp, the same every time where the decay is, is 5e-6 of a state that
            // lasts 10^4 tokens.  Slow decay is 1 + d with d good to its own last bits, and the rest of the sum kept.
            w.log = all_hi + all_lo;
            float f = ex2f(w.log), f_lo = 0.f;
            if (w.log > -1.f) {
              const float d = expm1f(w.log * 0.6931471805599453f);
              f = 1.f + d;
              f_lo = d - (f - 1.f);
            }
            w.all = f;
            w.all_lo = f_lo;
          }
          if (WITH_O) {
            reinterpret_cast<float2 *>(w.ghi)[lane] = gh;
            reinterpret_cast<float2 *>(w.glo)[lane] = gl;
            above(w.eg, 0.f, 0.f);
            const int block = lane >> 3;  // B: the last token before this lane's block of 16
            const float bh = __shfl_sync(0xffffffffu, sum_hi, block * 8 - 1), bl = __shfl_sync(0xffffffffu, sum_lo, block * 8 - 1);
            above(w.row, block == 0 ? 0.f : bh, block == 0 ? 0.f : bl);
#pragma unroll 1
            for (int b = 0; b < 3; ++b) {
              const float h = __shfl_sync(0xffffffffu, sum_hi, 8 * b + 7), l = __shfl_sync(0xffffffffu, sum_lo, 8 * b + 7);
              if (block <= b) below(w.col[b], h, l);
            }
          }
          arrive_warp(&m->dec_full[slot(n)], lane);
        }
        if (x.n < 0) break;
      }
    } else {
      const auto gave_up = [&]() { return uni(m->abort_flag) != 0; };  // (one answer for the whole warp)
      const auto next = [&](int n) {  // is there a chunk n?
        const bool yes = uni(there(n));
        if (lane == 0) mbar_arrive(&m->dec_empty[slot(n)]);
        return yes;
      };
      if (warp == WARP_MMA) {
        constexpr uint32_t ID_KV = idesc_bf16(128, 128, false, true);
        // Test hook: a first, short wait for operands that cannot be there yet.
        if (a.poll_limit_first_wait) {
          bool done = false;
          for (uint32_t i = 0; i < a.poll_limit_first_wait && !done; ++i) done = mbar_test_wait(&m->k_ready[0], 0);
          if (!done) m->abort_flag = 1;
        }
#pragma unroll 1
        for (int n = 0; next(n); ++n) {
          const uint32_t par = n & 1u;
          wait_bar(&m->v_ready[par], phase2(n), m);
          if (n > 0) wait_bar(&m->d_free, par ^ 1u, m);
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {  // 32 tokens each, so that the next Kw can follow behind
            wait_bar(&m->k_ready[half], par, m);
            tc_fence_after_sync();
            if (gave_up()) break;
            if (elect_one()) {
              const uint32_t v = tm + COL_V + par * 32 + half * 16, kw = desc_lo_mn(sbase + OFF_KW, BLOCK) + half * (2 * 2048 >> 4);
              if (half == 0)
                mma16_ts<false>(tm + COL_D, v, kw, ID_KV);
              else
                mma16_ts<true>(tm + COL_D, v, kw, ID_KV);
#pragma unroll
              for (int i = 1; i < 2 * KSPLIT; ++i)
                mma16_ts<true>(tm + COL_D, v + (i & 1) * 8, kw + (((i >> 1) * TILE + (i & 1) * 2048) >> 4), ID_KV);
              mma_commit(half == 0 ? &m->bar_kw : &m->bar_d);
            }
            __syncwarp();
          }
        }
      } else if constexpr (WITH_O) {
        constexpr uint32_t ID_QK = idesc_bf16(64, 64), ID_QS = idesc_bf16(128, 64);
        Ring<NS> kq;  // of the chunk QK is for
        uint32_t q_before = 0;
        bool more = next(0);
        // QK of chunk n + 1 goes ahead of PV of chunk n: its accumulator has been read, and the next P is waited for longest
#pragma unroll 1
        for (int n = -1;; ++n) {
          const uint32_t par = n & 1u;
          if (n >= 0) {
            // QS
            wait_bar(&m->s_ready, par, m);
            if (n > 0) wait_bar(&m->o_free, par ^ 1u, m);
            tc_fence_after_sync();
            if (gave_up()) break;
            if (elect_one()) {
              const uint32_t q = desc_lo_k(sbase + OFF_Q) + q_before * (TILE >> 4);
              const uint32_t d = tm + COL_OI;
              mma16_ts<false>(d, tm + COL_SH, q, ID_QS);
#pragma unroll
              for (int i = 1; i < 8 * OSPLIT; ++i) {
                const int kk = i & 7;
                mma16_ts<true>(d, tm + (i < 8 ? COL_SH : COL_SL) + kk * 8, q + (((kk >> 2) * BLOCK + (kk & 3) * 32) >> 4), ID_QS);
              }
              mma_commit(&m->bar_s);
              mma_commit(&m->empty_q[q_before]);
            }
            __syncwarp();
            more = next(n + 1);
            wait_bar(&m->p_ready, par, m);
            wait_bar(&m->v_ready[par], phase2(n), m);
          }
          if (more) {
            wait_bar(&m->full_k[kq.i], kq.ph, m);
            wait_bar(&m->full_q[kq.i], kq.ph, m);
          }
          tc_fence_after_sync();
          if (gave_up()) break;
          if (elect_one()) {
            if (more) {
              const uint32_t q = desc_lo_k(sbase + OFF_Q) + kq.i * (TILE >> 4), k = desc_lo_k(sbase + OFF_K) + kq.i * (TILE >> 4);
              mma16_ss<false>(tm + COL_P, q, k, ID_QK);
#pragma unroll
              for (int kk = 1; kk < 8; ++kk) {
                const uint32_t o = ((kk >> 2) * BLOCK + (kk & 3) * 32) >> 4;
                mma16_ss<true>(tm + COL_P, q + o, k + o, ID_QK);
              }
              mma_commit(&m->bar_p);
              mma_commit(&m->empty_k[kq.i]);
            }
            if (n >= 0) {
              // PV: tokens 16 s ... 16 s + 15 reach the rows from 16 s on
              const uint32_t v = tm + COL_V + par * 32, p = desc_lo_k(sbase + OFF_PH);
              mma16_ts<false>(tm + COL_OT, v, p, idesc_bf16(128, 64));
#pragma unroll
              for (int i = 1; i < 4 * OSPLIT; ++i) {
                const uint32_t s = i & 3;
                mma16_ts<true>(tm + COL_OT + 16 * s, v + 8 * s, p + (((i < 4 ? 0 : OFF_PL - OFF_PH) + s * 2048 + s * 32) >> 4), idesc_bf16(128, 64 - 16 * s));
              }
              mma_commit(&m->bar_o[par]);
            }
          }
          __syncwarp();
          if (!more) break;
          q_before = kq.i;
          kq.step();
        }
      }
      // products in flight end before their memory is given back, whoever has given up waiting for them
      uint64_t *const drain = &m->drain[warp == WARP_MMA ? 0 : 1];
      if (elect_one()) mma_commit(drain);
      __syncwarp();
#pragma unroll 1
      for (uint32_t p = 0; p < kMaxPolls && !mbar_try_wait(drain, 0); ++p) {
      }
    }
  } else if (warp < WARP_O) {
    // ---- P ----
    regs_down<REGS_P>();
    if constexpr (WITH_O) {
      const int quad = warp & 3, g = lane >> 2, tig = lane & 3;
      const uint32_t tp = tm + (static_cast<uint32_t>(quad * 32) << 16) + COL_P;
      const int t0 = quad * 16 + g, t1 = t0 + 8;  // this thread's rows; columns 16 s + 2 tig, + 1, + 8, + 9
      unsigned char *const ps = smem + OFF_PH + t0 * 128 + tig * 4;
#pragma unroll 1
      for (int n = 0; uni(there(n)); ++n) {
        const Chunk &w = m->ch[slot(n)];
        wait_bar(&m->bar_p, n & 1u, m);
        if (n > 0) wait_bar(&m->bar_o[(n - 1) & 1], phase2(n - 1), m);  // PV of the chunk before has read its P
        tc_fence_after_sync();
#pragma unroll 1
        for (int s = 0; s <= quad; ++s) {
          uint32_t p[8];
          tmem_ld_16x256b(tp + 16 * s, p);
          uint64_t f[4];  // weights of p's pairs: rows t0, t1, columns + 0, 1; the same rows, columns + 8, 9
          if (s < quad) {
            const float r0 = w.row[t0], r1 = w.row[t1];
            const uint64_t rr0 = dpack2(r0, r0), rr1 = dpack2(r1, r1);
            const uint64_t *const col = reinterpret_cast<const uint64_t *>(&w.col[quad - 1][16 * s]) + tig;
            f[0] = dmul2(rr0, col[0]);
            f[1] = dmul2(rr1, col[0]);
            f[2] = dmul2(rr0, col[4]);
            f[3] = dmul2(rr1, col[4]);
            tmem_ld_wait();
          } else {
            tmem_ld_wait();
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const int t = b & 1 ? t1 : t0, i = 16 * s + (b >> 1) * 8 + 2 * tig;
              const float2 hi = *reinterpret_cast<const float2 *>(&w.ghi[i]), lo = *reinterpret_cast<const float2 *>(&w.glo[i]);
              const float h = w.ghi[t], l = w.glo[t];
              f[b] = dpack2(a.q_scale * ex2f((h - hi.x) + (l - lo.x)), a.q_scale * ex2f((h - hi.y) + (l - lo.y)));
              // (masked places may hold anything, and above the diagonal weights may not be finite)
              if (i > t) p[2 * b] = 0;
              if (i + 1 > t) p[2 * b + 1] = 0;
              const float2 y = dunpack2(f[b]);
              f[b] = dpack2(i > t ? 0.f : y.x, i + 1 > t ? 0.f : y.y);
            }
          }
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            uint64_t rest = dmul2(dpack2(__uint_as_float(p[2 * b]), __uint_as_float(p[2 * b + 1])), f[b]);
            unsigned char *const to = ps + (((2 * s + (b >> 1)) ^ (t0 & 7)) << 4) + (b & 1) * (8 * 128);
#pragma unroll
            for (int part = 0; part < OSPLIT; ++part) *reinterpret_cast<uint32_t *>(to + part * (OFF_PL - OFF_PH)) = take_bf16x2(rest);
          }
        }
        fence_smem_to_async();
        tc_fence_before_sync();
        arrive_warp(&m->p_ready, lane);
        if (lane == 0) mbar_arrive(&m->dec_empty[slot(n)]);
      }
    }
  } else if (warp < WARP_K) {
    // ---- outputs ----
    regs_down<REGS_O>();
    if constexpr (WITH_O) {
      const int quad = warp & 3, g = lane >> 2, tig = lane & 3;
      const uint32_t tl = tm + (static_cast<uint32_t>(quad * 32) << 16);
      const int64_t v_stride = static_cast<int64_t>(a.H_v) * D;
      unsigned char *const ost = smem + OFF_O + quad * 4096;
#pragma unroll 1
      for (int n = 0; uni(there(n)); ++n) {
        const Chunk &w = m->ch[slot(n)];
        const int rows = w.rows;
        OT *const o = static_cast<OT *>(a.o) + w.out + quad * 32;
        wait_bar(&m->bar_o[n & 1], phase2(n), m);
        if (uni(m->abort_flag)) break;
        tc_fence_after_sync();
#pragma unroll 1
        for (int part = 0; part < 4; ++part) {  // 16 columns of d_v (part & 1), 32 tokens (part >> 1)
          const int half = part & 1, tb = part >> 1;
          uint32_t oi[16], ot[16];
          const uint32_t at = tl + (static_cast<uint32_t>(half * 16) << 16) + tb * 32;
          tmem_ld_16x256b(at + COL_OI, oi);
          tmem_ld_16x256b(at + COL_OT, ot);
          tmem_ld_wait();
          if (part == 3) {
            tc_fence_before_sync();
            arrive_warp(&m->o_free, lane);
          }
          const int v0 = half * 16 + g;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = tb * 32 + 8 * j + 2 * tig;
            const uint64_t e = *reinterpret_cast<const uint64_t *>(&w.eg[t]);
            const auto pair = [](uint32_t x, uint32_t y) { return dpack2(__uint_as_float(x), __uint_as_float(y)); };
            const float2 y0 = dunpack2(dfma2(e, pair(oi[4 * j], oi[4 * j + 1]), pair(ot[4 * j], ot[4 * j + 1])));
            const float2 y1 = dunpack2(dfma2(e, pair(oi[4 * j + 2], oi[4 * j + 3]), pair(ot[4 * j + 2], ot[4 * j + 3])));
            if constexpr (sizeof(OT) == 2) {
              ot[2 * j] = bf16x2(y0.x, y0.y);
              ot[2 * j + 1] = bf16x2(y1.x, y1.y);
            } else {
              OT *const p = o + t * v_stride + v0;
              if (t < rows) {
                p[0] = y0.x;
                p[8] = y1.x;
              }
              if (t + 1 < rows) {
                p[v_stride] = y0.y;
                p[v_stride + 8] = y1.y;
              }
            }
          }
          if constexpr (sizeof(OT) == 2) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              const int t = tb * 32 + 8 * (j + (lane >> 4)) + (lane & 7), ch = half * 2 + (lane >> 3 & 1);
              stmatrix_x4_trans(smem_u32(ost) + t * 64 + ((ch ^ (t >> 1 & 3)) << 4), ot[2 * j], ot[2 * j + 1], ot[2 * j + 2], ot[2 * j + 3]);
            }
          }
        }
        __syncwarp();
        if constexpr (sizeof(OT) == 2) {
#pragma unroll 4
          for (int i8 = 0; i8 < 8; ++i8) {
            const int t = i8 * 8 + (lane >> 2), ch = lane & 3;
            const uint4 y = *reinterpret_cast<const uint4 *>(ost + t * 64 + ((ch ^ (t >> 1 & 3)) << 4));
            if (t < rows) *reinterpret_cast<uint4 *>(o + t * v_stride + ch * 8) = y;
          }
          __syncwarp();
        }
        if (w.has_bad[quad * 2] | w.has_bad[quad * 2 + 1]) {  // a lane per column, over what the warp has just stored
          const OT nan = static_cast<OT>(__int_as_float(0x7fffffff));
#pragma unroll 1
          for (int t = w.has_bad[quad * 2 + (lane >> 4)] ? w.bad[quad * 32 + lane] : C; t < rows; ++t) o[t * v_stride + lane] = nan;
        }
        arrive_warp(&m->dec_empty[slot(n)], lane);
      }
    }
  } else if (warp < WARP_S) {
    // ---- Kw ----
    regs_down<REGS_K>();
    const int kt = tid - WARP_K * 32;
    Ring<NS> kq;
#pragma unroll 1
    for (int n = 0; uni(there(n)); ++n, kq.step()) {
      const Chunk &w = m->ch[slot(n)];
      const int rows = w.rows;
      wait_bar(&m->full_k[kq.i], kq.ph, m);
      const unsigned char *const kr = smem + OFF_K + kq.i * TILE + kt * 16;
      unsigned char *const kw = smem + OFF_KW + kt * 16;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {  // 32 tokens at a time
        if (n > 0) wait_bar(half == 0 ? &m->bar_kw : &m->bar_d, (n - 1) & 1u, m);  // KV of the chunk before has read this half
#pragma unroll 2
        for (int i = 0; i < 4; ++i) {
          const int row = (kt >> 3) + (half * 2 + (i & 1)) * 16;
          const uint32_t at = ((i >> 1) * 4 + half * 2 + (i & 1)) * 2048;
          const float f = w.w[row];
          const uint64_t ff = dpack2(f, f);
          uint4 y = *reinterpret_cast<const uint4 *>(kr + at);
          if (row >= rows) y = make_uint4(0u, 0u, 0u, 0u);
          uint64_t rest[4] = {dmul2(dpack2(bf_lo(y.x), bf_hi(y.x)), ff), dmul2(dpack2(bf_lo(y.y), bf_hi(y.y)), ff),
                              dmul2(dpack2(bf_lo(y.z), bf_hi(y.z)), ff), dmul2(dpack2(bf_lo(y.w), bf_hi(y.w)), ff)};
#pragma unroll
          for (int part = 0; part < KSPLIT; ++part) {
            uint4 b;
            b.x = take_bf16x2(rest[0]);
            b.y = take_bf16x2(rest[1]);
            b.z = take_bf16x2(rest[2]);
            b.w = take_bf16x2(rest[3]);
            *reinterpret_cast<uint4 *>(kw + part * TILE + at) = b;
          }
        }
        fence_smem_to_async();
        arrive_warp(&m->k_ready[half], lane);
      }
      if (lane == 0) {
        mbar_arrive(&m->empty_k[kq.i]);
        mbar_arrive(&m->dec_empty[slot(n)]);
      }
    }
  } else {
    // ---- the state ----
    regs_up<REGS_S>();
    const int quad = warp & 3, half = (warp - WARP_S) >> 2;
    const uint32_t tl = tm + (static_cast<uint32_t>(quad * 32) << 16);
    const int v = quad * 32 + lane, k0 = half * 64;
    uint64_t S[32];
    float decay = 0.f;  // the unit's, in log2 units
    uint32_t units = 0;
    // V^T of chunk n, if there is one.
    const auto values = [&](int n) {
      if (!uni(there(n))) return false;
      Chunk &w = m->ch[slot(n)];
      const uint32_t par = n & 1u;
      const int rows = w.rows;
      // This warp's 16 columns.  A value that is none would reach every row of its column through products with weights that are
      // zero, so it is taken out and remembered; 0 * x + sum is NaN from the first of them on.
      wait_bar(&m->full_v[par], phase2(n), m);
      // the products of the chunk before the last have read their V^T (their KV has been waited for)
      if (WITH_O && n > 1) wait_bar(&m->bar_o[par], phase2(n - 2), m);
      tc_fence_after_sync();
      {
        unsigned char *const vt = smem + OFF_V + par * TILE + (quad >> 1) * BLOCK;
        const int ch = (quad & 1) * 4 + half * 2;  // two of the 16-byte places of a row
        if (rows < C) {  // nothing from behind the last token
#pragma unroll 1
          for (int t = rows + (lane >> 1); t < C; t += 16)
            *reinterpret_cast<uint4 *>(vt + t * 128 + (((ch + (lane & 1)) ^ (t & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          fence_smem_to_async();  // (the next tile lands here)
          __syncwarp();
        }
        bool looked = false;
        uint32_t r[16];
#pragma unroll 1
        for (;;) {
          __nv_bfloat162 probe = __floats2bfloat162_rn(0.f, 0.f);
          const __nv_bfloat162 zero2 = probe;
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const int t = 8 * (j + (lane >> 4)) + (lane & 7);
            ldmatrix_x4_trans(r[2 * j], r[2 * j + 1], r[2 * j + 2], r[2 * j + 3],
                              smem_u32(vt) + t * 128 + (((ch + (lane >> 3 & 1)) ^ (t & 7)) << 4));
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) probe = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&r[j]), zero2, probe);
          const bool none = __isnan(__low2float(probe)) || __isnan(__high2float(probe));
          if (!__any_sync(0xffffffffu, none) || looked) break;
          looked = true;
          if (lane < 16) {
            int first = C;  // of this lane's column
#pragma unroll 1
            for (int t = rows - 1; t >= 0; --t) {
              uint16_t *const e = reinterpret_cast<uint16_t *>(vt + t * 128 + (((ch + (lane >> 3)) ^ (t & 7)) << 4) + (lane & 7) * 2);
              if ((*e & 0x7F80u) == 0x7F80u) {
                *e = 0;
                first = t;
              }
            }
            w.bad[quad * 32 + half * 16 + lane] = first;
          }
          fence_smem_to_async();  // (the next tile lands here)
          __syncwarp();
        }
        if (lane == 0) w.has_bad[quad * 2 + half] = looked;
        tmem_st_16x128b(tl + COL_V + par * 32 + (static_cast<uint32_t>(half * 16) << 16), r);
        tmem_st_wait();
        tc_fence_before_sync();
        arrive_warp(&m->v_ready[par], lane);
        if (lane == 0) mbar_arrive(&m->empty_v[par]);
      }
      return true;
    };
    // The state goes where it belongs, and the next unit's takes its place (null: from nowhere), 16 values of a thread at a time, so that the loads
    // are under way beside the stores.
    const auto exchange = [&](float *dst, const float *src) {
      const bool out = dst != nullptr, in = src != nullptr;
      dst += k0 * D + v;
      src += k0 * D + v;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (out) {
#pragma unroll
          for (int j = 8 * b; j < 8 * b + 8; ++j) {
            const float2 y = dunpack2(S[j]);
            dst[2 * j * D] = y.x;
            dst[(2 * j + 1) * D] = y.y;
          }
        }
#pragma unroll
        for (int j = 8 * b; j < 8 * b + 8; ++j) S[j] = 0;
        if (in) {
#pragma unroll
          for (int j = 8 * b; j < 8 * b + 8; ++j) S[j] = dpack2(src[2 * j * D], src[(2 * j + 1) * D]);
        }
      }
    };
    // V^T goes a chunk ahead: a chunk's own products are under way meanwhile.
    bool more = false;
#pragma unroll 1
    for (int n = -1;; ++n) {
      Chunk &w = m->ch[slot(n)];
      if (n >= 0) {
        if constexpr (WITH_O) {
          if (n > 0) wait_bar(&m->bar_s, (n - 1) & 1u, m);  // QS of the chunk before has read its state
          tc_fence_after_sync();
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            uint64_t rest[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] = S[b * 8 + j];
#pragma unroll
            for (int part = 0; part < OSPLIT; ++part) {
              uint32_t r[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) r[j] = take_bf16x2(rest[j]);
              tmem_st8(tl + COL_SH + part * (COL_SL - COL_SH) + half * 32 + b * 8, r);
            }
          }
          tmem_st_wait();
          tc_fence_before_sync();
          arrive_warp(&m->s_ready, lane);
        }
      }
      more = values(n + 1);
      if (n >= 0) {
        float f = w.all;
        const float f_lo = w.all_lo;
        decay += w.log;
        wait_bar(&m->bar_d, n & 1u, m);
        tc_fence_after_sync();
        if (w.has_bad[quad * 2 + (lane >> 4)] != 0 && w.bad[v] < C) f = __int_as_float(0x7fffffff);  // the column is none from here on
        const uint64_t ff = dpack2(f, f), ll = dpack2(f_lo, f_lo);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t d[16];
          tmem_ld16(tl + COL_D + k0 + b * 16, d);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 8; ++j)
            S[b * 8 + j] = dfma2(S[b * 8 + j], ff, dfma2(S[b * 8 + j], ll, dpack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1]))));
        }
        tc_fence_before_sync();
        arrive_warp(&m->d_free, lane);
        if (w.last) {
          // A unit is written as a whole or, after a time-out, not at all: every warp that has got through it arrives, and it is written
          // if all have.
          if (uni(m->abort_flag)) break;
          arrive_warp(&m->s_whole, lane);
          wait_bar(&m->s_whole, units & 1u, m);
          if (!uni(mbar_test_wait(&m->s_whole, units & 1u))) break;
          ++units;
          exchange(w.dst, more ? m->ch[slot(n + 1)].src : nullptr);
          if (w.decay && warp == WARP_S && lane == 0) *w.decay = exp2f(decay);
          decay = 0.f;
        }
        arrive_warp(&m->dec_empty[slot(n)], lane);
      }
      else if (more) {
        exchange(nullptr, m->ch[0].src);
      }
      if (!more) break;
    }
  }
  stream_order_release();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == WARP_MMA) tmem_dealloc(tm, 512);
  // every block says how it ended, the first one also for the blocks there are not: nobody has to clear the words beforehand
  if (tid == 0) sp.status[blockIdx.x] = m->abort_flag;
  if (blockIdx.x == 0) {
    for (uint32_t i = gridDim.x + tid; i < kStatusWords; i += NT) sp.status[i] = 0;
    if (sp.phase == 0)
      for (uint32_t i = tid; i < kStatusWords; i += NT) sp.status[kStatusWords + i] = 0;
  }
}

// States at the starts of a unit's segments: seg_state[unit][0] = its own, [s] = e^{G of segment s-1} [s-1] + what segment s-1 adds
// (which [s] held).  One thread per four values.
__global__ void __launch_bounds__(256) decay_join_kernel(const __grid_constant__ DascDecayArgs a, const __grid_constant__ Split sp) {
  const int64_t unit = blockIdx.x / (D * D / 1024);
  const int at = (blockIdx.x % (D * D / 1024)) * 1024 + threadIdx.x * 4;
  const int h = static_cast<int>(unit % a.H_v), lc = static_cast<int>(unit / a.H_v % a.n_layers_in_call);
  const int r = static_cast<int>(unit / a.H_v / a.n_layers_in_call);
  stream_order_begin();
  const int req = a.req_idx[r];
  if (req < 0) return;
  const int segs = segments_of(sp, chunks_of(decay_range(a, r).n));
  if (segs <= 1) return;
  const bool merge = a.mode == DASC_DECAY_SCRATCH_MERGE_LOCAL;
  const int layer = a.layer_begin + lc;
  if (!a.o && (a.mode == DASC_DECAY_SCORE || (merge && a.row_keep[layer * a.rows_per_layer + h * D]))) return;
  float4 run = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!merge && !(a.from_zero && a.from_zero[r] != 0))
    run = *reinterpret_cast<const float4 *>(a.state + req * a.req_stride + layer * a.layer_stride + static_cast<int64_t>(h) * (D * D) + at);
  float *const seg = sp.seg_state + unit * sp.nseg * (D * D) + at;
  *reinterpret_cast<float4 *>(seg) = run;
  for (int s = 1; s < segs; ++s) {
    const float f = sp.seg_decay[unit * sp.nseg + s - 1];
    const float4 y = *reinterpret_cast<const float4 *>(seg + static_cast<int64_t>(s) * (D * D));
    run = make_float4(fmaf(f, run.x, y.x), fmaf(f, run.y, y.y), fmaf(f, run.z, y.z), fmaf(f, run.w, y.w));
    *reinterpret_cast<float4 *>(seg + static_cast<int64_t>(s) * (D * D)) = run;
  }
}

// cuTensorMapEncodeTiled is a driver entry point, looked up through the runtime at first use (no link-time dependency on libcuda).
using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                   const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// How long requests are split: into as many segments as make the longest chain of chunks on one SM shortest, by the caller's bound on
// the length.  All but the last segment are then run twice (their states first, without outputs).  The model counts time in chunks with
// outputs (2.4 to 2.5 us): one without takes 0.58 to 0.60 of it (148 heads of 8192 tokens, 184 against 315 us), so a split chunk counts 1.6, and the two
// more launches and the join about 10 (2048 tokens of 32 heads in 4 segments: 52 us, 31 of them chunks).  Measured, us, unsplit / as the model has it /
// the best of up to 16 segments: 32 heads of 32,768 tokens 1124 / 462 / 457, of 8192 320 / 153 / 151, of 2048 77 / 52 / 52, of 1024 42 / 42 / 37; 4 heads
// of 4096 169 / 41 / 38; 4, 8 and 9 requests of 32 heads and 2048 or 4096 tokens are best left whole, as it has them (two segments of four
// requests 221 against 153).  One of 32,768 beside 8 of 100 1218 / 722 / 665: the model weighs the batch, not its one long request,
// and with more units than twice the SMs nothing is split however long one of them is.
struct SplitSizes {
  int32_t nseg, seg_chunks;
};
constexpr int64_t kMaxSplitUnits = 2 * kSms, kMaxSegments = 16, kMaxSplitItems = 1024, kMinSplitChunks = 16, kMinSegmentChunks = 4;
int64_t longest_chunks(int64_t total_tokens, int32_t max_seqlen) {
  return (std::max<int64_t>(std::min<int64_t>(max_seqlen, total_tokens), 1) + C - 1) / C;
}
SplitSizes split_sizes(int32_t n_req, int32_t layers, int32_t H_v, int64_t total_tokens, int32_t max_seqlen) {
  const int64_t units = static_cast<int64_t>(n_req) * layers * H_v;
  const int64_t longest = longest_chunks(total_tokens, max_seqlen);
  SplitSizes best{1, static_cast<int32_t>(longest)};
  if (units == 0 || units > kMaxSplitUnits || longest < kMinSplitChunks) return best;
  const double even = static_cast<double>(std::min<int64_t>(total_tokens / C + n_req, longest * n_req)) * layers * H_v / longest;  // units as long as the longest
  double cost = 0;
  for (int nseg = 1; nseg <= kMaxSegments && units * nseg <= kMaxSplitItems && n_req * nseg <= kMaxSorted; ++nseg) {
    const int64_t chunks = (longest + nseg - 1) / nseg;
    if (nseg > 1 && chunks < kMinSegmentChunks) break;
    const double rounds = std::max(1.0, static_cast<double>(static_cast<int64_t>((even * nseg + kSms - 1) / kSms)));
    const double t = rounds * chunks * (nseg > 1 ? 1.6 : 1.0) + (nseg > 1 ? 10.0 : 0.0);
    if (nseg == 1 || t < cost) {
      cost = t;
      best = {nseg, static_cast<int32_t>(chunks)};
    }
  }
  return best;
}

template <bool WITH_O, typename OT>
cudaError_t launch(const DascDecayArgs &a, const Split &sp, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, void *stream) {
  auto kern = decay_chunked_kernel<WITH_O, OT>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(SMEM_BYTES));
  if (e != cudaSuccess) return e;
  const int64_t items = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v * sp.nseg;
  return launch_blocks(kern, dim3(static_cast<unsigned>(std::min<int64_t>(items, kSms))), dim3(NT), SMEM_BYTES, stream, a, sp, q, k, v);
}

}  // namespace

static size_t workspace_of(int64_t segments) {
  return kDecayStatusWords * sizeof(uint32_t) + (segments * sizeof(float) + 255) / 256 * 256 + segments * D * D * sizeof(float);
}

size_t dasc_decay_chunked_workspace_bytes(int32_t n_req, int32_t n_layers_in_call, int32_t H_v, int64_t total_tokens, int32_t max_seqlen) {
  const SplitSizes s = split_sizes(n_req, n_layers_in_call, H_v, total_tokens, max_seqlen);
  return workspace_of(s.nseg > 1 ? static_cast<int64_t>(n_req) * n_layers_in_call * H_v * s.nseg : 0);
}

// Few long requests are split where many are not, so a call may need more than a larger one.  The most that any call up to these sizes
// needs: as many units as are split at all, times as many segments as the longest request may have.
size_t dasc_decay_chunked_workspace_bound(int32_t n_req, int32_t n_layers_in_call, int32_t H_v, int64_t total_tokens, int32_t max_seqlen) {
  const int64_t longest = longest_chunks(total_tokens, max_seqlen);
  if (longest < kMinSplitChunks) return workspace_of(0);
  const int64_t units = std::min(static_cast<int64_t>(n_req) * n_layers_in_call * H_v, kMaxSplitUnits / H_v * H_v);
  const int64_t segments = std::min(kMaxSegments, (longest - 1) / (kMinSegmentChunks - 1));  // ceil(longest / n) >= kMinSegmentChunks
  return workspace_of(std::min(units * segments, kMaxSplitItems));
}

int dasc_launch_decay_chunked(const DascDecayArgs &args, void *stream) {
  if (args.d_k != D || args.d_v != D || !args.io_bf16) return -1;
  DascDecayArgs a = args;
  a.poll_limit_first_wait = __atomic_load_n(&g_dasc_debug_poll_limit, __ATOMIC_RELAXED);
  CUtensorMap tmap_q{}, tmap_k{}, tmap_v{};
  const EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) return static_cast<int>(cudaErrorNotSupported);
  // the streams [Lc*T tokens][heads][128]: boxes of 64 tokens x one head x 64 channels, 128 bytes, swizzled as the operand tiles are
  const auto make_map = [&](CUtensorMap *map, const void *base, int heads) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(heads),
                                static_cast<cuuint64_t>(a.n_layers_in_call) * static_cast<cuuint64_t>(a.total_tokens)};
    const cuuint64_t strides[2] = {D * 2, static_cast<cuuint64_t>(heads) * D * 2};
    const cuuint32_t box[3] = {64, 1, static_cast<cuuint32_t>(C)}, ones[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!make_map(&tmap_k, a.k, a.H_k) || !make_map(&tmap_v, a.v, a.H_v) || (a.o && !make_map(&tmap_q, a.q, a.H_k)))
    return static_cast<int>(cudaErrorInvalidValue);
  const SplitSizes sizes = split_sizes(a.n_req, a.n_layers_in_call, a.H_v, a.total_tokens, a.max_seqlen);
  uint32_t *const ws = static_cast<uint32_t *>(a.workspace);
  Split sp{sizes.nseg, sizes.seg_chunks, 0, nullptr, nullptr, ws};
  cudaError_t e = cudaSuccess;
  if (sp.nseg > 1) {
    const int64_t units = static_cast<int64_t>(a.n_req) * a.n_layers_in_call * a.H_v;
    unsigned char *const p = static_cast<unsigned char *>(a.workspace) + kDecayStatusWords * sizeof(uint32_t);
    sp.seg_decay = reinterpret_cast<float *>(p);
    sp.seg_state = reinterpret_cast<float *>(p + (units * sp.nseg * sizeof(float) + 255) / 256 * 256);
    sp.phase = 1;
    sp.status = ws + kStatusWords;
    e = launch<false, __nv_bfloat16>(a, sp, tmap_q, tmap_k, tmap_v, stream);
    if (e == cudaSuccess)
      e = launch_blocks(decay_join_kernel, dim3(static_cast<unsigned>(units * (D * D / 1024))), dim3(256), 0, stream, a, sp);
    sp.phase = 2;
    sp.status = ws;
  }
  if (e != cudaSuccess) return static_cast<int>(e);
  if (!a.o) return static_cast<int>(launch<false, __nv_bfloat16>(a, sp, tmap_q, tmap_k, tmap_v, stream));
  return static_cast<int>(a.o_bf16 ? launch<true, __nv_bfloat16>(a, sp, tmap_q, tmap_k, tmap_v, stream)
                                   : launch<true, float>(a, sp, tmap_q, tmap_k, tmap_v, stream));
}
