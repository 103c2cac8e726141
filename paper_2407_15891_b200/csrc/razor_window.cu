// Attention of prompt tokens over dense K and V, causal, with a sliding window and sink tokens per KV head: what a prefill
// computes from the rows that razor_compress packs afterwards (Algorithm 1 keeps the same sets: the first N0 and the last
// L_h tokens of a head, everything of a retrieval head).
//
//   out[m] = sum_n e^(s_mn) v_n / sum_n e^(s_mn),  s_mn = sm_scale q_m.k_n,  n <= m and (n < N0 or m - n < L_h or L_h < 0)
//
// Flash attention on the 5th-generation tensor cores.  A CTA (one to an SM) takes a unit: two tiles of 128 query rows (128 / G
// query tokens x the G query heads that share a KV head), for which K and V are read once.  It walks over the 128-token key
// tiles that some of its queries see (razor_window.h).  Roles:
//   * warps 0-3 and 4-7: softmax of tile 0 and of tile 1, a thread per query row (tensor-memory lane): 128 scores out of
//     tensor memory, mask, running maximum, weights as bf16 back into tensor memory, over the scores, and the sum of those;
//   * warp 8: TMA copies (Q per tile, a ring of K tiles, a ring of V tiles, 128-byte swizzle) and the walk over the units;
//   * warp 9, one thread: the matrix instructions.  S_i = Q_i K^T (both operands in shared memory), O_i += P_i V (P out of
//     tensor memory, as soon as its first half is there).  While one tile is in its softmax the other one's products run:
//     PV_0, QK_0, PV_1, QK_1, ..;
//   * warps 10, 11: look over the V tiles that are partly masked.  A weight of zero times a NaN or an infinity is a NaN, so
//     such values are zeroed in shared memory, and put back into the rows that do see them at the end (rows that a mask
//     hides from a token are never touched by it, whatever it holds).  Where no query of the unit sees one there is nothing to
//     put back: one token over 4 x 8000, NaN behind them, 63 us for 58 (looked through all the same, 759).
// Tensor memory: S_0, S_1 (P over their lower halves), O_0, O_1: 4 x 128 columns, all there is.
// The reference maximum of a row may lag behind the true one by a factor of 2^8; only a row that outruns it has its
// accumulator rescaled, by its own softmax thread: when S_i of a step is there, the product of the step before has run.
//
// Work: up to 1024 units are laid end to end, step by step, and cut into one span per CTA, on the device (lengths and windows
// live there): a long context with few queries is spread over all SMs, and equal units fill the last wave.  Units that were
// cut leave partial records (m, l, o) per row, which window_combine_kernel folds in order.  More units than that are handed
// out whole from a queue, the last queries first: the longest first among equal sequences and heads, but a unit of a head that
// sees everything is not put before one of a short window.  (1024: units then come to seven waves and their ends even out.  What
// is lost at the border, and with ragged lengths behind it, has not been measured.)
//
// What bounds it.  Long contexts, D = 128: a step of both tiles is 2048 cycles of products (128 x 128 x 16 in 64 cycles) and
// takes 3550: a tile's softmax (2000: 128 exponentials a thread, as many again for scale, maximum, sum and conversion) and its
// way through the products (1450) follow each other, and two tiles fill no more than that.  32768 tokens, 32 query heads over
// 8, all in sight: 7.25 ms in short runs (1213 TFLOP/s, 0.78 of the measured cuBLAS burst rate), 8.3 under continuous load,
// where the power cap holds the clock (1060 TFLOP/s, 0.79 of cuBLAS's sustained rate); 8192 tokens 0.54 ms, a window of 1024 at
// 32768 0.68 ms.  Short units pay their start (8500 cycles to the first scores of a launch, about half of it before the first
// copy) and their results' way out (4400 cycles: a thread writes a row of its own).  One token over dense K and V is bound by the
// same chain, a tile's step being short of rows but not of latency: 164 MB in 50 us.
// Tried and dropped: an issuing thread for each tile (9.0 ms for 8.5 as it stood then: the tiles drift into step); sixteen
// softmax warps, two threads to a row (10.3 ms for 7.6: the threads' exchange, twice the waits); every third, fifth or eighth
// pair of exponentials as a polynomial (7.6, 7.6, 7.5 ms for 7.1: instructions are shorter than the unit); P in four parts.
//
// Every wait is bounded in time; a wait that runs out ends the CTA through the common exit (copies and instructions in flight
// are waited for, tensor memory is released).  Rows that it was working on, and those of cut units that it had a part of, are
// NaN; rows of its own that it had not come to stay as they were.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "razor_common.cuh"
#include "razor_sync.cuh"
#include "razor_tc.cuh"
#include "razor_window.h"

namespace razor {
namespace {

constexpr int kWinThreads = 384;
// Registers: 168 a thread at launch; the softmax threads, which hold a row of 128 scores, take over what the others give up.
constexpr int kWinLaunchRegs = 168, kWinSoftmaxRegs = 216, kWinOtherRegs = 72;
static_assert(256 * kWinSoftmaxRegs + 128 * kWinOtherRegs <= kWinThreads * kWinLaunchRegs, "no more than the block was launched with");
constexpr int kParts = 2;                    // P is handed over in so many parts (32K tokens, before the sums of rounded weights: 7.1 ms; in four parts 7.3)
constexpr int kHalfBytes = kWinTile * 128;   // 128 rows of 64 elements

template <int D>
struct WinCfg {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kKStages = D == 128 ? 3 : 4;
  static constexpr int kVStages = D == 128 ? 2 : 4;
};

struct WinCall {
  const int32_t* q_len;     // [B] or NULL: n_tokens
  const int32_t* ctx_len;   // [B] or NULL: n_ctx
  const int32_t* window;    // [B, Hkv] or NULL: everything
  const __nv_bfloat16* v;   // for values that are not finite
  __nv_bfloat16* out;       // [B, n_tokens, Hq, D]
  int64_t v_stride_b, v_stride_h, v_stride_n;
  int32_t batch, n_tokens, n_ctx, n_q_heads, n_kv_heads, group, tpt;   // tpt: query tokens of a tile
  int32_t n_sink, n_units, pairs, spans;   // spans: 1: the steps are cut into spans; 0: units from the queue
  int32_t rec_rows;         // rows of a record: those of two tiles
  int32_t rec_tile;         // query tokens of a tile in it
  int32_t out_whole;        // out begins at a 32-byte boundary
  float scale_log2;
  int32_t stopped_cta;      // -1; a self-test has this CTA give up its waits at once
  // workspace
  int32_t* queue;
  uint8_t* done;            // [CTAs]: this CTA came to its end without giving up a wait
  int2* table;              // [n_units]: the first span with a part of the unit, and its parts (0: no query in it)
  float2* rec_ml;           // [2 * kWinMaxSpans][rec_rows]
  float* rec_o;             // [2 * kWinMaxSpans][rec_rows][D]
};

struct WinItem {
  int32_t unit, b, g, window, ctx;   // unit < 0: no more
  int32_t j0, j1;                    // steps of this part
  int32_t slot;                      // record, -1: the whole unit is here
  int32_t poison;                    // values that are not finite were taken out of V
  WinUnit u;
};

struct WinCtl {
  uint64_t q_full[2], q_empty[2];
  uint64_t k_full[4], k_empty[4], v_full[4], v_clean[4], v_empty[4];
  uint64_t s_full[2], p_full[2][kParts], o_full[2];   // (P in parts: its product begins with the first)
  uint64_t item_full[2], item_empty[2];
  uint64_t drain;
  WinItem item[2];
  uint32_t tmem_base;
  int abort_flag;
  unsigned issued_k, issued_v, issued_q[2];   // copies, by the copying thread when it leaves
  int first_unit, first_step;        // of this CTA's span
  long long scan[kWinThreads / 32];
};
constexpr int kItemReaders = 8 + 1 + 2;   // softmax warps, the MMA thread, the looking warps

template <int D>
constexpr size_t win_smem_bytes() {
  return 1024 + (size_t)(2 + WinCfg<D>::kKStages + WinCfg<D>::kVStages) * WinCfg<D>::kTileBytes + sizeof(WinCtl);
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void win_tmem_st32(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      :
      : "r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]),
        "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]),
        "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ void win_tmem_st16(uint32_t taddr, const uint32_t* o) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      :
      : "r"(taddr), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "r"(o[8]),
        "r"(o[9]), "r"(o[10]), "r"(o[11]), "r"(o[12]), "r"(o[13]), "r"(o[14]), "r"(o[15])
      : "memory");
}
// Scales 16 columns of this thread's lane.
__device__ __forceinline__ void win_tmem_scale16(uint32_t taddr, float f) {
  uint32_t o[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]), "=r"(o[8]),
        "=r"(o[9]), "=r"(o[10]), "=r"(o[11]), "=r"(o[12]), "=r"(o[13]), "=r"(o[14]), "=r"(o[15])
      : "r"(taddr)
      : "memory");
  tmem_ld_wait_all();
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    asm volatile("" : "+r"(o[e]));
    o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
  }
  win_tmem_st16(taddr, o);
}
__device__ __forceinline__ void win_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t win_pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t*)&v;
}
// a, b += the two bf16 values of `pair`, in fp32
__device__ __forceinline__ void win_sum2(float& a, float& b, uint32_t pair) {
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "add.rn.f32.bf16 %0, lo, %0;\n\t"
      "add.rn.f32.bf16 %1, hi, %1;\n\t}"
      : "+f"(a), "+f"(b)
      : "r"(pair));
}
// One matrix instruction, the descriptors as (low word, high word); the second with operand A out of tensor memory.
__device__ __forceinline__ void win_umma(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 a, {%1, %2};\n\t"
      "mov.b64 b, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
      :
      : "r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate));
}
__device__ __forceinline__ void win_umma_tmem_a(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 b, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
      :
      : "r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate));
}
// 32 bytes at a 32-byte boundary, or at a 16-byte one.  (A row's pieces go to lines of their own, so it is the number of
// stores that counts: half as many took a unit's way out from 5800 cycles to 4400.)
__device__ __forceinline__ void win_store32(void* p, bool whole, const uint32_t (&u)[8]) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
                 "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
  } else {
    ((uint4*)p)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    ((uint4*)p)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}
// the larger of three values, NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool finite_bf16(__nv_bfloat16 x) { return (__bfloat16_as_ushort(x) & 0x7f80) != 0x7f80; }

// Unit number -> its place and steps.  Units run over (sequence, KV head) fastest; out of the queue the last queries come first.
__device__ __forceinline__ WinUnit find_unit(const WinCall& c, int unit, int& b, int& g, int& window, int& ctx) {
  const int bh = unit % (c.batch * c.n_kv_heads);
  int pr = unit / (c.batch * c.n_kv_heads);
  if (!c.spans) pr = c.pairs - 1 - pr;
  b = bh / c.n_kv_heads;
  g = bh % c.n_kv_heads;
  ctx = c.ctx_len ? min(max(c.ctx_len[b], 0), c.n_ctx) : c.n_ctx;
  const int q_len = c.q_len ? min(max(c.q_len[b], 0), c.n_tokens) : c.n_tokens;
  window = c.window ? min(c.window[bh], 1 << 30) : -1;   // (no context is longer; differences stay in range)
  return win_unit(pr * 2 * c.tpt, c.tpt, q_len, ctx, window, c.n_sink);
}

// Zeroes the bf16 values of `w` that are not finite.
__device__ __forceinline__ uint32_t finite_or_zero2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
  return w;
}

// Infinities and NaNs of V that were zeroed for the sake of rows that do not see them, added to a row that does: positions
// of the masked tiles among the row's steps.  Slow (a thread looks through them by itself), and only where a query of the unit
// sees such a value: what lies behind the end of a context or before the windows costs next to nothing.
template <int D, typename Add>
__device__ __forceinline__ void restore_non_finite(const WinCall& c, const WinItem& it, const WinTileSteps& t, int pos, Add add) {
  const __nv_bfloat16* v = c.v + it.b * c.v_stride_b + it.g * c.v_stride_h;
#pragma unroll 1
  for (int j = it.j0; j < it.j1; ++j) {
    const int kt = it.u.key_tile(j);
    // (looked over: the tiles that are masked for either tile of the unit)
    bool looked = false;
    for (int i = 0; i < 2; ++i) {
      const WinTileSteps& o = it.u.tile[i];
      looked |= o.active(j) && win_masked(kt, o.pos, o.pos + o.n_tok - 1, it.window, c.n_sink);
    }
    if (!looked || !t.active(j)) continue;
#pragma unroll 1
    for (int n = kt * kWinTile; n < kt * kWinTile + kWinTile && n <= pos; ++n) {
      if (!(it.window < 0 || n < c.n_sink || pos - n < it.window)) continue;
      const __nv_bfloat16* row = v + (int64_t)n * c.v_stride_n;
#pragma unroll 4
      for (int d = 0; d < D; d += 8) {
        const uint4 u = __ldg((const uint4*)(row + d));
        if (finite_or_zero2(u.x) == u.x && finite_or_zero2(u.y) == u.y && finite_or_zero2(u.z) == u.z && finite_or_zero2(u.w) == u.w) continue;
#pragma unroll 1
        for (int x = d; x < d + 8; ++x)
          if (!finite_bf16(row[x])) add(x, __bfloat162float(row[x]));
      }
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kWinThreads, 1)
    window_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ WinCall c) {
  using Cfg = WinCfg<D>;
  constexpr int TB = Cfg::kTileBytes, KS = Cfg::kKStages, VS = Cfg::kVStages, HALVES = Cfg::kHalves;
  constexpr uint32_t kIdescQK = instr_desc_bf16(kWinTile, kWinTile, false);
  constexpr uint32_t kIdescPV = instr_desc_bf16(kWinTile, D, true);
  constexpr uint32_t kTmemCols = 512;
  extern __shared__ uint8_t win_smem_raw[];
  uint8_t* base = win_smem_raw + ((1024u - (smem_u32(win_smem_raw) & 1023u)) & 1023u);
  uint8_t* q_tile = base;
  uint8_t* k_tile = q_tile + 2 * TB;
  uint8_t* v_tile = k_tile + KS * TB;
  WinCtl* ctl = (WinCtl*)(v_tile + VS * TB);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &ctl->abort_flag;

  cudaTriggerProgrammaticLaunchCompletion();   // (the combine kernel waits for this whole grid before it reads)
  if (threadIdx.x < 3 * 32 && lane == 0)
    asm volatile("prefetch.tensormap [%0];" ::"l"(warp == 0 ? &map_q : (warp == 1 ? &map_k : &map_v)) : "memory");
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl->q_full[i], 1);
      mbar_init(&ctl->q_empty[i], 1);
      mbar_init(&ctl->s_full[i], 1);
      for (int k = 0; k < kParts; ++k) mbar_init(&ctl->p_full[i][k], 128);
      mbar_init(&ctl->o_full[i], 1);
      mbar_init(&ctl->item_full[i], 1);
      mbar_init(&ctl->item_empty[i], kItemReaders);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&ctl->k_full[s], 1);
      mbar_init(&ctl->k_empty[s], 1);
      mbar_init(&ctl->v_full[s], 1);
      mbar_init(&ctl->v_clean[s], 64);
      mbar_init(&ctl->v_empty[s], 1);
    }
    mbar_init(&ctl->drain, 1);
    ctl->abort_flag = (int)blockIdx.x == c.stopped_cta;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  long long total = 0, span_end = 0, span_at = 0;   // steps of the launch; this CTA's span
  int n_spans = 1;
  if (c.spans) {
    // ---- prefix sums of the units' weights, three consecutive units to a thread.  (The weights are put down in the K stages,
    // which nothing fills yet.)
    constexpr int PER = (kWinSpanUnits + kWinThreads - 1) / kWinThreads;
    int* weights = (int*)k_tile;
#pragma unroll 1
    for (int unit = threadIdx.x; unit < c.n_units; unit += kWinThreads) {
      int b, g, window, ctx;
      weights[unit] = find_unit(c, unit, b, g, window, ctx).weight();
    }
    __syncthreads();
    int w[PER];
    long long sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int unit = (int)threadIdx.x * PER + i;
      w[i] = unit < c.n_units ? weights[unit] : 0;
      sum += w[i];
    }
    long long upto = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    if (lane == 31) ctl->scan[warp] = upto;
    __syncthreads();
    long long before = upto - sum;
    for (int k = 0; k < kWinThreads / 32; ++k) {
      if (k < warp) before += ctl->scan[k];
      total += ctl->scan[k];
    }
    n_spans = total > 0 ? win_n_spans(total, (int)gridDim.x) : 1;
    if (blockIdx.x == gridDim.x - 1) {   // (the CTA that is likeliest to have no span)
      long long at = before;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int unit = (int)threadIdx.x * PER + i;
        int first = 0, parts = 0;
        if (w[i] > 0) win_unit_spans(total, n_spans, at, w[i], first, parts);
        if (unit < c.n_units) c.table[unit] = make_int2(first, parts);
        at += w[i];
      }
    }
    if (total > 0 && (int)blockIdx.x < n_spans) {
      span_at = win_span_begin(total, n_spans, blockIdx.x);
      span_end = win_span_begin(total, n_spans, blockIdx.x + 1);
    }   // (otherwise there is nothing for this CTA: it goes through the motions with no item)
    long long at = before;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (span_at < span_end && span_at >= at && span_at < at + w[i]) {
        ctl->first_unit = (int)threadIdx.x * PER + i;
        ctl->first_step = (int)(span_at - at);
      }
      at += w[i];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the weights have been read: TMA may write there)
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;

  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWinSoftmaxRegs));
    // ================================================================ softmax and epilogue: a thread per query row
    const int ti = warp >> 2;                     // tile
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_addr + (uint32_t)(ti * kWinTile), o_addr = lane_addr + 2 * kWinTile + (uint32_t)(ti * kWinTile);
    const int G = c.group, r_tok = row / G, r_head = row % G;
    const float scale_log2 = c.scale_log2;
    unsigned n_s = 0, n_o = 0;
    bool ok = true;
    for (unsigned gi = 0; ok; ++gi) {
      ok = __all_sync(0xffffffffu, mbar_wait(&ctl->item_full[gi & 1], (gi >> 1) & 1, abort_flag));
      if (!ok) break;
      const WinItem& it = ctl->item[gi & 1];
      if (it.unit < 0) break;
      const WinTileSteps t = it.u.tile[ti];
      const int j0 = it.j0, j1 = it.j1, window = it.window;
      const int cnt = t.steps_in(j0, j1);
      const bool row_live = r_tok < t.n_tok;      // (r_tok >= tpt for the rows that 128 / G leaves over: n_tok <= tpt)
      const bool warp_live = __any_sync(0xffffffffu, row_live);
      const int pos = t.pos + r_tok;
      constexpr float kLag = 8.f;
      float m_ref = -CUDART_INF_F, l_run = 0.f;
      bool first = true;
      for (int j = j0; j < j1 && ok && cnt > 0; ++j) {
        if (!t.active(j)) continue;
        ok = __all_sync(0xffffffffu, mbar_wait(&ctl->s_full[ti], n_s & 1, abort_flag));
        if (!ok) break;
        ++n_s;
        tc_fence_after();
        if (!warp_live) {   // nobody reads these rows
#pragma unroll
          for (int h = 0; h < kParts; ++h) mbar_arrive(&ctl->p_full[ti][h]);
          continue;
        }
        uint32_t v[kWinTile];
#pragma unroll
        for (int k = 0; k < kWinTile / 32; ++k) tmem_ld32_issue(s_addr + (uint32_t)(k * 32), v + k * 32);
        tmem_ld_wait_all();
#pragma unroll
        for (int e = 0; e < kWinTile; ++e) asm volatile("" : "+r"(v[e]));
        const int kt = it.u.key_tile(j);
        if (win_masked(kt, t.pos, t.pos + t.n_tok - 1, window, c.n_sink)) {
          const int k0 = kt * kWinTile, hi = pos - k0 + 1, sink = c.n_sink - k0;   // columns [0, hi) are not in the future
          const int lo = window < 0 ? 0 : hi - window;                            // columns from lo on are in the window
          auto below = [](int x) -> uint32_t { return x <= 0 ? 0u : (x >= 32 ? 0xffffffffu : (1u << x) - 1u); };
#pragma unroll
          for (int k = 0; k < kWinTile / 32; ++k) {
            const uint32_t see = below(hi - k * 32) & (below(sink - k * 32) | ~below(lo - k * 32));
            if (__all_sync(0xffffffffu, see == 0xffffffffu)) continue;   // (most of a boundary tile is in sight of a warp's rows)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(see & (1u << e))) v[k * 32 + e] = 0xff800000u;
          }
        }
        float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
        for (int e = 0; e < kWinTile; e += 2) mx[(e >> 1) & 3] = max3_nan(mx[(e >> 1) & 3], __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
        // (the scale is positive or zero: the maximum of the scaled scores is the scaled maximum)
        const float m_blk = max3_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3], mx[3]) * scale_log2;
        // a score that is NaN or +infinity leaves no weights to speak of: the row is NaN
        if (!(m_blk < CUDART_INF_F)) l_run = CUDART_NAN_F;
        const bool want = m_blk > m_ref + kLag || (m_ref == -CUDART_INF_F && m_blk > -CUDART_INF_F);
        if (__any_sync(0xffffffffu, want)) {
          const float m_to = fmaxf(m_ref, m_blk);
          const float f = (m_to == -CUDART_INF_F || m_ref == -CUDART_INF_F) ? 0.f : fast_exp2(m_ref - m_to);
          if (!first) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) win_tmem_scale16(o_addr + (uint32_t)(k * 16), f);
          }
          l_run *= f;
          m_ref = m_to;
        }
        const float m_use = (m_ref == -CUDART_INF_F) ? 0.f : m_ref;
        const uint64_t scale2 = f2_pack(scale_log2, scale_log2), neg_m2 = f2_pack(-m_use, -m_use);
        // Weights go to the product with V in bf16: the instruction takes both operands in one type, and V is bf16.  (Their
        // remainders would be a second product, half as much again of the instructions' time, for a result in bf16.)
        uint32_t pw[kWinTile / 2];
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
          constexpr int PAIRS = kWinTile / kParts / 2;
          uint32_t* const p = pw + h * PAIRS;
#pragma unroll
          for (int e2 = 0; e2 < PAIRS; ++e2) {
            const int e = (h * PAIRS + e2) * 2;
            const uint64_t t2 = f2_fma(f2_pack(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), scale2, neg_m2);
            float w0, w1;
            f2_unpack(t2, w0, w1);
            w0 = fast_exp2(w0);
            w1 = fast_exp2(w1);
            p[e2] = win_pack2(w0, w1);
          }
          static_assert(PAIRS == 32, "a part is one store");
          win_tmem_st32(s_addr + (uint32_t)(h * PAIRS), p);
          win_tmem_st_wait();
          tc_fence_before();
          mbar_arrive(&ctl->p_full[ti][h]);
        }
        // The sum takes the weights as the product has them, rounded: a row is an average of the values it sees, whatever the
        // rounding.  (With the unrounded ones a row of equal values came out up to a step of bf16 off, and so did a row whose
        // largest weight is not 1, the reference lagging.)  Added up while the products run: 32K tokens 7.14 -> 7.28 ms, a window
        // of 1024 there 0.674 -> 0.702; before the hand-over 7.37 and 0.712.
        float psum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
        for (int e = 0; e < kWinTile / 2; ++e) win_sum2(psum[e & 1][0], psum[e & 1][1], pw[e]);
        l_run += (psum[0][0] + psum[1][0]) + (psum[0][1] + psum[1][1]);
        first = false;
      }
      if (ok && cnt > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(&ctl->o_full[ti], n_o & 1, abort_flag));
        ++n_o;
        tc_fence_after();
      }
      // ---- the row's result
      const bool direct = it.slot < 0;
      float inv = 1.f;
      if (direct) inv = m_ref == -CUDART_INF_F && !isnan(l_run) ? 0.f : 1.f / l_run;
      if (!ok) inv = CUDART_NAN_F;
      const int tok = t.tok + r_tok;
      __nv_bfloat16* dst = c.out + (((size_t)it.b * c.n_tokens + tok) * c.n_q_heads + (size_t)it.g * G + r_head) * D;
      const size_t rec = (size_t)max(it.slot, 0) * c.rec_rows + (size_t)(ti * c.rec_tile + r_tok) * G + r_head;
      if (warp_live) {
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          uint32_t o[32];
          if (ok && cnt > 0) {
            tmem_ld32_issue(o_addr + (uint32_t)(k * 32), o);
            tmem_ld_wait_all();
#pragma unroll
            for (int e = 0; e < 32; ++e) asm volatile("" : "+r"(o[e]));
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0u;
          }
          if (row_live) {
            if (direct) {
#pragma unroll
              for (int e = 0; e < 32; e += 16) {
                uint32_t u[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) u[x] = win_pack2(__uint_as_float(o[e + 2 * x]) * inv, __uint_as_float(o[e + 2 * x + 1]) * inv);
                win_store32(dst + k * 32 + e, c.out_whole, u);
              }
            } else {
              float* ro = c.rec_o + rec * D + k * 32;
#pragma unroll
              for (int e = 0; e < 32; e += 8) {
                const uint32_t u[8] = {o[e], o[e + 1], o[e + 2], o[e + 3], o[e + 4], o[e + 5], o[e + 6], o[e + 7]};
                win_store32(ro + e, true, u);
              }
            }
          }
        }
        if (row_live && !direct) c.rec_ml[rec] = make_float2(m_ref, ok ? l_run : CUDART_NAN_F);
        if (ok && row_live && *(volatile int*)&it.poison) {
          if (direct) {
            restore_non_finite<D>(c, it, t, pos, [&](int d, float x) { dst[d] = __float2bfloat16_rn(__bfloat162float(dst[d]) + x); });
          } else {
            float* ro = c.rec_o + rec * D;
            restore_non_finite<D>(c, it, t, pos, [&](int d, float x) { ro[d] += x; });
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl->item_empty[gi & 1]);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWinOtherRegs));
    if (warp == 8) {
    // ================================================================ work and copies: one thread
    if (lane == 0) {
      unsigned kc = 0, vc = 0, nq[2] = {0, 0};
      int unit = c.spans ? ctl->first_unit : (int)blockIdx.x;
      int step = c.spans ? ctl->first_step : 0;
      bool ok = true;
      unsigned gi = 0;
      for (; ok;) {
        const bool more = c.spans ? span_at < span_end && unit < c.n_units : unit < c.n_units;
        WinItem w;
        w.unit = -1;
        if (more) {
          w.u = find_unit(c, unit, w.b, w.g, w.window, w.ctx);
          const int weight = w.u.weight();
          if (weight == 0) {   // no query in it
            if (c.spans) ++unit, step = 0;
            else unit = (int)gridDim.x + atomicAdd(c.queue, 1);
            continue;
          }
          w.unit = unit;
          w.poison = 0;
          if (c.spans) {
            const long long z = min((long long)weight, step + (span_end - span_at));
            const bool some = w.u.part(step, z, w.j0, w.j1);
            span_at += z - step;
            if (z == weight) ++unit, step = 0;
            else step = (int)z;
            if (!some) continue;
            w.slot = w.j0 == 0 && w.j1 == w.u.n_steps ? -1 : 2 * (int)blockIdx.x + (w.j0 == 0 ? 1 : 0);
            if (w.slot >= 0 && w.u.live <= c.tpt) w.u.share_steps();
          } else {
            w.j0 = 0;
            w.j1 = w.u.n_steps;
            w.slot = -1;
            unit = (int)gridDim.x + atomicAdd(c.queue, 1);
          }
        }
        if (gi >= 2) ok = mbar_wait(&ctl->item_empty[gi & 1], ((gi >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        ctl->item[gi & 1] = w;
        mbar_arrive(&ctl->item_full[gi & 1]);
        ++gi;
        if (!more) break;
        auto load_q = [&](int i) -> bool {
          const WinTileSteps& t = w.u.tile[i];
          if (t.steps_in(w.j0, w.j1) == 0) return true;
          if (nq[i] > 0 && !mbar_wait(&ctl->q_empty[i], (nq[i] - 1) & 1, abort_flag)) return false;
          mbar_arrive_expect_tx(&ctl->q_full[i], (uint32_t)(c.tpt * c.group * 128 * HALVES));
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
            tma_load_4d(q_tile + i * TB + h * kHalfBytes, &map_q, h * 64, w.g * c.group, t.tok, w.b, &ctl->q_full[i]);
          ++nq[i];
          return true;
        };
        ok = load_q(0);
        for (int j = w.j0; j < w.j1 && ok; ++j) {
          const int kt = w.u.key_tile(j);
          const int ks = kc % KS, vs = vc % VS;
          if (kc >= KS) ok = mbar_wait(&ctl->k_empty[ks], (kc / KS - 1) & 1, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(&ctl->k_full[ks], (uint32_t)TB);
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
            tma_load_4d(k_tile + ks * TB + h * kHalfBytes, &map_k, h * 64, kt * kWinTile, w.g, w.b, &ctl->k_full[ks]);
          ++kc;
          if (j == w.j0) ok = load_q(1);
          if (ok && vc >= VS) ok = mbar_wait(&ctl->v_empty[vs], (vc / VS - 1) & 1, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(&ctl->v_full[vs], (uint32_t)TB);
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
            tma_load_4d(v_tile + vs * TB + h * kHalfBytes, &map_v, h * 64, kt * kWinTile, w.g, w.b, &ctl->v_full[vs]);
          ++vc;
        }
      }
      ctl->issued_k = kc;
      ctl->issued_v = vc;
      ctl->issued_q[0] = nq[0];
      ctl->issued_q[1] = nq[1];
    }
    __syncwarp();
  } else if (warp == 9) {
    // ================================================================ matrix instructions: one thread
    if (lane == 0) {
      unsigned kc = 0, vc = 0, nq[2] = {0, 0}, np[2] = {0, 0};
      bool ok = true;
      // descriptors as words: only the start address (low word, 16-byte units) changes
      const uint64_t q_desc = operand_desc(smem_u32(q_tile)), k_desc = operand_desc(smem_u32(k_tile));
      const uint64_t v_desc = operand_desc_mn(smem_u32(v_tile), kHalfBytes, 1024);
      const uint32_t q_lo = (uint32_t)q_desc, k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc;
      const uint32_t kmajor_hi = (uint32_t)(k_desc >> 32), v_hi = (uint32_t)(v_desc >> 32);
      for (unsigned gi = 0; ok; ++gi) {
        ok = mbar_wait(&ctl->item_full[gi & 1], (gi >> 1) & 1, abort_flag);
        if (!ok) break;
        const WinItem& it = ctl->item[gi & 1];
        if (it.unit < 0) break;
        const int j0 = it.j0, j1 = it.j1;
        const WinTileSteps t0 = it.u.tile[0], t1 = it.u.tile[1];
        mbar_arrive(&ctl->item_empty[gi & 1]);
        const int cnt[2] = {t0.steps_in(j0, j1), t1.steps_in(j0, j1)};
        int left_q[2] = {cnt[0], cnt[1]}, left_p[2] = {cnt[0], cnt[1]};
        // S_i = Q_i K^T of the K tile in stage ks
        auto qk = [&](const int i, uint32_t ks) -> bool {
          if (left_q[i] == cnt[i]) {
            if (!mbar_wait(&ctl->q_full[i], nq[i] & 1, abort_flag)) return false;
            ++nq[i];
          }
          tc_fence_after();
          const uint32_t a_lo = q_lo + (uint32_t)i * (TB >> 4), b_lo = k_lo + ks * (TB >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = (uint32_t)((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
            win_umma(tmem + (uint32_t)(i * kWinTile), a_lo + off, kmajor_hi, b_lo + off, kmajor_hi, kIdescQK, kk > 0);
          }
          umma_commit(&ctl->s_full[i]);
          if (--left_q[i] == 0) umma_commit(&ctl->q_empty[i]);
          return true;
        };
        // O_i += P_i V of the V tile in stage vs
        auto pv = [&](const int i, uint32_t vs) -> bool {
          const uint32_t b_lo = v_lo + vs * (TB >> 4), s_col = tmem + (uint32_t)(i * kWinTile);
          const uint32_t more = left_p[i] != cnt[i];   // the accumulator holds products of this item
#pragma unroll
          for (int kk = 0; kk < kWinTile / 16; ++kk) {   // 16 tokens per instruction: 8 columns of bf16 pairs
            if (kk % (kWinTile / 16 / kParts) == 0) {
              if (!mbar_wait(&ctl->p_full[i][kk / (kWinTile / 16 / kParts)], np[i] & 1, abort_flag)) return false;
              tc_fence_after();
            }
            win_umma_tmem_a(tmem + 2 * kWinTile + (uint32_t)(i * kWinTile), s_col + (uint32_t)(kk * 8),
                            b_lo + (uint32_t)(kk * 16 * 128 >> 4), v_hi, kIdescPV, kk > 0 ? 1u : more);
          }
          ++np[i];
          if (--left_p[i] == 0) umma_commit(&ctl->o_full[i]);
          return true;
        };
        if (j0 < j1) {
          const uint32_t ks = kc % KS;
          ok = mbar_wait(&ctl->k_full[ks], (kc / KS) & 1, abort_flag);
          if (ok && t0.active(j0)) ok = qk(0, ks);
          if (ok && t1.active(j0)) ok = qk(1, ks);
          if (!ok) break;
          umma_commit(&ctl->k_empty[ks]);
          ++kc;
        }
        for (int j = j0; j < j1 && ok; ++j) {
          const uint32_t ks = kc % KS, vs = vc % VS;
          const bool next = j + 1 < j1;
          ok = mbar_wait(&ctl->v_clean[vs], (vc / VS) & 1, abort_flag);
          if (ok && t0.active(j)) ok = pv(0, vs);
          if (ok && next) {
            ok = mbar_wait(&ctl->k_full[ks], (kc / KS) & 1, abort_flag);
            if (ok && t0.active(j + 1)) ok = qk(0, ks);
          }
          if (ok && t1.active(j)) ok = pv(1, vs);
          if (!ok) break;
          umma_commit(&ctl->v_empty[vs]);
          ++vc;
          if (next) {
            if (t1.active(j + 1)) ok = qk(1, ks);
            if (!ok) break;
            umma_commit(&ctl->k_empty[ks]);
            ++kc;
          }
        }
      }
    }
    __syncwarp();
  } else {
    // ================================================================ a look over the V tiles that are partly masked
    const int me = (int)threadIdx.x - 320;   // 0 .. 63
    unsigned vc = 0;
    bool ok = true;
    for (unsigned gi = 0; ok; ++gi) {
      ok = __all_sync(0xffffffffu, mbar_wait(&ctl->item_full[gi & 1], (gi >> 1) & 1, abort_flag));
      if (!ok) break;
      WinItem& it = ctl->item[gi & 1];
      if (it.unit < 0) break;
      for (int j = it.j0; j < it.j1 && ok; ++j, ++vc) {
        const int vs = vc % VS, kt = it.u.key_tile(j);
        ok = __all_sync(0xffffffffu, mbar_wait(&ctl->v_full[vs], (vc / VS) & 1, abort_flag));
        if (!ok) break;
        bool look = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const WinTileSteps& t = it.u.tile[i];
          look |= t.active(j) && win_masked(kt, t.pos, t.pos + t.n_tok - 1, it.window, c.n_sink);
        }
        if (look) {
          uint4* p = (uint4*)(v_tile + vs * TB);
          const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
          __nv_bfloat162 acc = zero;   // x * 0 is 0 or NaN
#pragma unroll 8
          for (int k = me; k < TB / 16; k += 64) {
            const uint4 u = p[k];
            acc = __hfma2(*(const __nv_bfloat162*)&u.x, zero, acc);
            acc = __hfma2(*(const __nv_bfloat162*)&u.y, zero, acc);
            acc = __hfma2(*(const __nv_bfloat162*)&u.z, zero, acc);
            acc = __hfma2(*(const __nv_bfloat162*)&u.w, zero, acc);
          }
          if (!finite_bf16(acc.x) || !finite_bf16(acc.y)) {
            // zeroed; whether a query of the unit sees one of them decides on the looking for them later
            bool seen = false;
            for (int k = me; k < TB / 16; k += 64) {
              const uint4 u = p[k];
              const uint4 f = make_uint4(finite_or_zero2(u.x), finite_or_zero2(u.y), finite_or_zero2(u.z), finite_or_zero2(u.w));
              if (f.x == u.x && f.y == u.y && f.z == u.z && f.w == u.w) continue;
              p[k] = f;
              const int n = kt * kWinTile + k * 16 % kHalfBytes / 128;   // (the swizzle stays within a row)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const WinTileSteps& t = it.u.tile[i];
                seen |= t.active(j) && win_seen(n, t.pos, t.pos + t.n_tok - 1, it.window, c.n_sink);
              }
            }
            if (seen) {
              *(volatile int*)&it.poison = 1;
              __threadfence_block();
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        mbar_arrive(&ctl->v_clean[vs]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl->item_empty[gi & 1]);
    }
    }
  }
  tc_fence_before();
  __syncthreads();
  // Every role has left, so the flag and the counts are final.  A role that gave up may have left behind copies or instructions
  // that nobody waited for, of roles that had long ended well: the copies must land before the CTA may exit, the instructions
  // finish before tensor memory is released.
  if (*abort_flag) {
    if (warp == 8 && lane == 0) {
      const unsigned kc = ctl->issued_k, vc = ctl->issued_v;
      for (int i = 0; i < 2; ++i)
        if (ctl->issued_q[i] > 0) (void)mbar_wait_drain(&ctl->q_full[i], (ctl->issued_q[i] - 1) & 1);
      for (unsigned x = kc > KS ? kc - KS : 0; x < kc; ++x) (void)mbar_wait_drain(&ctl->k_full[x % KS], (x / KS) & 1);
      for (unsigned x = vc > VS ? vc - VS : 0; x < vc; ++x) (void)mbar_wait_drain(&ctl->v_full[x % VS], (x / VS) & 1);
    }
    if (warp == 9 && lane == 0) {
      umma_commit(&ctl->drain);
      (void)mbar_wait_drain(&ctl->drain, 0);
    }
    __syncwarp();
  }
  if (c.spans && threadIdx.x == 0) c.done[blockIdx.x] = *abort_flag == 0;
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Folds the records of the units that spans have cut, part by part in order: a warp per row.  A CTA that gave up has left
// records unwritten, so a unit with a part of such a one is NaN.  grid = (units, row blocks), block = 256.
template <int D>
__global__ void __launch_bounds__(256) window_combine_kernel(const __grid_constant__ WinCall c) {
  cudaGridDependencySynchronize();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int2 spans = __ldcg(&c.table[blockIdx.x]);
  const int s0 = spans.x, parts = spans.y;
  if (parts <= 1) return;   // in one piece
  bool lost = false;
  for (int p = lane; p < parts; p += 32) lost |= __ldcg(&c.done[s0 + p]) == 0;
  lost = __any_sync(0xffffffffu, lost);
  int b, g, window, ctx;
  const WinUnit u = find_unit(c, blockIdx.x, b, g, window, ctx);
  const int rows = u.live * c.group;   // (query token of the unit, query head)
  for (int row = blockIdx.y * 8 + warp; row < rows; row += gridDim.y * 8) {
  // (a unit whose queries fit a tile has been shared by both: two records a part)
  const int per = u.live <= c.tpt ? 2 : 1, records = parts * per;
  float m = -CUDART_INF_F, l = 0.f;
  LaneVec<D> acc;
  acc.zero();
  constexpr int U = 8;
  for (int p0 = 0; p0 < records; p0 += U) {
    float2 mls[U];
    LaneVec<D> os[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int p = min(p0 + i, records - 1), part = p / per;   // beyond the end: read again, unused
      const size_t r = (size_t)(2 * (s0 + part) + (part == 0 ? 1 : 0)) * c.rec_rows + (size_t)(p % per) * c.rec_tile * c.group + row;
      mls[i] = __ldcg(&c.rec_ml[r]);
      os[i].load_l2(c.rec_o + r * D, lane);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (p0 + i >= records) break;
      const float2 ml = mls[i];
      const float mn = fmaxf(m, ml.x);
      const float mu = (mn == -CUDART_INF_F) ? 0.f : mn;
      const float c_old = fast_exp2(m - mu), c_new = fast_exp2(ml.x - mu);
      l = l * c_old + ml.y * c_new;
      acc.scale(c_old);
      acc.fma(c_new, os[i]);
      m = mn;
    }
  }
  acc.scale(lost ? CUDART_NAN_F : (m == -CUDART_INF_F && !isnan(l) ? 0.f : 1.f / l));
  __nv_bfloat16* dst = c.out + (((size_t)b * c.n_tokens + u.tile[0].tok + row / c.group) * c.n_q_heads + (size_t)g * c.group + row % c.group) * D;
  if constexpr (D == 128) {
    *(uint2*)(dst + lane * 4) = make_uint2(win_pack2(acc.v.x, acc.v.y), win_pack2(acc.v.z, acc.v.w));
  } else {
    *(uint32_t*)(dst + lane * 2) = win_pack2(acc.v.x, acc.v.y);
  }
  }
}

// X[d3][d2][d1][D] bf16 with boxes of 64 elements x n1 x n2 rows, 128-byte swizzle; what lies outside reads as zero.
// Strides in elements; one of a dimension of size 1 does not matter.
bool make_map(CUtensorMap* map, const void* X, int D, int64_t d1, int64_t s1, int64_t d2, int64_t s2, int64_t d3, int64_t s3,
              int n1, int n2) {
  const EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) return false;
  if (d1 == 1) s1 = D;
  if (d2 == 1) s2 = D;
  if (d3 == 1) s3 = D;
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)d1, (cuuint64_t)d2, (cuuint64_t)d3};
  const cuuint64_t strides[3] = {(cuuint64_t)s1 * 2, (cuuint64_t)s2 * 2, (cuuint64_t)s3 * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)n1, (cuuint32_t)n2, 1};
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(X), dims, strides, box, es,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch_window(const WinCall& c, const void* q, int64_t q_b, int64_t q_t, const void* k, const void* v, int64_t kv_b,
                          int64_t kv_h, int64_t kv_n, int n_sms, cudaStream_t s) {
  CUtensorMap map_q, map_k, map_v;
  if (!make_map(&map_q, q, D, c.n_q_heads, D, c.n_tokens, q_t, c.batch, q_b, c.group, c.tpt) ||
      !make_map(&map_k, k, D, c.n_ctx, kv_n, c.n_kv_heads, kv_h, c.batch, kv_b, kWinTile, 1) ||
      !make_map(&map_v, v, D, c.n_ctx, kv_n, c.n_kv_heads, kv_h, c.batch, kv_b, kWinTile, 1))
    return cudaErrorInvalidValue;
  static bool opted_in[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !opted_in[dev]) {
    // (a block launched with fewer registers than its warpgroups share out would wait for them for ever)
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, window_kernel<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs < kWinLaunchRegs) return cudaErrorInvalidConfiguration;
    e = cudaFuncSetAttribute(window_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)win_smem_bytes<D>());
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) opted_in[dev] = true;
  }
  const int ctas = std::min(n_sms, kWinMaxSpans);
  if (!c.spans) {
    e = cudaMemsetAsync(c.queue, 0, sizeof(int32_t), s);
    if (e != cudaSuccess) return e;
  }
  window_kernel<D><<<ctas, kWinThreads, win_smem_bytes<D>(), s>>>(map_q, map_k, map_v, c);
  e = cudaGetLastError();
  if (e != cudaSuccess || !c.spans) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(c.n_units, std::min(16, (c.rec_rows + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, window_combine_kernel<D>, c);
}

// Workspace: queue and `done` (256 bytes) | table of units | (m, l) records | o records.
constexpr size_t kWinDoneOffset = 64;
static_assert(kWinDoneOffset + kWinMaxSpans <= 256, "beside the queue");
struct WinLayout {
  size_t table, rec_ml, rec_o, total;
  int group, tpt, pairs, rec_rows;
  long long units;
};
int win_layout(int batch, int n_q_heads, int n_kv_heads, int head_dim, int n_tokens, WinLayout& l) {
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_tokens < 0 || n_tokens > (1 << 30)) return RAZOR_E_INVALID_ARG;
  if (n_q_heads % n_kv_heads) return RAZOR_E_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || n_q_heads / n_kv_heads > kWinTile) return RAZOR_E_UNSUPPORTED_DIM;
  l.group = n_q_heads / n_kv_heads;
  l.tpt = kWinTile / l.group;
  l.pairs = (n_tokens + 2 * l.tpt - 1) / (2 * l.tpt);
  l.units = (long long)l.pairs * batch;
  if (l.units > (1LL << 30)) return RAZOR_E_CAPACITY;   // (before the next factor: all three need not fit 64 bits)
  l.units *= n_kv_heads;
  if (l.units > (1LL << 30)) return RAZOR_E_CAPACITY;
  l.rec_rows = 2 * std::min(l.tpt, n_tokens) * l.group;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t off = 256;
  l.table = l.rec_ml = l.rec_o = off;
  if (l.units <= kWinSpanUnits) {
    off = up(off + (size_t)l.units * sizeof(int2));
    l.rec_ml = off;
    off = up(off + (size_t)2 * kWinMaxSpans * l.rec_rows * sizeof(float2));
    l.rec_o = off;
    off = up(off + (size_t)2 * kWinMaxSpans * l.rec_rows * head_dim * sizeof(float));
  }
  l.total = off;
  return RAZOR_OK;
}

}  // namespace
}  // namespace razor

extern "C" int razor_window_attention_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                      int32_t n_tokens, size_t* bytes) {
  if (!bytes) return RAZOR_E_NULL_PTR;
  razor::WinLayout l;
  const int rc = razor::win_layout(batch, n_q_heads, n_kv_heads, head_dim, n_tokens, l);
  if (rc) return rc;
  *bytes = l.total;
  return RAZOR_OK;
}

namespace razor {
namespace {
int window_call(const void* q, int64_t q_stride_b, int64_t q_stride_t, const void* K, const void* V, int64_t kv_stride_b,
                int64_t kv_stride_h, int64_t kv_stride_n, const int32_t* window, const int32_t* q_len, const int32_t* ctx_len,
                int32_t batch, int32_t n_tokens, int32_t n_ctx, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                int32_t n_sink, float sm_scale, void* out, void* workspace, size_t workspace_bytes, int32_t stopped_cta, void* stream) {
  WinLayout l;
  const int rc = win_layout(batch, n_q_heads, n_kv_heads, head_dim, n_tokens, l);
  if (rc) return rc;
  if (dtype != RAZOR_BF16) return RAZOR_E_UNSUPPORTED_DIM;
  if (n_ctx < 1 || n_ctx > (1 << 30) || n_sink < 0) return RAZOR_E_INVALID_ARG;
  if (!(sm_scale >= 0.f) || std::isinf(sm_scale)) return RAZOR_E_INVALID_ARG;
  if (n_tokens == 0) return RAZOR_OK;
  if (!q || !K || !V || !out || !workspace) return RAZOR_E_NULL_PTR;
  if (((uintptr_t)q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)out) & 15) return RAZOR_E_MISALIGNED;
  if ((uintptr_t)workspace & 255) return RAZOR_E_MISALIGNED;
  if (((uintptr_t)window | (uintptr_t)q_len | (uintptr_t)ctx_len) & 3) return RAZOR_E_MISALIGNED;
  // strides that separate nothing are not looked at
  const int64_t st[5] = {batch > 1 ? q_stride_b : head_dim, n_tokens > 1 ? q_stride_t : head_dim, batch > 1 ? kv_stride_b : head_dim,
                         n_kv_heads > 1 ? kv_stride_h : head_dim, n_ctx > 1 ? kv_stride_n : head_dim};
  for (int i = 0; i < 5; ++i) {
    if (st[i] < head_dim || st[i] > (1LL << 36)) return RAZOR_E_INVALID_ARG;
    if ((st[i] * 2) & 15) return RAZOR_E_MISALIGNED;
  }
  if (workspace_bytes < l.total) return RAZOR_E_POOL_TOO_SMALL;
  WinCall c = {};
  c.q_len = q_len; c.ctx_len = ctx_len; c.window = window;
  c.v = (const __nv_bfloat16*)V; c.out = (__nv_bfloat16*)out;
  c.v_stride_b = st[2]; c.v_stride_h = st[3]; c.v_stride_n = st[4];
  c.batch = batch; c.n_tokens = n_tokens; c.n_ctx = n_ctx; c.n_q_heads = n_q_heads; c.n_kv_heads = n_kv_heads;
  c.group = l.group; c.tpt = l.tpt; c.n_sink = n_sink; c.n_units = (int)l.units; c.pairs = l.pairs;
  c.spans = l.units <= kWinSpanUnits;
  c.out_whole = ((uintptr_t)out & 31) == 0;
  c.rec_rows = l.rec_rows;
  c.rec_tile = std::min(l.tpt, n_tokens);
  c.scale_log2 = (sm_scale == 0.f ? 1.0f / sqrtf((float)head_dim) : sm_scale) * 1.4426950408889634f;
  c.stopped_cta = stopped_cta;
  uint8_t* ws = (uint8_t*)workspace;
  c.queue = (int32_t*)ws;
  c.done = ws + kWinDoneOffset;
  c.table = (int2*)(ws + l.table);
  c.rec_ml = (float2*)(ws + l.rec_ml);
  c.rec_o = (float*)(ws + l.rec_o);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess)
    e = head_dim == 128
            ? launch_window<128>(c, q, st[0], st[1], K, V, st[2], st[3], st[4], sms, (cudaStream_t)stream)
            : launch_window<64>(c, q, st[0], st[1], K, V, st[2], st[3], st[4], sms, (cudaStream_t)stream);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    return RAZOR_E_CUDA;
  }
  return RAZOR_OK;
}

}  // namespace
}  // namespace razor

extern "C" int razor_window_attention(const void* q, int64_t q_stride_b, int64_t q_stride_t, const void* K, const void* V,
                                      int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_n, const int32_t* window,
                                      const int32_t* q_len, const int32_t* ctx_len, int32_t batch, int32_t n_tokens, int32_t n_ctx,
                                      int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t n_sink,
                                      float sm_scale, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return razor::window_call(q, q_stride_b, q_stride_t, K, V, kv_stride_b, kv_stride_h, kv_stride_n, window, q_len, ctx_len, batch,
                            n_tokens, n_ctx, n_q_heads, n_kv_heads, head_dim, dtype, n_sink, sm_scale, out, workspace,
                            workspace_bytes, -1, stream);
}

extern "C" int razor_window_attention_wait_selftest(const void* q, int64_t q_stride_b, int64_t q_stride_t, const void* K,
                                                    const void* V, int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_n,
                                                    const int32_t* window, const int32_t* q_len, const int32_t* ctx_len,
                                                    int32_t batch, int32_t n_tokens, int32_t n_ctx, int32_t n_q_heads,
                                                    int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t n_sink,
                                                    float sm_scale, void* out, void* workspace, size_t workspace_bytes,
                                                    int32_t cta, void* stream) {
  if (cta < 0) return RAZOR_E_INVALID_ARG;
  return razor::window_call(q, q_stride_b, q_stride_t, K, V, kv_stride_b, kv_stride_h, kv_stride_n, window, q_len, ctx_len, batch,
                            n_tokens, n_ctx, n_q_heads, n_kv_heads, head_dim, dtype, n_sink, sm_scale, out, workspace,
                            workspace_bytes, cta, stream);
}
