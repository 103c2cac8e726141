// Attention of a tree of drafted tokens over a bf16 cache, on the tensor cores.
//
// The work per KV head is a short block of query rows (nodes x query heads of the group: from one to a thousand)
// against a long stream of tokens, so the products are taken the other way round from a prompt's: TOKENS are the
// 128-row operand and the query rows the narrow one,
//     S^T = K Q^T          [128 tokens x R rows],     R = 32, 64 or 128 rows of a tile,
//     O^T = V^T P^T        [D x R rows], contraction over the tokens,
// and no lane of the tensor memory, no tensor-core row and no softmax thread stands idle when the rows are few.  A thread
// owns one token, which also makes masks cheap: beyond the head's end, or which nodes see this draft, is decided per
// thread.  Query rows are columns, independent of one another: whatever a dead or poisoned row holds stays in its own
// column.  P goes through shared memory as a bf16 head plus a bf16 remainder, side by side as 2R columns of one product
// (the V operand is read once for both), so that a weight keeps fp32-like accuracy; the two halves of the accumulator are
// added at the end.
//
// Work: every head's slots in steps of 128 tokens plus one step for the tree's own tokens (their visibility is a bit mask
// per thread).  All heads' steps are laid end to end and cut into equal spans, one per CTA; with several tiles of rows
// the tiles of a span run in neighbouring CTAs at the same time, so that the cache comes out of HBM once and out of L2 for
// the others.  The cut is made on the device from the head states - a scan over the heads, about a microsecond - so a
// call costs the host nothing but the launch, and a captured graph follows the cache as it grows.  A head that a cut runs
// through leaves one partial record per span; tree_combine_kernel folds them.
//
// A CTA (one per SM): softmax warps (one per tensor-memory lane quarter and group of columns), a producer
// warp (TMA: pages of the pool, whose rows are stored in the swizzle of the operand layout; drafts and queries through
// maps of their own) and a warp that issues the matrix instructions.  S is double-buffered, so the scores of the next
// step are computed during the softmax of this one.
//
// The running maximum of a row is a reference that may lag: weights are 2^(s - m), floats, as exact at 2^20 as at one.  It
// is moved (and the accumulator rescaled) only when a score outruns it by 2^kLag; the four warps of a column group agree on
// that once per step, and compute their weights while the agreement is on its way.
//
// Every wait is bounded in time; a wait that runs out sets the CTA's abort flag and a bit of the device status word,
// copies and instructions in flight are waited for, tensor memory is released.
#include <math_constants.h>

#include <algorithm>

#include "razor_common.cuh"
#include "razor_sync.cuh"
#include "razor_tc.cuh"
#include "razor_tree.cuh"

namespace razor {
namespace {

constexpr int kTok = 128;                       // tokens of a step = tensor-memory lanes
constexpr int kStepPages = kTok / kPageTokens;
// Eight softmax warps: two groups of columns, four warps each (one per tensor-memory lane quarter).  (Sixteen warps with
// half as many columns each had 104 registers apiece and spilled, and next to 227 KB of shared memory there is no L1 to
// spill to: slower for 64 rows and for 128.)  Two further warps feed them, and two have no part.
constexpr int kGroups = 2, kSoftWarps = 4 * kGroups, kTreeThreads = (kSoftWarps + 4) * 32;
constexpr int kFlush = 16;                      // steps whose products add up in tensor memory
constexpr int kItemSlots = 3;
constexpr int kMaxStages = 4;                   // of K and of V
constexpr float kLag = 20.f;                    // log2 of how far a weight may outgrow the reference maximum
constexpr float kLow = -3.0e38f;                // stands for a reference maximum of minus infinity in the arithmetic

struct TreeItem {
  int32_t head;          // b * Hkv + kv_head; -1: no more items
  int32_t begin, end;    // steps of the cache
  int32_t draft;         // 1: the tree's own tokens follow
  int32_t rec;           // record this part leaves; -1: the head is whole and its output is written
  int32_t seed;          // 1: carries the compensation token
  HeadState st;
};

template <int R>
struct TreeCtl {
  uint64_t q_full, q_empty;
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
  uint64_t s_full[2], s_empty[2];     // per S buffer
  uint64_t p_full, p_done;            // the weights are in shared memory; the product that read them has run
  uint64_t o_read;                    // the accumulator has been read out
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  uint64_t agree[kGroups];   // the four warps of a column group among themselves
  uint64_t all_sync;                  // the softmax warps among themselves
  uint64_t drain;
  uint32_t tmem_base;
  int abort_flag;
  uint32_t need[kGroups][2]; // [column group][step parity]: step + 1 when a score outran the reference
  uint32_t bad_v[2][kTreeMaxNodes / 32];   // [item parity]: drafts whose V holds a NaN or an infinity
  TreeItem item[kItemSlots];
  alignas(16) float neg_m[R];                     // minus the reference maximum of each row (log2 domain)
  int32_t top[2][R];                  // column maxima while the reference moves, as ordered integers
  alignas(16) float slope[R];
  alignas(16) float depth[R];           // ALiBi only
};

template <int D, int R>
struct TreeSmem {
  static constexpr int kKv = kTok * D * 2;             // one stage of K or of V
  static constexpr int kQ = R * D * 2;
  static constexpr int kP = kTok * 2 * R * 2;
  static constexpr int kMax = 232448;
  static constexpr int kRoom = kMax - kQ - kP - (int)sizeof(TreeCtl<R>);
  static constexpr int kK = kRoom / (2 * kKv) < kMaxStages ? kRoom / (2 * kKv) : kMaxStages;   // stages
  static constexpr int kV = kRoom / kKv - kK < kMaxStages ? kRoom / kKv - kK : kMaxStages;     // (one left over goes to V: it is held a step longer)
  static constexpr int kBytes = (kK + kV) * kKv + kQ + kP + (int)sizeof(TreeCtl<R>);
  static_assert(kV >= 2 && kK >= 2 && kBytes <= kMax, "shared memory");
};

__device__ __forceinline__ void tma5(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, int c4, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::
          "r"(smem_u32(dst)),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
// One matrix instruction with the operand descriptors given as (low word, high word).  The start address is in the low
// word, in 16-byte units, so a walk along an operand is one 32-bit addition.
__device__ __forceinline__ void umma_words(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                           uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
      :
      : "r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// NC consecutive columns of this thread's lane, in registers when the function returns.
template <int NC>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&v)[NC]) {
#pragma unroll
  for (int c = 0; c < NC; c += 16) tmem_ld16_issue(taddr + (uint32_t)c, v + c);
  tmem_ld_wait_all();
#pragma unroll
  for (int c = 0; c < NC; ++c) asm volatile("" : "+r"(v[c]));
}
// Floats as integers of the same order.
__device__ __forceinline__ int ordered(float x) { const int i = __float_as_int(x); return i < 0 ? i ^ 0x7fffffff : i; }
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }

// Sums (or maxima) over the warp of NC (16 or 32) values per lane: lane c (mod NC) gets that of x[c].  Destroys x.
template <int NC, bool kMax>
__device__ __forceinline__ float across_warp(float* x, int lane) {
  auto join = [](float a, float b) { return kMax ? fmaxf(a, b) : a + b; };
  if constexpr (NC == 16) {
#pragma unroll
    for (int c = 0; c < 16; ++c) x[c] = join(x[c], __shfl_xor_sync(0xffffffffu, x[c], 16));
  }
#pragma unroll
  for (int half = NC / 2; half > 0; half >>= 1) {
    const bool up = (lane & half) != 0;
#pragma unroll
    for (int c = 0; c < half; ++c) {
      const float send = up ? x[c] : x[c + half], keep = up ? x[c + half] : x[c];
      x[c] = join(keep, __shfl_xor_sync(0xffffffffu, send, half));
    }
  }
  return x[0];
}

// A whole warp waits; every lane gets the same answer.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
// One arrival for a warp's 32 threads, behind everything they did.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

__device__ __forceinline__ int head_steps(int len) { return (len + kTok - 1) / kTok; }

// Is node n node t or an ancestor of it?  (Straight from the parents: only where a draft holds a NaN or an infinity.)
__device__ __noinline__ bool walk_sees(const int32_t* parent, int t, int n) {
  while (t > n) {
    const int a = parent[t];
    if (a < -1 || a >= t) return false;
    t = a;
  }
  return t == n;
}

template <int D, int R, bool kAlibi>
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_mma_kernel(DeviceView dv, const __grid_constant__ CUtensorMap map_pool, const __grid_constant__ CUtensorMap map_q,
                    const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, int layer, TreeCall tc) {
  using Smem = TreeSmem<D, R>;
  using Ctl = TreeCtl<R>;
  constexpr int HALVES = D / 64, KV = Smem::kKv, NK = Smem::kK, NV = Smem::kV;
  constexpr int SW = kSoftWarps, NT = kTreeThreads;
  constexpr int NC = R / kGroups;                       // columns of a softmax warp: 16, 32, 64
  constexpr int LC = NC > 32 ? 2 : 1, LW = NC / LC;     // columns whose bookkeeping a lane carries, LW apart
  constexpr uint32_t kOctet = 8 * D * 2;                // bytes of eight tokens in a stage: [octet][64-element half][8][128 B]
  constexpr uint32_t kTmemCols = 4 * R, kOCol = 2 * R;  // S, S, O (heads), O (remainders)
  constexpr uint32_t kIdescS = instr_desc_bf16(kTok, R, false);
  constexpr uint32_t kIdescO = instr_desc_bf16(kTok, 2 * R, true) | (1u << 15);   // (bit 15: A is MN-major too)

  extern __shared__ __align__(1024) uint8_t tree_smem[];
  uint8_t* k_ring = tree_smem;
  uint8_t* v_ring = k_ring + NK * KV;
  uint8_t* p_tile = v_ring + NV * KV;                   // [64-column block][token][128 B], chunks swizzled by the token
  uint8_t* q_tile = p_tile + Smem::kP;                  // [half][row][128 B]
  Ctl* ctl = (Ctl*)(q_tile + Smem::kQ);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &ctl->abort_flag;
  const int G = dv.group, lg = __ffs(G) - 1, n_nodes = tc.n_nodes;   // (the group is a power of two)
  const int tile = blockIdx.x % tc.n_tiles, span = blockIdx.x / tc.n_tiles;
  const HeadState* states = dv.state + (size_t)layer * dv.n_heads;
  if (smem_u32(tree_smem) & 1023u) {   // (the operand layouts need it; the first byte of a CTA's dynamic shared memory is)
    if (tid == 0) atomicOr(dv.status, kStatusProducerTimeout);
    return;
  }

  if (tid == 0) {
    mbar_init(&ctl->q_full, 1);
    mbar_init(&ctl->q_empty, 1);
    for (int s = 0; s < NK; ++s) { mbar_init(&ctl->k_full[s], 1); mbar_init(&ctl->k_empty[s], 1); }
    for (int s = 0; s < NV; ++s) { mbar_init(&ctl->v_full[s], 1); mbar_init(&ctl->v_empty[s], 1); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&ctl->s_full[s], 1);
      mbar_init(&ctl->s_empty[s], SW);
    }
    for (int s = 0; s < kGroups; ++s) {
      mbar_init(&ctl->agree[s], 4);
      ctl->need[s][0] = ctl->need[s][1] = 0;
    }
    mbar_init(&ctl->p_full, SW);
    mbar_init(&ctl->p_done, 1);
    mbar_init(&ctl->o_read, SW);
    for (int s = 0; s < kItemSlots; ++s) { mbar_init(&ctl->item_full[s], 1); mbar_init(&ctl->item_empty[s], SW + 1); }
    mbar_init(&ctl->all_sync, SW);
    mbar_init(&ctl->drain, 1);
    ctl->abort_flag = 0;
    for (int k = 0; k < 2 * kTreeMaxNodes / 32; ++k) ctl->bad_v[0][k] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == SW + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int c = tid; c < 2 * R; c += NT) ctl->top[0][c] = ordered(-CUDART_INF_F);

  // ---- this CTA's span: a scan over the heads' steps (scratch: the tile of P)
  long long* warp_tot = (long long*)p_tile;
  int* found = (int*)(p_tile + 256);   // head and step the span begins with, and the head's state
  long long* bounds = (long long*)(p_tile + 512);
  {
    const int per = (dv.n_heads + NT - 1) / NT;
    const int h0 = min(dv.n_heads, tid * per), h1 = min(dv.n_heads, h0 + per);
    long long mine = 0;
    for (int h = h0; h < h1; ++h) mine += head_steps(states[h].len) + 1;
    long long upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += y;
    }
    if (lane == 31) warp_tot[warp] = upto;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    long long before = 0, total = 0;
    for (int w = 0; w < NT / 32; ++w) {
      if (w < warp) before += warp_tot[w];
      total += warp_tot[w];
    }
    before += upto - mine;
    const int n = (int)min((long long)tc.n_spans, max(1LL, (total + tc.min_span - 1) / tc.min_span));
    auto cut = [&](int s) { return total * s / n; };
    const long long x0 = span < n ? cut(span) : total, x1 = span < n ? cut(span + 1) : total;
    if (x0 < x1 && before <= x0 && x0 < before + mine) {
      long long u0 = before;
      int h = h0, w = head_steps(states[h0].len) + 1;
      while (u0 + w <= x0) {
        u0 += w;
        h += 1;
        w = head_steps(states[h].len) + 1;
      }
      found[0] = h;
      found[1] = (int)(x0 - u0);
      *(HeadState*)(found + 4) = states[h];
      bounds[0] = x1 - x0;
      // the span in which a head is cut for the first time lists it for the combine kernel
      TreeUnit u{h, span - 1, 0, 0};
      if (x0 > u0 && cut(span - 1) <= u0) {
        int e = span;
        while (e + 1 < n && cut(e + 1) < u0 + w) e += 1;
        u.n_parts = e - span + 2;
      }
      if (tile == 0) dv.tree_units[span] = u;
    }
    if (x0 >= x1 && tile == 0 && tid == 0) dv.tree_units[span] = TreeUnit{0, 0, 0, 0};
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem_base;
  const int first_head = found[0], first_step = found[1];
  const long long span_len = first_head >= 0 ? bounds[0] : 0;
  const HeadState first_state = first_head >= 0 ? *(const HeadState*)(found + 4) : HeadState{0, 0, 0, 0};
  __syncthreads();   // (the scratch becomes the tile of P)

  // Registers: the last warpgroup hands over what it does not need (3 x 128 x 168 at launch = 2 x 128 x 224 + 128 x 56).
  if (warp >= SW) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == SW) {
    // ================================================================ producer: items and TMA copies
    unsigned gk = 0, gi = 0, gq = 0;   // steps issued, items published, query tiles issued
    int head = first_head, y = first_step;
    long long todo = span_len;
    bool ok = true;
    HeadState st = first_state;
    for (;; ++gi) {
      TreeItem it;
      it.head = todo > 0 ? head : -1;
      it.begin = it.end = it.draft = it.seed = 0;
      it.rec = -1;
      it.st = st;
      const int steps = head_steps(st.len);
      if (todo > 0) {
        const int y1 = (int)min((long long)(steps + 1), y + todo);
        it.begin = y;
        it.end = min(y1, steps);
        it.draft = y1 == steps + 1;
        it.seed = y == 0 && dv.use_comp && st.n_drop > 0 && st.window >= 0;
        if (y > 0 || !it.draft) it.rec = ((int)blockIdx.x * 2 + (y > 0 ? 0 : 1));
        todo -= y1 - y;
      }
      const int slot = gi % kItemSlots;
      if (gi >= kItemSlots) ok = warp_wait(&ctl->item_empty[slot], (gi / kItemSlots - 1) & 1, abort_flag);
      if (!ok) break;
      if (lane == 0) {
        ctl->item[slot] = it;
        mbar_arrive(&ctl->item_full[slot]);
      }
      if (it.head < 0) break;
      const HeadState st_next = todo > 0 ? states[head + 1] : st;
      const int b = head / dv.n_kv_heads, g = head % dv.n_kv_heads;
      const size_t hs = (size_t)layer * dv.n_heads + head;
      const int32_t* pt = dv.page_table + hs * dv.max_pages;
      const int head_pages = (st.len + kPageTokens - 1) / kPageTokens;
      auto page_of = [&](int step) { return lane < kStepPages && step * kStepPages + lane < head_pages ? pt[step * kStepPages + lane] : 0; };
      int pid = it.begin < it.end ? page_of(it.begin) : 0;
      // the tile's queries: free once the scores of the item before have been computed
      if (gi >= 1) ok = warp_wait(&ctl->q_empty, (gi - 1) & 1, abort_flag);
      if (!ok) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(&ctl->q_full, (uint32_t)Smem::kQ);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) tma5(q_tile + h * R * 128, &map_q, 0, g * G, tile * (R / G), h, b, &ctl->q_full);
      }
      gq += 1;
      for (int step = it.begin; step < it.end + it.draft; ++step, ++gk) {
        const bool draft = step == it.end;
        const int sk = gk % NK, sv = gk % NV;
        const int n_pages = draft ? 0 : min(kStepPages, head_pages - step * kStepPages);
        const int n_oct = (n_nodes + 15) / 16 * 2;   // (the matrix instruction takes 16 tokens at a time; rows beyond the tree read zero)
        const uint32_t bytes = draft ? (uint32_t)n_oct * kOctet : (uint32_t)n_pages * 2 * kOctet;
        const int pid_next = step + 1 < it.end ? page_of(step + 1) : 0;
        if (gk >= (unsigned)NK) ok = warp_wait(&ctl->k_empty[sk], (gk / NK - 1) & 1, abort_flag);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&ctl->k_full[sk], bytes);
        __syncwarp();
        if (draft) {
          if (lane < n_oct) tma5(k_ring + sk * KV + lane * kOctet, &map_k, 0, lane * 8, 0, g, b, &ctl->k_full[sk]);
        } else if (lane < n_pages) {
          tma5(k_ring + sk * KV + lane * 2 * kOctet, &map_pool, 0, 0, 0, 0, 2 * pid, &ctl->k_full[sk]);
        }
        if (gk >= (unsigned)NV) ok = warp_wait(&ctl->v_empty[sv], (gk / NV - 1) & 1, abort_flag);
        if (lane == 0 && ok) mbar_arrive_expect_tx(&ctl->v_full[sv], bytes);
        __syncwarp();
        if (!ok) { gk |= 0x80000000u; break; }        // (K of this step is in flight, V is not)
        if (draft) {
          if (lane < n_oct) tma5(v_ring + sv * KV + lane * kOctet, &map_v, 0, lane * 8, 0, g, b, &ctl->v_full[sv]);
        } else if (lane < n_pages) {
          tma5(v_ring + sv * KV + lane * 2 * kOctet, &map_pool, 0, 0, 0, 0, 2 * pid + 1, &ctl->v_full[sv]);
        }
        pid = pid_next;
      }
      if (!ok) break;
      head += 1;
      y = 0;
      st = st_next;
    }
    if (*abort_flag) {   // copies in flight must land before the CTA may exit
      if (lane == 0) {
        atomicOr(dv.status, kStatusProducerTimeout);
        const bool k_only = (gk & 0x80000000u) != 0;
        const unsigned n = gk & 0x7fffffffu, nk = n + (k_only ? 1 : 0);
        for (unsigned i = nk > (unsigned)NK ? nk - NK : 0; i < nk; ++i)
          if (!mbar_wait_drain(&ctl->k_full[i % NK], (i / NK) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
        for (unsigned i = n > (unsigned)NV ? n - NV : 0; i < n; ++i)
          if (!mbar_wait_drain(&ctl->v_full[i % NV], (i / NV) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
        if (gq > 0 && !mbar_wait_drain(&ctl->q_full, (gq - 1) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
      }
    }
    __syncwarp();
  } else if (warp == SW + 1) {
    // ================================================================ matrix instructions: one thread
    if (lane == 0) {
      bool ok = true, pending = false, pend_first = false;
      unsigned g = 0;                  // steps whose scores have been issued
      unsigned pend_flush = 0, n_flush = 0;   // accumulators begun before the pending one; begun so far
      int pend_kk = 0;
      // descriptors of the operands' first rows
      const uint64_t v_desc = operand_desc_mn(smem_u32(v_ring), 1024, kOctet), p_desc = operand_desc_mn(smem_u32(p_tile), 128 * kTok, 1024);
      const uint64_t k_desc = operand_desc_mn(smem_u32(k_ring), 16, kOctet), q_desc = operand_desc(smem_u32(q_tile));
      const uint32_t v_lo = (uint32_t)v_desc, v_hi = (uint32_t)(v_desc >> 32), p_lo = (uint32_t)p_desc, p_hi = (uint32_t)(p_desc >> 32);
      const uint32_t k_lo = (uint32_t)k_desc, k_hi = (uint32_t)(k_desc >> 32), q_lo = (uint32_t)q_desc, q_hi = (uint32_t)(q_desc >> 32);
      // O^T of step g - 1
      auto issue_o = [&](unsigned step) -> bool {
        const int s = step % NV;
        if (!mbar_wait(&ctl->p_full, step & 1, abort_flag)) return false;
        if (!mbar_wait(&ctl->v_full[s], (step / NV) & 1, abort_flag)) return false;
        // the first product of an accumulator overwrites the one before, which must have been read out
        if (pend_first && pend_flush >= 1 && !mbar_wait(&ctl->o_read, (pend_flush - 1) & 1, abort_flag)) return false;
        tc_fence_after();
        const uint32_t a_lo = v_lo + (uint32_t)s * (KV >> 4), d = tmem + kOCol;
        if (pend_kk == kTok / 16) {
#pragma unroll
          for (int kk = 0; kk < kTok / 16; ++kk)   // 16 tokens per instruction
            umma_words(d, a_lo + kk * (2 * kOctet >> 4), v_hi, p_lo + kk * (2048 >> 4), p_hi, kIdescO, kk > 0 ? 1u : (pend_first ? 0u : 1u));
        } else {
          for (int kk = 0; kk < pend_kk; ++kk)
            umma_words(d, a_lo + kk * (2 * kOctet >> 4), v_hi, p_lo + kk * (2048 >> 4), p_hi, kIdescO, (kk > 0 || !pend_first) ? 1u : 0u);
        }
        umma_commit(&ctl->v_empty[s]);
        umma_commit(&ctl->p_done);
        return true;
      };
      for (unsigned gi = 0; ok; ++gi) {
        const int slot = gi % kItemSlots;
        ok = mbar_wait(&ctl->item_full[slot], (gi / kItemSlots) & 1, abort_flag);
        if (!ok) break;
        const TreeItem it = ctl->item[slot];
        mbar_arrive(&ctl->item_empty[slot]);
        if (it.head < 0) break;
        // the last product of the item before is not kept waiting for copies of this one
        if (pending && !(mbar_try_wait(&ctl->q_full, gi & 1) && mbar_try_wait(&ctl->k_full[g % NK], (g / NK) & 1))) {
          ok = issue_o(g - 1);
          pending = false;
          if (!ok) break;
        }
        ok = mbar_wait(&ctl->q_full, gi & 1, abort_flag);
        const int n = it.end - it.begin + it.draft;
        for (int i = 0; i < n && ok; ++i, ++g) {
          const int s = g % NK;
          ok = mbar_wait(&ctl->k_full[s], (g / NK) & 1, abort_flag);
          if (ok && g >= 2) ok = mbar_wait(&ctl->s_empty[g & 1], (g / 2 - 1) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a_lo = k_lo + (uint32_t)s * (KV >> 4), d = tmem + (g & 1) * R;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)   // 16 elements = 32 bytes along the swizzled half row
            umma_words(d, a_lo + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), k_hi, q_lo + (((kk >> 2) * R * 128 + (kk & 3) * 32) >> 4), q_hi, kIdescS, kk > 0);
          umma_commit(&ctl->k_empty[s]);
          umma_commit(&ctl->s_full[g & 1]);
          if (i == n - 1) umma_commit(&ctl->q_empty);
          if (pending) ok = issue_o(g - 1);   // behind the next step's scores, so that its softmax overlaps this product
          const bool draft = it.draft && i == n - 1;
          const int left = draft ? n_nodes : it.st.len - (it.begin + i) * kTok;
          pending = true;
          pend_first = i % kFlush == 0;
          pend_flush = pend_first ? n_flush++ : n_flush;
          pend_kk = min(kTok / 16, (left + 15) / 16);
        }
      }
      if (ok && pending) ok = issue_o(g - 1);
      if (!ok) {   // leaving early: let the instructions in flight finish before tensor memory is released
        atomicOr(dv.status, kStatusConsumerTimeout);
        umma_commit(&ctl->drain);
        (void)mbar_wait_drain(&ctl->drain, 0);
      }
    }
    __syncwarp();
  }
  } else {
    // ================================================================ softmax and epilogue: a thread per token
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int grp = warp >> 2, quarter = warp & 3;          // column group; tensor-memory lane quarter
    const int tk = quarter * 32 + lane;                     // token of the step; in the epilogue, dimension of the output
    const int c0 = grp * NC;                                // first column
    const uint32_t o_cols = kOCol + c0;                      // accumulator of the first column (heads; remainders R further)
    const int my_c = c0 + lane % LW;                         // the column(s) whose bookkeeping this lane carries: my_c + k LW
    const bool keeper = lane < LW;
    const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
    const float scale_log2 = dv.scale_log2;
    const uint64_t scale2 = f2_pack(scale_log2, scale_log2);
    const int rows = n_nodes * G, row0 = tile * R;
    unsigned g = 0, n_agree = 0, n_all = 0, n_top = 0;
    int mask_b = -1;              // the sequence whose tree the next three belong to
    uint32_t vis[LC] = {}, live[LC] = {};   // columns that see this thread's draft; columns that are a node of the tree
    float my_depth = 0.f;         // this thread's draft's
    bool ok = true;
    auto group_sync = [&]() -> bool {   // the four warps of this column group
      warp_arrive(&ctl->agree[grp], lane);
      return warp_wait(&ctl->agree[grp], n_agree++ & 1, abort_flag);
    };
    auto all_sync = [&]() -> bool {
      warp_arrive(&ctl->all_sync, lane);
      return warp_wait(&ctl->all_sync, n_all++ & 1, abort_flag);
    };
    for (unsigned gi = 0; ok; ++gi) {
      const int slot = gi % kItemSlots;
      ok = warp_wait(&ctl->item_full[slot], (gi / kItemSlots) & 1, abort_flag);
      if (!ok) break;
      const TreeItem it = ctl->item[slot];
      warp_arrive(&ctl->item_empty[slot], lane);
      if (it.head < 0) break;
      const size_t hs = (size_t)layer * dv.n_heads + it.head;
      const int b = it.head / dv.n_kv_heads, g_kv = it.head % dv.n_kv_heads;
      const int total = it.st.len + it.st.n_drop;
      const int32_t* parent = tc.parent + (size_t)b * n_nodes;
      // this lane's columns: their nodes, and where their rows stand in the output (from the KV head's first row on)
      int my_node[LC], place[LC];
#pragma unroll
      for (int k = 0; k < LC; ++k) {
        const int r = min(row0 + my_c + k * LW, rows - 1);
        my_node[k] = r >> lg;
        place[k] = (my_node[k] * dv.n_kv_heads * G + (r & (G - 1))) * D;
      }

      // ---- the tree (items that hold its tokens; with ALiBi, all: a row's position is its node's depth)
      // (the heads of a sequence follow one another: its tree is worked out once)
      if ((it.draft || kAlibi) && b != mask_b) {
        mask_b = b;
        TreeMask* mask = (TreeMask*)p_tile;   // (no weights are in there between items)
        static_assert(sizeof(TreeMask) <= (size_t)Smem::kP, "scratch");
        tree_mask_load(*mask, parent, n_nodes, tid, SW * 32);
        if (!(ok = all_sync())) break;
        tree_mask_walk(*mask, n_nodes, tid, SW * 32);
        if (!(ok = all_sync())) break;
#pragma unroll
        for (int k = 0; k < LC; ++k) {
          live[k] = __ballot_sync(0xffffffffu, keeper && row0 + my_c + k * LW < rows && tree_sees(*mask, my_node[k], my_node[k]));
          vis[k] = 0;
#pragma unroll 8
          for (int c = 0; c < LW; ++c) {   // (tokens are nodes here: this warp's are bits of one word)
            const int t = __shfl_sync(0xffffffffu, my_node[k], c);
            vis[k] |= (mask->see[t][quarter] >> lane & live[k] >> c & 1u) << c;
          }
        }
        if constexpr (kAlibi) {
          my_depth = (float)mask->depth[min(tk, n_nodes - 1)];
#pragma unroll
          for (int k = 0; k < LC; ++k)
            if (quarter == 0 && keeper) ctl->depth[my_c + k * LW] = (float)mask->depth[my_node[k]];
        }
        if (!(ok = all_sync())) break;
      }
      if constexpr (kAlibi) {
#pragma unroll
        for (int k = 0; k < LC; ++k)
          if (quarter == 0 && keeper)
            ctl->slope[my_c + k * LW] = dv.alibi_slopes[((size_t)layer * dv.n_kv_heads + g_kv) * G + (min(row0 + my_c + k * LW, rows - 1) & (G - 1))];
      }
      if (tid < kTreeMaxNodes / 32) ctl->bad_v[(gi + 1) & 1][tid] = 0;   // (last read before the barrier that ended the item before, next written behind this item's)
      uint32_t* bad_v = ctl->bad_v[gi & 1];
      // ---- reference maxima: minus infinity, or the compensation token's logit (Eq. 5: weight N_d exp(s_c), value v_hat),
      // whose weight is carried apart and added at the end
      if (it.seed) {
        const float* k_hat = dv.comp_mean + hs * 2 * D;
        const float count_log2 = log2f((float)it.st.n_drop);
        constexpr int EPL = D / 32;
        float kh[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) kh[e] = k_hat[lane * EPL + e];
#pragma unroll 4
        for (int k = 0; k < NC / 4; ++k) {
          const int c = c0 + quarter * (NC / 4) + k, r = min(row0 + c, rows - 1);
          const __nv_bfloat16* src = (const __nv_bfloat16*)tc.q + (size_t)b * tc.q_stride_b + (size_t)(r >> lg) * tc.q_stride_t + ((size_t)g_kv * G + (r & (G - 1))) * D + lane * EPL;
          uint32_t x[EPL / 2];
#pragma unroll
          for (int e = 0; e < EPL / 2; ++e) x[e] = __ldg((const uint32_t*)src + e);
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < EPL; ++e) s = fmaf(__uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16), kh[e], s);
          s = row_sum<32>(s);
          if (lane == 0) ctl->neg_m[c] = -fmaf(s, scale_log2, count_log2);
        }
      } else {
        if (tk < NC) ctl->neg_m[c0 + tk] = -kLow;
      }
      if (!(ok = group_sync())) break;
      float m_lane[LC], w_seed[LC];
#pragma unroll
      for (int k = 0; k < LC; ++k) {
        m_lane[k] = it.seed ? -ctl->neg_m[my_c + k * LW] : -CUDART_INF_F;
        w_seed[k] = it.seed ? 1.f : 0.f;
      }
      // Sums of the weights of this thread's tokens, and this thread's dimension of the rows' outputs: the accumulator in
      // tensor memory is added on every kFlush steps.  (The matrix unit truncates when it adds to the accumulator; over
      // the thousand products of a long span that bias reached 1.6e-5 of the result, 4e-6 with sixteen steps.)
      // (With 64 columns to a thread the sum lives in local memory - its loops are not unrolled -, which costs less than
      // spilling what the steps use.)
      constexpr int kUnroll = LC == 2 ? 1 : NC / 16;
      float l[NC], acc[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) l[c] = 0.f;
#pragma unroll kUnroll
      for (int c = 0; c < NC; c += 16)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c + e] = 0.f;
      auto flush = [&]() {
        tc_fence_after();
#pragma unroll kUnroll
        for (int c = 0; c < NC; c += 16) {
          uint32_t oh[16], ol[16];
          tmem_load<16>(lane_addr + o_cols + (uint32_t)c, oh);
          tmem_load<16>(lane_addr + o_cols + (uint32_t)(R + c), ol);
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[c + e] += __uint_as_float(oh[e]) + __uint_as_float(ol[e]);
        }
        tc_fence_before();
        warp_arrive(&ctl->o_read, lane);
      };

      const int n = it.end - it.begin + it.draft;
      for (int i = 0; i < n && ok; ++i, ++g) {
        const bool draft = it.draft && i == n - 1;
        const int slot0 = (it.begin + i) * kTok;
        const bool valid = draft ? tk < n_nodes : slot0 + tk < it.st.len;
        float rel = 0.f;   // ALiBi: this token's position, counted from the first position after the cache
        if constexpr (kAlibi)
          rel = draft ? my_depth : (float)(slot_position(min(slot0 + tk, it.st.len - 1), dv.n_sink, it.st, total) - total);
        ok = warp_wait(&ctl->s_full[g & 1], (g / 2) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[NC];
        // scores to the log2 domain, minus the reference; returns whether one outran it
        auto scores = [&]() -> bool {
          tmem_load<NC>(lane_addr + (g & 1) * R + c0, v);
          float mx = -CUDART_INF_F;
#pragma unroll
          for (int c = 0; c < NC; c += 4) {
            const float4 nm = *(const float4*)&ctl->neg_m[c0 + c];
            float t[4];
            f2_unpack(f2_fma(f2_pack(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), scale2, f2_pack(nm.x, nm.y)), t[0], t[1]);
            f2_unpack(f2_fma(f2_pack(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), scale2, f2_pack(nm.z, nm.w)), t[2], t[3]);
            if constexpr (kAlibi) {
              const float4 sl = *(const float4*)&ctl->slope[c0 + c], de = *(const float4*)&ctl->depth[c0 + c];
              t[0] = fmaf(sl.x, rel - de.x, t[0]);
              t[1] = fmaf(sl.y, rel - de.y, t[1]);
              t[2] = fmaf(sl.z, rel - de.z, t[2]);
              t[3] = fmaf(sl.w, rel - de.w, t[3]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) v[c + k] = __float_as_uint(t[k]);
            if (!draft) mx = max3(mx, max3(t[0], t[1], t[2]), t[3]);
          }
          if (draft) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (!(vis[c / LW] >> (c % LW) & 1)) v[c] = 0xff800000u;
              mx = fmaxf(mx, __uint_as_float(v[c]));
            }
          } else if (!valid) {
            mx = -CUDART_INF_F;
#pragma unroll
            for (int c = 0; c < NC; ++c) v[c] = 0xff800000u;
          }
          return mx > kLag;
        };
        auto weights = [&]() {
#pragma unroll
          for (int c = 0; c < NC; ++c) v[c] = __float_as_uint(fast_exp2(__uint_as_float(v[c])));
        };
        const bool outran = scores();
        if (__any_sync(0xffffffffu, outran) && lane == 0) *(volatile uint32_t*)&ctl->need[grp][g & 1] = g + 1;
        warp_arrive(&ctl->agree[grp], lane);
        weights();
        ok = warp_wait(&ctl->agree[grp], n_agree++ & 1, abort_flag);
        if (!ok) break;
        bool flush_now = i > 0 && i % kFlush == 0;
        if (*(volatile uint32_t*)&ctl->need[grp][g & 1] == g + 1) {
          // ---- move the references that were outrun to the maximum of what has been seen
          if (g > 0) {
            ok = warp_wait(&ctl->p_done, (g - 1) & 1, abort_flag);
            if (!ok) break;
          }
          if (flush_now) flush();
          flush_now = false;
          int32_t* top = ctl->top[n_top & 1];
#pragma unroll
          for (int k = 0; k < LC; ++k) {
            uint32_t s[LW];
            float t[LW];
            tmem_load<LW>(lane_addr + (g & 1) * R + c0 + k * LW, s);
#pragma unroll
            for (int c = 0; c < LW; ++c) {
              t[c] = __uint_as_float(s[c]) * scale_log2;
              if constexpr (kAlibi) t[c] = fmaf(ctl->slope[c0 + k * LW + c], rel - ctl->depth[c0 + k * LW + c], t[c]);
              if (draft ? !(vis[k] >> c & 1) : !valid) t[c] = -CUDART_INF_F;
            }
            const float mx = across_warp<LW, true>(t, lane);
            if (keeper) atomicMax(&top[my_c + k * LW], ordered(mx));
          }
          if (!(ok = group_sync())) break;
          float f[LC];
#pragma unroll
          for (int k = 0; k < LC; ++k) {
            // (a row moves only when it has been outrun itself: what it computes does not depend on the rows beside it)
            const float seen = from_ordered(top[my_c + k * LW]);
            const float m_new = m_lane[k] == -CUDART_INF_F || seen > m_lane[k] + kLag ? fmaxf(m_lane[k], seen) : m_lane[k];
            f[k] = m_lane[k] == -CUDART_INF_F ? 0.f : fast_exp2(m_lane[k] - m_new);
            m_lane[k] = m_new;
            w_seed[k] *= f[k];
            if (quarter == 0 && keeper) {
              ctl->neg_m[my_c + k * LW] = m_new == -CUDART_INF_F ? -kLow : -m_new;
              ctl->top[(n_top + 1) & 1][my_c + k * LW] = ordered(-CUDART_INF_F);   // (its last readers are two moves back)
            }
          }
          n_top += 1;
          if (!(ok = group_sync())) break;
          if (i > 0) {   // (an item's first step finds nothing to rescale)
#pragma unroll
            for (int c = 0; c < NC; ++c) l[c] *= __shfl_sync(0xffffffffu, f[c / LW], c % LW);
            tc_fence_after();
#pragma unroll kUnroll
            for (int c = 0; c < NC; c += 16) {
              const float f16 = LC == 2 && c >= 32 ? f[LC - 1] : f[0];
              float fc[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                fc[e] = __shfl_sync(0xffffffffu, f16, (c + e) % LW);
                acc[c + e] *= fc[e];
              }
              if (i % kFlush != 0) {   // the accumulator holds products of this item
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                  const uint32_t addr = lane_addr + o_cols + (uint32_t)(part * R + c);
                  uint32_t o[16];
                  tmem_load<16>(addr, o);
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fc[e]);
                  tmem_st16(addr, o);
                }
              }
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
          (void)scores();
          weights();
        } else if (g > 0) {   // the product of the step before must have read its weights
          ok = warp_wait(&ctl->p_done, (g - 1) & 1, abort_flag);
          if (!ok) break;
        }
        // S is read out
        tc_fence_before();
        warp_arrive(&ctl->s_empty[g & 1], lane);
        if (flush_now) flush();
        // ---- sums; a weight is written as a bf16 head (its upper 16 bits) plus a bf16 remainder
        uint8_t* p_row = p_tile + tk * 128;
#pragma unroll
        for (int c = 0; c < NC; c += 8) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int e = c + 2 * k;
            const uint32_t b0 = v[e], b1 = v[e + 1];
            const uint64_t w2 = f2_pack(__uint_as_float(b0), __uint_as_float(b1));
            f2_unpack(f2_add(f2_pack(l[e], l[e + 1]), w2), l[e], l[e + 1]);
            hi[k] = __byte_perm(b0, b1, 0x7632);
            float r0, r1;
            f2_unpack(f2_sub(w2, f2_pack(__uint_as_float(b0 & 0xffff0000u), __uint_as_float(b1 & 0xffff0000u))), r0, r1);
            const __nv_bfloat162 r = __floats2bfloat162_rn(r0, r1);
            lo[k] = *(const uint32_t*)&r;
          }
          const int ch = c0 + c, cl = R + ch;   // columns of heads and remainders in the 2R-column operand
          *(uint4*)(p_row + (ch >> 6) * (128 * kTok) + ((((ch & 63) >> 3) ^ (tk & 7)) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *(uint4*)(p_row + (cl >> 6) * (128 * kTok) + ((((cl & 63) >> 3) ^ (tk & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        // ---- V rows that no weight may meet: a zero weight times a NaN is a NaN.  Behind the head's last token the pool
        // may hold anything; a draft is hidden from the nodes of other branches.
        const int sv = g % NV;
        if (draft) {
          ok = warp_wait(&ctl->v_full[sv], (g / NV) & 1, abort_flag);
          if (!ok) break;
          if (tk < n_nodes) {
            constexpr int kChunks = D / 8 / kGroups;
            bool bad = false;
#pragma unroll 4
            for (int c = grp * kChunks; c < (grp + 1) * kChunks; ++c) {   // 16-byte chunks: this group's share of the row
              uint4* at = (uint4*)(v_ring + sv * KV + (tk >> 3) * kOctet + (c >> 3) * 1024 + (tk & 7) * 128 + (((c & 7) ^ (tk & 7)) << 4));
              uint4 x = *at;
              uint32_t* w = (uint32_t*)&x;
              bool hit = false;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; hit = true; }
                if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; hit = true; }
              }
              if (hit) *at = x;
              bad |= hit;
            }
            if (bad) atomicOr(&bad_v[tk >> 5], 1u << (tk & 31));
          }
        } else if (slot0 + kTok > it.st.len) {
          ok = warp_wait(&ctl->v_full[sv], (g / NV) & 1, abort_flag);
          if (!ok) break;
          const int first = it.st.len - slot0, last = (first + 15) / 16 * 16;
          for (int idx = tid; idx < (last - first) * (D / 8); idx += SW * 32) {
            const int t = first + idx / (D / 8), c = idx % (D / 8);
            *(uint4*)(v_ring + sv * KV + (t >> 3) * kOctet + (c >> 3) * 1024 + (t & 7) * 128 + ((c & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        warp_arrive(&ctl->p_full, lane);
      }
      if (!ok) break;
      // ---- the rows' results
      ok = warp_wait(&ctl->p_done, (g - 1) & 1, abort_flag);
      if (!ok) break;
      flush();
      float* l_part = (float*)(p_tile + 8192) + grp * 4 * NC;   // [quarter][NC]
      static_assert(8192 + 16 * R <= Smem::kP, "scratch");
#pragma unroll
      for (int k = 0; k < LC; ++k) {
        const float x = across_warp<LW, false>(l + k * LW, lane);
        if (keeper) l_part[quarter * NC + lane + k * LW] = x;
      }
      if (!(ok = group_sync())) break;
      const bool direct = it.rec < 0;
      // what a column's results need, for every lane to read: factor, the compensation token's share, place, liveness
      float4* table = (float4*)(p_tile + 10240 + warp * NC * 16);
      static_assert(10240 + SW * NC * 16 <= Smem::kP, "scratch");
#pragma unroll
      for (int k = 0; k < LC; ++k) {
        if (!keeper) continue;
        const int c = lane + k * LW;
        const float* lp = l_part + c;
        const float l_all = ((lp[0] + lp[NC]) + (lp[2 * NC] + lp[3 * NC])) + w_seed[k];
        const float inv = direct ? 1.f / l_all : 1.f;
        const bool is_node = (live[k] >> lane & 1) != 0;
        table[c] = make_float4(inv, w_seed[k] * inv, __int_as_float(direct ? place[k] : c * D), __int_as_float(row0 + c0 + c < rows && (!direct || is_node)));
        if (!direct && quarter == 0)   // (a negative sum marks an absent node's row for the combine kernel)
          dv.rec_ml[(size_t)it.rec * R + c0 + c] = make_float2(m_lane[k], it.draft && !is_node ? -1.f : l_all);
      }
      __syncwarp();
      if (quarter * 32 < D) {
        const float v_hat = it.seed ? dv.comp_mean[hs * 2 * D + D + tk] : 0.f;
        float* dst = direct ? tc.out + ((size_t)b * n_nodes * dv.n_kv_heads + g_kv) * G * D + tk : dv.rec_o + ((size_t)it.rec * R + c0) * D + tk;
        const int n_cols = min(NC, rows - (row0 + c0));   // (rows behind the last are nobody's)
#pragma unroll kUnroll
        for (int cb = 0; cb < NC; cb += 16) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float4 w = table[cb + e];
            if (__float_as_int(w.w)) dst[__float_as_int(w.z)] = fmaf(w.y, v_hat, w.x * acc[cb + e]);
          }
        }
        // The NaN and infinities that were taken out of the drafts' V reach the rows that see them.
        if (it.draft && (bad_v[0] | bad_v[1] | bad_v[2] | bad_v[3]) != 0) {
#pragma unroll 1
          for (int c = 0; c < n_cols; ++c) {
            const int t = (row0 + c0 + c) >> lg;
            float bad = 0.f;
#pragma unroll 1
            for (int nd = 0; nd <= t; ++nd) {
              if (!(bad_v[nd >> 5] >> (nd & 31) & 1) || !walk_sees(parent, t, nd)) continue;
              const float y = __bfloat162float(((const __nv_bfloat16*)tc.v)[(size_t)b * tc.kv_stride_b + (size_t)nd * tc.kv_stride_t + (size_t)g_kv * D + tk]);
              if (!(fabsf(y) < CUDART_INF_F)) bad += y;
            }
            if (bad != 0.f && __float_as_int(table[c].w)) dst[__float_as_int(table[c].z)] += bad;   // (this thread's own store)
          }
        }
      }
      if (!(ok = all_sync())) break;   // (the scratch in P's tile, and bad_v, are done with)
    }
    if (!ok && lane == 0) atomicOr(dv.status, kStatusReducerTimeout);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == SW + 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Folds the partial records of the heads that a cut ran through, parts in order: a warp per query row.
// grid = (spans, tiles, R / 32), eight warps of four rows each.
template <int D, int R>
__global__ void __launch_bounds__(256) tree_combine_kernel(DeviceView dv, TreeCall tc) {
  cudaGridDependencySynchronize();
  const TreeUnit u = dv.tree_units[blockIdx.x];
  if (u.n_parts == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tile = blockIdx.y, G = dv.group;
  const int b = u.head / dv.n_kv_heads, g = u.head % dv.n_kv_heads;
  // the first part is the last item of its span, the others are the first of theirs
  auto record = [&](int p) { return ((size_t)((u.first_span + p) * tc.n_tiles + tile) * 2 + (p == 0 ? 1 : 0)) * R; };
  for (int k = 0; k < 4; ++k) {
    const int c = blockIdx.z * 32 + k * 8 + warp, r = tile * R + c;
    if (r >= tc.n_nodes * G) return;
    if (dv.rec_ml[record(u.n_parts - 1) + c].y < 0.f) continue;   // an absent node (the last part holds the tree)
    float m = -CUDART_INF_F, l = 0.f;
    LaneVec<D> acc;
    acc.zero();
    constexpr int U = 4;   // records in flight
    for (int p0 = 0; p0 < u.n_parts; p0 += U) {
      float2 ml[U];
      LaneVec<D> o[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const size_t rec = record(min(p0 + i, u.n_parts - 1)) + c;
        ml[i] = __ldcg(&dv.rec_ml[rec]);
        o[i].load_l2(dv.rec_o + rec * D, lane);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (p0 + i >= u.n_parts) break;
        const float mn = fmaxf(m, ml[i].x), mu = mn == -CUDART_INF_F ? 0.f : mn;
        const float c_old = fast_exp2(m - mu), c_new = fast_exp2(ml[i].x - mu);
        l = l * c_old + ml[i].y * c_new;
        acc.scale(c_old);
        acc.fma(c_new, o[i]);
        m = mn;
      }
    }
    acc.scale(1.f / l);
    const int t = r / G, j = r % G;
    acc.store(tc.out + (((size_t)b * tc.n_nodes + t) * dv.n_kv_heads * G + (size_t)g * G + j) * D, lane);
  }
}

bool make_map(CUtensorMap* map, const void* base, const cuuint64_t (&dims)[5], const cuuint64_t (&strides)[4],
              const cuuint32_t (&box)[5], CUtensorMapSwizzle swizzle) {
  const EncodeTiledFn encode = encode_tiled_fn();
  const cuuint32_t es[5] = {1, 1, 1, 1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, es,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int R, bool kAlibi>
cudaError_t mma_launch(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& call, long long rec_rows,
                       int n_sms, cudaStream_t s) {
  constexpr cuuint64_t RB = D * 2;
  constexpr cuuint32_t H = D / 64;
  TreeCall tc = call;
  const cuuint64_t B = (cuuint64_t)(dv.n_heads / dv.n_kv_heads), T = (cuuint64_t)tc.n_nodes, G = (cuuint64_t)dv.group;
  const cuuint64_t Hkv = (cuuint64_t)dv.n_kv_heads, Hq = Hkv * G;
  // (a stride that separates nothing may be anything in the call, and must be a legal one in the map)
  const cuuint64_t qt = T > 1 ? (cuuint64_t)tc.q_stride_t * 2 : Hq * RB, kt = T > 1 ? (cuuint64_t)tc.kv_stride_t * 2 : Hkv * RB;
  const cuuint64_t qb = B > 1 ? (cuuint64_t)tc.q_stride_b * 2 : Hq * RB, kb = B > 1 ? (cuuint64_t)tc.kv_stride_b * 2 : Hkv * RB;
  CUtensorMap pool, q, k, v;
  // pool: eight tokens of a 64-element half are 1 KB in the stage; [octet][half] as the operand layout has them
  const bool made =
      make_map(&pool, dv.pool, {64, 8, H, 2, 2 * (cuuint64_t)pool_pages}, {RB, 128, 8 * RB, 16 * RB}, {64, 8, H, 2, 1}, CU_TENSOR_MAP_SWIZZLE_NONE) &&
      make_map(&q, tc.q, {64, Hq, T, H, B}, {RB, qt, 128, qb}, {64, (cuuint32_t)G, (cuuint32_t)(R / G), 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B) &&
      make_map(&k, tc.k, {64, T, H, Hkv, B}, {kt, 128, RB, kb}, {64, 8, H, 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B) &&
      make_map(&v, tc.v, {64, T, H, Hkv, B}, {kt, 128, RB, kb}, {64, 8, H, 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B);
  if (!made) return cudaErrorInvalidValue;
  tc.n_tiles = (int)((T * G + R - 1) / R);
  tc.n_spans = std::max(1, std::min({n_sms / tc.n_tiles, kTreeMaxSpans, (int)(rec_rows / (2LL * R * tc.n_tiles))}));
  tc.min_span = 4;
  constexpr int kBytes = TreeSmem<D, R>::kBytes;
  static bool opted_in[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !opted_in[dev]) {
    e = cudaFuncSetAttribute(tree_mma_kernel<D, R, kAlibi>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) opted_in[dev] = true;
  }
  tree_mma_kernel<D, R, kAlibi><<<tc.n_spans * tc.n_tiles, kTreeThreads, kBytes, s>>>(dv, pool, q, k, v, layer, tc);
  e = cudaGetLastError();
  if (e != cudaSuccess || tc.n_spans == 1) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tc.n_spans, tc.n_tiles, R / 32);
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, tree_combine_kernel<D, R>, dv, tc);
}

template <int D, bool kAlibi>
cudaError_t mma_rows(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& tc, long long rec_rows, int n_sms,
                     cudaStream_t s) {
  const int rows = tc.n_nodes * dv.group;
  if (rows <= 32) return mma_launch<D, 32, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  if (rows <= 64) return mma_launch<D, 64, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  return mma_launch<D, 128, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
}

}  // namespace

cudaError_t launch_tree_mma(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& tc, long long rec_rows,
                            int n_sms, cudaStream_t s) {
  if (dv.alibi)
    return dv.head_dim == 128 ? mma_rows<128, true>(dv, pool_pages, layer, tc, rec_rows, n_sms, s)
                              : mma_rows<64, true>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  return dv.head_dim == 128 ? mma_rows<128, false>(dv, pool_pages, layer, tc, rec_rows, n_sms, s)
                            : mma_rows<64, false>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
}

}  // namespace razor
