// What the two tensor-core kernels of tree attention share: how the work is cut into spans, the producer warp that feeds
// them, barriers, tensor-memory accesses, and the kernel that folds partial records.
#ifndef RAZOR_TREE_TC_CUH_
#define RAZOR_TREE_TC_CUH_

#include <math_constants.h>

#include <algorithm>

#include "razor_common.cuh"
#include "razor_sync.cuh"
#include "razor_tc.cuh"
#include "razor_tree.cuh"

namespace razor {
namespace {

constexpr int kTok = 128;                       // tokens of a step
constexpr int kStepPages = kTok / kPageTokens;
constexpr int kSoftWarps = 8, kTreeThreads = (kSoftWarps + 4) * 32;   // softmax warps; of four more, one copies, one issues the scores' products, one the outputs', and one has no part
// Steps whose products add up in tensor memory before the softmax warps take the sum out.  The matrix unit truncates when it
// adds to an accumulator: over a span of the 32K shape (147 steps, 1200 additions) that bias alone put 1.6e-5 of the
// result's norm into it (2.2e-5 to 4.5e-5 over single heads of 150 steps a span, where every eight steps leave 2.5e-6 to 3.4e-6,
// everything else included).
constexpr int kFlush = 8;
// What a head costs beside its steps, in steps.  Chosen on two shapes (33 nodes on 32 short D = 64 heads: 0 32-34 us, 3 30-33,
// 5 28-30, 8 32; 26 nodes on 128 ragged heads: 0 133-137, 3 130-132, 5 122-129, 8 121).  On fifteen others, eight drawn at random
// among them, 0 costs up to a quarter more where heads are short and many (40 heads of 1114 tokens, 236 rows each: 36
// against 29 us; 240 of 92 tokens, 32 rows: 23 against 20), is level on long ones, and is 1.5-2 us faster for twenty
// short heads or fewer (16 -> 14 us: there the smallest span, which is longer than this, leaves SMs idle); 8 stays within 8 %
// either way.
constexpr int kHeadCost = 5;
constexpr int kItemSlots = 3;
constexpr int kMaxStages = 4;                   // of K and of V
constexpr int kSmemMax = 232448;
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

// Barriers between the producer, the warp that issues the matrix instructions and the softmax warps.
struct TreePipe {
  uint64_t q_full, q_empty;
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
  uint64_t s_full[2], s_empty[2];     // per S buffer
  uint64_t p_full, p_done;            // the weights are in place; the product that read them has run
  uint64_t o_read;                    // the accumulator has been read out
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  uint64_t all_sync;                  // the softmax warps among themselves
  uint64_t drain[2];                  // of the two issuing warps
  uint32_t tmem_base;
  int abort_flag;
  uint32_t bad_v[2][kTreeMaxNodes / 32];   // [item parity]: drafts whose V holds a NaN or an infinity
  TreeItem item[kItemSlots];
};
__device__ __forceinline__ void tree_pipe_init(TreePipe* p, int nk, int nv) {
  mbar_init(&p->q_full, 1);
  mbar_init(&p->q_empty, 1);
  for (int s = 0; s < nk; ++s) { mbar_init(&p->k_full[s], 1); mbar_init(&p->k_empty[s], 1); }
  for (int s = 0; s < nv; ++s) { mbar_init(&p->v_full[s], 1); mbar_init(&p->v_empty[s], 1); }
  for (int s = 0; s < 2; ++s) { mbar_init(&p->s_full[s], 1); mbar_init(&p->s_empty[s], kSoftWarps); }
  mbar_init(&p->p_full, kSoftWarps);
  mbar_init(&p->p_done, 1);
  mbar_init(&p->o_read, kSoftWarps);
  for (int s = 0; s < kItemSlots; ++s) { mbar_init(&p->item_full[s], 1); mbar_init(&p->item_empty[s], kSoftWarps + 2); }
  mbar_init(&p->all_sync, kSoftWarps);
  mbar_init(&p->drain[0], 1);
  mbar_init(&p->drain[1], 1);
  p->abort_flag = 0;
  for (int k = 0; k < 2 * kTreeMaxNodes / 32; ++k) p->bad_v[0][k] = 0;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
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
// The same with operand A out of tensor memory.
__device__ __forceinline__ void umma_words_tmem_a(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                                  uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
      :
      : "r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
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

// The warps that issue matrix instructions, one thread each: one the scores of a step, the other its output - two, because a
// thread that did both had its waits and commits add up to more than the tensor cores' own time.  Each goes through the
// items and their steps: step(g, i, it) issues global step g, the item's i-th, and returns false when a wait has run out; first(gi) comes
// before an item's steps.
template <typename First, typename Step>
__device__ __forceinline__ void tree_issue(TreePipe* p, const DeviceView& dv, uint64_t* drain, First&& first, Step&& step) {
  volatile int* abort_flag = &p->abort_flag;
  bool ok = true;
  unsigned g = 0;
  for (unsigned gi = 0; ok; ++gi) {
    const int slot = gi % kItemSlots;
    ok = mbar_wait(&p->item_full[slot], (gi / kItemSlots) & 1, abort_flag);
    if (!ok) break;
    const TreeItem it = p->item[slot];
    mbar_arrive(&p->item_empty[slot]);
    if (it.head < 0) break;
    ok = first(gi);
    const int n = it.end - it.begin + it.draft;
    for (int i = 0; i < n && ok; ++i, ++g) ok = step(g, i, n, it);
  }
  if (!ok) {   // leaving early: let the instructions in flight finish before tensor memory is released
    atomicOr(dv.status, kStatusConsumerTimeout);
    umma_commit(drain);
    (void)mbar_wait_drain(drain, 0);
  }
}

// Is node n node t or an ancestor of it?  (Straight from the parents: only where a draft holds a NaN or an infinity.)
__device__ __noinline__ bool walk_sees(const int32_t* parent, int t, int n) {
  while (t > n) {
    const int a = parent[t];
    if (a < -1 || a >= t) return false;
    t = a;
  }
  return t == n;
}

// A pair of weights as bf16 heads and bf16 remainders: together within 2^-18 of a weight (the head is off by at most 2^-9,
// the remainder by 2^-9 of that); a head alone would put 2^-9 of a large weight's V row into the result.
__device__ __forceinline__ void split_weights(uint64_t w2, float w0, float w1, uint32_t& heads, uint32_t& remainders) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(w0, w1);
  heads = *(const uint32_t*)&h;
  float r0, r1;
  f2_unpack(f2_sub(w2, f2_pack(__uint_as_float(heads << 16), __uint_as_float(heads & 0xffff0000u))), r0, r1);
  const __nv_bfloat162 r = __floats2bfloat162_rn(r0, r1);
  remainders = *(const uint32_t*)&r;
}
// NaN and infinities in eight bf16 values to zero; returns whether there were any.
__device__ __forceinline__ bool drop_non_finite(uint4& x) {
  uint32_t* w = (uint32_t*)&x;
  bool hit = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; hit = true; }
    if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; hit = true; }
  }
  return hit;
}

// What a CTA is to do: the steps begin .. end of all the heads' steps laid end to end, the first of them step `step` of head
// `head` (state `st`); head < 0: nothing.
struct TreeSpan {
  int head, step;
  long long begin, end;
  HeadState st;
};
// All heads' steps laid end to end (a head's cache steps, then one for the tree), cut into spans of equal cost; the CTA's own
// span is left at scratch + 256 (1 KB of shared memory), to be read behind a barrier.  A head costs its steps and kHeadCost
// more (queries, the compensation token's logit, results); that much lies in front of its first step, and a cut there is a
// cut between two heads.
__device__ __forceinline__ void tree_find_span(const DeviceView& dv, const HeadState* states, const TreeCall& tc, int span,
                                               int tile, uint8_t* scratch) {
  constexpr int NT = kTreeThreads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  long long* warp_tot = (long long*)scratch;
  TreeSpan* out = (TreeSpan*)(scratch + 256);
  const int per = (dv.n_heads + NT - 1) / NT;
  const int h0 = min(dv.n_heads, tid * per), h1 = min(dv.n_heads, h0 + per);
  auto cost = [&](int h) { return head_steps(states[h].len) + 1 + kHeadCost; };
  long long mine = 0;
  for (int h = h0; h < h1; ++h) mine += cost(h);
  long long upto = mine;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto, off);
    if (lane >= off) upto += y;
  }
  if (lane == 31) warp_tot[warp] = upto;
  if (tid == 0) *out = TreeSpan{-1, 0, 0, 0, HeadState{0, 0, 0, 0}};
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += warp_tot[w];
    total += warp_tot[w];
  }
  before += upto - mine;
  const int n = (int)min((long long)tc.n_spans, max(1LL, total / tc.min_span));   // (a span is longer than kHeadCost)
  auto cut = [&](int s) { return total * s / n; };
  // where a cut is: head h, whose cost starts at u0 (kHeadCost of each head before it are no steps)
  auto find = [&](long long x, int& h, long long& u0) {
    u0 = before;
    h = h0;
    for (int w; u0 + (w = cost(h)) <= x; ++h) u0 += w;
  };
  const long long x0 = span < n ? cut(span) : total, x1 = span < n ? cut(span + 1) : total;
  if (x0 < x1 && before <= x0 && x0 < before + mine) {
    int h;
    long long u0;
    find(x0, h, u0);
    const long long u = u0 + kHeadCost, step = max(0LL, x0 - u);   // (u: the head's first step)
    out->head = h;
    out->step = (int)step;
    out->begin = u0 - (long long)kHeadCost * h + step;
    out->st = states[h];
    // the spans that start inside a head share the work of folding its parts
    TreeUnit t{h, 0, 0, 0};
    if (step > 0) {
      auto span_of = [&](long long x) {   // the span that a step lies in
        int s = (int)(x * n / total);
        while (cut(s) > x) s -= 1;
        while (cut(s + 1) <= x) s += 1;
        return s;
      };
      t.first_span = span_of(u);
      t.n_parts = span_of(u0 + cost(h) - 1) - t.first_span + 1;
      t.turn = span - t.first_span - 1;
    }
    if (tile == 0) tc.units[span] = t;
  }
  if (x1 < total && before <= x1 && x1 < before + mine) {
    int h;
    long long u0;
    find(x1, h, u0);
    out->end = u0 - (long long)kHeadCost * h + max(0LL, x1 - u0 - kHeadCost);
  }
  if (x1 == total && tid == 0) out->end = total - (long long)kHeadCost * dv.n_heads;
  if (x0 >= x1 && tile == 0 && tid == 0) tc.units[span] = TreeUnit{0, 0, 0, 0};
}

// The next item of a span that has `todo` steps left, from step y of a head on; takes its steps off todo.
__device__ __forceinline__ TreeItem tree_item(const DeviceView& dv, int head, int y, long long& todo, const HeadState& st) {
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
  return it;
}

// The producer warp: publishes the span's items and copies queries, pages and drafts into their rings.  A stage holds 128
// tokens of K or of V as [octet][64-element half][8 tokens][128 B], each KB in the 128-byte swizzle: for the matrix unit
// the tokens are rows of a K-major operand or the contraction index of an MN-major one.
template <int D, int R, int NK, int NV>
__device__ __forceinline__ void tree_produce(const DeviceView& dv, const CUtensorMap& map_pool, const CUtensorMap& map_q,
                                             const CUtensorMap& map_k, const CUtensorMap& map_v, int layer, const TreeCall& tc,
                                             const TreeSpan& sp, int tile, TreePipe* p, uint8_t* k_ring, uint8_t* v_ring,
                                             uint8_t* q_tile, int lane) {
  constexpr int HALVES = D / 64, KV = kTok * D * 2;
  constexpr uint32_t kOctet = 8 * D * 2;
  const int G = dv.group, n_nodes = tc.n_nodes;
  const HeadState* states = dv.state + (size_t)layer * dv.n_heads;
  volatile int* abort_flag = &p->abort_flag;
  unsigned gk = 0, gi = 0, gq = 0;   // steps issued, items published, query tiles issued
  int head = sp.head, y = sp.step;
  long long todo = sp.head < 0 ? 0 : sp.end - sp.begin;
  bool ok = true;
  HeadState st = sp.st;
  for (;; ++gi) {
    const TreeItem it = tree_item(dv, head, y, todo, st);
    const int slot = gi % kItemSlots;
    if (gi >= kItemSlots) ok = warp_wait(&p->item_empty[slot], (gi / kItemSlots - 1) & 1, abort_flag);
    if (!ok) break;
    if (lane == 0) {
      p->item[slot] = it;
      mbar_arrive(&p->item_full[slot]);
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
    if (gi >= 1) ok = warp_wait(&p->q_empty, (gi - 1) & 1, abort_flag);
    if (!ok) break;
    if (lane == 0) {
      mbar_arrive_expect_tx(&p->q_full, (uint32_t)R * D * 2);
#pragma unroll
      for (int h = 0; h < HALVES; ++h) tma5(q_tile + h * R * 128, &map_q, 0, g * G, tile * (R / G), h, b, &p->q_full);
    }
    gq += 1;
    for (int step = it.begin; step < it.end + it.draft; ++step, ++gk) {
      const bool draft = step == it.end;
      const int sk = gk % NK, sv = gk % NV;
      const int n_pages = draft ? 0 : min(kStepPages, head_pages - step * kStepPages);
      const int n_oct = (n_nodes + 15) / 16 * 2;   // (the matrix instruction takes 16 tokens at a time; rows beyond the tree read zero)
      const uint32_t bytes = draft ? (uint32_t)n_oct * kOctet : (uint32_t)n_pages * 2 * kOctet;
      const int pid_next = step + 1 < it.end ? page_of(step + 1) : 0;
      if (gk >= (unsigned)NK) ok = warp_wait(&p->k_empty[sk], (gk / NK - 1) & 1, abort_flag);
      if (!ok) break;
      if (lane == 0) mbar_arrive_expect_tx(&p->k_full[sk], bytes);
      __syncwarp();
      if (draft) {
        if (lane < n_oct) tma5(k_ring + sk * KV + lane * kOctet, &map_k, 0, lane * 8, 0, g, b, &p->k_full[sk]);
      } else if (lane < n_pages) {
        tma5(k_ring + sk * KV + lane * 2 * kOctet, &map_pool, 0, 0, 0, 0, 2 * pid, &p->k_full[sk]);
      }
      if (gk >= (unsigned)NV) ok = warp_wait(&p->v_empty[sv], (gk / NV - 1) & 1, abort_flag);
      if (lane == 0 && ok) mbar_arrive_expect_tx(&p->v_full[sv], bytes);
      __syncwarp();
      if (!ok) { gk |= 0x80000000u; break; }        // (K of this step is in flight, V is not)
      if (draft) {
        if (lane < n_oct) tma5(v_ring + sv * KV + lane * kOctet, &map_v, 0, lane * 8, 0, g, b, &p->v_full[sv]);
      } else if (lane < n_pages) {
        tma5(v_ring + sv * KV + lane * 2 * kOctet, &map_pool, 0, 0, 0, 0, 2 * pid + 1, &p->v_full[sv]);
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
        if (!mbar_wait_drain(&p->k_full[i % NK], (i / NK) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
      for (unsigned i = n > (unsigned)NV ? n - NV : 0; i < n; ++i)
        if (!mbar_wait_drain(&p->v_full[i % NV], (i / NV) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
      if (gq > 0 && !mbar_wait_drain(&p->q_full, (gq - 1) & 1)) atomicOr(dv.status, kStatusDrainTimeout);
    }
  }
}

// Folds the partial records of the heads that a cut ran through, in an order that depends on their number alone.
// grid = (spans, tiles, R / 8).  The spans that start inside a head take its rows in turn; a row's records are shared out to
// as many warps as leave each about eight, since what costs here is the latency of one record after the other (32 nodes over
// two long heads of 54 parts each: the whole call 79 us when the rows of a head were one span's and a warp took each, 56 so).
template <int D, int R>
__global__ void __launch_bounds__(256) tree_combine_kernel(DeviceView dv, TreeCall tc) {
  constexpr int U = 8;   // records in flight
  __shared__ float part_o[8][D];
  __shared__ float2 part_ml[8];
  cudaGridDependencySynchronize();
  const TreeUnit u = tc.units[blockIdx.x];
  if (u.n_parts == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tile = blockIdx.y, G = dv.group;
  const int b = u.head / dv.n_kv_heads, g = u.head % dv.n_kv_heads;
  // the first part is the last item of its span, the others are the first of theirs
  auto record = [&](int p) { return ((size_t)((u.first_span + p) * tc.n_tiles + tile) * 2 + (p == 0 ? 1 : 0)) * R; };
  const int rows = min(R, tc.n_nodes * G - tile * R), among = u.n_parts - 1;
  const int W = u.n_parts <= U ? 1 : (u.n_parts <= 2 * U ? 2 : (u.n_parts <= 4 * U ? 4 : 8));   // warps to a row
  const int rows_at_once = 8 / W;
  for (int k0 = blockIdx.z * rows_at_once; u.turn + k0 * among < rows; k0 += gridDim.z * rows_at_once) {
    const int c = u.turn + (k0 + warp / W) * among;
    const bool mine = c < rows;
    float m = -CUDART_INF_F, l = 0.f;
    LaneVec<D> acc;
    acc.zero();
    auto add = [&](const float2& ml, const LaneVec<D>& o) {
      const float mn = fmaxf(m, ml.x), mu = mn == -CUDART_INF_F ? 0.f : mn;
      const float c_old = fast_exp2(m - mu), c_new = fast_exp2(ml.x - mu);
      l = l * c_old + ml.y * c_new;
      acc.scale(c_old);
      acc.fma(c_new, o);
      m = mn;
    };
    bool live = mine;
    if (mine) {
      const float2 last = __ldcg(&dv.rec_ml[record(u.n_parts - 1) + c]);
      for (int p0 = warp % W; p0 < u.n_parts; p0 += U * W) {
        float2 ml[U];
        LaneVec<D> o[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const size_t rec = record(min(p0 + i * W, u.n_parts - 1)) + c;
          ml[i] = __ldcg(&dv.rec_ml[rec]);
          o[i].load_l2(dv.rec_o + rec * D, lane);
        }
        live = !(last.y < 0.f);   // (an absent node otherwise: the last part holds the tree; the sum of a row that sees a NaN is a NaN)
        if (!live) break;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (p0 + i * W >= u.n_parts) break;
          add(ml[i], o[i]);
        }
      }
    }
    if (W > 1) {
      __syncthreads();   // (the turn before has been read)
      if (warp % W != 0) {
        acc.store(part_o[warp], lane);
        if (lane == 0) part_ml[warp] = make_float2(m, l);
      }
      __syncthreads();
      if (warp % W != 0) continue;
      for (int i = 1; i < W; ++i) {
        LaneVec<D> o;
        o.load_shared(part_o[warp + i], lane);
        add(part_ml[warp + i], o);
      }
    }
    if (!live) continue;
    acc.scale(1.f / l);
    const int r = tile * R + c, t = r / G, j = r % G;
    acc.store(tc.out + (((size_t)b * tc.n_nodes + t) * dv.n_kv_heads * G + (size_t)g * G + j) * D, lane);
  }
}

[[maybe_unused]] bool make_map(CUtensorMap* map, const void* base, const cuuint64_t (&dims)[5], const cuuint64_t (&strides)[4],
              const cuuint32_t (&box)[5], CUtensorMapSwizzle swizzle) {
  const EncodeTiledFn encode = encode_tiled_fn();
  const cuuint32_t es[5] = {1, 1, 1, 1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, es,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct TreeMaps {
  CUtensorMap pool, q, k, v;
};
// How a call is cut: tiles of R rows, spans (at most one CTA to an SM).
template <int R>
void tree_cut(const DeviceView& dv, long long rec_rows, int n_sms, TreeCall& tc) {
  tc.n_tiles = (int)(((long long)tc.n_nodes * dv.group + R - 1) / R);
  tc.n_spans = std::max(1, std::min({n_sms / tc.n_tiles, kTreeMaxSpans, (int)(rec_rows / (2LL * R * tc.n_tiles))}));
  tc.min_span = kHeadCost + 1;
}
// Tensor maps of a call.
template <int D, int R>
bool tree_maps(const DeviceView& dv, long long pool_pages, const TreeCall& tc, TreeMaps& m) {
  constexpr cuuint64_t RB = D * 2;
  constexpr cuuint32_t H = D / 64;
  const cuuint64_t B = (cuuint64_t)(dv.n_heads / dv.n_kv_heads), T = (cuuint64_t)tc.n_nodes, G = (cuuint64_t)dv.group;
  const cuuint64_t Hkv = (cuuint64_t)dv.n_kv_heads, Hq = Hkv * G;
  // (a stride that separates nothing may be anything in the call, and must be a legal one in the map)
  const cuuint64_t qt = T > 1 ? (cuuint64_t)tc.q_stride_t * 2 : Hq * RB, kt = T > 1 ? (cuuint64_t)tc.kv_stride_t * 2 : Hkv * RB;
  const cuuint64_t qb = B > 1 ? (cuuint64_t)tc.q_stride_b * 2 : Hq * RB, kb = B > 1 ? (cuuint64_t)tc.kv_stride_b * 2 : Hkv * RB;
  // pool: eight tokens of a 64-element half are 1 KB in the stage; [octet][half] as the operand layout has them
  return make_map(&m.pool, dv.pool, {64, 8, H, 2, 2 * (cuuint64_t)pool_pages}, {RB, 128, 8 * RB, 16 * RB}, {64, 8, H, 2, 1}, CU_TENSOR_MAP_SWIZZLE_NONE) &&
         make_map(&m.q, tc.q, {64, Hq, T, H, B}, {RB, qt, 128, qb}, {64, (cuuint32_t)G, (cuuint32_t)(R / G), 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B) &&
         make_map(&m.k, tc.k, {64, T, H, Hkv, B}, {kt, 128, RB, kb}, {64, 8, H, 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B) &&
         make_map(&m.v, tc.v, {64, T, H, Hkv, B}, {kt, 128, RB, kb}, {64, 8, H, 1, 1}, CU_TENSOR_MAP_SWIZZLE_128B);
}
// The kernel over all spans and tiles, and the one that folds its records.  Both are launched as programmatic dependents:
// barriers, tensor memory and descriptors are set up while the kernel before finishes, and everything else waits for it.
template <int D, int R, typename... P, typename... A>
cudaError_t tree_run(void (*kernel)(P...), int smem_bytes, const DeviceView& dv, const TreeCall& tc, cudaStream_t s, A... args) {
  // (set at every call: it costs less than a microsecond, and is kept per device)
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(tc.n_spans * tc.n_tiles);
  cfg.blockDim = dim3(kTreeThreads);
  cfg.dynamicSmemBytes = smem_bytes;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e != cudaSuccess || tc.n_spans == 1) return e;
  cfg.gridDim = dim3(tc.n_spans, tc.n_tiles, R / 8);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, tree_combine_kernel<D, R>, dv, tc);
}
template <int D, int R, typename Kernel>
cudaError_t tree_launch(Kernel kernel, int smem_bytes, const DeviceView& dv, long long pool_pages, int layer, const TreeCall& call,
                        long long rec_rows, int n_sms, cudaStream_t s) {
  TreeCall tc = call;
  tree_cut<R>(dv, rec_rows, n_sms, tc);
  TreeMaps m;
  if (!tree_maps<D, R>(dv, pool_pages, tc, m)) return cudaErrorInvalidValue;
  return tree_run<D, R>(kernel, smem_bytes, dv, tc, s, dv, m.pool, m.q, m.k, m.v, layer, tc);
}

}  // namespace
}  // namespace razor
#endif
