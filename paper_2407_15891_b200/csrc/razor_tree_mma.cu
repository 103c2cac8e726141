// Attention of a tree of drafted tokens over a bf16 cache, on the tensor cores: up to 64 query rows per KV head (nodes x
// query heads of the group), and every ALiBi cache.
//
// A short block of query rows stands against a long stream of tokens, so the products are taken the other way round from
// a prompt's: TOKENS are the 128-row operand and the query rows the narrow one,
//     S^T = K Q^T          [128 tokens x R rows],     R = 32, 64 or 128 (ALiBi) rows of a tile,
//     O^T = V^T P^T        [D x R rows], contraction over the tokens,
// and no lane of the tensor memory, no tensor-core row and no softmax thread stands idle when the rows are few.  A thread
// owns one token, which also makes masks cheap: beyond the head's end, or which nodes see this draft, is decided per
// thread.  Query rows are columns, independent of one another: whatever a dead or poisoned row holds stays in its own
// column.  P goes through shared memory as a bf16 head plus a bf16 remainder, side by side as 2R columns of one product
// (the V operand is read once for both), so that a weight keeps fp32-like accuracy; the two halves of the accumulator are
// added at the end.
//
// What bounds it is the stream of pages out of HBM: 8 nodes on the 32K multi-head shape (8 x 32 heads, 1.40 GB of kept
// pages) 224-226 us under continuous load = 6.2 TB/s, 0.97 of the measured copy rate (210-214 us in runs of 60 calls); 64
// nodes 286-290 us with the clock held near 1.5 GHz by the power cap, where the softmax warps (2500 cycles a step against
// the copies' 2640 at full clock) fall behind, 240 us at full clock.
//
// Work: every head's slots in steps of 128 tokens plus one step for the tree's own tokens (their visibility is a bit mask
// per thread).  All heads' steps are laid end to end and cut into equal spans, one per CTA; with several tiles of rows
// the tiles of a span run in neighbouring CTAs at the same time, so that the cache comes out of HBM once and out of L2 for
// the others.  The cut is made on the device from the head states - a scan over the heads, two microseconds with the rest of
// the set-up - so a call costs the host nothing but the launch, and a captured graph follows the cache as it grows.  A
// head that a cut runs through leaves one partial record per span; tree_combine_kernel folds them.
//
// A CTA (one per SM): eight softmax warps (one per tensor-memory lane quarter and group of columns), a producer warp (TMA:
// pages of the pool, whose rows are stored in the swizzle of the operand layout; drafts and queries through maps of their
// own) and two warps that issue the matrix instructions.  S is double-buffered, so the scores of the next step are
// computed during the softmax of this one.
//
// The running maximum of a row is a reference that may lag: weights are 2^(s - m), floats, as exact at 2^20 as at one.  It
// is moved (and the accumulator rescaled) only when a score outruns it by 2^kLag; the four warps of a column group agree on
// that once per step, and compute their weights while the agreement is on its way.
//
// Every wait is bounded in time; a wait that runs out sets the CTA's abort flag and a bit of the device status word,
// copies and instructions in flight are waited for, tensor memory is released.
#include "razor_tree_tc.cuh"

namespace razor {
namespace {

// Two groups of columns, four softmax warps each (one per tensor-memory lane quarter).  (Four groups, sixteen warps with
// half as many columns each, had 104 registers apiece and spilled, and next to 227 KB of shared memory there is no L1 to
// spill to: slower for 64 rows and for 128.)
constexpr int kGroups = 2;

template <int R>
struct TreeCtl {
  TreePipe pipe;
  uint64_t agree[kGroups];            // the four warps of a column group among themselves
  uint32_t need[kGroups][2];          // [column group][step parity]: step + 1 when a score outran the reference
  alignas(16) float neg_m[R];         // minus the reference maximum of each row (log2 domain)
  int32_t top[2][R];                  // column maxima while the reference moves, as ordered integers
  alignas(16) float slope[R];         // ALiBi only
  alignas(16) float depth[R];
};

template <int D, int R>
struct TreeSmem {
  static constexpr int kKv = kTok * D * 2;             // one stage of K or of V
  static constexpr int kQ = R * D * 2;
  static constexpr int kP = kTok * 2 * R * 2;
  static constexpr int kRoom = kSmemMax - kQ - kP - (int)sizeof(TreeCtl<R>);
  static constexpr int kK = kRoom / (2 * kKv) < kMaxStages ? kRoom / (2 * kKv) : kMaxStages;   // stages
  static constexpr int kV = kRoom / kKv - kK < kMaxStages ? kRoom / kKv - kK : kMaxStages;     // (one left over goes to V: it is held a step longer)
  static constexpr int kBytes = (kK + kV) * kKv + kQ + kP + (int)sizeof(TreeCtl<R>);
  static_assert(kV >= 2 && kK >= 2 && kBytes <= kSmemMax, "shared memory");
};

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

template <int D, int R, bool kAlibi>
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_mma_kernel(DeviceView dv, const __grid_constant__ CUtensorMap map_pool, const __grid_constant__ CUtensorMap map_q,
                    const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, int layer, TreeCall tc) {
  using Smem = TreeSmem<D, R>;
  using Ctl = TreeCtl<R>;
  constexpr int KV = Smem::kKv, NK = Smem::kK, NV = Smem::kV;
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
  TreePipe* p = &ctl->pipe;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &p->abort_flag;
  const int G = dv.group, lg = __ffs(G) - 1, n_nodes = tc.n_nodes;   // (the group is a power of two)
  const int tile = blockIdx.x % tc.n_tiles, span = blockIdx.x / tc.n_tiles;
  if (smem_u32(tree_smem) & 1023u) {   // (the operand layouts need it; the first byte of a CTA's dynamic shared memory is)
    if (tid == 0) atomicOr(dv.status, kStatusProducerTimeout);
    return;
  }

  if (tid == 0) {
    tree_pipe_init(p, NK, NV);
    for (int s = 0; s < kGroups; ++s) {
      mbar_init(&ctl->agree[s], 4);
      ctl->need[s][0] = ctl->need[s][1] = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == SW + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&p->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int c = tid; c < 2 * R; c += NT) ctl->top[0][c] = ordered(-CUDART_INF_F);

  if (warp == SW && lane == 0) {
    prefetch_map(&map_pool);
    prefetch_map(&map_q);
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  cudaGridDependencySynchronize();   // (so far nothing in global memory has been touched)
  tree_find_span(dv, dv.state + (size_t)layer * dv.n_heads, tc, span, tile, p_tile);   // (scratch: the tile of P)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = p->tmem_base;
  const TreeSpan sp = *(const TreeSpan*)(p_tile + 256);
  __syncthreads();   // (the scratch becomes the tile of P)

  // Registers: the last warpgroup hands over what it does not need (3 x 128 x 168 at launch = 2 x 128 x 224 + 128 x 56).
  if (warp >= SW) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == SW) {
    tree_produce<D, R, NK, NV>(dv, map_pool, map_q, map_k, map_v, layer, tc, sp, tile, p, k_ring, v_ring, q_tile, lane);
    __syncwarp();
  } else if (warp == SW + 1) {
    // ================================================================ S^T = K Q^T
    if (lane == 0) {
      const uint64_t k_desc = operand_desc_mn(smem_u32(k_ring), 16, kOctet), q_desc = operand_desc(smem_u32(q_tile));
      const uint32_t k_lo = (uint32_t)k_desc, k_hi = (uint32_t)(k_desc >> 32), q_lo = (uint32_t)q_desc, q_hi = (uint32_t)(q_desc >> 32);
      tree_issue(p, dv, &p->drain[0], [&](unsigned gi) { return mbar_wait(&p->q_full, gi & 1, abort_flag); },
                 [&](unsigned g, int i, int n, const TreeItem&) {
        const int s = g % NK;
        if (g >= 2 && !mbar_wait(&p->s_empty[g & 1], (g / 2 - 1) & 1, abort_flag)) return false;
        if (!mbar_wait(&p->k_full[s], (g / NK) & 1, abort_flag)) return false;
        tc_fence_after();
        const uint32_t a_lo = k_lo + (uint32_t)s * (KV >> 4), d = tmem + (g & 1) * R;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)   // 16 elements = 32 bytes along the swizzled half row
          umma_words(d, a_lo + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), k_hi, q_lo + (((kk >> 2) * R * 128 + (kk & 3) * 32) >> 4), q_hi, kIdescS, kk > 0);
        umma_commit(&p->s_full[g & 1]);
        umma_commit(&p->k_empty[s]);
        if (i == n - 1) umma_commit(&p->q_empty);
        return true;
      });
    }
    __syncwarp();
  } else if (warp == SW + 2) {
    // ================================================================ O^T = V^T P^T
    if (lane == 0) {
      const uint64_t v_desc = operand_desc_mn(smem_u32(v_ring), 1024, kOctet), p_desc = operand_desc_mn(smem_u32(p_tile), 128 * kTok, 1024);
      const uint32_t v_lo = (uint32_t)v_desc, v_hi = (uint32_t)(v_desc >> 32), p_lo = (uint32_t)p_desc, p_hi = (uint32_t)(p_desc >> 32);
      const uint32_t d = tmem + kOCol;
      unsigned n_flush = 0;   // accumulators begun
      tree_issue(p, dv, &p->drain[1], [](unsigned) { return true; }, [&](unsigned g, int i, int n, const TreeItem& it) {
        const int s = g % NV;
        const int left = it.draft && i == n - 1 ? n_nodes : it.st.len - (it.begin + i) * kTok;
        const bool first = i % kFlush == 0;
        // the first product of an accumulator overwrites the one before, which must have been read out
        if (first && n_flush >= 1 && !mbar_wait(&p->o_read, (n_flush - 1) & 1, abort_flag)) return false;
        if (first) n_flush += 1;
        if (!mbar_wait(&p->v_full[s], (g / NV) & 1, abort_flag)) return false;
        if (!mbar_wait(&p->p_full, g & 1, abort_flag)) return false;
        tc_fence_after();
        const uint32_t a_lo = v_lo + (uint32_t)s * (KV >> 4);
        if (left > kTok - 16) {
#pragma unroll
          for (int kk = 0; kk < kTok / 16; ++kk)   // 16 tokens per instruction
            umma_words(d, a_lo + kk * (2 * kOctet >> 4), v_hi, p_lo + kk * (2048 >> 4), p_hi, kIdescO, kk > 0 ? 1u : (first ? 0u : 1u));
        } else {
          for (int kk = 0; kk * 16 < left; ++kk)
            umma_words(d, a_lo + kk * (2 * kOctet >> 4), v_hi, p_lo + kk * (2048 >> 4), p_hi, kIdescO, (kk > 0 || !first) ? 1u : 0u);
        }
        umma_commit(&p->p_done);
        umma_commit(&p->v_empty[s]);
        return true;
      });
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
      warp_arrive(&p->all_sync, lane);
      return warp_wait(&p->all_sync, n_all++ & 1, abort_flag);
    };
    for (unsigned gi = 0; ok; ++gi) {
      const int slot = gi % kItemSlots;
      ok = warp_wait(&p->item_full[slot], (gi / kItemSlots) & 1, abort_flag);
      if (!ok) break;
      const TreeItem it = p->item[slot];
      warp_arrive(&p->item_empty[slot], lane);
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
        place[k] = my_node[k] * dv.n_kv_heads * G + (r & (G - 1));
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
      if (tid < kTreeMaxNodes / 32) p->bad_v[(gi + 1) & 1][tid] = 0;   // (last read before the barrier that ended the item before, next written behind this item's)
      uint32_t* bad_v = p->bad_v[gi & 1];
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
      // tensor memory is added on every kFlush steps.
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
        warp_arrive(&p->o_read, lane);
      };

      const int n = it.end - it.begin + it.draft;
      for (int i = 0; i < n && ok; ++i, ++g) {
        const bool draft = it.draft && i == n - 1;
        const int slot0 = (it.begin + i) * kTok;
        const bool valid = draft ? tk < n_nodes : slot0 + tk < it.st.len;
        float rel = 0.f;   // ALiBi: this token's position, counted from the first position after the cache
        if constexpr (kAlibi)
          rel = draft ? my_depth : (float)(slot_position(min(slot0 + tk, it.st.len - 1), dv.n_sink, it.st, total) - total);
        ok = warp_wait(&p->s_full[g & 1], (g / 2) & 1, abort_flag);
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
            ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
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
          ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
          if (!ok) break;
        }
        // S is read out
        tc_fence_before();
        warp_arrive(&p->s_empty[g & 1], lane);
        if (flush_now) flush();
        // ---- sums; a weight is written as a bf16 head plus a bf16 remainder
        uint8_t* p_row = p_tile + tk * 128;
#pragma unroll
        for (int c = 0; c < NC; c += 8) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int e = c + 2 * k;
            const float w0 = __uint_as_float(v[e]), w1 = __uint_as_float(v[e + 1]);
            const uint64_t w2 = f2_pack(w0, w1);
            f2_unpack(f2_add(f2_pack(l[e], l[e + 1]), w2), l[e], l[e + 1]);
            split_weights(w2, w0, w1, hi[k], lo[k]);
          }
          const int ch = c0 + c, cl = R + ch;   // columns of heads and remainders in the 2R-column operand
          *(uint4*)(p_row + (ch >> 6) * (128 * kTok) + ((((ch & 63) >> 3) ^ (tk & 7)) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *(uint4*)(p_row + (cl >> 6) * (128 * kTok) + ((((cl & 63) >> 3) ^ (tk & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        // ---- V rows that no weight may meet: a zero weight times a NaN is a NaN.  Behind the head's last token the pool
        // may hold anything; a draft is hidden from the nodes of other branches.
        const int sv = g % NV;
        if (draft) {
          ok = warp_wait(&p->v_full[sv], (g / NV) & 1, abort_flag);
          if (!ok) break;
          if (tk < n_nodes) {
            constexpr int kChunks = D / 8 / kGroups;
            bool bad = false;
#pragma unroll 4
            for (int c = grp * kChunks; c < (grp + 1) * kChunks; ++c) {   // 16-byte chunks: this group's share of the row
              uint4* at = (uint4*)(v_ring + sv * KV + (tk >> 3) * kOctet + (c >> 3) * 1024 + (tk & 7) * 128 + (((c & 7) ^ (tk & 7)) << 4));
              uint4 x = *at;
              const bool hit = drop_non_finite(x);
              if (hit) *at = x;
              bad |= hit;
            }
            if (bad) atomicOr(&bad_v[tk >> 5], 1u << (tk & 31));
          }
        } else if (slot0 + kTok > it.st.len) {
          ok = warp_wait(&p->v_full[sv], (g / NV) & 1, abort_flag);
          if (!ok) break;
          const int first = it.st.len - slot0, last = (first + 15) / 16 * 16;
          for (int idx = tid; idx < (last - first) * (D / 8); idx += SW * 32) {
            const int t = first + idx / (D / 8), c = idx % (D / 8);
            *(uint4*)(v_ring + sv * KV + (t >> 3) * kOctet + (c >> 3) * 1024 + (t & 7) * 128 + ((c & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        warp_arrive(&p->p_full, lane);
      }
      if (!ok) break;
      // ---- the rows' results
      ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
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
        table[c] = make_float4(inv, w_seed[k] * inv, __int_as_float(direct ? place[k] : c), __int_as_float(row0 + c0 + c < rows && (!direct || is_node)));
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
            if (__float_as_int(w.w)) dst[(size_t)__float_as_int(w.z) * D] = fmaf(w.y, v_hat, w.x * acc[cb + e]);
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
            if (bad != 0.f && __float_as_int(table[c].w)) dst[(size_t)__float_as_int(table[c].z) * D] += bad;   // (this thread's own store)
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

template <int D, int R, bool kAlibi>
cudaError_t mma_launch(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& tc, long long rec_rows, int n_sms,
                       cudaStream_t s) {
  return tree_launch<D, R>(tree_mma_kernel<D, R, kAlibi>, TreeSmem<D, R>::kBytes, dv, pool_pages, layer, tc, rec_rows, n_sms, s);
}

template <int D, bool kAlibi>
cudaError_t mma_rows(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& tc, long long rec_rows, int n_sms,
                     cudaStream_t s) {
  const int rows = tc.n_nodes * dv.group;
  if (rows <= 32) return mma_launch<D, 32, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  if (rows <= 64) return mma_launch<D, 64, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  if constexpr (kAlibi) return mma_launch<D, 128, kAlibi>(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
  else return launch_tree_wide(dv, pool_pages, layer, tc, rec_rows, n_sms, s);
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
