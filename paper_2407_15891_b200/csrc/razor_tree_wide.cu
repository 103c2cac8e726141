// Tree attention on the tensor cores for more than 64 query rows per KV head: tiles of 128 rows.
//
// With a full tile of rows the narrow-operand form of the other kernel has no idle lanes to save, and its weights cost: P
// goes through shared memory, whose port then carries the matrix unit's operand reads, the copies and the softmax stores
// (2560 cycles of it per step, against 1536 of the tensor cores).  So here the QUERY ROWS are the 128-row operand,
//     S = Q K^T   [128 rows x 128 tokens],     O = P V   [128 rows x D],
// and P is written into tensor memory and read by the matrix unit from there.  Two threads share a row, each with half of
// a step's tokens and half of the output's dimensions; a row's bookkeeping is a register.  Heads and remainders of the
// weights are two products against the same V.  Spans, producer, masks of hidden rows and the lagging maximum are the other
// kernel's (so are the reasons for them); the two warps that share rows agree on a move of the maximum.
//
// 64 nodes on the 128K grouped-query shape (256 rows against 16 KV heads, 0.37 GB of kept pages): 173-175 us under continuous
// load = 540 TFLOP/s over 4 D flops a (row, token) pair, 0.38 of cuBLAS's measured rate under the same power cap and 0.32 of
// its burst rate (147 us in short runs at full clock); the other form took 214 there.
// What bounds it has not been found.  A step takes about 2700 cycles (weights and their splitting 1160, loads of S and
// maxima 480, waits and stores the rest) against 1536 of the tensor cores, but no pipe is over 42 % and the schedulers issue
// in 39 % of the cycles: two softmax warps to a scheduler wait for most of a step.  Timing-only variants moved little: 148 us
// for 151 without the remainder product, 143 with every page out of L2, and the same within 2 % with two groups of warps
// that take turns at the steps or with four threads to a row.
//
// Tensor memory (512 columns): S twice 128, P 64 columns of bf16 pairs for the heads and 64 for the remainders, O D.
// ALiBi caches stay with the other kernel: there a token's position is one thread's, here it would be every thread's.
#include "razor_tree_tc.cuh"

namespace razor {
namespace {

constexpr int kRows = 128;

struct WideCtl {
  TreePipe pipe;
  uint64_t agree[4];          // the two warps that share rows
  uint32_t need[4][2];        // [lane quarter][step parity]: step + 1 when a score outran the reference
  float top[2][2][kRows];     // [move parity][half]: a row's maximum in that half of a step
  float sum[2][kRows];        // [half]: a row's sum of weights
  alignas(16) float turn[kSoftWarps][32][20];   // a warp's rows, on their way from a thread each to neighbouring lanes
};

template <int D>
struct WideSmem {
  static constexpr int kKv = kTok * D * 2, kQ = kRows * D * 2;
  static constexpr int kRoom = kSmemMax - kQ - (int)sizeof(TreeMask) - (int)sizeof(WideCtl);
  static constexpr int kK = kRoom / (2 * kKv) < kMaxStages ? kRoom / (2 * kKv) : kMaxStages;   // stages
  static constexpr int kV = kRoom / kKv - kK < kMaxStages ? kRoom / kKv - kK : kMaxStages;     // (one left over goes to V: it is held a step longer)
  static constexpr int kBytes = (kK + kV) * kKv + kQ + (int)sizeof(TreeMask) + (int)sizeof(WideCtl);
  static_assert(kV >= 2 && kK >= 2 && kBytes <= kSmemMax && sizeof(TreeMask) >= 1024 && sizeof(TreeMask) % 16 == 0, "shared memory");
};

// 32 consecutive columns of this thread's lane into tensor memory; complete after tcgen05.wait::st.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
  tmem_st16(taddr, v);
  tmem_st16(taddr + 16, v + 16);
}

template <int D>
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_wide_kernel(DeviceView dv, const __grid_constant__ CUtensorMap map_pool, const __grid_constant__ CUtensorMap map_q,
                     const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, int layer, TreeCall tc) {
  using Smem = WideSmem<D>;
  constexpr int KV = Smem::kKv, NK = Smem::kK, NV = Smem::kV, SW = kSoftWarps;
  constexpr int HT = kTok / 2, HD = D / 2;                // tokens and output dimensions of a thread
  constexpr uint32_t kOctet = 8 * D * 2;
  constexpr uint32_t kTmemCols = 512, kPCol = 2 * kTok, kPLo = kTok / 2, kOCol = 3 * kTok;
  constexpr uint32_t kIdescS = instr_desc_bf16(kRows, kTok, false), kIdescO = instr_desc_bf16(kRows, D, true);

  extern __shared__ __align__(1024) uint8_t wide_smem[];
  uint8_t* k_ring = wide_smem;
  uint8_t* v_ring = k_ring + NK * KV;
  uint8_t* q_tile = v_ring + NV * KV;                     // [half][row][128 B]
  TreeMask* mask = (TreeMask*)(q_tile + Smem::kQ);
  WideCtl* ctl = (WideCtl*)(mask + 1);
  TreePipe* p = &ctl->pipe;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &p->abort_flag;
  const int G = dv.group, lg = __ffs(G) - 1, n_nodes = tc.n_nodes;   // (the group is a power of two)
  const int tile = blockIdx.x % tc.n_tiles, span = blockIdx.x / tc.n_tiles;
  if (smem_u32(wide_smem) & 1023u) {   // (the operand layouts need it; the first byte of a CTA's dynamic shared memory is)
    if (tid == 0) atomicOr(dv.status, kStatusProducerTimeout);
    return;
  }
  if (tid == 0) {
    tree_pipe_init(p, NK, NV);
    for (int s = 0; s < 4; ++s) {
      mbar_init(&ctl->agree[s], 2);
      ctl->need[s][0] = ctl->need[s][1] = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == SW + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&p->tmem_base)), "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == SW && lane == 0) {
    prefetch_map(&map_pool);
    prefetch_map(&map_q);
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  cudaGridDependencySynchronize();   // (so far nothing in global memory has been touched)
  tree_find_span(dv, dv.state + (size_t)layer * dv.n_heads, tc, span, tile, (uint8_t*)mask);   // (scratch: the mask)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = p->tmem_base;
  const TreeSpan sp = *(const TreeSpan*)((const uint8_t*)mask + 256);
  __syncthreads();   // (the scratch becomes the mask)

  // Registers: the last warpgroup hands over what it does not need (3 x 128 x 168 at launch = 2 x 128 x 224 + 128 x 56).
  if (warp >= SW) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == SW) {
      tree_produce<D, kRows, NK, NV>(dv, map_pool, map_q, map_k, map_v, layer, tc, sp, tile, p, k_ring, v_ring, q_tile, lane);
      __syncwarp();
    } else if (warp == SW + 1) {
      // ============================================================== S = Q K^T
      if (lane == 0) {
        const uint64_t k_desc = operand_desc_mn(smem_u32(k_ring), 16, kOctet), q_desc = operand_desc(smem_u32(q_tile));
        const uint32_t k_lo = (uint32_t)k_desc, k_hi = (uint32_t)(k_desc >> 32), q_lo = (uint32_t)q_desc, q_hi = (uint32_t)(q_desc >> 32);
        tree_issue(p, dv, &p->drain[0], [&](unsigned gi) { return mbar_wait(&p->q_full, gi & 1, abort_flag); },
                   [&](unsigned g, int i, int n, const TreeItem&) {
          const int s = g % NK;
          if (g >= 2 && !mbar_wait(&p->s_empty[g & 1], (g / 2 - 1) & 1, abort_flag)) return false;
          if (!mbar_wait(&p->k_full[s], (g / NK) & 1, abort_flag)) return false;
          tc_fence_after();
          const uint32_t b_lo = k_lo + (uint32_t)s * (KV >> 4), d = tmem + (g & 1) * kTok;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)   // 16 elements = 32 bytes along the swizzled half row
            umma_words(d, q_lo + (((kk >> 2) * kRows * 128 + (kk & 3) * 32) >> 4), q_hi, b_lo + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), k_hi, kIdescS, kk > 0);
          umma_commit(&p->s_full[g & 1]);
          umma_commit(&p->k_empty[s]);
          if (i == n - 1) umma_commit(&p->q_empty);
          return true;
        });
      }
      __syncwarp();
    } else if (warp == SW + 2) {
      // ============================================================== O = P V
      if (lane == 0) {
        const uint64_t v_desc = operand_desc_mn(smem_u32(v_ring), 1024, kOctet);
        const uint32_t v_lo = (uint32_t)v_desc, v_hi = (uint32_t)(v_desc >> 32), d = tmem + kOCol, a = tmem + kPCol;
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
          const uint32_t b_lo = v_lo + (uint32_t)s * (KV >> 4);
          if (left > kTok - 16) {
#pragma unroll
            for (int kk = 0; kk < kTok / 16; ++kk) {   // 16 tokens per instruction: 8 columns of pairs
              umma_words_tmem_a(d, a + kk * 8, b_lo + kk * (2 * kOctet >> 4), v_hi, kIdescO, kk > 0 ? 1u : (first ? 0u : 1u));
              umma_words_tmem_a(d, a + kPLo + kk * 8, b_lo + kk * (2 * kOctet >> 4), v_hi, kIdescO, 1u);
            }
          } else {
            for (int kk = 0; kk * 16 < left; ++kk) {
              umma_words_tmem_a(d, a + kk * 8, b_lo + kk * (2 * kOctet >> 4), v_hi, kIdescO, (kk > 0 || !first) ? 1u : 0u);
              umma_words_tmem_a(d, a + kPLo + kk * 8, b_lo + kk * (2 * kOctet >> 4), v_hi, kIdescO, 1u);
            }
          }
          umma_commit(&p->p_done);
          umma_commit(&p->v_empty[s]);
          return true;
        });
      }
      __syncwarp();
    }
  } else {
    // ================================================================ softmax and epilogue: two threads per row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int half = warp >> 2, quarter = warp & 3;         // half of a step's tokens; tensor-memory lane quarter
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_cols = half * HT, o_cols = kOCol + half * HD, p_cols = kPCol + half * (HT / 2);
    const float scale_log2 = dv.scale_log2;
    const uint64_t scale2 = f2_pack(scale_log2, scale_log2);
    const int rows = n_nodes * G, r = tile * kRows + row;
    const bool is_row = r < rows, warp_live = tile * kRows + quarter * 32 < rows;   // (a warp behind the last row only keeps pace)
    const int node = min(r, rows - 1) >> lg, j = min(r, rows - 1) & (G - 1);
    unsigned g = 0, n_agree = 0, n_all = 0, n_top = 0;
    int mask_b = -1;              // the sequence whose tree the next two belong to
    uint32_t vis[2] = {0, 0};     // tokens of this thread's half of the tree that the row sees
    bool live = false;            // the row is a node of the tree
    bool ok = true;
    auto pair_sync = [&]() -> bool {   // the other warp of these rows
      warp_arrive(&ctl->agree[quarter], lane);
      return warp_wait(&ctl->agree[quarter], n_agree++ & 1, abort_flag);
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
      const int32_t* parent = tc.parent + (size_t)b * n_nodes;
      if (it.draft && b != mask_b) {   // (the heads of a sequence follow one another: its tree is worked out once)
        mask_b = b;
        tree_mask_load(*mask, parent, n_nodes, tid, SW * 32);
        if (!(ok = all_sync())) break;
        tree_mask_walk(*mask, n_nodes, tid, SW * 32);
        if (!(ok = all_sync())) break;
        live = is_row && tree_sees(*mask, node, node);
#pragma unroll
        for (int k = 0; k < 2; ++k) vis[k] = live ? mask->see[node][half * 2 + k] : 0u;
        if (!(ok = all_sync())) break;
      }
      if (tid < kTreeMaxNodes / 32) p->bad_v[(gi + 1) & 1][tid] = 0;   // (last read before the barrier that ended the item before, next written behind this item's)
      uint32_t* bad_v = p->bad_v[gi & 1];
      // ---- reference maximum: minus infinity, or the compensation token's logit (Eq. 5: weight N_d exp(s_c), value v_hat),
      // whose weight is carried apart and added at the end
      float m_ref = -CUDART_INF_F, w_seed = 0.f, l = 0.f;
      if (it.seed && warp_live) {
        const uint4* src = (const uint4*)((const __nv_bfloat16*)tc.q + (size_t)b * tc.q_stride_b + (size_t)node * tc.q_stride_t + ((size_t)g_kv * G + j) * D);
        const float4* k_hat = (const float4*)(dv.comp_mean + hs * 2 * D);
        float s = 0.f;
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          float x[8];
          Elem<__nv_bfloat16>::unpack(__ldg(src + c), x);
          const float4 k0 = k_hat[2 * c], k1 = k_hat[2 * c + 1];
          s = fmaf(x[0], k0.x, fmaf(x[1], k0.y, fmaf(x[2], k0.z, fmaf(x[3], k0.w, s))));
          s = fmaf(x[4], k1.x, fmaf(x[5], k1.y, fmaf(x[6], k1.z, fmaf(x[7], k1.w, s))));
        }
        m_ref = fmaf(s, scale_log2, log2f((float)it.st.n_drop));
        w_seed = 1.f;
      }
      // This thread's half of the row's output; the accumulator in tensor memory is added on every kFlush steps.
      float acc[HD];
#pragma unroll
      for (int c = 0; c < HD; ++c) acc[c] = 0.f;
      auto flush = [&]() {
        if (warp_live) {
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < HD; c += 16) {
            uint32_t o[16];
            tmem_load<16>(lane_addr + o_cols + (uint32_t)c, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[c + e] += __uint_as_float(o[e]);
          }
          tc_fence_before();
        }
        warp_arrive(&p->o_read, lane);
      };

      const int n = it.end - it.begin + it.draft;
      for (int i = 0; i < n && ok; ++i, ++g) {
        const bool draft = it.draft && i == n - 1;
        const int slot0 = (it.begin + i) * kTok;
        const int n_valid = (draft ? kTok : it.st.len - slot0) - half * HT;   // of this thread's tokens, from its first on
        bool flush_now = i > 0 && i % kFlush == 0;
        ok = warp_wait(&p->s_full[g & 1], (g / 2) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (warp_live) {
          uint32_t v[HT];
          // scores to the log2 domain, minus the reference; returns whether one outran it
          auto scores = [&]() -> bool {
            tmem_load<HT>(lane_addr + (g & 1) * kTok + s_cols, v);
            const float nm = m_ref == -CUDART_INF_F ? -kLow : -m_ref;
            const uint64_t nm2 = f2_pack(nm, nm);
#pragma unroll
            for (int c = 0; c < HT; c += 2) {
              float t0, t1;
              f2_unpack(f2_fma(f2_pack(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), scale2, nm2), t0, t1);
              v[c] = __float_as_uint(t0);
              v[c + 1] = __float_as_uint(t1);
            }
            if (draft) {
#pragma unroll
              for (int c = 0; c < HT; ++c)
                if (!(vis[c >> 5] >> (c & 31) & 1)) v[c] = 0xff800000u;
            } else if (n_valid < HT) {
#pragma unroll
              for (int c = 0; c < HT; ++c)
                if (c >= n_valid) v[c] = 0xff800000u;
            }
            float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F;
#pragma unroll
            for (int c = 0; c < HT; c += 4) {
              m0 = max3(m0, __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
              m1 = max3(m1, __uint_as_float(v[c + 2]), __uint_as_float(v[c + 3]));
            }
            return fmaxf(m0, m1) > kLag;
          };
          // Weights, their sum, and their two halves for the product: a bf16 head plus a bf16 remainder,
          // column c of either holding the pair of tokens 2 c and 2 c + 1 (remainders replace the scores).  One loop: the
          // exponentials of a pair go to the special-function unit while the pair before is split.
          uint32_t hi[HT / 2];
          float step_sum;
          auto weights = [&]() {
            uint64_t sum2[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < HT / 2; ++c) {
              const float w0 = fast_exp2(__uint_as_float(v[2 * c])), w1 = fast_exp2(__uint_as_float(v[2 * c + 1]));
              const uint64_t w2 = f2_pack(w0, w1);
              sum2[c & 1] = f2_add(sum2[c & 1], w2);
              split_weights(w2, w0, w1, hi[c], v[c]);
            }
            float a0, a1;
            f2_unpack(f2_add(sum2[0], sum2[1]), a0, a1);
            step_sum = a0 + a1;
          };
          const bool outran = scores();
          if (__any_sync(0xffffffffu, outran) && lane == 0) *(volatile uint32_t*)&ctl->need[quarter][g & 1] = g + 1;
          warp_arrive(&ctl->agree[quarter], lane);
          weights();
          ok = warp_wait(&ctl->agree[quarter], n_agree++ & 1, abort_flag);
          if (!ok) break;
          if (*(volatile uint32_t*)&ctl->need[quarter][g & 1] == g + 1) {
            // ---- move the references that were outrun to the maximum of what has been seen
            if (g > 0) {
              ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
              if (!ok) break;
            }
            if (flush_now) flush();
            flush_now = false;
            float mx = -CUDART_INF_F;
#pragma unroll 1
            for (int c = 0; c < HT; c += 16) {
              uint32_t s[16];
              tmem_load<16>(lane_addr + (g & 1) * kTok + s_cols + c, s);
              const uint32_t see = draft ? (c < 32 ? vis[0] : vis[1]) >> (c & 31) : 0xffffu;
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if ((see >> e & 1) && c + e < n_valid) mx = fmaxf(mx, __uint_as_float(s[e]) * scale_log2);
            }
            float (*top)[kRows] = ctl->top[n_top++ & 1];   // (the other half of a pair may still read the move before's)
            top[half][row] = mx;
            if (!(ok = pair_sync())) break;
            const float seen = fmaxf(mx, top[half ^ 1][row]);
            // (a row moves only when it has been outrun itself: what it computes does not depend on the rows beside it)
            const float m_new = m_ref == -CUDART_INF_F || seen > m_ref + kLag ? fmaxf(m_ref, seen) : m_ref;
            const float f = m_ref == -CUDART_INF_F ? 0.f : fast_exp2(m_ref - m_new);
            m_ref = m_new;
            w_seed *= f;
            if (i > 0) {   // (an item's first step finds nothing to rescale)
              l *= f;
#pragma unroll
              for (int c = 0; c < HD; ++c) acc[c] *= f;
              if (i % kFlush != 0) {   // the accumulator holds products of this item
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < HD; c += 16) {
                  uint32_t o[16];
                  tmem_load<16>(lane_addr + o_cols + (uint32_t)c, o);
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                  tmem_st16(lane_addr + o_cols + (uint32_t)c, o);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
              }
            }
            (void)scores();
            weights();
          } else if (g > 0) {   // the product of the step before must have read its weights
            ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
            if (!ok) break;
          }
          tc_fence_after();   // (P's columns are written again)
          // S is read out
          tc_fence_before();
          warp_arrive(&p->s_empty[g & 1], lane);
          if (flush_now) flush();
          tmem_st32(lane_addr + p_cols, hi);
          tmem_st32(lane_addr + p_cols + kPLo, v);
          l += step_sum;
        } else {
          tc_fence_before();
          warp_arrive(&p->s_empty[g & 1], lane);
          if (g > 0) ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
          if (!ok) break;
          if (flush_now) flush();
        }
        // ---- V rows that no weight may meet: a zero weight times a NaN is a NaN.  Behind the head's last token the pool
        // may hold anything; a draft is hidden from the nodes of other branches.
        const int sv = g % NV;
        if (draft) {
          ok = warp_wait(&p->v_full[sv], (g / NV) & 1, abort_flag);
          if (!ok) break;
          if (row < n_nodes) {   // (this thread looks after the draft with its row's number, its half of the dimensions)
            bool bad = false;
#pragma unroll 4
            for (int c = half * (D / 16); c < (half + 1) * (D / 16); ++c) {
              uint4* at = (uint4*)(v_ring + sv * KV + (row >> 3) * kOctet + (c >> 3) * 1024 + (row & 7) * 128 + (((c & 7) ^ (row & 7)) << 4));
              uint4 x = *at;
              const bool hit = drop_non_finite(x);
              if (hit) *at = x;
              bad |= hit;
            }
            if (bad) atomicOr(&bad_v[row >> 5], 1u << (row & 31));
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
        if (warp_live) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        warp_arrive(&p->p_full, lane);
      }
      if (!ok) break;
      // ---- the rows' results
      ok = warp_wait(&p->p_done, (g - 1) & 1, abort_flag);
      if (!ok) break;
      flush();
      if (warp_live) {
        ctl->sum[half][row] = l;
        if (!(ok = pair_sync())) break;
        const float l_all = (ctl->sum[0][row] + ctl->sum[1][row]) + w_seed;
        const bool direct = it.rec < 0;
        const float inv = direct ? 1.f / l_all : 1.f;
        if (!direct && half == 0)   // (a negative sum marks an absent node's row for the combine kernel)
          dv.rec_ml[(size_t)it.rec * kRows + row] = make_float2(m_ref, it.draft && !live ? -1.f : l_all);
        // Sixteen dimensions at a time through shared memory, so that four neighbouring lanes store a row's 64 bytes.
        const size_t row_at = direct ? (((size_t)b * n_nodes + node) * dv.n_kv_heads * G + (size_t)g_kv * G + j) * D : ((size_t)it.rec * kRows + row) * D;
        const uint32_t wanted = __ballot_sync(0xffffffffu, direct ? live : is_row);
        float* all = direct ? tc.out : dv.rec_o;
        const float4* v_hat = (const float4*)(dv.comp_mean + hs * 2 * D + D + half * HD);
        float (*turn)[20] = ctl->turn[warp];   // (rows 80 bytes apart: 16-byte accesses of eight lanes hit different banks)
#pragma unroll
        for (int c = 0; c < HD; c += 16) {
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 vh = it.seed ? v_hat[(c + e) / 4] : make_float4(0.f, 0.f, 0.f, 0.f);
            *(float4*)&turn[lane][e] = make_float4(fmaf(w_seed, vh.x, acc[c + e]) * inv, fmaf(w_seed, vh.y, acc[c + e + 1]) * inv,
                                                   fmaf(w_seed, vh.z, acc[c + e + 2]) * inv, fmaf(w_seed, vh.w, acc[c + e + 3]) * inv);
          }
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int to = k * 8 + lane / 4;
            const size_t at = __shfl_sync(0xffffffffu, row_at, to);
            if (wanted >> to & 1) *(float4*)(all + at + half * HD + c + lane % 4 * 4) = *(const float4*)&turn[to][lane % 4 * 4];
          }
          __syncwarp();
        }
        // The NaN and infinities that were taken out of the drafts' V reach the rows that see them.
        if (it.draft && (bad_v[0] | bad_v[1] | bad_v[2] | bad_v[3]) != 0 && (direct ? live : is_row)) {
          float* dst = all + row_at + half * HD;   // (stored by lanes of this warp, before its last __syncwarp)
#pragma unroll 1
          for (int nd = 0; nd <= node; ++nd) {
            if (!(bad_v[nd >> 5] >> (nd & 31) & 1) || !walk_sees(parent, node, nd)) continue;
            const __nv_bfloat16* src = (const __nv_bfloat16*)tc.v + (size_t)b * tc.kv_stride_b + (size_t)nd * tc.kv_stride_t + (size_t)g_kv * D + half * HD;
#pragma unroll 1
            for (int c = 0; c < HD; ++c) {
              const float y = __bfloat162float(src[c]);
              if (!(fabsf(y) < CUDART_INF_F)) dst[c] += y;
            }
          }
        }
      }
      if (!(ok = all_sync())) break;   // (the sums, the mask and bad_v are done with)
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

}  // namespace

cudaError_t launch_tree_wide(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& tc, long long rec_rows,
                             int n_sms, cudaStream_t s) {
  return dv.head_dim == 128 ? tree_launch<128, kRows>(tree_wide_kernel<128>, WideSmem<128>::kBytes, dv, pool_pages, layer, tc, rec_rows, n_sms, s)
                            : tree_launch<64, kRows>(tree_wide_kernel<64>, WideSmem<64>::kBytes, dv, pool_pages, layer, tc, rec_rows, n_sms, s);
}

}  // namespace razor
