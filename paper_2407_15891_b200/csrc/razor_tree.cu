// Attention of a tree of drafted tokens over an fp32 cache (the reference configurations; a bf16 cache runs on the
// tensor-core kernels).
//
// A node attends to every kept token of its head, to the compensation token with its count (Eq. 5), and to itself and
// its ancestors in the tree; the drafts' K and V are read from the caller's buffers and the cache stays as it is.
// Query rows of a KV head: r = t * group + j for node t and query head j of the group.
//
// The tensor cores have no fp32 product, so this runs on the CUDA cores.  The work is cut as the tensor-core kernels cut
// theirs (spans of the heads' steps laid end to end, records of the heads that a cut runs through); inside a CTA each of
// twelve warps streams groups of eight tokens of its own through two stages of shared memory, with its own running maximum,
// sum and output for the eight rows of the tile, so that warps meet only when an item ends.
//   scores: a lane has one token and a quarter of the dimensions and goes through the rows, whose queries are the same for
//           eight lanes; the quarters are added by exchanging halves, which leaves a lane with two finished scores;
//   output: a lane has four dimensions of every row; the weights come back through shared memory, the same for all lanes.
// Every K and V value read from shared memory meets eight rows, two multiply-adds to an instruction.  What bounds it: up to
// eight rows the stream of pages (4 x 16 heads of 16384 tokens, a quarter of them whole, 0.47 GB: 90 us = 5.2 TB/s = 0.81
// of the measured copy rate); with more, the shared-memory port, since queries and weights are read again for every group
// of tokens (64 rows: 600 us = 25 TFLOP/s).
#include <math_constants.h>

#include <algorithm>

#include "razor_common.cuh"
#include "razor_tc.cuh"
#include "razor_tree_tc.cuh"

namespace razor {
namespace {

constexpr int kGroup = 8;                          // tokens of a warp's turn: half a page
constexpr int kRowWarps = kTreeThreads / 32;
constexpr int R = 8;                               // query rows of a CTA (sixteen: 9 to 16 rows 171 us for 165, 17 to 24 rows 317 for 240)

template <int D>
struct RowsSmem {
  static constexpr int kStage = 2 * kGroup * D * 4;   // K rows, V rows
  static constexpr int kStages = kRowWarps * 2 * kStage;
  static constexpr int kFold = kRowWarps * R * D * 4;   // the warps' outputs, in the place of the stages
  static constexpr int kQ = R * D * 4, kW = kRowWarps * kGroup * R * 4;
  static constexpr int kBytes = kStages + kQ + kW + kRowWarps * R * 8 + (int)sizeof(TreeMask);
  static_assert(kFold <= kStages && kBytes <= kSmemMax && sizeof(TreeMask) % 16 == 0, "shared memory");
};

__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_rows_kernel(DeviceView dv, int layer, TreeCall tc) {
  using Geo = RowGeom<float, D>;
  using Smem = RowsSmem<D>;
  constexpr int LPR = Geo::kLpr, RL = R / 4;            // 16-byte chunks of a row; finished scores of a lane
  constexpr int TPI = 32 / LPR;                         // tokens that a warp's V load covers
  extern __shared__ __align__(1024) uint8_t rows_smem[];
  float* q_tile = (float*)(rows_smem + Smem::kStages);  // [row][D]
  float* w_all = q_tile + R * D;                        // [warp][token][row]
  float2* ml = (float2*)(w_all + kRowWarps * kGroup * R);   // [warp][row]
  TreeMask* mask = (TreeMask*)(ml + kRowWarps * R);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* stage = rows_smem + warp * 2 * Smem::kStage;
  float* w_tile = w_all + warp * kGroup * R;
  const int tile = blockIdx.x % tc.n_tiles, span = blockIdx.x / tc.n_tiles;
  const int G = dv.group, n_nodes = tc.n_nodes, rows = n_nodes * G, row0 = tile * R;
  cudaGridDependencySynchronize();   // (so far nothing in global memory has been touched)
  const HeadState* states = dv.state + (size_t)layer * dv.n_heads;
  tree_find_span(dv, states, tc, span, tile, rows_smem);
  __syncthreads();
  const TreeSpan sp = *(const TreeSpan*)(rows_smem + 256);
  __syncthreads();   // (the scratch becomes stages)

  const int tok = lane & 7, quarter = lane >> 3;        // of the scores
  const int my_row = (quarter & 1) * (R / 2) + (quarter >> 1) * (R / 4);   // first of the rows whose scores end up here
  const int chunk = lane % LPR, sub = lane / LPR;       // of the output
  int node[RL];
  float slope[RL];
#pragma unroll
  for (int e = 0; e < RL; ++e) node[e] = min(row0 + my_row + e, rows - 1) / G;
  int head = sp.head, y = sp.step, mask_b = -1;
  long long todo = sp.head < 0 ? 0 : sp.end - sp.begin;
  HeadState st = sp.st;
  while (todo > 0) {
    const TreeItem it = tree_item(dv, head, y, todo, st);
    const int b = head / dv.n_kv_heads, g = head % dv.n_kv_heads;
    const size_t hs = (size_t)layer * dv.n_heads + head;
    const int32_t* pt = dv.page_table + hs * dv.max_pages;
    const int total = st.len + st.n_drop;
    const bool alibi = dv.alibi != 0;
    // ---- the item's turns: the compensation token, half pages of the cache, eights of the drafts
    const int h0 = it.begin * (kTok / kGroup), n_cache = (int)((min((long long)it.end * kTok, (long long)st.len) - (long long)it.begin * kTok + kGroup - 1) / kGroup);
    const int first_cache = it.seed, first_draft = first_cache + max(n_cache, 0), n_turns = first_draft + (it.draft ? (n_nodes + kGroup - 1) / kGroup : 0);
    auto page_of = [&](int x) { return x >= first_cache && x < first_draft ? pt[(h0 + x - first_cache) >> 1] : 0; };
    auto issue = [&](int x, int page, uint8_t* dst) {
      if (x >= first_draft) {
        const int n0 = (x - first_draft) * kGroup;
#pragma unroll
        for (int i = 0; i < kGroup / TPI; ++i) {
          const int t = i * TPI + sub;
          const size_t at = (size_t)b * tc.kv_stride_b + (size_t)min(n0 + t, n_nodes - 1) * tc.kv_stride_t + (size_t)g * D + chunk * 4;
          copy16(dst + (t * LPR + swz(t, chunk)) * 16, (const float*)tc.k + at);
          copy16(dst + Smem::kStage / 2 + (t * LPR + swz(t, chunk)) * 16, (const float*)tc.v + at);
        }
      } else if (x >= first_cache) {   // (rows behind the head's last token are the page's own and are not looked at)
        const uint8_t* src = dv.pool + (size_t)page * dv.page_bytes + (size_t)((h0 + x - first_cache) & 1) * kGroup * Geo::kRowBytes + lane * 16;
#pragma unroll
        for (int i = 0; i < kGroup / TPI; ++i) {
          copy16(dst + (i * 32 + lane) * 16, src + i * 512);
          copy16(dst + Smem::kStage / 2 + (i * 32 + lane) * 16, src + kPageTokens * Geo::kRowBytes + i * 512);
        }
      } else if (lane < LPR) {
        const float* mean = dv.comp_mean + hs * 2 * D;
        copy16(dst + lane * 16, mean + lane * 4);
        copy16(dst + Smem::kStage / 2 + lane * 16, mean + D + lane * 4);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int page_next = warp + kRowWarps < n_turns ? page_of(warp + kRowWarps) : 0;
    if (warp < n_turns) issue(warp, page_of(warp), stage);
    // ---- queries and, for a new sequence, its tree
    for (int i = tid; i < R * LPR; i += kTreeThreads) {
      const int r = min(row0 + i / LPR, rows - 1), c = i % LPR;
      const float* src = (const float*)tc.q + (size_t)b * tc.q_stride_b + (size_t)(r / G) * tc.q_stride_t + ((size_t)g * G + r % G) * D + c * 4;
      *(float4*)(q_tile + (i / LPR) * D + c * 4) = __ldg((const float4*)src);
    }
    const bool new_tree = b != mask_b;
    mask_b = b;
    if (new_tree) tree_mask_load(*mask, tc.parent + (size_t)b * n_nodes, n_nodes, tid, kTreeThreads);
    __syncthreads();
    if (new_tree) {
      tree_mask_walk(*mask, n_nodes, tid, kTreeThreads);
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < RL; ++e)
      slope[e] = alibi ? dv.alibi_slopes[(size_t)layer * dv.n_kv_heads * G + (size_t)g * G + min(row0 + my_row + e, rows - 1) % G] : 0.f;

    float m[RL], l[RL];
    uint64_t o[R][2];
#pragma unroll
    for (int e = 0; e < RL; ++e) { m[e] = -CUDART_INF_F; l[e] = 0.f; }
#pragma unroll
    for (int r = 0; r < R; ++r) o[r][0] = o[r][1] = f2_pack(0.f, 0.f);
    int at_stage = 0;
    for (int x = warp; x < n_turns; x += kRowWarps, at_stage ^= 1) {
      if (x + kRowWarps < n_turns) {
        issue(x + kRowWarps, page_next, stage + (at_stage ^ 1) * Smem::kStage);
        page_next = page_of(x + 2 * kRowWarps);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncwarp();
      const uint8_t* ks = stage + at_stage * Smem::kStage;
      const uint8_t* vs = ks + Smem::kStage / 2;
      // ---- scores
      float s[R];
      {
        uint64_t s2[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s2[r] = f2_pack(0.f, 0.f);
#pragma unroll 4
        for (int c = quarter; c < LPR; c += 4) {
          const ulonglong2 k = *(const ulonglong2*)(ks + (tok * LPR + swz(tok, c)) * 16);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const ulonglong2 q = *(const ulonglong2*)(q_tile + r * D + c * 4);
            s2[r] = f2_fma(q.y, k.y, f2_fma(q.x, k.x, s2[r]));
          }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float a0, a1;
          f2_unpack(s2[r], a0, a1);
          s[r] = a0 + a1;
        }
      }
      const bool up0 = quarter & 1, up1 = quarter >> 1;
#pragma unroll
      for (int r = 0; r < R / 2; ++r) {
        const float give = up0 ? s[r] : s[r + R / 2], keep = up0 ? s[r + R / 2] : s[r];
        s[r] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
      }
#pragma unroll
      for (int r = 0; r < R / 4; ++r) {
        const float give = up1 ? s[r] : s[r + R / 4], keep = up1 ? s[r + R / 4] : s[r];
        s[r] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
      }
      // ---- what kind of token this lane has, and which of its rows see it
      const bool draft = x >= first_draft, cache = !draft && x >= first_cache;
      const int at = draft ? (x - first_draft) * kGroup + tok : (h0 + x - first_cache) * kGroup + tok;
      const int n_tok = draft ? min(kGroup, n_nodes - (x - first_draft) * kGroup) : (cache ? min(kGroup, st.len - (h0 + x - first_cache) * kGroup) : 1);
      uint32_t see = 0;
      const int pos = draft ? total + mask->depth[min(at, n_nodes - 1)] : slot_position(at, dv.n_sink, st, total);
      const float count_log2 = cache || draft ? 0.f : log2f((float)st.n_drop);
      bool rises = false;
      float up[RL];
#pragma unroll
      for (int e = 0; e < RL; ++e) {
        const bool sees = tok < n_tok && (!draft || tree_sees(*mask, node[e], at));
        see |= (sees ? 1u : 0u) << (my_row + e);
        float z = fmaf(s[e], dv.scale_log2, count_log2);
        if (alibi && (cache || draft)) z -= slope[e] * (float)(total + mask->depth[node[e]] - pos);
        s[e] = sees ? z : -CUDART_INF_F;
        float mx = s[e];
#pragma unroll
        for (int off = 1; off < 8; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float mn = fmaxf(m[e], mx), mu = mn == -CUDART_INF_F ? 0.f : mn;
        up[e] = fast_exp2(m[e] - mu);
        rises |= mn > m[e];
        m[e] = mn;
        s[e] = fast_exp2(s[e] - mu);
        l[e] = fmaf(l[e], up[e], s[e]);
      }
#pragma unroll
      for (int e = 0; e < RL; e += 2) *(float2*)(w_tile + tok * R + my_row + e) = make_float2(s[e], s[e + 1]);
      if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int q = (r / (R / 2)) | ((r / (R / 4)) & 1) << 1;
          const float c = __shfl_sync(0xffffffffu, up[r % (R / 4)], q * 8);
          const uint64_t c2 = f2_pack(c, c);
          o[r][0] = f2_fma(o[r][0], c2, f2_pack(0.f, 0.f));
          o[r][1] = f2_fma(o[r][1], c2, f2_pack(0.f, 0.f));
        }
      }
      __syncwarp();
      // ---- output
      if (draft) {   // (a draft that a row does not see must not reach it, whatever it holds)
        see |= __shfl_xor_sync(0xffffffffu, see, 8);
        see |= __shfl_xor_sync(0xffffffffu, see, 16);
#pragma unroll 1
        for (int t0 = 0; t0 < kGroup; t0 += TPI) {
          const int t = t0 + sub;
          const uint32_t who = __shfl_sync(0xffffffffu, see, t);
          const ulonglong2 v = *(const ulonglong2*)(vs + (t * LPR + swz(t, chunk)) * 16);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float w = w_tile[t * R + r];
            if (who >> r & 1) {
              o[r][0] = f2_fma(f2_pack(w, w), v.x, o[r][0]);
              o[r][1] = f2_fma(f2_pack(w, w), v.y, o[r][1]);
            }
          }
        }
      } else {
#pragma unroll 2
        for (int t0 = 0; t0 < n_tok; t0 += TPI) {
          const int t = t0 + sub;
          if (TPI > 1 && t >= n_tok) continue;
          const ulonglong2 v = *(const ulonglong2*)(vs + (t * LPR + swz(t, chunk)) * 16);
#pragma unroll
          for (int r = 0; r < R; r += 4) {
            const float4 w = *(const float4*)(w_tile + t * R + r);
            o[r][0] = f2_fma(f2_pack(w.x, w.x), v.x, o[r][0]);
            o[r][1] = f2_fma(f2_pack(w.x, w.x), v.y, o[r][1]);
            o[r + 1][0] = f2_fma(f2_pack(w.y, w.y), v.x, o[r + 1][0]);
            o[r + 1][1] = f2_fma(f2_pack(w.y, w.y), v.y, o[r + 1][1]);
            o[r + 2][0] = f2_fma(f2_pack(w.z, w.z), v.x, o[r + 2][0]);
            o[r + 2][1] = f2_fma(f2_pack(w.z, w.z), v.y, o[r + 2][1]);
            o[r + 3][0] = f2_fma(f2_pack(w.w, w.w), v.x, o[r + 3][0]);
            o[r + 3][1] = f2_fma(f2_pack(w.w, w.w), v.y, o[r + 3][1]);
          }
        }
      }
      __syncwarp();   // (the stage and the weights are written again)
    }
    // ---- the warps' states of each row, folded in order
#pragma unroll
    for (int e = 0; e < RL; ++e) {
      float sum = l[e];
#pragma unroll
      for (int off = 1; off < 8; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      if (tok == 0) ml[warp * R + my_row + e] = make_float2(m[e], sum);
    }
    __syncthreads();   // (every warp is through with its stages)
    float* fold = (float*)rows_smem;   // [warp][row][D]
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float4 x;
      f2_unpack(o[r][0], x.x, x.y);
      f2_unpack(o[r][1], x.z, x.w);
      if (TPI > 1) {
        x.x += __shfl_xor_sync(0xffffffffu, x.x, 16);
        x.y += __shfl_xor_sync(0xffffffffu, x.y, 16);
        x.z += __shfl_xor_sync(0xffffffffu, x.z, 16);
        x.w += __shfl_xor_sync(0xffffffffu, x.w, 16);
      }
      if (lane < LPR) *(float4*)(fold + ((size_t)warp * R + r) * D + chunk * 4) = x;
    }
    __syncthreads();
    for (int i = tid; i < R * LPR; i += kTreeThreads) {
      const int r = i / LPR, c = i % LPR, rr = row0 + r;
      if (rr >= rows) continue;
      float mx = -CUDART_INF_F, lt = 0.f;
      for (int k = 0; k < kRowWarps; ++k) mx = fmaxf(mx, ml[k * R + r].x);
      const float mu = mx == -CUDART_INF_F ? 0.f : mx;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < kRowWarps; ++k) {
        const float f = fast_exp2(ml[k * R + r].x - mu);
        const float4 z = *(const float4*)(fold + ((size_t)k * R + r) * D + c * 4);
        lt = fmaf(ml[k * R + r].y, f, lt);
        acc.x = fmaf(z.x, f, acc.x); acc.y = fmaf(z.y, f, acc.y); acc.z = fmaf(z.z, f, acc.z); acc.w = fmaf(z.w, f, acc.w);
      }
      const int t = rr / G, j = rr % G;
      const bool live = tree_sees(*mask, t, t);
      if (it.rec < 0) {
        const float inv = 1.f / lt;
        if (live) *(float4*)(tc.out + (((size_t)b * n_nodes + t) * dv.n_kv_heads * G + (size_t)g * G + j) * D + c * 4) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      } else {
        const size_t rec = (size_t)it.rec * R + r;
        *(float4*)(dv.rec_o + rec * D + c * 4) = acc;
        // (a negative sum marks the row of an absent node for the combine kernel)
        if (c == 0) dv.rec_ml[rec] = make_float2(mx, it.draft && !live ? -1.f : lt);
      }
    }
    __syncthreads();   // (stages, queries, records of the warps are written again)
    head += 1;
    y = 0;
    if (todo > 0) st = states[head];
  }
}

template <int D>
cudaError_t rows_launch(const DeviceView& dv, int layer, const TreeCall& call, long long rec_rows, int n_sms, cudaStream_t s) {
  TreeCall tc = call;
  tree_cut<R>(dv, rec_rows, n_sms, tc);
  return tree_run<D, R>(tree_rows_kernel<D>, RowsSmem<D>::kBytes, dv, tc, s, dv, layer, tc);
}

}  // namespace

cudaError_t launch_tree_rows(const DeviceView& dv, int layer, const TreeCall& call, long long rec_rows, int n_sms, cudaStream_t s) {
  return dv.head_dim == 128 ? rows_launch<128>(dv, layer, call, rec_rows, n_sms, s) : rows_launch<64>(dv, layer, call, rec_rows, n_sms, s);
}

}  // namespace razor
