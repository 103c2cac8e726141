// Attention of a tree of drafted tokens over an fp32 cache (the reference configurations; a bf16 cache runs on the
// tensor-core kernels).
//
// A node attends to every kept token of its head, to the compensation token with its count (Eq. 5), and to itself and
// its ancestors in the tree; the drafts' K and V are read from the caller's buffers and the cache stays as it is.
// Query rows of a KV head: r = t * group + j for node t and query head j of the group.
//
// The tensor cores have no fp32 product, so this runs on the CUDA cores: groups of lanes that cover a row of 16 bytes a
// lane take the tokens of a part in turn, each keeping the online softmax of eight query rows in registers (a K row is
// then used eight times); parts leave partial records that a combine kernel folds.  What bounds it is the shuffles of the
// dot products: about a hundred instructions a token and eight rows.
#include <math_constants.h>

#include <algorithm>

#include "razor_common.cuh"
#include "razor_tree.cuh"

namespace razor {
namespace {

constexpr int kRowsThreads = 256;
constexpr int kRowsTile = 8;    // query rows of a CTA

template <int D>
__global__ void __launch_bounds__(kRowsThreads) tree_rows_kernel(DeviceView dv, int layer, TreeCall tc) {
  using T = float;
  using Geo = RowGeom<T, D>;
  constexpr int LPR = Geo::kLpr, EPL = Geo::kEpl, NGRP = kRowsThreads / LPR;
  __shared__ TreeMask mask;
  __shared__ float g_o[NGRP][D];
  __shared__ float2 g_ml[NGRP];
  const int head = blockIdx.x, tile = blockIdx.y, split = blockIdx.z;
  const size_t hs = (size_t)layer * dv.n_heads + head;
  const HeadState st = dv.state[hs];
  const int b = head / dv.n_kv_heads, g = head % dv.n_kv_heads, G = dv.group, n_nodes = tc.n_nodes;
  const int rows = n_nodes * G, row0 = tile * kRowsTile;
  const int lir = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const int total = st.len + st.n_drop;
  tree_mask_load(mask, tc.parent + (size_t)b * n_nodes, n_nodes, threadIdx.x, kRowsThreads);
  __syncthreads();
  tree_mask_walk(mask, n_nodes, threadIdx.x, kRowsThreads);
  __syncthreads();

  float qf[kRowsTile][EPL], o[kRowsTile][EPL], m[kRowsTile], l[kRowsTile], slope[kRowsTile];
  int node[kRowsTile];
#pragma unroll
  for (int i = 0; i < kRowsTile; ++i) {
    const int r = row0 + i, t = min(r, rows - 1) / G, j = min(r, rows - 1) % G;
    node[i] = t;
    const T* src = (const T*)tc.q + (size_t)b * tc.q_stride_b + (size_t)t * tc.q_stride_t + ((size_t)g * G + j) * D;
    Elem<T>::unpack(__ldg((const uint4*)src + lir), qf[i]);
    slope[i] = dv.alibi ? dv.alibi_slopes[(size_t)layer * dv.n_kv_heads * G + (size_t)g * G + j] : 0.f;
    m[i] = -CUDART_INF_F;
    l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[i][e] = 0.f;
  }
  // one token against the eight rows; `pos` is its position, `see` the rows that may attend to it
  auto take = [&](const float (&kf)[EPL], const float (&vf)[EPL], int pos, unsigned see) {
#pragma unroll
    for (int i = 0; i < kRowsTile; ++i) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) s = fmaf(qf[i][e], kf[e], s);
      s = row_sum<LPR>(s);
      if (!(see >> i & 1)) continue;
      s *= dv.scale_log2;
      if (dv.alibi) s -= slope[i] * (float)(total + mask.depth[node[i]] - pos);
      const float mn = fmaxf(m[i], s), mu = mn == -CUDART_INF_F ? 0.f : mn;
      const float c = fast_exp2(m[i] - mu), w = fast_exp2(s - mu);
      m[i] = mn;
      l[i] = l[i] * c + w;
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[i][e] = fmaf(w, vf[e], o[i][e] * c);
    }
  };

  const int lo = (int)((long long)st.len * split / tc.n_splits), hi = (int)((long long)st.len * (split + 1) / tc.n_splits);
  const int32_t* pt = dv.page_table + hs * dv.max_pages;
  // (all groups of a warp run the same number of turns: row_sum is warp-wide)
  for (int base = lo; base < hi; base += NGRP) {
    const int s = base + grp, at = min(s, hi - 1);
    const uint4* src = (const uint4*)(dv.pool + (size_t)pt[at >> 4] * dv.page_bytes + (size_t)(at & 15) * Geo::kRowBytes) + swz(at, lir);
    float kf[EPL], vf[EPL];
    Elem<T>::unpack(ld_stream(src), kf);
    Elem<T>::unpack(ld_stream(src + kPageTokens * LPR), vf);
    take(kf, vf, slot_position(at, dv.n_sink, st, total), s < hi ? 0xffu : 0u);
  }
  const bool drafts = split == tc.n_splits - 1;   // the last part takes the tree's own tokens
  if (drafts) {
    for (int base = 0; base < n_nodes; base += NGRP) {
      const int n = base + grp, at = min(n, n_nodes - 1);
      const size_t off = (size_t)b * tc.kv_stride_b + (size_t)at * tc.kv_stride_t + (size_t)g * D;
      float kf[EPL], vf[EPL];
      Elem<T>::unpack(__ldg((const uint4*)((const T*)tc.k + off) + lir), kf);
      Elem<T>::unpack(__ldg((const uint4*)((const T*)tc.v + off) + lir), vf);
      unsigned see = 0;
#pragma unroll
      for (int i = 0; i < kRowsTile; ++i) see |= (n < n_nodes && tree_sees(mask, node[i], at) ? 1u : 0u) << i;
      take(kf, vf, total + mask.depth[at], see);
    }
  }
  if (split == 0 && dv.use_comp && st.n_drop > 0 && st.window >= 0) {   // the compensation token, once
    float kf[EPL], vf[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      kf[e] = dv.comp_mean[hs * 2 * D + lir * EPL + e];
      vf[e] = dv.comp_mean[hs * 2 * D + D + lir * EPL + e];
    }
    const float count_log2 = log2f((float)st.n_drop);
#pragma unroll
    for (int i = 0; i < kRowsTile; ++i) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) s = fmaf(qf[i][e], kf[e], s);
      s = fmaf(row_sum<LPR>(s), dv.scale_log2, count_log2);
      if (grp != 0) continue;
      const float mn = fmaxf(m[i], s), mu = mn == -CUDART_INF_F ? 0.f : mn;
      const float c = fast_exp2(m[i] - mu), w = fast_exp2(s - mu);
      m[i] = mn;
      l[i] = l[i] * c + w;
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[i][e] = fmaf(w, vf[e], o[i][e] * c);
    }
  }
  // ---- the groups' states of each row, folded in order
#pragma unroll
  for (int i = 0; i < kRowsTile; ++i) {
    __syncthreads();
    if (lir == 0) g_ml[grp] = make_float2(m[i], l[i]);
#pragma unroll
    for (int e = 0; e < EPL; ++e) g_o[grp][lir * EPL + e] = o[i][e];
    __syncthreads();
    const int r = row0 + i, d = threadIdx.x;
    if (r < rows && d < D) {
      const int t = r / G, j = r % G;
      float mx = -CUDART_INF_F, lt = 0.f, x = 0.f;
      for (int k = 0; k < NGRP; ++k) mx = fmaxf(mx, g_ml[k].x);
      const float mu = mx == -CUDART_INF_F ? 0.f : mx;
      for (int k = 0; k < NGRP; ++k) {
        const float c = fast_exp2(g_ml[k].x - mu);
        lt = fmaf(g_ml[k].y, c, lt);
        x = fmaf(g_o[k][d], c, x);
      }
      const bool live = tree_sees(mask, t, t);
      if (tc.n_splits == 1) {
        if (live) tc.out[(((size_t)b * n_nodes + t) * dv.n_kv_heads * G + (size_t)g * G + j) * D + d] = x / lt;
      } else {
        const size_t rec = ((size_t)head * tc.n_splits + split) * tc.rec_rows + r;
        dv.rec_o[rec * D + d] = x;
        // (a negative sum marks the row of an absent node for the combine kernel)
        if (d == 0) dv.rec_ml[rec] = make_float2(mx, drafts && !live ? -1.f : lt);
      }
    }
  }
}

// Folds the records of the parts, in order: a warp per query row.
template <int D>
__global__ void __launch_bounds__(128) tree_rows_combine_kernel(DeviceView dv, TreeCall tc) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, head = blockIdx.x, G = dv.group;
  const int r = blockIdx.y * 4 + warp;
  if (r >= tc.n_nodes * G) return;
  const size_t rec0 = (size_t)head * tc.n_splits * tc.rec_rows + r;
  if (dv.rec_ml[rec0 + (size_t)(tc.n_splits - 1) * tc.rec_rows].y < 0.f) return;
  float m = -CUDART_INF_F, l = 0.f;
  LaneVec<D> acc;
  acc.zero();
  for (int p = 0; p < tc.n_splits; ++p) {
    const size_t rec = rec0 + (size_t)p * tc.rec_rows;
    const float2 ml = dv.rec_ml[rec];
    LaneVec<D> x;
    x.load_l2(dv.rec_o + rec * D, lane);
    const float mn = fmaxf(m, ml.x), mu = mn == -CUDART_INF_F ? 0.f : mn;
    const float c_old = fast_exp2(m - mu), c_new = fast_exp2(ml.x - mu);
    l = l * c_old + ml.y * c_new;
    acc.scale(c_old);
    acc.fma(c_new, x);
    m = mn;
  }
  acc.scale(1.f / l);
  const int b = head / dv.n_kv_heads, g = head % dv.n_kv_heads, t = r / G, j = r % G;
  acc.store(tc.out + (((size_t)b * tc.n_nodes + t) * dv.n_kv_heads * G + (size_t)g * G + j) * D, lane);
}

template <int D>
cudaError_t rows_launch(const DeviceView& dv, int layer, const TreeCall& tc, cudaStream_t s) {
  const int rows = tc.n_nodes * dv.group;
  tree_rows_kernel<D><<<dim3(dv.n_heads, (rows + kRowsTile - 1) / kRowsTile, tc.n_splits), kRowsThreads, 0, s>>>(dv, layer, tc);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || tc.n_splits == 1) return e;
  tree_rows_combine_kernel<D><<<dim3(dv.n_heads, (rows + 3) / 4), 128, 0, s>>>(dv, tc);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_tree_rows(const DeviceView& dv, int layer, const TreeCall& call, int longest, long long rec_rows,
                        int n_sms, cudaStream_t s) {
  TreeCall tc = call;
  // Parts: about four CTAs per SM in all, at least 256 tokens to a part, no more than the records have rows for.
  const long long rows = (long long)tc.n_nodes * dv.group, tiles = (rows + kRowsTile - 1) / kRowsTile;
  const long long want = (4LL * n_sms + dv.n_heads * tiles - 1) / (dv.n_heads * tiles);
  const long long room = rec_rows / (dv.n_heads * rows);
  tc.n_splits = (int)std::max(1LL, std::min({want, (longest + 255LL) / 256, room, 65535LL}));
  tc.rec_rows = (int)rows;
  return dv.head_dim == 128 ? rows_launch<128>(dv, layer, tc, s) : rows_launch<64>(dv, layer, tc, s);
}

}  // namespace razor
