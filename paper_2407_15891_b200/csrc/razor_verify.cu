// Verification of drafted tokens against the target's probabilities (the accept / reject walk of speculative
// decoding, for a tree of drafts).
//
// At a node with target row p and draft row q its children are tried in index order.  With W = p, S = 1, Z = 1, A = 0
// at the first child, child x is accepted when u q(x) S < W(x) Z - that is u < P(x) / Q(x) for the residual target
// P = W / S and the draft distribution Q = q / Z without the children rejected so far.  A rejected child moves both
// on: A += S / Z, Z -= q(x), and, because a maximum of maxima subtracting a growing multiple of q collapses into one,
//     W(y) = max(p(y) - A q(y), 0), zero at the rejected children;   S = sum_y W(y).
// Without draft probabilities (drafts that were looked up, not drawn) q is one at the child: W = p without the
// rejected children and S = 1 - their probabilities, no pass over the row needed.  Where the walk ends, the next token
// is the first y whose running sum of W exceeds r sum(W).
//
// What bounds it: for large batches one read of the last node's rows (64 chains of 7 over 128256 tokens, 66 MB in fp32: 27 us,
// 0.37 of the measured copy rate; what keeps the streaming loop below that has not been measured), for small ones a chain of
// dependent steps (16 trees of 63: up to a dozen rejections in one sequence, 38-53 us with the inputs).  So a
// sequence is a cluster of CTAs that share the row: each takes a contiguous run of segments, keeps the segment sums in
// shared memory, and the CTAs trade their warps' partial sums once a pass through distributed shared memory.  The walk
// itself runs in every CTA of the cluster on values fetched up front (one p and one q value per node), with the same
// arithmetic on the same operands, so all of them take the same decisions without talking.  The token is found by the
// CTA whose run the threshold falls into: it scans its segment sums and reads one segment again.  Everything is summed in
// 64 bits: a running sum in 32 would move the border between two tokens by more than a rare token's whole probability.
#include <cooperative_groups.h>
#include <math_constants.h>

#include <algorithm>

#include "razor_common.cuh"
#include "razor_spec.h"

namespace cg = cooperative_groups;

namespace razor {
namespace {

constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyCluster = 8;       // most CTAs that share a sequence (the portable cluster size)
constexpr int kMaxSegs = 1024;          // segments of a CTA's share of a row
constexpr int kUnroll = 8;              // neighbouring values of a row that a lane takes at a time
constexpr int kSegUnit = 32 * kUnroll;  // a segment is a multiple of this
constexpr int kKeepSegs = 4;            // segments of one unit each that a warp can keep in registers

__device__ __forceinline__ float raw_prob(const float* x) { return __ldg(x); }
__device__ __forceinline__ float raw_prob(const __nv_bfloat16* x) {
  return __uint_as_float((uint32_t)__ldg((const unsigned short*)x) << 16);
}
// What is not a positive finite number counts as zero.
__device__ __forceinline__ float clean(float x) { return x < CUDART_INF_F ? fmaxf(x, 0.f) : 0.f; }
__device__ __forceinline__ double prob(float x) { return (double)clean(x); }
// kUnroll values of a row from position i on (none at or beyond hi), cleaned; wide: 16-byte loads will do.
__device__ __forceinline__ void load_row(const float* row, int i, int hi, bool wide, float (&x)[kUnroll]) {
  if (wide && i + kUnroll <= hi) {
    const float4 a = __ldg((const float4*)(row + i)), b = __ldg((const float4*)(row + i) + 1);
    x[0] = clean(a.x); x[1] = clean(a.y); x[2] = clean(a.z); x[3] = clean(a.w);
    x[4] = clean(b.x); x[5] = clean(b.y); x[6] = clean(b.z); x[7] = clean(b.w);
  } else {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) x[k] = i + k < hi ? clean(raw_prob(row + i + k)) : 0.f;
  }
}
__device__ __forceinline__ void load_row(const __nv_bfloat16* row, int i, int hi, bool wide, float (&x)[kUnroll]) {
  if (wide && i + kUnroll <= hi) {
    Elem<__nv_bfloat16>::unpack(__ldg((const uint4*)(row + i)), x);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) x[k] = clean(x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) x[k] = i + k < hi ? clean(raw_prob(row + i + k)) : 0.f;
  }
}
// max(x, 0) by the sign bit: the library's maximum of two doubles runs at a quarter of an addition's rate.  (x is no NaN.)
__device__ __forceinline__ double at_least_0(double x) { return __double2hiint(x) < 0 ? 0.0 : x; }

constexpr int kParts = kVerifyCluster * kVerifyWarps;
static_assert(kParts == 128 && kUnroll == 8, "four sums to a lane; eight values to a tree of sums");

struct VerifySmem {
  double seg_sum[kMaxSegs];
  double part[2][kVerifyCluster][kVerifyWarps];   // every warp's sum of every CTA's share, written by its owner; passes take turns
  float p_child[kTreeMaxNodes], q_child[kTreeMaxNodes], u[kTreeMaxNodes];
  int32_t parent[kTreeMaxNodes], token[kTreeMaxNodes];
  int32_t gone[kTreeMaxNodes];      // rejected children of the current node
  int32_t path[kTreeMaxNodes];
  int32_t n_gone, row;              // row: the current node + 1
  int32_t draw;                     // 1: the walk has ended and the segment sums are those of its last W
  int32_t again;                    // 1: the pass is over the target's own row, rejected children among it
  double minus;                     // A
};

// W at position i of the current row.
template <typename T>
__device__ __forceinline__ double weight_at(const VerifySmem& sm, const T* p_row, const T* q_row, double a, int i) {
  double w = prob(raw_prob(p_row + i));
  if (q_row) w = at_least_0(fma(-a, prob(raw_prob(q_row + i)), w));
  for (int j = 0; j < sm.n_gone; ++j)
    if (sm.gone[j] == i) w = 0.0;
  return w;
}

// Sum of x over the lanes at or below this one.
__device__ __forceinline__ double running_sum(double x, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  return x;
}

// The CTAs' sums from their warps': lane r < kVerifyCluster gets CTA r's, and all lanes the whole (in the same order in
// every CTA of the cluster).
__device__ __forceinline__ double cta_part(const double (*part)[kVerifyWarps], int lane) {
  const double* p = &part[0][0] + lane * 4;   // a CTA's sixteen sums lie in four neighbouring lanes
  double x = (p[0] + p[1]) + (p[2] + p[3]);
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  x += __shfl_xor_sync(0xffffffffu, x, 2);
  return __shfl_sync(0xffffffffu, x, (lane & 7) * 4);
}
__device__ __forceinline__ double all_parts(const double (*part)[kVerifyWarps], int lane) {
  double x = cta_part(part, lane);
#pragma unroll
  for (int off = 1; off < kVerifyCluster; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}

// kKeep: a row's values stay in registers while its node is the current one, so that every rejected child after the
// first costs no memory access (needs rows of at most kVerifyCluster * kVerifyWarps * kKeepSegs units, 131072 values).
template <typename T, bool kKeep>
__global__ void __launch_bounds__(kVerifyThreads, kKeep ? 1 : 2) verify_kernel(VerifyCall vc) {
  __shared__ VerifySmem sm;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), n_ranks = (int)cluster.num_blocks();
  const int b = blockIdx.x / n_ranks;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_nodes = vc.n_nodes, V = vc.vocab;
  const T* target = (const T*)vc.target + (size_t)b * vc.target_stride_b;
  const T* draft = vc.draft ? (const T*)vc.draft + (size_t)b * vc.draft_stride_b : nullptr;

  // ---- the values the walk compares, all at once
  for (int t = tid; t < n_nodes; t += kVerifyThreads) {
    const int a = vc.parent[(size_t)b * n_nodes + t], x = vc.tokens[(size_t)b * n_nodes + t];
    const bool ok = a >= -1 && a < t && x >= 0 && x < V;   // otherwise it is nobody's child
    sm.parent[t] = ok ? a : -2;
    sm.token[t] = x;
    sm.u[t] = vc.u_accept[(size_t)b * n_nodes + t];
    sm.p_child[t] = ok ? raw_prob(target + (size_t)(a + 1) * vc.target_stride_row + x) : 0.f;
    sm.q_child[t] = ok && draft ? raw_prob(draft + (size_t)(a + 1) * vc.draft_stride_row + x) : 1.f;
  }
  for (int i = tid; i < 2 * kParts; i += kVerifyThreads) (&sm.part[0][0][0])[i] = 0.0;   // (a smaller cluster's missing CTAs add nothing)
  // this CTA's share of a row: n_segs segments of seg_len values from segment seg0 on
  const int seg_len = vc.seg_len, all_segs = (V + seg_len - 1) / seg_len;
  const int per = (all_segs + n_ranks - 1) / n_ranks;
  const int seg0 = min(all_segs, rank * per), n_segs = min(all_segs, seg0 + per) - seg0;
  cluster.sync();   // the values are there, and every CTA of the cluster runs (its shared memory may be written)

  // ---- walk and passes.  The walk's state lives in warp 0, the same in every lane and in every CTA.
  int cur = -1, last = -1, taken = 0, n_gone = 0;
  double minus = 0.0, left = 1.0, total = 1.0;
  bool fresh = false, whole = false;   // the segment sums belong to the current W; the residual was empty
  unsigned pass = 0;
  float p_kept[kKeep ? kKeepSegs : 1][kUnroll], q_kept[kKeep ? kKeepSegs : 1][kUnroll];
  int p_row_kept = -1, q_row_kept = -1;
  for (;; ++pass) {
    if (warp == 0) {
      bool draw = false;
      double sum = 0.0;   // of the last pass
      if (pass > 0) sum = all_parts(sm.part[(pass - 1) & 1], lane);
      if (fresh && draft && !whole) total = sum;
      for (;;) {
        int t = -1;       // the next child of `cur` behind `last`
        for (int base = 0; base < n_nodes && t < 0; base += 32) {
          const int i = base + lane;
          const unsigned hit = __ballot_sync(0xffffffffu, i < n_nodes && i > last && sm.parent[i] == cur);
          if (hit) t = base + __ffs(hit) - 1;
        }
        if (t < 0) {
          draw = fresh;
          if (fresh && !(sum > 0.0) && !whole) {   // nothing left (p nowhere above A q): the target's own row
            whole = true;
            draw = false;
            n_gone = 0;
            minus = 0.0;
          }
          fresh = true;   // (after the pass that follows)
          break;
        }
        last = t;
        const int x = sm.token[t];
        bool was = false;
        for (int i = lane; i < n_gone; i += 32) was |= sm.gone[i] == x;
        was = __any_sync(0xffffffffu, was);
        const double px = prob(sm.p_child[t]);
        const double qx = !draft ? 1.0 : was ? 0.0 : prob(sm.q_child[t]);
        const double w = was ? 0.0 : draft ? fmax(px - minus * qx, 0.0) : px;
        if ((double)sm.u[t] * qx * total < w * left) {   // accepted: its children are next
          if (lane == 0) sm.path[taken] = t;
          taken += 1;
          cur = t;
          n_gone = 0;
          minus = 0.0;
          left = total = 1.0;
          fresh = false;
          continue;
        }
        if (!was) {
          if (lane == 0) sm.gone[n_gone] = x;
          n_gone += 1;
          __syncwarp();
        }
        if (draft) {
          minus += left > 0.0 ? total / left : 0.0;
          left -= qx;
          fresh = true;   // after the pass for its S
          break;
        }
        total = fmax(total - w, 0.0);
        fresh = false;
      }
      if (lane == 0) {
        sm.draw = draw;
        sm.again = whole;
        sm.row = cur + 1;
        sm.minus = minus;
        sm.n_gone = n_gone;
      }
    }
    __syncthreads();
    if (sm.draw) break;
    // ---- one pass over this CTA's share of the row: segment sums of W
    const double a = sm.minus;
    const int gone = sm.n_gone;
    if (kKeep && sm.again) p_row_kept = -1;   // (the kept row has lost its rejected children)
    const T* p_row = target + (size_t)sm.row * vc.target_stride_row;
    const T* q_row = a != 0.0 ? draft + (size_t)sm.row * vc.draft_stride_row : nullptr;
    double mine = 0.0;
    const bool wide = (((uintptr_t)p_row | (uintptr_t)q_row) & 15) == 0;
    // does a rejected child lie in [lo, hi)?
    auto any_gone = [&](int lo, int hi) -> bool {
      bool hit = false;
      for (int i = lane; i < gone; i += 32) hit |= sm.gone[i] >= lo && sm.gone[i] < hi;
      return __any_sync(0xffffffffu, hit);
    };
    // the sum of W over kUnroll values from position i on
    auto weigh = [&](float (&pv)[kUnroll], const float (&qv)[kUnroll], int i, bool has_gone) -> double {
      if (has_gone) {
#pragma unroll 1
        for (int j = 0; j < gone; ++j)
#pragma unroll
          for (int k = 0; k < kUnroll; ++k)
            if (sm.gone[j] == i + k) pv[k] = 0.f;
      }
      double s0 = 0.0, s1 = 0.0;
#pragma unroll
      for (int k = 0; k < kUnroll; k += 2) {
        const double x = (double)pv[k], y = (double)pv[k + 1];
        s0 += q_row ? at_least_0(fma(-a, (double)qv[k], x)) : x;
        s1 += q_row ? at_least_0(fma(-a, (double)qv[k + 1], y)) : y;
      }
      return s0 + s1;
    };
    if constexpr (kKeep) {   // (a segment is one unit here)
      const bool fresh_p = p_row_kept != sm.row, fresh_q = q_row && q_row_kept != sm.row;
#pragma unroll
      for (int k = 0; k < kKeepSegs; ++k) {
        const int i = (seg0 + warp + k * kVerifyWarps) * kSegUnit + lane * kUnroll, hi = warp + k * kVerifyWarps < n_segs ? V : 0;
        if (fresh_p) load_row(p_row, i, hi, wide, p_kept[k]);
        if (fresh_q) load_row(q_row, i, hi, wide, q_kept[k]);
      }
      if (fresh_p) p_row_kept = sm.row;
      if (fresh_q) q_row_kept = sm.row;
      double sum[kKeepSegs];
#pragma unroll
      for (int k = 0; k < kKeepSegs; ++k) {
        const int lo = (seg0 + warp + k * kVerifyWarps) * kSegUnit;
        sum[k] = weigh(p_kept[k], q_kept[k], lo + lane * kUnroll, any_gone(lo, lo + kSegUnit));
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < kKeepSegs; ++k) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], off);
#pragma unroll
      for (int k = 0; k < kKeepSegs; ++k) {
        if (lane == 0 && warp + k * kVerifyWarps < n_segs) sm.seg_sum[warp + k * kVerifyWarps] = sum[k];
        mine += sum[k];
      }
    } else {
      for (int s = warp; s < n_segs; s += kVerifyWarps) {
        const int lo = (seg0 + s) * seg_len, hi = min(V, lo + seg_len);
        const bool has_gone = any_gone(lo, hi);
        double sum = 0.0;
#pragma unroll 1
        for (int i = lo + lane * kUnroll; i < hi; i += kSegUnit) {
          float pv[kUnroll], qv[kUnroll] = {};
          load_row(p_row, i, hi, wide, pv);
          if (q_row) load_row(q_row, i, hi, wide, qv);
          sum += weigh(pv, qv, i, has_gone);
        }
        __syncwarp();
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (lane == 0) sm.seg_sum[s] = sum;
        mine += sum;
      }
    }
    if (lane < n_ranks) *cluster.map_shared_rank(&sm.part[pass & 1][rank][warp], lane) = mine;   // to every CTA of the cluster
    cluster.sync();   // (no CTA writes the same half of part[] again before all have come through the next pass's)
  }

  // ---- results
  if (rank == 0 && warp == 0) {
    if (lane == 0) vc.n_accepted[b] = taken;
    for (int t = lane; t < n_nodes; t += 32) vc.path[(size_t)b * n_nodes + t] = t < taken ? sm.path[t] : -1;
  }
  // The draw: the token is in the share of the first CTA whose running sum exceeds the threshold.  (Sums taken in
  // another order may differ in the last bit, so the last one with any weight stands in where none does.)
  if (warp != 0) return;
  const double (*part)[kVerifyWarps] = sm.part[(pass - 1) & 1];   // (the walk draws after at least one pass)
  const double threshold = (double)vc.u_sample[b] * all_parts(part, lane);
  const double cta_sum = cta_part(part, lane), mine = lane < n_ranks ? cta_sum : 0.0;
  const double upto_cta = running_sum(mine, lane);
  const unsigned cta_over = __ballot_sync(0xffffffffu, lane < n_ranks && mine > 0.0 && upto_cta > threshold);
  const unsigned cta_with = __ballot_sync(0xffffffffu, lane < n_ranks && mine > 0.0);
  const int owner = cta_over ? __ffs(cta_over) - 1 : cta_with ? 31 - __clz(cta_with) : -1;
  double run, before = owner >= 0 ? __shfl_sync(0xffffffffu, upto_cta - mine, owner) : 0.0;
  if (owner < 0 && rank == 0 && lane == 0) vc.next_token[b] = -1;   // a target row without any weight
  if (rank != owner) return;
  // the segment, then the position in it: the first whose running sum exceeds the threshold, else the last with weight
  int seg = -1;
  run = before;
  for (int s0 = 0; s0 < n_segs; s0 += 32) {
    const double v = s0 + lane < n_segs ? sm.seg_sum[s0 + lane] : 0.0;
    const double upto = run + running_sum(v, lane);
    const unsigned over = __ballot_sync(0xffffffffu, v > 0.0 && upto > threshold), with = __ballot_sync(0xffffffffu, v > 0.0);
    const int pick = over ? __ffs(over) - 1 : with ? 31 - __clz(with) : -1;
    if (pick >= 0) {
      seg = s0 + pick;
      before = __shfl_sync(0xffffffffu, upto - v, pick);
    }
    if (over) break;
    run = __shfl_sync(0xffffffffu, upto, 31);
  }
  const double a = sm.minus;
  const T* p_row = target + (size_t)sm.row * vc.target_stride_row;
  const T* q_row = a != 0.0 ? draft + (size_t)sm.row * vc.draft_stride_row : nullptr;
  const int lo = (seg0 + seg) * seg_len, hi = min(V, lo + seg_len);
  int token = -1;
  run = before;
  for (int i0 = lo; i0 < hi; i0 += kSegUnit) {   // kUnroll neighbours to a lane
    double w[kUnroll], mine = 0.0;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int i = i0 + lane * kUnroll + k;
      w[k] = i < hi ? weight_at(sm, p_row, q_row, a, i) : 0.0;
      mine += w[k];
    }
    const double upto = run + running_sum(mine, lane);
    const unsigned over = __ballot_sync(0xffffffffu, mine > 0.0 && upto > threshold), with = __ballot_sync(0xffffffffu, mine > 0.0);
    if (over || with) {
      const int pick = over ? __ffs(over) - 1 : 31 - __clz(with);
      double r = upto - mine;
      int at = -1;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (w[k] > 0.0 && (at < 0 || !(over && r > threshold))) at = k;   // the first whose sum is beyond the threshold, or the last
        r += w[k];
      }
      token = i0 + pick * kUnroll + __shfl_sync(0xffffffffu, at, pick);
    }
    if (over) break;
    run = __shfl_sync(0xffffffffu, upto, 31);
  }
  if (lane == 0) vc.next_token[b] = token;
}

}  // namespace

cudaError_t launch_verify(const VerifyCall& call, int dtype, int n_sms, cudaStream_t stream) {
  VerifyCall vc = call;
  // CTAs to a sequence: as many as are resident at once (two to an SM), so that a large batch does not run in a wave and a
  // bit (64 sequences over 128256 tokens, one pass each: 8 to a sequence 33.6 us, 4 27 us).
  int ranks = kVerifyCluster;
  while (ranks > 1 && (long long)vc.batch * ranks > 2LL * n_sms) ranks /= 2;
  // segments: at most kMaxSegs to a CTA
  const long long units = ((long long)vc.vocab + kSegUnit - 1) / kSegUnit;
  vc.seg_len = (int)(kSegUnit * ((units + (long long)ranks * kMaxSegs - 1) / ((long long)ranks * kMaxSegs)));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)vc.batch * ranks);
  cfg.blockDim = dim3(kVerifyThreads);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ranks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  // Rows in registers: when the clusters have an SM to each CTA anyway (the registers of a CTA fill most of an SM; with
  // more sequences the SMs are kept busy by CTAs waiting side by side).
  const bool keep = vc.seg_len == kSegUnit && units <= (long long)kVerifyCluster * kVerifyWarps * kKeepSegs &&
                    (long long)vc.batch * kVerifyCluster <= n_sms;
  if (dtype == RAZOR_BF16)
    return keep ? cudaLaunchKernelEx(&cfg, verify_kernel<__nv_bfloat16, true>, vc) : cudaLaunchKernelEx(&cfg, verify_kernel<__nv_bfloat16, false>, vc);
  return keep ? cudaLaunchKernelEx(&cfg, verify_kernel<float, true>, vc) : cudaLaunchKernelEx(&cfg, verify_kernel<float, false>, vc);
}

}  // namespace razor
