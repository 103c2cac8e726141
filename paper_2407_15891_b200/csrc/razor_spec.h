// Speculative decoding: what the host code and the kernels of a round of drafted tokens share (razor_tree*.cu,
// razor_verify.cu, append_tree_kernel in razor_cache_kernels.cu).
#ifndef RAZOR_SPEC_H_
#define RAZOR_SPEC_H_

#include "razor_internal.h"

namespace razor {

constexpr int kTreeMaxNodes = RAZOR_TREE_MAX_NODES;
constexpr int kTreeMaxSpans = 1024;
// A head that a span starts inside (listed under that span): its parts lie in the spans first_span, first_span + 1, ..;
// n_parts = 0: the span starts with a head.  turn: the span's number among those that start inside the head.
struct TreeUnit {
  int32_t head, first_span, n_parts, turn;
};
// One razor_decode_attention_tree call.  Strides in elements, between sequences (b) and between nodes (t).
struct TreeCall {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* parent;   // device [B, n_nodes]
  float* out;
  TreeUnit* units;         // [kTreeMaxSpans] in the workspace: heads that the launch has cut
  int64_t q_stride_b, q_stride_t, kv_stride_b, kv_stride_t;
  int32_t n_nodes;
  // set by the launchers: tiles of query rows, spans of the heads' steps laid end to end, steps a span has at least
  int32_t n_tiles, n_spans, min_span;
};
cudaError_t launch_tree_wide(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& call, long long rec_rows,
                             int n_sms, cudaStream_t stream);   // more than 64 query rows per KV head, no ALiBi
cudaError_t launch_tree_mma(const DeviceView& dv, long long pool_pages, int layer, const TreeCall& call, long long rec_rows,
                            int n_sms, cudaStream_t stream);
cudaError_t launch_tree_rows(const DeviceView& dv, int layer, const TreeCall& call, long long rec_rows, int n_sms,
                             cudaStream_t stream);   // fp32 caches
// Appends n_accept[b] (host, [B]) rows of k, v to every sequence, picked by path (device [B, n_nodes] or NULL).
cudaError_t launch_append_tree(const DeviceView& dv, int dtype, int layer, const void* k, const void* v, int64_t kv_stride_b,
                               int64_t kv_stride_t, const int32_t* path, int n_nodes, const int32_t* n_accept, int batch,
                               cudaStream_t stream);
struct VerifyCall {
  const void* target;
  const void* draft;       // NULL: the drafts were not drawn at random
  const int32_t* tokens;
  const int32_t* parent;
  const float* u_accept;
  const float* u_sample;
  int32_t* n_accepted;
  int32_t* path;
  int32_t* next_token;
  int64_t target_stride_b, target_stride_row, draft_stride_b, draft_stride_row;   // elements
  int32_t batch, n_nodes, vocab;
  int32_t seg_len;         // set by the launcher
};
cudaError_t launch_verify(const VerifyCall& call, int dtype, int n_sms, cudaStream_t stream);

}  // namespace razor
#endif
