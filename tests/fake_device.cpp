// The CUDA runtime and the kernel launchers as the host code of the library sees them, for tests without a GPU: nothing runs,
// and what would have been launched or copied is counted.  Compiled together with razor_api.cu and razor_schedule.cpp.
#include <cstdlib>
#include <cstring>
#include <map>

#include "razor_internal.h"
#include "razor_spec.h"

namespace {
std::map<void*, unsigned long long> capturing;   // stream -> the capture it is part of
struct Seen {
  int append_early = -1;        // of the last append: may it read ahead of its wait?
  int decode_stable = -1;       // of the last decode launch: may it load head states ahead?
  int decode_early = -1;        // and how many pages, all CTAs together
  int uploads = 0;              // copies to the device on streams that run
  int captured_uploads = 0;     // and on capturing ones
  int launches = 0;             // kernels
  int records = 0, captured_records = 0;   // of events
} seen;
int launched() {
  seen.launches += 1;
  return 0;
}
}  // namespace

extern "C" {
#define FAKE __attribute__((visibility("default")))
FAKE void fake_reset() {
  capturing.clear();
  seen = Seen();
}
FAKE void fake_capture(void* stream, unsigned long long id) {   // 0: no longer
  if (id) capturing[stream] = id;
  else capturing.erase(stream);
}
FAKE void fake_seen(int* out) { std::memcpy(out, &seen, sizeof(seen)); }

cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
cudaError_t cudaHostAlloc(void** p, size_t n, unsigned) { *p = std::calloc(1, n); return cudaSuccess; }
cudaError_t cudaFreeHost(void* p) { std::free(p); return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void*, const void*, size_t, cudaMemcpyKind, cudaStream_t s) {
  (capturing.count(s) ? seen.captured_uploads : seen.uploads) += 1;
  return cudaSuccess;
}
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) { *e = (cudaEvent_t)std::malloc(1); return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t e) { std::free(e); return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t s) {
  (capturing.count(s) ? seen.captured_records : seen.records) += 1;
  return cudaSuccess;
}
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus* st) {
  *st = capturing.count(s) ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
cudaError_t cudaStreamGetCaptureInfo(cudaStream_t s, cudaStreamCaptureStatus* st, unsigned long long* id, cudaGraph_t*,
                                     const cudaGraphNode_t**, size_t*) {
  const auto it = capturing.find(s);
  *st = it == capturing.end() ? cudaStreamCaptureStatusNone : cudaStreamCaptureStatusActive;
  if (id && it != capturing.end()) *id = it->second;
  return cudaSuccess;
}
}  // extern "C"

namespace razor {
cudaError_t launch_compress(const DeviceView&, int, int, int, int, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_append(const DeviceView&, int, int, const void*, const void*, int early_reads, cudaStream_t) {
  seen.append_early = early_reads;
  return (cudaError_t)launched();
}
cudaError_t launch_append_many(const DeviceView&, int, int, const void*, const void*, int, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_decode(const DeviceView&, int, int, const DecodeJobs& jb, const void*, float*, int, const DecodeTuning&, cudaStream_t) {
  seen.decode_stable = jb.state_stable;
  seen.decode_early = 0;
  for (int i = 0; i < kEarlyCtas; ++i) seen.decode_early += jb.early[i];
  return (cudaError_t)launched();
}
cudaError_t launch_round(const DeviceView&, long long, int, const RoundJobs&, const void*, float*, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_wait_selftest(const DeviceView&, unsigned long long, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_export(const DeviceView&, int, int, int, int32_t*, void*, void*, float*, float*, float*, float*, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_tree_mma(const DeviceView&, long long, int, const TreeCall&, long long, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_tree_rows(const DeviceView&, int, const TreeCall&, long long, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_append_tree(const DeviceView&, int, int, const void*, const void*, int64_t, int64_t, const int32_t*, int, const int32_t*, int, cudaStream_t) { return (cudaError_t)launched(); }
cudaError_t launch_verify(const VerifyCall&, int, int, cudaStream_t) { return (cudaError_t)launched(); }
}  // namespace razor
