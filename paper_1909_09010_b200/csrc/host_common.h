// Host-side helpers shared by the translation units of libgbmuf (gbmuf.cu, local_ops.cu).
#ifndef GBMUF_CSRC_HOST_COMMON_H
#define GBMUF_CSRC_HOST_COMMON_H

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <string>
#include <vector>

#include "gbmuf.h"

// Sets what gbmuf_last_error(NULL) returns on this thread.
__attribute__((visibility("hidden"))) void gbmuf_set_thread_error(const std::string& text);

namespace {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { prev = -1; }
    if (prev != dev) ok = (cudaSetDevice(dev) == cudaSuccess);
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

// Is `st` recording a stream capture?  (The legacy default stream never is.)
inline bool is_capturing(cudaStream_t st) {
  if (!st) return false;
  cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(st, &cs) != cudaSuccess) { cudaGetLastError(); return false; }
  return cs != cudaStreamCaptureStatusNone;
}

// Which streams a handle has put work into, as one event per stream recorded after the latest
// piece of work.  Re-partitioning and destruction wait for these events: for the handle's own
// work and nothing else on the device.  Events outlive the streams they were recorded in, so a
// stream the caller has destroyed in the meantime is no problem.  Work recorded into a stream
// capture is not tracked (an event recorded there cannot be waited for from the host); the
// caller keeps the handle alive while such a graph can still run.
struct WorkMarks {
  struct Mark { cudaStream_t s; cudaEvent_t ev; };
  std::vector<Mark> marks;
  static constexpr size_t kMaxStreams = 16;
  // false: the work went into a stream capture
  bool note(cudaStream_t st) {
    if (is_capturing(st)) return false;
    for (Mark& mk : marks)
      if (mk.s == st) { cudaEventRecord(mk.ev, st); return true; }
    if (marks.size() == kMaxStreams) {               // many streams: retire the oldest mark
      cudaEventSynchronize(marks.front().ev);
      cudaEventDestroy(marks.front().ev);
      marks.erase(marks.begin());
    }
    Mark mk{st, nullptr};
    if (cudaEventCreateWithFlags(&mk.ev, cudaEventDisableTiming) != cudaSuccess) { cudaGetLastError(); return true; }
    cudaEventRecord(mk.ev, st);
    marks.push_back(mk);
    return true;
  }
  cudaError_t wait() {
    cudaError_t first = cudaSuccess;
    for (Mark& mk : marks) {
      const cudaError_t e = cudaEventSynchronize(mk.ev);
      if (e != cudaSuccess && first == cudaSuccess) first = e;
    }
    return first;
  }
  void release() {
    for (Mark& mk : marks) cudaEventDestroy(mk.ev);
    marks.clear();
  }
};

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up until it is found; NULL if the driver has none.
inline EncodeTiledFn encode_tiled_fn() {
  static std::atomic<EncodeTiledFn> found{nullptr};
  EncodeTiledFn fn = found.load(std::memory_order_relaxed);
  if (fn) return fn;
  void* f = nullptr;
  cudaDriverEntryPointQueryResult qres;
  const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &qres);
  if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !f) return nullptr;
  fn = reinterpret_cast<EncodeTiledFn>(f);
  found.store(fn, std::memory_order_relaxed);
  return fn;
}

}  // namespace

#endif  // GBMUF_CSRC_HOST_COMMON_H
