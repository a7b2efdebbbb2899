// dc_outside.h -- allocations and uploads of plans and handles, beside whatever streams do.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

#include "dc_device.h"

namespace dc {

// While one lives, this thread's allocations, frees and waits are no part of a stream capture that is under way here or in
// another thread: under the default mode each of them is refused, and the capture lost.
class OutsideCapture {
 public:
  OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode_); }
  ~OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode_); }
  OutsideCapture(const OutsideCapture&) = delete;
  OutsideCapture& operator=(const OutsideCapture&) = delete;

 private:
  cudaStreamCaptureMode mode_ = cudaStreamCaptureModeRelaxed;
};

// Copies to or from the device and waits until it is done, whatever stream the next call is on. (cudaMemcpy may return once
// pageable memory is staged, and orders the rest on the legacy stream only, which a non-blocking stream does not wait
// for; and it waits for all that the legacy stream is busy with. A stream of its own does neither. It is kept, one a
// device: making one took 18 us of a small plan's 39.)
inline cudaError_t copy_now(void* dst, const void* src, size_t bytes, cudaMemcpyKind kind) {
  static std::atomic<cudaStream_t> kept[kDevices];
  const int dev = device_slot();
  cudaStream_t s = dev >= 0 ? kept[dev].load(std::memory_order_acquire) : nullptr;
  bool drop = false;
  if (!s) {
    cudaError_t e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
    if (e != cudaSuccess) return e;
    cudaStream_t none = nullptr;
    drop = dev < 0 || !kept[dev].compare_exchange_strong(none, s);
  }
  const cudaError_t e = cudaMemcpyAsync(dst, src, bytes, kind, s), done = cudaStreamSynchronize(s);
  if (drop) cudaStreamDestroy(s);
  return e != cudaSuccess ? e : done;
}
inline cudaError_t upload_now(void* dst, const void* src, size_t bytes) { return copy_now(dst, src, bytes, cudaMemcpyHostToDevice); }

// Waits for a stream and fetches the status words that its kernels write. A capture that is under way goes on: of another
// stream in any case, of this one because it is not waited for (*captures; a captured kernel has not run).
inline cudaError_t fetch_status(cudaStream_t s, const unsigned* status, unsigned (&words)[16], bool* captures) {
  cudaStreamCaptureStatus how = cudaStreamCaptureStatusNone;
  const cudaError_t is = cudaStreamIsCapturing(s, &how);
  if (is != cudaSuccess) cudaGetLastError();
  // (the legacy stream would wait for a blocking stream that captures)
  *captures = how != cudaStreamCaptureStatusNone || is == cudaErrorStreamCaptureImplicit;
  if (*captures) return cudaSuccess;
  const OutsideCapture outside;
  const cudaError_t e = cudaStreamSynchronize(s);
  return e != cudaSuccess ? e : copy_now(words, status, sizeof words, cudaMemcpyDeviceToHost);
}

}  // namespace dc
