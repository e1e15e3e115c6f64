// Library-internal calls between the translation units of libas2d.so
// (not part of the C ABI in include/as2d.h; hidden from the export table).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/as2d.h"

// Capture, if not yet captured, the verification graphs of one-request
// passes of 1..max_rows rows under the context's current execution mode
// and keep_logits setting (nothing is launched).  A caller that is about
// to run two contexts from two host threads calls it for both first, so
// that no graph is captured while another thread captures.
__attribute__((visibility("hidden"))) int as2d_prepare_graphs(as2d_ctx* ctx, int32_t max_rows);

namespace as2d {

// Another device for the calling thread, the one before at the end of the scope.
struct OnDevice {
  int before = -1;
  explicit OnDevice(int dev) {
    int now = 0;
    if (hipGetDevice(&now) == hipSuccess && now != dev && hipSetDevice(dev) == hipSuccess) before = now;
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

// Whether a stream is being captured: what ran on it before can then not be
// waited for (an event recorded there would be a node of the caller's graph,
// and a host wait would end the capture with an error).  The null stream counts
// as captured while a stream that it synchronises with is.
inline bool being_captured(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing(s, &st);
  if (e == hipSuccess) return st != hipStreamCaptureStatusNone;
  (void)hipGetLastError();   // another error: the stream may be gone
  return e == hipErrorStreamCaptureImplicit;
}

// Whether a stream is confined to part of the current device by a CU mask
// (hipExtStreamCreateWithCUMask).  Such streams are refused: the first
// concurrent run on masked streams ended in a host segmentation fault whose
// cause has not been found, so the library never runs on one.  A stream
// whose mask cannot be read is taken as unrestricted.
constexpr const char* kRestrictedStream =
    "streams restricted by a CU mask are not supported (use as2d_set_cu_budget to share the device)";
inline bool stream_restricted(hipStream_t s) {
  int dev = 0, dev_cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&dev_cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || dev_cus < 1)
    return false;
  uint32_t mask[32] = {0};
  const uint32_t words = (uint32_t)((dev_cus + 31) / 32);
  if (words > 32) return false;
  if (hipExtStreamGetCUMask(s, words, mask) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  int n = 0;
  for (uint32_t i = 0; i < words; ++i) n += __builtin_popcount(mask[i]);
  return n > 0 && n < dev_cus;
}

}  // namespace as2d
