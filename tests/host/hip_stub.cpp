// A HIP runtime and kernel launchers that run nothing: the library's host code
// (as2d.cpp, sampler.cpp, ..) linked against it shows, without a GPU, in which
// order it launches, waits and allocates, and what it does when a call fails.
//
// Device memory is host memory.  Every call that matters for order is a line
// of the log: "launch NAME STREAM", "copy STREAM", "record EVENT STREAM",
// "wait STREAM EVENT", "sync STREAM", "sync device", "malloc", "malloc failed".
// Streams are numbers (0: the default one), given by the test or made here.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

#include "../../paper_2609_37617_amd/csrc/kernels.h"

namespace {

struct Stream {
  bool capturing = false, masked = false;
  int device = 0;
};
std::string g_log, g_fail_launch;
std::map<size_t, Stream> g_streams;
size_t g_next_stream = 1000, g_next_event = 1;
long long g_malloc_limit = -1;   // larger allocations fail; -1: none does
int g_device = 0;
hipError_t g_error = hipSuccess;   // what hipGetLastError returns next

size_t num(const void* p) { return reinterpret_cast<size_t>(p); }
template <class... A> void note(const char* fmt, A... a) {
  char line[128];
  snprintf(line, sizeof line, fmt, a...);
  g_log += line;
  g_log += '\n';
}
hipError_t error(hipError_t e) {
  if (e != hipSuccess) g_error = e;
  return e;
}
// What a launcher does: the runtime's pending error is its result, as hipGetLastError gives it after a launch.
hipError_t launch(const char* name, hipStream_t s) {
  const bool fails = g_fail_launch == name;
  note("launch %s %zu%s", name, num(s), fails ? " failed" : "");
  if (fails) error(hipErrorLaunchFailure);
  return hipGetLastError();
}

}  // namespace

extern "C" {

// ---- the test's side ----------------------------------------------------------
const char* stub_log() { return g_log.c_str(); }
void stub_reset() {
  g_log.clear();
  g_fail_launch.clear();
  g_streams.clear();
  g_malloc_limit = -1;
  g_next_stream = 1000;
  g_device = 0;
  g_error = hipSuccess;
}
void stub_clear_log() { g_log.clear(); }
void stub_malloc_limit(long long bytes) { g_malloc_limit = bytes; }
void stub_fail_launch(const char* name) { g_fail_launch = name; }
void stub_stream(size_t s, int capturing, int masked, int device) { g_streams[s] = Stream{capturing != 0, masked != 0, device}; }
int stub_device() { return g_device; }
int stub_pending_error() { return g_error; }

// ---- the runtime ----------------------------------------------------------------
hipError_t hipGetLastError() {
  const hipError_t e = g_error;
  g_error = hipSuccess;
  return e;
}
const char* hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipGetDevice(int* d) { return *d = g_device, hipSuccess; }
hipError_t hipSetDevice(int d) { return g_device = d, hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipDeviceSynchronize() { return note("sync device"), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) {
  if (g_malloc_limit >= 0 && (long long)n > g_malloc_limit) return note("malloc failed"), *p = nullptr, error(hipErrorOutOfMemory);
  note("malloc");
  return *p = malloc(n ? n : 1), hipSuccess;
}
hipError_t hipFree(void* p) { return free(p), hipSuccess; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return *p = calloc(1, n ? n : 1), hipSuccess; }
hipError_t hipHostFree(void* p) { return free(p), hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { return memmove(d, s, n), hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t st) {
  note("copy %zu", num(st));
  return memmove(d, s, n), hipSuccess;
}
hipError_t hipMemset(void* d, int v, size_t n) { return memset(d, v, n), hipSuccess; }
hipError_t hipMemsetAsync(void* d, int v, size_t n, hipStream_t) { return memset(d, v, n), hipSuccess; }
hipError_t hipStreamCreateWithFlags(hipStream_t* s, unsigned) { return *s = reinterpret_cast<hipStream_t>(g_next_stream++), hipSuccess; }
hipError_t hipStreamDestroy(hipStream_t) { return hipSuccess; }
hipError_t hipStreamGetDevice(hipStream_t s, hipDevice_t* d) { return *d = g_streams[num(s)].device, hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* st) {
  if (!s && g_streams[0].capturing) return error(hipErrorStreamCaptureImplicit);   // a stream it synchronises with is
  *st = g_streams[num(s)].capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipExtStreamGetCUMask(hipStream_t s, uint32_t words, uint32_t* mask) {
  for (uint32_t i = 0; i < words; ++i) mask[i] = g_streams[num(s)].masked && i ? 0 : 0xffffffffu;
  return hipSuccess;
}
// A capturing stream can be neither waited for by the host nor recorded for another stream.
hipError_t hipStreamSynchronize(hipStream_t s) {
  note("sync %zu%s", num(s), g_streams[num(s)].capturing ? " capturing" : "");
  return g_streams[num(s)].capturing ? error(hipErrorStreamCaptureUnsupported) : hipSuccess;
}
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = reinterpret_cast<hipEvent_t>(g_next_event++), hipSuccess; }
hipError_t hipEventCreate(hipEvent_t* e) { return hipEventCreateWithFlags(e, 0); }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  return note("record %zu %zu%s", num(e), num(s), g_streams[num(s)].capturing ? " capturing" : ""), hipSuccess;
}
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float* ms, hipEvent_t, hipEvent_t) { return *ms = 0.f, hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t e, unsigned) { return note("wait %zu %zu", num(s), num(e)), hipSuccess; }
hipError_t hipStreamBeginCapture(hipStream_t, hipStreamCaptureMode) { return error(hipErrorNotSupported); }
hipError_t hipStreamEndCapture(hipStream_t, hipGraph_t*) { return error(hipErrorNotSupported); }
hipError_t hipGraphDestroy(hipGraph_t) { return hipSuccess; }
hipError_t hipGraphExecDestroy(hipGraphExec_t) { return hipSuccess; }
hipError_t hipGraphInstantiate(hipGraphExec_t*, hipGraph_t, hipGraphNode_t*, char*, size_t) { return error(hipErrorNotSupported); }
hipError_t hipGraphLaunch(hipGraphExec_t, hipStream_t) { return error(hipErrorNotSupported); }

}  // extern "C"

// ---- the launchers ----------------------------------------------------------------
namespace as2d {

hipError_t prepare_kernels() { return hipSuccess; }
bool range_plan_ok(const GemmArgs&) { return true; }
int step_ra_slice(bool, int, int) { return 0; }
hipError_t step_occupancy(bool, int, int, int, int, int* n) { return *n = 0, hipSuccess; }   // no persistent step kernel
hipError_t static_scratch(void** p, size_t* n) {
  static char scratch[4 << 20];
  return *p = scratch, *n = sizeof scratch, hipSuccess;
}
hipError_t launch_pack(bool, const void*, uint4*, int, int, int, int, hipStream_t s) { return launch("pack", s); }
hipError_t launch_embed(bool, const RowDesc*, const PassDesc&, int, const void*, const void*, int, const float*, float*, float*,
                        void*, long long, hipStream_t s) {
  return launch("embed", s);
}
hipError_t launch_gemm(bool, int, int, const GemmArgs&, hipStream_t s) { return launch("gemm", s); }
hipError_t launch_step(bool, int, int, int, const StepArgs&, int, int, hipStream_t s) { return launch("step", s); }
hipError_t launch_attention(bool, const AttnArgs&, int, int, bool, hipStream_t s) { return launch("attention", s); }
hipError_t launch_tree_attention(bool, const AttnArgs&, const TreeOp&, int, hipStream_t s) { return launch("tree_attention", s); }
hipError_t launch_finish(const RowDesc*, const ReqDesc*, int, int, const float*, const float*, const int*, int, int*, int*, int*,
                         const HostOut&, hipStream_t s) {
  return launch("finish", s);
}
hipError_t launch_put_rows(bool, bool, const PutRows&, int, hipStream_t s) { return launch("put_rows", s); }
hipError_t launch_tree_walk(const RowDesc*, const ReqDesc*, int, const int*, const int*, const TreeOut&, hipStream_t s) {
  return launch("tree_walk", s);
}
hipError_t launch_move_path(bool, const MovePath&, int, int, hipStream_t s) { return launch("move_path", s); }
hipError_t launch_sample(const SampleArgs&, bool, hipStream_t s) { return launch("sample", s); }
hipError_t launch_fill_zero(int* p, int n, hipStream_t s) {
  memset(p, 0, sizeof(int) * n);
  return launch("fill_zero", s);
}
hipError_t launch_stream_read(const uint4*, long long, int, unsigned*, hipStream_t s) { return launch("stream_read", s); }

}  // namespace as2d
