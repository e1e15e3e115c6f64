// C ABI of the sampler (include/as2d.h): verification of drafted tokens by
// sampling, on device tensors, with the kernels of sample.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <string>

#include "internal.h"
#include "kernels.h"

using namespace as2d;

struct as2d_sampler {
  int max_requests = 0, max_k = 0, max_vocab = 0, dev = 0;
  void* work = nullptr;
  hipEvent_t ev = nullptr;
  hipStream_t last = nullptr;   // stream of the last call
  bool used = false;
  std::string err;
};

namespace {

thread_local std::string t_create_err;

int fail(as2d_sampler* s, int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  (s ? s->err : t_create_err) = buf;
  return code;
}

int hip_fail(as2d_sampler* s, const char* what, hipError_t e) {
  (void)hipGetLastError();   // reported here: the next launch must not report it
  return fail(s, e == hipErrorOutOfMemory ? AS2D_ENOMEM : AS2D_EHIP, "sampler: %s: %s", what, hipGetErrorString(e));
}

// The workspace is the last call's until it has run: stream st waits for it.
hipError_t after_last(as2d_sampler* s, hipStream_t st) {
  if (being_captured(s->last)) return hipErrorStreamCaptureUnsupported;
  hipError_t e = hipEventRecord(s->ev, s->last);
  e = e == hipSuccess ? hipStreamWaitEvent(st, s->ev, 0) : hipDeviceSynchronize();   // the stream may be gone
  if (e == hipSuccess) (void)hipGetLastError();   // of the queries
  return e;
}

}  // namespace

extern "C" {

const char* as2d_sampler_last_error(const as2d_sampler* s) {
  return s ? s->err.c_str() : t_create_err.empty() ? "null sampler" : t_create_err.c_str();
}

int as2d_sampler_create(int32_t max_requests, int32_t max_k, int32_t max_vocab, as2d_sampler** out) {
  if (!out) return AS2D_EINVAL;
  *out = nullptr;
  t_create_err.clear();
  if (max_requests < 1 || max_requests > 4096 || max_k < 0 || max_k > 31 || max_vocab < 1 || max_vocab > 1 << 24)
    return fail(nullptr, AS2D_EINVAL, "sampler: 1 <= max_requests <= 4096, 0 <= max_k <= 31, 1 <= max_vocab <= 2^24");
  auto* s = new (std::nothrow) as2d_sampler();
  if (!s) return fail(nullptr, AS2D_ENOMEM, "sampler: host memory");
  s->max_requests = max_requests;
  s->max_k = max_k;
  s->max_vocab = max_vocab;
  SampleArgs a{};
  a.n = max_requests;
  a.k = max_k;
  a.chunks = (max_vocab + kSampleChunk - 1) / kSampleChunk;
  a.max_children = max_k;
  hipError_t e = hipGetDevice(&s->dev);
  if (e == hipSuccess) e = hipMalloc(&s->work, sample_layout(a, max_requests, nullptr));
  if (e == hipSuccess) e = hipMemset(s->work, 0, sizeof(int) * max_requests);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipEventCreateWithFlags(&s->ev, hipEventDisableTiming);
  if (e != hipSuccess) {
    const int rc = hip_fail(nullptr, "create", e);
    (void)hipGetLastError();
    as2d_sampler_free(s);
    return rc;
  }
  *out = s;
  return AS2D_OK;
}

int as2d_sampler_free(as2d_sampler* s) {
  if (!s) return AS2D_EINVAL;
  OnDevice on(s->dev);
  if (s->work) hipFree(s->work);   // waits for the device
  if (s->ev) hipEventDestroy(s->ev);
  delete s;
  return AS2D_OK;
}

int as2d_sampler_verify(as2d_sampler* s, const as2d_sample_args* p, void* hip_stream) {
  if (!s) return AS2D_EINVAL;
  if (!p) return fail(s, AS2D_EINVAL, "sampler: null arguments");
  const int n = p->n, k = p->k, vocab = p->vocab;
  if (n < 0 || n > s->max_requests || k < 0 || k > s->max_k || vocab < 1 || vocab > s->max_vocab)
    return fail(s, AS2D_EINVAL, "sampler: %d requests of %d candidates over %d tokens, made for %d, %d and %d", n, k, vocab,
                s->max_requests, s->max_k, s->max_vocab);
  if (n == 0) return AS2D_OK;
  if (p->dtype != AS2D_F32 && p->dtype != AS2D_BF16) return fail(s, AS2D_EINVAL, "sampler: type %d", p->dtype);
  if (!p->logits || !p->uniforms || !p->accepted || !p->token || (k && (!p->cands || !p->path)))
    return fail(s, AS2D_EINVAL, "sampler: null tensor");
  if (p->row_stride < vocab || (p->draft_logits && p->draft_row_stride < vocab))
    return fail(s, AS2D_EINVAL, "sampler: rows overlap (stride below %d)", vocab);
  const auto good = [](double t) { return t >= kLeastTemp && t <= kMostTemp; };
  if ((!p->temperatures && !good(p->temperature)) || (p->draft_temperature != 0.0 && !good(p->draft_temperature)))
    return fail(s, AS2D_EINVAL, "sampler: temperature %g, of the drafter %g (1e-30 to 1e30)", p->temperature, p->draft_temperature);
  SampleArgs a{};
  int children[32] = {};
  for (int i = 1; i <= k; ++i) {
    const int up = p->parents ? p->parents[i - 1] : i - 2;
    if (up < -1 || up >= i - 1)
      return fail(s, AS2D_EINVAL, "sampler: candidate %d follows %d (a parent comes before its children, -1 is the root)", i - 1, up);
    a.parent[i] = (signed char)(up + 1);
    ++children[up + 1];
  }
  a.max_children = *std::max_element(children, children + 32);
  a.target = p->logits;
  a.draft = k ? p->draft_logits : nullptr;
  a.t_stride = p->row_stride;
  a.d_stride = p->draft_row_stride;
  a.n = n;
  a.k = k;
  a.vocab = vocab;
  a.chunks = (vocab + kSampleChunk - 1) / kSampleChunk;
  a.bf16 = p->dtype == AS2D_BF16;
  a.cands = p->cands;
  a.ks = p->ks;
  a.uniforms = p->uniforms;
  a.temps = p->temperatures;
  a.temp = p->temperature;
  a.draft_temp = p->draft_temperature;
  a.accepted = p->accepted;
  a.path = p->path;
  a.token = p->token;
  a.logp = p->logp;
  sample_layout(a, s->max_requests, (char*)s->work);

  OnDevice on(s->dev);
  hipStream_t st = (hipStream_t)hip_stream;
  hipDevice_t d = s->dev;
  hipError_t e = st ? hipStreamGetDevice(st, &d) : hipSuccess;
  if (e != hipSuccess) return hip_fail(s, "stream", e);
  if (d != s->dev) return fail(s, AS2D_EINVAL, "sampler: the stream belongs to device %d, the sampler to %d", d, s->dev);
  if (stream_restricted(st)) return fail(s, AS2D_EINVAL, "sampler: %s", kRestrictedStream);
  hipStreamCaptureStatus now = hipStreamCaptureStatusNone;
  if ((e = hipStreamIsCapturing(st, &now)) != hipSuccess) return hip_fail(s, "stream", e);
  if (now == hipStreamCaptureStatusNone) {   // a captured call runs nothing now: it is ordered by who replays the graph
    if (s->used && s->last != st && (e = after_last(s, st)) != hipSuccess)
      return e == hipErrorStreamCaptureUnsupported
                 ? fail(s, AS2D_ESTATE, "sampler: the last call's stream is being captured: that call cannot be waited for")
                 : hip_fail(s, "stream order", e);
    s->used = true;
    s->last = st;
  }
  e = launch_sample(a, a.draft != nullptr, st);
  return e == hipSuccess ? AS2D_OK : hip_fail(s, "launch", e);
}

}  // extern "C"
