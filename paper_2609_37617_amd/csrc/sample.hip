// Verification of drafted tokens by sampling: the candidates of a tree tested
// against the target's probabilities with given random numbers, and the
// token that follows the accepted path.
//
// p = softmax(l / T) of a row of target logits, q = softmax(l' / T') of the
// drafter's row that the row's children were drawn from.  At a node with
// distribution R (at first p, mass S = 1) its children are tried in order:
// child x with random number u is accepted where u S q(x) < R(x), and the
// walk goes on at the child; else R <- max(R - S q, 0), S <- sum of R.  Without
// a drafter's row the child is certain, q(x) = 1 and 0 elsewhere: R(x) <- 0.
// After the last child the token is the first j with R_0 + .. + R_j > u S.  The
// token then has the target's distribution whatever the candidates are.
//
// Two rejections subtract a q, then b q; max(max(p - a q, 0) - b q, 0) =
// max(p - (a + b) q, 0), so a node's state is the single number C (the sum of
// the masses so far) and a mass is one pass over two rows:
//   R = max(p - C q, 0),  C_1 = 1, C_{m+1} = C_m + S(C_m).
// Masses after one rejection depend on no random number, so they are
// computed for every node with a second child at once, and so on: as many
// passes as the most children of a node, less one, and none for a chain.
//
// Rounding.  Exponentials are float32 (2^x by the hardware, about 1 unit in
// the last place, with the argument's rounding put back: x is formed in 64
// bits, 2^x = 2^float(x) (1 + (x - float(x)) ln 2)); everything summed,
// compared or logged is 64 bits, so that a random number next to a border
// falls on the same side as in exact arithmetic.
#include "common.h"

namespace as2d {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = kSampleChunk / kThreads;   // logits of a thread
constexpr double kLog2E = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

// ---- requests ---------------------------------------------------------------

struct Req {
  int r, row0, drow0, k;   // request, its first rows, candidates
  double c, dc;            // log2(e) / temperature
  bool ok;
};

__device__ __forceinline__ Req load_req(const SampleArgs& a, int r) {
  Req q;
  q.r = r;
  double t, dt;
  if (a.reqs) {
    const SampleReq s = load_invariant(a.reqs + r);
    q.row0 = s.row0;
    q.drow0 = s.draft_row0;
    q.k = s.k;
    t = s.temp;
    dt = s.draft_temp;
  } else {
    q.row0 = r * (a.k + 1);
    q.drow0 = a.draft ? q.row0 : -1;
    q.k = a.ks ? a.ks[r] : a.k;
    t = a.temps ? (double)a.temps[r] : a.temp;
    dt = a.draft_temp > 0.0 ? a.draft_temp : t;
  }
  q.ok = q.k >= 0 && q.k <= a.k && t > 0.0 && t < INFINITY;
  if (!q.ok) q.k = 0;
  q.c = kLog2E / t;
  q.dc = kLog2E / dt;
  return q;
}

// Row that row i (1 .. k) follows.
__device__ __forceinline__ int parent_of(const SampleArgs& a, const Req& q, int i) {
  return a.reqs ? parent_row(a.rows[q.row0 + i].mask, i) : a.parent[i & 31];
}
__device__ __forceinline__ int cand_of(const SampleArgs& a, const Req& q, int i) {
  return a.reqs ? a.rows[q.row0 + i].token : a.cands[(size_t)q.r * a.k + i - 1];
}
// Random number of candidate row i, or with i = 0 of the token after the path.
__device__ __forceinline__ float uniform_of(const SampleArgs& a, const Req& q, int i) {
  return a.reqs ? a.rows[q.row0 + i].u : a.uniforms[(size_t)q.r * (a.k + 1) + (i ? i - 1 : a.k)];
}
// Children of row `row`; every lane of the wave gets the count.
__device__ __forceinline__ int children_of(const SampleArgs& a, const Req& q, int row) {
  const int lane = threadIdx.x & 63;
  const bool child = lane >= 1 && lane <= q.k && parent_of(a, q, lane) == row;
  return __popcll(__ballot(child));
}

// ---- rows of logits ---------------------------------------------------------

template <bool BF> __device__ __forceinline__ float logit(const void* base, long long i) {
  if constexpr (BF) return bf2f(ldg(static_cast<const uint16_t*>(base) + i));
  else return ldg(static_cast<const float*>(base) + i);
}

// A thread's kPer logits of a chunk: runs of 16 bytes, kThreads apart (rows may
// start at any element: the loads need no alignment past the element's).
// Element e is column chunk * kSampleChunk + column<BF>(e); columns past the row
// read -inf.
template <bool BF> __device__ __forceinline__ int column(int e) {
  constexpr int RUN = BF ? 8 : 4;
  return ((e / RUN) * kThreads + (int)threadIdx.x) * RUN + e % RUN;
}
template <bool BF> __device__ __forceinline__ void load_chunk(const void* base, long long row, int chunk, int vocab, float (&x)[kPer]) {
  constexpr int RUN = BF ? 8 : 4;
  const int c0 = chunk * kSampleChunk;
  if (c0 + kSampleChunk <= vocab) {
#pragma unroll
    for (int g = 0; g < kPer / RUN; ++g) {
      const long long at = row + c0 + column<BF>(g * RUN);
      if constexpr (BF) {
        typedef uint16_t run __attribute__((ext_vector_type(8), aligned(2)));
        const run v = *gmem(reinterpret_cast<const run*>(static_cast<const uint16_t*>(base) + at));
#pragma unroll
        for (int t = 0; t < RUN; ++t) x[g * RUN + t] = bf2f(v[t]);
      } else {
        typedef float run __attribute__((ext_vector_type(4), aligned(4)));
        const run v = *gmem(reinterpret_cast<const run*>(static_cast<const float*>(base) + at));
#pragma unroll
        for (int t = 0; t < RUN; ++t) x[g * RUN + t] = v[t];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int col = c0 + column<BF>(e);
      x[e] = col < vocab ? logit<BF>(base, row + col) : -INFINITY;
    }
  }
}

// 2^((x - m) c) for x <= m.
__device__ __forceinline__ float power(float x, float m, double c) {
  const double y = ((double)x - (double)m) * c;
  const float f = (float)y;
  if (!(f > -160.f)) return 0.f;   // below float32's range; x = -inf
  return __builtin_amdgcn_exp2f(f) * __builtin_fmaf((float)(y - (double)f), (float)kLn2, 1.0f);
}

// What is left of a column: max(p - C q, 0) from the two powers and the factors
// 1 / sum and C / sum.  One rounding per operation wherever it is formed, so
// that a chunk's sum is positive exactly where one of its columns is.
__device__ __forceinline__ double left_of(float p, double ps, float q, double qs) {
#pragma clang fp contract(off)
  return fmax((double)p * ps - (double)q * qs, 0.0);
}

// ---- reductions: fixed trees, the same bits in every lane -------------------

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double block_sum64(double v, double* s) {
  v = wave_sum64(v);
  __syncthreads();   // s may be in use
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ float block_max(float v, float* s) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}

// ---- workspace places ----------------------------------------------------------

__device__ __forceinline__ SamplePart* part_of(const SampleArgs& a, int r, int which, int row) {
  return a.part + (((size_t)r * 2 + which) * (a.k + 1) + row) * a.chunks;
}
__device__ __forceinline__ double* stage_of(const SampleArgs& a, int s, int r, int row) {
  return a.stage + (((size_t)(s - 1) * a.n + r) * (a.k + 1) + row) * a.chunks;
}
__device__ __forceinline__ double* cut_of(const SampleArgs& a, int s, int r, int row) {
  return a.cut + ((size_t)(s - 1) * a.n + r) * (a.k + 1) + row;
}

// A row's maximum, log2 of its sum and whether it has a value that is no
// logit, from its chunks' parts; one wave, every lane gets them.
struct RowStat {
  float max;
  double log_sum;
  bool bad;
};
__device__ __forceinline__ RowStat row_stat(const SamplePart* part, int chunks, double c) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  int bad = 0;
  for (int i = lane; i < chunks; i += 64) {
    m = fmaxf(m, part[i].max);
    bad |= part[i].bad;
  }
  m = wave_max(m);
  double s = 0.0;
  for (int i = lane; i < chunks; i += 64)
    if (part[i].max > -INFINITY) s += part[i].sum * exp2(((double)part[i].max - (double)m) * c);
  s = wave_sum64(s);
  return RowStat{m, log2(s), __ballot(bad) != 0 || !(m > -INFINITY)};
}
__device__ __forceinline__ double prob(float x, float max, double c, double log_sum) {
  return x > -INFINITY ? exp2(((double)x - (double)max) * c - log_sum) : 0.0;
}

// ---- kernels ----------------------------------------------------------------

// Maximum and sum of every chunk of the target's rows and of the drafter's
// rows with children.  The one pass over the logits that cannot be avoided.
template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_stats_kernel(const SampleArgs a) {
  __shared__ float s_max[4];
  __shared__ double s_sum[4];
  const int chunk = blockIdx.x, row = blockIdx.y, which = (int)blockIdx.z >= a.n, r = blockIdx.z - which * a.n;
  const Req q = load_req(a, r);
  if (!q.ok || row > q.k) return;
  if (which && (q.drow0 < 0 || children_of(a, q, row) == 0)) return;
  float x[kPer];
  load_chunk<BF>(which ? a.draft : a.target, (which ? q.drow0 + row : q.row0 + row) * (which ? a.d_stride : a.t_stride), chunk,
                 a.vocab, x);
  const double c = which ? q.dc : q.c;
  float m = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    bad |= !(x[e] < INFINITY);
    m = fmaxf(m, x[e]);
  }
  m = block_max(m, s_max);
  double s = 0.0;
  if (m > -INFINITY && m < INFINITY) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) s += (double)power(x[e], m, c);
  }
  s = block_sum64(s, s_sum);
  const bool any = __syncthreads_or(bad);
  if (threadIdx.x == 0) part_of(a, r, which, row)[chunk] = SamplePart{s, m, any};
}

// Sum of max(p - C q, 0) over a chunk.
template <bool BF>
__device__ __forceinline__ double chunk_left(const SampleArgs& a, long long trow, long long drow, int chunk, float max,
                                             double c, double log_sum, float dmax, double dc, double dlog_sum, double cut,
                                             double* s_sum) {
  float x[kPer], y[kPer];
  load_chunk<BF>(a.target, trow, chunk, a.vocab, x);
  load_chunk<BF>(a.draft, drow, chunk, a.vocab, y);
  const double ps = exp2(-log_sum), qs = cut * exp2(-dlog_sum);
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) s += left_of(power(x[e], max, c), ps, power(y[e], dmax, dc), qs);
  return block_sum64(s, s_sum);
}

// Stage s: the mass left at every node of more than s children after s
// rejections.  Its C is the earlier C and the earlier mass.
template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_stage_kernel(const SampleArgs a, const int s) {
  __shared__ double s_sum[4];
  const int chunk = blockIdx.x, row = blockIdx.y, r = blockIdx.z;
  const Req q = load_req(a, r);
  if (!q.ok || row > q.k || q.drow0 < 0 || children_of(a, q, row) <= s) return;
  double cut = 1.0;
  if (s > 1) {
    const double* before = stage_of(a, s - 1, r, row);
    double v = 0.0;
    for (int i = threadIdx.x & 63; i < a.chunks; i += 64) v += before[i];
    cut = *cut_of(a, s - 1, r, row) + wave_sum64(v);
  }
  const RowStat t = row_stat(part_of(a, r, 0, row), a.chunks, q.c), d = row_stat(part_of(a, r, 1, row), a.chunks, q.dc);
  const double left = t.bad || d.bad ? 0.0
                                     : chunk_left<BF>(a, (q.row0 + row) * a.t_stride, (q.drow0 + row) * a.d_stride, chunk, t.max,
                                                      q.c, t.log_sum, d.max, q.dc, d.log_sum, cut, s_sum);
  if (threadIdx.x == 0) {
    stage_of(a, s, r, row)[chunk] = left;
    if (chunk == 0) *cut_of(a, s, r, row) = cut;
  }
}

// The walk: rows' statistics and the candidates' probabilities, all at once,
// then the tests in order.  One workgroup per request.
template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_decide_kernel(const SampleArgs a) {
  __shared__ float s_max[2][32];
  __shared__ double s_log[2][32], s_p[32], s_q[32], s_cut[32], s_mass[32];
  __shared__ int s_parent[32], s_cand[32], s_bad;
  const int r = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const Req q = load_req(a, r);
  if (tid == 0) s_bad = !q.ok || (a.gate && a.gate[r].nan_flag);
  __syncthreads();
  for (int w = wave; w < 2 * (q.k + 1); w += 4) {
    const int which = w & 1, row = w >> 1;
    if (which && (q.drow0 < 0 || children_of(a, q, row) == 0)) continue;
    if (!q.ok) continue;
    const RowStat st = row_stat(part_of(a, r, which, row), a.chunks, which ? q.dc : q.c);
    if (lane == 0) {
      s_max[which][row] = st.max;
      s_log[which][row] = st.log_sum;
      if (st.bad) s_bad = 1;
    }
  }
  // for candidate row i, the m-th child of its node (m >= 1): C and the mass after m
  // rejections (the last child's mass is never used)
  if (q.drow0 >= 0)
    for (int i = 1 + wave; i <= q.k; i += 4) {
      const int p = parent_of(a, q, i);
      const bool before = lane >= 1 && lane <= i && parent_of(a, q, lane) == p;
      const int m = __popcll(__ballot(before));
      const bool more = m < children_of(a, q, p);
      double v = 0.0, cut = 0.0;
      if (more) {
        for (int j = lane; j < a.chunks; j += 64) v += stage_of(a, m, r, p)[j];
        cut = *cut_of(a, m, r, p);
      } else if (m > 1) {
        for (int j = lane; j < a.chunks; j += 64) v += stage_of(a, m - 1, r, p)[j];
        cut = *cut_of(a, m - 1, r, p);
      }
      v = wave_sum64(v);
      if (lane == 0) {
        s_mass[i] = more ? v : 0.0;
        s_cut[i] = more ? cut : m > 1 ? cut + v : 1.0;
      }
    }
  __syncthreads();
  const bool bad = s_bad;
  if (tid >= 1 && tid <= q.k) {
    const int p = parent_of(a, q, tid), x = cand_of(a, q, tid);
    const bool in = x >= 0 && x < a.vocab;
    s_parent[tid] = p;
    s_cand[tid] = x;
    const float l = in && !bad ? logit<BF>(a.target, (q.row0 + p) * a.t_stride + x) : -INFINITY;
    const float dl = in && !bad && q.drow0 >= 0 ? logit<BF>(a.draft, (q.drow0 + p) * a.d_stride + x) : -INFINITY;
    s_p[tid] = prob(l, s_max[0][p], q.c, s_log[0][p]);
    s_q[tid] = q.drow0 >= 0 ? prob(dl, s_max[1][p], q.dc, s_log[1][p]) : 1.0;
    if (a.logp)
      a.logp[(size_t)r * (a.k + 1) + tid - 1] =
          bad ? NAN : l > -INFINITY ? (float)((((double)l - (double)s_max[0][p]) * q.c - s_log[0][p]) * kLn2) : -INFINITY;
  }
  if (a.logp && tid > q.k && tid <= a.k) a.logp[(size_t)r * (a.k + 1) + tid - 1] = NAN;
  __syncthreads();
  if (tid) return;
  SampleDecision& d = a.dec[r];
  int* path = a.reqs ? a.tree.path + q.row0 : a.path + (size_t)r * a.k;
  int at = 0, n = 0, n_gone = 0;
  double cut = 0.0, mass = 1.0;
  if (!bad)
    for (int i = 1; i <= q.k; ++i) {
      if (s_parent[i] != at) continue;
      double left;
      if (q.drow0 >= 0) {
        left = fmax(s_p[i] - cut * s_q[i], 0.0);
      } else {
        left = s_p[i];
        for (int j = 0; j < n_gone; ++j)
          if (d.gone[j] == s_cand[i]) left = 0.0;
      }
      if ((double)uniform_of(a, q, i) * mass * s_q[i] < left) {
        path[n] = i - 1;
        if (a.reqs) a.tree.host_path[q.row0 + n] = i - 1;
        ++n;
        at = i;
        n_gone = 0;
        cut = 0.0;
        mass = 1.0;
      } else if (q.drow0 >= 0) {
        cut = s_cut[i];
        mass = s_mass[i];
      } else {
        mass = fmax(mass - left, 0.0);
        d.gone[n_gone++] = s_cand[i];
      }
    }
  d.bad = bad;
  d.accepted = bad ? -1 : n;
  d.node = at;
  d.n_gone = n_gone;
  d.u = (double)uniform_of(a, q, 0);
  d.cut = cut;
  d.c = q.c;
  d.dc = q.dc;
  d.max = s_max[0][at];
  d.log_sum = s_log[0][at];
  d.draft = cut > 0.0;
  d.dmax = cut > 0.0 ? s_max[1][at] : 0.f;
  d.dlog_sum = cut > 0.0 ? s_log[1][at] : 0.0;
  if (!a.reqs) {
    for (int j = bad ? 0 : n; j < a.k; ++j) path[j] = -1;
    a.accepted[r] = d.accepted;
  }
}

// What is left of each chunk at the node that gives the token, where a
// drafter's distribution has been taken off.
template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_left_kernel(const SampleArgs a) {
  __shared__ double s_sum[4];
  const int chunk = blockIdx.x, r = blockIdx.y;
  const SampleDecision& d = a.dec[r];
  if (d.bad || !d.draft) return;
  const Req q = load_req(a, r);
  const double left = chunk_left<BF>(a, (q.row0 + d.node) * a.t_stride, (q.drow0 + d.node) * a.d_stride, chunk, d.max, d.c,
                                     d.log_sum, d.dmax, d.dc, d.dlog_sum, d.cut, s_sum);
  if (threadIdx.x == 0) a.left[(size_t)r * a.chunks + chunk] = left;
}

// The token: the chunk in which the running sum passes u S, then the column.
// One workgroup per request.
template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_pick_kernel(const SampleArgs a) {
  __shared__ double s_sum[4], s_run[kThreads];
  __shared__ int s_chunk, s_tok, s_gone[32];
  __shared__ double s_before;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Req q = load_req(a, r);
  const SampleDecision& d = a.dec[r];
  int tok = -1;
  if (!d.bad) {
    const long long trow = (q.row0 + d.node) * a.t_stride, drow = d.draft ? (q.drow0 + d.node) * a.d_stride : 0;
    const SamplePart* part = part_of(a, r, 0, d.node);
    int n_gone = d.n_gone;
    double cut = d.cut;
    if (tid < n_gone) s_gone[tid] = d.gone[tid];
    __syncthreads();
    // this thread's columns of a chunk, in column order: a run of kPer, with what is left of each
    auto values = [&](int chunk, double (&v)[kPer]) {
      const int c0 = chunk * kSampleChunk + tid * kPer;
      const double ps = exp2(-d.log_sum), qs = cut > 0.0 ? cut * exp2(-d.dlog_sum) : 0.0;
      const float m = cut > 0.0 ? d.max : part[chunk].max;
      const double scale = m > -INFINITY ? exp2(((double)m - (double)d.max) * d.c - d.log_sum) : 0.0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int col = c0 + e;
        v[e] = 0.0;
        if (col >= a.vocab || !(m > -INFINITY)) continue;
        const float p = power(logit<BF>(a.target, trow + col), m, d.c);
        v[e] = cut > 0.0 ? left_of(p, ps, power(logit<BF>(a.draft, drow + col), d.dmax, d.dc), qs) : (double)p * scale;
        for (int j = 0; j < n_gone; ++j)
          if (s_gone[j] == col) v[e] = 0.0;
      }
    };
    auto chunk_sum = [&](int chunk) {
      double v[kPer], s = 0.0;
      values(chunk, v);
#pragma unroll
      for (int e = 0; e < kPer; ++e) s += v[e];
      return block_sum64(s, s_sum);
    };
    // what is left of chunk i; a chunk with a rejected token is summed again without it
    auto left = [&](int i) {
      if (cut > 0.0) return a.left[(size_t)r * a.chunks + i];
      return part[i].max > -INFINITY ? part[i].sum * exp2(((double)part[i].max - (double)d.max) * d.c - d.log_sum) : 0.0;
    };
    __shared__ double s_again[32];
    auto search = [&]() -> bool {   // false: nothing is left
      for (int j = 0; j < n_gone; ++j) {
        const double s = chunk_sum(min(max(s_gone[j], 0), a.vocab - 1) / kSampleChunk);
        if (tid == 0) s_again[j] = s;
      }
      __syncthreads();
      auto at = [&](int i) {
        double v = left(i);
        for (int j = 0; j < n_gone; ++j)
          if (min(max(s_gone[j], 0), a.vocab - 1) / kSampleChunk == i) v = s_again[j];
        return v;
      };
      // the first wave: 64 chunks at a time, running sums across lanes
      if (tid < 64) {
        double total = 0.0;
        for (int i0 = 0; i0 < a.chunks; i0 += 64) total += wave_sum64(i0 + tid < a.chunks ? at(i0 + tid) : 0.0);
        const double goal = d.u * total;
        double before = 0.0;
        int found = -1, last = -1;
        double found_before = 0.0, last_before = 0.0;
        for (int i0 = 0; i0 < a.chunks && found < 0; i0 += 64) {
          const double v = i0 + tid < a.chunks ? at(i0 + tid) : 0.0;
          double run = v;
#pragma unroll
          for (int o = 1; o < 64; o <<= 1) {
            const double t = __shfl_up(run, o);
            if (tid >= o) run += t;
          }
          const uint64_t hit = __ballot(v > 0.0 && before + run > goal), some = __ballot(v > 0.0);
          if (some) {
            const int w = 63 - __clzll((long long)some);
            last = i0 + w;
            last_before = before + __shfl(run - v, w);
          }
          if (hit) {
            const int w = __ffsll((unsigned long long)hit) - 1;
            found = i0 + w;
            found_before = before + __shfl(run - v, w);
          }
          before += __shfl(run, 63);
        }
        if (tid == 0) {
          s_chunk = found >= 0 ? found : last;
          s_before = goal - (found >= 0 ? found_before : last_before);
        }
      }
      __syncthreads();
      return s_chunk >= 0;
    };
    bool some = search();
    if (!some) {   // everything was taken off (a rounding: the candidate would have been accepted): the target's own
      __syncthreads();
      n_gone = 0;
      cut = 0.0;
      some = search();
    }
    const int chunk = max(s_chunk, 0);
    double v[kPer], sum = 0.0;
    values(chunk, v);
#pragma unroll
    for (int e = 0; e < kPer; ++e) sum += v[e];
    // running sums over the threads
    s_run[tid] = sum;
    if (tid == 0) s_tok = 0x7fffffff;
    __syncthreads();
    double run = sum;
    {
      const int lane = tid & 63;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(run, o);
        if (lane >= o) run += t;
      }
      if (lane == 63) s_sum[tid >> 6] = run;
      __syncthreads();
      for (int w = 0; w < (tid >> 6); ++w) run += s_sum[w];
    }
    double before = run - sum;
    int mine = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      before += v[e];
      if (v[e] > 0.0) {
        if (before > s_before && mine == 0x7fffffff) mine = chunk * kSampleChunk + tid * kPer + e;
        last = chunk * kSampleChunk + tid * kPer + e;
      }
    }
    if (mine != 0x7fffffff) atomicMin(&s_tok, mine);
    __syncthreads();
    if (s_tok == 0x7fffffff) {   // the goal is the chunk's whole sum, up to rounding: its last column
      __syncthreads();
      if (tid == 0) s_tok = -1;
      __syncthreads();
      if (last >= 0) atomicMax(&s_tok, last);
      __syncthreads();
    }
    tok = s_tok >= 0 ? s_tok : chunk * kSampleChunk;
  }
  if (tid) return;
  float lp = NAN;
  if (!d.bad) {
    const float l = logit<BF>(a.target, (q.row0 + d.node) * a.t_stride + tok);
    lp = (float)((((double)l - (double)d.max) * d.c - d.log_sum) * kLn2);
  }
  if (a.reqs) {
    const StepOut o{d.accepted, tok, d.bad, 0};
    a.tree.sel[r] = o;
    a.tree.host[r] = o;
  } else {
    a.token[r] = tok;
    if (a.logp) a.logp[(size_t)r * (a.k + 1) + a.k] = lp;
  }
}

template <bool BF> hipError_t run(const SampleArgs& a, bool draft, int max_children, hipStream_t s) {
  sample_stats_kernel<BF><<<dim3(a.chunks, a.k + 1, (draft ? 2 : 1) * a.n), kThreads, 0, s>>>(a);
  if (draft)
    for (int st = 1; st < max_children; ++st) sample_stage_kernel<BF><<<dim3(a.chunks, a.k + 1, a.n), kThreads, 0, s>>>(a, st);
  sample_decide_kernel<BF><<<a.n, kThreads, 0, s>>>(a);
  if (draft) sample_left_kernel<BF><<<dim3(a.chunks, a.n), kThreads, 0, s>>>(a);
  sample_pick_kernel<BF><<<a.n, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool draft, int max_children, hipStream_t s) {
  if (a.n < 1 || a.k < 0 || a.k > 31 || a.vocab < 1 || a.chunks != (a.vocab + kSampleChunk - 1) / kSampleChunk || a.n > 32767)
    return hipErrorInvalidValue;
  return a.bf16 ? run<true>(a, draft, max_children, s) : run<false>(a, draft, max_children, s);
}

}  // namespace as2d
