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
// committed token then has the target's distribution: without a drafter's row
// whatever the candidates are, with one if they are independent draws from it
// (a tree of a row's most likely tokens is biased).
//
// Two rejections subtract a q, then b q; max(max(p - a q, 0) - b q, 0) =
// max(p - (a + b) q, 0), so a node's state is the single number C (the sum of
// the masses so far) and a mass is one pass over two rows:
//   R = max(p - C q, 0),  C_1 = 1, C_{m+1} = C_m + S(C_m).
// A mass needs nothing from the walk, so those of one rejection are formed for
// every node with a second child at once (that reject their first: its test is
// made on the way), and so on: as many passes as the most children of a node,
// less one, and none for a chain.  Without a drafter's row a mass is the row's
// sum without the rejected tokens.
//
// What bounds it: few rows, latency (a chain of 8, 9 rows of 152,064 logits, 5.5
// MB: 1.1 us at a copy's 5.1 TB/s; 15.1 us in one launch: its start, the pass,
// the last workgroup's ticket and the rows' parts, the tests, the token's chunk
// and column, each waiting for the one before); many rows, the pass over them
// (16 requests, 13 rows of each that matter, 126 MB: 31 us, 4.1 TB/s, two thirds
// of it 64-bit operations, 17 a logit; 18.9 for those of the 64 nodes with a
// second child whose first is rejected: their two rows are read again; and 16
// to finish).
//
// Rounding.  Powers are good to 2^-33.8 and everything summed over a row,
// compared or logged has 64 bits, so that a random number falls on another side
// of a border than in exact arithmetic only within 2^-31 of it: a draw from
// 152,064 tokens differs with a probability of 10^-7.  (float32 powers: 3 10^-4;
// the pass over 126 MB 25 us, the whole call of a chain 13.9.)
#include "common.h"

namespace as2d {

namespace {

constexpr int kPer = kSampleChunk / 64;   // logits of a lane
constexpr int kBlock = 256, kWide = 1024;  // threads: one pass over the logits, and the kernels that also combine parts
constexpr double kLog2E = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

// ---- powers -----------------------------------------------------------------

// 2^(d c) of a difference d <= 0 of logits, c = log2(e) / temperature, in 64
// bits: d c = n + f, |f| <= 1/2, and 2^f = 1 + f g(f), g of degree 6 by weighted
// least squares (relative error 2^-33.8).  Differences, and not x c, because x c
// has no bits left after the point where the temperature is small.
struct Power {
  double c, low;   // 2^(low c) is 0
  __device__ explicit Power(double c) : c(c), low(-1100.0 * __builtin_amdgcn_rcp(c)) {}
  __device__ __forceinline__ double operator()(double d) const {
    constexpr double kRound = 6755399441055744.0;   // 1.5 2^52: a sum's low bits are the nearest integer
    constexpr double g[7] = {0.6931471805416539,    0.24022651075853424,   0.05550410962572529,  0.009618036910832413,
                             0.0013333430786686678, 0.0001546711034876234, 1.5314946856354705e-05};
    d = fmax(d, low);
    const double t = __builtin_fma(d, c, kRound);
    const double f = __builtin_fma(d, c, kRound - t);
    double v = g[6];
#pragma unroll
    for (int i = 5; i >= 0; --i) v = __builtin_fma(v, f, g[i]);
    return __builtin_amdgcn_ldexp(__builtin_fma(v, f, 1.0), (int)(uint32_t)__builtin_bit_cast(uint64_t, t));
  }
  // of logit x relative to top, the largest of its row or chunk
  __device__ __forceinline__ double operator()(float x, double top) const { return (*this)((double)x - top); }
};

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
  q.ok = q.k >= 0 && q.k <= a.k && t >= kLeastTemp && t <= kMostTemp;
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
// This lane's parent row (lane = row 1 .. k; -1 for the others), and the rows
// that follow a row, as bits.
__device__ __forceinline__ int lane_parent(const SampleArgs& a, const Req& q) {
  const int lane = threadIdx.x & 63;
  return lane >= 1 && lane <= q.k ? parent_of(a, q, lane) : -1;
}
__device__ __forceinline__ uint32_t children_of(int parent, int row) { return (uint32_t)__ballot(parent == row); }

// ---- rows of logits ---------------------------------------------------------

template <bool BF> __device__ __forceinline__ float logit(const void* base, long long i) {
  if constexpr (BF) return bf2f(ldg(static_cast<const uint16_t*>(base) + i));
  else return ldg(static_cast<const float*>(base) + i);
}

// A lane's kPer logits of a wave's chunk: runs of 16 bytes, 64 lanes apart (rows
// may start at any element: the loads need no alignment past the element's).
// Columns past the row read -inf.
template <bool BF> __device__ __forceinline__ int column(int e) {
  constexpr int RUN = BF ? 8 : 4;
  return ((e / RUN) * 64 + (int)(threadIdx.x & 63)) * RUN + e % RUN;
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

// What is left of a column: max(p - C q, 0) from the two powers and the factors
// 1 / sum and C / sum.  One rounding per operation wherever it is formed, so
// that a chunk's sum is positive exactly where one of its columns is.
__device__ __forceinline__ double left_of(double p, double ps, double q, double qs) {
#pragma clang fp contract(off)
  return fmax(p * ps - q * qs, 0.0);
}

// ---- reductions: fixed trees, the same bits in every lane -------------------

// (cross-lane moves that do not go through the LDS, a 32-bit half at a time)

template <int CTRL, int ROWS = 0xF> __device__ __forceinline__ double dpp_get64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// op of lane l's and lane l ^ 16's (SWAP32: l ^ 32's) values, in the lower lane's order.
template <bool SWAP32, class Op> __device__ __forceinline__ double swap64(double v, Op op) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t l = (uint32_t)u, h = (uint32_t)(u >> 32);
  const auto swap = [](uint32_t w) {
    if constexpr (SWAP32) return __builtin_amdgcn_permlane32_swap(w, w, false, false);
    else return __builtin_amdgcn_permlane16_swap(w, w, false, false);
  };
  const auto a = swap(l), b = swap(h);
  return op(__builtin_bit_cast(double, (uint64_t)b[0] << 32 | a[0]), __builtin_bit_cast(double, (uint64_t)b[1] << 32 | a[1]));
}
template <class Op> __device__ __forceinline__ double wave_reduce64(double v, Op op) {
  v = op(v, dpp_get64<kDppXor1>(v));
  v = op(v, dpp_get64<kDppXor2>(v));
  v = op(v, dpp_get64<kDppHalfMirror>(v));
  v = op(v, dpp_get64<kDppMirror>(v));
  return swap64<true>(swap64<false>(v, op), op);
}
__device__ __forceinline__ double wave_sum64(double v) {
  return wave_reduce64(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double wave_max64(double v) {
  return wave_reduce64(v, [](double a, double b) { return fmax(a, b); });
}
// Running sums, this lane's included: within 16 lanes, then the rows before.
__device__ __forceinline__ double wave_scan64(double v) {
  v += dpp_get64<0x111>(v);        // row_shr 1, 2, 4, 8 (0 from before the row)
  v += dpp_get64<0x112>(v);
  v += dpp_get64<0x114>(v);
  v += dpp_get64<0x118>(v);
  v += dpp_get64<0x142, 0xA>(v);   // lane 15 of rows 0 and 2 to rows 1 and 3
  v += dpp_get64<0x143, 0xC>(v);   // lane 31 to rows 2 and 3
  return v;
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

// A row's sum of 2^((x - top) c) from its chunks' parts, top its largest
// logit; bad: a value that is no logit, or none that is finite.  rest: the sum
// without the chunks that lanes `gone` (bits) have in `ours`.  One wave, every
// lane gets them.
struct RowStat {
  double sum, top, rest;
  int bad;
};
template <bool COH> __device__ __forceinline__ SamplePart load_part(const SamplePart* p) {
  if constexpr (COH) return SamplePart{ld_coherent(&p->sum), ld_coherent(&p->top)};
  else return *p;
}
__device__ __forceinline__ bool one_of(int chunk, int ours, uint32_t gone) {
  bool is = false;
  for (uint32_t b = gone; b; b &= b - 1) is |= __builtin_amdgcn_readlane(ours, __builtin_ctz(b)) == chunk;
  return is;
}
template <bool COH>
__device__ __forceinline__ RowStat row_stat(const SamplePart* part, int chunks, const Power& w, int ours = -1, uint32_t gone = 0) {
  const int lane = threadIdx.x & 63;
  constexpr int B = 4;   // a lane's first parts, kept (262,144 tokens: all of them)
  SamplePart p[B];
  double top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    p[i] = SamplePart{0.0, -INFINITY};
    if (64 * i + lane < chunks) p[i] = load_part<COH>(part + 64 * i + lane);
  }
#pragma unroll
  for (int i = 0; i < B; ++i) {
    bad |= p[i].top != p[i].top;
    top = fmax(top, p[i].top);
  }
  for (int i = 64 * B + lane; i < chunks; i += 64) {
    const double t = load_part<COH>(part + i).top;
    bad |= t != t;
    top = fmax(top, t);
  }
  top = wave_max64(top);
  double s = 0.0, rest = 0.0;
  const auto add = [&](const SamplePart& v, int chunk) {   // by every lane: one_of reads the others' candidates
    const bool is = gone && one_of(chunk, ours, gone);
    if (!(v.top > -INFINITY)) return;
    const double x = v.sum * w(v.top - top);
    s += x;
    rest += is ? 0.0 : x;
  };
#pragma unroll
  for (int i = 0; i < B; ++i) add(p[i], 64 * i + lane);
  for (int i0 = 64 * B; i0 < chunks; i0 += 64) {
    SamplePart v{0.0, -INFINITY};
    if (i0 + lane < chunks) v = load_part<COH>(part + i0 + lane);
    add(v, i0 + lane);
  }
  s = wave_sum64(s);
  return RowStat{s, top, gone ? wave_sum64(rest) : s, __ballot(bad) != 0 || !(top > -INFINITY)};
}
__device__ __forceinline__ double prob(float x, const RowStat& t, const Power& w) {
  return w(x, t.top) / t.sum;
}
// log p of a token in natural units, rounded once.
__device__ __forceinline__ float log_prob(float x, double top, double log_sum, double c) {
  return (float)((((double)x - top) * c - log_sum) * kLn2);
}

// A candidate's test from p(x), q(x), C and the mass S of what is left.  The
// stages and the walk have to agree on it to the last bit.
__device__ __forceinline__ double share_left(double p, double q, double cut) {
#pragma clang fp contract(off)
  return fmax(p - cut * q, 0.0);
}
__device__ __forceinline__ bool accepts(float u, double mass, double q, double left) {
#pragma clang fp contract(off)
  return (double)u * mass * q < left;
}

// ---- kernels ----------------------------------------------------------------

// A wave's chunk of a row: its largest logit and its sum relative to that.
template <bool BF> __device__ __forceinline__ SamplePart chunk_part(const void* base, long long row, int chunk, int vocab, const Power& w) {
  float x[kPer];
  load_chunk<BF>(base, row, chunk, vocab, x);
  float m = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    bad |= !(x[e] < INFINITY);
    m = fmaxf(m, x[e]);
  }
  m = wave_max(m);
  const double top = __ballot(bad) != 0 ? NAN : m;
  double s = 0.0;
  if (top > -INFINITY) {
#pragma unroll
    for (int e = 0; e < kPer; e += 4)
      s += (w(x[e], top) + w(x[e + 1], top)) + (w(x[e + 2], top) + w(x[e + 3], top));
    s = wave_sum64(s);
  }
  return SamplePart{s, top};
}

// Chunk of the vocabulary of a candidate.
__device__ __forceinline__ int chunk_of(int x, int vocab) { return x >= 0 && x < vocab ? x / kSampleChunk : -1; }
// A rejected candidate's chunk without the rejected tokens (x: lane i's
// candidate, gone: those of one node), 0 where an earlier one of them has the
// chunk; one wave.
template <bool BF, bool COH>
__device__ __forceinline__ SamplePart chunk_rest(const SampleArgs& a, long long row, const SamplePart* part, const Power& w, int x, int i,
                                                 uint32_t gone) {
  const int ours = chunk_of(x, a.vocab), ch = __builtin_amdgcn_readlane(ours, i);
  const uint32_t same = (uint32_t)__ballot(ours == ch) & gone;
  if (ch < 0 || __builtin_ctz(same) != i) return SamplePart{0.0, -INFINITY};
  float y[kPer];
  load_chunk<BF>(a.target, row, ch, a.vocab, y);
  const double top = load_part<COH>(part + ch).top;
  if (!(top > -INFINITY)) return SamplePart{0.0, -INFINITY};
  double v = 0.0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) v += one_of(ch * kSampleChunk + column<BF>(e), x, same) ? 0.0 : w(y[e], top);
  return SamplePart{wave_sum64(v), top};
}
__device__ __forceinline__ uint32_t but_last(uint32_t children) {
  return children ? children & ~(0x80000000u >> __builtin_clz(children)) : 0;
}

// The parts of every chunk of the target's rows and of the drafter's rows with
// children, a chunk per wave.  The one pass over the logits that cannot be
// avoided.
template <bool BF>
__global__ __launch_bounds__(kBlock) void sample_stats_kernel(const SampleArgs a) {
  const int chunk = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6), row = blockIdx.y;
  const int which = (int)blockIdx.z >= a.n, r = blockIdx.z - which * a.n;
  const Req q = load_req(a, r);
  if (!q.ok || row > q.k || chunk >= a.chunks) return;
  if (which && (q.drow0 < 0 || !children_of(lane_parent(a, q), row))) return;
  const SamplePart p =
      chunk_part<BF>(which ? a.draft : a.target, (which ? q.drow0 + row : q.row0 + row) * (which ? a.d_stride : a.t_stride),
                     chunk, a.vocab, Power(which ? q.dc : q.c));
  if ((threadIdx.x & 63) == 0) part_of(a, r, which, row)[chunk] = p;
}

// Sum of max(p - C q, 0) over a wave's chunk; ps, qs: 1 / sum and C / sum.
template <bool BF>
__device__ __forceinline__ double chunk_left(const SampleArgs& a, long long trow, long long drow, int chunk, double top,
                                             const Power& w, double ps, double dtop, const Power& dw, double qs) {
  float x[kPer], y[kPer];
  load_chunk<BF>(a.target, trow, chunk, a.vocab, x);
  load_chunk<BF>(a.draft, drow, chunk, a.vocab, y);
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) s += left_of(w(x[e], top), ps, dw(y[e], dtop), qs);
  return wave_sum64(s);
}

// Stage s: the mass left at every node of more than s children whose first s are
// all rejected (C < 0 marks the others: the walk never asks for theirs).  Its C
// is the earlier C and the earlier mass.  What that test saves depends on how
// often a first child is accepted: 16 requests of 8 candidates in twos over
// 152,064 float32 logits took 25.5 us without it and 18.9 with it; 4 requests of
// 15 in threes over 50,257 bf16 logits 9.2 a stage without it and 8.9 with it
// (the whole call 40.5 and 40.3).
template <bool BF>
__global__ __launch_bounds__(kWide) void sample_stage_kernel(const SampleArgs a, const int s) {
  __shared__ RowStat s_stat[2];
  __shared__ double s_cut, s_mass;
  __shared__ float s_u, s_l, s_dl;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int chunk = blockIdx.x * (kWide / 64) + wave, row = blockIdx.y, r = blockIdx.z;
  const Req q = load_req(a, r);
  if (!q.ok || row > q.k || q.drow0 < 0) return;
  uint32_t children = children_of(lane_parent(a, q), row);
  if (__popc(children) <= s) return;
  if (wave < 2) {
    const RowStat t = row_stat<false>(part_of(a, r, wave, row), a.chunks, Power(wave ? q.dc : q.c));
    if (lane == 0) s_stat[wave] = t;
  } else if (wave == 2) {
    double cut = 0.0, mass = 1.0;   // before the s-th child
    if (s > 1) {
      cut = *cut_of(a, s - 1, r, row);
      const double* before = stage_of(a, s - 1, r, row);
      double v = 0.0;
      if (cut >= 0.0)
        for (int i = lane; i < a.chunks; i += 64) v += before[i];
      mass = wave_sum64(v);
    }
    if (lane == 0) {
      s_cut = cut;
      s_mass = mass;
    }
  } else if (wave == 3 && lane == 0) {   // the s-th child
    for (int i = 1; i < s; ++i) children &= children - 1;
    const int i = __builtin_ctz(children), x = cand_of(a, q, i);
    s_u = uniform_of(a, q, i);
    const bool in = x >= 0 && x < a.vocab;
    s_l = in ? logit<BF>(a.target, (q.row0 + row) * a.t_stride + x) : -INFINITY;
    s_dl = in ? logit<BF>(a.draft, (q.drow0 + row) * a.d_stride + x) : -INFINITY;
  }
  __syncthreads();
  const RowStat t = s_stat[0], d = s_stat[1];
  bool skip = s_cut < 0.0;
  if (!skip && !t.bad && !d.bad) {
    const double qx = prob(s_dl, d, Power(q.dc));
    skip = accepts(s_u, s_mass, qx, share_left(prob(s_l, t, Power(q.c)), qx, s_cut));
  }
  const double cut = s_cut + s_mass;
  if (blockIdx.x == 0 && threadIdx.x == 0) *cut_of(a, s, r, row) = skip ? -1.0 : cut;
  if (skip || chunk >= a.chunks) return;
  const double left = t.bad || d.bad ? 0.0
                                     : chunk_left<BF>(a, (q.row0 + row) * a.t_stride, (q.drow0 + row) * a.d_stride, chunk, t.top,
                                                      Power(q.c), 1.0 / t.sum, d.top, Power(q.dc), cut / d.sum);
  if (lane == 0) stage_of(a, s, r, row)[chunk] = left;
}

// A running sum over the workgroup: the first index with v > 0 whose sum up
// to and with it passes `goal`, or the last with v > 0 (the goal is the whole
// sum, up to rounding), or -1; *before receives the sum before it.  One value
// per thread, in order.
struct Find {
  double wave[kWide / 64], before;
  int first, last;
};
template <class Goal> __device__ __forceinline__ int find_in_run(double v, Goal&& goal_of, Find& f, double* before) {
  const int tid = threadIdx.x, wave = tid >> 6;
  const double run = wave_scan64(v);
  __syncthreads();   // f may be in use
  if (tid == 0) {
    f.first = 0x7fffffff;
    f.last = -1;
  }
  if ((tid & 63) == 63) f.wave[wave] = run;
  __syncthreads();
  double base = 0.0, total = 0.0;
#pragma unroll
  for (int w = 0; w < kWide / 64; ++w) {
    if (w == wave) base = total;
    total += f.wave[w];
  }
  const double goal = goal_of(total);
  const bool some = v > 0.0, hit = some && base + run > goal;
  const uint64_t hits = __ballot(hit), any = __ballot(some);
  if ((tid & 63) == 0) {
    if (hits) atomicMin(&f.first, (wave << 6) + __ffsll((unsigned long long)hits) - 1);
    if (any) atomicMax(&f.last, (wave << 6) + 63 - __clzll((long long)any));
  }
  __syncthreads();
  const int at = f.first != 0x7fffffff ? f.first : f.last;
  if (tid == at) f.before = base + run - v;
  __syncthreads();
  if (before) *before = goal - f.before;
  return at;
}

// The walk and the token.  Every test's outcome follows from its node's
// earlier siblings having failed, so all are made at once, a candidate per
// lane, and the walk follows bits.  `blocks` workgroups per request: more
// than one where a drafter's distribution may have to be taken off the
// node's; each then makes the same walk, sums its share of what is left, and
// the last to finish draws the token.  FUSED: one workgroup, in the kernel that
// made the parts.
template <bool BF, bool FUSED> __device__ __forceinline__ void sample_finish(const SampleArgs& a, const Req& q, int block, int blocks) {
  constexpr int kWavesW = kWide / 64;
  __shared__ RowStat s_stat[2][32];
  __shared__ double s_left[32], s_again[32], s_log[32];
  __shared__ SamplePart s_rest[32];
  __shared__ uint32_t s_children[32];
  __shared__ int s_cand[32], s_bad, s_at, s_n, s_path[32], s_last;
  __shared__ double s_cut, s_cutoff[32];
  __shared__ Find s_find;
  const int r = q.r, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const bool writes = block == 0;
  const bool drafted = q.drow0 >= 0;
  if (tid == 0) s_bad = !q.ok || (a.gate && a.gate[r].nan_flag);
  const int parent = lane_parent(a, q);
  // candidates: what they need from memory, in flight while the rows' parts are combined
  const bool cand = wave < 2 && lane >= 1 && lane <= q.k;   // wave 0: the tests, wave 1: log-probabilities
  const float u_tok = uniform_of(a, q, 0);
  const bool several = !drafted && a.max_children > 1;
  int x = -1;
  float u = 0.f, l = -INFINITY, dl = -INFINITY;
  if ((cand || several) && lane >= 1 && lane <= q.k) x = cand_of(a, q, lane);
  if (cand) {
    u = uniform_of(a, q, lane);
    if (x >= 0 && x < a.vocab) {
      l = logit<BF>(a.target, (q.row0 + parent) * a.t_stride + x);
      if (drafted) dl = logit<BF>(a.draft, (q.drow0 + parent) * a.d_stride + x);
    }
  }
  if (several)
    for (int i = 1 + wave; i <= q.k; i += kWavesW) {
      const int p = __shfl(parent, i);
      const uint32_t gone = but_last(children_of(parent, p));
      if (!(gone >> i & 1)) continue;
      const SamplePart v = chunk_rest<BF, FUSED>(a, (q.row0 + p) * a.t_stride, part_of(a, r, 0, p), Power(q.c), x, i, gone);
      if (lane == 0) s_rest[i] = v;
    }
  __syncthreads();
  for (int w = wave; w < 2 * (q.k + 1) && q.ok; w += kWavesW) {
    const int which = w > q.k, row = w - which * (q.k + 1);
    const uint32_t children = children_of(parent, row);
    if (!which && lane == 0) s_children[row] = children;
    if (which && (!drafted || !children)) continue;
    // Without a drafter's row: what is left once every child but the last is
    // rejected, summed from what is left (1 less their probabilities would have
    // nothing but roundings where a child is near certain).
    const uint32_t gone = several ? but_last(children) : 0;
    const bool mine = lane < 32 && gone >> (lane & 31) & 1;
    const Power pw(which ? q.dc : q.c);
    RowStat st = row_stat<FUSED>(part_of(a, r, which, row), a.chunks, pw, chunk_of(x, a.vocab), gone);
    if (gone) {
      const SamplePart v = mine ? s_rest[lane] : SamplePart{0.0, -INFINITY};
      st.rest += wave_sum64(v.top > -INFINITY ? v.sum * pw(v.top - st.top) : 0.0);
    }
    if (lane == 0) {
      s_stat[which][row] = st;
      if (st.bad) s_bad = 1;
    }
  }
  // candidate i of a drafter's row: C and the mass once its m earlier siblings have been rejected
  if (drafted && a.max_children > 1)
    for (int i = 1 + wave; i <= q.k; i += kWavesW) {
      const int p = __shfl(parent, i);
      const int m = __popc(children_of(parent, p) & ((1u << i) - 1));
      double v = 1.0, cut = 0.0;
      if (m) {
        cut = *cut_of(a, m, r, p);
        v = 0.0;
        if (cut >= 0.0)   // else an earlier sibling is accepted: this one is not asked for
          for (int j = lane; j < a.chunks; j += 64) v += stage_of(a, m, r, p)[j];
        v = wave_sum64(v);
      }
      if (lane == 0) {
        s_cutoff[i] = fmax(cut, 0.0);
        s_left[i] = v;
      }
    }
  __syncthreads();
  const bool bad = s_bad;
  if (wave == 0) {
    const bool siblings = drafted && a.max_children > 1 && cand;
    const double cut = siblings ? s_cutoff[lane] : 0.0;
    double mass = siblings ? s_left[lane] : 1.0;
    double p = 0.0, qx = 1.0;
    if (cand && !bad) {
      p = prob(l, s_stat[0][parent], Power(q.c));
      if (drafted) qx = prob(dl, s_stat[1][parent], Power(q.dc));
    }
    double left = drafted ? share_left(p, qx, cut) : p;
    if (lane < 32) s_cand[lane] = x;
    uint32_t before = cand && !bad && !drafted ? s_children[parent] & ((1u << lane) - 1) : 0;
    for (uint32_t b = before; b; b &= b - 1)   // a sibling that was rejected has taken the token
      if (s_cand[__builtin_ctz(b)] == x) left = 0.0;
    if (lane < 32) s_left[lane] = left;
    if (before) {   // what all children but the last leave, and those of them that are not tried yet
      mass = s_stat[0][parent].rest / s_stat[0][parent].sum;
      for (uint32_t b = but_last(s_children[parent]) & ~((1u << lane) - 1); b; b &= b - 1) mass += s_left[__builtin_ctz(b)];
    }
    const bool yes = cand && !bad && accepts(u, mass, qx, left);
    const uint32_t accepted = (uint32_t)__ballot(yes);
    if (lane < 32) s_cutoff[lane] = cut + mass;   // C once this child is rejected too
    if (lane == 0) {
      int at = 0, n = 0;
      for (uint32_t next; !bad && (next = s_children[at] & accepted); ) {
        at = __builtin_ctz(next);   // a child's row is past its parent's: the walk ends
        s_path[n++] = at - 1;
      }
      const uint32_t tried = bad ? 0 : s_children[at];
      s_at = at;
      s_n = n;
      s_cut = tried && drafted ? s_cutoff[31 - __builtin_clz(tried)] : 0.0;
    }
  }
  if (wave == 1 && a.logp) {
    if (lane <= q.k && !bad) s_log[lane] = log2(s_stat[0][lane].sum);
    __builtin_amdgcn_wave_barrier();
    if (writes && lane >= 1 && lane <= a.k)
      a.logp[(size_t)r * (a.k + 1) + lane - 1] = bad || lane > q.k ? NAN : log_prob(l, s_stat[0][parent].top, s_log[parent], q.c);
  }
  __syncthreads();
  const int at = s_at, n = s_n;
  if (writes) {
    if (a.reqs) {
      if (tid < n) a.tree.path[q.row0 + tid] = a.tree.host_path[q.row0 + tid] = s_path[tid];
    } else {
      if (tid < a.k) a.path[(size_t)r * a.k + tid] = tid < n ? s_path[tid] : -1;
      if (tid == 0) a.accepted[r] = bad ? -1 : n;
    }
  }
  double taken = s_cut;   // multiples of the drafter's distribution
  if (bad || !(taken > 0.0)) {
    if (!writes) return;
  }
  const RowStat t = s_stat[0][at];
  const long long trow = (q.row0 + at) * a.t_stride, drow = drafted ? (q.drow0 + at) * a.d_stride : 0;
  const double ps = 1.0 / t.sum;
  RowStat d{};
  double qs = 0.0;
  if (taken > 0.0) {
    d = s_stat[1][at];
    qs = taken / d.sum;
    double* out = a.left + (size_t)r * a.chunks;
    for (int chunk = block * kWavesW + wave; chunk < a.chunks; chunk += blocks * kWavesW) {
      const double v = chunk_left<BF>(a, trow, drow, chunk, t.top, Power(q.c), ps, d.top, Power(q.dc), qs);
      if (lane == 0) st<true>(out + chunk, v);
    }
    if (blocks > 1) {
      wait_vmem();
      __syncthreads();
      if (tid == 0) {
        s_last = counter_add(a.ticket + r, 1) == blocks - 1;
        if (s_last) st<true>(a.ticket + r, 0);   // ready for the next call
      }
      __syncthreads();
      if (!s_last) return;
    } else {
      wait_vmem();
      __syncthreads();
    }
  }
  // by the thread that has the token's logit
  const auto give = [&](int tok, float y) {
    if (a.reqs) {
      const StepOut o{bad ? -1 : n, tok, bad, 0};
      a.tree.sel[r] = o;
      a.tree.host[r] = o;
      return;
    }
    a.token[r] = tok;
    if (a.logp) a.logp[(size_t)r * (a.k + 1) + a.k] = bad ? NAN : log_prob(y, t.top, s_log[at], q.c);
  };
  if (bad) {
    if (tid == 0) give(-1, 0.f);
    return;
  }
  {
    const SamplePart* part = part_of(a, r, 0, at);
    uint32_t gone = drafted ? 0 : s_children[at];   // rejected rows
    const auto is_gone = [&](int col) {
      bool g = false;
      for (uint32_t b = gone; b; b &= b - 1) g |= s_cand[__builtin_ctz(b)] == col;
      return g;
    };
    int chunk = -1;
    double rest = 0.0;
    for (int round = 0; round < 2 && chunk < 0; ++round) {
      if (round) {   // nothing is left (a rounding: the last child would have been accepted): the target's own
        taken = 0.0;
        gone = 0;
      }
      // chunks of rejected tokens are summed again without them, a wave each
      for (int i = wave; i <= q.k; i += kWavesW)
        if (gone >> i & 1) {
          const int ch = chunk_of(s_cand[i], a.vocab);
          double v = 0.0;
          if (ch >= 0) {
            float y[kPer];
            load_chunk<BF>(a.target, trow, ch, a.vocab, y);
            const double top = load_part<FUSED>(part + ch).top;
            if (top > -INFINITY) {
#pragma unroll
              for (int e = 0; e < kPer; ++e)
                v += is_gone(ch * kSampleChunk + column<BF>(e)) ? 0.0 : Power(q.c)(y[e], top);
            }
            v = wave_sum64(v);
          }
          if (lane == 0) s_again[i] = v;
        }
      __syncthreads();
      const auto left = [&](int i) -> double {
        if (taken > 0.0) return ld_coherent(a.left + (size_t)r * a.chunks + i);
        const SamplePart p = load_part<FUSED>(part + i);
        double v = p.sum;
        for (uint32_t b = gone; b; b &= b - 1)
          if (chunk_of(s_cand[__builtin_ctz(b)], a.vocab) == i) v = s_again[__builtin_ctz(b)];
        return v > 0.0 ? v * Power(q.c)(p.top - t.top) : 0.0;
      };
      // a run of chunks per thread (up to 1,048,576 tokens: one chunk)
      const int per = (a.chunks + kWide - 1) / kWide;
      double v = 0.0;
      for (int i = tid * per; i < min((tid + 1) * per, a.chunks); ++i) v += left(i);
      const int who = find_in_run(v, [&](double total) { return (double)u_tok * total; }, s_find, &rest);
      chunk = who;
      if (who >= 0 && per > 1) {
        if (tid == who) {
          int c = -1;
          double goal = rest, at_c = 0.0;
          for (int i = tid * per; i < min((tid + 1) * per, a.chunks); ++i) {
            const double w = left(i);
            if (!(w > 0.0)) continue;
            c = i;
            at_c = goal;
            if (w > goal) break;
            goal -= w;
          }
          s_at = c;
          s_find.before = at_c;
        }
        __syncthreads();
        chunk = s_at;
        rest = s_find.before;
      }
    }
    chunk = max(chunk, 0);
    // the chunk's columns, one per thread: each summed as its chunk's sum took it
    const int col = chunk * kSampleChunk + tid;
    double v = 0.0;
    float y = -INFINITY;
    if (col < a.vocab) {
      y = logit<BF>(a.target, trow + col);
      if (taken > 0.0) {
        v = left_of(Power(q.c)(y, t.top), ps, Power(q.dc)(logit<BF>(a.draft, drow + col), d.top), qs);
      } else {
        const double top = load_part<FUSED>(part + chunk).top;
        if (top > -INFINITY && !is_gone(col)) v = Power(q.c)(y, top) * Power(q.c)(top - t.top);
      }
    }
    int who = find_in_run(v, [&](double) { return rest; }, s_find, nullptr);
    if (who < 0)   // columns that are 0 one by one (2^-1075), their sum is not: the first of them
      who = find_in_run(y > -INFINITY && !is_gone(col) ? 1.0 : 0.0, [](double) { return 0.0; }, s_find, nullptr);
    if (tid == max(who, 0)) give(min(col, a.vocab - 1), y);
  }
}

template <bool BF> __global__ __launch_bounds__(kWide) void sample_finish_kernel(const SampleArgs a) {
  sample_finish<BF, false>(a, load_req(a, blockIdx.y), blockIdx.x, gridDim.x);
}

// Both in one launch, without a drafter's rows: the last workgroup of a request
// to have made its parts finishes it.
template <bool BF> __global__ __launch_bounds__(kWide) void sample_fused_kernel(const SampleArgs a) {
  __shared__ int s_last;
  const int row = blockIdx.y, r = blockIdx.z, chunk = blockIdx.x * (kWide / 64) + (threadIdx.x >> 6);
  const Req q = load_req(a, r);
  if (row > q.k) return;
  if (q.ok) {
    if (chunk < a.chunks) {
      const SamplePart p = chunk_part<BF>(a.target, (q.row0 + row) * a.t_stride, chunk, a.vocab, Power(q.c));
      if ((threadIdx.x & 63) == 0) {
        SamplePart* out = part_of(a, r, 0, row) + chunk;
        st<true>(&out->sum, p.sum);
        st<true>(&out->top, p.top);
      }
    }
    wait_vmem();
    __syncthreads();   // the workgroup's parts are stored
    if (threadIdx.x == 0) {
      s_last = counter_add(a.ticket + r, 1) == (int)gridDim.x * (q.k + 1) - 1;
      if (s_last) st<true>(a.ticket + r, 0);   // ready for the next call
    }
    __syncthreads();
    if (!s_last) return;
  } else if (blockIdx.x) {
    return;   // refused: nothing to wait for
  }
  sample_finish<BF, true>(a, q, 0, 1);
}

// Up to this many workgroups (one per compute unit) a call without a drafter is
// one launch: 16 requests of one row of 152,064 logits (160 workgroups) 13.2 us
// against 15.4 in two, 1 request of 32 rows (320) 23.7 against 21.4, 16 of 9
// (1,440) 45.7 against 30.7: past one workgroup a unit the larger kernel's fewer
// waves hold the pass back.
constexpr long long kFusedBlocks = 256;

template <bool BF> hipError_t run(const SampleArgs& a, bool draft, hipStream_t s) {
  static_assert(kSampleChunk == kWide, "the token's chunk: a column per thread");
  const auto blocks = [&](int threads) { return (a.chunks + threads / 64 - 1) / (threads / 64); };
  if (!draft && (long long)blocks(kWide) * (a.k + 1) * a.n <= kFusedBlocks) {
    sample_fused_kernel<BF><<<dim3(blocks(kWide), a.k + 1, a.n), kWide, 0, s>>>(a);
    return hipGetLastError();
  }
  sample_stats_kernel<BF><<<dim3(blocks(kBlock), a.k + 1, (draft ? 2 : 1) * a.n), kBlock, 0, s>>>(a);
  if (draft)
    for (int st = 1; st < a.max_children; ++st)
      sample_stage_kernel<BF><<<dim3(blocks(kWide), a.k + 1, a.n), kWide, 0, s>>>(a, st);
  sample_finish_kernel<BF><<<dim3(draft ? blocks(kWide) : 1, a.n), kWide, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool draft, hipStream_t s) {
  if (a.n < 1 || a.k < 0 || a.k > 31 || a.vocab < 1 || a.chunks != (a.vocab + kSampleChunk - 1) / kSampleChunk || a.n > 32767)
    return hipErrorInvalidValue;
  return a.bf16 ? run<true>(a, draft, s) : run<false>(a, draft, s);
}

}  // namespace as2d
