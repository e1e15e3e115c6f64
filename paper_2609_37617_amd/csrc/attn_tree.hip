// Attention of trees of candidates over long caches (bf16 models).
//
// A row's result is sum_j 2^(s_j - M) v_j / sum_j 2^(s_j - M) over the keys it
// sees, s_j = (q . k_j) log2(e) / sqrt(d); the products take the cache's (hi,
// lo) pairs as attn.h does.  No result has to have the bits of another path
// here (a tree's keys are summed in an order of their own), so the keys are
// split into a run per workgroup and a run keeps one running state, instead of
// one state per 128 keys.
//
// A workgroup of eight waves takes 64 T rows of the query heads that share a KV
// head and a run of keys, 64 at a time through LDS (two buffers): four waves
// of T row tiles each on the first 32 keys, four on the other 32; the halves'
// states meet once, at the end.  Both products are formed transposed (s: keys
// x rows, A: dimensions x rows), so a lane holds values of one query row; its
// sum stays the lane's own until the end, and its maximum is raised (and the
// sums rescaled) only where a score passes it by more than 2^8.
//
// What bounds it: 64 keys of a head are 64 KiB, read by the LDS eight times
// (2,048 cycles a step at 128 bytes a cycle) and multiplied by 16 T + 24 T
// products a wave (two waves on each SIMD: 1,280 T cycles), so two tiles a wave
// balance the two; one tile leaves the LDS as the limit, but shares the keys among
// twice the workgroups (as2d.cpp has the rule).  Measured, 7B heads, 32 rows (224
// per KV head): over 7,564 keys, one tile, 24.5 us and 5 us for the join (one
// layer; the cache's 31 MB at a copy's 5.1 TB/s: 6 us), over 32,704 keys, two
// tiles, 55.5 and 6.5 (134 MB: 26 us); workgroups of 128 keys and 16 rows took 68 and 225.  A step
// of 64 keys takes 2.7 us: the loads alone 2.5 (a step's burst, one in flight),
// the products and powers alone 2.3, matrix cores a quarter busy.  All rows of a
// KV head in one workgroup with two smaller steps in flight (256 rows): 55 us and
// 9.8 for twice the states; the second half's value products a step late: 59;
// operands two groups ahead of their products: 40 registers spilled, 55.
#include "attn.h"

namespace as2d {

constexpr int kTreeWaves = 8;
constexpr int kTreeThreads = 64 * kTreeWaves;
constexpr int kTreeStep = 64;                                 // keys of a step
constexpr int kTreeStepsPerSpan = kAttnSpanKeys / kTreeStep;   // runs are whole spans
constexpr float kTreeSlack = 8.0f;                             // 2^8 over the maximum before it is raised

template <int D> __host__ __device__ constexpr int tree_units() { return kTreeStep * D * 4 / 16; }   // of a step's keys, or values
template <int D> __host__ __device__ constexpr int tree_lds_bytes() { return 2 * 2 * tree_units<D>() * 16; }

// Spans per run and items of a launch of G workgroups with T tiles a wave: of a
// pass's requests (device), or of one (host).
__host__ __device__ inline int tree_spans(const ReqDesc& rq) { return (rq.L0 + rq.W - 1) / kAttnSpanKeys + 1; }
struct TreeItems {
  int n_kv, hpg, rows;   // rows of a workgroup
  __host__ __device__ int per(const ReqDesc& rq) const { return (hpg * rq.W + rows - 1) / rows; }
  __host__ __device__ int operator()(const ReqDesc& rq) const { return n_kv * per(rq); }
  __host__ __device__ int operator()(const ReqDesc& rq, int r) const { return n_kv * per(rq) * ((tree_spans(rq) + r - 1) / r); }
};

// One item: spans [sp0, sp1) of rq for rows u0 .. of KV head g.
template <int D, int T, bool OP>
__device__ __forceinline__ void tree_run(const AttnArgs& p, const TreeOp* op, TreeLds* tree, const ReqDesc& rq, const AttnRows& rows,
                                         int g, int sp0, int sp1, int j, bool only, unsigned char* smem) {
  constexpr int KS = D / 32, DT = D / 16, U = tree_units<D>(), NV = U / kTreeThreads, KU = D / 4;
  const int tid = threadIdx.x, lane = tid & 63, lg = lane >> 4, lr = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rp = wave & 3, kh = wave >> 2;
  const int last = rq.L0 + rq.W - 1;
  const size_t head = (size_t)rq.slot * p.slot_stride + (size_t)g * p.kv_cap * D;   // float32 units
  const uint4* kb = reinterpret_cast<const uint4*>(p.k_cache + head);
  const uint4* vb = reinterpret_cast<const uint4*>(p.v_cache + head);
  u32x4* L = reinterpret_cast<u32x4*>(smem);   // keys [2][U], values [2][U]
  // Keys: unit u (16 bytes) of key k at u ^ (k % 16), so that the 16 keys a
  // fragment read takes at one u lie in 16 different bank groups.  Values:
  // fragment order (block of 16 dimensions and one part, lane).
  uint4 kr[NV], vr[NV];
  auto request = [&](int step) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      kr[i] = ldg(kb + (size_t)step * U + tid + i * kTreeThreads);
      vr[i] = ldg(vb + (size_t)step * U + (wave * 64 + i * kTreeThreads) + frag_lane_unit(lane));
    }
  };
  auto stage = [&](int step) {
    const int buf = step & 1;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int u = tid + i * kTreeThreads, key = u / KU, ku = u % KU;
      L[buf * U + key * KU + (ku ^ (key & 15))] = __builtin_bit_cast(u32x4, kr[i]);
      // values past the last row (never written, or left by an earlier
      // request) are set to zero: their weight is 0
      const int kc = step * kTreeStep + (i / (NV / 2)) * kAttnChunk;
      if (kc + kAttnChunk > last + 1) {
        const int n0 = min(max(last + 1 - (kc + 4 * lg), 0), 4), n1 = min(max(last + 1 - (kc + 16 + 4 * lg), 0), 4);
        const uint4 a = keep_first<true>(make_uint4(vr[i].x, vr[i].y, 0, 0), n0);
        const uint4 b = keep_first<true>(make_uint4(vr[i].z, vr[i].w, 0, 0), n1);
        vr[i] = make_uint4(a.x, a.y, b.x, b.y);
      }
      L[(2 + buf) * U + u] = __builtin_bit_cast(u32x4, vr[i]);
    }
  };
  const int s0 = sp0 * kTreeStepsPerSpan, s1 = min(sp1 * kTreeStepsPerSpan, last / kTreeStep + 1);
  // (the first step's reads ahead of this, where they do not take the rows: 64
  // us instead of 56 over 32,704 keys, the loop's waits change with it)
  if constexpr (OP)
    if (sp1 * kAttnSpanKeys > rq.L0) tree_put<true, D, kTreeThreads>(p, *op, g, tree);
  request(s0);

  // this lane's rows, one per tile; rows past the group's repeat the last one
  const bool active = rows.u0 + 16 * T * rp < rows.n;
  const auto row_of = [&](int t) { return 16 * (T * rp + t) + lr; };
  Op2 q[T][KS];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int row = rows.row(row_of(t)), h = rows.head(row_of(t));
    if constexpr (OP) {
      typedef uint16_t run __attribute__((ext_vector_type(8), aligned(2)));
      const uint16_t* src = static_cast<const uint16_t*>(op->q.data) + row * op->q.row_stride + h * op->q.head_stride + 8 * lg;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[t][ks].h = __builtin_bit_cast(uint4, *gmem(reinterpret_cast<const run*>(src + 32 * ks)));
    } else {
      const float4* src = reinterpret_cast<const float4*>(p.q + (size_t)(rq.row_start + row) * p.n_q * D + h * D + 8 * lg);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const float4 v[2] = {ldg(src + 8 * ks), ldg(src + 8 * ks + 1)};
        q[t][ks] = split_op<true>(v);
      }
    }
  }
  float M[T], S[T];
  f4 A[T][DT];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    M[t] = -INFINITY;
    S[t] = 0.f;
#pragma unroll
    for (int n = 0; n < DT; ++n) A[t][n] = f4{0.f, 0.f, 0.f, 0.f};
  }

  auto chunk = [&](int step) {
    const int buf = step & 1, kc = step * kTreeStep + kh * kAttnChunk;
    if (!active || kc > last) return;
    f4 sa[T][2];
#pragma unroll
    for (int t = 0; t < T; ++t) sa[t][0] = sa[t][1] = f4{0.f, 0.f, 0.f, 0.f};
    const u32x4* K = L + buf * U + (kh * kAttnChunk + lr) * KU;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const uint4 hi = __builtin_bit_cast(uint4, K[16 * kt * KU + ((4 * ks + lg) ^ lr)]);
        const uint4 lo = __builtin_bit_cast(uint4, K[16 * kt * KU + ((KU / 2 + 4 * ks + lg) ^ lr)]);
#pragma unroll
        for (int t = 0; t < T; ++t) {
          sa[t][kt] = mma_step<true>(hi, q[t][ks].h, sa[t][kt]);
          if constexpr (!OP) sa[t][kt] = mma_step<true>(hi, q[t][ks].l, sa[t][kt]);
          sa[t][kt] = mma_step<true>(lo, q[t][ks].h, sa[t][kt]);
        }
      }
    Op2 pp[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float s[2][4];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kt][i] = sa[t][kt][i] * p.scale;
      if (kc + kAttnChunk > rq.L0) {   // the tree's rows
        asm volatile("");              // a branch: the other chunks do without the masks
        const int row = rows.row(row_of(t));
        const uint32_t mask = OP ? tree->mask[row] : ldg(&p.rows[rq.row_start + row].mask);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!tree_sees(mask, kc + 16 * kt + 4 * lg + i, rq.L0, rq.L0 + row)) s[kt][i] = -INFINITY;
        if constexpr (OP)
          if (mask & tree->bad) S[t] = NAN;
      }
      float mx = s[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e >> 2][e & 3]);
      mx = swap_combine<false>(mx, FMax{});
      mx = swap_combine<true>(mx, FMax{});
      const bool raise = mx > M[t] + kTreeSlack || (M[t] == -INFINITY && mx > -INFINITY);
      if (__ballot(raise)) {
        const float Mn = raise ? mx : M[t], ref = Mn == -INFINITY ? 0.0f : Mn, a = exp2_hw(M[t] - ref);
        S[t] *= a;
#pragma unroll
        for (int n = 0; n < DT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) A[t][n][i] *= a;
        M[t] = Mn;
      }
      const float ref = M[t] == -INFINITY ? 0.0f : M[t];   // no visible key yet: 2^(-inf - 0) = 0
      float pj[2][4];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) pj[kt][i] = exp2_hw(s[kt][i] - ref);
      S[t] += (((pj[0][0] + pj[0][1]) + pj[0][2]) + pj[0][3]) + (((pj[1][0] + pj[1][1]) + pj[1][2]) + pj[1][3]);
      uint32_t hw[4], lw[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // keys 2 (e % 2), 2 (e % 2) + 1 of tile e / 2
        const float v0 = pj[e >> 1][2 * (e & 1)], v1 = pj[e >> 1][2 * (e & 1) + 1];
        hw[e] = f2bf2(v0, v1);
        lw[e] = f2bf2(v0 - bf2f(hw[e]), v1 - __uint_as_float(hw[e] & 0xffff0000u));
      }
      pp[t] = Op2{make_uint4(hw[0], hw[1], hw[2], hw[3]), make_uint4(lw[0], lw[1], lw[2], lw[3])};
    }
    const u32x4* V = L + (2 + buf) * U + kh * (U / 2) + lane;
#pragma unroll
    for (int n = 0; n < DT; ++n) {
      const uint4 hi = __builtin_bit_cast(uint4, V[n * 64]), lo = __builtin_bit_cast(uint4, V[(DT + n) * 64]);
#pragma unroll
      for (int t = 0; t < T; ++t) A[t][n] = mma_step<true>(hi, pp[t].h, A[t][n]);
#pragma unroll
      for (int t = 0; t < T; ++t) A[t][n] = mma_step<true>(lo, pp[t].h, A[t][n]);
#pragma unroll
      for (int t = 0; t < T; ++t) A[t][n] = mma_step<true>(hi, pp[t].l, A[t][n]);
    }
  };
  stage(s0);
  lds_sync();
  for (int s = s0; s < s1; ++s) {
    if (s + 1 < s1) request(s + 1);
    chunk(s);
    if (s + 1 < s1) stage(s + 1);   // its buffer was last read a step ago
    lds_sync();
  }

  // the two halves' states, the second's through LDS [t][M, S, A][row wave][lane]
  f4* X = reinterpret_cast<f4*>(smem) + rp * 64 + lane;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    S[t] = swap_combine<false>(S[t], FAdd{});
    S[t] = swap_combine<true>(S[t], FAdd{});
  }
  if (kh && active) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      X[(t * (DT + 1)) * 256] = f4{M[t], S[t], 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < DT; ++n) X[(t * (DT + 1) + 1 + n) * 256] = A[t][n];
    }
  }
  lds_sync();
  if (!kh && active) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const f4 m = X[(t * (DT + 1)) * 256];
      const float Mn = fmaxf(M[t], m[0]), ref = Mn == -INFINITY ? 0.0f : Mn;
      const float a = exp2_hw(M[t] - ref), c = exp2_hw(m[0] - ref);
      S[t] = S[t] * a + m[1] * c;
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        const f4 x = X[(t * (DT + 1) + 1 + n) * 256];
#pragma unroll
        for (int i = 0; i < 4; ++i) A[t][n][i] = A[t][n][i] * a + x[i] * c;
      }
      if (!rows.valid(row_of(t))) continue;
      const int row = rq.row_start + rows.row(row_of(t)), h = rows.head(row_of(t));
      if (only) {   // one run holds every key
#pragma unroll
        for (int n = 0; n < DT; ++n) {
          const float o[4] = {A[t][n][0] / S[t], A[t][n][1] / S[t], A[t][n][2] / S[t], A[t][n][3] / S[t]};
          attn_store_out<true, D, false, 4>(p, OP ? op : nullptr, row, h * D + 16 * n + 4 * lg, o);
        }
      } else {
        const size_t at = ((size_t)row * p.n_q + h) * p.part_spans + j;
#pragma unroll
        for (int n = 0; n < DT; ++n) *gmem(reinterpret_cast<f4*>(p.pacc + at * D + 16 * n + 4 * lg)) = A[t][n];
        if (lg == 0) *gmem(reinterpret_cast<f2*>(p.pml + at * 2)) = f2{Mn, S[t]};
      }
    }
  }
  lds_sync();   // the next item writes the LDS
}

// Items (run, KV head, row group) of one tree's rows from tensors, a run per
// workgroup.
template <int D, int T>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_op_kernel(const AttnArgs p, const TreeOp op, const int R, const int total) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ TreeLds tree;
  tree_masks_to_lds(op, &tree);
  __syncthreads();
  const ReqDesc rq = tree_req(op);
  const int hpg = p.n_q / p.n_kv, ns = tree_spans(rq), per = TreeItems{p.n_kv, hpg, 64 * T}.per(rq);
  for (int t = xcd_contiguous(blockIdx.x, gridDim.x); t < total; t += gridDim.x) {
    const int j = t / (p.n_kv * per), v = t - j * p.n_kv * per, g = v / per, b = v - g * per;
    const AttnRows rows{g * hpg, rq.W, hpg * rq.W, b * 64 * T};
    tree_run<D, T, true>(p, &op, &tree, rq, rows, g, j * R, min((j + 1) * R, ns), j, R >= ns, smem);
  }
}

// The same of a pass's requests (a fixed grid takes their items in turn, so
// that a captured graph serves any cache length).
template <int D, int T>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_pass_kernel(const AttnArgs p, int n_reqs) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int hpg = p.n_q / p.n_kv;
  const TreeItems items{p.n_kv, hpg, 64 * T};
  int R, total;
  attn_run_length(p.reqs, n_reqs, gridDim.x, items, items, R, total);
  for (int t = xcd_contiguous(blockIdx.x, gridDim.x); t < total; t += gridDim.x) {
    int u = t, r = 0;
    if (n_reqs > 1) r = find_request(p.reqs, n_reqs, u, [&](const ReqDesc& q) { return items(q, R); });
    const ReqDesc rq = load_invariant(p.reqs + r);
    const int n = items.per(rq), ns = tree_spans(rq), j = u / (p.n_kv * n), v = u - j * p.n_kv * n, g = v / n, b = v - g * n;
    const AttnRows rows{g * hpg, rq.W, hpg * rq.W, b * 64 * T};
    tree_run<D, T, false>(p, nullptr, nullptr, rq, rows, g, j * R, min((j + 1) * R, ns), j, R >= ns, smem);
  }
}

// The runs' states of a row and head joined in order, one wave each.
template <int D>
__global__ __launch_bounds__(64) void tree_op_join_kernel(const AttnArgs p, const TreeOp op, const int runs) {
  const int i = blockIdx.x / p.n_q;
  attn_merge_wave<true, D>(p, tree_req(op), i, blockIdx.x - i * p.n_q, &op, runs);
}
template <int D>
__global__ __launch_bounds__(64) void tree_pass_join_kernel(const AttnArgs p, int n_reqs, int T, int G) {
  int u = blockIdx.x, r = 0, R, total;
  const TreeItems items{p.n_kv, p.n_q / p.n_kv, 64 * T};
  attn_run_length(p.reqs, n_reqs, G, items, items, R, total);
  if (n_reqs > 1) r = find_request(p.reqs, n_reqs, u, [&](const ReqDesc& q) { return q.W * p.n_q; });
  if (r < 0) return;
  const ReqDesc rq = load_invariant(p.reqs + r);
  if (u >= rq.W * p.n_q) return;
  const int ns = tree_spans(rq), i = u / p.n_q;
  if (R < ns) attn_merge_wave<true, D>(p, rq, i, u - i * p.n_q, nullptr, (ns + R - 1) / R);
}

template <int D, int T> static hipError_t tree_op(const AttnArgs& a, const TreeOp& op, int G, hipStream_t s) {
  const TreeItems items{a.n_kv, a.n_q / a.n_kv, 64 * T};
  int R, total;
  run_length_of(tree_req(op), G, items, items, R, total);
  tree_op_kernel<D, T><<<std::min(G, total), kTreeThreads, tree_lds_bytes<D>(), s>>>(a, op, R, total);
  const hipError_t e = hipGetLastError();
  const int runs = (tree_spans(tree_req(op)) + R - 1) / R;
  if (e != hipSuccess || runs == 1) return e;
  tree_op_join_kernel<D><<<op.W * a.n_q, 64, 0, s>>>(a, op, runs);
  return hipGetLastError();
}
template <int D, int T> static hipError_t tree_pass(const AttnArgs& a, int n_reqs, int G, hipStream_t s) {
  tree_pass_kernel<D, T><<<G, kTreeThreads, tree_lds_bytes<D>(), s>>>(a, n_reqs);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  tree_pass_join_kernel<D><<<a.M * a.n_q, 64, 0, s>>>(a, n_reqs, T, G);
  return hipGetLastError();
}

// a.wave_tiles: row tiles a wave.
hipError_t launch_tree_op(const AttnArgs& a, const TreeOp& op, int grid, hipStream_t s) {
  if (op.W < 1 || op.W > 32 || grid < 1) return hipErrorInvalidValue;
  const bool two = a.wave_tiles == 2;
  if (a.head_dim == 128) return two ? tree_op<128, 2>(a, op, grid, s) : tree_op<128, 1>(a, op, grid, s);
  if (a.head_dim == 64) return two ? tree_op<64, 2>(a, op, grid, s) : tree_op<64, 1>(a, op, grid, s);
  return hipErrorInvalidValue;
}
hipError_t launch_tree_pass(const AttnArgs& a, int n_reqs, int grid, hipStream_t s) {
  if (n_reqs < 1 || grid < 1) return hipErrorInvalidValue;
  const bool two = a.wave_tiles == 2;
  if (a.head_dim == 128) return two ? tree_pass<128, 2>(a, n_reqs, grid, s) : tree_pass<128, 1>(a, n_reqs, grid, s);
  if (a.head_dim == 64) return two ? tree_pass<64, 2>(a, n_reqs, grid, s) : tree_pass<64, 1>(a, n_reqs, grid, s);
  return hipErrorInvalidValue;
}

hipError_t prepare_tree() {
  hipError_t e = hipSuccess;
  const auto allow = [&](const void* k) {
    if (e == hipSuccess) e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, tree_lds_bytes<128>());
  };
  allow(reinterpret_cast<const void*>(&tree_op_kernel<64, 1>));   // 64 KiB, and the masks
  allow(reinterpret_cast<const void*>(&tree_op_kernel<64, 2>));
  allow(reinterpret_cast<const void*>(&tree_op_kernel<128, 1>));
  allow(reinterpret_cast<const void*>(&tree_op_kernel<128, 2>));
  allow(reinterpret_cast<const void*>(&tree_pass_kernel<128, 1>));
  allow(reinterpret_cast<const void*>(&tree_pass_kernel<128, 2>));
  return e;
}

}  // namespace as2d
