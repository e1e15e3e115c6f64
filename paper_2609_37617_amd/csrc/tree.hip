// Passes over trees of candidates: greedy verification along a tree and the
// accepted path's cache rows moved together; rows from device tensors into a
// cache layer.
//
// Row i of a request sits in cache row L0 + i and sees the committed keys and
// the rows in its mask (attn.h); its rotary position is L0 and its depth.
// After a pass the rows of the accepted path, at rising cache rows, become
// the rows L0 + 1, L0 + 2, ..: what as many chain steps would have appended.
#include "common.h"

namespace as2d {

// ---------------------------------------------------------------------------
// Keys and values [n][n_kv][D] of any strides into cache rows pos0 .. of a
// layer (layout: kernels.h), one workgroup per row.

template <bool SRC16> __device__ __forceinline__ float src_value(const void* p, long long i) {
  if constexpr (SRC16) return bf2f(ldg(static_cast<const uint16_t*>(p) + i));
  else return ldg(static_cast<const float*>(p) + i);
}

template <bool BF, bool SRC16>
__global__ __launch_bounds__(256) void put_rows_kernel(const PutRows a) {
  const int r = blockIdx.x, D = a.head_dim, pos = a.pos0 + r;
  const size_t base = (size_t)a.slot * a.slot_stride;
  for (int i = threadIdx.x; i < a.n_kv * D; i += 256) {
    const int g = i / D, dd = i - g * D;
    const float k = src_value<SRC16>(a.k.data, r * a.k.row_stride + g * a.k.head_stride + dd);
    const float v = src_value<SRC16>(a.v.data, r * a.v.row_stride + g * a.v.head_stride + dd);
    float* kb = a.k_cache + base + (size_t)g * a.kv_cap * D;
    float* vb = a.v_cache + base + (size_t)g * a.kv_cap * D;
    if constexpr (BF) {
      uint16_t* k16 = reinterpret_cast<uint16_t*>(kb) + (size_t)pos * 2 * D + dd;
      uint16_t* v16 = reinterpret_cast<uint16_t*>(vb);
      const BfPair hk = split_val(k), hv = split_val(v);
      *gmem(k16) = hk.hi;
      *gmem(k16 + D) = hk.lo;
      *gmem(v16 + v_elem(pos, 0, dd, D, true)) = hv.hi;
      *gmem(v16 + v_elem(pos, 1, dd, D, true)) = hv.lo;
    } else {
      *gmem(kb + (size_t)pos * D + dd) = k;
      *gmem(vb + v_elem(pos, 0, dd, D, false)) = v;
    }
  }
}

hipError_t launch_put_rows(bool bf16, bool src_bf16, const PutRows& a, int n, hipStream_t s) {
  if (n < 1) return hipErrorInvalidValue;
  if (bf16 && src_bf16) put_rows_kernel<true, true><<<n, 256, 0, s>>>(a);
  else if (bf16) put_rows_kernel<true, false><<<n, 256, 0, s>>>(a);
  else if (src_bf16) put_rows_kernel<false, true><<<n, 256, 0, s>>>(a);
  else put_rows_kernel<false, false><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Greedy verification along a tree, one wave per request, from the rows'
// greedy tokens (finish_kernel, earlier in the pass): from the root, the
// lowest-numbered child whose candidate is its node's greedy token, as long
// as there is one; the token after the path is the greedy token of its last
// row.  A request with a non-finite logit accepts nothing (-1) and the move
// below leaves its cache as it is.

__global__ __launch_bounds__(64) void tree_walk_kernel(const RowDesc* __restrict__ rows, const ReqDesc* __restrict__ reqs,
                                                       const int* __restrict__ row_tok, const int* __restrict__ row_bad,
                                                       const TreeOut out) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const ReqDesc rq = load_invariant(reqs + r);
  const bool row = lane < rq.W;
  const int at = rq.row_start + (row ? lane : 0);
  const int tok = row_tok[at], cand = rows[at].token;
  const uint32_t mask = rows[at].mask;
  const int parent = row && lane > 0 ? parent_row(mask, lane) : -1;
  const bool bad = __ballot(row && row_bad[at]) != 0;
  int cur = 0, a = 0;
  if (!bad)
    for (;;) {
      const int want = __shfl(tok, cur);   // every lane takes part
      const uint64_t next = __ballot(parent == cur && cand == want);
      if (!next) break;
      cur = __ffsll((unsigned long long)next) - 1;   // a child's row is past its parent's: the walk ends
      if (lane == 0) {
        out.path[rq.row_start + a] = cur - 1;
        out.host_path[rq.row_start + a] = cur - 1;
      }
      ++a;
    }
  const int next_tok = __shfl(tok, cur);
  if (lane == 0) {
    const StepOut o{bad ? -1 : a, next_tok, bad, 0};
    out.sel[r] = o;
    out.host[r] = o;
  }
}

hipError_t launch_tree_walk(const RowDesc* rows, const ReqDesc* reqs, int n_reqs, const int* row_tok, const int* row_bad,
                            const TreeOut& out, hipStream_t s) {
  tree_walk_kernel<<<n_reqs, 64, 0, s>>>(rows, reqs, row_tok, row_bad, out);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The accepted path's cache rows, moved down to follow the root's.  One
// workgroup per (layer, KV head) and request; a thread moves one 16-byte unit
// of the key rows and one element of the value rows for every row of the
// path, in order: path[j] >= j, so a row is read before any later one lands
// on it, and no other thread touches the thread's columns.

template <bool BF>
__global__ __launch_bounds__(256) void move_path_kernel(const MovePath a) {
  using T = typename ET<BF>::T;
  constexpr int kB = 8;   // rows whose reads are in flight together
  const int r = blockIdx.y, D = a.head_dim, tid = threadIdx.x;
  const ReqDesc rq = load_invariant(a.reqs + r);
  const int n = a.sel[r].accepted;
  if (n < 1) return;
  const int* path = a.path + rq.row_start;
  if (path[n - 1] == n - 1) return;   // rising: the first n candidates, in place already
  const int l = blockIdx.x / a.n_kv, g = blockIdx.x - l * a.n_kv;
  const size_t head = (size_t)rq.slot * a.slot_stride + (size_t)l * a.layer_stride + (size_t)g * a.kv_cap * D;
  const int units = D * 4 / 16, vals = BF ? 2 * D : D;
  const int part = tid / D, dd = tid - part * D;
  uint4* kb = reinterpret_cast<uint4*>(a.k_cache + head);
  T* vb = reinterpret_cast<T*>(a.v_cache + head);
  for (int j0 = 0; j0 < n; j0 += kB) {
    uint4 k[kB];
    T v[kB];
    int src[kB];
#pragma unroll
    for (int j = 0; j < kB; ++j) {
      src[j] = rq.L0 + 1 + path[min(j0 + j, n - 1)];
      if (tid < units) k[j] = ldg(kb + (size_t)src[j] * units + tid);
      if (tid < vals) v[j] = ldg(vb + v_elem(src[j], part, dd, D, BF));
    }
#pragma unroll
    for (int j = 0; j < kB; ++j) {
      const int dst = rq.L0 + 1 + j0 + j;
      if (j0 + j >= n || dst == src[j]) continue;
      if (tid < units) *gmem(reinterpret_cast<u32x4*>(kb + (size_t)dst * units + tid)) = u32x4{k[j].x, k[j].y, k[j].z, k[j].w};
      if (tid < vals) *gmem(vb + v_elem(dst, part, dd, D, BF)) = v[j];
    }
  }
}

hipError_t launch_move_path(bool bf16, const MovePath& a, int n_layers, int n_reqs, hipStream_t s) {
  if (a.head_dim != 64 && a.head_dim != 128) return hipErrorInvalidValue;
  const dim3 grid(n_layers * a.n_kv, n_reqs);
  if (bf16) move_path_kernel<true><<<grid, 256, 0, s>>>(a);
  else move_path_kernel<false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace as2d
