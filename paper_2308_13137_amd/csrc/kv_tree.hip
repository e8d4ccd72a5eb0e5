// A tree of drafted tokens over the paged 8-bit cache: its rows into the windows,
// attention of every node over the sequence and its own ancestors, and the accepted
// path kept.
//
// A sequence of L tokens whose tree has n nodes holds node j's key and value in row
// L + j of its window: no page is closed by drafts (a full page's codes share one step,
// so rejected tokens would change what the others stand for), and a tree of at most a
// page's tokens lies in the two pages that a window holds.  RoPE turns node j by
// L + its depth, so an accepted path only has to be moved together: its rows are then
// bit for bit those of its tokens appended one after another, and so are the codes of
// a page that they fill.
#include "kv_cache.h"

namespace oq {
namespace {

// ------------------------------------------------------------------ append
// One workgroup takes one sequence's tree: the keys and values of one head
// (blockIdx.y < kv heads), or a slice of the queries.
template <typename TI>
__global__ __launch_bounds__(256) void tree_append_kernel(CacheArgs c, RowIn<TI> in, int H,
                                                         const float* __restrict__ rope, int64_t n_rope,
                                                         const float* __restrict__ sa, uint16_t* __restrict__ Qout) {
  __shared__ uint32_t s_anc[TREE_MAX][4];
  __shared__ int s_up[TREE_MAX];
  const int i = blockIdx.x, u = blockIdx.y, tid = threadIdx.x, d = c.d, half = d / 2, P = c.P;
  const Seq s = seq_of(c, i);
  if (s.n == 0) return;
  const int slice = u - c.Hkv, slices = int(gridDim.y) - c.Hkv;
  const bool good = tree_ancestors(c.parent, s, s_anc, s_up);
  if (!good || !s.ok) {                                    // nothing is cached; the queries are NaN
    if (slice < 0) return;
    const int64_t wide = int64_t(H) * d;
    for (int64_t e = tid + 256 * int64_t(slice); e < s.n * wide; e += 256 * int64_t(slices))
      Qout[int64_t(s.b) * wide + e] = 0x7fc0;
    return;
  }
  // a node's depth is the number of its ancestors
  if (tid < s.n) s_up[tid] = s.L + __popc(s_anc[tid][0]) + __popc(s_anc[tid][1]) + __popc(s_anc[tid][2]) + __popc(s_anc[tid][3]) - 1;
  __syncthreads();
  if (slice >= 0) {
    append_queries(c, s, in, H, rope, n_rope, sa, Qout, s.L, s.L + s.n, slice, slices,
                   [&](int pos) { return s_up[pos - s.L]; });
    return;
  }
  const int64_t win = int64_t(P) * d;
  auto window = [&](uint16_t* w, int pos) {
    return w + ((int64_t(s.slot) * 2 + ((pos >> c.lgP) & 1)) * c.Hkv + u) * win;
  };
  const int lq = c.lgd - 3, q4 = 1 << lq;
  for (int e = tid; e < s.n * q4; e += 256) {
    const int j = e >> lq, p = 4 * (e & (q4 - 1)), pos = s.L + j;
    float x[4], y[4];
    turned4(in.k + (int64_t(s.b) + j) * in.ldk + int64_t(u) * d, rope, n_rope, s_up[j], p, half, x, y);
    if (sa) {
      float s0[4], s1[4];
      load4(sa + u * d + p, s0);
      load4(sa + u * d + p + half, s1);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = x[k] * s0[k];
        y[k] = y[k] * s1[k];
      }
    }
    uint16_t* kw = window(c.kw, pos) + (pos & (P - 1)) * d + p;
    *reinterpret_cast<uint2*>(kw) = pack4(x);
    *reinterpret_cast<uint2*>(kw + half) = pack4(y);
  }
  // values: four channels of four tokens that lie together in the operand order
  const int lv = c.lgd - 2, t0 = s.L & ~3, end = s.L + s.n;
  for (int e = tid; e < ((end - t0 + 3) >> 2) << lv; e += 256) {
    const int t = t0 + 4 * (e >> lv), p = 4 * (e & ((1 << lv) - 1));
    uint2 row[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = min(max(t + k - s.L, 0), s.n - 1);     // (outside the tree: not stored)
      float x[4];
      load4(in.v + (int64_t(s.b) + j) * in.ldv + int64_t(u) * d + p, x);
      row[k] = pack4(x);
    }
    uint16_t* vw = window(c.vw, t);
#pragma unroll
    for (int ch = 0; ch < 4; ++ch) {
      uint32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = ((ch < 2 ? row[k].x : row[k].y) >> (16 * (ch & 1))) & 0xffffu;
      uint16_t* dst = vw + vw_at(t & (P - 1), p + ch, d);
      if (t >= s.L && t + 4 <= end) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (t + k >= s.L && t + k < end) dst[k] = uint16_t(v[k]);
      }
    }
  }
}

// ------------------------------------------------------------------ commit
// One workgroup: one head of one sequence.  The path's rows go through LDS, since a row
// is written where another one is read; then the page that they fill, if any (a tree
// of at most a page's tokens fills no second one), becomes codes.
__global__ __launch_bounds__(256) void tree_commit_kernel(CacheArgs c, const int32_t* __restrict__ path, int max_path,
                                                         const int32_t* __restrict__ count) {
  extern __shared__ uint4 s_page[];                        // K [P][d], then V, bf16
  __shared__ int s_max[2][8];
  __shared__ int s_path[TREE_MAX];
  const int i = blockIdx.x, u = blockIdx.y, tid = threadIdx.x, d = c.d, P = c.P;
  const Seq s = seq_of(c, i);
  const int n = count[i];
  if (!s.ok || n <= 0 || n > min(s.n, max_path)) return;
  bool fine = true;
  if (tid < n) {
    const int32_t* p = path + int64_t(i) * max_path;
    const int at = p[tid];
    s_path[tid] = at;
    fine = at < s.n && (tid == 0 ? at >= 0 : at > p[tid - 1]);
  }
  if (!__syncthreads_and(fine)) return;
  const int64_t win = int64_t(P) * d;
  auto window = [&](uint16_t* w, int pos) {
    return w + ((int64_t(s.slot) * 2 + ((pos >> c.lgP) & 1)) * c.Hkv + u) * win;
  };
  // (a path's first nodes may stand where they belong; from the first that does not on,
  // every one is to be moved)
  uint16_t* sk = reinterpret_cast<uint16_t*>(s_page);
  uint16_t* sv = sk + P * d;
  const int lk = c.lgd - 3;
  for (int e = tid; e < n << lk; e += 256) {
    const int k = e >> lk, pos = s.L + s_path[k];
    if (s_path[k] != k)
      s_page[e] = *reinterpret_cast<const uint4*>(window(c.kw, pos) + (pos & (P - 1)) * d + 8 * (e & ((1 << lk) - 1)));
  }
  for (int e = tid; e < n << c.lgd; e += 256) {
    const int k = e >> c.lgd, pos = s.L + s_path[k];
    if (s_path[k] != k) sv[e] = window(c.vw, pos)[vw_at(pos & (P - 1), e & (d - 1), d)];
  }
  __syncthreads();
  for (int e = tid; e < n << lk; e += 256) {
    const int k = e >> lk, pos = s.L + k;
    if (s_path[k] != k)
      *reinterpret_cast<uint4*>(window(c.kw, pos) + (pos & (P - 1)) * d + 8 * (e & ((1 << lk) - 1))) = s_page[e];
  }
  for (int e = tid; e < n << c.lgd; e += 256) {
    const int k = e >> c.lgd, pos = s.L + k;
    if (s_path[k] != k) window(c.vw, pos)[vw_at(pos & (P - 1), e & (d - 1), d)] = sv[e];
  }
  if ((s.L & (P - 1)) + n < P) return;
  __syncthreads();
  const uint4* kw = reinterpret_cast<const uint4*>(window(c.kw, s.L));
  const uint4* vw = reinterpret_cast<const uint4*>(window(c.vw, s.L));
  for (int e = tid; e < P * d / 8; e += 256) {
    s_page[e] = kw[e];
    s_page[P * d / 8 + e] = vw[e];
  }
  __syncthreads();
  page_to_codes(c, i, s.L >> c.lgP, u, s_page, s_max);
}

}  // namespace

hipError_t cache_append_tree(const CacheArgs& c, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                             const void* V, int64_t ldv, bool in_bf16, int H, const float* rope, int64_t n_rope,
                             const float* s_a, uint16_t* Qout, hipStream_t st) {
  // query slices: eight items of a thread each
  const int64_t items = int64_t(c.max_q) * H * (c.d / 8);
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(items / (8 * 256), 65535 - c.Hkv));
  const dim3 grid(unsigned(c.n_seq), unsigned(c.Hkv + slices));
  auto go = [&](auto ti) {
    using TI = decltype(ti);
    const RowIn<TI> in{static_cast<const TI*>(Q), static_cast<const TI*>(K), static_cast<const TI*>(V), ldq, ldk, ldv};
    hipLaunchKernelGGL(tree_append_kernel<TI>, grid, dim3(256), 0, st, c, in, H, rope, n_rope, s_a, Qout);
  };
  if (in_bf16) go(uint16_t{});
  else go(float{});
  return hipGetLastError();
}

hipError_t cache_attend_tree(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                             float* ws, const AttendPlan& p, hipStream_t st) {
  return attend_launch<true>(c, Q, ldq, H, O, LSE, ws, p, st);
}

hipError_t cache_commit(const CacheArgs& c, const int32_t* path, int max_path, const int32_t* count, hipStream_t st) {
  const dim3 grid(unsigned(c.n_seq), unsigned(c.Hkv));
  hipLaunchKernelGGL(tree_commit_kernel, grid, dim3(256), unsigned(c.P) * c.d * 4, st, c, path, max_path, count);
  return hipGetLastError();
}

}  // namespace oq
