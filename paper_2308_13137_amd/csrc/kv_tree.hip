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

// A tree of drafted tokens: node j of a sequence's new tokens stands behind the sequence
// (parent -1) or behind an earlier node.  It sees the sequence's tokens and its own
// ancestors, itself counted: a bit each, TREE_MAX nodes at most.
constexpr int TREE_MAX = 128;
// Every node's ancestors, by one wave in registers: lane j has nodes j and 64 + j.  Each round
// doubles the part of its way that a node knows.
struct Ancestors {
  uint64_t low, high[2];                 // of node `lane`, of node 64 + `lane`
  bool ok;                               // every parent is an earlier node or none
  OQ_DEV Ancestors(const int32_t* parent, const Seq& s) {
    const int lane = threadIdx.x & 63;
    const int32_t* p = parent + s.b;
    int up = lane < s.n ? p[lane] : -1, far = lane + 64 < s.n ? p[lane + 64] : -1;
    ok = !__any(up < -1 || up >= lane + (up < 0) || far < -1 || far >= lane + 64);
    if (!ok) up = far = -1;
    low = high[1] = uint64_t(1) << lane;
    high[0] = 0;
    while (__any(up >= 0 || far >= 0)) {
      const int a = max(up, 0), b = max(far, 0) & 63;
      const uint64_t m = __shfl(low, a);
      const int next = __shfl(up, a);
      if (s.n > 64) {
        const uint64_t l0 = __shfl(low, b), h0 = __shfl(high[0], b), h1 = __shfl(high[1], b);
        const int n0 = __shfl(up, b), n1 = __shfl(far, b);
        if (far >= 64) {
          high[0] |= h0;
          high[1] |= h1;
          far = n1;
        } else if (far >= 0) {
          high[0] |= l0;
          far = n0;
        }
      }
      if (up >= 0) {
        low |= m;
        up = next;
      }
    }
  }
};
// The same in LDS, by the whole workgroup; a barrier is the caller's.  False where a parent
// is none.
OQ_DEV bool tree_ancestors(const int32_t* parent, const Seq& s, uint32_t (*s_anc)[4]) {
  const Ancestors a(parent, s);
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    reinterpret_cast<uint4*>(s_anc)[lane] = make_uint4(uint32_t(a.low), uint32_t(a.low >> 32), 0u, 0u);
    reinterpret_cast<uint4*>(s_anc)[lane + 64] = make_uint4(uint32_t(a.high[0]), uint32_t(a.high[0] >> 32),
                                                            uint32_t(a.high[1]), uint32_t(a.high[1] >> 32));
  }
  return a.ok;
}
// Which of the 32 tokens from t0 on a node sees: the sequence's L, its ancestors behind them.
OQ_DEV uint32_t tree_sees(const uint32_t (*s_anc)[4], int node, int L, int t0) {
  const int o = t0 - L, w = o >> 5;
  const uint32_t lo = unsigned(w) < 4u ? s_anc[node][w] : 0u, hi = unsigned(w + 1) < 4u ? s_anc[node][w + 1] : 0u;
  const uint32_t kin = uint32_t(((uint64_t(hi) << 32) | lo) >> (o & 31));
  return kin | (o >= 0 ? 0u : o <= -32 ? ~0u : (1u << -o) - 1u);
}

// ------------------------------------------------------------------ append
// One workgroup takes one sequence's tree: the keys and values of one head
// (blockIdx.y < kv heads), or a slice of the queries.  Large batches are bound by HBM (64 trees of up
// to 64 nodes, 64 heads, float32, 137 MB: 38 us, 3.6 TB/s, of which reading the rotation, again for
// every head, is 3; 27 us with inputs that the last-level cache holds), few rows by a chain of three
// loads (five nodes, 32 heads, 5.2 us; with a barrier for each round of the ancestors' search 10.8).
template <typename TI>
__global__ __launch_bounds__(256) void tree_append_kernel(CacheArgs c, RowIn<TI> in, int H,
                                                         const float* __restrict__ rope, int64_t n_rope,
                                                         const float* __restrict__ sa, uint16_t* __restrict__ Qout) {
  __shared__ int s_pos[TREE_MAX];                          // where RoPE has a node: a position per ancestor
  const int i = blockIdx.x, u = blockIdx.y, tid = threadIdx.x, d = c.d, half = d / 2, P = c.P;
  const Seq s = seq_of(c, i);
  if (s.n == 0) return;
  const int slice = u - c.Hkv, slices = int(gridDim.y) - c.Hkv;
  const Ancestors anc(c.parent, s);
  if (!anc.ok || !s.ok) {                                    // nothing is cached; the queries are NaN
    if (slice < 0) return;
    const int64_t wide = int64_t(H) * d;
    for (int64_t e = tid + 256 * int64_t(slice); e < s.n * wide; e += 256 * int64_t(slices))
      Qout[int64_t(s.b) * wide + e] = 0x7fc0;
    return;
  }
  if (tid < 64) {
    s_pos[tid] = s.L + __popcll(anc.low) - 1;
    s_pos[tid + 64] = s.L + __popcll(anc.high[0]) + __popcll(anc.high[1]) - 1;
  }
  __syncthreads();
  if (slice >= 0) {
    append_queries(c, s, in, H, rope, n_rope, sa, Qout, s.L, s.L + s.n, slice, slices,
                   [&](int pos) { return s_pos[pos - s.L]; });
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
    turned4(in.k + (int64_t(s.b) + j) * in.ldk + int64_t(u) * d, rope, n_rope, s_pos[j], p, half, x, y);
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
// of at most a page's tokens fills no second one), becomes codes.  Bound by its chain of loads: four
// heads' or 64 sequences' 6.7 and 9.4 us.
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
  // (a path's first nodes may stand where they belong)
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

// ------------------------------------------------------------------ attention
// A chunk of 32 tokens against a row tile of 16 R rows costs the codes' way to the registers and
// their widening, which any number of rows shares, and each 16 rows' products and softmax: 8, 32
// and 64 rows a key head over 131,072 tokens, 8 key heads of 128, took 55, 59 and 79 us (4.8, 4.5
// and 3.4 TB/s with all of a call; the chunks alone run at 6.2, 5.9 and 4.5), 512 rows over 131,072
// tokens, whose codes come from the caches, 400 (690 TFLOP/s).  With 64 rows a wave's own chain
// of reads, products, softmax and products bounds a chunk (3 us, two waves to a SIMD): exponentials left out
// would save 3%, codes out of the L2 6 to 17%.
OQ_DEV int tile_cost(int rows) { return rows <= 16 ? 3 : rows <= 32 ? 4 : 6; }
constexpr int TILE_ROWS = 64;
// What a tile costs more than its chunks, in chunks: some 3 us before the first one (the search on
// the line, page numbers, queries), 1 to 3 after the last, 4 to 6 for the window.  In a graph 32 trees of
// up to 16 and of up to 8 nodes over up to 4,096 tokens, 64 heads, 8 key heads, took 75 and 59 us with 8, 69
// and 54 with 16, 76 and 53 with 24, 79 and 57 with 32; without it workgroups ended after 46 to 83 us.
constexpr int TILE_MORE = 16;

// What a workgroup's share of the line of all tiles' chunks is made of: row tile `row0` of
// sequence s, chunks c0 .. c1 - 1.
struct Piece {
  int row0, rows, c0, c1;
};

template <int DH, int RMAX>
struct Shared {
  static constexpr int KS = DH / 32, JD = DH / 16;
  union {
    // the queries as operands, f16 (scaled) for codes, bf16 for the window
    struct {
      u32x4_t h[RMAX * KS * 64], b[RMAX * KS * 64];
    } q;
    f32x4_t o[4][RMAX * JD / 2][64];     // half of the waves' results
  };
  float2 ml[4][16 * RMAX], all[16 * RMAX];
  float qs[16 * RMAX];                   // what a row's f16 queries are in units of
  int4 line[4][64];                      // a wave's own: 64 sequences of the batch
  uint32_t anc[TREE_MAX][4];
};

// Bits 15 and 31: whether one of eight bf16 values has the largest exponent.
OQ_DEV unsigned not_finite(u32x4_t w) {
  unsigned x = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) x |= (w[i] & 0x7fff7fffu) + 0x00800080u;
  return x;
}

// One piece: the chunks are dealt to the four waves, each with all rows and a softmax of its
// own; codes go from memory straight into operand registers (ONCE: sequences of one tile, whose
// codes nobody else reads, go past the caches).  Joined in LDS, the result goes to the output or
// to a slot of the workspace.
//   S^T = K Q^T: a lane holds query row r, tokens 4 g + 0..3 of both 16-token
//   tiles, which is the B operand of O^T = V^T P^T as it stands.
template <int DH, int R, bool ONCE, int RMAX>
OQ_DEV void attend_piece(const CacheArgs& c, const Seq& s, const Piece& pc, int i, int u, int G, const uint16_t* Q,
                         int64_t ldq, const Out& out, Shared<DH, RMAX>& sh) {
  constexpr int KS = DH / 32, JD = DH / 16;
  // (a thread's place is read anew here, before the window and before the join: addresses made from it
  // would be kept in registers over the loops that need all of them)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  int lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int P = c.P, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto anew = [&] {
    tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    lane = tid & 63;
    r = lane & 15;
    g = lane >> 4;
  };
  const int total = s.ok ? s.L + s.n : 0, closed = (s.ok ? s.L : 0) & ~(P - 1);
  const int ncode = closed / 32, last = min(pc.c1, (total + 31) / 32), cend = min(last, ncode);
  const float sc = 1.4426950408889634f / sqrtf(float(DH));
  auto row_of = [&](int h) { return pc.row0 + min(16 * h + r, pc.rows - 1); };
  int ch = pc.c0 + wave;

  // (page numbers and steps by vector loads, though the whole wave reads one word: scalar ones share
  // a counter with the LDS reads, whose waits would then last until memory has answered)
  auto word = [&](const auto* p) {
    uint32_t zero = 0;
    asm volatile("" : "+v"(zero));
    return *reinterpret_cast<decltype(p)>(reinterpret_cast<const char*>(p) + zero);
  };
  // (the piece's chunks of full pages; none: not called)
  auto entry_of = [&](int ch) { return word(c.table + int64_t(i) * c.max_pages + ((32 * ch) >> c.lgP)); };
  u32x4_t kr[KS], vr[KS];
  float ks = 0.0f, vs = 0.0f;
  auto take = [&](const int8_t* p, int64_t at, u32x4_t (&x)[KS]) {
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + at) + lane;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      if constexpr (ONCE) x[j] = __builtin_nontemporal_load(q + 64 * j);
      else x[j] = q[64 * j];
    }
  };
  int64_t at = 0;                        // of the chunk's codes, in both tensors
  int page = -1, tin = 32 * ch & (P - 1);
  auto take_keys = [&] {
    const int id = page_in(c, __builtin_amdgcn_readfirstlane(page));
    const int64_t blk = int64_t(max(id, 0)) * c.Hkv + u;
    at = blk * P * DH + tin * DH;
    ks = word(c.ks + blk);
    vs = word(c.vs + blk);
    if (id < 0) vs = NAN;
    take(c.kc, at, kr);
  };
  // What a piece begins with is under way together: page numbers, queries, the first codes,
  // the tree.
  int entry_next = 0;
  if (ch < cend) {
    page = entry_of(ch);
    entry_next = entry_of(min(ch + 4, cend - 1));
  }
  u32x4_t q_in[KS];
  if (wave < R) {
    bf16x8_t qf[KS];
    load_q<DH>(qf, Q, ldq, s, u, G, row_of(wave), g);
#pragma unroll
    for (int k = 0; k < KS; ++k) q_in[k] = __builtin_bit_cast(u32x4_t, qf[k]);
  }
  if (ch < cend) {
    // (in the order of the loop's loads: its waits hold for both)
    __builtin_amdgcn_sched_barrier(0);
    take_keys();
    __builtin_amdgcn_sched_barrier(0);
    take(c.vc, at, vr);
    __builtin_amdgcn_sched_barrier(0);
  }
  bool tree_ok = true;
  if (last > ncode) tree_ok = tree_ancestors(c.parent, s, sh.anc);
  // the queries as f16 times a power of two that puts the row's largest entry between 2^14 and 2^15
  if (wave < R) {
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = fmaxf(top, fmaxf(fabsf(__uint_as_float(q_in[k][e] << 16)), fabsf(__uint_as_float(q_in[k][e] & 0xffff0000u))));
    const int e = min(max(int(__float_as_uint(row_max(top)) >> 23), 56), 253);
    const float up = __uint_as_float(uint32_t(268 - e) << 23);   // 2^(14 - exponent)
    if (g == 0) sh.qs[16 * wave + r] = __uint_as_float(uint32_t(e - 14) << 23);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4_t w;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = pack_f16(__uint_as_float(q_in[k][q] << 16) * up, __uint_as_float(q_in[k][q] & 0xffff0000u) * up);
      sh.q.h[(wave * KS + k) * 64 + lane] = w;
      sh.q.b[(wave * KS + k) * 64 + lane] = q_in[k];
    }
  }
  f32x4_t acc[R][JD];
  float m[R], l[R], vref = VREF0;
  auto nothing = [&](int h) {
    m[h] = -INFINITY;
    l[h] = 0.0f;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  };
  __syncthreads();
  // The window first, while few registers are in use: wave w takes row tile w mod R, and where there are
  // fewer tiles than waves, they share its chunks.  (Its code is run a few times a piece and comes from
  // memory as it runs: with all rows in every wave, four times the code, a chunk took 8 us.)
  const int tile = wave % R;
  int wch = max(pc.c0, ncode) + wave / R;
  if (wch < last) {
    f32x4_t a1[JD];
    float m1 = -INFINITY, l1 = 0.0f;
#pragma unroll
    for (int j = 0; j < JD; ++j) a1[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const Step sp[1] = {step_of(step_parts(sc, 1.0f), 1.0f, false)};   // its step is 1
    const int node = row_of(tile) / G;
#pragma unroll 1
    for (; wch < last; wch += 4 / R) {
      const int t0 = 32 * wch;
      const Window<DH> win(c, s, u, t0, total, lane);
      unsigned bad = 0;
      u32x4_t kw[2][KS], vw[JD];
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int k = 0; k < KS; ++k) kw[a][k] = win.key(a, k);
      auto values = [&] {
#pragma unroll
        for (int j = 0; j < JD; ++j) vw[j] = win.value(j);
      };
      if constexpr (RMAX > 1) values();
      unsigned odd = 0;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int k = 0; k < KS; ++k) odd |= not_finite(kw[a][k]);
      if (__any(odd & 0x80008000u)) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int k = 0; k < KS; ++k) win.check_key(kw[a][k], a, bad);
      }
      f32x4_t st[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8_t qf = __builtin_bit_cast(bf16x8_t, sh.q.b[(tile * KS + k) * 64 + lane]);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          st[a] = mfma(__builtin_bit_cast(bf16x8_t, kw[a][k]), qf, st[a]);
        }
      }
      if constexpr (RMAX == 1) {                         // (three waves' registers: where the keys were)
        __builtin_amdgcn_sched_barrier(0);
        values();
      }
      const uint32_t sees = tree_sees(sh.anc, node, s.L, t0);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (!((sees >> (4 * g)) & (1u << (16 * a + q)))) st[a][q] = -INFINITY;
      const float alpha = softmax_step<1>(st, sp, m1, l1);
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int j = 0; j < JD; ++j) a1[j] = a1[j] * alpha;
      }
      // (rows behind the sequence's end too are whatever the window holds: their weights are zeros, and
      // zero times a value that is finite is one)
      odd = 0;
#pragma unroll
      for (int j = 0; j < JD; ++j) odd |= not_finite(vw[j]);
      if (__any(odd & 0x80008000u)) {
#pragma unroll
        for (int j = 0; j < JD; ++j) vw[j] = win.check_value(vw[j], bad);
      }
      u32x4_t wh, wl;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = st[e >> 1][2 * (e & 1)], y = st[e >> 1][2 * (e & 1) + 1];
        wh[e] = f2bf2(x, y);
        wl[e] = f2bf2(x - __uint_as_float(wh[e] << 16), y - __uint_as_float(wh[e] & 0xffff0000u));
      }
#pragma unroll
      for (int j = 0; j < JD; ++j) {
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, vw[j]);
        a1[j] = mfma(vf, __builtin_bit_cast(bf16x8_t, wh), a1[j]);
        a1[j] = mfma(vf, __builtin_bit_cast(bf16x8_t, wl), a1[j]);
      }
      bad = wave_or(bad);
      if (bad & sees) l1 = NAN;
    }
    // in the units that the codes begin with: a page's weights keep their bits however small its step
#pragma unroll
    for (int h = 0; h < R; ++h)
      if (tile == h) {
#pragma unroll
        for (int j = 0; j < JD; ++j) acc[h][j] = a1[j] * (1.0f / VREF0);
        m[h] = m1;
        l[h] = l1;
      } else {
        nothing(h);
      }
  } else {
#pragma unroll
    for (int h = 0; h < R; ++h) nothing(h);
  }
  auto rescale = [&](int h, float alpha) {
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * alpha;
    }
  };
  // Scores of a 16-token tile: operands read from LDS AH ahead of their products (64 rows' would not
  // fit the registers: they are read at every use).
  auto scores = [&](const u32x4_t* sq, auto key, auto product, f32x4_t (&st)[R][2], int a) {
    constexpr int AH = R * KS < 4 ? R * KS : 4;
    int ql = lane;
    if constexpr (R > 2) asm volatile("" : "+v"(ql));
    auto query = [&](int x) { return sq[(x % R * KS + x / R) * 64 + ql]; };
    u32x4_t qf[AH];
#pragma unroll
    for (int x = 0; x < AH; ++x) qf[x] = query(x);
#pragma unroll
    for (int x = 0; x < R * KS; ++x) {
      const int h = x % R, k = x / R;
      if (k == 0) st[h][a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      st[h][a] = product(key(k), qf[x % AH], st[h][a]);
      if (x + AH < R * KS) qf[x % AH] = query(x + AH);
      if constexpr (R > 2) __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (; ch < cend; ch += 4) {
    // a page that stands for NaN: every row sees it, any finite step will do
    if (!(ks < INFINITY && vs < INFINITY)) {
#pragma unroll
      for (int h = 0; h < R; ++h) l[h] = NAN;
      ks = vs = 1.0f;
    }
    ks = fmaxf(ks, KS_MIN);
    vs = fmaxf(vs, VS_MIN);
    const float unit = fmaxf(vref, pow2_above(vs)), shrink = vref * pow2_inv(unit);
    const Step step = step_of(step_parts(ks * sc, vs), unit, true);
    vref = unit;
    f32x4_t st[R][2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      f16x8_t kf[KS];
#pragma unroll
      for (int j = 0; j < KS / 2; ++j) {
        const u32x4_t w = kr[a * (KS / 2) + j];
        kf[2 * j] = codes_f16(w[0], w[1]);
        kf[2 * j + 1] = codes_f16(w[2], w[3]);
      }
      scores(sh.q.h, [&](int k) { return kf[k]; },
             [](f16x8_t x, u32x4_t y, f32x4_t z) { return mfma_h(x, __builtin_bit_cast(f16x8_t, y), z); }, st, a);
    }
    // The next chunk's codes, as this one's registers become free.  (Without a next one this one's once
    // more: loads that only some iterations have would make every wait one for all of them, and the last
    // chunk's own copy of this loop would come from memory as it runs, 3 us.)
    const int id = entry_next;
    if (ch + 4 < cend) {
      page = id;
      tin = 32 * (ch + 4) & (P - 1);
    }
    entry_next = entry_of(min(ch + 8, cend - 1));
    take_keys();
    u32x4_t pb[R];
#pragma unroll
    for (int h = 0; h < R; ++h) {
      const Step sp[1] = {{step.f * sh.qs[16 * h + r], step.lw, step.winv}};
      rescale(h, softmax_step<1>(st[h], sp, m[h], l[h]) * shrink);
#pragma unroll
      for (int e = 0; e < 4; ++e) pb[h][e] = pack_f16(st[h][e >> 1][2 * (e & 1)], st[h][e >> 1][2 * (e & 1) + 1]);
    }
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const f16x8_t v0 = codes_f16(vr[j][0], vr[j][1]), v1 = codes_f16(vr[j][2], vr[j][3]);
#pragma unroll
      for (int h = 0; h < R; ++h) {
        acc[h][2 * j] = mfma_h(v0, __builtin_bit_cast(f16x8_t, pb[h]), acc[h][2 * j]);
        acc[h][2 * j + 1] = mfma_h(v1, __builtin_bit_cast(f16x8_t, pb[h]), acc[h][2 * j + 1]);
      }
    }
    take(c.vc, at, vr);
  }
  // The waves' results, each scaled to the row's maximum over all four, go through LDS, half of the operand
  // tiles at a time, and are summed in the order of the waves.
  anew();
#pragma unroll
  for (int h = 0; h < R; ++h) {
    l[h] = row_sum(l[h]);
    if (g == 0) sh.ml[wave][16 * h + r] = make_float2(m[h], l[h]);
  }
  __syncthreads();                                       // (the queries are read, too)
  const float unit = vref / WUNIT;
#pragma unroll
  for (int h = 0; h < R; ++h) {
    float2 x[4];
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[w] = sh.ml[w][16 * h + r];
      mm = fmaxf(mm, x[w].x);
    }
    float ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += x[w].x == -INFINITY ? x[w].y : __builtin_amdgcn_exp2f(x[w].x - mm) * x[w].y;
    const float f = m[h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[h] - mm) * unit;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * f;
    if (wave == 0 && g == 0) sh.all[16 * h + r] = make_float2(mm, !s.ok || !tree_ok ? NAN : ll);
  }
  constexpr int JH = JD / 2;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int p = 0; p < R * JH; ++p) sh.o[wave][p][lane] = acc[p / JH][half * JH + p % JH];
    __syncthreads();
    // (wave w: operand tiles w, w + 4, ..)
#pragma unroll 2
    for (int p = wave; p < R * JH; p += 4) {
      const int j = half * JH + p % JH, row = 16 * (p / JH) + r;
      f32x4_t o = sh.o[0][p][lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) o = o + sh.o[w][p][lane];
      if (row >= pc.rows) continue;
      const float2 x = sh.all[row];
      int64_t t = 0, hd = 0;
      if (out.splits == 1) {
        t = int64_t(s.b) + (pc.row0 + row) / G;
        hd = int64_t(u) * G + (pc.row0 + row) % G;
      }
      put4(out, row, t, hd, DH, 16 * j + 4 * g, make_float4(o[0], o[1], o[2], o[3]), x.y);
      if (j == 0 && g == 0) put_ml(out, row, t, hd, x.x, x.y);
    }
  }
  __syncthreads();
}

// An inclusive sum over the wave's lanes.
OQ_DEV uint32_t lanes_upto(uint32_t v) {
  auto from = [&](auto ctrl, auto rows) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
  };
  v += from(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});   // 1, 2, 4, 8 lanes below
  v += from(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
  v += from(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
  v += from(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
  v += from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});   // the row below's last
  v += from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});   // lane 31's
  return v;
}

// The row tiles of all sequences, one behind the other, each as long as its chunks cost, are a
// line that the nw workgroups of a key head cut into equal shares: the lengths are on the
// device, and a ragged batch is as evenly spread as one long sequence.  A tile's steps are of
// 2^shift chunks (one, unless the line would pass 30 bits); a step belongs to the share that it
// begins in, but for a tile's first and last few, which go with their neighbours: a piece costs
// more than they do.  A tile that several workgroups have goes to slots of the workspace (a share
// begins with at most one such piece and ends with at most one) and is joined by
// tree_join_kernel, whom the workgroup where it begins tells so.
// Against the batch attention's kernels with a tree's mask (a number of splits for all sequences, row
// and tile kernels one after the other): 32 trees of up to 16 nodes over up to 4,096 tokens, 64 heads, 8
// key heads, 107 -> 71 us (65 with TILE_MORE); 8 nodes over 131,072 81 -> 75; 64 over 16,384, where
// matrix and vector work bound both, 66 -> 65.  No instance spills vector registers; 57 to 91 scalar
// ones (the line's and the piece's numbers) wait in lanes of vector registers.
struct Cut {
  int token, head, rows, w, pieces;      // its first row as a token and a head of the group; w: where it begins,
};                                       // pieces: workgroups that go on with it
template <int DH, int RMAX, bool ONCE>
__global__ __launch_bounds__(256, 2) void tree_attend_kernel(CacheArgs c, const uint16_t* __restrict__ Q, int64_t ldq,
                                                             int H, uint16_t* __restrict__ O, float* __restrict__ LSE,
                                                             float* __restrict__ part, Cut* __restrict__ cuts,
                                                             int tiles, int nw, int least, int shift) {
  __shared__ Shared<DH, RMAX> sh;
  const int lane = threadIdx.x & 63, G = H / c.Hkv;
  int4* line = sh.line[threadIdx.x >> 6];
  // key heads fastest (an XCD keeps its heads' pages in its L2)
  const int u = int(blockIdx.x) % c.Hkv, w = int(blockIdx.x) / c.Hkv;
  // sequence i as (tokens, first row, new tokens, slot or -1)
  auto fetch = [&](int i) {
    if (i >= c.n_seq) return make_int4(0, 0, 0, -1);
    const Seq s = seq_of(c, i);
    return make_int4(s.L, s.b, s.n, s.ok ? s.slot : -1);
  };
  auto steps_of = [&](int4 x) {          // of a tile
    const int nch = x.w < 0 ? 1 : (x.x + x.z + 31) / 32;
    return uint32_t((nch + (1 << shift) - 1) >> shift);
  };
  // A tile costs TILE_MORE steps more than its chunks: the queries, the window, the join.
  auto cost_of = [&](int4 x) {           // of the sequence
    const int rows = x.z * G, rest = rows % TILE_ROWS;
    return (steps_of(x) + TILE_MORE) * uint32_t(rows / TILE_ROWS * 6 + (rest ? tile_cost(rest) : 0));
  };
  auto tiles_of = [&](int4 x) { return uint32_t(x.z * G + TILE_ROWS - 1) / TILE_ROWS; };
  uint32_t whole = 0, there = 0;         // the line's length, its tiles
  for (int base = 0; base < c.n_seq; base += 64) {
    const int4 x = fetch(base + lane);
    if (base == 0) line[lane] = x;
    whole += uint32_t(__builtin_amdgcn_readlane(int(lanes_upto(cost_of(x))), 63));
    there += uint32_t(__builtin_amdgcn_readlane(int(lanes_upto(tiles_of(x))), 63));
  }
  const uint32_t share = max((whole + nw - 1) / uint32_t(nw), uint32_t(least)), lo = w * share, hi = lo + share;
  const uint32_t snap = min(uint32_t(TILE_MORE) >> shift, share / 24);
  // (a tile's entry is written where it begins; of tiles that the host allowed for and that are not there, here)
  for (int k = int(there) + w * 256 + threadIdx.x; k < tiles; k += nw * 256) cuts[int64_t(k) * c.Hkv + u] = Cut{0, 0, 0, 0, 0};
  // from tile to tile: where the next one is looked for, what lies before `base`
  uint32_t pos = lo, run = 0, run_tiles = 0;
  for (int base = 0; base < c.n_seq && pos < hi && pos < whole;) {
    const int4 x = line[lane];
    const uint32_t cost = cost_of(x), upto = run + lanes_upto(cost);
    const uint64_t past = __ballot(upto > pos);
    if (!past) {
      run = uint32_t(__builtin_amdgcn_readlane(int(upto), 63));
      run_tiles += uint32_t(__builtin_amdgcn_readlane(int(lanes_upto(tiles_of(x))), 63));
      base += 64;
      line[lane] = fetch(base + lane);
      continue;
    }
    const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
    const int4 y = make_int4(of(x.x), of(x.y), of(x.z), of(x.w));
    const Seq s{y.x, y.y, y.z, y.w, y.w >= 0};
    const int rows = s.n * G, nch = s.ok ? (s.L + s.n + 31) / 32 : 1;
    const uint32_t begin = uint32_t(of(int(upto - cost))), steps = steps_of(y), place = steps + TILE_MORE;
    const int row0 = rows <= TILE_ROWS || pos < begin ? 0 : int((pos - begin) / (place * 6)) * TILE_ROWS;
    const int n = min(rows - row0, TILE_ROWS);
    const uint32_t cost1 = tile_cost(n), t0 = begin + uint32_t(row0 / TILE_ROWS) * place * 6, t1 = t0 + steps * cost1;
    pos = t0 + place * cost1;
    // the steps that begin in [lo, hi)
    auto steps_below = [&](uint32_t p) {
      const uint32_t d = min(max(p, t0), t1) - t0 + cost1 - 1;
      const uint32_t n = min(cost1 == 3 ? d / 3 : cost1 == 4 ? d / 4 : d / 6, steps);
      return n == steps ? n : n < snap ? 0u : n + snap > steps ? steps : n;
    };
    const uint32_t s0 = steps_below(lo), s1 = steps_below(hi);
    if (s0 >= s1) continue;
    const int64_t slot = (int64_t(w) * c.Hkv + u) * 2 + (s0 == 0);
    if (s0 == 0) {
      const uint32_t end = min((t0 + (steps - 1) * cost1) / share, uint32_t(nw - 1));
      const uint32_t to = max(steps_below(end * share) < steps ? end : end - 1, uint32_t(w));
      const uint32_t tile = run_tiles + uint32_t(of(int(lanes_upto(tiles_of(x)) - tiles_of(x)))) + row0 / TILE_ROWS;
      // (row ranges that overlap may make more tiles than there is room for)
      if (threadIdx.x == 0 && tile < uint32_t(tiles))
        cuts[int64_t(tile) * c.Hkv + u] = Cut{s.b + row0 / G, row0 % G, n, w, int(to) - w};
    }
    const Out out{O, LSE, part, s0 > 0 || s1 < steps ? 2 : 1, H, c.T, slot * (16 * RMAX),
                  int64_t(nw) * c.Hkv * 2 * (16 * RMAX) * DH};
    const Piece pc{row0, n, int(s0 << shift), min(nch, int(s1 << shift))};
    const int i = base + at;
    if (RMAX == 1 || n <= 16) attend_piece<DH, 1, ONCE>(c, s, pc, i, u, G, Q, ldq, out, sh);
    else if (RMAX == 2 || n <= 32) attend_piece<DH, RMAX == 1 ? 1 : 2, ONCE>(c, s, pc, i, u, G, Q, ldq, out, sh);
    else attend_piece<DH, RMAX, ONCE>(c, s, pc, i, u, G, Q, ldq, out, sh);
  }
}

// Joins the tiles that were cut: a workgroup takes `rows` rows of one tile, DH / 4 lanes a row.  With few
// pieces a group of lanes has a row to itself, with many the groups deal its pieces among themselves.
template <int DH>
__global__ __launch_bounds__(256) void tree_join_kernel(CacheArgs c, int H, const float* __restrict__ part,
                                                        const Cut* __restrict__ cuts, int nw, int unit_rows, int rows,
                                                        uint16_t* __restrict__ O, float* __restrict__ LSE) {
  constexpr int Q4 = DH / 4, NG = 256 / Q4;
  __shared__ float4 s_o[NG][Q4];
  __shared__ float2 s_ml[NG];
  const Cut cut = cuts[blockIdx.x];                        // [tile][key head]
  const int q = threadIdx.x % Q4, ng = threadIdx.x / Q4, u = int(blockIdx.x) % c.Hkv, G = H / c.Hkv;
  const int row0 = int(blockIdx.y) * rows, row1 = min(row0 + rows, cut.rows);
  if (cut.pieces <= 0 || row0 >= row1) return;
  const float2* ml = reinterpret_cast<const float2*>(part + int64_t(nw) * c.Hkv * 2 * unit_rows * DH);
  const bool few = cut.pieces < NG && rows > 1;
  for (int row = few ? row0 + ng : row0; row < row1; row += few ? NG : 1) {
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto join = [&](float2 x, float4 y) {
      const float mn = fmaxf(m, x.x);
      const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
      const float fk = x.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.x - mn);
      // (without a token l is 0 or, for a NaN row, NaN: it stays)
      l = (m == -INFINITY ? l : f * l) + (x.x == -INFINITY ? x.y : fk * x.y);
      o = make_float4(f * o.x + fk * y.x, f * o.y + fk * y.y, f * o.z + fk * y.z, f * o.w + fk * y.w);
      m = mn;
    };
    // eight pieces' loads at a time (past the last: none, which changes nothing)
    constexpr int AT = 8;
    for (int k0 = few ? 0 : ng; k0 <= cut.pieces; k0 += few ? AT : AT * NG) {
      float2 x[AT];
      float4 y[AT];
#pragma unroll
      for (int e = 0; e < AT; ++e) {
        const int k = k0 + e * (few ? 1 : NG), kk = min(k, cut.pieces);
        const int64_t p = ((int64_t(cut.w + kk) * c.Hkv + u) * 2 + (kk == 0)) * unit_rows + row;
        x[e] = ml[p];
        y[e] = *reinterpret_cast<const float4*>(part + p * DH + 4 * q);
        if (k > cut.pieces) {
          x[e] = make_float2(-INFINITY, 0.0f);
          y[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
#pragma unroll
      for (int e = 0; e < AT; ++e) join(x[e], y[e]);
    }
    if (!few) {
      __syncthreads();                                     // (the last row is read)
      s_o[ng][q] = o;
      if (q == 0) s_ml[ng] = make_float2(m, l);
      __syncthreads();
      if (ng > 0) continue;
#pragma unroll
      for (int k = 1; k < NG; ++k) join(s_ml[k], s_o[k][q]);
    }
    const float inv = 1.0f / l;
    const int64_t t = int64_t(cut.token) + (cut.head + row) / G, hd = int64_t(u) * G + (cut.head + row) % G;
    *reinterpret_cast<uint2*>(O + (t * H + hd) * DH + 4 * q) =
        make_uint2(f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv));
    if (LSE && q == 0) LSE[hd * c.T + t] = lse_of(m, l);
  }
}

}  // namespace

hipError_t cache_append_tree(const CacheArgs& c, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                             const void* V, int64_t ldv, bool in_bf16, int H, const float* rope, int64_t n_rope,
                             const float* s_a, uint16_t* Qout, hipStream_t st) {
  // query slices: eight items of a thread each where that fills the card, else two
  const int64_t items = int64_t(c.max_q) * H * (c.d / 8), each = c.n_seq * items >= 1024 * 8 * 256 ? 8 : 2;
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(items / (each * 256), 65535 - c.Hkv));
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

// Workgroups: two to a compute unit, as many as run at once (three with 16 rows each spill: one node over
// 131,072 tokens, 64 heads, 70 us, with two 55).  The smallest share is 256 tokens of a tile.
TreePlan tree_attend_plan(int n_seq, int Hkv, int H, int64_t tokens, int max_q, int64_t max_len, int d) {
  const int64_t rows = int64_t(max_q) * (H / Hkv);
  TreePlan p;
  p.row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.one_tile = rows <= TILE_ROWS;
  p.nw = std::max(1, (512 + Hkv / 2) / Hkv);
  p.least = 8 * (p.row_tiles == 1 ? 3 : p.row_tiles == 2 ? 4 : 6);
  p.all_tiles = n_seq * ((rows + TILE_ROWS - 1) / TILE_ROWS);
  p.tiles = std::min(tokens * (H / Hkv) / TILE_ROWS + std::min<int64_t>(n_seq, tokens), p.all_tiles);
  // (2^23 tiles of a step and TILE_MORE still fit 30 bits, more are refused; all_tiles, since row ranges that
  // overlap may make more tiles than the tokens do, and the line must not wrap for them either)
  p.shift = 0;
  while (p.shift < 30 && p.all_tiles * (((max_len + 31) / 32 >> p.shift) + 1 + TILE_MORE) * 6 >= (int64_t(1) << 30))
    ++p.shift;
  p.part_floats = size_t(p.nw) * size_t(Hkv) * 2 * size_t(16 * p.row_tiles) * size_t(d + 2);
  p.bytes = p.part_floats * 4 + size_t(p.tiles) * size_t(Hkv) * sizeof(Cut);
  return p;
}

hipError_t cache_attend_tree(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                             float* ws, const TreePlan& p, hipStream_t st) {
  Cut* cuts = reinterpret_cast<Cut*>(ws + p.part_floats);
  auto run = [&](auto dh, auto rt, auto once) {
    constexpr int DH = decltype(dh)::value, RMAX = decltype(rt)::value;
    const unsigned units = unsigned(p.nw) * unsigned(c.Hkv);
    hipLaunchKernelGGL((tree_attend_kernel<DH, RMAX, decltype(once)::value>), dim3(units), dim3(256), 0, st, c, Q, ldq,
                       H, O, LSE, ws, cuts, int(p.tiles), p.nw, p.least, p.shift);
    // (a key head's only workgroup cuts nothing; rows by eight where tiles have few pieces)
    const int by = p.nw > 16 * p.tiles ? 1 : 8;
    if (p.nw > 1)
      hipLaunchKernelGGL(tree_join_kernel<DH>, dim3(unsigned(p.tiles) * unsigned(c.Hkv), 16 * RMAX / by), dim3(256), 0,
                         st, c, H, ws, cuts, p.nw, 16 * RMAX, by, O, LSE);
  };
  auto rows = [&](auto dh) {
    if (p.row_tiles == 1) run(dh, std::integral_constant<int, 1>{}, std::true_type{});
    else if (p.row_tiles == 2) run(dh, std::integral_constant<int, 2>{}, std::true_type{});
    else if (p.one_tile) run(dh, std::integral_constant<int, 4>{}, std::true_type{});
    else run(dh, std::integral_constant<int, 4>{}, std::false_type{});
  };
  if (c.d == 64) rows(std::integral_constant<int, 64>{});
  else rows(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

hipError_t cache_commit(const CacheArgs& c, const int32_t* path, int max_path, const int32_t* count, hipStream_t st) {
  const dim3 grid(unsigned(c.n_seq), unsigned(c.Hkv));
  hipLaunchKernelGGL(tree_commit_kernel, grid, dim3(256), unsigned(c.P) * c.d * 4, st, c, path, max_path, count);
  return hipGetLastError();
}

}  // namespace oq
