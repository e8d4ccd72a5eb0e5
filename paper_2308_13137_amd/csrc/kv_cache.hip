// The paged key/value cache in 8 bits and attention over it.
//
// A sequence's tokens fill pages of P tokens.  A full page is int8 codes with
// one step per page, head and tensor (the symmetric quantiser of the whole
// block: h = max(max|x| / 127, 1e-5), code = rint(x (1/h))), written once from
// the bf16 rows, so the codes do not depend on how the tokens arrived.  The
// rows of the page being filled, and of the one before it, are bf16 in the
// sequence's window (page p in half p mod 2): a page is quantised from there,
// and a caller that drops its newest tokens (down to the start of the page
// before the last) only has to set the length back.
//
// Layouts are operand layouts of v_mfma_f32_16x16x32_bf16 (lane = 16 g + r):
//   K codes   [P/16][d/64][g][r][16]: token 16 a + r, channels 64 j + 16 g + b
//   V codes   [P/32][d/32][g][r][2][8]: channel 32 jj + 16 hh + r, tokens
//             32 c + 4 g + e (e < 4) and 32 c + 16 + 4 g + e - 4
//   K window  [P][d];  V window [P/32][d/16][g][r][8], tokens as in V codes
// One 16-byte load per lane, 1 KiB in a row per wave, fills an operand.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "serve.h"

namespace oq {
namespace {

typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

OQ_DEV f32x4_t mfma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Byte (element) offsets inside a page-and-head block.
OQ_DEV int k_at(int t, int c, int d) {
  return ((t >> 4) * (d >> 6) + (c >> 6)) * 1024 + ((c >> 4) & 3) * 256 + (t & 15) * 16 + (c & 15);
}
OQ_DEV int v_at(int t, int c, int d) {
  return ((t >> 5) * (d >> 5) + (c >> 5)) * 1024 + ((t >> 2) & 3) * 256 + (c & 15) * 16 + ((c >> 4) & 1) * 8 +
         ((t >> 4) & 1) * 4 + (t & 3);
}
OQ_DEV int vw_at(int t, int c, int d) {
  return ((t >> 5) * (d >> 4) + (c >> 4)) * 512 + ((t >> 2) & 3) * 128 + (c & 15) * 8 + ((t >> 4) & 1) * 4 +
         (t & 3);
}

// One sequence of the batch, with everything read from device memory checked:
// a sequence that does not fit the tensors has ok = false.
struct Seq {
  int L, b, n, slot;
  bool ok;
};
OQ_DEV Seq seq_of(const CacheArgs& c, int i) {
  Seq s;
  const int64_t b = c.q_start[i], e = c.q_start[i + 1];
  s.L = c.length[i];
  s.slot = c.slot ? c.slot[i] : i;
  s.ok = s.slot >= 0 && s.slot < c.n_slots && s.L >= 0;
  const int64_t bb = min(max(b, int64_t(0)), c.T), ee = min(max(e, bb), c.T);
  s.b = int(bb);
  s.n = int(min(ee - bb, int64_t(c.max_q)));
  if (b < 0 || e < b || e > c.T || e - b > c.max_q) s.ok = false;
  if (int64_t(s.L) + s.n > int64_t(c.max_pages) * c.P) s.ok = false;
  return s;
}
OQ_DEV int page_of(const CacheArgs& c, int i, int pg) {
  const int p = c.table[int64_t(i) * c.max_pages + pg];
  return p >= 0 && p < c.n_pages ? p : -1;
}

// ------------------------------------------------------------------ append
constexpr int AT = 256;

template <typename TI>
struct RowIn {
  const TI *q, *k, *v;
  int64_t ldq, ldk, ldv;
};

// Channels p and p + d/2 of a turned row, in the block step's order of operations.
OQ_DEV float2 turn(float a, float b, const float* rope, int64_t n_rope, int pos, int p, int half) {
  if (!rope) return make_float2(a, b);
  if (pos >= n_rope) return make_float2(NAN, NAN);
  const float2 cs = reinterpret_cast<const float2*>(rope)[int64_t(pos) * half + p];
  return make_float2(a * cs.x - b * cs.y, b * cs.x + a * cs.y);
}

template <typename TI>
__global__ __launch_bounds__(AT) void cache_append_kernel(CacheArgs c, RowIn<TI> in, int H,
                                                          const float* __restrict__ rope, int64_t n_rope,
                                                          const float* __restrict__ sa,
                                                          uint16_t* __restrict__ Qout) {
  extern __shared__ uint16_t s_rows[];                     // K [P][d], then V [P][d]
  __shared__ int s_max[2][AT / 64];
  const int u = blockIdx.y, i = blockIdx.z, tid = threadIdx.x;
  const int d = c.d, half = d / 2, P = c.P, G = H / c.Hkv;
  const Seq s = seq_of(c, i);
  const int pg0 = s.L / P, pg = pg0 + int(blockIdx.x);
  if (s.n == 0) return;
  const int end = s.L + s.n;                               // (ok: fits an int)
  if (!s.ok) {                                             // nothing is cached; the queries are NaN
    for (int64_t e = tid + int64_t(AT) * blockIdx.x; e < int64_t(s.n) * G * d; e += int64_t(AT) * gridDim.x)
      Qout[(int64_t(s.b) + e / (G * d)) * H * d + int64_t(u) * G * d + e % (G * d)] = 0x7fc0;
    return;
  }
  const int lo = max(s.L, pg * P), hi = min(end, (pg + 1) * P);
  if (lo >= hi) return;
  const int last = (end - 1) / P;
  // the queries
  for (int e = tid; e < (hi - lo) * G * half; e += AT) {
    const int p = e % half, hh = (e / half) % G, pos = lo + e / (half * G);
    const int64_t t = int64_t(s.b) + (pos - s.L);
    const int64_t col = int64_t(u * G + hh) * d + p;
    const float2 y = turn(load1(in.q + t * in.ldq + col), load1(in.q + t * in.ldq + col + half), rope, n_rope,
                          pos, p, half);
    const float s0 = sa ? sa[u * d + p] : 1.0f, s1 = sa ? sa[u * d + p + half] : 1.0f;
    Qout[t * H * d + col] = f2bf(y.x / s0);
    Qout[t * H * d + col + half] = f2bf(y.y / s1);
  }
  const int64_t win = int64_t(P) * d;
  auto window = [&](uint16_t* w, int page) { return w + ((int64_t(s.slot) * 2 + (page & 1)) * c.Hkv + u) * win; };
  auto new_row = [&](int pos, int p, uint32_t& k2, uint32_t& v2) {
    const int64_t t = int64_t(s.b) + (pos - s.L);
    const int64_t col = int64_t(u) * d + p;
    float2 y = turn(load1(in.k + t * in.ldk + col), load1(in.k + t * in.ldk + col + half), rope, n_rope, pos, p,
                    half);
    if (sa) y = make_float2(y.x * sa[u * d + p], y.y * sa[u * d + p + half]);
    k2 = f2bf2(y.x, y.y);
    v2 = f2bf2(load1(in.v + t * in.ldv + col), load1(in.v + t * in.ldv + col + half));
  };
  auto to_window = [&](int page, int r, int p, uint32_t k2, uint32_t v2) {
    uint16_t* kw = window(c.kw, page);
    uint16_t* vw = window(c.vw, page);
    kw[r * d + p] = uint16_t(k2);
    kw[r * d + p + half] = uint16_t(k2 >> 16);
    vw[vw_at(r, p, d)] = uint16_t(v2);
    vw[vw_at(r, p + half, d)] = uint16_t(v2 >> 16);
  };
  const bool full = hi == (pg + 1) * P;
  uint16_t* sk = s_rows;
  uint16_t* sv = s_rows + P * d;
  // rows of this page that were there before the call
  const int old = blockIdx.x == 0 ? s.L - pg * P : 0;
  if (full) {
    const uint16_t* kw = window(c.kw, pg);
    const uint16_t* vw = window(c.vw, pg);
    for (int e = tid; e < old * d; e += AT) {
      sk[e] = kw[e];
      sv[e] = vw[vw_at(e / d, e % d, d)];
    }
  }
  // this page's new rows: to LDS where the page fills up, to the window where
  // it is one of the last two.  A later page of the same half as the first must
  // wait until the first one's old rows are read: workgroup 0 writes it.
  const bool old_rows = s.L % P != 0;
  const bool keep = pg >= last - 1 && !(blockIdx.x > 0 && old_rows && ((pg - pg0) & 1) == 0);
  for (int e = tid; e < (hi - lo) * half; e += AT) {
    const int p = e % half, pos = lo + e / half, r = pos - pg * P;
    uint32_t k2, v2;
    new_row(pos, p, k2, v2);
    if (full) {
      sk[r * d + p] = uint16_t(k2);
      sk[r * d + p + half] = uint16_t(k2 >> 16);
      sv[r * d + p] = uint16_t(v2);
      sv[r * d + p + half] = uint16_t(v2 >> 16);
    }
    if (keep) to_window(pg, r, p, k2, v2);
  }
  if (!full) return;
  __syncthreads();
  if (blockIdx.x == 0 && old_rows) {
    for (int page = max(last - 1, pg0 + 1); page <= last; ++page) {
      if ((page - pg0) & 1) continue;
      const int a = page * P, b = min(end, a + P);
      for (int e = tid; e < (b - a) * half; e += AT) {
        const int p = e % half, pos = a + e / half;
        uint32_t k2, v2;
        new_row(pos, p, k2, v2);
        to_window(page, pos - a, p, k2, v2);
      }
    }
  }
  // the largest magnitude as an integer: NaN and infinity order above all
  int mk = 0, mv = 0;
  for (int e = tid; e < P * d; e += AT) {
    mk = max(mk, int(sk[e] & 0x7fff));
    mv = max(mv, int(sv[e] & 0x7fff));
  }
  for (int off = 1; off < 64; off <<= 1) {
    mk = max(mk, __shfl_xor(mk, off));
    mv = max(mv, __shfl_xor(mv, off));
  }
  if ((tid & 63) == 0) {
    s_max[0][tid >> 6] = mk;
    s_max[1][tid >> 6] = mv;
  }
  __syncthreads();
  for (int w = 0; w < AT / 64; ++w) {
    mk = max(mk, s_max[0][w]);
    mv = max(mv, s_max[1][w]);
  }
  const int id = page_of(c, i, pg);
  if (id < 0) return;
  // a block with a value that is not finite stands for NaN as a whole
  const float hk = mk >= 0x7f80 ? NAN : fmaxf(div_rn(bf2f(uint16_t(mk)), 127.0f), 1e-5f);
  const float hv = mv >= 0x7f80 ? NAN : fmaxf(div_rn(bf2f(uint16_t(mv)), 127.0f), 1e-5f);
  const float rk = div_rn(1.0f, hk), rv = div_rn(1.0f, hv);
  const int64_t blk = int64_t(id) * c.Hkv + u;
  if (tid == 0) {
    c.ks[blk] = hk;
    c.vs[blk] = hv;
  }
  auto code = [](uint16_t x, float r) {
    const float q = rintf(bf2f(x) * r);
    return int8_t(int(fminf(fmaxf(q, -127.0f), 127.0f)));
  };
  for (int e = tid; e < P * d; e += AT) {
    c.kc[blk * win + k_at(e / d, e % d, d)] = code(sk[e], rk);
    c.vc[blk * win + v_at(e / d, e % d, d)] = code(sv[e], rv);
  }
}

// ------------------------------------------------------------------ read
// Rows begin[i] .. length[i] + new - 1 of every sequence, as values.
template <typename TO>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs c, const int32_t* __restrict__ begin,
                                                         const int32_t* __restrict__ row_start, int64_t rows,
                                                         TO* __restrict__ K, TO* __restrict__ V) {
  const int i = blockIdx.y, d = c.d, W = c.Hkv * d;
  const Seq s = seq_of(c, i);
  const int64_t b = max(row_start[i], 0), e = min(int64_t(row_start[i + 1]), rows);
  const int64_t r = b + blockIdx.x;
  if (r >= e) return;
  const int64_t pos = int64_t(begin[i]) + blockIdx.x;
  const bool ok = s.ok && pos >= 0 && pos < int64_t(s.L) + s.n;
  const int64_t win = int64_t(c.P) * d;
  const int pg = ok ? int(pos / c.P) : 0, t = ok ? int(pos % c.P) : 0;
  const bool full = ok && int64_t(pg + 1) * c.P <= int64_t(s.L) + s.n;
  const int id = full ? page_of(c, i, pg) : -1;
  for (int x = threadIdx.x; x < W; x += 256) {
    const int u = x / d, ch = x % d;
    float k = NAN, v = NAN;
    if (ok && !full) {
      const int64_t at = ((int64_t(s.slot) * 2 + (pg & 1)) * c.Hkv + u) * win;
      k = bf2f(c.kw[at + t * d + ch]);
      v = bf2f(c.vw[at + vw_at(t, ch, d)]);
    } else if (id >= 0) {
      const int64_t blk = int64_t(id) * c.Hkv + u;
      k = float(c.kc[blk * win + k_at(t, ch, d)]) * c.ks[blk];
      v = float(c.vc[blk * win + v_at(t, ch, d)]) * c.vs[blk];
    }
    if (K) store1(K + r * W + x, k);
    if (V) store1(V + r * W + x, v);
  }
}

// ------------------------------------------------------------------ attention
// int8 -> bf16, exact: eight codes of two dwords.
OQ_DEV bf16x8_t codes_bf16(unsigned a, unsigned b) {
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned v = i < 2 ? a : b;
    const int sh = 16 * (i & 1);
    const float lo = float(int8_t(v >> sh)), hi = float(int8_t(v >> (sh + 8)));
    w[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

// Is one of eight bf16 values not finite?
OQ_DEV bool not_finite(u32x4_t w) {
  bool b = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) b = b || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return b;
}

// One workgroup: 16 R rows (query x head of the group) of one key head, chunks
// of 32 tokens dealt to the four waves; each wave runs its own online softmax
// in registers, the four are joined in LDS and the splits by a second kernel.
//   S^T = K Q^T: a lane holds query row r, tokens 4 g + 0..3 of both 16-token
//   tiles, which is the B operand of O^T = V^T P^T as it stands.
template <int DH, int R>
__global__ __launch_bounds__(256) void cache_attend_kernel(CacheArgs c, const uint16_t* __restrict__ Q,
                                                           int64_t ldq, int H, uint16_t* __restrict__ O,
                                                           float* __restrict__ LSE, float* __restrict__ part,
                                                           int splits) {
  constexpr int KS = DH / 32, JD = DH / 16;
  __shared__ float s_o[4][16 * R][DH + 4];
  __shared__ float s_ml[4][16 * R][2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int split = int(blockIdx.x) % splits, rt = int(blockIdx.x) / splits, u = blockIdx.y, i = blockIdx.z;
  const int G = H / c.Hkv, P = c.P;
  const Seq s = seq_of(c, i);
  const int rows = s.n * G, row0 = rt * 16 * R;
  if (row0 >= rows) return;
  const int total = s.ok ? s.L + s.n : 0;
  const int closed = total / P * P;
  const float sc = 1.4426950408889634f / sqrtf(float(DH));
  const int64_t win = int64_t(P) * DH;

  bf16x8_t qf[R][KS];
  int lim[R];                                            // the last token this lane's row sees
#pragma unroll
  for (int h = 0; h < R; ++h) {
    const int row = min(row0 + 16 * h + r, rows - 1), j = row / G;
    lim[h] = s.L + j;
    const uint16_t* qp = Q + (int64_t(s.b) + j) * ldq + int64_t(u * G + row % G) * DH;
#pragma unroll
    for (int k = 0; k < KS; ++k)
      qf[h][k] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(qp + 64 * (k >> 1) + 16 * g + 8 * (k & 1)));
  }
  f32x4_t acc[R][JD];
  float m[R], l[R];
#pragma unroll
  for (int h = 0; h < R; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.0f;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int jmax = min(row0 + 16 * R - 1, rows - 1) / G;
  const int seen = s.ok ? s.L + jmax + 1 : 0;            // tokens some row of the tile sees
  const int nch = (seen + 31) / 32, per = (nch + splits - 1) / splits;
  const int c1 = min(nch, (split + 1) * per);
  for (int ch = split * per + wave; ch < c1; ch += 4) {
    const int t0 = 32 * ch, pg = t0 / P, tin = t0 - pg * P;
    bf16x8_t kf[2][KS], vf[JD];
    float ks = 1.0f, vs = 1.0f;
    unsigned badtok = 0;
    if (t0 < closed) {
      const int id = page_of(c, i, pg);
      const int64_t blk = int64_t(max(id, 0)) * c.Hkv + u;
      ks = id < 0 ? NAN : c.ks[blk];
      vs = id < 0 ? NAN : c.vs[blk];
      const u32x4_t* kp = reinterpret_cast<const u32x4_t*>(c.kc + blk * win + tin * DH) + lane;
      const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(c.vc + blk * win + tin * DH) + lane;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < DH / 64; ++j) {
          const u32x4_t w = kp[64 * (a * (DH / 64) + j)];
          kf[a][2 * j] = codes_bf16(w[0], w[1]);
          kf[a][2 * j + 1] = codes_bf16(w[2], w[3]);
        }
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) {
        const u32x4_t w = vp[64 * j];
        vf[2 * j] = codes_bf16(w[0], w[1]);
        vf[2 * j + 1] = codes_bf16(w[2], w[3]);
      }
    } else {
      // the open page: rows behind the end are whatever the window holds
      const int64_t at = ((int64_t(s.slot) * 2 + (pg & 1)) * c.Hkv + u) * win;
      const uint16_t* kp = c.kw + at + int64_t(tin) * DH;
      const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(c.vw + at + int64_t(tin) * DH) + lane;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4_t w =
              *reinterpret_cast<const u32x4_t*>(kp + (16 * a + r) * DH + 64 * (k >> 1) + 16 * g + 8 * (k & 1));
          if (t0 + 16 * a + r < total && not_finite(w)) badtok |= 1u << (16 * a + r);
          kf[a][k] = __builtin_bit_cast(bf16x8_t, w);
        }
#pragma unroll
      for (int j = 0; j < JD; ++j) {
        u32x4_t w = vp[64 * j];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int tok = 16 * (e >> 2) + 4 * g + (e & 3);
          const unsigned mask = 0xffffu << (16 * (e & 1));
          const unsigned x = (w[e >> 1] >> (16 * (e & 1))) & 0x7fffu;
          if (t0 + tok >= total) w[e >> 1] &= ~mask;
          else if (x >= 0x7f80u) {                       // not finite: see below
            badtok |= 1u << tok;
            w[e >> 1] &= ~mask;
          }
        }
        vf[j] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
    // a value that is not finite would reach every row of the product, those
    // that do not see its token too: it enters as zero, and the rows that see
    // it (or a key that is not finite) become NaN
    if (__any(badtok != 0)) {
      for (int off = 1; off < 64; off <<= 1) badtok |= __shfl_xor(badtok, off);
      const int first = t0 + __ffs(int(badtok)) - 1;
#pragma unroll
      for (int h = 0; h < R; ++h)
        if (lim[h] >= first) l[h] = NAN;
    }
#pragma unroll
    for (int h = 0; h < R; ++h) {
      f32x4_t st[2];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        st[a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k) st[a] = mfma(kf[a][k], qf[h][k], st[a]);
      }
      const float f = ks * sc;
      float mt = -INFINITY;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          st[a][q] = t0 + 16 * a + 4 * g + q > lim[h] ? -INFINITY : st[a][q] * f;
          mt = fmaxf(mt, st[a][q]);
        }
      mt = fmaxf(mt, __shfl_xor(mt, 16));
      mt = fmaxf(mt, __shfl_xor(mt, 32));
      const float mn = fmaxf(m[h], ceilf(mt));
      const float off = mn == -INFINITY ? 0.0f : mn;     // no token seen yet: weights 2^-inf = 0
      float ls = 0.0f;
      u32x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int a = e >> 1, q = 2 * (e & 1);
        const float p0 = __builtin_amdgcn_exp2f(st[a][q] - off), p1 = __builtin_amdgcn_exp2f(st[a][q + 1] - off);
        ls += p0 + p1;
        // (a page whose step is NaN must not reach rows that see none of it)
        w[e] = f2bf2(st[a][q] == -INFINITY ? 0.0f : p0 * vs, st[a][q + 1] == -INFINITY ? 0.0f : p1 * vs);
      }
      const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, w);
      ls += __shfl_xor(ls, 16);
      ls += __shfl_xor(ls, 32);
      if (__any(mn != m[h])) {
        const float alpha = m[h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[h] - mn);
        l[h] *= alpha;
#pragma unroll
        for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * alpha;
      }
      l[h] += ls;
      m[h] = mn;
#pragma unroll
      for (int j = 0; j < JD; ++j) acc[h][j] = mfma(vf[j], pb, acc[h][j]);
    }
  }
#pragma unroll
  for (int h = 0; h < R; ++h) {
#pragma unroll
    for (int j = 0; j < JD; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) s_o[wave][16 * h + r][16 * j + 4 * g + q] = acc[h][j][q];
    if (g == 0) {
      s_ml[wave][16 * h + r][0] = m[h];
      s_ml[wave][16 * h + r][1] = l[h];
    }
  }
  __syncthreads();
  for (int e = tid; e < 16 * R * DH; e += 256) {
    const int rr = e / DH, ch = e % DH, row = row0 + rr;
    if (row >= rows) break;
    float mm = -INFINITY, ll = 0.0f, o = 0.0f;
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_ml[w][rr][0]);
    for (int w = 0; w < 4; ++w) {
      const float mw = s_ml[w][rr][0];
      const float f = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - mm);
      ll += mw == -INFINITY ? s_ml[w][rr][1] : f * s_ml[w][rr][1];
      o += f * s_o[w][rr][ch];
    }
    if (!s.ok) ll = NAN;
    const int64_t t = int64_t(s.b) + row / G, hd = int64_t(u) * G + row % G;
    if (splits == 1) {
      O[(t * H + hd) * DH + ch] = f2bf(o / ll);
      if (LSE && ch == 0) LSE[hd * c.T + t] = mm + log2f(ll);
    } else {
      const int64_t at = (int64_t(split) * c.T + t) * H + hd;
      part[at * DH + ch] = o;
      if (ch == 0) {
        float* ml = part + int64_t(splits) * c.T * H * DH + 2 * at;
        ml[0] = mm;
        ml[1] = ll;
      }
    }
  }
}

// Joins the splits of a row: one thread per output value.
__global__ __launch_bounds__(256) void cache_join_kernel(CacheArgs c, int H, int DH,
                                                         const float* __restrict__ part, int splits,
                                                         uint16_t* __restrict__ O, float* __restrict__ LSE) {
  const Seq s = seq_of(c, blockIdx.y);
  const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (e >= int64_t(s.n) * H * DH) return;
  const int64_t at = int64_t(s.b) * H + e / DH;
  const int ch = int(e % DH);
  const float* ml = part + int64_t(splits) * c.T * H * DH;
  float mm = -INFINITY, ll = 0.0f, o = 0.0f;
  for (int k = 0; k < splits; ++k) mm = fmaxf(mm, ml[2 * (k * c.T * H + at)]);
  for (int k = 0; k < splits; ++k) {
    const float mk = ml[2 * (k * c.T * H + at)], lk = ml[2 * (k * c.T * H + at) + 1];
    const float f = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - mm);
    ll += mk == -INFINITY ? lk : f * lk;
    if (mk != -INFINITY) o += f * part[(k * c.T * H + at) * DH + ch];
  }
  O[at * DH + ch] = f2bf(o / ll);
  if (LSE && ch == 0) LSE[(at % H) * c.T + at / H] = mm + log2f(ll);
}

}  // namespace

hipError_t cache_append(const CacheArgs& c, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                        const void* V, int64_t ldv, bool in_bf16, int H, const float* rope, int64_t n_rope,
                        const float* s_a, uint16_t* Qout, hipStream_t st) {
  const dim3 grid(unsigned((c.max_q + c.P - 2) / c.P + 1), unsigned(c.Hkv), unsigned(c.n_seq));
  const unsigned lds = unsigned(c.P) * c.d * 4;
  if (in_bf16) {
    RowIn<uint16_t> in{static_cast<const uint16_t*>(Q), static_cast<const uint16_t*>(K),
                       static_cast<const uint16_t*>(V), ldq, ldk, ldv};
    hipLaunchKernelGGL(cache_append_kernel<uint16_t>, grid, dim3(AT), lds, st, c, in, H, rope, n_rope, s_a, Qout);
  } else {
    RowIn<float> in{static_cast<const float*>(Q), static_cast<const float*>(K), static_cast<const float*>(V),
                    ldq, ldk, ldv};
    hipLaunchKernelGGL(cache_append_kernel<float>, grid, dim3(AT), lds, st, c, in, H, rope, n_rope, s_a, Qout);
  }
  return hipGetLastError();
}

hipError_t cache_read(const CacheArgs& c, const int32_t* begin, const int32_t* row_start, int64_t rows,
                      int max_rows, void* K, void* V, bool bf16, hipStream_t st) {
  const dim3 grid(unsigned(max_rows), unsigned(c.n_seq));
  if (bf16)
    hipLaunchKernelGGL(cache_read_kernel<uint16_t>, grid, dim3(256), 0, st, c, begin, row_start, rows,
                       static_cast<uint16_t*>(K), static_cast<uint16_t*>(V));
  else
    hipLaunchKernelGGL(cache_read_kernel<float>, grid, dim3(256), 0, st, c, begin, row_start, rows,
                       static_cast<float*>(K), static_cast<float*>(V));
  return hipGetLastError();
}

int cache_attend_splits(int n_seq, int Hkv, int H, int max_q, int64_t max_len) {
  const int64_t tiles = (int64_t(max_q) * (H / Hkv) + 15) / 16;
  const int64_t wgs = tiles * Hkv * n_seq, chunks = (max_len + 31) / 32;
  const int64_t want = (1024 + wgs - 1) / wgs;
  return int(std::max<int64_t>(1, std::min<int64_t>({want, chunks / 8, 64})));
}

hipError_t cache_attend(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                        float* ws, int splits, hipStream_t st) {
  const int64_t rows = int64_t(c.max_q) * (H / c.Hkv);
  auto go = [&](auto dh, auto rr) {
    constexpr int DH = decltype(dh)::value, R = decltype(rr)::value;
    const dim3 grid(unsigned((rows + 16 * R - 1) / (16 * R) * splits), unsigned(c.Hkv), unsigned(c.n_seq));
    hipLaunchKernelGGL((cache_attend_kernel<DH, R>), grid, dim3(256), 0, st, c, Q, ldq, H, O, LSE, ws, splits);
  };
  if (c.d == 64) go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else go(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const dim3 grid(unsigned((int64_t(c.max_q) * H * c.d + 255) / 256), unsigned(c.n_seq));
  hipLaunchKernelGGL(cache_join_kernel, grid, dim3(256), 0, st, c, H, c.d, ws, splits, O, LSE);
  return hipGetLastError();
}

}  // namespace oq
