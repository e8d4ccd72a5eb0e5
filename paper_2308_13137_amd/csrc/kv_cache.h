// Device code of the paged 8-bit key/value cache that kv_cache.hip (a sequence's new
// tokens in a row) and kv_tree.hip (a tree of drafted tokens) share: what is read
// from device memory and checked, rows on their way into the cache, pages turned
// into codes, and attention.
#pragma once
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

// Where channel c of token t lies in a V window's block.
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

OQ_DEV int page_in(const CacheArgs& c, int p) { return p >= 0 && p < c.n_pages ? p : -1; }
OQ_DEV int page_of(const CacheArgs& c, int i, int pg) { return page_in(c, c.table[int64_t(i) * c.max_pages + pg]); }

// ------------------------------------------------------------------ rows on their way in
template <typename TI>
struct RowIn {
  const TI *q, *k, *v;
  int64_t ldq, ldk, ldv;
};

OQ_DEV void load4(const uint16_t* p, float v[4]) {
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(q.x << 16);
  v[1] = __uint_as_float(q.x & 0xffff0000u);
  v[2] = __uint_as_float(q.y << 16);
  v[3] = __uint_as_float(q.y & 0xffff0000u);
}
OQ_DEV void load4(const float* p, float v[4]) {
  const float4 q = *reinterpret_cast<const float4*>(p);
  v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
}
OQ_DEV uint2 pack4(const float v[4]) { return make_uint2(f2bf2(v[0], v[1]), f2bf2(v[2], v[3])); }

// Channels p .. p + 3 and p + d/2 .. of one head's row: loaded, turned by RoPE, in
// the block step's order of operations.
template <typename TI>
OQ_DEV void turned4(const TI* row, const float* rope, int64_t n_rope, int pos, int p, int half, float (&lo)[4],
                    float (&hi)[4]) {
  load4(row + p, lo);
  load4(row + p + half, hi);
  if (!rope) return;
  if (pos >= n_rope) {
#pragma unroll
    for (int e = 0; e < 4; ++e) lo[e] = hi[e] = NAN;
    return;
  }
  const float4* cs = reinterpret_cast<const float4*>(rope + 2 * (int64_t(pos) * half + p));
  const float4 c0 = cs[0], c1 = cs[1];
  const float c[4] = {c0.x, c0.z, c1.x, c1.z}, sn[4] = {c0.y, c0.w, c1.y, c1.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = lo[e], b = hi[e];
    lo[e] = a * c[e] - b * sn[e];
    hi[e] = b * c[e] + a * sn[e];
  }
}

// Channels p .. p + 3 and p + d/2 .. of one query head's row, U rows (or heads) at
// a time so that their loads are in flight together; turn(pos): where RoPE has the token
// at position pos.
template <typename TI, typename F>
OQ_DEV void append_queries(const CacheArgs& c, const Seq& s, const RowIn<TI>& in, int H, const float* rope,
                           int64_t n_rope, const float* sa, uint16_t* Qout, int lo, int hi, int slice, int slices,
                           F turn) {
  constexpr int U = 4;
  const int d = c.d, half = d / 2, lq = c.lgd - 3, G = H / c.Hkv;
  const int items = ((hi - lo) * H) << lq, step = slices * int(blockDim.x);      // (below 2^28: H <= 2^17)
  for (int e0 = slice * int(blockDim.x) + int(threadIdx.x); e0 < items; e0 += U * step) {
    float x[U][4], y[U][4];
    int64_t at[U];
    int sc[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int e = min(e0 + k * step, items - 1);         // (past the end: the last one, not stored)
      const int row = (e >> lq) / H, hh = (e >> lq) - row * H, p = 4 * (e & ((1 << lq) - 1)), pos = lo + row;
      const int64_t t = int64_t(s.b) + (pos - s.L);
      turned4(in.q + t * in.ldq + int64_t(hh) * d, rope, n_rope, turn(pos), p, half, x[k], y[k]);
      at[k] = (t * H + hh) * d + p;
      sc[k] = (hh / G) * d + p;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (e0 + k * step >= items) break;
      if (sa) {
        float s0[4], s1[4];
        load4(sa + sc[k], s0);
        load4(sa + sc[k] + half, s1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[k][i] = x[k][i] / s0[i];
          y[k][i] = y[k][i] / s1[i];
        }
      }
      *reinterpret_cast<uint2*>(Qout + at[k]) = pack4(x[k]);
      *reinterpret_cast<uint2*>(Qout + at[k] + half) = pack4(y[k]);
    }
  }
}

// A page that has filled up, in LDS (K rows [P][d], then V in the window's operand
// order, bf16), becomes page pg of sequence i, head u, in codes.  By the whole workgroup,
// after a barrier; s_max: two words a wave.
OQ_DEV void page_to_codes(const CacheArgs& c, int i, int pg, int u, const uint4* s_page, int (*s_max)[8]) {
  const int tid = threadIdx.x, AT = blockDim.x, d = c.d, P = c.P;
  const int64_t win = int64_t(P) * d;
  // the largest magnitude as an integer: NaN and infinity order above all
  uint32_t mk = 0, mv = 0;
  auto top = [](uint4 x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max(m, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
    return m;
  };
  for (int e = tid; e < P * d / 8; e += AT) {
    mk = max(mk, top(s_page[e]));
    mv = max(mv, top(s_page[P * d / 8 + e]));
  }
  for (int off = 1; off < 64; off <<= 1) {
    mk = max(mk, uint32_t(__shfl_xor(int(mk), off)));
    mv = max(mv, uint32_t(__shfl_xor(int(mv), off)));
  }
  if ((tid & 63) == 0) {
    s_max[0][tid >> 6] = int(mk);
    s_max[1][tid >> 6] = int(mv);
  }
  __syncthreads();
  for (int w = 0; w < AT / 64; ++w) {
    mk = max(mk, uint32_t(s_max[0][w]));
    mv = max(mv, uint32_t(s_max[1][w]));
  }
  const int id = page_of(c, i, pg);
  if (id < 0) return;
  // a block with a value that is not finite stands for NaN as a whole
  const float hk = mk >= 0x7f80u ? NAN : fmaxf(div_rn(bf2f(uint16_t(mk)), 127.0f), 1e-5f);
  const float hv = mv >= 0x7f80u ? NAN : fmaxf(div_rn(bf2f(uint16_t(mv)), 127.0f), 1e-5f);
  const float rk = div_rn(1.0f, hk), rv = div_rn(1.0f, hv);
  const int64_t blk = int64_t(id) * c.Hkv + u;
  if (tid == 0) {
    c.ks[blk] = hk;
    c.vs[blk] = hv;
  }
  // eight bf16 values as codes
  auto codes8 = [](uint4 x, float r) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t o[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = __uint_as_float((k & 1) ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
      const int q = int(fminf(fmaxf(rintf(v * r), -127.0f), 127.0f));
      o[k >> 2] |= (uint32_t(q) & 255u) << (8 * (k & 3));
    }
    return make_uint2(o[0], o[1]);
  };
  uint4* kd = reinterpret_cast<uint4*>(c.kc + blk * win);
  uint4* vd = reinterpret_cast<uint4*>(c.vc + blk * win);
  const int lk = c.lgd - 6, lv = c.lgd - 5;                // 64- and 32-channel pieces of a row
  for (int e = tid; e < P * d / 16; e += AT) {
    const int ln = e & 63, f = e >> 6, r = ln & 15, g = ln >> 4;
    // keys: piece (16-token tile, 64-channel half, g, r)
    const uint4* ks = &s_page[((f >> lk) * 16 + r) * (d / 8) + (f & ((1 << lk) - 1)) * 8 + 2 * g];
    const uint2 k0 = codes8(ks[0], rk), k1 = codes8(ks[1], rk);
    kd[e] = make_uint4(k0.x, k0.y, k1.x, k1.y);
    // values: piece (32-token chunk, 32 channels, g, r), two channels of eight tokens
    const uint4* vs = &s_page[P * d / 8 + ((f >> lv) * (d / 16) + 2 * (f & ((1 << lv) - 1))) * 64 + ln];
    const uint2 v0 = codes8(vs[0], rv), v1 = codes8(vs[64], rv);
    vd[e] = make_uint4(v0.x, v0.y, v1.x, v1.y);
  }
}

// ------------------------------------------------------------------ attention
// Query x key products on bf16 operands (codes are exact in bf16), weight x
// value products on f16 operands: codes are exact in f16 too, and a weight
// times its page's V step, over a power of two no smaller than any step so far
// (vref), is at most 1 and keeps 11 bits there (8 in bf16: the output's error
// against 64 bits was 2.5e-3 with bf16 weights and is 1.7e-3, a bf16 rounding's
// own, with f16 ones).  It enters times 2^15, so what f16 cannot hold is below
// 2^-40 of the largest.  The window's rows are bf16, of any size: their weights
// enter as a pair of bf16 terms, in the same unit.
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

OQ_DEV f32x4_t mfma_h(f16x8_t a, f16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// int8 -> f16, exact: code + 128 as the low bits of 1024, then minus 1152.
OQ_DEV f16x8_t codes_f16(unsigned a, unsigned b) {
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned v = (i < 2 ? a : b) ^ 0x80808080u;
    const unsigned h = __builtin_amdgcn_perm(0x64646464u, v, (i & 1) ? 0x04030402u : 0x04010400u);
    const f16x2_t f = __builtin_bit_cast(f16x2_t, h) - f16x2_t{(_Float16)1152.0f, (_Float16)1152.0f};
    w[i] = __builtin_bit_cast(unsigned, f);
  }
  return __builtin_bit_cast(f16x8_t, w);
}
OQ_DEV unsigned pack_f16(float a, float b) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2_t{a, b}, f16x2_t));
}

// The smallest power of two no smaller than a positive finite x.
OQ_DEV float pow2_above(float x) { return __uint_as_float((__float_as_uint(x) + 0x7fffffu) & 0x7f800000u); }
OQ_DEV float pow2_inv(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }
constexpr float VREF0 = 7.62939453125e-06f;              // 2^-17, below any step
constexpr float WUNIT = 32768.0f;                        // weights are in units of vref / WUNIT

// 32 tokens of the open page, one bf16 operand at a time.  Rows behind the
// sequence's end are whatever the window holds: their values become zeros (their
// scores are masked).  A value that is not finite would reach every row of the
// product, those that do not see its token too: it enters as zero and its token
// is marked in `bad` (a bit per token), as are those of keys that are not
// finite; rows that see a marked token are made NaN.
template <int DH>
struct Window {
  const uint16_t* k;
  const u32x4_t* v;
  int left, lane;                                        // tokens of the chunk inside the sequence
  OQ_DEV Window(const CacheArgs& c, const Seq& s, int u, int t0, int total, int ln) : left(total - t0), lane(ln) {
    const int pg = t0 >> c.lgP, tin = t0 & (c.P - 1);
    const int64_t at = ((int64_t(s.slot) * 2 + (pg & 1)) * c.Hkv + u) * c.P * DH + int64_t(tin) * DH;
    k = c.kw + at;
    v = reinterpret_cast<const u32x4_t*>(c.vw + at) + ln;
  }
  // operands as they lie there: keys 16 a + r, channels of k-step ks; values 16 j + r
  OQ_DEV u32x4_t key(int a, int ks) const {
    const int r = lane & 15, g = lane >> 4;
    return *reinterpret_cast<const u32x4_t*>(k + (16 * a + r) * DH + 64 * (ks >> 1) + 16 * g + 8 * (ks & 1));
  }
  OQ_DEV u32x4_t value(int j) const { return v[64 * j]; }
  OQ_DEV void check_key(u32x4_t w, int a, unsigned& bad) const {
    const int tok = 16 * a + (lane & 15);
    bool inf = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      inf = inf || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    if (inf && tok < left) bad |= 1u << tok;
  }
  OQ_DEV u32x4_t check_value(u32x4_t w, unsigned& bad) const {
    const int g = lane >> 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int tok = 16 * (e >> 2) + 4 * g + (e & 3);
      const unsigned mask = 0xffffu << (16 * (e & 1));
      const bool out = tok >= left, inf = ((w[e >> 1] >> (16 * (e & 1))) & 0x7f80u) == 0x7f80u;
      if (inf && !out) bad |= 1u << tok;
      if (out || inf) w[e >> 1] &= ~mask;
    }
    return w;
  }
};
OQ_DEV unsigned wave_or(unsigned bad) {
  if (__any(bad != 0))
    for (int off = 1; off < 64; off <<= 1) bad |= __shfl_xor(bad, off);
  return bad;
}

// Four lanes (16 apart) share a query row: v of lane l combined over l ^ 16, l ^ 32.
OQ_DEV float over16(float v, bool sum) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float a = __uint_as_float(x[0]), b = __uint_as_float(x[1]);
  return sum ? a + b : fmaxf(a, b);
}
OQ_DEV float over32(float v, bool sum) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float a = __uint_as_float(x[0]), b = __uint_as_float(x[1]);
  return sum ? a + b : fmaxf(a, b);
}
OQ_DEV float row_max(float v) { return over32(over16(v, false), false); }
OQ_DEV float row_sum(float v) { return over32(over16(v, true), true); }

// A chunk's factors: its scores' (key step x log2(e) / sqrt(d)), and its weights'
// (value step over the unit vref / WUNIT) as an exponent and inverted.
struct Step {
  float f, lw, winv;
};
// A page that was never written has steps of zero and stands for zeros, whatever its
// codes (a pool's pages are used again): its steps count as these.  A score of its codes
// is at most 2^7 d |q| times that, below 2^-25 for queries below 2^20, while the smallest
// query factor leaves a masked score -inf (times zero it would be NaN); every weight
// vanishes as fp16.  (A branch that clears the codes cost the tile kernel 1 to 3%.)
constexpr float KS_MIN = 8.6736173798840355e-19f;        // 2^-60
constexpr float VS_MIN = 8.6736173798840355e-19f;        // 2^-60
// `q` = (key step x scale, value step, its log2, its inverse); vr = vref, a power of two.
OQ_DEV float4 step_parts(float ks_sc, float vs) {
  return make_float4(ks_sc, vs, __builtin_amdgcn_logf(vs), 1.0f / vs);
}
// A full page's weights lie below 2^LW_MIN only where fp16 holds none of them: they stay
// there (their exponential would leave fp32 with V steps far apart), so that the sum,
// which takes the factor out again, has them all.  The open page's step is 1, its factor
// 2^-106 at least, and its weights have to be what they are.
constexpr float LW_MIN = -70.0f, WINV_MAX = 1.1805916207174113e+21f;
OQ_DEV Step step_of(float4 q, float vr, bool full) {
  const float e = float(int(__float_as_uint(vr) >> 23) - 127 - 15);
  const float lw = q.z - e, winv = q.w * (vr * (1.0f / WUNIT));
  return {q.x, full ? fmaxf(lw, LW_MIN) : lw, full ? fminf(winv, WINV_MAX) : winv};
}

// A row's running softmax: m, the maximum of its logits in base 2 rounded up to an
// integer (so it seldom moves), and l, this lane's share of the sum of its
// weights 2^(t - m).  A lane holds the row's scores of NC chunks of 32 tokens (two
// 16-token tiles each), masked ones -inf; they become the weights times their
// chunk's factor, which the sum takes out again.  Returns the factor that the
// row's numerators need.
// (The maximum that passes NaN on takes two values an instruction straight from the
// matrix unit; fmaxf would first quiet each.  A NaN score makes its weight NaN.)
template <int NC>
OQ_DEV float softmax_step(f32x4_t (&st)[2 * NC], const Step (&sp)[NC], float& m, float& l) {
  auto top = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };
  float mt = -INFINITY;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const f32x4_t x = st[2 * c], y = st[2 * c + 1];
    mt = fmaxf(mt, sp[c].f * top(top(top(top(x[0], x[1]), x[2]), top(x[3], y[0])), top(top(y[1], y[2]), y[3])));
  }
  const float mn = fmaxf(m, ceilf(row_max(mt)));
  const float off = mn == -INFINITY ? 0.0f : mn;         // no token seen yet: weights 2^-inf = 0
  const float alpha = mn == m ? 1.0f : m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
  l *= alpha;
  m = mn;
  float f[NC], less = off;
#pragma unroll
  for (int c = 0; c < NC; ++c) f[c] = sp[c].f;
  // From 2^12 on the maximum is subtracted from rounded products before the factor is
  // added: in the one multiply-add below, lw - off would lose the factor's bits, and from
  // 2^24 on the exact product may pass the rounded maximum and its weight fp16 (NaN).
  // Rows that are not there keep their bits.  (It costs prompts 1 to 2%; a second
  // run over the tokens in this form, only where it is needed, cost 10 to 50%, since the
  // kernels then spill.)
  if (__any(fabsf(off) >= 4096.0f)) {
    const bool far = fabsf(off) >= 4096.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int a = 2 * c; a < 2 * c + 2; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float x = __fsub_rn(__fmul_rn(st[a][q], f[c]), off);
          st[a][q] = far ? x : st[a][q];
        }
      f[c] = far ? 1.0f : f[c];
    }
    less = far ? 0.0f : off;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const float e = sp[c].lw - less;
    float w = 0.0f;
#pragma unroll
    for (int a = 2 * c; a < 2 * c + 2; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        st[a][q] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[a][q], f[c], e));
        w += st[a][q];
      }
    l = __builtin_fmaf(w, sp[c].winv, l);
  }
  return alpha;
}
// The query rows of one key head (query x head of the group) in matrix operands.
template <int DH>
OQ_DEV void load_q(bf16x8_t (&qf)[DH / 32], const uint16_t* Q, int64_t ldq, const Seq& s, int u, int G, int row,
                   int g) {
  const uint16_t* qp = Q + (int64_t(s.b) + row / G) * ldq + int64_t(u * G + row % G) * DH;
#pragma unroll
  for (int k = 0; k < DH / 32; ++k)
    qf[k] = __builtin_bit_cast(bf16x8_t,
                               *reinterpret_cast<const u32x4_t*>(qp + 64 * (k >> 1) + 16 * g + 8 * (k & 1)));
}

// Where a row's result goes: the output, or a split's share for cache_join_kernel.
// Shares: numerators [split][unit][row][DH], then (m, l) [split][unit][row]; a unit is
// a workgroup's rows.
struct Out {
  uint16_t* O;
  float *LSE, *part;
  int splits, H;
  int64_t T, at, ml;                 // at: the workgroup's first share; ml: where the pairs begin, in floats
};
// A row whose every score is -inf (an infinite query) is NaN, like its output 0 / 0.
OQ_DEV float lse_of(float m, float l) { return l > 0.0f ? m + log2f(l) : NAN; }
OQ_DEV void put_ml(const Out& o, int row, int64_t t, int64_t hd, float m, float l) {
  if (o.splits > 1) reinterpret_cast<float2*>(o.part + o.ml)[o.at + row] = make_float2(m, l);
  else if (o.LSE) o.LSE[hd * o.T + t] = lse_of(m, l);
}
OQ_DEV void put4(const Out& o, int row, int64_t t, int64_t hd, int DH, int ch, float4 x, float l) {
  if (o.splits > 1) {
    *reinterpret_cast<float4*>(o.part + (o.at + row) * DH + ch) = x;
  } else {
    const float inv = 1.0f / l;
    *reinterpret_cast<uint2*>(o.O + (t * o.H + hd) * DH + ch) =
        make_uint2(f2bf2(x.x * inv, x.y * inv), f2bf2(x.z * inv, x.w * inv));
  }
}

}  // namespace
}  // namespace oq
