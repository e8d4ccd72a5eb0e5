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
// Ragged batches: unit w of all sequences' units (pages, row tiles), in the order of
// the sequences, as (sequence, its unit); (-1, 0) past the last.  By every wave for
// itself.  Batches whose grid of n_seq times the longest sequence's units is no
// larger than the units' bound, or small, are numbered directly instead (a search
// costs some 4 us: 15 chunks of up to 152 tokens 26 us, searched 30).  With 63
// decoding sequences beside a prompt of 4,096 tokens at 64 heads the empty
// workgroups of the direct grid took most of the time: attention 2,340 us, searched
// 390; the append 786 and 45.
struct Unit {
  int i, k;
};
template <typename F>
OQ_DEV Unit unit_of(int n_seq, int w, bool direct, F units) {
  if (direct) return {w % n_seq, w / n_seq};
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < n_seq; i0 += 64) {
    const int n = i0 + lane < n_seq ? units(i0 + lane) : 0;
    int sum = min(n, 0x3fffffff);                          // (row ranges may overlap: no sum overflows)
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(sum, off);
      if (lane >= off) sum = min(sum + o, 0x3fffffff);
    }
    const uint64_t past = __ballot(sum > w);
    if (past) {
      const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const int before = l > 0 ? __shfl(sum, l - 1) : 0;
      return {__builtin_amdgcn_readfirstlane(i0 + l), __builtin_amdgcn_readfirstlane(w - before)};
    }
    w -= __shfl(sum, 63);
  }
  return {-1, 0};
}

// A tree of drafted tokens: node j of a sequence's new tokens stands behind the sequence
// (parent -1) or behind an earlier node.  It sees the sequence's tokens and its own
// ancestors, itself counted: a bit each, TREE_MAX nodes at most.
constexpr int TREE_MAX = 128;
// By the whole workgroup (at least TREE_MAX threads): every node's ancestors, each round
// doubling the part of its way that a node knows.  False where a parent is none.
OQ_DEV bool tree_ancestors(const int32_t* parent, const Seq& s, uint32_t (*s_anc)[4], int* s_up) {
  const int j = threadIdx.x;
  const bool in = j < s.n;
  uint32_t m[4];
  int up = -1;
  bool good = true;
  if (in) {
    const int p = parent[int64_t(s.b) + j];
    good = p >= -1 && p < j;
    up = good ? p : -1;
#pragma unroll
    for (int w = 0; w < 4; ++w) s_anc[j][w] = m[w] = (j >> 5) == w ? 1u << (j & 31) : 0u;
    s_up[j] = up;
  }
  good = __syncthreads_and(good);
  while (true) {
    int further = -1;
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < 4; ++w) m[w] |= s_anc[up][w];
      further = s_up[up];
    }
    if (!__syncthreads_or(up >= 0)) return good;
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < 4; ++w) s_anc[j][w] = m[w];
      s_up[j] = up = further;
    }
    __syncthreads();
  }
}
// Which of the 32 tokens from t0 on a node sees: the sequence's L, its ancestors behind them.
OQ_DEV uint32_t tree_sees(const uint32_t (*s_anc)[4], int node, int L, int t0) {
  const int o = t0 - L, w = o >> 5;
  const uint32_t lo = unsigned(w) < 4u ? s_anc[node][w] : 0u, hi = unsigned(w + 1) < 4u ? s_anc[node][w + 1] : 0u;
  const uint32_t kin = uint32_t(((uint64_t(hi) << 32) | lo) >> (o & 31));
  return kin | (o >= 0 ? 0u : o <= -32 ? ~0u : (1u << -o) - 1u);
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

// 32 tokens of a full page as they lie in memory, with the page's steps.
template <int DH>
struct Codes {
  u32x4_t k[DH / 32], v[DH / 32];
  float ks, vs;
  // (entry: the table's, checked here: at its load the check would wait for memory)
  OQ_DEV void load(const CacheArgs& c, int entry, int u, int tin, int lane) {
    const int id = page_in(c, entry);
    const int64_t blk = int64_t(max(id, 0)) * c.Hkv + u;
    ks = id < 0 ? NAN : c.ks[blk];
    vs = id < 0 ? NAN : c.vs[blk];
    const int64_t at = blk * c.P * DH + tin * DH;
    const u32x4_t* kp = reinterpret_cast<const u32x4_t*>(c.kc + at) + lane;
    const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(c.vc + at) + lane;
    // read once: past the caches (64 sequences of up to 8,192 tokens 130 -> 111 us)
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) k[j] = __builtin_nontemporal_load(kp + 64 * j);
#pragma unroll
    for (int j = 0; j < DH / 32; ++j) v[j] = __builtin_nontemporal_load(vp + 64 * j);
  }
};

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
OQ_DEV Out out_of(uint16_t* O, float* LSE, float* part, int splits, int split, int H, int64_t T, int64_t units,
                  int64_t unit, int unit_rows, int DH) {
  return {O, LSE, part, splits, H, T, (split * units + unit) * unit_rows, splits * units * unit_rows * DH};
}
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

// Few rows (decoding): one workgroup takes 16 R rows of one key head and a split's
// tokens, dealt to its four waves in chunks of 32.  Codes go from memory straight
// into operand registers, the next chunk's in flight meanwhile; each wave has a
// softmax of its own, the four are joined in LDS and the splits by a second kernel.
//   S^T = K Q^T: a lane holds query row r, tokens 4 g + 0..3 of both 16-token
//   tiles, which is the B operand of O^T = V^T P^T as it stands.
// HBM-bound: 131,072 tokens x 8 key heads 44 us (6.1 TB/s, some from the last-level
// cache), 64 sequences of up to 8,192 x 8 heads 100 us (5.1 TB/s).  Three waves to a
// SIMD and loads past the caches: 256 sequences of up to 1,024 x 32 heads took 218 us,
// 254 with two waves, 302 without either.  Sequences with more rows are the tile
// kernel's.
template <int DH, int R, bool TREE>
__global__ __launch_bounds__(256, R == 1 ? 3 : 2) void cache_attend_kernel(CacheArgs c, const uint16_t* __restrict__ Q,
                                                           int64_t ldq, int H, uint16_t* __restrict__ O,
                                                           float* __restrict__ LSE, float* __restrict__ part,
                                                           int splits) {
  constexpr int KS = DH / 32, JD = DH / 16;
  __shared__ float s_o[4][16 * R][DH + 4];
  __shared__ float s_ml[4][16 * R][2];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = blockIdx.x, u = blockIdx.y, i = blockIdx.z;
  const int G = H / c.Hkv, P = c.P;
  const Seq s = seq_of(c, i);
  const int rows = s.n * G;
  if (rows == 0 || rows > 16 * R) return;
  const int total = s.ok ? s.L + s.n : 0;
  // the tokens in full pages: of a tree's, drafts fill no page
  const int closed = (TREE ? (s.ok ? s.L : 0) : total) & ~(P - 1);
  const float sc = 1.4426950408889634f / sqrtf(float(DH));

  bf16x8_t qf[R][KS];
  int lim[R];                                            // the last token this lane's row sees; of a tree, its node
  f32x4_t acc[R][JD];
  float m[R], l[R], vref = VREF0;
#pragma unroll
  for (int h = 0; h < R; ++h) {
    const int row = min(16 * h + r, rows - 1);
    lim[h] = TREE ? row / G : s.L + row / G;
    load_q<DH>(qf[h], Q, ldq, s, u, G, row, g);
    m[h] = -INFINITY;
    l[h] = 0.0f;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int nch = (total + 31) / 32, ncode = closed / 32, per = (nch + splits - 1) / splits;
  const int c0 = split * per + wave, c1 = min(nch, (split + 1) * per), c1c = min(c1, ncode);
  __shared__ uint32_t s_anc[TREE ? TREE_MAX : 1][4];
  __shared__ int s_up[TREE ? TREE_MAX : 1];
  bool tree_ok = true;
  if (TREE && c1 > ncode) tree_ok = tree_ancestors(c.parent, s, s_anc, s_up);
  auto id_of = [&](int ch) { return ch < c1c ? c.table[int64_t(i) * c.max_pages + ((32 * ch) >> c.lgP)] : -1; };
  auto scores = [&](int h, const bf16x8_t (&kf)[2][KS], int t0, f32x4_t (&st)[2], auto open) {
    constexpr bool OPEN = decltype(open)::value;
    const uint32_t sees = TREE && OPEN ? tree_sees(s_anc, lim[h], s.L, t0) >> (4 * g) : 0u;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      st[a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) st[a] = mfma(kf[a][k], qf[h][k], st[a]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (!TREE) st[a][q] = t0 + 16 * a + 4 * g + q > lim[h] ? -INFINITY : st[a][q];
        else if constexpr (OPEN) st[a][q] = sees & (1u << (16 * a + q)) ? st[a][q] : -INFINITY;
      }
    }
  };
  auto rescale = [&](int h, float alpha) {
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * alpha;
    }
  };
  int ch = c0;
  if (ch < c1c) {
    Codes<DH> nx;
    nx.load(c, id_of(ch), u, 32 * ch & (P - 1), lane);
    int idn = id_of(ch + 4);
    for (; ch < c1c; ch += 4) {
      const int t0 = 32 * ch;
      Codes<DH> cur = nx;
      if (ch + 4 < c1c) {
        nx.load(c, idn, u, 32 * (ch + 4) & (P - 1), lane);
        idn = id_of(ch + 8);
      }
      // a page that stands for NaN: rows that see it are NaN, any finite step will do
      if (!(cur.ks < INFINITY && cur.vs < INFINITY)) {
#pragma unroll
        for (int h = 0; h < R; ++h)
          if (TREE || lim[h] >= t0) l[h] = NAN;
        cur.ks = cur.vs = 1.0f;
      }
      cur.ks = fmaxf(cur.ks, KS_MIN);
      cur.vs = fmaxf(cur.vs, VS_MIN);
      const float vr = fmaxf(vref, pow2_above(cur.vs));
      const float shrink = vref * pow2_inv(vr);
      const Step sp[1] = {step_of(step_parts(cur.ks * sc, cur.vs), vr, true)};
      bf16x8_t kf[2][KS];
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < KS / 2; ++j) {
          const u32x4_t w = cur.k[a * (KS / 2) + j];
          kf[a][2 * j] = codes_bf16(w[0], w[1]);
          kf[a][2 * j + 1] = codes_bf16(w[2], w[3]);
        }
      f16x8_t pb[R];
#pragma unroll
      for (int h = 0; h < R; ++h) {
        f32x4_t st[2];
        scores(h, kf, t0, st, std::false_type{});
        rescale(h, softmax_step<1>(st, sp, m[h], l[h]) * shrink);
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_f16(st[e >> 1][2 * (e & 1)], st[e >> 1][2 * (e & 1) + 1]);
        pb[h] = __builtin_bit_cast(f16x8_t, w);
      }
      vref = vr;
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const f16x8_t v0 = codes_f16(cur.v[j][0], cur.v[j][1]), v1 = codes_f16(cur.v[j][2], cur.v[j][3]);
#pragma unroll
        for (int h = 0; h < R; ++h) {
          acc[h][2 * j] = mfma_h(v0, pb[h], acc[h][2 * j]);
          acc[h][2 * j + 1] = mfma_h(v1, pb[h], acc[h][2 * j + 1]);
        }
      }
    }
  }
  if (ch < c1) {                                         // the open page's step is 1
    const float vr = fmaxf(vref, 1.0f), shrink = vref * pow2_inv(vr);
#pragma unroll
    for (int h = 0; h < R; ++h)
#pragma unroll
      for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * shrink;
    vref = vr;
  }
  for (; ch < c1; ch += 4) {
    const int t0 = 32 * ch;
    bf16x8_t kf[2][KS], vf[JD];
    const Window<DH> win(c, s, u, t0, total, lane);
    unsigned bad = 0;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[a][k] = __builtin_bit_cast(bf16x8_t, win.key(a, k));
#pragma unroll
    for (int j = 0; j < JD; ++j) vf[j] = __builtin_bit_cast(bf16x8_t, win.value(j));
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int k = 0; k < KS; ++k) win.check_key(__builtin_bit_cast(u32x4_t, kf[a][k]), a, bad);
#pragma unroll
    for (int j = 0; j < JD; ++j)
      vf[j] = __builtin_bit_cast(bf16x8_t, win.check_value(__builtin_bit_cast(u32x4_t, vf[j]), bad));
    bad = wave_or(bad);
    const Step sp[1] = {step_of(step_parts(sc, 1.0f), vref, false)};
#pragma unroll
    for (int h = 0; h < R; ++h) {
      if (bad && (TREE ? (bad & tree_sees(s_anc, lim[h], s.L, t0)) != 0 : lim[h] >= t0 + __ffs(int(bad)) - 1))
        l[h] = NAN;
      f32x4_t st[2];
      scores(h, kf, t0, st, std::true_type{});
      rescale(h, softmax_step<1>(st, sp, m[h], l[h]));
      u32x4_t wh, wl;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = st[e >> 1][2 * (e & 1)], y = st[e >> 1][2 * (e & 1) + 1];
        wh[e] = f2bf2(x, y);
        wl[e] = f2bf2(x - __uint_as_float(wh[e] << 16), y - __uint_as_float(wh[e] & 0xffff0000u));
      }
#pragma unroll
      for (int j = 0; j < JD; ++j) {
        acc[h][j] = mfma(vf[j], __builtin_bit_cast(bf16x8_t, wh), acc[h][j]);
        acc[h][j] = mfma(vf[j], __builtin_bit_cast(bf16x8_t, wl), acc[h][j]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < R; ++h) {
    l[h] = row_sum(l[h]);
#pragma unroll
    for (int j = 0; j < JD; ++j)
      *reinterpret_cast<f32x4_t*>(&s_o[wave][16 * h + r][16 * j + 4 * g]) = acc[h][j] * (vref / WUNIT);
    if (g == 0) {
      s_ml[wave][16 * h + r][0] = m[h];
      s_ml[wave][16 * h + r][1] = l[h];
    }
  }
  __syncthreads();
  const Out out = out_of(O, LSE, part, splits, split, H, c.T, int64_t(c.n_seq) * c.Hkv, int64_t(i) * c.Hkv + u, 16 * R, DH);
  for (int e = tid; e < 4 * R * DH; e += 256) {          // 16 R rows of DH / 4 fours
    const int row = e / (DH / 4), c4 = 4 * (e % (DH / 4));
    if (row >= rows) break;
    float mm = -INFINITY, ll = 0.0f;
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_ml[w][row][0]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < 4; ++w) {
      const float mw = s_ml[w][row][0], lw = s_ml[w][row][1];
      const float f = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - mm);
      ll += mw == -INFINITY ? lw : f * lw;               // (no token, or NaN)
      const float4 x = *reinterpret_cast<const float4*>(&s_o[w][row][c4]);
      o = make_float4(o.x + f * x.x, o.y + f * x.y, o.z + f * x.z, o.w + f * x.w);
    }
    if (!s.ok || !tree_ok) ll = NAN;
    const int64_t t = int64_t(s.b) + row / G, hd = int64_t(u) * G + row % G;
    put4(out, row, t, hd, DH, c4, o, ll);
    if (c4 == 0) put_ml(out, row, t, hd, mm, ll);
  }
}

// Tiles of `qw` rows of one key head's rows: the w-th of all sequences' as (sequence,
// tile), (-1, 0) past the last.  Where up to 32 sequences have several tiles each, the
// tiles that see the most tokens come first, against an order by place (the k-th tile
// from the end of each sequence in turn): 16 chunks of up to 512 tokens over up to
// 4,096, 16 heads, 188 -> 142 us; two of up to 2,048 over up to 4,096, 32 heads, 216
// -> 202; but 60 chunks of up to 256 tokens 157 -> 172, and 8 of 16 tokens (one tile
// each) 63 -> 77.  A tile's level is its place from the sequence's beginning, in
// tiles; from level b up there are sum_i clamp(end_i - b, 0, tiles_i), which 64 lanes
// evaluate at 64 levels at once.
enum TileOrder { BY_PLACE, BY_SEARCH, BY_LEVEL };
OQ_DEV Unit row_tile(const CacheArgs& c, int G, int qw, int rows_min, int w, int order, int levels) {
  auto tiles = [&](const Seq& s) { return s.n * G < rows_min ? 0 : (s.n * G + qw - 1) / qw; };
  if (order != BY_LEVEL) {
    Unit un = unit_of(c.n_seq, w, order == BY_PLACE, [&](int j) { return tiles(seq_of(c, j)); });
    // a sequence's last tile first
    if (un.i >= 0) un.k = (order == BY_PLACE ? (c.max_q * G + qw - 1) / qw : tiles(seq_of(c, un.i))) - 1 - un.k;
    return un;
  }
  const int lane = threadIdx.x & 63;
  int n = 0, first = 0;                                    // the lane's sequence: tiles, the first one's level
  if (lane < c.n_seq) {
    const Seq s = seq_of(c, lane);
    n = tiles(s);
    first = s.ok ? int(int64_t(s.L) * G / qw) : 0;
  }
  const uint64_t some = __ballot(n > 0);
  auto from = [&](int b) {                                 // tiles of level b and up
    int sum = 0;
    for (uint64_t left = some; left; left &= left - 1) {
      const int i = __ffsll(static_cast<unsigned long long>(left)) - 1;
      const int ni = __builtin_amdgcn_readlane(n, i), end = __builtin_amdgcn_readlane(first, i) + ni;
      sum += min(max(end - b, 0), ni);
    }
    return sum;
  };
  int lo = 0, hi = levels;                                 // the level is in [lo, hi)
  while (true) {
    const int step = (hi - lo + 63) / 64, b = lo + lane * step, over = from(b);
    const uint64_t past = __ballot(b < hi && over > w);
    if (!past) return {-1, 0};
    lo += (__popcll(past) - 1) * step;
    if (step == 1) break;
    hi = min(hi, lo + step);
  }
  uint64_t at = __ballot(n > 0 && first <= lo && lo < first + n);
  for (int j = w - from(lo + 1); j > 0; --j) at &= at - 1;
  const int i = __ffsll(static_cast<unsigned long long>(at)) - 1;
  return {i, lo - __builtin_amdgcn_readlane(first, i)};
}

// Many rows (prompts): one workgroup of four waves takes 64 R rows of one key head,
// 16 R per wave, over tiles of 64 tokens.  The waves turn a tile's codes into f16
// operands once, in LDS, a tile ahead; the raw codes of the one after are in
// flight meanwhile.  Two workgroups to a compute unit.  Neither unit is busy all the
// time: over a whole launch the vector units (softmax, conversion) 48%, the matrix
// units 26%, at 1.5 of 2 waves a SIMD, so a wave's products, softmax and products again
// mostly follow one another, and a quarter of the wave slots is empty at the ends.  Two
// chunks of up to 2,048 tokens over up to 4,096, 32 heads of 128, 203 us, 652 TFLOP/s;
// 4,096 tokens at 64 heads, 8 key heads, 339 us, 812 TFLOP/s.
//
// Queries enter Q K^T as f16 too, each row scaled by a power of two that puts its
// largest entry between 2^14 and 2^15: bf16's 8 bits fit, and what is lost is below
// 2^-39 of that entry.  (Of a row below 2^-71 what is lost is below 2^-110: a smaller
// factor times KS_MIN would leave fp32.)
//
// TWO: pages of 32 tokens, a tile's chunks lie in two pages.  A row's unit of the weights
// is its own then: rows that see only the first chunk must not lose bits to the other
// page's V step (two chunks of up to 2,048 tokens over up to 4,096, 32 heads of 128, 210
// -> 217 us).  Larger pages hold both chunks: one step and one unit for all rows.
template <int DH, int R, bool TWO, bool TREE>
__global__ __launch_bounds__(256, 2) void cache_attend_tile_kernel(CacheArgs c, const uint16_t* __restrict__ Q,
                                                                       int64_t ldq, int H,
                                                                       uint16_t* __restrict__ O,
                                                                       float* __restrict__ LSE,
                                                                       float* __restrict__ part, int splits,
                                                                       int rows_min, int units, int order, int levels) {
  constexpr int KS = DH / 32, JD = DH / 16, QW = 64 * R;
  constexpr int TILE = 64 * DH / 8;                      // 16-byte pieces of one operand's tile
  constexpr int CW = 2, LPW = JD / CW;                   // waves of a chunk, loads of a wave
  static_assert(LPW == KS, "half a chunk's keys are one 16-token tile");
  __shared__ u32x4_t s_k[2][TILE], s_v[2][TILE];
  __shared__ float4 s_step[2][2];                        // [buffer][chunk], step_parts
  __shared__ unsigned s_bad[2][2][CW];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // key heads fastest (an XCD keeps its heads' pages in its L2)
  const int G = H / c.Hkv, P = c.P;
  int x = int(blockIdx.x);
  const int u = x % c.Hkv;
  x /= c.Hkv;
  const int split = x % splits, w = x / splits;
  const Unit un = row_tile(c, G, QW, rows_min, w, order, levels);
  if (un.i < 0) return;
  const int i = un.i;
  const Seq s = seq_of(c, i);
  const int rows = s.n * G, row0 = un.k * QW;
  if (rows < rows_min || row0 >= rows) return;
  const int total = s.ok ? s.L + s.n : 0, closed = (TREE ? (s.ok ? s.L : 0) : total) & ~(P - 1);
  const float sc = 1.4426950408889634f / sqrtf(float(DH));

  bf16x8_t qf[R][KS];                                    // f16 (times 1 / qs), bf16 for the open page
  float qs[R];
  int lim[R];                                            // the last token this lane's row sees; of a tree, its node
  f32x4_t acc[R][JD];
  float m[R], l[R], vref[TWO ? R : 1];
  auto row_of = [&](int h) { return min(row0 + 16 * (R * wave + h) + r, rows - 1); };
#pragma unroll
  for (int h = 0; h < R; ++h) {
    lim[h] = TREE ? row_of(h) / G : s.L + row_of(h) / G;
    load_q<DH>(qf[h], Q, ldq, s, u, G, row_of(h), g);
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(float(qf[h][k][e])));
    const int e = min(max(int(__float_as_uint(row_max(top)) >> 23), 56), 253);
    const float up = __uint_as_float(uint32_t(268 - e) << 23);   // 2^(14 - exponent)
    qs[h] = __uint_as_float(uint32_t(e - 14) << 23);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4_t w;
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = pack_f16(float(qf[h][k][2 * q]) * up, float(qf[h][k][2 * q + 1]) * up);
      qf[h][k] = __builtin_bit_cast(bf16x8_t, w);
    }
    m[h] = -INFINITY;
    l[h] = 0.0f;
    vref[TWO ? h : 0] = VREF0;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int first_lim = TREE ? s.L - 1 : s.L + row0 / G;  // what every row of the tile sees
  const int seen = TREE ? total : s.ok ? s.L + min(row0 + QW - 1, rows - 1) / G + 1 : 0;
  const int nt = (seen + 63) / 64, per = (nt + splits - 1) / splits;
  const int k0 = split * per, k1 = min(nt, (split + 1) * per);
  const int ntc = closed / 64;                           // tiles of full pages only
  __shared__ uint32_t s_anc[TREE ? TREE_MAX : 1][4];
  __shared__ int s_up[TREE ? TREE_MAX : 1];
  bool tree_ok = true;
  if (TREE && k1 > ntc) tree_ok = tree_ancestors(c.parent, s, s_anc, s_up);
  // this wave's share of a tile: the keys or the values of chunk cc
  const int cc = wave >> 1, hw = wave & 1;
  const bool vals = hw != 0;
  u32x4_t raw[LPW];
  float ks = 0.0f, vs = 0.0f;
  // The page of this wave's chunk of tile t (a page number is a load of its own: it
  // is fetched a tile before the codes are).  Page numbers and steps come by vector
  // loads, though the whole wave reads one word: scalar loads share a counter with
  // the LDS reads, whose waits would then last until memory has answered.
  int zero = 0;
  asm("" : "+v"(zero));
  auto id_of = [&](int t) {
    return t < k1 && 64 * t + 32 * cc < closed
               ? c.table[int64_t(i) * c.max_pages + ((64 * t + 32 * cc) >> c.lgP) + zero]
               : -1;
  };
  int idn = id_of(k0);
  auto load = [&](int t) __attribute__((always_inline)) {   // tile t, if its chunk is in a full page
    const int t0 = 64 * t + 32 * cc, id = page_in(c, __builtin_amdgcn_readfirstlane(idn));
    if (t0 < closed) {
      const int64_t blk = int64_t(max(id, 0)) * c.Hkv + u;
      if (hw == 0) {
        ks = id < 0 ? NAN : c.ks[blk + zero];
        vs = id < 0 ? NAN : c.vs[blk + zero];
      }
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>((vals ? c.vc : c.kc) + blk * P * DH + (t0 & (P - 1)) * DH) + lane;
#pragma unroll
      for (int j = 0; j < LPW; ++j) raw[j] = p[64 * j];
      idn = id_of(t + 1);
    }
  };
  auto steps = [&](int b) {
    if (hw == 0 && lane == 0) {
      const bool fine = ks < INFINITY && vs < INFINITY;
      s_step[b][cc] = step_parts(fine ? fmaxf(ks, KS_MIN) * sc : sc, fine ? fmaxf(vs, VS_MIN) : 1.0f);
      s_bad[b][cc][0] = fine ? 0u : 1u;
    }
    if (hw > 0 && lane == 0) s_bad[b][cc][hw] = 0u;
  };
  // Operands of tile t into buffer b, fragment f of a chunk (64 lanes) at 64 f: f16,
  // or bf16 where the tile reaches into the open page (from ntc on).
  auto store = [&](int t, int b) __attribute__((always_inline)) {
    const int t0 = 64 * t + 32 * cc;
    u32x4_t* dst = (vals ? s_v[b] : s_k[b]) + cc * JD * 64 + lane;
    if (t0 < closed) {
      if (t < ntc) {
#pragma unroll
        for (int j = 0; j < 2 * LPW; ++j)
          dst[64 * j] = __builtin_bit_cast(u32x4_t, codes_f16(raw[j / 2][2 * (j & 1)], raw[j / 2][2 * (j & 1) + 1]));
      } else {
#pragma unroll
        for (int j = 0; j < 2 * LPW; ++j)
          dst[64 * j] = __builtin_bit_cast(u32x4_t, codes_bf16(raw[j / 2][2 * (j & 1)], raw[j / 2][2 * (j & 1) + 1]));
      }
      steps(b);
    } else {
      // (past every row's limit zeros, any finite operands)
      unsigned bad = 0;
      if (t0 < seen) {
        const Window<DH> win(c, s, u, t0, total, lane);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          u32x4_t w[LPW];
#pragma unroll
          for (int j = 0; j < LPW; ++j) w[j] = vals ? win.value(LPW * half + j) : win.key(half, j);
#pragma unroll
          for (int j = 0; j < LPW; ++j) {
            if (vals) w[j] = win.check_value(w[j], bad);
            else win.check_key(w[j], half, bad);
            dst[64 * (half * LPW + j)] = w[j];
          }
        }
      } else {
#pragma unroll
        for (int f = 0; f < 2 * LPW; ++f) dst[64 * f] = u32x4_t{0u, 0u, 0u, 0u};
      }
      bad = wave_or(bad);
      if (lane == 0) {
        if (hw == 0) s_step[b][cc] = step_parts(sc, 1.0f);
        s_bad[b][cc][hw] = bad;
      }
    }
  };
  if (k0 < k1) {
    load(k0);
    store(k0, 0);
    if (k0 + 1 < k1) load(k0 + 1);
  }
  // OPEN: the tile reaches into the open page; the weights enter as pairs of bf16 terms.
  auto tile = [&](int t, auto open) __attribute__((always_inline)) {
    constexpr bool OPEN = decltype(open)::value;
    const int b = (t - k0) & 1, t0 = 64 * t;
    __syncthreads();                                     // tile t is in buffer b, the other is free
    // operands are read from LDS AH ahead of their products
    constexpr int AH = 4;
    const u32x4_t *sk = &s_k[b][lane], *sv = &s_v[b][lane];
    u32x4_t kf[AH];
#pragma unroll
    for (int x = 0; x < AH; ++x) kf[x] = sk[64 * x];
    if (t + 1 < k1) {
      store(t + 1, b ^ 1);
      if (t + 2 < k1) load(t + 2);
    }
    f32x4_t st[R][4];
#pragma unroll
    for (int x = 0; x < 4 * KS; ++x) {
      const int a = x / KS, k = x % KS;
      const u32x4_t f = kf[x % AH];
#pragma unroll
      for (int h = 0; h < R; ++h) {
        if (k == 0) st[h][a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if constexpr (OPEN) st[h][a] = mfma(__builtin_bit_cast(bf16x8_t, f), qf[h][k], st[h][a]);
        else st[h][a] = mfma_h(__builtin_bit_cast(f16x8_t, f), __builtin_bit_cast(f16x8_t, qf[h][k]), st[h][a]);
      }
      if (x + AH < 4 * KS) kf[x % AH] = sk[64 * (x + AH)];
      __builtin_amdgcn_sched_barrier(0);
    }
    if ((OPEN || !TREE) && t0 + 63 > first_lim) {
#pragma unroll
      for (int h = 0; h < R; ++h)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const uint32_t sees = TREE ? tree_sees(s_anc, lim[h], s.L, t0 + 32 * (a >> 1)) >> (4 * g) : 0u;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (TREE ? !(sees & (1u << (16 * (a & 1) + q))) : t0 + 16 * a + 4 * g + q > lim[h]) st[h][a][q] = -INFINITY;
        }
    }
    unsigned bad0 = 0, bad1 = 0;
#pragma unroll
    for (int w = 0; w < CW; ++w) {
      bad0 |= s_bad[b][0][w];
      bad1 |= s_bad[b][1][w];
    }
    if (bad0 | bad1) {
      // (a full page that stands for NaN: from its chunk's first token on)
#pragma unroll
      for (int h = 0; h < R; ++h) {
        if constexpr (!TREE) {
          if (bad0 && lim[h] >= t0 + __ffs(int(bad0)) - 1) l[h] = NAN;
          if (bad1 && lim[h] >= t0 + 32 + __ffs(int(bad1)) - 1) l[h] = NAN;
        } else if constexpr (!OPEN) {
          l[h] = NAN;
        } else if ((bad0 & tree_sees(s_anc, lim[h], s.L, t0)) | (bad1 & tree_sees(s_anc, lim[h], s.L, t0 + 32))) {
          l[h] = NAN;
        }
      }
    }
    const float4 q0 = s_step[b][0], q1 = TWO ? s_step[b][1] : q0;
    float shrink;
    Step s0, s1;
    auto unit = [&](float& vref, bool both) {
      const float vr = fmaxf(vref, TWO && both ? fmaxf(pow2_above(q0.y), pow2_above(q1.y)) : pow2_above(q0.y));
      shrink = vref * pow2_inv(vr);
      vref = vr;
      s0 = step_of(q0, vr, !OPEN || (TWO && t0 < closed));
      s1 = TWO ? step_of(q1, vr, !OPEN) : s0;
    };
    if constexpr (!TWO) unit(vref[0], true);
    u32x4_t vf[AH];
#pragma unroll
    for (int x = 0; x < AH; ++x) vf[x] = sv[64 * x];
#pragma unroll
    for (int h = 0; h < R; ++h) {
      if constexpr (TWO) unit(vref[h], TREE || lim[h] >= t0 + 32);   // (a tree's rows all meet the window's step)
      Step sp[2] = {s0, s1};
      if constexpr (!OPEN) {
        sp[0].f *= qs[h];
        sp[1].f *= qs[h];
      }
      const float alpha = softmax_step<2>(st[h], sp, m[h], l[h]) * shrink;
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int j = 0; j < JD; ++j) acc[h][j] = acc[h][j] * alpha;
      }
    }
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      u32x4_t ph[R], pl[OPEN ? R : 1];
#pragma unroll
      for (int h = 0; h < R; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = st[h][2 * k2 + (e >> 1)][2 * (e & 1)], p1 = st[h][2 * k2 + (e >> 1)][2 * (e & 1) + 1];
          if constexpr (OPEN) {
            ph[h][e] = f2bf2(p0, p1);
            pl[h][e] = f2bf2(p0 - __uint_as_float(ph[h][e] << 16), p1 - __uint_as_float(ph[h][e] & 0xffff0000u));
          } else {
            ph[h][e] = pack_f16(p0, p1);
          }
        }
#pragma unroll
      for (int j = 0; j < JD; ++j) {
        const int x = k2 * JD + j;
        const u32x4_t v = vf[x % AH];
#pragma unroll
        for (int h = 0; h < R; ++h) {
          if constexpr (OPEN) {
            acc[h][j] = mfma(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, ph[h]), acc[h][j]);
            acc[h][j] = mfma(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, pl[h]), acc[h][j]);
          } else {
            acc[h][j] = mfma_h(__builtin_bit_cast(f16x8_t, v), __builtin_bit_cast(f16x8_t, ph[h]), acc[h][j]);
          }
        }
        if (x + AH < 2 * JD) vf[x % AH] = sv[64 * (x + AH)];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  int t = k0;
  for (; t < min(k1, ntc); ++t) tile(t, std::false_type{});
  if (t < k1) {
#pragma unroll
    for (int h = 0; h < R; ++h) load_q<DH>(qf[h], Q, ldq, s, u, G, row_of(h), g);
  }
  for (; t < k1; ++t) tile(t, std::true_type{});
  const Out out = out_of(O, LSE, part, splits, split, H, c.T, int64_t(units) * c.Hkv, int64_t(w) * c.Hkv + u, QW, DH);
#pragma unroll
  for (int h = 0; h < R; ++h) {
    l[h] = row_sum(l[h]);
    const int row = row0 + 16 * (R * wave + h) + r;
    if (row >= rows) continue;
    if (!s.ok || !tree_ok) l[h] = NAN;
    const int64_t tok = int64_t(s.b) + row / G, hd = int64_t(u) * G + row % G;
#pragma unroll
    for (int j = 0; j < JD; ++j) {
      const f32x4_t o = acc[h][j] * (vref[TWO ? h : 0] / WUNIT);
      put4(out, row - row0, tok, hd, DH, 16 * j + 4 * g, make_float4(o[0], o[1], o[2], o[3]), l[h]);
    }
    if (g == 0) put_ml(out, row - row0, tok, hd, m[h], l[h]);
  }
}

// Joins a row's splits: DH / 4 lanes of four output values each, NG groups of them
// dealing the splits among themselves; 256 threads take RW rows of a unit, of the
// row kernel's first.
struct JoinArgs {
  const float *few, *many;           // shares of the two kernels
  int few_splits, many_splits, row_rows, tile_rows, units;
  int few_rows;                      // rows of a unit of the row kernel that can be in use
  int few_blocks;
  int order, levels;
};
template <int DH, int NG>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheArgs c, int H, JoinArgs a, uint16_t* __restrict__ O,
                                                         float* __restrict__ LSE) {
  constexpr int Q4 = DH / 4, RW = 256 / (Q4 * NG);
  __shared__ float4 s_o[NG][RW][Q4];
  __shared__ float2 s_ml[NG][RW];
  const int G = H / c.Hkv;
  const bool few = int(blockIdx.x) < a.few_blocks;
  const int unit_rows = few ? a.row_rows : a.tile_rows, blocks = ((few ? a.few_rows : a.tile_rows) + RW - 1) / RW;
  const int bid = int(blockIdx.x) - (few ? 0 : a.few_blocks), unit = bid / blocks, u = unit % c.Hkv;
  const Unit un = few ? Unit{unit / c.Hkv, 0}
                      : row_tile(c, G, a.tile_rows, a.row_rows + 1, unit / c.Hkv, a.order, a.levels);
  if (un.i < 0) return;
  const Seq s = seq_of(c, un.i);
  const int rows = s.n * G, row0 = un.k * unit_rows;
  const int lane = threadIdx.x % Q4, ng = (threadIdx.x / Q4) % NG, rw = threadIdx.x / (Q4 * NG);
  const int at0 = (bid % blocks) * RW;                     // the block's first row of the unit
  if (few != (rows <= a.row_rows) || row0 + at0 >= rows) return;
  const bool in = at0 + rw < unit_rows && row0 + at0 + rw < rows;
  const int row = in ? row0 + at0 + rw : row0 + at0, j = row / G, hd = u * G + row % G;
  const int splits = few ? a.few_splits : a.many_splits;
  const int64_t units = int64_t(few ? c.n_seq : a.units) * c.Hkv, at = int64_t(unit) * unit_rows + (row - row0);
  const float* part = few ? a.few : a.many;
  const float2* ml = reinterpret_cast<const float2*>(part + splits * units * unit_rows * DH);
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto join = [&](float mk, float lk, float4 x) {
    const float mn = fmaxf(m, mk);
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    const float fk = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - mn);
    // (without a token l is 0 or, for a NaN row, NaN: it stays)
    l = (m == -INFINITY ? l : f * l) + (mk == -INFINITY ? lk : fk * lk);
    o = make_float4(f * o.x + fk * x.x, f * o.y + fk * x.y, f * o.z + fk * x.z, f * o.w + fk * x.w);
    m = mn;
  };
#pragma unroll 4
  for (int k = ng; k < splits; k += NG) {
    const int64_t p = k * units * unit_rows + at;
    const float2 w = ml[p];
    join(w.x, w.y, *reinterpret_cast<const float4*>(part + p * DH + 4 * lane));
  }
  if constexpr (NG > 1) {
    s_o[ng][rw][lane] = o;
    if (lane == 0) s_ml[ng][rw] = make_float2(m, l);
    __syncthreads();
    if (ng > 0) return;
#pragma unroll
    for (int k = 1; k < NG; ++k) {
      const float2 w = s_ml[k][rw];
      join(w.x, w.y, s_o[k][rw][lane]);
    }
  }
  if (!in) return;
  const float inv = 1.0f / l;
  const int64_t t = int64_t(s.b) + j;
  *reinterpret_cast<uint2*>(O + (t * H + hd) * DH + 4 * lane) =
      make_uint2(f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv));
  if (LSE && lane == 0) LSE[hd * c.T + t] = lse_of(m, l);
}

template <bool TREE>
hipError_t attend_launch(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                         float* ws, const AttendPlan& p, hipStream_t st) {
  const int G = H / c.Hkv;
  float* ws_many = ws + p.few_floats;
  auto few = [&](auto dh, auto rr) {
    constexpr int DH = decltype(dh)::value, R = decltype(rr)::value;
    const dim3 grid(unsigned(p.few), unsigned(c.Hkv), unsigned(c.n_seq));
    hipLaunchKernelGGL((cache_attend_kernel<DH, R, TREE>), grid, dim3(256), 0, st, c, Q, ldq, H, O, LSE, ws, p.few);
  };
  auto many_of = [&](auto dh, auto rr, auto two) {
    constexpr int DH = decltype(dh)::value, R = decltype(rr)::value;
    constexpr bool TWO = decltype(two)::value;
    const dim3 grid(unsigned(p.units * p.many * c.Hkv));
    hipLaunchKernelGGL((cache_attend_tile_kernel<DH, R, TWO, TREE>), grid, dim3(256), 0, st, c, Q, ldq, H, O, LSE, ws_many,
                       p.many, p.row_rows + 1, int(p.units), p.order, int(p.levels));
  };
  auto many = [&](auto dh, auto rr) {
    if (c.P == 32) many_of(dh, rr, std::true_type{});
    else many_of(dh, rr, std::false_type{});
  };
  auto join = [&](auto dh, auto ng) {
    constexpr int DH = decltype(dh)::value, NG = decltype(ng)::value, RW = 1024 / (DH * NG);
    const int few_rows = int(std::min<int64_t>(p.row_rows, int64_t(c.max_q) * G));
    const int64_t few_blocks = p.few > 1 ? int64_t((few_rows + RW - 1) / RW) * c.Hkv * c.n_seq : 0;
    const int64_t many_blocks = p.many > 1 ? p.units * c.Hkv * (p.tile_rows / RW) : 0;
    const JoinArgs a{ws, ws_many, p.few, p.many, p.row_rows, p.tile_rows, int(p.units), few_rows, int(few_blocks),
                     p.order, int(p.levels)};
    hipLaunchKernelGGL((cache_join_kernel<DH, NG>), dim3(unsigned(few_blocks + many_blocks)), dim3(256), 0, st, c, H,
                       a, O, LSE);
  };
  auto run = [&](auto dh) {
    const std::integral_constant<int, 1> i1{};
    const std::integral_constant<int, 2> i2{};
    if (p.tile_rows == 64) many(dh, i1);
    else if (p.tile_rows) many(dh, i2);
    if (p.row_rows == 16) few(dh, std::integral_constant<int, 1>{});
    else if (p.row_rows) few(dh, std::integral_constant<int, 2>{});
    const int splits = std::max(p.few, p.many);
    if (splits > 8) join(dh, std::integral_constant<int, 8>{});
    else if (splits > 1) join(dh, std::integral_constant<int, 1>{});
  };
  if (c.d == 64) run(std::integral_constant<int, 64>{});
  else run(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace
}  // namespace oq
