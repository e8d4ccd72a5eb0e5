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
#include "kv_cache.h"

namespace oq {
namespace {

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

// ------------------------------------------------------------------ append
// One workgroup takes one page's worth of one sequence's new tokens: the keys and
// values of one head (blockIdx.y < kv heads), or a slice of the queries.  A thread
// takes channels p .. p + 3 and p + d/2 .. of a head's row at a time.  HBM-bound for
// prompts (each row read once, written once: two prompts of up to 4,096 tokens and
// ten single ones, 64 heads, float32, 84 us, 99 with all of it read back, 4.1 TB/s);
// for decoding a few loads deep (8 sequences, 32 heads, 7 us; 63, 6 us where no page
// fills up).  A
// page that fills up is gathered in LDS, the keys as rows, the values in the
// window's operand order, so that its codes are written in whole 16-byte pieces.
template <typename TI>
__global__ __launch_bounds__(512) void cache_append_kernel(CacheArgs c, RowIn<TI> in, int H,
                                                          const float* __restrict__ rope, int64_t n_rope,
                                                          const float* __restrict__ sa,
                                                          uint16_t* __restrict__ Qout, bool direct) {
  extern __shared__ uint4 s_page[];                        // K [P][d], then V in operand order, bf16
  __shared__ int s_max[2][8];
  const int u = blockIdx.y, tid = threadIdx.x, AT = blockDim.x;
  const int d = c.d, half = d / 2, P = c.P;
  const Unit un = unit_of(c.n_seq, int(blockIdx.x), direct, [&](int j) {
    const Seq s = seq_of(c, j);
    return s.n == 0 ? 0 : s.ok ? ((s.L + s.n - 1) >> c.lgP) - (s.L >> c.lgP) + 1 : (s.n + P - 1) >> c.lgP;
  });
  if (un.i < 0) return;
  const int i = un.i;
  const Seq s = seq_of(c, i);
  if (s.n == 0) return;
  const int slice = u - c.Hkv, slices = int(gridDim.y) - c.Hkv;
  if (!s.ok) {                                             // nothing is cached; the queries are NaN
    if (slice < 0) return;
    const int64_t wide = int64_t(H) * d, at = int64_t(un.k) * P, n = min(int64_t(s.n), at + P) * wide;
    for (int64_t e = at * wide + tid + int64_t(AT) * slice; e < n; e += int64_t(AT) * slices)
      Qout[int64_t(s.b) * wide + e] = 0x7fc0;
    return;
  }
  const int pg0 = s.L >> c.lgP, pg = pg0 + un.k, end = s.L + s.n;
  const int lo = max(s.L, pg * P), hi = min(end, (pg + 1) * P);
  if (lo >= hi) return;
  if (slice >= 0) {
    append_queries(c, s, in, H, rope, n_rope, sa, Qout, lo, hi, slice, slices, [](int pos) { return pos; });
    return;
  }
  const int last = (end - 1) >> c.lgP;
  const int64_t win = int64_t(P) * d;
  auto window = [&](uint16_t* w, int page) { return w + ((int64_t(s.slot) * 2 + (page & 1)) * c.Hkv + u) * win; };
  const bool full = hi == (pg + 1) * P;
  uint16_t* sk = reinterpret_cast<uint16_t*>(s_page);
  uint16_t* sv = sk + P * d;
  const bool old_rows = (s.L & (P - 1)) != 0;
  if (full && un.k == 0 && old_rows) {
    // the page's rows from before the call (with whatever lies behind them: the new
    // rows overwrite that)
    const uint4* kw = reinterpret_cast<const uint4*>(window(c.kw, pg));
    const uint4* vw = reinterpret_cast<const uint4*>(window(c.vw, pg));
    for (int e = tid; e < P * d / 8; e += AT) {
      s_page[e] = kw[e];
      s_page[P * d / 8 + e] = vw[e];
    }
    __syncthreads();
  }
  // a key or value row's eight channels to the window
  auto to_window = [&](int page, int r, int p, bool key, uint2 a, uint2 b) {
    if (key) {
      uint16_t* kw = window(c.kw, page) + r * d + p;
      *reinterpret_cast<uint2*>(kw) = a;
      *reinterpret_cast<uint2*>(kw + half) = b;
    } else {
      uint16_t* vw = window(c.vw, page);
      const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        vw[vw_at(r, p + e, d)] = uint16_t(w[e >> 1] >> (16 * (e & 1)));
        vw[vw_at(r, p + half + e, d)] = uint16_t(w[2 + (e >> 1)] >> (16 * (e & 1)));
      }
    }
  };
  auto key_row = [&](int pos, int p, uint2& a, uint2& b) {
    float x[4], y[4];
    turned4(in.k + (int64_t(s.b) + (pos - s.L)) * in.ldk + int64_t(u) * d, rope, n_rope, pos, p, half, x, y);
    if (sa) {
      float s0[4], s1[4];
      load4(sa + u * d + p, s0);
      load4(sa + u * d + p + half, s1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = x[e] * s0[e];
        y[e] = y[e] * s1[e];
      }
    }
    a = pack4(x);
    b = pack4(y);
  };
  auto value_row = [&](int pos, int p, uint2& a, uint2& b) {
    const TI* row = in.v + (int64_t(s.b) + (pos - s.L)) * in.ldv + int64_t(u) * d;
    float x[4];
    load4(row + p, x);
    a = pack4(x);
    load4(row + p + half, x);
    b = pack4(x);
  };
  // this page's new rows: to LDS where the page fills up, to the window where it is
  // one of the last two.  A later page of the same half as the first must wait until
  // the first one's old rows are read: the first page's workgroup writes it.
  const bool keep = pg >= last - 1 && !(un.k > 0 && old_rows && ((pg - pg0) & 1) == 0);
  const int lq = c.lgd - 3, q4 = 1 << lq;
  for (int e = tid; e < (hi - lo) * 2 * q4; e += AT) {
    const int pos = lo + (e >> (lq + 1)), p = 4 * (e & (q4 - 1));
    uint2 a, b;
    const bool key = (e >> lq) & 1;
    const int r = pos - pg * P;
    if (key) key_row(pos, p, a, b);
    else value_row(pos, p, a, b);
    if (full) {
      if (key) {
        *reinterpret_cast<uint2*>(sk + r * d + p) = a;
        *reinterpret_cast<uint2*>(sk + r * d + p + half) = b;
      } else {
        const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sv[vw_at(r, p + k, d)] = uint16_t(w[k >> 1] >> (16 * (k & 1)));
          sv[vw_at(r, p + half + k, d)] = uint16_t(w[2 + (k >> 1)] >> (16 * (k & 1)));
        }
      }
    }
    if (keep) to_window(pg, r, p, key, a, b);
  }
  if (!full) return;
  __syncthreads();
  if (un.k == 0 && old_rows) {
    for (int page = max(last - 1, pg0 + 1); page <= last; ++page) {
      if ((page - pg0) & 1) continue;
      const int a0 = page * P, b0 = min(end, a0 + P);
      for (int e = tid; e < (b0 - a0) * 2 * q4; e += AT) {
        const int pos = a0 + (e >> (lq + 1)), p = 4 * (e & (q4 - 1));
        const bool key = (e >> lq) & 1;
        uint2 a, b;
        if (key) key_row(pos, p, a, b);
        else value_row(pos, p, a, b);
        to_window(page, pos - a0, p, key, a, b);
      }
    }
  }
  page_to_codes(c, i, pg, u, s_page, s_max);
}

// ------------------------------------------------------------------ read
// One workgroup: one head of 32 tokens of a sequence (a chunk lies in one page):
// its operand pieces to rows in LDS, then to the output (the batch above 15 us, the
// rate of a copy; 8 sequences' single rows 7 us, a few loads deep).
template <typename TO>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs c, const int32_t* __restrict__ begin,
                                                         const int32_t* __restrict__ row_start, int64_t rows,
                                                         int max_rows, TO* __restrict__ K, TO* __restrict__ V,
                                                         bool direct) {
  __shared__ float s_x[32][132];
  const int u = blockIdx.y, d = c.d, tid = threadIdx.x, lk = c.lgd - 6;
  // rows b .. e - 1 of sequence j, from its position `first` on
  int64_t first, b, e;
  auto range = [&](int j) {
    first = max(begin[j], 0);
    b = max(row_start[j], 0);
    e = min(min(int64_t(row_start[j + 1]), rows), b + max_rows);
  };
  const Unit un = unit_of(c.n_seq, int(blockIdx.x), direct, [&](int j) {
    range(j);
    return b < e ? int((first % 32 + (e - b) + 31) / 32) : 0;
  });
  if (un.i < 0) return;
  const int i = un.i;
  const Seq s = seq_of(c, i);
  range(i);
  // chunks of 32 from the one that holds the first position
  const int64_t t0 = (first / 32 + un.k) * 32;
  const int64_t at0 = b + (t0 - first);                   // the chunk's first row of the output
  if (b >= e || at0 >= e) return;
  const int64_t total = int64_t(s.L) + s.n, win = int64_t(c.P) * d;
  const bool ok = s.ok && begin[i] >= 0 && t0 < total;
  const int pg = ok ? int(t0 >> c.lgP) : 0, tin = ok ? int(t0) & (c.P - 1) : 0;
  const bool full = ok && int64_t(pg + 1) * c.P <= total;
  const int id = full ? page_of(c, i, pg) : -1;
  const int64_t blk = int64_t(max(id, 0)) * c.Hkv + u;
  const int64_t wat = ok ? ((int64_t(s.slot) * 2 + (pg & 1)) * c.Hkv + u) * win : 0;
  for (int kv = 0; kv < 2; ++kv) {
    TO* out = kv ? V : K;
    if (!out) continue;
    const float h = id < 0 ? NAN : kv ? c.vs[blk] : c.ks[blk];
    if (kv) __syncthreads();
    if (full) {
      for (int p = tid; p < 2 * d; p += 256) {             // 16-byte pieces
        const int ln = p & 63, f = p >> 6, r = ln & 15, g = ln >> 4;
        const uint4 q = reinterpret_cast<const uint4*>((kv ? c.vc : c.kc) + blk * win + tin * d)[p];
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float x = float(int8_t(w[k >> 2] >> (8 * (k & 3)))) * h;
          if (kv) s_x[16 * ((k >> 2) & 1) + 4 * g + (k & 3)][32 * f + 16 * (k >> 3) + r] = x;
          else s_x[16 * (f >> lk) + r][64 * (f & ((1 << lk) - 1)) + 16 * g + k] = x;
        }
      }
    } else if (ok) {
      for (int p = tid; p < 4 * d; p += 256) {
        const uint16_t* src = (kv ? c.vw : c.kw) + wat + int64_t(tin) * d;
        float x[8];
        load8(src + 8 * p, x);
        const int ln = p & 63, f = p >> 6, r = ln & 15, g = ln >> 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (kv) s_x[16 * (k >> 2) + 4 * g + (k & 3)][16 * f + r] = x[k];
          else s_x[p >> (c.lgd - 3)][8 * (p & (d / 8 - 1)) + k] = x[k];
        }
      }
    }
    __syncthreads();
    for (int p = tid; p < 32 * d / 8; p += 256) {
      const int t = p >> (c.lgd - 3), ch = 8 * (p & (d / 8 - 1));
      const int64_t pos = t0 + t, row = at0 + t;
      if (pos < first || row < b || row >= e) continue;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = ok && pos < total ? s_x[t][ch + k] : NAN;
      store8(out + (row * c.Hkv + u) * d + ch, x);
    }
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

OQ_DEV Out out_of(uint16_t* O, float* LSE, float* part, int splits, int split, int H, int64_t T, int64_t units,
                  int64_t unit, int unit_rows, int DH) {
  return {O, LSE, part, splits, H, T, (split * units + unit) * unit_rows, splits * units * unit_rows * DH};
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
template <int DH, int R>
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
  const float sc = 1.4426950408889634f / sqrtf(float(DH));

  bf16x8_t qf[R][KS];
  int lim[R];                                            // the last token this lane's row sees
  f32x4_t acc[R][JD];
  float m[R], l[R], vref = VREF0;
#pragma unroll
  for (int h = 0; h < R; ++h) {
    const int row = min(16 * h + r, rows - 1);
    lim[h] = s.L + row / G;
    load_q<DH>(qf[h], Q, ldq, s, u, G, row, g);
    m[h] = -INFINITY;
    l[h] = 0.0f;
#pragma unroll
    for (int j = 0; j < JD; ++j) acc[h][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int nch = (total + 31) / 32, ncode = (total >> c.lgP) * (P / 32), per = (nch + splits - 1) / splits;
  const int c0 = split * per + wave, c1 = min(nch, (split + 1) * per), c1c = min(c1, ncode);
  auto id_of = [&](int ch) { return ch < c1c ? c.table[int64_t(i) * c.max_pages + ((32 * ch) >> c.lgP)] : -1; };
  auto scores = [&](int h, const bf16x8_t (&kf)[2][KS], int t0, f32x4_t (&st)[2]) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      st[a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) st[a] = mfma(kf[a][k], qf[h][k], st[a]);
#pragma unroll
      for (int q = 0; q < 4; ++q) st[a][q] = t0 + 16 * a + 4 * g + q > lim[h] ? -INFINITY : st[a][q];
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
          if (lim[h] >= t0) l[h] = NAN;
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
        scores(h, kf, t0, st);
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
      if (bad && lim[h] >= t0 + __ffs(int(bad)) - 1) l[h] = NAN;
      f32x4_t st[2];
      scores(h, kf, t0, st);
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
    if (!s.ok) ll = NAN;
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
template <int DH, int R, bool TWO>
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
  const int total = s.ok ? s.L + s.n : 0, closed = total & ~(P - 1);
  const float sc = 1.4426950408889634f / sqrtf(float(DH));

  bf16x8_t qf[R][KS];                                    // f16 (times 1 / qs), bf16 for the open page
  float qs[R];
  int lim[R];                                            // the last token this lane's row sees
  f32x4_t acc[R][JD];
  float m[R], l[R], vref[TWO ? R : 1];
  auto row_of = [&](int h) { return min(row0 + 16 * (R * wave + h) + r, rows - 1); };
#pragma unroll
  for (int h = 0; h < R; ++h) {
    lim[h] = s.L + row_of(h) / G;
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
  const int first_lim = s.L + row0 / G;                  // what every row of the tile sees
  const int seen = s.ok ? s.L + min(row0 + QW - 1, rows - 1) / G + 1 : 0;
  const int nt = (seen + 63) / 64, per = (nt + splits - 1) / splits;
  const int k0 = split * per, k1 = min(nt, (split + 1) * per);
  const int ntc = closed / 64;                           // tiles of full pages only
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
    if (t0 + 63 > first_lim) {
#pragma unroll
      for (int h = 0; h < R; ++h)
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (t0 + 16 * a + 4 * g + q > lim[h]) st[h][a][q] = -INFINITY;
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
        if (bad0 && lim[h] >= t0 + __ffs(int(bad0)) - 1) l[h] = NAN;
        if (bad1 && lim[h] >= t0 + 32 + __ffs(int(bad1)) - 1) l[h] = NAN;
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
      if constexpr (TWO) unit(vref[h], lim[h] >= t0 + 32);
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
    if (!s.ok) l[h] = NAN;
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

}  // namespace

hipError_t cache_append(const CacheArgs& c, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                        const void* V, int64_t ldv, bool in_bf16, int H, const float* rope, int64_t n_rope,
                        const float* s_a, uint16_t* Qout, hipStream_t st) {
  // 512 threads where the pages' workgroups are few (a page that fills up is then a
  // long walk: 25 us against 33 for 11 sequences of 142 tokens at one key head),
  // 256 where they fill the card (29 us against 33 for four chunks of up to 325
  // tokens at 32 key heads).  Query slices: eight items of a thread each.
  // Pages: of the longest sequence times n_seq, or, where that is less, what T tokens
  // in at most min(n_seq, T) sequences can touch.
  const int64_t grid_pages = ((int64_t(c.max_q) + c.P - 2) / c.P + 1) * c.n_seq;
  const int64_t most = c.T / c.P + 2 * std::min<int64_t>(c.n_seq, c.T);
  const bool direct = grid_pages <= most || grid_pages * c.Hkv <= 1024;
  const int64_t units = direct ? grid_pages : most, items = std::min<int64_t>(c.max_q, c.P) * H * (c.d / 8);
  const unsigned threads = units * c.Hkv <= 1024 ? 512 : 256;
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(items / (8 * threads), 65535 - c.Hkv));
  const dim3 grid(unsigned(units), unsigned(c.Hkv + slices));
  const unsigned lds = unsigned(c.P) * c.d * 4;
  auto go = [&](auto ti) {
    using TI = decltype(ti);
    const RowIn<TI> in{static_cast<const TI*>(Q), static_cast<const TI*>(K), static_cast<const TI*>(V), ldq, ldk, ldv};
    hipLaunchKernelGGL(cache_append_kernel<TI>, grid, dim3(threads), lds, st, c, in, H, rope, n_rope, s_a, Qout,
                       direct);
  };
  if (in_bf16) go(uint16_t{});
  else go(float{});
  return hipGetLastError();
}

hipError_t cache_read(const CacheArgs& c, const int32_t* begin, const int32_t* row_start, int64_t rows,
                      int max_rows, void* K, void* V, bool bf16, hipStream_t st) {
  const int64_t grid_chunks = ((int64_t(max_rows) + 30) / 32 + 1) * c.n_seq;
  const int64_t most = rows / 32 + 2 * std::min<int64_t>(c.n_seq, rows);
  const bool direct = grid_chunks <= most || grid_chunks * c.Hkv <= 1024;
  const dim3 grid(unsigned(direct ? grid_chunks : most), unsigned(c.Hkv));
  if (bf16)
    hipLaunchKernelGGL(cache_read_kernel<uint16_t>, grid, dim3(256), 0, st, c, begin, row_start, rows, max_rows,
                       static_cast<uint16_t*>(K), static_cast<uint16_t*>(V), direct);
  else
    hipLaunchKernelGGL(cache_read_kernel<float>, grid, dim3(256), 0, st, c, begin, row_start, rows, max_rows,
                       static_cast<float*>(K), static_cast<float*>(V), direct);
  return hipGetLastError();
}

// How a call is cut up, from its sizes alone (the lengths are on the device: a table
// wider than they need makes the plan one for longer sequences; a prompt of 512 tokens
// at 32 heads 17.6 us, 30.3 with a table eight times as wide, which takes 128-row tiles;
// 8 sequences decoding at 1,000 tokens 11.2 and 12.4; 64 of them the same).
// Rows of a key head: up to 32 go to the row kernel, more to the tile kernel; a batch of
// prompts and decoding sequences (fewer tokens than three quarters of n_seq * max_q) runs
// both, each on its own: of 16 sequences over 2,000 tokens with 64 or 1 new ones at 32
// heads, 8 key heads, 84 -> 81 us at 63% of n_seq * max_q, 75 -> 61 at 51%, 66 -> 50 at 8%,
// but 91 -> 97 at 88% (at 75% 86 and 84); 32 key heads 93 -> 96, 91 -> 89, 86 -> 82, 98
// -> 113 (95 and 102).
// Rows of a tile: 128 where such tiles, split into pieces of 512 tokens, are more than
// the 512 workgroups that run at once, else 64 (a prompt of 512 tokens at 32 heads
// 23 -> 17 us, of 1,024 38 -> 29, but 256 tokens over 8,192 62 -> 71).
// Splits of the tokens: as many as fill the card once with the row kernel, three
// workgroups of 16 rows to a compute unit or two of 32, to the nearest (against 1024
// rounded up: one row of 8 heads over 131,072 tokens 53 -> 49 us, four rows 62 -> 53,
// 16 sequences of four over up to 4,096 33 -> 26; rounded down, 64 sequences of up to
// 8,192 102 -> 107); 1024 where it has only a ragged batch's shorter sequences (8 of up
// to 48 tokens 154 -> 130).  Tiles of 128 rows are bound by arithmetic, and 512 workgroups
// are all that run at once (4 times as many: 119 -> 145 us for 512 rows a head over
// 32768 tokens, the join's traffic), or twice that for several sequences, whose lengths
// the host does not know.  Uneven ones gain (18 chunks of up to 84 tokens over up to 5,318
// at 32 heads, 8 key heads, 176 -> 138 us; 8 of up to 512 over up to 4,096, 8 heads, 135
// -> 112), equal ones lose 3 to 7% (8 of 512 over 4,096, 8 heads, 116 -> 123; 4 of 256
// over 8,192 184 -> 190; 18 of 84 over 5,318, 16 heads, 140 -> 149); three times loses for
// most.  64 rows or fewer wait for memory like the row
// kernel's and lengths are ragged, so 1536 (200 -> 126 us for 35 sequences of up to 27
// tokens at 4 key heads of 8, up to 16741 long; 252 -> 136 us for 8 of 48, up to 16384).
// Smallest splits: 256 tokens for the row kernel (one row over 1,024 tokens, 32 heads, 8.9
// us, with 512 10.7, with 128 8.7; 256 tokens 5.8 unsplit, 7.7 in two; over 2,048 to 16,384
// within 15% either way), 512 for the tile kernel (512 tokens 17.4, with 256 24.7; 64 over
// 4,096, 32 heads, 24.2 and 26.6, with 1,024 33.5; at 8 heads 22.0 and 18.2, 31.5).
AttendPlan cache_attend_plan(int n_seq, int Hkv, int H, int64_t tokens, int max_q, int64_t max_len, int d) {
  const int64_t rows = int64_t(max_q) * (H / Hkv), heads = int64_t(n_seq) * Hkv;
  const bool mixed = n_seq > 1 && 4 * tokens < 3 * int64_t(n_seq) * max_q;
  AttendPlan p;
  // (a double: sizes that are refused later must not wrap here)
  const double wide = double((rows + 127) / 128) * double(heads) * double(std::max<int64_t>(1, max_len / 512));
  p.tile_rows = rows <= 32 ? 0 : rows <= 64 || wide <= 512 ? 64 : 128;
  p.row_rows = rows <= 16 ? 16 : rows <= 32 || mixed ? 32 : 0;
  auto cut = [](int64_t want, int64_t most) { return int(std::max<int64_t>(1, std::min(want, most))); };
  const int64_t fit = p.tile_rows ? 1024 : p.row_rows == 16 ? 768 : 512;
  p.few = p.row_rows ? cut((fit + heads / 2) / heads, std::min<int64_t>(128, max_len / 256)) : 1;
  p.units = 0;
  p.order = BY_PLACE;
  p.levels = 0;
  if (p.tile_rows) {
    // tiles of the longest sequence times n_seq, or, where that is less, what T tokens can fill
    const int64_t G = H / Hkv, grid = (rows + p.tile_rows - 1) / p.tile_rows * n_seq;
    const int64_t most = tokens * G / p.tile_rows + std::min<int64_t>(n_seq, tokens * G / (p.row_rows + 1));
    p.levels = std::max(max_len * G, rows) / p.tile_rows + 1;   // (a chunk that does not fit counts from 0)
    if (n_seq > 1 && n_seq <= 32 && rows > p.tile_rows && p.levels <= (1 << 24)) p.order = BY_LEVEL;
    else if (grid > most && grid > 1024 / Hkv) p.order = BY_SEARCH;
    p.units = p.order == BY_PLACE ? grid : std::min(grid, most);
  }
  const int64_t tiles = p.units * Hkv;
  p.many = tiles ? cut((rows <= 64 ? 1536 : n_seq > 1 ? 1024 : 512) / tiles, std::min<int64_t>(64, max_len / 512)) : 1;
  p.few_floats = p.few > 1 ? size_t(p.few) * size_t(heads) * size_t(p.row_rows) * size_t(d + 2) : 0;
  p.many_floats = p.many > 1 ? size_t(p.many) * size_t(tiles) * size_t(p.tile_rows) * size_t(d + 2) : 0;
  return p;
}

hipError_t cache_attend(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                        float* ws, const AttendPlan& p, hipStream_t st) {
  const int G = H / c.Hkv;
  float* ws_many = ws + p.few_floats;
  auto few = [&](auto dh, auto rr) {
    constexpr int DH = decltype(dh)::value, R = decltype(rr)::value;
    const dim3 grid(unsigned(p.few), unsigned(c.Hkv), unsigned(c.n_seq));
    hipLaunchKernelGGL((cache_attend_kernel<DH, R>), grid, dim3(256), 0, st, c, Q, ldq, H, O, LSE, ws, p.few);
  };
  auto many_of = [&](auto dh, auto rr, auto two) {
    constexpr int DH = decltype(dh)::value, R = decltype(rr)::value;
    constexpr bool TWO = decltype(two)::value;
    const dim3 grid(unsigned(p.units * p.many * c.Hkv));
    hipLaunchKernelGGL((cache_attend_tile_kernel<DH, R, TWO>), grid, dim3(256), 0, st, c, Q, ldq, H, O, LSE, ws_many,
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

}  // namespace oq
