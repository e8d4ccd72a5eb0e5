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
  return attend_launch<false>(c, Q, ldq, H, O, LSE, ws, p, st);
}

}  // namespace oq
