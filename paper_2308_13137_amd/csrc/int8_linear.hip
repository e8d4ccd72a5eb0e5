// Y = Q_a(X) Q_w(W)^T + B from integer codes, on 8-bit matrix cores: the linear
// of a weight-activation quantised block.  With a = q_x - 128 and b = q_w - 128
// (both int8) and z' = z - 128,
//   sum_c (q_x - z_x)(q_w - z_w) = sum a b - z_x' (sum b - K z_w') - z_w' sum a,
// where sum a b is exact in int32, sum b comes with the packed weight and
// sum a = sum q_x - 128 K is formed beside the product.  The correction is fp64 (its terms are
// larger than the result), the two scales and the bias fp32.
#include <math.h>

#include <type_traits>

#include "common.h"
#include "serve.h"

namespace oq {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
constexpr uint32_t FLIP = 0x80808080u;      // code -> code - 128 as int8, four at once

OQ_DEV i32x4_t mfma_i8(i32x4_t a, i32x4_t b, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}
OQ_DEV i32x4_t flip(i32x4_t v) {
  return i32x4_t{int(uint32_t(v[0]) ^ FLIP), int(uint32_t(v[1]) ^ FLIP), int(uint32_t(v[2]) ^ FLIP),
                 int(uint32_t(v[3]) ^ FLIP)};
}
// s + the sum of 16 codes (bytes as unsigned): v_sad_u8 against zero, one
// instruction per four (a dot product with ones measured 10-13% of the tiled
// kernel's time, this next to nothing).
OQ_DEV uint32_t sum_codes(i32x4_t v, uint32_t s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_sad_u8(uint32_t(v[i]), 0u, s);
  return s;
}

// Channels n .. n + 3 (past the last: the last) as the epilogue needs them.
struct Chan {
  double zw[4], c[4];        // z_w', sum b - K z_w'
  float hw[4], b[4];
};
OQ_DEV Chan load_chan(const I8Args& a, int64_t n) {
  Chan k;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t o = min(n + i, a.N - 1);
    k.zw[i] = double(a.zw[o]) - 128.0;
    k.c[i] = double(a.wsum[o]) - double(a.K) * k.zw[i];
    k.hw[i] = a.hw[o];
    k.b[i] = a.bias ? a.bias[o] : 0.0f;
  }
  return k;
}
// Channels n .. n + 3 of token t from their integer sums, sum a, h_x and z_x'.
// (Stores of four need rows of a multiple of four.)
template <bool YBF>
OQ_DEV void store_out(const I8Args& a, int64_t t, int64_t n, const Chan& k, i32x4_t acc, int sx, float hx,
                      double zx) {
  float y[4];
  const double s = double(sx);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double v = __builtin_fma(-zx, k.c[i], __builtin_fma(-k.zw[i], s, double(acc[i])));
    y[i] = float(v) * (hx * k.hw[i]);
    if (a.bias) y[i] = y[i] + k.b[i];
  }
  const bool four = (a.N & 3) == 0 && n + 4 <= a.N;
  if (YBF) {
    uint16_t* p = static_cast<uint16_t*>(a.y) + t * a.N + n;
    if (four) {
      *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) p[i] = f2bf(y[i]);
    }
  } else {
    float* p = static_cast<float*>(a.y) + t * a.N + n;
    if (four) {
      *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) p[i] = y[i];
    }
  }
}

// ------------------------------------------------------------------ few tokens
// 16 channels x 16 tokens per workgroup, the K range dealt to its 16 waves in
// one piece each: every weight fragment is one 1-KiB load straight into the
// matrix instruction's registers, U k-steps of them in flight per wave (a
// compute unit needs some 32 KiB in flight to draw its share of HBM's rate).
constexpr int SW = 16;                    // waves per workgroup
template <int U, bool YBF>
__global__ __launch_bounds__(64 * SW) void i8_small_kernel(I8Args a) {
  __shared__ i32x4_t s_acc[SW][64];
  __shared__ uint32_t s_sum[SW][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r = lane & 15, g = lane >> 4;
  const int kt = int(i8_cols(a.K) / 64);
  const int per = (kt + SW - 1) / SW;
  const int k0 = wave * per, k1 = min(kt, k0 + per);
  const i32x4_t* wp = reinterpret_cast<const i32x4_t*>(a.w) + int64_t(blockIdx.x) * kt * 64 + lane;
  const uint8_t* xp = a.x + min(int64_t(r), a.T - 1) * a.K + 16 * g;
  i32x4_t acc = {0, 0, 0, 0};
  uint32_t sx = 0;
  // k-steps k .. k + U - 1; TAIL: those past the wave's range and the columns past
  // K (where the packed weight is zero) are read from inside and do not count
  auto steps = [&](int k, auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    i32x4_t w[U], x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int kk = TAIL ? min(k + i, k1 - 1) : k + i;
      w[i] = wp[64 * kk];
      const bool in = !TAIL || 64 * kk + 16 * g < a.K;
      x[i] = *reinterpret_cast<const i32x4_t*>(xp + (in ? 64 * kk : -16 * g));
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (TAIL && k + i >= k1) break;
      const uint32_t s = sum_codes(x[i], sx);
      sx = !TAIL || 64 * (k + i) + 16 * g < a.K ? s : sx;
      acc = mfma_i8(w[i], flip(x[i]), acc);
    }
  };
  int k = k0;
  for (; k + U < k1; k += U) steps(k, std::false_type{});
  if (k < k1) steps(k, std::true_type{});
  s_acc[wave][lane] = acc;
  s_sum[wave][lane] = sx;
  __syncthreads();
  const int64_t n = 16 * int64_t(blockIdx.x) + 4 * g;
  if (wave > 0 || r >= a.T || n >= a.N) return;
  const Chan kc = load_chan(a, n);
  acc = i32x4_t{0, 0, 0, 0};
  sx = 0;
#pragma unroll
  for (int w = 0; w < SW; ++w) {
    acc += s_acc[w][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) sx += s_sum[w][16 * e + r];
  }
  store_out<YBF>(a, r, n, kc, acc, int(sx) - 128 * int(a.K), a.hx[r], double(a.zx[r]) - 128.0);
}

// ------------------------------------------------------------------ many tokens
// 256 channels x 256 tokens per workgroup, stages of 128 inputs (two k-steps of
// 64), eight waves of 128 x 64.  Both operands come to LDS by asynchronous
// copies: the channels in matrix-operand order, as the weight is packed; the
// tokens as rows of 128 bytes (a copy fetches whole cache lines), chunk c of row
// r at slot c ^ (r & 7) ^ ((r >> 4) & 1), free of bank conflicts for the fragment
// reads.  Tokens' tiles in three buffers, channels' in two, as the bf16 product.
typedef __attribute__((address_space(3))) const char lds_cchar;
constexpr int BT = 256;                   // tile side
constexpr int TNT = 512;                  // threads
constexpr int GROUP = 8;                  // tile rows swept together

OQ_DEV void dma16_s(const void* base, uint32_t vofs, uint32_t lds_addr) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds_addr);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(m0v), "v"(vofs), "s"(base)
      : "memory");
}
OQ_DEV void wait_vm0() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
OQ_DEV void wait_vm4() { asm volatile("s_waitcnt vmcnt(4)" ::: "memory"); }
OQ_DEV i32x4_t frag(lds_cchar* tile, int block, int kk, int lane) {
  typedef __attribute__((address_space(3))) const i32x4_t lds_v4;
  return *(lds_v4*)(tile + (2 * block + kk) * 1024 + 16 * lane);
}
OQ_DEV i32x4_t tok_frag(lds_cchar* tile, int block, int kk, int lane) {
  typedef __attribute__((address_space(3))) const i32x4_t lds_v4;
  const int row = 16 * block + (lane & 15), c = 4 * kk + (lane >> 4);
  return *(lds_v4*)(tile + row * 128 + 16 * (c ^ (row & 7) ^ ((row >> 4) & 1)));
}
// One k-step: 8 groups of four matrix instructions; the next step's 12 fragment
// reads in groups 0..5, one asynchronous copy in each even group when DMA, and
// the next token fragments' conversion and sums (of lanes with `in`) in the last two.
template <bool DMA>
OQ_DEV void i8_step(i32x4_t (&acc)[8][4], uint32_t (&sx)[4], const i32x4_t (&au)[8], const i32x4_t (&bu)[4],
                    lds_cchar* ra, lds_cchar* rb, int kk, int wm, int wn, int lane, i32x4_t (&ad)[8],
                    i32x4_t (&bd)[4], const void* src, const uint32_t (&off)[4], uint32_t wr, int wave) {
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    if (g < 2) {
      bd[2 * g] = tok_frag(rb, 4 * wn + 2 * g, kk, lane);
      bd[2 * g + 1] = tok_frag(rb, 4 * wn + 2 * g + 1, kk, lane);
    } else if (g < 6) {
      ad[2 * g - 4] = frag(ra, 8 * wm + 2 * g - 4, kk, lane);
      ad[2 * g - 3] = frag(ra, 8 * wm + 2 * g - 3, kk, lane);
    } else {
      // (every lane's columns are inside K here: the last stage is not read so)
#pragma unroll
      for (int j = 2 * g - 12; j < 2 * g - 10; ++j) {
        sx[j] = sum_codes(bd[j], sx[j]);
        bd[j] = flip(bd[j]);
      }
    }
    if constexpr (DMA) {
      if ((g & 1) == 0) dma16_s(src, off[g >> 1], wr + (8 * (g >> 1) + wave) * 1024);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[g][j] = mfma_i8(au[g], bu[j], acc[g][j]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <bool YBF>
__global__ __launch_bounds__(TNT, 1) void i8_tile_kernel(I8Args a, int tiles_m, int tiles_n) {
  __shared__ uint4 lds[5 * 2048];         // tokens at 0, 32, 64 KiB, channels at 96, 128 KiB
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r = lane & 15, g4 = lane >> 4;
  // contiguous tiles per XCD, GROUP tile rows swept column by column
  const int nblk = gridDim.x, bid = blockIdx.x;
  const int xcd = bid & 7, local = bid >> 3, q = nblk >> 3, rem = nblk & 7;
  const int L = xcd * q + min(xcd, rem) + local;
  const int group_sz = GROUP * tiles_n;
  const int gr = L / group_sz, first_m = gr * GROUP;
  const int gm = min(GROUP, tiles_m - first_m), li = L - gr * group_sz;
  const int64_t n0 = int64_t(first_m + li % gm) * BT, t0 = int64_t(li / gm) * BT;

  const int kt = int(i8_cols(a.K) / 64), ns = (kt + 1) / 2;
  const int64_t nb = i8_rows(a.N) / 16;
  const int8_t* wbase = a.w + (n0 / 16) * kt * 1024;
  const uint8_t* xbase = a.x + t0 * a.K;
  // copy i of this wave fills 1 KiB of either tile: operand block 4 i + wave / 2,
  // k-step wave % 2 of the channels; rows 8 (8 i + wave) .. + 7 of the tokens, lane
  // l the chunk of row l / 8 that belongs in slot l % 8
  uint32_t aoff[4], boff[4];
  const int half = wave & 1;
  int chunk[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = 4 * i + (wave >> 1);
    aoff[i] = uint32_t(min(int64_t(b), nb - 1 - n0 / 16) * kt * 1024 + half * 1024 + 16 * lane);
    const int row = 8 * (8 * i + wave) + (lane >> 3);
    chunk[i] = (lane & 7) ^ (row & 7) ^ ((row >> 4) & 1);
    boff[i] = uint32_t(min(int64_t(row), a.T - 1 - t0) * a.K + 16 * chunk[i]);
  }
  // the last stage: a k-step or columns past the end are read from the stage's
  // first ones instead (which the row has); the packed zeros and the sums'
  // masks leave them out
  auto last = [&](int st) {
    if (st == ns - 1) {
      if (2 * st + half >= kt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) aoff[i] -= 1024;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (128 * int64_t(st) + 16 * chunk[i] >= a.K) boff[i] -= uint32_t(16 * chunk[i]);
    }
  };
  const uint32_t lds0 = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(&lds[0])));
  lds_cchar* lbase = (lds_cchar*)(&lds[0]);
  const int wm = wave >> 2, wn = wave & 3;
  auto b_lds = [&](int s) { return lds0 + uint32_t(s % 3) * 32768u; };
  auto a_lds = [&](int s) { return lds0 + 98304u + uint32_t(s & 1) * 32768u; };
  auto b_tile = [&](int s) { return lbase + (s % 3) * 32768; };
  auto a_tile = [&](int s) { return lbase + 98304 + (s & 1) * 32768; };
  // (offsets of the stage are added to the bases; the last stage's are changed first)
  auto copy_a = [&](int s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) dma16_s(wbase + int64_t(s) * 2048, aoff[i], a_lds(s) + (8 * i + wave) * 1024);
  };
  auto copy_b = [&](int s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) dma16_s(xbase + int64_t(s) * 128, boff[i], b_lds(s) + (8 * i + wave) * 1024);
  };
  // token fragments of k-step k as int8, with their sums: columns past K do not count
  auto take_b = [&](i32x4_t (&b)[4], uint32_t (&sx)[4], int k) {
    const bool in = 64 * int64_t(k) + 16 * g4 < a.K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t s = sum_codes(b[j], sx[j]);
      sx[j] = in ? s : sx[j];
      b[j] = flip(b[j]);
    }
  };
  auto read = [&](i32x4_t (&x)[8], i32x4_t (&y)[4], int st, int kk) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = frag(a_tile(st), 8 * wm + i, kk, lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = tok_frag(b_tile(st), 4 * wn + j, kk, lane);
  };
  i32x4_t acc[8][4];
  uint32_t sx[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  auto mul = [&](const i32x4_t (&x)[8], const i32x4_t (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mfma_i8(x[i], y[j], acc[i][j]);
  };

  last(0);
  copy_a(0);
  copy_b(0);
  wait_vm0();
  __syncthreads();
  i32x4_t a0[8], b0[4], a1[8], b1[4];
  read(a0, b0, 0, 0);
  take_b(b0, sx, 0);
  if (ns > 1) {
    last(1);
    copy_a(1);
    copy_b(1);
  }
  // iteration s: the first k-step copies the tokens of stage s + 2 (their buffer
  // held stage s - 1), the second the channels of stage s + 2 (held stage s, whose
  // last reads end at the middle barrier), which waits for stage s + 1 with the
  // tokens of stage s + 2 still in flight.  The last two stages run below.
  int s = 0;
  for (; s + 2 < ns; ++s) {
    last(s + 2);
    i8_step<true>(acc, sx, a0, b0, a_tile(s), b_tile(s), 1, wm, wn, lane, a1, b1, xbase + int64_t(s + 2) * 128,
                  boff, b_lds(s + 2), wave);
    wait_vm4();
    __syncthreads();
    i8_step<true>(acc, sx, a1, b1, a_tile(s + 1), b_tile(s + 1), 0, wm, wn, lane, a0, b0,
                  wbase + int64_t(s + 2) * 2048, aoff, a_lds(s + 2), wave);
  }
  for (; s < ns; ++s) {
    if (2 * s + 1 < kt) {
      read(a1, b1, s, 1);
      take_b(b1, sx, 2 * s + 1);
    }
    mul(a0, b0);
    if (s + 1 < ns) wait_vm0();
    __syncthreads();
    if (s + 1 < ns) {
      read(a0, b0, s + 1, 0);
      take_b(b0, sx, 2 * s + 2);
    }
    if (2 * s + 1 < kt) mul(a1, b1);
  }
  // a token's sum: its four lanes hold every k-step's quarter
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sx[j] += __shfl_xor(sx[j], 16);
    sx[j] += __shfl_xor(sx[j], 32);
  }
  float hx[4];
  double zx[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t t = min(t0 + 64 * wn + 16 * j + r, a.T - 1);
    hx[j] = a.hx[t];
    zx[j] = double(a.zx[t]) - 128.0;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t n = n0 + 128 * wm + 16 * i + 4 * g4;
    if (n < a.N) {
      const Chan kc = load_chan(a, n);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t t = t0 + 64 * wn + 16 * j + r;
        if (t < a.T) store_out<YBF>(a, t, n, kc, acc[i][j], int(sx[j]) - 128 * int(a.K), hx[j], zx[j]);
      }
    }
  }
}

// ------------------------------------------------------------------ a medium number of tokens
// 16 MB channels x 16 NB tokens per workgroup, the same stages of 128 inputs in
// a ring of S: S - 1 stages are in flight or in use while one is computed, so the
// copies' latency is hidden also where a compute unit has one workgroup.
template <int N>
OQ_DEV void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int MB, int NB, int WM, int WN, int KG, int S, bool YBF>
__global__ __launch_bounds__(64 * WM * WN * KG) void i8_ring_kernel(I8Args a, int tiles_m, int tiles_n) {
  constexpr int GW = WM * WN;                      // waves of one K group
  constexpr int CA = 2 * MB / GW, CB = 2 * NB / GW;
  constexpr int MT = MB / WM, NT = NB / WN;
  constexpr int SUB = (MB + NB) * 2048, STAGE = KG * SUB;
  static_assert(CA * GW == 2 * MB && CB * GW == 2 * NB && GW % 2 == 0, "whole copies per wave");
  static_assert((KG - 1) * GW * 64 * (MT * NT * 16 + NT * 4) <= S * STAGE, "the groups' sums fit the ring");
  __shared__ uint4 lds[S * STAGE / 16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int kg = (tid >> 6) / GW, wave = (tid >> 6) % GW;
  const int r = lane & 15, g4 = lane >> 4;
  // contiguous tiles per XCD, token tiles fastest: a weight tile is fetched once
  const int nblk = gridDim.x, bid = blockIdx.x;
  const int xcd = bid & 7, local = bid >> 3, q = nblk >> 3, rem = nblk & 7;
  const int L = xcd * q + min(xcd, rem) + local;
  const int64_t n0 = int64_t(L / tiles_n) * (16 * MB), t0 = int64_t(L % tiles_n) * (16 * NB);
  const int kt = int(i8_cols(a.K) / 64), ns = (kt + 2 * KG - 1) / (2 * KG);
  const int64_t nb = i8_rows(a.N) / 16;
  const int8_t* wbase = a.w + (n0 / 16) * kt * 1024;
  const uint8_t* xbase = a.x + t0 * a.K;
  uint32_t aoff[CA], boff[CB];
  int chunk[CB];
  const int half = wave & 1;
#pragma unroll
  for (int i = 0; i < CA; ++i) {
    const int b = (GW * i + wave) >> 1;
    aoff[i] = uint32_t(min(int64_t(b), nb - 1 - n0 / 16) * kt * 1024 + kg * 2048 + half * 1024 + 16 * lane);
  }
#pragma unroll
  for (int i = 0; i < CB; ++i) {
    const int row = 8 * (GW * i + wave) + (lane >> 3);
    chunk[i] = (lane & 7) ^ (row & 7) ^ ((row >> 4) & 1);
    boff[i] = uint32_t(min(int64_t(row), a.T - 1 - t0) * a.K + kg * 128 + 16 * chunk[i]);
  }
  const uint32_t lds0 = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(&lds[0])));
  lds_cchar* lbase = (lds_cchar*)(&lds[0]);
  auto copy = [&](int st) {
    if (st == ns - 1) {
      // past the end: the weight's last k-step and the row's first columns of the
      // stage instead (both exist); neither is used
      const int k = 2 * (st * KG + kg) + half;
      if (k >= kt) {
#pragma unroll
        for (int i = 0; i < CA; ++i) aoff[i] -= uint32_t(k - (kt - 1)) * 1024;
      }
#pragma unroll
      for (int i = 0; i < CB; ++i)
        if (128 * int64_t(st * KG + kg) + 16 * chunk[i] >= a.K) boff[i] -= uint32_t(kg * 128 + 16 * chunk[i]);
    }
    const uint32_t at = lds0 + uint32_t(st % S) * STAGE + uint32_t(kg) * SUB;
#pragma unroll
    for (int i = 0; i < CA; ++i) dma16_s(wbase + int64_t(st) * (KG * 2048), aoff[i], at + (GW * i + wave) * 1024);
#pragma unroll
    for (int i = 0; i < CB; ++i)
      dma16_s(xbase + int64_t(st) * (KG * 128), boff[i], at + MB * 2048 + (GW * i + wave) * 1024);
  };
  const int wm = wave / WN, wn = wave % WN;
  i32x4_t acc[MT][NT];
  uint32_t sx[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    sx[j] = 0;
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i][j] = i32x4_t{0, 0, 0, 0};
  }
#pragma unroll
  for (int st = 0; st < S - 1; ++st)
    if (st < ns) copy(st);
  for (int st = 0; st < ns; ++st) {
    // stage st has landed once only the S - 2 later ones are outstanding
    if (st + S - 2 < ns) wait_vm<(S - 2) * (CA + CB)>();
    else wait_vm<0>();
    __syncthreads();                       // every wave is done with stage st - 1
    if (st + S - 1 < ns) copy(st + S - 1);
    lds_cchar* at = lbase + (st % S) * STAGE + kg * SUB;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int k = 2 * (st * KG + kg) + kk;
      if (k < kt) {
        i32x4_t x[MT], y[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) y[j] = tok_frag(at + MB * 2048, NT * wn + j, kk, lane);
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = frag(at, MT * wm + i, kk, lane);
        const bool in = 64 * int64_t(k) + 16 * g4 < a.K;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint32_t s = sum_codes(y[j], sx[j]);
          sx[j] = in ? s : sx[j];
          y[j] = flip(y[j]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma_i8(x[i], y[j], acc[i][j]);
      }
    }
  }
  if constexpr (KG > 1) {
    // the K groups' sums, in the ring's memory
    i32x4_t* pa = reinterpret_cast<i32x4_t*>(&lds[0]);
    uint32_t* ps = reinterpret_cast<uint32_t*>(&lds[(KG - 1) * GW * MT * NT * 64]);
    __syncthreads();
    if (kg > 0) {
      const int w = (kg - 1) * GW + wave;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        ps[(w * NT + j) * 64 + lane] = sx[j];
#pragma unroll
        for (int i = 0; i < MT; ++i) pa[((w * MT + i) * NT + j) * 64 + lane] = acc[i][j];
      }
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int k = 0; k < KG - 1; ++k) {
      const int w = k * GW + wave;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        sx[j] += ps[(w * NT + j) * 64 + lane];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][j] += pa[((w * MT + i) * NT + j) * 64 + lane];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    sx[j] += __shfl_xor(sx[j], 16);
    sx[j] += __shfl_xor(sx[j], 32);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t n = n0 + 16 * (MT * wm + i) + 4 * g4;
    if (n < a.N) {
      const Chan kc = load_chan(a, n);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int64_t t = t0 + 16 * (NT * wn + j) + r;
        if (t < a.T)
          store_out<YBF>(a, t, n, kc, acc[i][j], int(sx[j]) - 128 * int(a.K), a.hx[t], double(a.zx[t]) - 128.0);
      }
    }
  }
}

__global__ __launch_bounds__(256) void i8_pack_kernel(const uint8_t* __restrict__ codes, int64_t N,
                                                      int64_t K, int8_t* __restrict__ packed,
                                                      int32_t* __restrict__ wsum) {
  // one workgroup per block row of 16 channels; thread t: row t % 16, chunks t / 16 + 16 i
  __shared__ uint32_t s_sum[256];
  const int r = threadIdx.x & 15, c0 = threadIdx.x >> 4;
  const int64_t n = 16 * int64_t(blockIdx.x) + r;
  const int64_t kt = (K + 63) / 64;
  uint32_t s = 0;
  for (int64_t c = c0; c < 4 * kt; c += 16) {
    i32x4_t v = {0, 0, 0, 0};
    if (n < N && 16 * c < K) {
      v = *reinterpret_cast<const i32x4_t*>(codes + n * K + 16 * c);
      s = sum_codes(v, s);
      v = flip(v);
    }
    reinterpret_cast<i32x4_t*>(packed)[(int64_t(blockIdx.x) * kt + c / 4) * 64 + 16 * (c & 3) + r] = v;
  }
  s_sum[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 16 && n < N) {
    for (int q = 1; q < 16; ++q) s += s_sum[16 * q + r];
    wsum[n] = int(s) - 128 * int(K);
  }
}

}  // namespace

hipError_t int8_pack(const uint8_t* codes, int64_t c_out, int64_t c_in, int8_t* packed, int32_t* wsum,
                     hipStream_t st) {
  if (c_out == 0) return hipSuccess;
  hipLaunchKernelGGL(i8_pack_kernel, dim3(unsigned(i8_rows(c_out) / 16)), dim3(256), 0, st, codes, c_out,
                     c_in, packed, wsum);
  return hipGetLastError();
}

namespace {

template <int MB, int NB, int WM, int WN, int KG, int S>
void launch_ring(const I8Args& a, bool y_bf16, hipStream_t st) {
  const int tm = int((a.N + 16 * MB - 1) / (16 * MB)), tn = int((a.T + 16 * NB - 1) / (16 * NB));
  const dim3 grid(unsigned(tm) * unsigned(tn)), blk(64 * WM * WN * KG);
  if (y_bf16) hipLaunchKernelGGL((i8_ring_kernel<MB, NB, WM, WN, KG, S, true>), grid, blk, 0, st, a, tm, tn);
  else hipLaunchKernelGGL((i8_ring_kernel<MB, NB, WM, WN, KG, S, false>), grid, blk, 0, st, a, tm, tn);
}

}  // namespace

hipError_t int8_linear(const I8Args& a, bool y_bf16, hipStream_t st) {
  // Kernels by tokens and channels (us, one graph of launches over weights that
  // do not stay in the caches, inputs x channels):
  //   up to 16 tokens and 4,096 channels, 16 channels a workgroup (all of them run
  //   at once, with every load of a token's weights in flight): 6.9 against the
  //   ring's 8.1 (1 token, 4,096 x 4,096), 12.7 against 15 (11,008 x 4,096); at
  //   6,144 channels 10.1 against 8.9;
  if (a.T <= 16 && a.N <= 4096) {
    const dim3 grid(unsigned(i8_rows(a.N) / 16));
    if (y_bf16) hipLaunchKernelGGL((i8_small_kernel<8, true>), grid, dim3(64 * SW), 0, st, a);
    else hipLaunchKernelGGL((i8_small_kernel<8, false>), grid, dim3(64 * SW), 0, st, a);
    return hipGetLastError();
  }
  //   else the smallest tile whose workgroups all run at once on 256 compute units
  //   (4,096 x 4,096, 64 tokens: 32 x 32 9.0, 64 x 32 10.9, 64 x 64 14.5; 256
  //   tokens: 28.7, 19.8, 14.7 and 128 x 64 20.6; 5,120 x 13,824, 256 tokens: 128 x
  //   64 52, 128 x 128 36, 256 x 256 63): small tiles split K over more waves and
  //   larger ones read the operands fewer times (the K halves in two groups of waves
  //   also with 128 x 64: 384 tokens of 4,096 x 4,096 20.6 -> 19.0, of 11,008 x 4,096
  //   46 -> 42; rings one or two stages deeper or shallower: no gain); two 128 x 128 workgroups fit a
  //   compute unit with rings of two stages (8,192 x 28,672, 256 tokens: 90
  //   against 123 by 256 x 256 tiles);
  //   256 x 256 tiles beyond (1,024 tokens, 4,096 x 11,008: 61 against 75).
  //   Over very many channels few tokens take these tiles too: they wait for the
  //   weight's bytes all the same up to 65,536 channels of 8,192 inputs (57,344: 1 to
  //   64 tokens 91 to 101 us, the bytes alone 93); by 256 x 256 tiles 128,256 channels
  //   take 221 us for one token and 251 to 259 for 4 to 128, the bytes alone 208.
  auto tiles = [&](int ch, int tok) { return ((a.N + ch - 1) / ch) * ((a.T + tok - 1) / tok); };
  if (tiles(32, 32) <= 256) launch_ring<2, 2, 2, 1, 4, 4>(a, y_bf16, st);
  else if (tiles(64, 32) <= 256) launch_ring<4, 2, 2, 2, 2, 4>(a, y_bf16, st);
  else if (tiles(64, 64) <= 256) launch_ring<4, 4, 2, 2, 2, 4>(a, y_bf16, st);
  else if (tiles(128, 64) <= 256) launch_ring<8, 4, 4, 2, 2, 3>(a, y_bf16, st);
  else if (tiles(128, 128) <= 256) launch_ring<8, 8, 2, 4, 1, 4>(a, y_bf16, st);
  else if (tiles(128, 128) <= 512) launch_ring<8, 8, 2, 4, 1, 2>(a, y_bf16, st);   // two per compute unit
  else {
    const int tm = int((a.N + BT - 1) / BT), tn = int((a.T + BT - 1) / BT);
    const dim3 grid(unsigned(tm) * unsigned(tn));
    if (y_bf16) hipLaunchKernelGGL((i8_tile_kernel<true>), grid, dim3(TNT), 0, st, a, tm, tn);
    else hipLaunchKernelGGL((i8_tile_kernel<false>), grid, dim3(TNT), 0, st, a, tm, tn);
  }
  return hipGetLastError();
}

}  // namespace oq
