// Y = Q_a(X) Q_w(W)^T + B from integer codes, on 8-bit matrix cores: the linear
// of a weight-activation quantised block.  With a = q_x - 128 and b = q_w - 128
// (both int8) and z' = z - 128,
//   sum_c (q_x - z_x)(q_w - z_w) = sum a b - z_x' (sum b - K z_w') - z_w' sum a,
// where sum a b is exact in int32, sum b comes with the packed weight and
// sum a is formed beside the product.  The correction is fp64 (its terms are
// larger than the result), the two scales and the bias fp32.
#include <math.h>

#include "common.h"
#include "serve.h"

namespace oq {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
constexpr uint32_t FLIP = 0x80808080u;      // code -> code - 128 as int8, four at once

OQ_DEV i32x4_t mfma_i8(i32x4_t a, i32x4_t b, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}
OQ_DEV i32x4_t flip(uint4 v) {
  return i32x4_t{int(v.x ^ FLIP), int(v.y ^ FLIP), int(v.z ^ FLIP), int(v.w ^ FLIP)};
}
OQ_DEV int sum_bytes(i32x4_t v, int s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_sdot4(v[i], 0x01010101, s, false);
  return s;
}

// Four channels n .. n + 3 of token t from their accumulators.
template <bool YBF>
OQ_DEV void store_out(const I8Args& a, int64_t t, int64_t n, i32x4_t acc, int sx, float hx, double zx) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t c = n + i < a.N ? n + i : a.N - 1;
    const double zw = double(a.zw[c]) - 128.0;
    const double s = double(acc[i]) - zx * (double(a.wsum[c]) - double(a.K) * zw) - zw * double(sx);
    y[i] = float(s) * (hx * a.hw[c]);
    if (a.bias) y[i] = y[i] + a.bias[c];
  }
  if (YBF) {
    uint16_t* p = static_cast<uint16_t*>(a.y) + t * a.N + n;
    if ((a.N & 3) == 0 && n + 4 <= a.N) {
      *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) p[i] = f2bf(y[i]);
    }
  } else {
    float* p = static_cast<float*>(a.y) + t * a.N + n;
    if ((a.N & 3) == 0 && n + 4 <= a.N) {
      *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) p[i] = y[i];
    }
  }
}

// 16 channels x 16 R tokens per workgroup, the K range split over the waves.
template <int R, bool YBF>
__global__ __launch_bounds__(256) void i8_small_kernel(I8Args a) {
  __shared__ i32x4_t s_acc[4][R][64];
  __shared__ int s_sum[4][R][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r = lane & 15, g = lane >> 4;
  const int64_t n0 = 16 * int64_t(blockIdx.x), t0 = 16 * R * int64_t(blockIdx.y);
  const int kt = int(i8_cols(a.K) / 64);
  const int per = (kt + 3) / 4;
  const int k0 = wave * per, k1 = min(kt, k0 + per);
  const uint4* wp = reinterpret_cast<const uint4*>(a.w) + (int64_t(blockIdx.x) * kt) * 64 + lane;
  const uint8_t* xp[R];
#pragma unroll
  for (int j = 0; j < R; ++j) xp[j] = a.x + min(t0 + 16 * j + r, a.T - 1) * a.K;
  i32x4_t acc[R];
  int sx[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    acc[j] = i32x4_t{0, 0, 0, 0};
    sx[j] = 0;
  }
  for (int k = k0; k < k1; ++k) {
    const uint4 w = wp[64 * k];
    const i32x4_t wf = {int(w.x), int(w.y), int(w.z), int(w.w)};
    const int64_t col = 64 * int64_t(k) + 16 * g;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      i32x4_t x = {0, 0, 0, 0};
      if (col < a.K) x = flip(*reinterpret_cast<const uint4*>(xp[j] + col));
      acc[j] = mfma_i8(wf, x, acc[j]);
      sx[j] = sum_bytes(x, sx[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    s_acc[wave][j][lane] = acc[j];
    s_sum[wave][j][lane] = sx[j];
  }
  __syncthreads();
  for (int j = wave; j < R; j += 4) {
    i32x4_t c = {0, 0, 0, 0};
    int s = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      c += s_acc[w][j][lane];
#pragma unroll
      for (int q = 0; q < 4; ++q) s += s_sum[w][j][16 * q + r];
    }
    const int64_t t = t0 + 16 * j + r, n = n0 + 4 * g;
    if (t < a.T && n < a.N) store_out<YBF>(a, t, n, c, s, a.hx[t], double(a.zx[t]) - 128.0);
  }
}

__global__ __launch_bounds__(256) void i8_pack_kernel(const uint8_t* __restrict__ codes, int64_t N,
                                                      int64_t K, int8_t* __restrict__ packed,
                                                      int32_t* __restrict__ wsum) {
  // one workgroup per block row of 16 channels; thread t: row t % 16, chunks t / 16 + 16 i
  __shared__ int s_sum[256];
  const int r = threadIdx.x & 15, c0 = threadIdx.x >> 4;
  const int64_t n = 16 * int64_t(blockIdx.x) + r;
  const int64_t kt = (K + 63) / 64;
  int s = 0;
  for (int64_t c = c0; c < 4 * kt; c += 16) {
    i32x4_t v = {0, 0, 0, 0};
    if (n < N && 16 * c < K) v = flip(*reinterpret_cast<const uint4*>(codes + n * K + 16 * c));
    s = sum_bytes(v, s);
    reinterpret_cast<i32x4_t*>(packed)[(int64_t(blockIdx.x) * kt + c / 4) * 64 + 16 * (c & 3) + r] = v;
  }
  s_sum[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 16 && n < N) {
    for (int q = 1; q < 16; ++q) s += s_sum[16 * q + r];
    wsum[n] = s;
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

hipError_t int8_linear(const I8Args& a, bool y_bf16, hipStream_t st) {
  const dim3 grid(unsigned(i8_rows(a.N) / 16), unsigned((a.T + 63) / 64));
  if (y_bf16) hipLaunchKernelGGL((i8_small_kernel<4, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((i8_small_kernel<4, false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace oq
