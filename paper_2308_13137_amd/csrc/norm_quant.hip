// The residual addition, RMSNorm and per-token activation quantiser of a
// deployed block in one pass over the row:
//   H = X + R (rounded to X's type),  y = (H rstd) g + b,  rstd = 1/sqrt(mean H^2 + eps)
//   h = max((max y - min y)/(2^N - 1), 1e-5), z = -rint(min y (1/h)),
//   code = clamp(rint(y (1/h)) + z, 0, 2^N - 1)
// (or the symmetric quantiser).  The norm is that of H as stored, so the call
// equals the addition followed by the norm of what the addition left.  g and b
// are the norm's gain and shift after LET is absorbed into them.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "serve.h"

namespace oq {
namespace {

// Eight elements as they lie in memory.
template <typename T>
struct Raw8 {
  uint4 q[sizeof(T) / 2];
  OQ_DEV void load(const T* p) {
    const uint4* s = reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) q[i] = s[i];
  }
  OQ_DEV void get(float (&v)[8]) const { load8(reinterpret_cast<const T*>(q), v); }
};

// One workgroup per row, the row in registers (CH chunks of 8 per thread)
// between its three uses: the sum of squares, the range, the codes.  Up to 2,048
// workgroups walk the rows: gain and shift are loaded once (per row from the L2
// they took a fifth of the time) and the next row's loads are in flight while one
// is reduced.  HBM-bound: 16,384 x 8,192 bf16 with residual and shift 185 us, 5.1
// TB/s, the rate of a copy (217 us without either).  Squares are summed in fp64: a
// row of any finite bf16 or fp32 values has a finite mean square there.
template <typename TX, typename TR, int NTH, int CH>
__global__ __launch_bounds__(NTH) void norm_quant_kernel(
    const TX* X, const TR* R, int64_t T, int64_t D,
    const float* __restrict__ gain, const float* __restrict__ bias, float eps, int bits, bool sym,
    TX* Hout, void* __restrict__ xdq, bool dq_bf16, uint8_t* __restrict__ codes,
    float* __restrict__ hout, float* __restrict__ zout) {
  constexpr int NW = NTH / 64;
  __shared__ double s_sum[NW];
  __shared__ float s_rng[3][NW];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int nch = int(D / 8);
  const bool quant = bits < 16;
  const float qmax = quant ? float((1 << bits) - 1) : 0.0f;
  // 1,024 threads have 128 registers each: gain and shift come from the caches per
  // row there, and a row's loads wait for the row before.  The row and its residual, raw
  // and as fp32, still pass the 128: 10 (bf16) to 77 (fp32) registers spill, 44 to 248
  // bytes a lane.  2,048 x 32,768 with both: bf16 146 us (3.2 TB/s; 291 with everything
  // held), fp32 380 us (2.3 TB/s); every narrower kernel keeps all of it in registers.
  constexpr bool KEEP = NTH < 1024;
  float gn[KEEP ? CH : 1][8], bs[KEEP ? CH : 1][8];
  auto gains = [&](int k, int j) {
    load8(gain + 8 * j, gn[k]);
    if (bias) load8(bias + 8 * j, bs[k]);
  };
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int j = tid + NTH * k;
#pragma unroll
      for (int e = 0; e < 8; ++e) gn[k][e] = bs[k][e] = 0.0f;
      if (j < nch) gains(k, j);
    }
  }
  Raw8<TX> nx[CH];
  Raw8<TR> nr[CH];
  auto fetch = [&](int64_t row) {
    if (row >= T) return;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int j = tid + NTH * k;
      if (j < nch) {
        nx[k].load(X + row * D + 8 * j);
        if (R) nr[k].load(R + row * D + 8 * j);
      }
    }
  };
  if constexpr (KEEP) fetch(blockIdx.x);
  for (int64_t row = blockIdx.x; row < T; row += gridDim.x) {
    float v[CH][8], rv[CH][8];
    double ss = 0.0;
    if constexpr (!KEEP) fetch(row);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      nx[k].get(v[k]);
      nr[k].get(rv[k]);
    }
    if constexpr (KEEP) fetch(row + gridDim.x);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int j = tid + NTH * k;
      if (j < nch) {
        if (R) {
          const float (&r)[8] = rv[k];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[k][e] = v[k][e] + r[e];
            if constexpr (sizeof(TX) == 2) v[k][e] = bf2f(f2bf(v[k][e]));
          }
          if (Hout) store8(Hout + row * D + 8 * j, v[k]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fma(double(v[k][e]), double(v[k][e]), ss);
      }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) ss += __shfl_xor(ss, off);
    if (lane == 0) s_sum[wave] = ss;
    __syncthreads();
    ss = s_sum[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) ss += s_sum[w];
    const double rstd = 1.0 / sqrt(ss / double(D) + double(eps));
    float rs = float(rstd);
    // one that fp32 holds with fewer bits, or not at all (subnormal rows, eps 0): a power of
    // two of it goes to the values first
    if (!(rs >= 0x1p-126f && rs <= 0x1p126f)) {
      const float k = rs < 1.0f ? 0x1p-64f : 0x1p64f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * k;
      rs = float(rstd / double(k));
    }
    float mx = -INFINITY, mn = INFINITY, bad = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int j = tid + NTH * k;
      if (j < nch) {
        const int kg = KEEP ? k : 0;
        if constexpr (!KEEP) gains(kg, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] = v[k][e] * rs * gn[kg][e];
        if (bias) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[k][e] = v[k][e] + bs[kg][e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          mx = fmaxf(mx, v[k][e]);
          mn = fminf(mn, v[k][e]);
          bad = __builtin_fmaf(v[k][e], 0.0f, bad);       // NaN once a value is not finite
        }
      }
    }
    if (!quant) {
      if (xdq) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const int j = tid + NTH * k;
          if (j < nch) {
            if (dq_bf16) store8(static_cast<uint16_t*>(xdq) + row * D + 8 * j, v[k]);
            else store8(static_cast<float*>(xdq) + row * D + 8 * j, v[k]);
          }
        }
      }
      __syncthreads();
      continue;
    }
    mx = wave_max(mx);
    mn = wave_min(mn);
    bad = wave_sum(bad);
    if (lane == 0) {
      s_rng[0][wave] = mx;
      s_rng[1][wave] = mn;
      s_rng[2][wave] = bad;
    }
    __syncthreads();
    mx = s_rng[0][0];
    mn = s_rng[1][0];
    bad = s_rng[2][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      mx = fmaxf(mx, s_rng[0][w]);
      mn = fminf(mn, s_rng[1][w]);
      bad += s_rng[2][w];
    }
    QParams p;
    if (sym) {
      int iab;
      float sgn;
      p = make_sym_qparams(mx, 0, mn, 0, float((1 << (bits - 1)) - 1), iab, sgn);
    } else {
      p = make_qparams(mx, mn, 1.0f, 1.0f, qmax);
    }
    // a row with a value that is not finite has no range: its step is NaN (so
    // is everything computed from its codes), its codes are zeros
    const bool fine = bad == 0.0f;
    if (!fine) {
      p.h = NAN;
      p.z = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int j = tid + NTH * k;
      if (j < nch) {
        float q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = fine ? quant_elem(v[k][e], p, qmax).q : 0.0f;
        if (codes) store8_codes(codes + row * D + 8 * j, q);
        if (xdq) {
#pragma unroll
          for (int e = 0; e < 8; ++e) q[e] = dequant(q[e], p);
          if (dq_bf16) store8(static_cast<uint16_t*>(xdq) + row * D + 8 * j, q);
          else store8(static_cast<float*>(xdq) + row * D + 8 * j, q);
        }
      }
    }
    if (tid == 0) {
      if (hout) hout[row] = p.h;
      if (zout) zout[row] = p.z;
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t rmsnorm_quant(const void* X, bool x_bf16, const void* R, bool r_bf16, int64_t T, int64_t D,
                         const float* gain, const float* bias, float eps, int bits, bool sym, void* H,
                         void* X_dq, bool dq_bf16, uint8_t* codes, float* h, float* z, hipStream_t st) {
  if (T == 0) return hipSuccess;
  const dim3 grid(unsigned(std::min<int64_t>(T, 2048)));
  auto go = [&](auto tx, auto tr, auto nth, auto ch) {
    using TX = decltype(tx);
    using TR = decltype(tr);
    constexpr int NTH = decltype(nth)::value, CH = decltype(ch)::value;
    hipLaunchKernelGGL((norm_quant_kernel<TX, TR, NTH, CH>), grid, dim3(NTH), 0, st,
                       static_cast<const TX*>(X), static_cast<const TR*>(R), T, D, gain, bias, eps, bits,
                       sym, static_cast<TX*>(H), X_dq, dq_bf16, codes, h, z);
  };
  auto by_d = [&](auto tx, auto tr) {
    const int64_t nch = D / 8;
    const std::integral_constant<int, 2> c2{};
    const std::integral_constant<int, 3> c3{};
    const std::integral_constant<int, 4> c4{};
    if (nch <= 128) go(tx, tr, std::integral_constant<int, 64>{}, c2);
    else if (nch <= 256) go(tx, tr, std::integral_constant<int, 128>{}, c2);
    else if (nch <= 512) go(tx, tr, std::integral_constant<int, 256>{}, c2);
    else if (nch <= 768) go(tx, tr, std::integral_constant<int, 256>{}, c3);
    else if (nch <= 1024) go(tx, tr, std::integral_constant<int, 256>{}, c4);
    else if (nch <= 2048) go(tx, tr, std::integral_constant<int, 512>{}, c4);
    else go(tx, tr, std::integral_constant<int, 1024>{}, c4);
  };
  if (x_bf16) {
    if (r_bf16) by_d(uint16_t{}, uint16_t{});
    else by_d(uint16_t{}, float{});
  } else {
    if (r_bf16) by_d(float{}, uint16_t{});
    else by_d(float{}, float{});
  }
  return hipGetLastError();
}

}  // namespace oq
