// Drafted tokens against the target: logits to probabilities, and the walk down a tree
// of drafts that keeps the target's distribution.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "serve.h"

namespace oq {
namespace {

constexpr int NT = 1024, NW = NT / 64;

// Rows of a vocabulary start at any element: 16 bytes at an address of any alignment.
template <typename T>
OQ_DEV T load_any(const void* p) {
  T v;
  __builtin_memcpy(&v, p, sizeof(T));
  return v;
}

// ------------------------------------------------------------------ probabilities
// P = softmax(logits / t) = 2^((x - max x) log2(e) / t) over their sum.  One workgroup
// a row: up to NV 16-byte pieces a thread stay in registers between the maximum, the sum
// and the output; what is beyond them is read again.  Many rows are bound by HBM (512 of 128,256
// bf16 logits 104 us, 3.8 TB/s, 7% longer with half the pieces held and two workgroups on a compute
// unit; fp32 logits, of which 49,152 a row stay in registers, 153 us).  With few rows gridDim.y
// workgroups read the same row, sum it in the same order and write a part each (five rows of 128,256:
// 19 us a call with one, 14.6 with eight).
template <typename TI, int NV>
__global__ __launch_bounds__(NT) void probs_kernel(const TI* __restrict__ X, int64_t ldx, int64_t V,
                                                   const float* __restrict__ temperature, float* __restrict__ P,
                                                   int64_t ldp) {
  constexpr int E = 16 / sizeof(TI);
  typedef unsigned raw_t __attribute__((ext_vector_type(4)));
  __shared__ float s_a[NW];
  __shared__ int s_i[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const TI* x = X + int64_t(blockIdx.x) * ldx;
  float* out = P + int64_t(blockIdx.x) * ldp;
  const int n = int(V / E), rest = int(V) - n * E;         // whole pieces, values behind them
  const int y = blockIdx.y, S = gridDim.y;                 // steps of NT pieces that are y modulo S
  const float t = temperature ? temperature[blockIdx.x] : 1.0f;
  auto value = [&](raw_t w, int e) {
    if constexpr (E == 8) return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    else return __uint_as_float(w[e]);
  };
  raw_t held[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (tid + NT * k < n) held[k] = load_any<raw_t>(x + int64_t(E) * (tid + NT * k));
  const float tail = tid < rest ? load1(x + int64_t(n) * E + tid) : -INFINITY;
  // f(piece number, its values) of every whole piece of this thread
  auto pieces = [&](auto f) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (tid + NT * k < n) f(tid + NT * k, held[k]);
    for (int i = tid + NT * NV; i < n; i += NT) f(i, load_any<raw_t>(x + int64_t(E) * i));
  };
  float m = tail;
  bool odd = !(tail < INFINITY);                           // NaN or +inf
  pieces([&](int, raw_t w) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      m = fmaxf(m, value(w, e));
      odd = odd || !(value(w, e) < INFINITY);
    }
  });
  m = wave_max(m);
  if (lane == 0) s_a[wave] = m;
  odd = __syncthreads_or(odd);
#pragma unroll
  for (int w = 0; w < NW; ++w) m = fmaxf(m, s_a[w]);
  // a row without a maximum, or without a temperature, is no distribution
  if (odd || m == -INFINITY || !(t >= 0.0f && t < INFINITY)) {
    for (int64_t i = tid + NT * y; i < V; i += NT * S) out[i] = NAN;
    return;
  }
  if (t == 0.0f) {                                         // all of it on the first maximum
    int first = tail == m ? n * E + tid : 0x7fffffff;
    pieces([&](int i, raw_t w) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (value(w, e) == m) first = min(first, i * E + e);
    });
    for (int off = 1; off < 64; off <<= 1) first = min(first, __shfl_xor(first, off));
    if (lane == 0) s_i[wave] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) first = min(first, s_i[w]);
    for (int64_t i = tid + NT * y; i < V; i += NT * S) out[i] = i == first ? 1.0f : 0.0f;
    return;
  }
  auto row_sum = [&](float v) {
    v = wave_sum(v);
    __syncthreads();                                       // s_a is read
    if (lane == 0) s_a[wave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += s_a[w];
    return v;
  };
  // Above a temperature of one x - max may pass fp32's range where its quotient does not, at huge ones the scale
  // itself lies below fp32's normal numbers, and at tiny ones differences there count, whose scale would be infinite:
  // all are scaled by a power of two first.  (Loops of their own: with the factor in the ones below, 512 rows of
  // 128,256 bf16 logits took 104.6 us a call instead of 104.2, five 14.7 instead of 14.5.)
  const bool tiny = t < 0x1p-100f;
  if (tiny || (t > 1.0f && fmaxf(m, t) > 0x1p100f)) {
    const bool far = tiny && fabsf(m) >= 0x1p90f;          // every difference that is not zero is 2^66 or more
    const float h = far ? 1.0f : tiny ? 0x1p32f : 0x1p-3f;
    const float k = far ? 3.0e38f : (1.4426950408889634f / h) / t;
    auto weight = [&](int64_t i) { return __builtin_amdgcn_exp2f(__builtin_fmaf(load1(x + i), h, -(m * h)) * k); };
    float sum = 0.0f;
    for (int64_t i = tid; i < V; i += NT) sum += weight(i);
    const float inv = 1.0f / row_sum(sum);
    for (int64_t i = tid + NT * y; i < V; i += NT * S) out[i] = weight(i) * inv;
    return;
  }
  const float k = 1.4426950408889634f / t;
  auto weight = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * k); };
  float sum = tid < rest ? weight(tail) : 0.0f;
  pieces([&](int, raw_t w) {
#pragma unroll
    for (int e = 0; e < E; ++e) sum += weight(value(w, e));
  });
  sum = row_sum(sum);
  const float inv = 1.0f / sum;
  pieces([&](int i, raw_t w) {
    if (i / NT % S != y) return;
    float p[E];
#pragma unroll
    for (int e = 0; e < E; ++e) p[e] = weight(value(w, e)) * inv;
    __builtin_memcpy(out + int64_t(i) * E, p, sizeof(p));
  });
  if (y == 0 && tid < rest) out[int64_t(n) * E + tid] = weight(tail) * inv;
}

// ------------------------------------------------------------------ verification
// The walk of one tree.  At node c the target's distribution is r = P[c]; its children
// are tried in order.  A child with token x that the draft took from q (its own row Q[c])
// is accepted if u q(x) / Z < r(x) / R; otherwise r becomes max(r / R - q / Z, 0), what the
// target has beyond the draft, and R its mass; where siblings differ, x leaves q and Z is
// what q has left.  (R = Z = 1 at first: rows are distributions.)  Without Q a child is
// certain: q is one at x, and r loses x.  After the last accepted node the next token
// is drawn from r.  Numbers that decide are fp64: a sum over the vocabulary that fp32 held
// would move the border between two tokens by more than most tokens have.
//
// After m rejections r(x) follows from p(x), q(x) and the masses of each step alone,
// so a child's test reads two numbers (all of them are fetched at the start), and only a
// mass needs a pass over the vocabulary: before a further sibling, and for the draw.  That pass repeats
// the rejections at every value, so many siblings cost their square: 8 rejected ones of 128,256 tokens
// 221 us, 32 of them 2,260 (without Q, one pass in all, 40 and 115).  With Q the kernel needs 15 registers
// more than 1,024 threads have (56 bytes a lane are spilled).
// r of N values of a row after `levels` rejections, from p and q.  (A NaN counts as zero here: sums over
// a row tell by themselves whether it holds values that are not finite.  With that in every value's own
// fp64 arithmetic, and sums of q that nobody asked for, 16 trees of up to 32 nodes over 128,256 tokens
// took 29.6 us, now 24.6.)
template <bool CERTAIN, int N>
OQ_DEV void residual(const float (&p)[N], const float (&q)[N], const int (&x)[N], int levels, const double* s_ir,
                     const double* s_iz, const int* s_rej, double (&r)[N]) {
  if constexpr (CERTAIN) {
    float y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = fmaxf(p[e], 0.0f);
    for (int t = 0; t < levels; ++t) {
      const int gone = s_rej[t];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = x[e] == gone ? 0.0f : y[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = y[e];
  } else {
    // (the first masses are ones)
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = fmax(levels > 0 ? double(p[e]) - double(q[e]) : double(p[e]), 0.0);
    for (int t = 1; t < levels; ++t) {
      const double ir = s_ir[t], iz = -s_iz[t];
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = fmax(__builtin_fma(r[e], ir, double(q[e]) * iz), 0.0);
    }
  }
}
template <bool CERTAIN>
OQ_DEV double residual(float p, float q, int x, int levels, const double* s_ir, const double* s_iz, const int* s_rej) {
  const float pp[1] = {p}, qq[1] = {q};
  const int xx[1] = {x};
  double r[1];
  residual<CERTAIN, 1>(pp, qq, xx, levels, s_ir, s_iz, s_rej, r);
  return r[0];
}
OQ_DEV double wave_sum64(double v) {
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
  return v;
}

template <bool CERTAIN>
__global__ __launch_bounds__(NT) void verify_kernel(VerifyArgs a) {
  constexpr int M = VERIFY_MAX_NODES;
  __shared__ int s_par[M], s_tok[M], s_rej[M], s_path[M];
  __shared__ float s_u[M], s_p[M], s_q[M];
  __shared__ double s_ir[M], s_iz[M], s_sum[NW], s_sumq[NW];
  __shared__ int s_hit;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = blockIdx.x;
  const int64_t b = a.q_start[i], e = a.q_start[i + 1];
  int32_t* path = a.path + int64_t(i) * a.max_path;
  const int V = int(a.V);
  bool none = b < 0 || e <= b || e > a.T || e - b > a.max_q;   // no tree, or one that does not fit
  const int n = none ? 0 : int(e - b);
  const int par_t = tid < n ? a.parent[b + tid] : -1;
  none = __syncthreads_or(none || par_t < -1 || (par_t >= 0 && par_t >= tid));
  if (none) {
    for (int k = tid; k < a.max_path; k += NT) path[k] = -1;
    if (tid == 0) {
      a.count[i] = 0;
      a.next[i] = -1;
    }
    return;
  }
  if (tid < n) {
    const int par = par_t, tok = a.token[b + tid];
    const bool fits = par >= 0 && par < tid && tok >= 0 && tok < V;
    s_par[tid] = par;
    s_tok[tid] = tok;
    s_u[tid] = a.u[b + tid];
    s_p[tid] = fits ? a.P[(b + par) * a.ldp + tok] : 0.0f;
    s_q[tid] = fits && !CERTAIN ? a.Q[(b + par) * a.ldq + tok] : 1.0f;
  }
  __syncthreads();
  const int par0 = lane < n ? s_par[lane] : -2, par1 = lane + 64 < n ? s_par[lane + 64] : -2;
  // the next child of c behind node j, n if there is none
  auto child_after = [&](int c, int j) {
    const uint64_t lo = __ballot(par0 == c && lane > j), hi = __ballot(par1 == c && lane + 64 > j);
    return lo ? __ffsll(static_cast<unsigned long long>(lo)) - 1 : hi ? __ffsll(static_cast<unsigned long long>(hi)) + 63 : n;
  };
  const float *p = a.P + b * a.ldp, *q = CERTAIN ? nullptr : a.Q + b * a.ldq;
  int levels = 0;
  // Sums of r (and of q without the rejected tokens) over values x0 .. x1 - 1 of the row, by one wave: four steps'
  // loads are under way together (16 trees of up to 32 nodes over 128,256 tokens 29.6 us, one step at a time 35.6).
  // (`walk`: for a further sibling; the draw's code has no use for q's sum)
  auto range_sum = [&](auto walk, int x0, int x1, double& sr, double& sq) {
    constexpr bool WALK = !CERTAIN && decltype(walk)::value;
    const bool of_q = WALK && !a.replace;
    double r = 0.0, w = 0.0;
    float finite = 0.0f;                                   // NaN once a value is not
    constexpr int U = 4;
    const bool with_q = !CERTAIN && levels > 0;
    int x = x0 + 4 * lane;
    // What is left of q is summed itself: a sum of all of it, less what has left it, would hold nothing of it where
    // one token had all but 2^-53 of the mass.  So the rejected tokens among these values, a few at most, are struck
    // out of both rows (r has nothing there, either).  (16 trees with many rejections 59 us a call with and without;
    // compared at every four values these tokens made it 62, all rejected tokens 67.)
    auto among = [&](int t) { return __ballot(of_q && t < levels && s_rej[t] >= x0 && s_rej[t] < x1); };
    const uint64_t here0 = WALK ? among(lane) : 0, here1 = WALK && levels > 64 ? among(lane + 64) : 0;
    auto strike = [&](int width, auto each) {              // each(token) of those in x .. x + width - 1 (lane 0's x)
      const int base = __builtin_amdgcn_readfirstlane(x);
      auto in = [&](uint64_t here, int t0) {
        for (; here; here &= here - 1) {
          const int t = t0 + __ffsll(static_cast<unsigned long long>(here)) - 1;
          const int tok = __builtin_amdgcn_readfirstlane(s_rej[t]);
          if (unsigned(tok - base) < unsigned(width)) each(tok);
        }
      };
      in(here0, 0);
      in(here1, 64);
    };
    auto four = [&](const float (&pv)[4], const float (&qv)[4], int at) {
      const int xx[4] = {at, at + 1, at + 2, at + 3};
      double rv[4];
      residual<CERTAIN, 4>(pv, qv, xx, levels, s_ir, s_iz, s_rej, rv);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        r += rv[k];
        finite = __builtin_fmaf(pv[k], 0.0f, __builtin_fmaf(qv[k], 0.0f, finite));
      }
      if (of_q) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w += double(qv[k]);
      }
    };
    for (; __all(x + 256 * (U - 1) + 4 <= x1); x += 256 * U) {
      float4 f[U], h[U];
#pragma unroll
      for (int i = 0; i < U; ++i) f[i] = load_any<float4>(p + x + 256 * i);
#pragma unroll
      for (int i = 0; i < U; ++i)
        h[i] = with_q ? load_any<float4>(q + x + 256 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
      if constexpr (WALK) strike(256 * U, [&](int tok) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int k = tok - (x + 256 * i);
          const float gp = k == 0 ? f[i].x : k == 1 ? f[i].y : k == 2 ? f[i].z : k == 3 ? f[i].w : 0.0f;
          const float gq = k == 0 ? h[i].x : k == 1 ? h[i].y : k == 2 ? h[i].z : k == 3 ? h[i].w : 0.0f;
          finite = __builtin_fmaf(gp, 0.0f, __builtin_fmaf(gq, 0.0f, finite));
          f[i] = make_float4(k == 0 ? 0.0f : f[i].x, k == 1 ? 0.0f : f[i].y, k == 2 ? 0.0f : f[i].z,
                             k == 3 ? 0.0f : f[i].w);
          h[i] = make_float4(k == 0 ? 0.0f : h[i].x, k == 1 ? 0.0f : h[i].y, k == 2 ? 0.0f : h[i].z,
                             k == 3 ? 0.0f : h[i].w);
        }
      });
#pragma unroll
      for (int i = 0; i < U; ++i)
        four({f[i].x, f[i].y, f[i].z, f[i].w}, {h[i].x, h[i].y, h[i].z, h[i].w}, x + 256 * i);
    }
    for (; x < x1; x += 256) {
      float pv[4], qv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        pv[k] = x + k < x1 ? p[x + k] : 0.0f;
        qv[k] = with_q && x + k < x1 ? q[x + k] : 0.0f;
      }
      if constexpr (WALK) strike(256, [&](int tok) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool it = x + k == tok;
          finite = it ? __builtin_fmaf(pv[k], 0.0f, __builtin_fmaf(qv[k], 0.0f, finite)) : finite;
          pv[k] = it ? 0.0f : pv[k];
          qv[k] = it ? 0.0f : qv[k];
        }
      });
      four(pv, qv, x);
    }
    sr = wave_sum64(r + double(finite));
    sq = wave_sum64(w);
  };
  // Values of a wave: sixteenths of the row, in whole steps of a wave.
  const int part = ((V + NW - 1) / NW + 255) / 256 * 256;
  auto row_sums = [&](auto walk, double& sr, double& sq) {
    __syncthreads();
    double r, w;
    range_sum(walk, min(V, wave * part), min(V, (wave + 1) * part), r, w);
    if (lane == 0) {
      s_sum[wave] = r;
      s_sumq[wave] = w;
    }
    __syncthreads();
    sr = sq = 0.0;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      sr += s_sum[k];
      sq += s_sumq[k];
    }
  };
  int cur = 0, count = 1;
  double R = 1.0, Z = 1.0;
  if (tid == 0) s_path[0] = 0;
  for (int j = child_after(0, 0); j < n;) {
    const int x = s_tok[j];
    if (x < 0 || x >= V) {                                 // no token: rejected, and nothing learned
      j = child_after(cur, j);
      continue;
    }
    const float px = s_p[j], qx = s_q[j];
    bool again = false;                                    // an earlier sibling had this token
    for (int t = 0; t < levels; ++t) again = again || s_rej[t] == x;
    const double r = residual<CERTAIN>(px, qx, x, levels, s_ir, s_iz, s_rej);
    const double qm = !CERTAIN && !a.replace && again ? 0.0 : double(qx);
    if (r > 0.0 && double(s_u[j]) * qm * R < r * Z) {
      cur = j;
      if (tid == 0) s_path[count] = j;
      ++count;
      p = a.P + (b + j) * a.ldp;
      if constexpr (!CERTAIN) q = a.Q + (b + j) * a.ldq;
      levels = 0;
      R = Z = 1.0;
      j = child_after(j, j);
      continue;
    }
    __syncthreads();                                       // (every wave has read this level's numbers)
    if (tid == 0) {
      s_rej[levels] = x;
      s_ir[levels] = 1.0 / R;
      s_iz[levels] = Z > 0.0 ? 1.0 / Z : 0.0;
    }
    __syncthreads();
    ++levels;
    j = child_after(cur, j);
    if constexpr (CERTAIN) {
      R -= r;
    } else {
      if (j < n) {
        double sr, sq;
        row_sums(std::true_type{}, sr, sq);
        if (sr == 0.0) break;                              // nothing is left: the draw steps back
        R = sr;
        if (!a.replace) Z = sq;
      }
    }
  }
  // the draw
  int next = -1;
  while (true) {
    double total, sq;
    row_sums(std::false_type{}, total, sq);
    if (total == 0.0 && levels > 0) {                      // no mass: from the distribution before
      --levels;
      continue;
    }
    if (!(total > 0.0 && total < INFINITY)) break;
    const double want = double(a.u_next[i]) * total;
    // the wave's part that holds it (the last one with mass, should rounding leave none), then the
    // sixteenth of that, then the value
    double before = 0.0, upto = 0.0;
    int at = 0;
    bool found = false;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const double v = s_sum[k];
      if (!found && v > 0.0) {
        before = upto;
        at = k;
        found = upto + v > want;
      }
      upto += v;
    }
    __syncthreads();
    const int x0 = at * part, sub = part / NW;             // (a multiple of 16)
    double r, w;
    range_sum(std::false_type{}, min(V, x0 + wave * sub), min(V, x0 + (wave + 1) * sub), r, w);
    if (lane == 0) s_sum[wave] = r;
    __syncthreads();
    upto = before;
    int at2 = 0;
    found = false;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const double v = s_sum[k];
      if (!found && v > 0.0) {
        before = upto;
        at2 = k;
        found = upto + v > want;
      }
      upto += v;
    }
    if (wave == 0) {
      // 64 values at a time
      const int lo = min(V, x0 + at2 * sub), hi = min(V, lo + sub);
      int hit = -1, last = -1;
      for (int y = lo; y < hi && hit < 0; y += 64) {
        const int xx = y + lane;
        const float pv = xx < hi ? p[xx] : 0.0f, qv = !CERTAIN && levels > 0 && xx < hi ? q[xx] : 0.0f;
        const double rv = residual<CERTAIN>(pv, qv, xx, levels, s_ir, s_iz, s_rej);
        double c = rv;
        for (int off = 1; off < 64; off <<= 1) {
          const double o = __shfl_up(c, off);
          if (lane >= off) c += o;
        }
        const uint64_t over = __ballot(rv > 0.0 && before + c > want), some = __ballot(rv > 0.0);
        if (over) hit = y + __ffsll(static_cast<unsigned long long>(over)) - 1;
        if (some) last = y + 63 - __clzll(static_cast<long long>(some));
        before += __shfl(c, 63);
      }
      if (lane == 0) s_hit = hit >= 0 ? hit : last;
    }
    __syncthreads();
    next = s_hit;
    break;
  }
  for (int k = tid; k < a.max_path; k += NT) path[k] = k < count ? s_path[k] : -1;
  if (tid == 0) {
    a.count[i] = count;
    a.next[i] = next;
  }
}

}  // namespace

// A launch's threads are below 2^32: as many workgroups of NT as one of them has.
constexpr int64_t AT_ONCE = int64_t(1) << 21;

hipError_t token_probs(const void* logits, bool bf16, int64_t ldl, int64_t T, int64_t V, const float* temperature,
                       float* P, int64_t ldp, hipStream_t st) {
  auto go = [&](auto ti, auto nv) {
    using TI = decltype(ti);
    // parts of a row: one for each of its steps of NT pieces, as long as all workgroups have a compute unit
    // and rows get four or more (us a call with parts | one: 64 rows of 128,256 21.2 | 24.1, but 100 rows of
    // 128,256 in two parts 28.0 | 27.0)
    const int64_t steps = V / (16 / int64_t(sizeof(ti))) / NT;
    const int64_t parts = T > 64 ? 1 : std::max<int64_t>(1, std::min<int64_t>({8, 256 / T, steps}));
    for (int64_t t = 0; t < T; t += AT_ONCE)
      hipLaunchKernelGGL((probs_kernel<TI, decltype(nv)::value>), dim3(unsigned(std::min(T - t, AT_ONCE)), unsigned(parts)),
                         dim3(NT), 0, st, static_cast<const TI*>(logits) + t * ldl, ldl, V,
                         temperature ? temperature + t : nullptr, P + t * ldp, ldp);
  };
  // as many pieces as the row has (code for more would come from memory as it runs: five rows of 32,000 bf16
  // logits 7.1 us with 4, 7.8 with 16); fp32 rows spill from 16 on
  auto held = [&](auto ti) {
    const int64_t pieces = V / (16 / int64_t(sizeof(ti))), per = (pieces + NT - 1) / NT;
    if (per <= 4) go(ti, std::integral_constant<int, 4>{});
    else if (per <= 8) go(ti, std::integral_constant<int, 8>{});
    else if constexpr (sizeof(ti) == 2) go(ti, std::integral_constant<int, 16>{});
    else go(ti, std::integral_constant<int, 12>{});
  };
  if (bf16) held(uint16_t{});
  else held(float{});
  return hipGetLastError();
}

hipError_t tree_verify(const VerifyArgs& a, hipStream_t st) {
  for (int64_t i = 0; i < a.n_seq; i += AT_ONCE) {
    VerifyArgs b = a;
    b.q_start += i;
    b.u_next += i;
    b.path += i * a.max_path;
    b.count += i;
    b.next += i;
    const dim3 grid(unsigned(std::min(a.n_seq - i, AT_ONCE)));
    if (a.Q) hipLaunchKernelGGL(verify_kernel<false>, grid, dim3(NT), 0, st, b);
    else hipLaunchKernelGGL(verify_kernel<true>, grid, dim3(NT), 0, st, b);
  }
  return hipGetLastError();
}

}  // namespace oq
