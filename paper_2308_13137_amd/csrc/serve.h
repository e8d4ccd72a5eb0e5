// Host-side launchers of the serving operators: RMSNorm to codes, the 8-bit
// integer linear, the paged 8-bit key/value cache and attention over it.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "oq.h"

namespace oq {

// ---------------------------------------------------------------- RMSNorm to codes
constexpr int64_t NORM_MAX_D = 32768;
hipError_t rmsnorm_quant(const void* X, bool x_bf16, const void* R, bool r_bf16, int64_t T, int64_t D,
                         const float* gain, const float* bias, float eps, int bits, bool sym, void* H,
                         void* X_dq, bool dq_bf16, uint8_t* codes, float* h, float* z, hipStream_t st);

// ---------------------------------------------------------------- 8-bit integer linear
// Packed weight: (codes - 128) as int8, rows padded to 16 and columns to 64 with
// zeros, in blocks of 16 rows x 64 columns (1 KiB): block [row / 16][column / 64],
// inside it byte 256 g + 16 r + b holds row 16 i + r, column 64 j + 16 g + b: a
// matrix instruction's A operand is one 16-byte load per lane, 1 KiB per wave.
constexpr int64_t I8_MAX_C_IN = 65536;   // |sum| <= 65536 * 2^14 = 2^30
constexpr int64_t i8_rows(int64_t c_out) { return (c_out + 15) / 16 * 16; }
constexpr int64_t i8_cols(int64_t c_in) { return (c_in + 63) / 64 * 64; }
hipError_t int8_pack(const uint8_t* codes, int64_t c_out, int64_t c_in, int8_t* packed, int32_t* wsum,
                     hipStream_t st);
struct I8Args {
  const uint8_t* x;        // [T, K] codes
  const float *hx, *zx;    // [T]
  int64_t T, K;
  const int8_t* w;         // packed
  const int32_t* wsum;     // [N]
  const float *hw, *zw;    // [N]
  const float* bias;       // [N] | nullptr
  int64_t N;
  void* y;                 // [T, N] fp32 or bf16
};
hipError_t int8_linear(const I8Args& a, bool y_bf16, hipStream_t st);

// ---------------------------------------------------------------- paged 8-bit cache
struct CacheArgs {
  int8_t *kc, *vc;          // [n_pages, Hkv, P d] operand order
  float *ks, *vs;           // [n_pages, Hkv]
  uint16_t *kw, *vw;        // [n_slots, 2, Hkv, P d] bf16 windows
  int n_pages, n_slots, P, lgP, Hkv, d, lgd;   // P = 2^lgP, d = 2^lgd
  const int32_t* table;     // [n_seq, max_pages]
  const int32_t* slot;      // [n_seq] | nullptr: the sequence's number
  const int32_t* length;    // [n_seq] tokens before the call
  const int32_t* q_start;   // [n_seq + 1]
  int n_seq, max_pages, max_q;
  int64_t T;                // rows of the batch's tensors
};
hipError_t cache_append(const CacheArgs& c, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                        const void* V, int64_t ldv, bool in_bf16, int H, const float* rope, int64_t n_rope,
                        const float* s_a, uint16_t* Qout, hipStream_t st);
hipError_t cache_read(const CacheArgs& c, const int32_t* begin, const int32_t* row_start, int64_t rows,
                      int max_rows, void* K, void* V, bool bf16, hipStream_t st);
struct AttendPlan {
  int row_rows;    // rows of a workgroup of the row kernel (16, 32; 0: not used)
  int tile_rows;   // rows of a workgroup of the tile kernel (64, 128; 0: not used)
  int few, many;   // splits of a row's tokens in the two
  int64_t units;   // row tiles of one key head, of all sequences, at most
  int order;       // how they are numbered, with levels (kv_cache.hip, row_tile)
  int64_t levels;
  size_t few_floats, many_floats;  // their shares in the workspace
};
AttendPlan cache_attend_plan(int n_seq, int Hkv, int H, int64_t tokens, int max_q, int64_t max_len, int d);
hipError_t cache_attend(const CacheArgs& c, const uint16_t* Q, int64_t ldq, int H, uint16_t* O, float* LSE,
                        float* ws, const AttendPlan& p, hipStream_t st);

}  // namespace oq
