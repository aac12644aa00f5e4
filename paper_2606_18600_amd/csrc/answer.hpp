// Host-side launchers of the answer operators: 8-bit products, token
// probabilities and draft verification. Like those of kernels.hpp they enqueue
// on the given stream, return the launch status and allocate nothing.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"

namespace stage_k {

// An 8-bit matrix: [rows, K] int8 values and one fp32 scale per row, for
// activations and weights alike. The values are whole operand fragments of
// v_mfma_i32_16x16x64_i8 (16 rows x 64 k, 1 KB, lane l holding row l % 16, k
// (l / 16) * 16 .. + 15): fragment (row / 16, k / 64) at index
// (row / 16) * (kp / 64) + k / 64, so that 16 rows are one contiguous strip.
// Rows are padded to 16 (undefined values, whose products nobody stores), K to
// kp, a multiple of 128, with zeros. The scales follow the values.
inline size_t quant_kp(int K) { return ((size_t)K + 127) / 128 * 128; }
inline size_t quant_rows16(int rows) { return ((size_t)rows + 15) / 16 * 16; }
inline size_t quant_scales_at(int rows, int K) { return quant_rows16(rows) * quant_kp(K); }
inline size_t quant_bytes(int rows, int K) {
  return quant_scales_at(rows, K) + quant_rows16(rows) * sizeof(float);
}
constexpr int kQuantMaxK = 131072;  // 127 * 127 * K stays below 2^31

// dst = the 8-bit matrix of src [rows, K] (fp32 or bf16, row stride ld).
hipError_t quant_rows(DType dt, const void* src, int64_t ld, int rows, int K, void* dst,
                      hipStream_t s);
// ... of int8 values and scales [rows] that the caller has.
hipError_t quant_pack(const int8_t* src, int64_t ld, const float* scales, int rows, int K,
                      void* dst, hipStream_t s);
// ... of RMSNorm(src) * gain in fp32 (K <= 16384, K % 128 == 0); row t is row
// idx[t] of src (idx: device, or nullptr for row t).
hipError_t quant_norm_rows(DType dt, const void* src, const int32_t* idx, const void* gain,
                           float eps, int rows, int K, void* dst, hipStream_t s);

// The kernels of a product (k_quant.hip): operands streamed into registers by
// blocks of 1 to 3 strips of 16 columns; the skinny kernel with NF strips for each
// of WC groups of waves; tiles of BM x BN strips.
enum QuantKernel {
  QUANT_STREAM_1,
  QUANT_STREAM_2,  // (rows quantised on the way only)
  QUANT_STREAM_3,
  QUANT_SKINNY_2X2,
  QUANT_SKINNY_4X2,
  QUANT_SKINNY_4X4,
  QUANT_SKINNY_4X8,
  QUANT_TILE_16X16,
  QUANT_TILE_12X8,
  QUANT_TILE_8X8,
  QUANT_TILE_4X8,
  QUANT_TILE_4X4,
  QUANT_TILE_4X4_K2  // two parts of k in a block: ranges of a multiple of 4 k tiles
};
constexpr int kStreamStrips = 4;   // row strips of 16 that the stream kernel takes
constexpr int kSkinnyStrips = 12;  // ... and the skinny kernel
// Row strips that the skinny kernel is built for: 1 and the even numbers.
constexpr int quant_skinny_strips(int strips) { return strips <= 1 ? 1 : (strips + 1) / 2 * 2; }
// A product's kernel and its k ranges of kt_len k tiles of 64. Several ranges
// leave an int32 plane [M][N rounded up to 16] each, which a last kernel adds.
// fused: the stream kernel quantises the rows itself (quant_linear).
struct QuantPlan {
  QuantKernel kernel = QUANT_TILE_4X4;
  int ranges = 1, kt_len = 0;
  bool fused = false;
};
constexpr int kFusedRows = 4;
// The plan of a product whose planes may take `room` bytes; with x_bytes, of rows
// that are still to be quantised, from values of so many bytes.
QuantPlan quant_plan(int M, int N, int K, size_t room, int x_bytes = 0);
size_t quant_plane_bytes(const QuantPlan& p, int M, int N);
// out [M, N] (fp32 or bf16, row stride ldo) = a b^T for the 8-bit matrices a
// [M, K] and b [N, K]; planes: quant_plane_bytes() bytes.
hipError_t quant_product(const QuantPlan& p, const void* a, int M, const void* b, int N, int K,
                         DType out_dt, void* out, int64_t ldo, void* planes, hipStream_t s);
// ... of rows x [M, K] (fp32 or bf16, row stride ld) that are quantised on the way.
// ws: quant_linear_bytes().
inline size_t quant_planes_at(int M, int K) { return (quant_bytes(M, K) + 15) / 16 * 16; }
inline size_t quant_linear_bytes(const QuantPlan& p, int M, int N, int K) {
  return p.fused ? 0 : quant_planes_at(M, K) + quant_plane_bytes(p, M, N);
}
hipError_t quant_linear(const QuantPlan& p, DType dt, const void* x, int64_t ld, int M,
                        const void* b, int N, int K, DType out_dt, void* out, int64_t ldo,
                        void* ws, hipStream_t s);

// probs[r] = softmax(logits[r] / temperature[r]) (temperature: device [rows],
// nullptr for 1). ws: token_probs_bytes().
size_t token_probs_bytes(int rows, int vocab);
hipError_t token_probs(DType in_dt, const void* logits, int64_t ld_in, int rows, int vocab,
                       const float* temperature, DType out_dt, void* probs, int64_t ld_out,
                       void* ws, hipStream_t s);

struct VerifyArgs {
  const void* target;  // [n_drafts + seqs, vocab]
  int64_t ld_target;
  const void* draft;  // [n_drafts, vocab] or nullptr
  int64_t ld_draft;
  int vocab;
  const int32_t* drafts;  // [n_drafts]
  const int32_t* starts;  // [seqs + 1]
  int seqs, n_drafts, most;
  const float* accept_u;  // [n_drafts]
  const float* sample_u;  // [seqs]
  int32_t* n_accepted;    // [seqs]
  int32_t* tokens;        // [seqs, most + 1]
};
size_t verify_bytes(int seqs, int vocab);
hipError_t verify_drafts(DType dt, const VerifyArgs& a, void* ws, hipStream_t s);

}  // namespace stage_k
