// Internal interface of the layer operators: dense and gated layers, their
// gradients, and 8-bit activation checkpoints.
//
// Every product is one of three forms of a sum over an inner index:
//   forward  z[m][n]  = sum over k of x[m][k] W[k][n]
//   dx       dx[m][k] = sum over n of dz[m][n] W[k][n]
//   dW       dW[k][n] = sum over m of x[m][k] dz[m][n]
// "left" is the operand that the result's rows index, "right" the one its columns
// index.  A gated layer has two right operands (two halves of one result).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "pointid.h"

namespace pointid {

// Values of a 16-bit or fp32 type at p[i * si + k * sk] (i: the result's row or
// column, k: the inner index), one of the strides 1.
struct Strided {
  const void* p;
  int64_t si, sk;
  int32_t dtype;               // POINTID_FP32, _BF16 or _FP16
};

// An 8-bit checkpoint, contiguous: codes [rows][cols], exponents [rows][ceil(cols / 32)].
struct Packed8 {
  uint8_t* codes;
  uint8_t* exponents;
};
constexpr int kBlock8 = 32;

// Where activations kept for the backward pass go to or come from: a matrix of the
// call's type, or a checkpoint (matrix == nullptr).
struct Kept {
  void* matrix;
  int64_t ld;
  Packed8 packed;
  __host__ __device__ bool any() const { return matrix || packed.codes; }
};

enum EndMode { kEndDense = 0, kEndGated = 1, kEndStore = 2, kEndPartial = 3 };

// What becomes of the finished sums of one result (or of two halves of one).
//   kEndDense    v = sum + bias0; keep0 <- v; y0 = act(v) + residual
//   kEndGated    g = sum0 + bias0, u = sum1 + bias1; keep0 <- g; keep1 <- u; y0 = act(g) u
//   kEndStore    y0 = sum0 (and y1 = sum1), fp16 times *unscale where that is given
//   kEndPartial  sums to part[(split * halves + half) * rows + row][part_ld] in fp32
struct End {
  int32_t mode;
  int32_t act;
  int32_t dtype;               // of y0, y1, residual, kept matrices
  int32_t halves;              // 1 or 2
  int64_t rows;
  int64_t cols;                // of each half
  const float* bias0;
  const float* bias1;
  const void* residual;
  int64_t ld_residual;
  void* y0;
  int64_t ld0;
  void* y1;
  int64_t ld1;
  Kept keep0, keep1;
  const float* unscale;
  float* part;
  int64_t part_ld;             // a multiple of 32
};

// One term of the sum: a left operand with one right operand for each half.
struct Term {
  const void* left;
  const void* right0;
  const void* right1;
};
constexpr int kMaxTerms = 12;

// ---- layers_rows.hip: forward products of 1..kFewRows rows; the weights
// [inner][cols] are read once.  splits > 1 leaves partials (end.mode is kEndPartial then).
constexpr int kFewRows = 8;
int few_rows_splits(int64_t inner, int64_t cols, int halves, int cus);
hipError_t launch_layers_rows(const Strided& x, const Strided* w, int64_t inner, const End& end, int splits,
                              hipStream_t stream);

// ---- layers_mm.h: products on the matrix cores.
enum Form { kForward = 0, kDx = 1, kDw = 2 };
struct ProductArgs {
  Term term[kMaxTerms];
  int32_t terms;
  int32_t splits;
  int32_t inner;
  int64_t ld_left;             // elements; 16-bit operands are 16-byte aligned, rows too
  int64_t ld_right;
  // set by the launch: tiles, how the blocks spread over the XCDs, stages a split
  int32_t tiles_m, tiles_n;
  int32_t xcd_each, xcd_more;
  int32_t stages, split_each, split_more;
  End end;
};
// The tile of a launch and its splits of the sum.
constexpr int kTiles = 4, kTiles32 = 4;        // 16-bit: two of 128 x 128, of 3 and 2 stages
constexpr int kTileM[kTiles] = {256, 128, 128, 64}, kTileN[kTiles] = {256, 128, 128, 128};
constexpr int kTileM32[kTiles32] = {256, 128, 64, 64}, kTileN32[kTiles32] = {128, 128, 128, 64};
struct ProductPlan {
  int tile;                    // index into kTileM, kTileN (fp32: kTileM32, kTileN32; columns of both halves)
  int splits;
};
ProductPlan plan_product(bool f32, int64_t rows, int64_t cols, int halves, int64_t inner, int terms, int cus);
hipError_t launch_product_bf16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream);
hipError_t launch_product_fp16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream);
// fp32 operands (4-byte aligned), in three bf16 parts each
hipError_t launch_product_f32(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream);
// Partials of `splits` parts added in order, then `end`.
hipError_t launch_layers_join(const End& end, const float* part, int64_t part_ld, int splits, hipStream_t stream);

// ---- layers_pass.hip: passes over one matrix
// What the products take from scratch: a matrix copied to rows of `ld` values (a multiple of
// 8), zero past its columns, or a checkpoint's values laid out so.
struct FillJob {
  enum Kind { kCopy = 0, kLoad = 1 };
  int32_t kind;
  int32_t dtype;
  const void* src;             // kCopy
  int64_t ld_src;
  Packed8 packed;              // kLoad
  int64_t rows, cols;
  void* out;
  int64_t ld;
  uint32_t first;              // set by the launch: the job's first block
};
struct FillJobs {
  FillJob job[3];
  int32_t count;
};
hipError_t launch_layers_fill(FillJobs jobs, hipStream_t stream);
// The column sums of a gradient from the sums of its blocks of rows: 32 columns of a half a
// block.
struct SumsJobs {
  const float* part;           // [rows][halves][cols]
  int64_t rows, cols;
  int32_t halves;
  float* out[2];               // nullptr: not wanted
  uint32_t half_blocks() const { return (uint32_t)((cols + 31) / 32); }
  uint32_t blocks() const { return half_blocks() * (uint32_t)halves; }
};
hipError_t launch_layers_sums(const SumsJobs& jobs, hipStream_t stream);
// A checkpoint's values as a matrix.
hipError_t launch_checkpoint_load(const Packed8& src, int64_t rows, int64_t cols, int dtype, void* out, int64_t ld,
                                  hipStream_t stream);
hipError_t launch_checkpoint_save(const void* src, int64_t ld, int dtype, int64_t rows, int64_t cols,
                                  const Packed8& out, hipStream_t stream);
hipError_t launch_layers_zero(void* out, int64_t ld, int dtype, int64_t rows, int64_t cols, hipStream_t stream);
// The gradient before the activation, and its column sums.
//   dense: dz = dy act'(z) (z absent: dy)     gated: dg = dy u act'(g), du = dy act(g)
// parts: 0 none written, 1 or 2 planes of the 16-bit type (2: value and remainder),
// -1 fp32 values.  col_part: [row blocks][halves][cols] sums of each block of rows, or
// nullptr.  maxima: nullptr, or (fp16) what launch_layers_grad_max left: the values written
// are those times the power of two that brings the largest finite magnitude to [2^14, 2^15),
// and *unscale <- the power that undoes it.
struct GradArgs {
  const void* dy;
  int64_t ld_dy;
  int32_t dtype;
  int32_t act;
  int32_t halves;
  Kept z[2];                   // dense: z; gated: g, u
  int64_t rows, cols;
  int32_t parts;
  void* out[2];                // each half: planes [parts][rows][ld], or fp32 [rows][ld]
  int64_t ld, plane;
  float* col_part;
  uint32_t* maxima;
  uint32_t maxima_count;
  float* unscale;
  uint32_t row_blocks, strips;  // set by the launch
};
// Rows of a block: 32, or 8 where that gives fewer than two blocks a CU.
int grad_rows(int64_t rows, int64_t cols, int cus);
// The largest finite magnitudes (their bits) of a fp16 gradient's values, one a block, in
// grad_max_blocks() words.
constexpr uint32_t kMostMaxima = 1024;
uint32_t grad_max_blocks(int64_t rows, int64_t cols);
hipError_t launch_layers_grad_max(const GradArgs& a, hipStream_t stream);
// `fill`: jobs that the same launch takes.
hipError_t launch_layers_grad(GradArgs a, int block_rows, FillJobs fill, hipStream_t stream);

// ---- layers_mm.h: the products dx and dW of a gradient by one launch of one tile shape, and
// its column sums.  splits of each; tile < 0: by launches of their own.
struct PairPlan {
  int tile;
  int dx_splits, dw_splits;
};
PairPlan plan_pair(bool f32, int64_t m, int64_t k, int64_t n, int halves, int parts, int cus);
hipError_t launch_pair_bf16(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream);
hipError_t launch_pair_f32(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream);
hipError_t launch_pair_fp16(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream);

}  // namespace pointid
