// Internal interface of the norms at the joint of two residual blocks, of dropout and of
// log probabilities.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "pointid.h"
#include "random.h"

namespace pointid {

// ---- dropout.hip
struct DropoutArgs {
  const char* x;
  const char* residual;        // or nullptr
  char* y;
  int64_t ld_x, ld_residual, ld_y;
  int64_t rows, cols;
  int32_t dtype;
  Drop drop;
  int32_t passing;             // set by the launch: see Passing
};
hipError_t launch_dropout(DropoutArgs a, hipStream_t stream);

// ---- norm.hip
// u = (v - mean) / deviation, or v / root of the mean square; u weight + bias.
struct NormOf {
  int32_t kind;                // POINTID_NORM_*
  float eps;
  const float* weight;         // nullptr: ones
  const float* bias;           // nullptr: zeros
};
struct Rows {
  char* p;                     // nullptr: not there
  int64_t ld;
};
// t = scale x + gate * drop(after(o)),  h = before(t); without o: t = x.
// stats: [rows][4] mean and 1 / deviation of `after`, then of `before`.
struct NormArgs {
  Rows x, o, t, h;
  NormOf after, before;
  const float* gate;
  float scale;
  Drop drop;
  float* stats;
  int64_t rows, cols;
  int32_t dtype;
  int32_t lanes, passing;      // set by the launch: a row's threads, and see Passing
};
hipError_t launch_norm(const NormArgs& a, hipStream_t stream);

// Gradients, from dh and dt, of x and o and (sums over rows) of the parameters.  The sums'
// order: before.weight, before.bias, after.weight, after.bias, gate.
constexpr int kNormSums = 5;
struct NormBackArgs {
  Rows dh, dt, t, o, dx, dout;
  NormOf after, before;
  const float* gate;
  float scale;
  Drop drop;
  const float* stats;
  float* out[kNormSums];       // nullptr: not wanted
  float* means;                // scratch [rows][4]: of e, e u, f, f u (see norm.hip)
  float* part;                 // scratch [blocks][wanted sums][cols]
  int32_t blocks;              // of rows
  int64_t rows, cols;
  int32_t dtype;
  int32_t lanes, passing;      // set by the launch: a row's threads, and see Passing
};
// The blocks that leave sums, and whether a block holds whole rows; if not, `means` has to be
// made first.
struct NormBackPlan {
  int32_t blocks;
  bool held;
};
NormBackPlan plan_norm_back(const NormBackArgs& a, int cus);
hipError_t launch_norm_means(const NormBackArgs& a, hipStream_t stream);
hipError_t launch_norm_back(const NormBackArgs& a, bool held, hipStream_t stream);
hipError_t launch_norm_sums(const NormBackArgs& a, hipStream_t stream);

// ---- logprobs.hip
constexpr int kMaxTop = 64;    // alternatives: a list is a wave's lanes
struct ScanArgs {
  Rows x;
  int64_t rows, cols;
  int32_t dtype;
  float scale;
  const int32_t* targets;
  float* logp;
  float* lse;
  float* entropy;
  int32_t top;
  int32_t* top_ids;
  float* top_logp;
  int32_t splits;              // of a row; more than one leave partials for the join
  int64_t split_cols;          // a multiple of 8
  float* part;                 // scratch [rows][splits][4]: maximum, sum, sum of e d
  uint64_t* part_top;          // scratch [rows][splits][top]
};
int32_t scan_splits(int64_t rows, int64_t cols, int cus);
hipError_t launch_logprobs(const ScanArgs& a, hipStream_t stream);
hipError_t launch_logprobs_join(const ScanArgs& a, hipStream_t stream);
struct ScanBackArgs {
  Rows x, dx;
  int64_t rows, cols;
  int32_t dtype;
  float scale;
  const int32_t* targets;
  const float *lse, *entropy, *dlogp, *dentropy, *dlse;
  int32_t lanes, passing;      // set by the launch: a row's threads, and see Passing
};
hipError_t launch_logprobs_back(ScanBackArgs a, hipStream_t stream);

}  // namespace pointid
