// The matrix-core products of fp16 operands.
#include "layers_mm.h"

namespace pointid {

hipError_t launch_product_fp16(Form form, const ProductPlan& plan, ProductArgs a, hipStream_t stream) {
  return mm::launch<true>(form, plan, a, stream);
}

hipError_t launch_pair_fp16(int tile, const ProductArgs& dx, const ProductArgs& dw, const SumsJobs& sums, hipStream_t stream) {
  return mm::launch_pair<true>(tile, dx, dw, sums, stream);
}

}  // namespace pointid
