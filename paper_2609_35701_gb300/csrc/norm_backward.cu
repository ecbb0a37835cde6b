// The norms' backward pass on rows that registers hold: one block per SM, partial sums over rows per block.
#include "norm_backward.cuh"

namespace meq {
namespace norm {

bool launch_row_backward(const BackwardArgs& a, int type, bool layer, int sms, int64_t* parts, cudaStream_t st, cudaError_t* e) {
  return launch_any<false>(a, type, layer, sms, parts, st, e);
}

}  // namespace norm
}  // namespace meq
