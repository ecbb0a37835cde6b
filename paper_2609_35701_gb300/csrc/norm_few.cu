// The norms' backward pass on few rows: one cluster, which adds up the sums over rows itself.
#include "norm_backward.cuh"

namespace meq {
namespace norm {

bool launch_few_backward(const BackwardArgs& a, int type, bool layer, cudaStream_t st, cudaError_t* e) {
  int64_t blocks = 0;
  return launch_any<true>(a, type, layer, 0, &blocks, st, e);
}

}  // namespace norm
}  // namespace meq
