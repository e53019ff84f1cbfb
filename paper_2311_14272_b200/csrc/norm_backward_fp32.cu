#include "norm_backward.cuh"

namespace crisp {
namespace norm {

cudaError_t backward_fp32(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st) { return backward<float>(p, q, one, vec, from8, st); }

}  // namespace norm
}  // namespace crisp
