#include "norm_backward.cuh"

namespace crisp {
namespace norm {

cudaError_t backward_fp16(const Plan &p, const Norm &q, bool one, bool vec, bool from8, cudaStream_t st) { return backward<__half>(p, q, one, vec, from8, st); }

}  // namespace norm
}  // namespace crisp
