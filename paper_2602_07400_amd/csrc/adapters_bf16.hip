// Low-rank adapters with bfloat16 weights.
#include "adapters_pass.h"

namespace bl {
namespace adapt {

template hipError_t launch_pass<kBf16>(const PassArgs &, bool, bool, hipStream_t);
template hipError_t launch_grads<kBf16>(const GradArgs &, hipStream_t);
template int32_t grad_block<kBf16>();
template bool fits_narrow<kBf16>(int32_t, int32_t, int32_t, bool);

}  // namespace adapt
}  // namespace bl
