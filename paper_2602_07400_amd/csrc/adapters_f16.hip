// Low-rank adapters with float16 weights.
#include "adapters_pass.h"

namespace bl {
namespace adapt {

template hipError_t launch_pass<kF16>(const PassArgs &, bool, bool, hipStream_t);
template hipError_t launch_grads<kF16>(const GradArgs &, hipStream_t);
template int32_t grad_block<kF16>();
template bool fits_narrow<kF16>(int32_t, int32_t, int32_t, bool);

}  // namespace adapt
}  // namespace bl
