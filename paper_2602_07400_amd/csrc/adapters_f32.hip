// Low-rank adapters with float32 weights.
#include "adapters_pass.h"

namespace bl {
namespace adapt {

template hipError_t launch_pass<kF32>(const PassArgs &, bool, bool, hipStream_t);
template hipError_t launch_grads<kF32>(const GradArgs &, hipStream_t);
template int32_t grad_block<kF32>();
template bool fits_narrow<kF32>(int32_t, int32_t, int32_t, bool);

}  // namespace adapt
}  // namespace bl
