#include "linear.hpp"

namespace prox {

hipError_t launch_linear_f16(const LinearArgs &a, hipStream_t s) { return launch_linear_dt<kF16>(a, s); }

}  // namespace prox
