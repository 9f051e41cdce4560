#include "linear.hpp"

namespace prox {

hipError_t launch_linear_bf16(const LinearArgs &a, hipStream_t s) { return launch_linear_dt<kBF16>(a, s); }

}  // namespace prox
