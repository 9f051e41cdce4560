#include "attn.hpp"

namespace prox {

hipError_t launch_attn_f16(AttnArgs &a, hipStream_t s) { return launch_attn_dt<kF16>(a, s); }

}  // namespace prox
