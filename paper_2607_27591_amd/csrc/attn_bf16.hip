#include "attn.hpp"

namespace prox {

hipError_t launch_attn_bf16(AttnArgs &a, hipStream_t s) { return launch_attn_dt<kBF16>(a, s); }

}  // namespace prox
