#include "attention.hpp"

namespace sv {
void launch_attention_bf16(const AttnArgs& a, const AttnLaunch& t) { launch_attention<SV_BF16, SV_BF16>(a, t); }
}  // namespace sv
