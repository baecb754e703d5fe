#include "attention.hpp"

namespace sv {
void launch_attention_bf16_f8(const AttnArgs& a, const AttnLaunch& t) { launch_attention<SV_BF16, SV_F8>(a, t); }
}  // namespace sv
