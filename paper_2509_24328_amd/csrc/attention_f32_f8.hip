#include "attention.hpp"

namespace sv {
void launch_attention_f32_f8(const AttnArgs& a, const AttnLaunch& t) { launch_attention<SV_F32, SV_F8>(a, t); }
}  // namespace sv
