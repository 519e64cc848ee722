// Attention over pages in bf16.
#include "photon_paged_attn.h"

namespace photon {

int32_t paged_attn_bf16(const PagedAttnArgs& a, bool f32_rows, hipStream_t st) { return paged_launch_types<bf16_t>(a, f32_rows, st); }

}  // namespace photon
