// Attention over pages in fp32.
#include "photon_paged_attn.h"

namespace photon {

int32_t paged_attn_f32(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st) {
  return paged_launch_types<float>(a, tile, f32_rows, st);
}

}  // namespace photon
