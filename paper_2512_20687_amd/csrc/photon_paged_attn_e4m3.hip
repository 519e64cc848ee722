// Attention over pages in E4M3.
#include "photon_paged_attn.h"

namespace photon {

int32_t paged_attn_e4m3(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st) {
  return paged_launch_types<fp8_t>(a, tile, f32_rows, st);
}

}  // namespace photon
