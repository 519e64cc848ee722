// Attention over pages in bf16.
#include "photon_paged_attn.h"
#include "photon_paged_attn_wide.h"

namespace photon {

int32_t paged_attn_bf16(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st) {
  if (!tile.wide) return paged_launch_types<bf16_t>(a, tile, f32_rows, st);
  switch (kv_row_elems(a.pool.d_h)) {
    case 32: return tile.waves == 4 ? paged_launch_wide<1, 4>(a, st) : paged_launch_wide<1, 8>(a, st);
    case 64: return tile.waves == 4 ? paged_launch_wide<2, 4>(a, st) : paged_launch_wide<2, 8>(a, st);
    default: return tile.waves == 4 ? paged_launch_wide<4, 4>(a, st) : paged_launch_wide<4, 8>(a, st);
  }
}

}  // namespace photon
