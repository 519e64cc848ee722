// Paged K/V cache: what its kernels share.  The layout is declared in photon.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "photon_attn.h"
#include "photon_host.h"

namespace photon {

constexpr int PAGED_LEAST = 16;                          // entries of the smallest page: an operand tile of 16 entries lies in one page
constexpr int PAGED_MOST_TREE = 64;                      // nodes of a drafted tree: a bit each
constexpr int64_t PAGED_MOST = (1ll << 31) - 256;        // entries of a sequence: the end of its last page is an int32, too

// The cache as kernels see it.
struct PagedPools {
  uint8_t* k;
  uint8_t* v;
  const int32_t* table;
  int32_t n_pages, page_shift, max_pages, H_kv, d_h;
  int32_t row_bytes;                                     // of a pool's row
  int64_t page_bytes, head_bytes;                        // a page; a page's part of one K/V head
};

inline bool element_aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Checks a cache and fills `out`; the message begins with `who`.
int32_t paged_pools(const char* who, const photon_paged_cache* c, int32_t Bt, int32_t T, PagedPools* out);

}  // namespace photon
