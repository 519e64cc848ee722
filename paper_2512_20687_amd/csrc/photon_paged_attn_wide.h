// Attention over a paged K/V cache of many rows that share a K/V head (trees, pieces of a prompt): bf16 rows, bf16 pages.
//
// The mathematics is photon_paged_attn.h's.  With more than 64 rows and many streams the matrix cores and the softmax bound it, not the entries: a workgroup
// of WAVES waves of 32 rows stages 64 entries of K and V at a time in LDS (K in two buffers, V in three, loads straight to LDS while the
// other buffers are worked on, one barrier per stage), so that entries are read once for all its rows.  Measured: 64 nodes under 4 heads,
// 16 x 8 streams of 4096 entries of 128 139 to 145 us; 2048 rows, 16 streams of 8191 entries 230 us, 580 TFLOP/s of the definition's products, 1160
// with the weights' second and third parts counted.  Matrix cores are busy for 54 % of the cycles, vector units for 52 %.
//   K     16-byte chunks of a row are permuted by row, so that the 16 rows of an operand lie in different banks
//   V     pairs of chunks likewise; ds_read_b64_tr_b16 hands a lane four entries of one element, as the contraction over entries takes
//         them: the interleaving of the register kernel is the LDS's work here
#pragma once
#include <atomic>

#include "photon_paged_attn.h"

namespace photon {

constexpr int WIDE_STAGE = 64;                 // entries of a stage
constexpr int WIDE_TILES = 2;                  // row tiles of a wave

constexpr int WIDE_VBUF = 3;                   // V is kept for a stage longer than K (see the loop)

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* lds_short4_t;

// load16_to_lds from a wave-uniform address and an offset per lane: no arithmetic per load.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load16_to_lds_from(const void* base, uint32_t offset, uint32_t lds_base) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  const uint64_t in = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(in), "s"(__builtin_amdgcn_readfirstlane(lds_base)) : "memory", "m0");
}
#pragma clang diagnostic pop

// Every load and LDS access of this wave is complete, and every wave of the workgroup is here.
__device__ __forceinline__ void wide_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// PAGES: of a stage (its 64 entries lie in one page, or in up to four).
template <int NB, int WAVES, int PAGES> __global__ __launch_bounds__(WAVES * 64, 2) void paged_attn_wide_kernel(PagedAttnArgs a) {
  using Y = PagedTypes<bf16_t, bf16_t, NB>;
  constexpr int DP = Y::DP, TILES = Y::TILES, R = WIDE_TILES, ROW = 2 * DP, CHUNKS = ROW / 16;
  constexpr int STAGE = WIDE_STAGE * ROW, VBUF = WIDE_VBUF;       // bytes of a stage's K, or V
  constexpr int LOADS = WIDE_STAGE * ROW / 1024, ROWS_LOAD = 1024 / ROW, PER = 2 * LOADS / WAVES;   // loads of a matrix; rows of one; a wave's, of both
  extern __shared__ __align__(16) char wide_lds[];                           // K [2 buffers][64][ROW], then V [VBUF buffers][64][ROW]
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)wide_lds));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;

  int row_group, hk, split, b;
  if (!paged_unit(a, row_group, hk, split, b)) return;
  int n, m, past;
  paged_sequence(a, paged_counts(a, b), n, m, past);
  const int rows = m * a.group, group_first = row_group * (WAVES * R * 16), first = group_first + wave * (R * 16);
  if (group_first >= rows) return;
  const int group_last = min(group_first + WAVES * R * 16, rows) - 1, last = min(first + R * 16, rows) - 1;
  const int hi = a.tree ? n : min(n, past + group_last / a.group + 1);
  const int stages = hi <= 0 ? 0 : (hi + WIDE_STAGE - 1) / WIDE_STAGE;
  const int s0 = (int)((int64_t)stages * split / a.n_splits), s1 = (int)((int64_t)stages * (split + 1) / a.n_splits);
  const bool has_rows = first < rows;
  const int wave_hi = !has_rows ? 0 : a.tree ? n : min(n, past + last / a.group + 1);

  PagedRows<bf16_t, bf16_t, NB, R> q;
  float top[R], sum[R];
  f32x4_t acc[R][TILES];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = PAGED_LOWEST;
    sum[r] = 0.f;
#pragma unroll
    for (int j = 0; j < TILES; ++j) acc[r][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // A row's 16-byte chunk i lies at chunk i ^ k_turn(row) of the row (K), i ^ v_turn(row) (V).
  auto k_turn = [](int row) { return (row * NB / 4) & (CHUNKS - 1); };
  auto v_turn = [](int row) { return ((row * NB / 4) & (CHUNKS / 2 - 1)) * 2; };
  const int32_t* table = a.pool.table + (int64_t)b * a.pool.max_pages;
  bool bad_page = false;
  constexpr int PART = WIDE_STAGE / PAGES;                                   // entries that are together for certain
  struct Pages { int32_t page[PAGES]; };
  auto pages = [&](int stage) {                                              // behind the last entry: the last one's
    Pages p;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) p.page[i] = table[min(stage * WIDE_STAGE + PART * i, max(n - 1, 0)) >> a.pool.page_shift];
    return p;
  };
  struct Places {
    int64_t at[PAGES];                                                       // where the parts lie (nowhere: the pool's first entries)
    uint32_t there;                                                          // bit i: tile i is somewhere
  };
  auto places = [&](const Pages& pages, int stage) {
    Places p;
    p.there = 0;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) {
      const int entry = stage * WIDE_STAGE + PART * i, page = __builtin_amdgcn_readfirstlane(pages.page[i]);
      const bool inside = page >= 0 && page < a.pool.n_pages, used = entry < n;
      bad_page = bad_page || (used && !inside);
      p.there |= used && inside ? (PAGES == 1 ? 15u : 1u << i) : 0u;
      const int64_t row = (((int64_t)(used && inside ? page : 0) * a.pool.H_kv + hk) << a.pool.page_shift) + (entry & ((1 << a.pool.page_shift) - 1));
      p.at[i] = row * ROW;
    }
    return p;
  };
  // Half of the waves load K, half V: load u of a wave is its matrix's load HALF u + wave % HALF, ROWS_LOAD rows of one tile.
  constexpr int HALF = WAVES / 2, SPAN = HALF > NB ? HALF / NB : 1;
  const int mine = wave % HALF;
  const uint8_t* const pool = wave < HALF ? a.pool.k : a.pool.v;
  const uint32_t lds_mine = lds + (wave < HALF ? 0 : 2 * STAGE) + mine * 1024;
  uint32_t from[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int row = (HALF * u + mine) * ROWS_LOAD + lane / CHUNKS, chunk = lane % CHUNKS;
    from[u] = row % PART * ROW + (chunk ^ (wave < HALF ? k_turn(row) : v_turn(row))) * 16;
  }
  auto load_in = [&](const Places& p, int buffer, int u) {                     // buffer: of this wave's matrix
    int64_t at = p.at[0];
    if constexpr (PAGES > 1) {
      at = p.at[HALF * u / NB];
#pragma unroll
      for (int i = 1; i < SPAN; ++i) at = mine / NB == i ? p.at[HALF * u / NB + i] : at;
    }
    load16_to_lds_from(pool + at, from[u], lds_mine + buffer * STAGE + u * (HALF * 1024));
  };
  // LDS places of this lane's operands in the first tile: K's of product f is k_at ^ 64 f, V's of elements 16 j .. is v_at ^ 32 j
  const uint32_t k_first = c * ROW + (g ^ k_turn(c)) * 16;
  const uint32_t v_first = (4 * g + (c >> 2)) * ROW + (((c & 3) >> 1) ^ v_turn(4 * g + (c >> 2))) * 16 + (c & 1) * 8;

  // A stage's scores and weights, its K in LDS at `in`.  CAREFUL: a row may not see every entry of it.
  float s[R][16];
  uint32_t seen[R] = {};
  auto weigh = [&](auto careful, const char* in, int base, uint32_t now, auto request) {
    constexpr bool CAREFUL = decltype(careful)::value;
    uint32_t k_at = k_first;
    asm volatile("" : "+v"(k_at));                                           // an exclusive-or a read, not a register for each over the whole loop
    f32x4_t d[R][4];
    // Two tiles side by side: a product whose sum the next but one continues waits for it, of four sums none does.  Operands of the
    // next two are requested as those of these are used up: the compiler, left to itself, reads each right before its use.
    uint4_t key[2][NB];
    auto read_keys = [&](int i, int f) {
#pragma unroll
      for (int t = 0; t < 2; ++t) key[t][f] = *reinterpret_cast<const uint4_t*>(in + (i + t) * 16 * ROW + (k_at ^ (64 * f)));
    };
#pragma unroll
    for (int f = 0; f < NB; ++f) read_keys(0, f);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) d[r][i + t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < NB; ++f) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < R; ++r)
            d[r][i + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(key[t][f]), q.operand(r, 0, f), d[r][i + t], 0, 0, 0);
        if (i == 0) read_keys(2, f);
        if (f % 2 == 0 && f / 2 < 2) request(i + f / 2);
      }
      if (NB < 4) request(i + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    settle(d);
    if constexpr (CAREFUL) {
      const bool there[4] = {(now & 1) != 0, (now & 2) != 0, (now & 4) != 0, (now & 8) != 0};
#pragma unroll
      for (int r = 0; r < R; ++r) seen[r] = q.template seen<4>(a, r, base, g, n, past, there);
    }
    paged_weights<CAREFUL, R, 4, TILES>(d, a.half_scale, seen, top, sum, acc, s);
  };
  // The values under those weights, V in LDS at `in`, 32 entries at a time.
  auto add_values = [&](auto careful, const char* in, int base, uint32_t now) {
    constexpr bool CAREFUL = decltype(careful)::value;
    uint32_t v_at = v_first;
    asm volatile("" : "+v"(v_at));
    const bool there[4] = {(now & 1) != 0, (now & 2) != 0, (now & 4) != 0, (now & 8) != 0};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const char* values = in + half * PAGED_STEP * ROW;
      uint4_t keep = {~0u, ~0u, ~0u, ~0u};                                   // of a lane's eight entries
      bool some = false;                                                     // an infinity or NaN that some row sees
      if constexpr (CAREFUL) {
        // Entries that no row sees may hold anything: zeros.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int entry = base + half * PAGED_STEP + i / 2 * 16 + 4 * g + i % 2 * 2;
          const bool tile = there[2 * half + i / 2];
          keep[i] = (entry < n && tile ? 0xffffu : 0u) | (entry + 1 < n && tile ? 0xffff0000u : 0u);
        }
        if (m > 1 || a.tree) {                                                // a node need not see itself
          const int mine = half * PAGED_STEP + lane / 2;                     // entry of the stage that this lane looks at, half of its row
          const bool used = base + mine < n && (lane < 32 ? there[2 * half] : there[2 * half + 1]);
          bool bad = false;
#pragma unroll
          for (int i = 0; i < CHUNKS / 2; ++i) {
            const uint4_t x = *reinterpret_cast<const uint4_t*>(in + mine * ROW + (lane % 2 * (CHUNKS / 2) + i) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) bad = bad || without_unbounded<bf16_t>(x[e]) != x[e];
          }
          some = __builtin_amdgcn_ballot_w64(bad && used) != 0;
        }
      }
      bf16x8_t p[R][Y::P_PARTS];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint4_t w[Y::P_PARTS];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = s[r][8 * half + 2 * i], y = s[r][8 * half + 2 * i + 1];
#pragma unroll
          for (int part = 0; part + 1 < Y::P_PARTS; ++part) {
            w[part][i] = high_halves(x, y);
            x -= high_part(x);
            y -= high_part(y);
          }
          w[Y::P_PARTS - 1][i] = pack_bf16x2(x, y);
        }
#pragma unroll
        for (int part = 0; part < Y::P_PARTS; ++part) p[r][part] = as_bf16x8(w[part]);
      }
      constexpr int SIDE = 2;                                                // operands side by side, as above, and as many requested ahead
      uint4_t ahead[SIDE];
      auto read_values = [&](int j) {
#pragma unroll
        for (int t = 0; t < SIDE; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint2v_t w = __builtin_bit_cast(uint2v_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(values + i * 16 * ROW + (v_at ^ (32 * (j + t))))));
            ahead[t][2 * i] = w[0];
            ahead[t][2 * i + 1] = w[1];
          }
      };
      read_values(0);
#pragma unroll
      for (int j = 0; j < TILES; j += SIDE) {
        uint4_t value[SIDE];
#pragma unroll
        for (int t = 0; t < SIDE; ++t) value[t] = ahead[t];
        if (j + SIDE < TILES) read_values(j + SIDE);
        __builtin_amdgcn_sched_barrier(6);                                   // arithmetic may pass
        if constexpr (CAREFUL) {
#pragma unroll
          for (int t = 0; t < SIDE; ++t) {
            value[t] &= keep;
            if (some) {
#pragma unroll
              for (int r = 0; r < R; ++r)
                add_unbounded(acc[r][j + t], __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unbounded_codes(value[t])), as_bf16x8(seen_operand(seen[r] >> (8 * half))),
                                                                                     f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0));
#pragma unroll
              for (int i = 0; i < 4; ++i) value[t][i] = without_unbounded<bf16_t>(value[t][i]);
            }
          }
        }
#pragma unroll
        for (int part = Y::P_PARTS - 1; part >= 0; --part)
#pragma unroll
          for (int t = 0; t < SIDE; ++t)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][j + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(value[t]), p[r][part], acc[r][j + t], 0, 0, 0);
      }
    }
  };

  // Stages that every row of the workgroup sees whole come first; from the first other one on, all steps are taken with care.  Code of
  // both in one loop would cost the ordinary steps their registers.
  const int group_sees = a.tree ? past : past + group_first / a.group + 1;
  Pages ahead = pages(s0);
  Places next = places(ahead, s0);
  uint32_t now = next.there;
  ahead = pages(s0 + 1);
  int stage = s0;
  if (s0 < s1) {
#pragma unroll
    for (int u = 0; u < PER; ++u) load_in(next, 0, u);
  }
  q.load(a, b, hk, first, c, g);                                        // behind the first stage's requests: one latency for both
  int k_buffer = 0, v_buffer = 0;                                            // this stage's
  auto begin = [&]() {                                                       // this stage is there, and what it is not to use no longer read
    next = places(ahead, stage + 1);
    ahead = pages(stage + 2);                                                // requested a stage before they are needed
    wide_barrier();
  };
  // The next stage's loads (behind the last one: of entries that nothing uses), a quarter at a time: a burst of them holds a wave up for
  // as long as its products take.
  auto request = [&](int quarter) {
    const int buffer = wave < HALF ? k_buffer ^ 1 : v_buffer + 1 == VBUF ? 0 : v_buffer + 1;
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (u * 4 / PER == quarter) load_in(next, buffer, u);
  };
  auto end = [&]() {
    ++stage;
    k_buffer ^= 1;
    v_buffer = v_buffer + 1 == VBUF ? 0 : v_buffer + 1;
    now = next.there;
  };
  auto keys = [&]() { return wide_lds + k_buffer * STAGE; };
  auto values = [&](int buffer) { return wide_lds + 2 * STAGE + buffer * STAGE; };
  // Two waves that share a SIMD and do the same at the same time wait for each other: both for the matrix core, then both for the vector
  // unit.  So the second half of a workgroup's waves adds a stage's values after the next barrier, when the first half is at its scores,
  // and is at its weights when they are at their values.  Of two workgroups of four waves, which share a unit's SIMDs, so does the one.
  const bool late = WAVES == 8 ? wave >= HALF : ((blockIdx.x >> 8) & 1) != 0;
#pragma unroll 1
  while (stage < s1 && (stage + 1) * WIDE_STAGE <= group_sees && now == 15) {
    begin();
    if (has_rows) {
      if (late && stage > s0) add_values(std::false_type{}, values(v_buffer == 0 ? VBUF - 1 : v_buffer - 1), 0, 15);
      weigh(std::false_type{}, keys(), 0, 15, request);
      if (!late) add_values(std::false_type{}, values(v_buffer), 0, 15);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) request(i);
    }
    end();
  }
  if (late && has_rows && stage > s0) add_values(std::false_type{}, values(v_buffer == 0 ? VBUF - 1 : v_buffer - 1), 0, 15);
  q.look(a, b, m, past, first, rows, c);
#pragma unroll 1
  while (stage < s1) {
    begin();
    const int base = stage * WIDE_STAGE;
    if (base < wave_hi) {
      weigh(std::true_type{}, keys(), base, now, request);
      add_values(std::true_type{}, values(v_buffer), base, now);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) request(i);
    }
    end();
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                         // no load outlives the workgroup's LDS
  settle(acc);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(any_unbounded(acc)) != 0, 0) && has_rows)
    restore_unbounded<bf16_t>(a, q, acc, table, hk, n, past, 2 * s0, 2 * s1, 1, c, g, [](int j, int i) { return 16 * j + i; });
  paged_say(a, bad_page, lane);

  // lane (c, g) holds elements 16 j + 4 g .. + 3 of its rows
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float l = over_row(sum[r], [](float x, float y) { return x + y; });
    const float mean = l == 0.f ? 0.f : 1.f / l;
    const int row = first + r * 16 + c;
    if (row >= rows) continue;
    const int64_t to = paged_row(a, b, hk, row);
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
      const float o[4] = {acc[r][j][0] * mean, acc[r][j][1] * mean, acc[r][j][2] * mean, acc[r][j][3] * mean};
      paged_emit<bf16_t, DP>(a, to, split, 16 * j + 4 * g, o, top[r], l);
    }
  }
}

template <int NB, int WAVES, int PAGES> int32_t paged_launch_wide_pages(const PagedAttnArgs& a, hipStream_t st) {
  const unsigned grid = a.row_groups > 1 ? (unsigned)((a.units + 7) / 8 * 8) * (unsigned)a.row_groups : (unsigned)a.units;
  constexpr unsigned LDS = (2 + WIDE_VBUF) * WIDE_STAGE * 64 * NB;
  if constexpr (LDS > (64u << 10)) {                             // has to be allowed once on every device
    static std::atomic<bool> allowed[64];
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64 || !allowed[device].load(std::memory_order_relaxed)) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(paged_attn_wide_kernel<NB, WAVES, PAGES>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS);
      if (e != hipSuccess) return fail(PHOTON_ERR_HIP, "paged_attn_wide_kernel: %u bytes of LDS: %s", LDS, hipGetErrorString(e));
      if (device >= 0 && device < 64) allowed[device].store(true, std::memory_order_relaxed);
    }
  }
  PHOTON_LAUNCH(KC_COARSE_ATTN, st, (paged_attn_wide_kernel<NB, WAVES, PAGES>), dim3(grid), dim3(WAVES * 64), LDS, st, a);
  return check_launch("paged_attn_wide_kernel");
}
template <int NB, int WAVES> int32_t paged_launch_wide(const PagedAttnArgs& a, hipStream_t st) {
  return (1 << a.pool.page_shift) >= WIDE_STAGE ? paged_launch_wide_pages<NB, WAVES, 1>(a, st) : paged_launch_wide_pages<NB, WAVES, 4>(a, st);
}

}  // namespace photon
