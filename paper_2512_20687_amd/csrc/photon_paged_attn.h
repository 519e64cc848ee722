// Attention over a paged K/V cache: the kernel.
//
// Mathematics.  For the rows q_r of a stream (token t, query head h; T * H / H_kv of them share a K/V head), one pass over the
// entries keeps per row the reference top_r, the sum l_r = sum_j 2^(s_rj - top_r) and o_r = sum_j 2^(s_rj - top_r) V_j, with
// s_rj = q_r . K_j * scale * log2 e.  top_r rises only when a lane's weights add up to more than 1 (then l_r and o_r shrink), and to 8 above
// the largest score, so that most steps need nothing from another lane and yet no weight is above 1: |o_r| stays within the sum of |V_j|.
// The result is o_r / l_r; parts of the entries are put together as means weighted by l_r 2^top_r.
// References are kept, compared and stored as half of that exponent: log2 e times a score of up to FLT_MAX would pass it.
//
// Operands.  A wave takes R tiles of 16 rows over steps of 32 entries, in registers alone:
//   S^T = K Q^T   A: 16 entries x elements, a lane's operand is what it loads of one entry's row; B: 16 rows x elements.  Lane
//                 (c, g) = (lane % 16, lane / 16) receives the scores of row c with entries 4 g .. 4 g + 3 of either tile of 16
//   O^T = V^T P^T B: those weights as they are: contraction index 8 g + i is entry 4 g + i of the first tile (i < 4) or
//                 4 g + i - 4 of the second.  A: elements x entries: a lane loads elements 2 NB c .. of eight entries and interleaves
//                 pairs of entries (v_perm_b32, one for every two values), since the contraction runs over entries
// so that neither the weights nor V change lanes, nothing goes through LDS, and a row's shrinking factor is in the lane that needs
// it.  fp32 pages: the same with 16x16x4 fp32 products, in which V needs no interleaving.
//
// What bounds it.  Up to 32 rows the entries, once streams fill the chip: 256 x 16 ragged streams of up to 2048 entries of 64 (fp32 rows, bf16
// pages, 1139 MB) 200 us, 5.7 TB/s; 8 x 4 streams of 32749 entries of 128 under 8 heads (537 MB) 101 us, 5.3 TB/s with the merge.  Few and
// short streams take the chain of one: counts, page, entries, two products, the waves' and the splits' merges (16 streams of 2048 fp32
// entries, 16.8 MB: 11.2 us in two launches, of which the merge is 3).
//
// Precision.  Products of bf16 and E4M3 entries (which bf16 holds exactly) run on the bf16 matrix cores.  fp32 queries enter as three
// bf16 parts and so do weights, whatever the rows are: all of their 24 bits.
#pragma once
#include <float.h>

#include <type_traits>

#include "photon_device.h"
#include "photon_paged.h"

namespace photon {

constexpr int PAGED_STEP = 32;                 // entries of a step
constexpr int PAGED_WAVES = 4;                 // of a workgroup
constexpr int64_t PAGED_MOST_ROWS = (1ll << 31) - 4096;   // that share a K/V head: row numbers, tiles' ends among them, are int32
constexpr float PAGED_ABOVE = 4.f;             // a reference that rises is set so far above the row's largest score: weights of 2^-8
constexpr float PAGED_RAISE = 1.f;             // sum of a lane's weights of a step from which on the reference rises
constexpr float PAGED_LOWEST = -FLT_MAX;       // a row's reference before it saw a score: below every score that fp32 holds, halved

struct PagedAttnArgs {
  PagedPools pool;
  const void* q;
  void* out;
  float* ws;                                   // n_splits > 1: [rows of out][n_splits][d_p], then [rows of out][n_splits][top, sum]
  const int32_t *seq_len, *n_new;
  const uint64_t* tree;
  int32_t* status;
  int64_t q_stride;
  int32_t S_max, Bt, T, H, group, row_groups, n_splits, units;   // units: streams * splits
  float half_scale;                            // scale * log2 e / 2
  bool q_pieces, out_pieces;                   // rows of q, of out: aligned to 4 elements
};

// How the rows that share a K/V head are taken: row tiles of a wave, waves side by side over rows, and by which kernel.  While the chip holds all
// workgroups of 32 rows at once (512: two a unit), these win whatever the rows: all four waves go along the entries.  From there on entries are to
// be read fewer times: by workgroups of 64 rows, or the wide kernel's of 128 and 256, where rows and pages are bf16.  Microseconds, bf16
// rows (32-row workgroups / 64-row ones / wide):
//   84 rows, 16 x 8 ragged streams of up to 3000 entries of 128    E4M3 pages 45 / 67     bf16 pages 50 / 71 / 71
//   128 rows, 8 streams of 3000                                    E4M3 19 / 25           bf16 21 / 24 / 34
//   512 rows, 4 x 8 streams of 3000                                E4M3 65 / 72           bf16 73 / 76 / 76
//   48 rows, 64 x 8 ragged streams of up to 1000                   E4M3 44 / 38           bf16 56 / 45 / 61
//   512 rows, 32 x 8 streams of 4096                               E4M3 560 / 534         bf16 676 / 643 / 467
// The wide kernel's eight waves instead of four for up to 128 rows cost ragged streams dear (1024 of up to 1000 entries of 32: 80 us, 57) and
// gain nothing elsewhere (80 rows, 208 streams of 8000 of 52: 191 both).  24 rows in two workgroups of one tile: 19.8 us for 32 streams of 3000
// (in one of two tiles 21.4), but 107 for 256 of 4096 (99).
struct PagedTile {
  int tiles, waves;
  bool wide;                                   // photon_paged_attn_wide.h's
  int rows() const { return 16 * tiles * waves; }
};
inline PagedTile paged_tile(int64_t rows, int64_t streams, bool f32_rows, photon_dtype kv_dt) {
  if (rows <= 16) return PagedTile{1, 1, false};
  if (streams * ((rows + 31) / 32) <= 512) return PagedTile{2, 1, false};
  if (rows <= 64 || f32_rows || kv_dt != PHOTON_BF16) return PagedTile{2, 2, false};
  return PagedTile{2, rows <= 128 ? 4 : 8, true};
}

// Launches over the tile of rows that `a` calls for; one translation unit per page type.
int32_t paged_attn_f32(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st);
int32_t paged_attn_bf16(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st);
int32_t paged_attn_e4m3(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st);

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v_t __attribute__((ext_vector_type(2)));

// x * y, not merged with a subtraction that follows: the reference was rounded, too.
__device__ __forceinline__ float rounded_product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}
__device__ __forceinline__ uint32_t high_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float high_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// Over the four lanes that share a row (16 apart).
template <typename F> __device__ __forceinline__ float over_row(float x, F f) {
  const uint2v_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint2v_t h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

template <int BYTES> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const uint4_t x = *reinterpret_cast<const uint4_t*>(p + 16 * i);
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
  } else if constexpr (BYTES == 8) {
    const uint2v_t x = *reinterpret_cast<const uint2v_t*>(p);
    w[0] = x[0]; w[1] = x[1];
  } else if constexpr (BYTES == 4) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    w[0] = *reinterpret_cast<const uint16_t*>(p);
  }
}

// A word of a pool's elements with zeros in place of infinities and NaN.
template <typename KV> __device__ __forceinline__ uint32_t without_unbounded(uint32_t w) {
  if constexpr (sizeof(KV) == 4) return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
  if constexpr (sizeof(KV) == 2) return w & ~(((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u));
  if constexpr (sizeof(KV) == 1) {
    const uint32_t nan = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;    // a one in every byte that is NaN
    return w & ~(nan * 255u);
  }
}

// What a kernel of these types holds: NB = d_p / 32.
template <typename KV, typename T, int NB> struct PagedTypes {
  static constexpr bool F32 = sizeof(KV) == 4;
  static constexpr int DP = 32 * NB, TILES = 2 * NB;                             // TILES of 16 elements: the value products of a row tile
  static constexpr int K_WORDS = 2 * NB * (int)sizeof(KV);                       // of a lane, per tile of 16 entries
  static constexpr int V_BYTES = 2 * NB * (int)sizeof(KV), V_WORDS = V_BYTES < 4 ? 1 : V_BYTES / 4;   // of a lane, per entry
  static constexpr int Q_PARTS = F32 || sizeof(T) == 2 ? 1 : 3, P_PARTS = 3;
  static constexpr int Q_WORDS = F32 ? 8 * NB : 4 * NB * Q_PARTS;
};

// Element that word 0 of product f's operand begins with in lane group g (bf16 operands: eight from there; fp32: four).
template <typename KV, int NB> __device__ __forceinline__ int operand_element(int f, int g) {
  if constexpr (sizeof(KV) == 4) return 16 * f + 4 * g;                          // f < 2 NB
  if constexpr (sizeof(KV) == 2) return 32 * f + 8 * g;                          // f < NB
  return NB == 4 ? (f / 2) * 64 + 16 * g + (f % 2) * 8 : NB == 2 ? 16 * g + 8 * f : 8 * g;
}

template <typename KV, int NB> __device__ __forceinline__ void load_keys(const uint8_t* row, int g, uint32_t (&w)[2 * NB * sizeof(KV)]) {
  if constexpr (sizeof(KV) == 1) {
    if constexpr (NB == 4) { load_words<16>(row + 16 * g, w); load_words<16>(row + 64 + 16 * g, w + 4); }
    else if constexpr (NB == 2) load_words<16>(row + 16 * g, w);
    else load_words<8>(row + 8 * g, w);
  } else {
#pragma unroll
    for (int f = 0; f < NB * (int)sizeof(KV) / 2; ++f) load_words<16>(row + 64 * f + 16 * g, w + 4 * f);
  }
}

// The bf16 operand of product f out of a lane's key words.
template <typename KV> __device__ __forceinline__ bf16x8_t key_operand(const uint32_t* w, int f) {
  uint4_t x;
  if constexpr (sizeof(KV) == 2) {
    x = uint4_t{w[4 * f], w[4 * f + 1], w[4 * f + 2], w[4 * f + 3]};
  } else {
    x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * f], 1.f, false));
    x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * f], 1.f, true));
    x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * f + 1], 1.f, false));
    x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * f + 1], 1.f, true));
  }
  return as_bf16x8(x);
}

// The bf16 operand of element j (of a lane's 2 NB): eight entries.
template <typename KV, int VW> __device__ __forceinline__ uint4_t value_operand(const uint32_t (&v)[8][VW], int j) {
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(KV) == 2) {
      x[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    } else {
      const uint32_t both = __builtin_amdgcn_perm(v[2 * i + 1][j / 4], v[2 * i][j / 4], j % 4 < 2 ? 0x05010400u : 0x07030602u);
      x[i] = j % 2 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(both, 1.f, true))
                   : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(both, 1.f, false));
    }
  }
  return uint4_t{x[0], x[1], x[2], x[3]};
}

// Four elements of a row of q from element d on; zeros behind the head.
template <typename T> __device__ __forceinline__ void load_query4(const T* row, int d, int d_h, bool pieces, float (&x)[4]) {
  if (pieces && d + 4 <= d_h) {
    if constexpr (sizeof(T) == 4) {
      const float4_t r = *reinterpret_cast<const float4_t*>(row + d);
      x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
    } else {
      const uint2v_t r = *reinterpret_cast<const uint2v_t*>(row + d);
      x[0] = bf16_lo(r[0]); x[1] = bf16_hi(r[0]); x[2] = bf16_lo(r[1]); x[3] = bf16_hi(r[1]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = d + e < d_h ? to_f32<T>(row[d + e]) : 0.f;
  }
}
// Four elements of a row of out.
template <typename T> __device__ __forceinline__ void store_result4(T* row, int d, int d_h, bool pieces, const float (&x)[4]) {
  if (pieces && d + 4 <= d_h) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4_t*>(row + d) = float4_t{x[0], x[1], x[2], x[3]};
    else *reinterpret_cast<uint2v_t*>(row + d) = uint2v_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d + e < d_h) row[d + e] = from_f32<T>(x[e]);
  }
}

// What one row sees and another does not may be an infinity or NaN, and 0 times it is not 0.  Such steps put zeros in the products, and
// a second product tells which rows see which: operands of 2^16 for NaN, 2^8 for -infinity, 1 for infinity, 0 else, times 1 where a
// row sees an entry.  Sums over 32 entries are exact, and their digits say what is added to the row's element.
//
// What all rows see may be infinite, too, and a weight, or one of its parts, may be 0.  Ordinary steps do not look: elements that end
// infinite or NaN are found out at the end, see restore_unbounded().
__device__ __forceinline__ float unbounded_code(float x) { return fabsf(x) <= FLT_MAX ? 0.f : x != x ? 0x1p16f : x < 0.f ? 0x1p8f : 1.f; }
__device__ __forceinline__ uint4_t unbounded_codes(uint4_t w) {               // of bf16 pairs
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = high_halves(unbounded_code(bf16_lo(w[i])), unbounded_code(bf16_hi(w[i])));
  return w;
}
__device__ __forceinline__ uint4_t seen_operand(uint32_t seen) {              // 1 where a lane's row sees its entry, in bf16
  uint4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ((seen >> (2 * i)) & 1u ? 0x3f80u : 0u) | ((seen >> (2 * i + 1)) & 1u ? 0x3f800000u : 0u);
  return w;
}
__device__ __forceinline__ void add_unbounded(f32x4_t& acc, const f32x4_t& digits) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t t = (uint32_t)digits[e];
    if (t != 0) acc[e] += t >= 0x10000u || (t >= 0x100u && (t & 0xffu)) ? NAN : t >= 0x100u ? -INFINITY : INFINITY;
  }
}

// Sequence b as its arrays say, then: the entries that count, its queries, and the entries before theirs (less than 0: the first own
// ones are not there).  A kernel asks for the former before anything else and uses them behind its own loads of q.
struct PagedCounts { int32_t len, fresh; };
__device__ __forceinline__ PagedCounts paged_counts(const PagedAttnArgs& a, int b) { return PagedCounts{a.seq_len[b], a.n_new ? a.n_new[b] : a.T}; }
__device__ __forceinline__ void paged_sequence(const PagedAttnArgs& a, const PagedCounts& counts, int& n, int& m, int& past) {
  n = __builtin_amdgcn_readfirstlane(counts.len);
  n = n < 0 ? 0 : n > a.S_max ? a.S_max : n;
  m = __builtin_amdgcn_readfirstlane(counts.fresh);
  m = m < 0 ? 0 : m > a.T ? a.T : m;
  past = n - m;
}

// Which stream, split and row group a workgroup takes.  The workgroups of a stream's row groups read the same entries: they are given
// numbers that are equal modulo 8, one die's, in turn.
__device__ __forceinline__ bool paged_unit(const PagedAttnArgs& a, int& row_group, int& hk, int& split, int& b) {
  int unit = blockIdx.x;
  row_group = 0;
  if (a.row_groups > 1) {
    const int y = blockIdx.x >> 3;
    row_group = y % a.row_groups;
    unit = (y / a.row_groups) * 8 + (blockIdx.x & 7);
    if (unit >= a.units) return false;
  }
  hk = unit % a.pool.H_kv;
  split = unit / a.pool.H_kv % a.n_splits;
  b = unit / a.pool.H_kv / a.n_splits;
  return true;
}

// Row `row` of stream (b, hk): its row of out.
__device__ __forceinline__ int64_t paged_row(const PagedAttnArgs& a, int b, int hk, int row) {
  const int t = row / a.group;
  return ((int64_t)b * a.T + t) * a.H + hk * a.group + (row - t * a.group);
}
// Four elements of a row's result: to out, or with its reference and sum to the workspace.
template <typename T, int DP>
__device__ __forceinline__ void paged_emit(const PagedAttnArgs& a, int64_t to, int split, int d, const float (&x)[4], float top, float sum) {
  if (a.n_splits == 1) {
    if (d < a.pool.d_h) store_result4<T>((T*)a.out + to * a.pool.d_h, d, a.pool.d_h, a.out_pieces, x);
    return;
  }
  const int64_t piece = to * a.n_splits + split;
  *reinterpret_cast<float4_t*>(a.ws + piece * DP + d) = float4_t{x[0], x[1], x[2], x[3]};
  if (d == 0) {
    float* st = a.ws + (int64_t)a.Bt * a.T * a.H * a.n_splits * DP + piece * 2;
    st[0] = top;
    st[1] = sum;
  }
}
// Where the 16 entries from `entry` on of a sequence of n lie, in the page that the table gives; < 0: nowhere (behind the last, or a page
// outside the pool, which `bad` remembers).
__device__ __forceinline__ int64_t paged_place(const PagedAttnArgs& a, int page, int hk, int entry, int n, bool& bad) {
  page = __builtin_amdgcn_readfirstlane(page);
  const bool used = entry < n, inside = page >= 0 && page < a.pool.n_pages;
  bad = bad || (used && !inside);
  const int64_t row = (((int64_t)page * a.pool.H_kv + hk) << a.pool.page_shift) + (entry & ((1 << a.pool.page_shift) - 1));
  return used && inside ? row * a.pool.row_bytes : -1;
}
__device__ __forceinline__ void paged_say(const PagedAttnArgs& a, bool bad, int lane) {
  if (bad && a.status && lane == 0) atomicOr(a.status, (int)PHOTON_STATUS_BAD_PAGE);
}

// What of an element x of q is left behind a part's 8 bits, for the next one.  Never 0 where entries may be infinite: 0 times infinity is NaN,
// and x times it is not.  2^-30 of x is added, below the digits that parts hold of x, so that only what would be 0 changes.
template <typename KV> __device__ __forceinline__ float rest_of_query(float part, float x) {
  const float rest = part - high_part(part);
  return sizeof(KV) == 2 ? fmaf(x, 0x1p-30f, rest) : rest;
}

// R tiles of 16 rows as a wave holds them: operands of the score products, and what each row sees.
template <typename KV, typename T, int NB, int R> struct PagedRows {
  using Y = PagedTypes<KV, T, NB>;
  uint32_t w[R][Y::Q_WORDS];
  int limit[R];                                // entries below are seen (without a tree); set by look(), as the next
  uint64_t bits[R];                            // own entries that are seen (with one)

  // Rows `first` .. of a stream; those behind its last are given that one's values.
  __device__ __forceinline__ void load(const PagedAttnArgs& a, int b, int hk, int first, int c, int g) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = min(first + r * 16 + c, a.T * a.group - 1), t = row / a.group, h = hk * a.group + (row - t * a.group);
      const T* from = (const T*)a.q + ((int64_t)b * a.T + t) * a.q_stride + (int64_t)h * a.pool.d_h;
      if constexpr (Y::F32) {
#pragma unroll
        for (int f = 0; f < 2 * NB; ++f) {
          float x[4];
          load_query4<T>(from, operand_element<KV, NB>(f, g), a.pool.d_h, a.q_pieces, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[r][4 * f + e] = __float_as_uint(x[e]);
        }
      } else {
#pragma unroll
        for (int f = 0; f < NB; ++f)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x[4];
            load_query4<T>(from, operand_element<KV, NB>(f, g) + 4 * half, a.pool.d_h, a.q_pieces, x);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              float u = x[e], v = x[e + 1];
#pragma unroll
              for (int part = 0; part < Y::Q_PARTS; ++part) {
                w[r][(part * NB + f) * 4 + half * 2 + e / 2] = high_halves(u, v);
                u = rest_of_query<KV>(u, x[e]);
                v = rest_of_query<KV>(v, x[e + 1]);
              }
            }
          }
      }
    }
  }
  __device__ __forceinline__ void look(const PagedAttnArgs& a, int b, int m, int past, int first, int rows, int c) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int t = min(first + r * 16 + c, rows - 1) / a.group;
      limit[r] = past + t + 1;
      bits[r] = 0;
      if (a.tree) bits[r] = a.tree[(int64_t)b * a.T + t] & (m == 64 ? ~0ull : (1ull << m) - 1);
    }
  }
  __device__ __forceinline__ bool visible(const PagedAttnArgs& a, int r, int entry, int past) const {
    if (!a.tree) return entry < limit[r];
    return entry < past || ((bits[r] >> ((unsigned)(entry - past) & 63u)) & 1u) != 0;
  }
  // Which of the lane's entries (4 g .. + 3 of the N tiles of 16 from base on) row tile r sees: bits.
  template <int N> __device__ __forceinline__ uint32_t seen(const PagedAttnArgs& a, int r, int base, int g, int n, int past, const bool (&there)[N]) const {
    uint32_t s = 0;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      const int entry = base + (i / 4) * 16 + 4 * g + i % 4;
      if (entry < n && there[i / 4] && visible(a, r, entry, past)) s |= 1u << i;
    }
    return s;
  }
  __device__ __forceinline__ bf16x8_t operand(int r, int part, int f) const {
    const uint32_t* x = w[r] + (part * NB + f) * 4;
    return as_bf16x8(uint4_t{x[0], x[1], x[2], x[3]});
  }
};

// Products are used behind a branch.  Where this compiler (clang 22 of ROCm 7.2) keeps their sums in accumulation registers, it reads them
// (v_accvgpr_read) without the distance that a matrix instruction's result needs on the path that skips the branch's body: entries 4 g + 3
// of a step were read too early.  The distance, 19 instructions for the longest product here, is kept by hand: results pass through this
// before anything reads them.
template <int R, int N> __device__ __forceinline__ void settle(f32x4_t (&d)[R][N]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(d[r][i]));            // volatile: these stay before the distance,
  asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(d[r][i]));            // and these behind it
}

// Weights of a lane's scores d of its rows: p = 2^(d scale - top).  Whether one exceeds the reference too far is told by the sums, so
// that an ordinary step has no comparisons; then references rise to ABOVE over the rows' maxima, and what was summed shrinks.  The product with
// the scale is rounded, as the reference was: fused with the subtraction it would keep digits that the reference lost, which are an
// exponent of their own once scores pass 2^24.  Where it passes FLT_MAX, or no score was seen before, sums are infinite or NaN; then,
// and with care, scores are halved as references are (scaling by 2 rounds nothing, so that weights are the same bits in either form).
// CAREFUL: 0 where `seen` has no bit.
template <bool CAREFUL, int R, int N, int TILES>
__device__ __forceinline__ void paged_weights(const f32x4_t (&d)[R][N], float half_scale, const uint32_t (&seen)[R], float (&top)[R], float (&sum)[R],
                                              f32x4_t (&acc)[R][TILES], float (&p)[R][4 * N]) {
  float s[R];
  const float scale = 2.f * half_scale;
  auto weigh = [&](auto halved) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float whole = rounded_product(top[r], 2.f);          // may be infinite: fused with the subtraction it would not be
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) {
        const float x = d[r][i / 4][i % 4];
        p[r][i] = decltype(halved)::value ? 2.f * (rounded_product(x, half_scale) - top[r]) : rounded_product(x, scale) - whole;
      }
      if constexpr (CAREFUL) {
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) p[r][i] = (seen[r] >> i) & 1u ? p[r][i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) p[r][i] = fast_exp2(p[r][i]);
      float part[N];
#pragma unroll
      for (int i = 0; i < N; ++i) part[i] = (p[r][4 * i] + p[r][4 * i + 1]) + (p[r][4 * i + 2] + p[r][4 * i + 3]);
      s[r] = part[0] + part[1];
      if constexpr (N == 4) s[r] += part[2] + part[3];
    }
  };
  weigh(std::bool_constant<CAREFUL>{});
  bool above = !(s[0] <= PAGED_RAISE);
  if constexpr (R == 2) above = above || !(s[1] <= PAGED_RAISE);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(above) != 0, 0)) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float highest = PAGED_LOWEST;
#pragma unroll
      for (int i = 0; i < 4 * N; ++i)
        if (!CAREFUL || ((seen[r] >> i) & 1u)) highest = fmaxf(highest, rounded_product(d[r][i / 4][i % 4], half_scale));
      const float higher = fmaxf(top[r], over_row(highest, [](float x, float y) { return fmaxf(x, y); }) + PAGED_ABOVE);
      const float shrink = fast_exp2(2.f * (top[r] - higher));
      top[r] = higher;
      sum[r] *= shrink;
#pragma unroll
      for (int j = 0; j < TILES; ++j) acc[r][j] *= shrink;
    }
    weigh(std::true_type{});
  }
#pragma unroll
  for (int r = 0; r < R; ++r) sum[r] += s[r];
}

// Whether one of a lane's sums is infinite or NaN.
template <int R, int TILES> __device__ __forceinline__ bool any_unbounded(const f32x4_t (&acc)[R][TILES]) {
  f32x4_t x = acc[0][0] * 0.f;                                               // four chains, not one of them all
#pragma unroll
  for (int i = 1; i < R * TILES; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(acc[i / TILES][i % TILES][e], 0.f, x[e]);
  const float y = (x[0] + x[1]) + (x[2] + x[3]);
  return y != y;
}

// Elements of a wave's rows that are infinite or NaN: infinite, or NaN, as the V that the row sees in the steps `step`, `step` + `by`, ... before
// `end` are, whatever their weights were; left as they are where none of those is (weights are NaN, sums too large).  Every element of V is
// looked at once more, which nothing else waits for.  element(j, i): which of a head's acc[.][j][i % 4] of lane group i / 4 is.
template <typename KV, typename Rows, int R, int TILES, typename Element>
__device__ __forceinline__ void restore_unbounded(const PagedAttnArgs& a, const Rows& q, f32x4_t (&acc)[R][TILES], const int32_t* table, int hk, int n,
                                                  int past, int step, int end, int by, int c, int g, Element element) {
  uint32_t found[R][TILES] = {};                                             // three bits an element: infinity, -infinity, NaN
#pragma unroll 1
  for (; step < end; step += by) {
    int64_t at[2];
    bool there[2], bad = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int entry = step * PAGED_STEP + 16 * i;
      at[i] = paged_place(a, table[min(entry, n - 1) >> a.pool.page_shift], hk, entry, n, bad);
      there[i] = at[i] >= 0;
    }
    uint4_t sees[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sees[r] = seen_operand(q.template seen<2>(a, r, step * PAGED_STEP, g, n, past, there));
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
      float code[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint8_t* from = a.pool.v + (at[i / 4] < 0 ? 0 : at[i / 4]) + (4 * g + i % 4) * a.pool.row_bytes;
        const float x = to_f32<KV>(reinterpret_cast<const KV*>(from)[element(j, c)]);
        code[i] = step * PAGED_STEP + (i / 4) * 16 + 4 * g + i % 4 < n && there[i / 4] ? unbounded_code(x) : 0.f;
      }
      const uint4_t codes = {high_halves(code[0], code[1]), high_halves(code[2], code[3]), high_halves(code[4], code[5]), high_halves(code[6], code[7])};
      f32x4_t digits[R][1];
#pragma unroll
      for (int r = 0; r < R; ++r)
        digits[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(codes), as_bf16x8(sees[r]), f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      settle(digits);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t t = (uint32_t)digits[r][0][e];
          found[r][j] |= ((t & 0xffu ? 1u : 0u) | (t & 0xff00u ? 2u : 0u) | (t >> 16 ? 4u : 0u)) << (3 * e);
        }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t t = (found[r][j] >> (3 * e)) & 7u;
        if (t != 0 && !(fabsf(acc[r][j][e]) <= FLT_MAX)) acc[r][j][e] = t == 1 ? INFINITY : t == 2 ? -INFINITY : NAN;
      }
}

// o = the sum of y w over the pairs that `each` hands on, where y is a mean of what was seen: an infinite one stays infinite however small
// its weight is.  Ordinary sums pay for one comparison.
template <typename Each> __device__ __forceinline__ void weighted_sum(float (&o)[4], Each each) {
  each([&](const float4_t& y, float w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], w, o[e]);
  });
  if (__builtin_expect(!(fabsf(fmaf(o[0], 0.f, fmaf(o[1], 0.f, fmaf(o[2], 0.f, o[3] * 0.f)))) <= 0.f), 0)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = 0.f;
    each([&](const float4_t& y, float w) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fabsf(y[e]) <= FLT_MAX ? fmaf(y[e], w, o[e]) : o[e] + y[e];
    });
  }
}

// R row tiles a wave, RW waves side by side over rows; the KW waves of the same rows deal the steps among themselves.  Fewer waves lose even
// where streams are many (256 x 16 ragged streams of up to 2048 entries of 64 fp32-row bf16 pages: 206 us, 215 with two waves, 231 with one).
// Two waves a SIMD are asked for wherever their registers suffice: left to itself, the compiler moves sums to accumulation registers and back
// and then fits one (13 nodes over E4M3 pages, 1024 streams of up to 1000 entries: 21.3 us, now 17.6; 512 rows over fp32 pages, 256 streams of
// 4096: 1439 us, now 1306).  Two tiles of 128 elements with fp32 rows or pages spill 130 registers and more at two waves (512 rows, 32
// streams of 2000: 84 us, 54 at one).
constexpr bool paged_two_waves(int d_p, int tiles, bool f32) { return !(d_p == 128 && tiles == 2 && f32); }
// Waves a SIMD that are asked for.  One tile of 32 fp32 elements takes 97 registers if it may, one more than five waves have (3480 streams of
// up to 7 entries: 17.4 us, 16.0 with five).
template <typename KV, typename T, int NB, int R> constexpr int paged_least_waves() {
  return sizeof(KV) == 4 && NB == 1 && R == 1 ? 5 : paged_two_waves(32 * NB, R, sizeof(KV) == 4 || sizeof(T) == 4) ? 2 : 1;
}

template <typename KV, typename T, int NB, int R, int RW>
__global__ __launch_bounds__(PAGED_WAVES * 64, (paged_least_waves<KV, T, NB, R>())) void paged_attn_kernel(PagedAttnArgs a) {
  using Y = PagedTypes<KV, T, NB>;
  constexpr int DP = Y::DP, TILES = Y::TILES, KW = PAGED_WAVES / RW, PITCH = DP + 4;
  __shared__ __align__(16) float results[PAGED_WAVES * 16 * PITCH];
  __shared__ float stats[PAGED_WAVES][16][2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int kw = wave % KW, rw = wave / KW;

  int row_group, hk, split, b;
  if (!paged_unit(a, row_group, hk, split, b)) return;
  // What is needed first is asked for at once: lengths, q, and (where a wave's first step does not depend on lengths) its pages.
  const PagedCounts counts = paged_counts(a, b);
  const int32_t* table = a.pool.table + (int64_t)b * a.pool.max_pages;
  struct Pages { int32_t page[2]; };                                         // of a step's tiles; behind `most` entries: the last one's
  auto pages = [&](int step, int most) {
    Pages p;
#pragma unroll
    for (int i = 0; i < 2; ++i) p.page[i] = table[min(step * PAGED_STEP + 16 * i, most - 1) >> a.pool.page_shift];
    return p;
  };
  Pages ahead = pages(kw, a.S_max);
  __builtin_amdgcn_sched_barrier(0);
  const int group_first = row_group * (RW * R * 16), first = group_first + rw * (R * 16);
  PagedRows<KV, T, NB, R> q;
  q.load(a, b, hk, first, c, g);
  __builtin_amdgcn_sched_barrier(0);
  int n, m, past;
  paged_sequence(a, counts, n, m, past);
  const int rows = m * a.group;
  if (group_first >= rows) return;
  const int group_last = min(group_first + RW * R * 16, rows) - 1;
  const int hi = a.tree ? n : min(n, past + group_last / a.group + 1);                     // entries that a row of the workgroup sees
  const int steps = hi <= 0 ? 0 : (hi + PAGED_STEP - 1) / PAGED_STEP;
  const int s0 = (int)((int64_t)steps * split / a.n_splits), s1 = (int)((int64_t)steps * (split + 1) / a.n_splits);
  const int all_see = a.tree ? past : past + min(first, rows - 1) / a.group + 1;           // entries that every row of the wave sees

  float top[R], sum[R];
  f32x4_t acc[R][TILES];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = PAGED_LOWEST;
    sum[r] = 0.f;
#pragma unroll
    for (int j = 0; j < TILES; ++j) acc[r][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  bool bad = false;
  auto places = [&](const Pages& p, int step, int64_t (&at)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i] = paged_place(a, p.page[i], hk, step * PAGED_STEP + 16 * i, n, bad);
  };
  const int k_lane = c * a.pool.row_bytes, v_lane = 4 * g * a.pool.row_bytes + c * Y::V_BYTES;
  uint32_t kx[2][Y::K_WORDS], vx[8][Y::V_WORDS];
  // From nowhere: the pool's first entries, in bounds, not used.
  auto load_k = [&](const int64_t (&at)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) load_keys<KV, NB>(a.pool.k + (at[i] < 0 ? 0 : at[i]) + k_lane, g, kx[i]);
  };
  auto load_v = [&](const int64_t (&at)[2]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) load_words<Y::V_BYTES>(a.pool.v + (at[i / 4] < 0 ? 0 : at[i / 4]) + v_lane + (i % 4) * a.pool.row_bytes, vx[i]);
  };

  const bool has_rows = first < rows;
  int step = s0 + kw;
  int64_t at[2] = {-1, -1};
  if (has_rows && step < s1) {
    if (s0 > 0) ahead = pages(step, n);
    places(ahead, step, at);
    load_k(at);
    load_v(at);
    ahead = pages(min(step + KW, steps - 1), n);                             // requested a step before they are needed
  }
  // One step; the next one's entries are requested as soon as their registers are free.  CAREFUL: a row may not see every entry of it.
  auto take = [&](auto careful) {
    constexpr bool CAREFUL = decltype(careful)::value;
    const bool there[2] = {at[0] >= 0, at[1] >= 0};
    const int base = step * PAGED_STEP, next = step + KW;
    int64_t next_at[2] = {-1, -1};
    if (next < s1) {
      places(ahead, next, next_at);
      ahead = pages(min(next + KW, steps - 1), n);
    }
    f32x4_t d[R][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < R; ++r) d[r][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (Y::F32) {
#pragma unroll
        for (int f = 0; f < 8 * NB; ++f)
#pragma unroll
          for (int r = 0; r < R; ++r)
            d[r][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kx[i][f]), __uint_as_float(q.w[r][f]), d[r][i], 0, 0, 0);
      } else {
#pragma unroll
        for (int f = 0; f < NB; ++f) {
          const bf16x8_t key = key_operand<KV>(kx[i], f);
#pragma unroll
          for (int part = Y::Q_PARTS - 1; part >= 0; --part)
#pragma unroll
            for (int r = 0; r < R; ++r) d[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q.operand(r, part, f), d[r][i], 0, 0, 0);
        }
      }
    }
    settle(d);
    if (next < s1) load_k(next_at);

    float s[R][8];
    uint32_t seen[R] = {};
    if constexpr (CAREFUL) {
#pragma unroll
      for (int r = 0; r < R; ++r) seen[r] = q.template seen<2>(a, r, base, g, n, past, there);
    }
    paged_weights<CAREFUL, R, 2, TILES>(d, a.half_scale, seen, top, sum, acc, s);
    bool some = false;                                                      // an infinity or NaN that some row sees
    if constexpr (CAREFUL) {
      // Entries that no row sees may hold anything: zeros.
      bool unbounded = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool used = base + (i / 4) * 16 + 4 * g + i % 4 < n && there[i / 4];
#pragma unroll
        for (int w = 0; w < Y::V_WORDS; ++w) {
          vx[i][w] = used ? vx[i][w] : 0u;
          unbounded = unbounded || without_unbounded<KV>(vx[i][w]) != vx[i][w];
        }
      }
      some = (m > 1 || a.tree) && __builtin_amdgcn_ballot_w64(unbounded) != 0;   // a node need not see itself
    }
    if constexpr (Y::F32 && CAREFUL) {
      if (some) {
#pragma unroll
        for (int j = 0; j < TILES; ++j) {
#pragma unroll
          for (int r = 0; r < R; ++r) {
            f32x4_t digits = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 8; ++i)
              digits = __builtin_amdgcn_mfma_f32_16x16x4f32(unbounded_code(__uint_as_float(vx[i][j])), (seen[r] >> i) & 1u ? 1.f : 0.f, digits, 0, 0, 0);
            add_unbounded(acc[r][j], digits);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) vx[i][j] = without_unbounded<KV>(vx[i][j]);
        }
      }
    }
    if constexpr (Y::F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < TILES; ++j)
#pragma unroll
          for (int r = 0; r < R; ++r)
            acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vx[i][j]), s[r][i], acc[r][j], 0, 0, 0);
    } else {
      bf16x8_t p[R][Y::P_PARTS];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        uint32_t w[Y::P_PARTS][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = s[r][2 * i], y = s[r][2 * i + 1];
#pragma unroll
          for (int part = 0; part + 1 < Y::P_PARTS; ++part) {
            w[part][i] = high_halves(x, y);
            x -= high_part(x);
            y -= high_part(y);
          }
          w[Y::P_PARTS - 1][i] = pack_bf16x2(x, y);
        }
#pragma unroll
        for (int part = 0; part < Y::P_PARTS; ++part) p[r][part] = as_bf16x8(uint4_t{w[part][0], w[part][1], w[part][2], w[part][3]});
      }
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        uint4_t value = value_operand<KV, Y::V_WORDS>(vx, j);
        if constexpr (CAREFUL) {
          if (some) {
#pragma unroll
            for (int r = 0; r < R; ++r)
              add_unbounded(acc[r][j], __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(unbounded_codes(value)), as_bf16x8(seen_operand(seen[r])),
                                                                               f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0));
#pragma unroll
            for (int i = 0; i < 4; ++i) value[i] = without_unbounded<bf16_t>(value[i]);
          }
        }
#pragma unroll
        for (int part = Y::P_PARTS - 1; part >= 0; --part)
#pragma unroll
          for (int r = 0; r < R; ++r) acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(value), p[r][part], acc[r][j], 0, 0, 0);
      }
    }
    if (next < s1) load_v(next_at);
    at[0] = next_at[0];
    at[1] = next_at[1];
    step = next;
  };
  // Steps that every row sees whole come first; from the first other one on, all are taken with care.  Code of both
  // in one loop would cost the ordinary steps their registers.
#pragma unroll 1
  while (has_rows && step < s1 && (step + 1) * PAGED_STEP <= all_see && at[0] >= 0 && at[1] >= 0) take(std::false_type{});
  q.look(a, b, m, past, first, rows, c);
#pragma unroll 1
  while (has_rows && step < s1) take(std::true_type{});
  settle(acc);
  if constexpr (sizeof(KV) > 1) {                                            // E4M3 has no infinities
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(any_unbounded(acc)) != 0, 0) && has_rows)
      restore_unbounded<KV>(a, q, acc, table, hk, n, past, s0 + kw, s1, KW, c, g, [](int j, int i) { return 2 * NB * i + j; });
  }
  paged_say(a, bad, lane);

  // Results: lane (c, g) holds elements 8 NB g .. + 8 NB - 1 of its rows.  Each wave divides by its sum, and waves are put together as
  // weighted means: no sum of values leaves the range that a wave's own is in.
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float l = over_row(sum[r], [](float x, float y) { return x + y; });
    const float mean = l == 0.f ? 0.f : 1.f / l;
    const int row = first + r * 16 + c;
    if (r > 0) __syncthreads();
    if (row < rows) {
#pragma unroll
      for (int x = 0; x < 8 * NB; x += 4) {
        float4_t o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = acc[r][(x + e) % TILES][(x + e) / TILES] * mean;
        *reinterpret_cast<float4_t*>(results + (wave * 16 + c) * PITCH + 8 * NB * g + x) = o;
      }
      if (g == 0) { stats[wave][c][0] = top[r]; stats[wave][c][1] = l; }
    }
    __syncthreads();
    for (int x = tid; x < RW * 16 * (DP / 4); x += PAGED_WAVES * 64) {
      const int d = x % (DP / 4) * 4, i = x / (DP / 4) % 16, of = x / (DP / 4) / 16;     // of: which of the waves side by side
      const int to = group_first + of * (R * 16) + r * 16 + i;
      if (to >= rows) continue;
      float w_top = PAGED_LOWEST, w_sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f}, weight[KW];
#pragma unroll
      for (int w = 0; w < KW; ++w) w_top = fmaxf(w_top, stats[of * KW + w][i][0]);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        weight[w] = stats[of * KW + w][i][1] * fast_exp2(2.f * (stats[of * KW + w][i][0] - w_top));
        w_sum += weight[w];
      }
      const float inverse = w_sum == 0.f ? 0.f : 1.f / w_sum;
      weighted_sum(o, [&](auto add) {
#pragma unroll
        for (int w = 0; w < KW; ++w) add(*reinterpret_cast<const float4_t*>(results + ((of * KW + w) * 16 + i) * PITCH + d), weight[w] * inverse);
      });
      paged_emit<T, DP>(a, paged_row(a, b, hk, to), split, d, o, w_top, w_sum);
    }
  }
}

// The splits' results of a row.  DP / 4 lanes hold a row's elements; with many splits a workgroup's SIDE groups of lanes take every
// SIDE-th one, and their results are put together in order (16 streams of 512 entries in 64 splits: 12 us in all, 24 with one group).
// References and sums of all splits are read by every lane in either case.
template <typename T, int NB, int SIDE> __global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int DP = 32 * NB, LANES = DP / 4, ROWS = 256 / (LANES * SIDE);
  __shared__ __align__(16) float part[SIDE > 1 ? 256 * 4 : 4];
  const int lane = threadIdx.x % LANES, side = threadIdx.x / LANES % SIDE, d = lane * 4;
  const int64_t to = (int64_t)blockIdx.x * ROWS + threadIdx.x / (LANES * SIDE);
  const int64_t token = to / a.H;
  const int b = (int)(token / a.T), t = (int)(token - (int64_t)b * a.T);
  if (to >= (int64_t)a.Bt * a.T * a.H || t >= (a.n_new ? a.n_new[b] : a.T)) return;    // with SIDE > 1 ROWS is 1: the whole workgroup's
  const float* values = a.ws + to * a.n_splits * DP + d;
  const float2_native* stats = reinterpret_cast<const float2_native*>(a.ws + (int64_t)a.Bt * a.T * a.H * a.n_splits * DP) + to * a.n_splits;
  float top = PAGED_LOWEST, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < a.n_splits; ++s) top = fmaxf(top, stats[s].x);
#pragma unroll 8
  for (int s = 0; s < a.n_splits; ++s) sum += stats[s].y * fast_exp2(2.f * (stats[s].x - top));
  const float inverse = sum == 0.f ? 0.f : 1.f / sum;
  weighted_sum(o, [&](auto add) {
#pragma unroll 4
    for (int s = side; s < a.n_splits; s += SIDE)
      add(*reinterpret_cast<const float4_t*>(values + (int64_t)s * DP), stats[s].y * fast_exp2(2.f * (stats[s].x - top)) * inverse);
  });
  if constexpr (SIDE > 1) {
    *reinterpret_cast<float4_t*>(part + threadIdx.x * 4) = float4_t{o[0], o[1], o[2], o[3]};
    __syncthreads();
    if (side != 0) return;
#pragma unroll
    for (int s = 1; s < SIDE; ++s) {
      const float4_t y = *reinterpret_cast<const float4_t*>(part + (s * LANES + lane) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += y[e];
    }
  }
  if (d < a.pool.d_h) store_result4<T>((T*)a.out + to * a.pool.d_h, d, a.pool.d_h, a.out_pieces, o);
}

template <typename KV, typename T, int NB, int R, int RW> int32_t paged_launch(const PagedAttnArgs& a, hipStream_t st) {
  const unsigned grid = a.row_groups > 1 ? (unsigned)((a.units + 7) / 8 * 8) * (unsigned)a.row_groups : (unsigned)a.units;
  PHOTON_LAUNCH(KC_COARSE_ATTN, st, (paged_attn_kernel<KV, T, NB, R, RW>), dim3(grid), dim3(PAGED_WAVES * 64), 0, st, a);
  return check_launch("paged_attn_kernel");
}
template <typename KV, typename T, int NB> int32_t paged_launch_rows(const PagedAttnArgs& a, const PagedTile& tile, hipStream_t st) {
  if (tile.tiles == 1) return paged_launch<KV, T, NB, 1, 1>(a, st);
  if (tile.waves == 1) return paged_launch<KV, T, NB, 2, 1>(a, st);
  return paged_launch<KV, T, NB, 2, 2>(a, st);
}
template <typename KV> int32_t paged_launch_types(const PagedAttnArgs& a, const PagedTile& tile, bool f32_rows, hipStream_t st) {
  const int nb = kv_row_elems(a.pool.d_h) / 32;
  if (f32_rows) return nb == 1 ? paged_launch_rows<KV, float, 1>(a, tile, st) : nb == 2 ? paged_launch_rows<KV, float, 2>(a, tile, st) : paged_launch_rows<KV, float, 4>(a, tile, st);
  return nb == 1 ? paged_launch_rows<KV, bf16_t, 1>(a, tile, st) : nb == 2 ? paged_launch_rows<KV, bf16_t, 2>(a, tile, st) : paged_launch_rows<KV, bf16_t, 4>(a, tile, st);
}

}  // namespace photon
