// Paged K/V cache: rows appended with the rotary encoding on the way, entries moved within a sequence.
//
// Both are copies: bytes bound them.  An append reads k, v and q once and writes the entries and q_out once; a row's heads are
// consecutive in memory, an entry's are head_bytes apart, so that every head of an entry is a run of whole 64- or 128-byte lines.
// Measured: four prompts of 8192 rows (805 MB) 153 us, 5.3 TB/s where a copy reaches 4.9; 64 ragged prompts into E4M3 pages (167 MB) 34.4 us,
// 4.9 TB/s; one entry of four sequences 7.5 us and 256 sequences' (10 MB) 8.1 us, which are the call's and a launch's.
#include <math.h>

#include "photon_device.h"
#include "photon_paged.h"

namespace photon {

int32_t paged_pools(const char* who, const photon_paged_cache* c, int32_t Bt, int32_t T, PagedPools* out) {
  PHOTON_REQUIRE(c != nullptr, PHOTON_ERR_INVALID_ARG, "%s: cache is null", who);
  PHOTON_REQUIRE(c->kv_dt == PHOTON_F32 || c->kv_dt == PHOTON_BF16 || c->kv_dt == PHOTON_FP8_E4M3, PHOTON_ERR_UNSUPPORTED,
                 "%s: pages are fp32, bf16 or E4M3, not dtype %d", who, (int)c->kv_dt);
  PHOTON_REQUIRE(Bt >= 0 && T >= 0 && c->H_kv > 0 && c->n_pages > 0 && c->max_pages > 0, PHOTON_ERR_INVALID_ARG,
                 "%s: Bt=%d T=%d H_kv=%d n_pages=%d max_pages=%d invalid", who, Bt, T, c->H_kv, c->n_pages, c->max_pages);
  PHOTON_REQUIRE(c->d_h >= 1 && c->d_h <= 128, PHOTON_ERR_UNSUPPORTED, "%s: d_h=%d not in [1, 128]", who, c->d_h);
  PHOTON_REQUIRE(c->page_size >= PAGED_LEAST && c->page_size <= 256 && (c->page_size & (c->page_size - 1)) == 0, PHOTON_ERR_UNSUPPORTED,
                 "%s: page_size=%d is not 16, 32, 64, 128 or 256", who, c->page_size);
  PHOTON_REQUIRE((int64_t)c->max_pages * c->page_size <= PAGED_MOST, PHOTON_ERR_UNSUPPORTED, "%s: %d pages of %d entries a sequence exceed 2^31 - 256",
                 who, c->max_pages, c->page_size);
  PHOTON_REQUIRE(Bt <= 65535 && c->H_kv <= 65535, PHOTON_ERR_UNSUPPORTED, "%s: Bt=%d, H_kv=%d streams: at most 65535 each", who, Bt, c->H_kv);
  PagedPools& p = *out;
  p.k = (uint8_t*)c->k_pages;
  p.v = (uint8_t*)c->v_pages;
  p.table = c->page_table;
  p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.H_kv = c->H_kv; p.d_h = c->d_h;
  p.page_shift = __builtin_ctz(c->page_size);
  p.row_bytes = kv_row_elems(c->d_h) * (int)dtype_size(c->kv_dt);
  p.head_bytes = (int64_t)p.row_bytes * c->page_size;
  p.page_bytes = p.head_bytes * c->H_kv;
  if (Bt == 0 || T == 0) return PHOTON_OK;               // nothing is touched
  PHOTON_REQUIRE(p.k && p.v && aligned16(p.k) && aligned16(p.v), PHOTON_ERR_INVALID_ARG, "%s: the pools must be non-null, 16-byte aligned device pointers", who);
  PHOTON_REQUIRE(p.table != nullptr && element_aligned(p.table, 4), PHOTON_ERR_INVALID_ARG, "%s: page_table must be a non-null device pointer to int32", who);
  const uintptr_t a = reinterpret_cast<uintptr_t>(p.k), b = reinterpret_cast<uintptr_t>(p.v);
  PHOTON_REQUIRE((a < b ? b - a : a - b) / (uint64_t)p.page_bytes >= (uint64_t)p.n_pages, PHOTON_ERR_INVALID_ARG,
                 "%s: K and V need a pool each: these overlap", who);
  return PHOTON_OK;
}

namespace {

constexpr int MOST_PAIRS = 64;            // rotary pairs of a row
constexpr int ROPE_ROWS = 32;             // rows of a workgroup, at most

// frequency i in turns per position, as a fraction of 2^64: positions times it, modulo 2^64, are exact phases
struct RopeTable { uint64_t turns[MOST_PAIRS]; };

struct WriteArgs {
  PagedPools pool;
  const void *k, *v, *q;
  void* q_out;
  int64_t row_stride, q_stride, q_out_stride;
  const int32_t *start, *n_new, *position;
  int32_t* status;
  int32_t T, H, rows, half, rotate;       // rows: of a workgroup; half: elements from one member of a rotary pair to the other
  uint32_t by_half, by_pieces;            // ceil(2^32 / half), ceil(2^32 / (half / VEC)): see quotient()
};

// x / d by a multiplication, m = ceil(2^32 / d): exact where x d < 2^32 (x below 2^24 here, d up to 64).  A division is 20 instructions and more (128
// sequences of 31 rows, one row a workgroup, and the move: 19.7 us with divisions, 19.2; the four prompts 155, 152).
__device__ __forceinline__ int quotient(int x, int d, uint32_t m) { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }

// Two values as E4M3: saturated, and NaN stays NaN.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  const float a = lo != lo ? lo : fminf(fmaxf(lo, -448.f), 448.f), b = hi != hi ? hi : fminf(fmaxf(hi, -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

template <typename T, int VEC> __device__ __forceinline__ void load_piece(const T* p, float (&x)[VEC]) {
  // as one access: the launch chose VEC so that pieces are aligned to their size
  struct alignas(VEC * sizeof(T)) Raw { T e[VEC]; };
  const Raw r = *reinterpret_cast<const Raw*>(p);
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = to_f32<T>(r.e[e]);
}
template <typename T, int VEC> __device__ __forceinline__ void store_piece(T* p, const float (&x)[VEC]) {
  struct alignas(VEC * sizeof(T)) Raw { T e[VEC]; };
  Raw r;
  if constexpr (sizeof(T) == 2 && VEC > 1) {
#pragma unroll
    for (int e = 0; e < VEC; e += 2) reinterpret_cast<uint32_t*>(r.e)[e / 2] = pack_bf16x2(x[e], x[e + 1]);
  } else if constexpr (sizeof(T) == 1 && VEC > 1) {
#pragma unroll
    for (int e = 0; e < VEC; e += 2) reinterpret_cast<uint16_t*>(r.e)[e / 2] = (uint16_t)pack_e4m3x2(x[e], x[e + 1]);
  } else if constexpr (sizeof(T) == 1) {
    r.e[0] = T{(uint8_t)pack_e4m3x2(x[0], 0.f)};
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) r.e[e] = from_f32<T>(x[e]);
  }
  *reinterpret_cast<Raw*>(p) = r;
}

// A thread holds VEC rotary pairs of one head (elements i .. and i + half ..) and takes them through the rows of its workgroup, so
// that what it works on follows from its index once.  Heads: H of q (none without q), H_kv of K, H_kv of V.  Cosines and sines are
// made once per row and pair, in LDS: heads share them.  A phase is position * frequency in turns, in 64 bits of fixed point, where
// a product wraps as angles do: far positions lose nothing, and no arithmetic in double is needed.
template <typename T, typename KV, int VEC>
__global__ __launch_bounds__(256) void paged_write_kernel(WriteArgs a, RopeTable rope) {
  __shared__ float2_native angle[ROPE_ROWS][MOST_PAIRS];
  __shared__ int64_t place[ROPE_ROWS];                                       // byte offset of the entry of head 0; -1: none
  const int b = blockIdx.z, tid = threadIdx.x, t0 = blockIdx.x * a.rows;
  const int pieces = (int)((uint32_t)a.half / VEC), x = blockIdx.y * blockDim.x + tid;
  const int q_heads = a.q ? a.H : 0, H_kv = a.pool.H_kv, d_h = a.pool.d_h, heads = q_heads + 2 * H_kv;
  const int nth = quotient(x, pieces, a.by_pieces), head = min(nth, heads - 1), c = (x - nth * pieces) * VEC;         // threads behind the last head only help with the table
  const int kind = head < q_heads ? 0 : head < q_heads + H_kv ? 1 : 2;       // q, K, V
  const int h = kind == 0 ? head : kind == 1 ? head - q_heads : head - q_heads - H_kv;
  const int64_t stride = kind == 0 ? a.q_stride : a.row_stride;
  const T* from = (const T*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) + ((int64_t)b * a.T + t0) * stride + (int64_t)h * d_h + c;
  const bool pair = c + a.half < d_h;                                        // an odd head's last element has no partner
  constexpr int AT_ONCE = 4;                                                 // rows in flight
  float lo[AT_ONCE][VEC], hi[AT_ONCE][VEC];
  auto request = [&](int r0, int rows) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int r = min(r0 + u, rows - 1);
      load_piece<T, VEC>(from + r * stride, lo[u]);
      load_piece<T, VEC>(from + r * stride + (pair ? a.half : 0), hi[u]);
    }
  };
  // The first rows are on their way while places and angles are found out, and counts, too, where most workgroups will have rows (64
  // prompts of 1 .. 133 rows, in the larger workgroups of that time: 42 us, 53 with all of the padding's rows requested).
  const bool early = a.n_new == nullptr || a.T <= AT_ONCE;
  if (early) request(0, min(a.rows, a.T - t0));
  int m = a.n_new ? a.n_new[b] : a.T;
  m = m < 0 ? 0 : m > a.T ? a.T : m;
  const int rows = min(a.rows, m - t0);
  if (rows <= 0) return;
  if (!early) request(0, rows);
  const int start = a.start ? a.start[b] : 0;
  if (tid < rows) {
    const int64_t entry = (int64_t)start + t0 + tid;
    const int64_t at = entry >> a.pool.page_shift;
    int64_t to = -1;
    int bad = 0;
    if (entry < 0 || at >= a.pool.max_pages) bad = PHOTON_STATUS_CACHE_FULL;
    else {
      const int page = a.pool.table[(int64_t)b * a.pool.max_pages + at];
      if (page < 0 || page >= a.pool.n_pages) bad = PHOTON_STATUS_BAD_PAGE;
      else to = page * a.pool.page_bytes + (entry & ((1 << a.pool.page_shift) - 1)) * a.pool.row_bytes;
    }
    place[tid] = to;
    if (bad && a.status && blockIdx.y == 0) atomicOr(a.status, bad);
  }
  if (a.rotate) {
    for (int y = tid; y < rows * a.half; y += blockDim.x) {
      const int r = quotient(y, a.half, a.by_half), i = y - r * a.half;
      // the low word of the position and its sign: start + t may pass 2^31 (q_out is written all the same), and stays below 2^32
      const int given = a.position ? a.position[(int64_t)b * a.T + t0 + r] : start;
      const uint32_t low = (uint32_t)given + (a.position ? 0u : (uint32_t)(t0 + r)), frequency = (uint32_t)rope.turns[i];
      const bool negative = given < 0 && (int)low < 0;
      // the nearest quarter turn is taken off before the phase becomes a float: what is left is at most an eighth, rounded to 2^-28 turns
      const uint32_t turn = __umulhi(low, frequency) + low * (uint32_t)(rope.turns[i] >> 32) - (negative ? frequency : 0u), quarter = (turn + 0x20000000u) >> 30;
      float sn, cs;
      sincospif((float)(int32_t)(turn - (quarter << 30)) * 0x1p-31f, &sn, &cs);
      const float co = quarter & 1 ? -sn : cs, si = quarter & 1 ? cs : sn;
      angle[r][i] = quarter & 2 ? float2_native{-co, -si} : float2_native{co, si};
    }
  }
  __syncthreads();
  if (nth >= heads) return;
  T* q_to = (T*)a.q_out + ((int64_t)b * a.T + t0) * a.q_out_stride + (int64_t)h * d_h + c;
  uint8_t* pool = (kind == 1 ? a.pool.k : a.pool.v) + h * a.pool.head_bytes;
  const int d_p = a.pool.row_bytes / (int)sizeof(KV);
  for (int r0 = 0; r0 < rows; r0 += AT_ONCE) {
    if (r0 > 0) request(r0, rows);
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int r = r0 + u;
      if (r >= rows) break;
      if (kind != 2 && a.rotate) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2_native cs = angle[r][c + e];
          rotate_pair(lo[u][e], hi[u][e], cs.x, cs.y, lo[u][e], hi[u][e]);
        }
      }
      if (kind == 0) {
        store_piece<T, VEC>(q_to + r * a.q_out_stride, lo[u]);
        if (pair) store_piece<T, VEC>(q_to + r * a.q_out_stride + a.half, hi[u]);
      } else if (place[r] >= 0) {
        KV* to = (KV*)(pool + place[r]);
        store_piece<KV, VEC>(to + c, lo[u]);
        if (pair) store_piece<KV, VEC>(to + c + a.half, hi[u]);
        // the columns behind a head's elements: VEC divides 32 and, where it is not 1, d_h
        const float zero[VEC] = {};
        for (int e = d_h + c; e < d_p; e += pieces * VEC) store_piece<KV, VEC>(to + e, zero);
      }
    }
  }
}

struct MoveArgs {
  PagedPools pool;
  const int32_t *start, *from, *n;
  int32_t* status;
  int32_t T;
};

// One workgroup per stream and pool: the entries, 16 bytes a thread and step, into LDS, then to their places.  All of them are read
// before one is written: the barrier waits for the reads, whose values are in LDS by then.
__global__ __launch_bounds__(256) void paged_move_kernel(MoveArgs a) {
  extern __shared__ __align__(16) uint4_t kept[];                            // [T][row in 16 bytes]
  __shared__ int64_t src[PAGED_MOST_TREE], dst[PAGED_MOST_TREE];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  uint8_t* pool = blockIdx.z ? a.pool.v : a.pool.k;
  int n = a.n ? a.n[b] : a.T;
  n = n < 0 ? 0 : n > a.T ? a.T : n;
  if (n == 0) return;
  if (tid < n) {
    const int64_t start = a.start ? a.start[b] : 0;
    const int64_t entry[2] = {start + a.from[(int64_t)b * a.T + tid], start + tid};
    int64_t at[2];
    int bad = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t place = entry[i] >> a.pool.page_shift;
      at[i] = -1;
      if (entry[i] < 0 || place >= a.pool.max_pages) { bad |= PHOTON_STATUS_CACHE_FULL; continue; }
      const int page = a.pool.table[(int64_t)b * a.pool.max_pages + place];
      if (page < 0 || page >= a.pool.n_pages) { bad |= PHOTON_STATUS_BAD_PAGE; continue; }
      at[i] = page * a.pool.page_bytes + h * a.pool.head_bytes + (entry[i] & ((1 << a.pool.page_shift) - 1)) * a.pool.row_bytes;
    }
    if (bad || at[0] == at[1]) at[0] = -1;                                   // nothing to do
    src[tid] = at[0];
    dst[tid] = at[1];
    if (bad && a.status && h == 0 && blockIdx.z == 0) atomicOr(a.status, bad);
  }
  __syncthreads();
  const int row = a.pool.row_bytes / 16, all = n * row;
  for (int x = tid; x < all; x += blockDim.x) {
    const int i = x / row, c = (x - i * row) * 16;
    if (src[i] < 0) continue;
    kept[x] = load16(pool + src[i] + c);
  }
  __syncthreads();
  for (int x = tid; x < all; x += blockDim.x) {
    const int i = x / row, c = (x - i * row) * 16;
    if (src[i] < 0) continue;
    *reinterpret_cast<uint4_t*>(pool + dst[i] + c) = kept[x];
  }
}

template <typename T, typename KV, int VEC> void launch_write(WriteArgs a, const RopeTable& rope, int Bt, hipStream_t st) {
  // Threads of a row: a multiple of 64, in as few idle ones as workgroups of at most 256 leave.
  const int64_t items = (int64_t)((a.q ? a.H : 0) + 2 * a.pool.H_kv) * (a.half / VEC);
  const int64_t groups = (items + 255) / 256;
  const int threads = (int)(((items + groups - 1) / groups + 63) / 64 * 64);
  // Rows of a workgroup: as many as share a table of angles well, but fewer while workgroups are few: several rounds of them even out what
  // their rows take (two sets of inputs in turn; at least 2048, 4096, 8192 workgroups: four prompts of 8192 rows 172, 164, 155 us; 64 ragged
  // prompts into 8 bits 38, 33, 31; four of 4096 fp32 rows 134, 131, 125; rows and move of 128 trees 21 all).
  int rows = ROPE_ROWS;
  while (rows > 1 && ((int64_t)Bt * ((a.T + rows - 1) / rows) * groups < 8192 || rows / 2 >= a.T)) rows /= 2;
  a.rows = rows;
  const uint32_t pieces = (uint32_t)a.half / VEC;
  a.by_half = (uint32_t)((0x100000000ull + a.half - 1) / a.half);          // 0 for 1, not used
  a.by_pieces = (uint32_t)((0x100000000ull + pieces - 1) / pieces);
  PHOTON_LAUNCH(KC_PAGED_CACHE, st, (paged_write_kernel<T, KV, VEC>), dim3((unsigned)((a.T + rows - 1) / rows), (unsigned)groups, Bt), dim3(threads), 0, st, a, rope);
}
template <typename T, typename KV> void launch_write_vec(const WriteArgs& a, const RopeTable& rope, int vec, int Bt, hipStream_t st) {
  switch (vec) {
    case 4: return launch_write<T, KV, 4>(a, rope, Bt, st);
    case 2: return launch_write<T, KV, 2>(a, rope, Bt, st);
    default: return launch_write<T, KV, 1>(a, rope, Bt, st);
  }
}
template <typename T> void launch_write_t(const WriteArgs& a, const RopeTable& rope, int vec, photon_dtype kv_dt, int Bt, hipStream_t st) {
  switch (kv_dt) {
    case PHOTON_F32: return launch_write_vec<T, float>(a, rope, vec, Bt, st);
    case PHOTON_BF16: return launch_write_vec<T, bf16_t>(a, rope, vec, Bt, st);
    default: return launch_write_vec<T, fp8_t>(a, rope, vec, Bt, st);
  }
}

}  // namespace
}  // namespace photon

// ------------------------------------------------------------------ C ABI

using namespace photon;

extern "C" int32_t photon_paged_cache_write(const photon_paged_cache* cache, const void* k, const void* v, int64_t row_stride, const void* q,
                                            int64_t q_stride, void* q_out, int64_t q_out_stride, const int32_t* start, const int32_t* n_new,
                                            const int32_t* position, int32_t* status, int32_t Bt, int32_t T, int32_t H, float rope_theta,
                                            photon_dtype dt, void* stream) {
  clear_error();
  WriteArgs a;
  PHOTON_TRY(paged_pools(__func__, cache, Bt, T, &a.pool));
  const int d_h = cache->d_h, H_kv = cache->H_kv;
  PHOTON_REQUIRE(valid_dtype(dt), PHOTON_ERR_UNSUPPORTED, "%s: rows are fp32 or bf16, not dtype %d", __func__, (int)dt);
  PHOTON_REQUIRE(rope_theta == 0.f || (rope_theta >= 1.f && isfinite(rope_theta)), PHOTON_ERR_INVALID_ARG, "%s: rope_theta=%g is neither 0 nor at least 1",
                 __func__, (double)rope_theta);
  PHOTON_REQUIRE(rope_theta == 0.f || d_h % 2 == 0, PHOTON_ERR_UNSUPPORTED, "%s: d_h=%d is odd: no rotary pairs", __func__, d_h);
  PHOTON_REQUIRE((q != nullptr) == (q_out != nullptr), PHOTON_ERR_INVALID_ARG, "%s: q and q_out go together", __func__);
  PHOTON_REQUIRE(q == nullptr || (H > 0 && H <= 65535), PHOTON_ERR_INVALID_ARG, "%s: H=%d invalid", __func__, H);
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const size_t esz = dtype_size(dt);
  PHOTON_REQUIRE(k && v && element_aligned(k, esz) && element_aligned(v, esz), PHOTON_ERR_INVALID_ARG, "%s: k and v must be non-null device pointers to whole elements", __func__);
  PHOTON_REQUIRE(row_stride >= (int64_t)H_kv * d_h, PHOTON_ERR_INVALID_ARG, "%s: row_stride=%lld is less than a row of %d heads of %d", __func__,
                 (long long)row_stride, H_kv, d_h);
  if (q) {
    PHOTON_REQUIRE(element_aligned(q, esz) && element_aligned(q_out, esz), PHOTON_ERR_INVALID_ARG, "%s: q and q_out must point to whole elements", __func__);
    PHOTON_REQUIRE(q_stride >= (int64_t)H * d_h && q_out_stride >= (int64_t)H * d_h, PHOTON_ERR_INVALID_ARG,
                   "%s: q_stride=%lld, q_out_stride=%lld: a row of %d heads of %d is longer", __func__, (long long)q_stride, (long long)q_out_stride, H, d_h);
    PHOTON_REQUIRE(q != q_out || q_stride == q_out_stride, PHOTON_ERR_INVALID_ARG, "%s: q rotated in place keeps its stride", __func__);
  }
  a.k = k; a.v = v; a.q = q; a.q_out = q_out;
  a.row_stride = row_stride; a.q_stride = q_stride; a.q_out_stride = q_out_stride;
  a.start = start; a.n_new = n_new; a.position = position; a.status = status;
  a.T = T; a.H = q ? H : 0; a.rows = 1; a.half = (d_h + 1) / 2; a.rotate = rope_theta != 0.f;
  RopeTable rope;
  if (a.rotate) {
    // theta^(-2i/d_h) / (2 pi) as fractions of 2^128, one a product of the one before with theta^(-2/d_h) as a fraction of 2^64, which is
    // within 2^-64: the last of 64 within 63 / (2 pi) 2^-64, which is 2^-28 turns at positions of up to 2^32.
    const long double ratio = powl((long double)rope_theta, -2.0L / d_h);
    const uint64_t r = ratio < 1.0L ? (uint64_t)ldexpl(ratio, 64) : 0;       // 0: all alike
    uint64_t high = 0x28be60db9391054aull, low = 0x7f09d5f47d4d3770ull;      // 1 / (2 pi)
    for (int i = 0; i < a.half; ++i) {
      rope.turns[i] = high + (low >> 63);
      if (r == 0) continue;
      const unsigned __int128 next = (unsigned __int128)high * r + (uint64_t)(((unsigned __int128)low * r) >> 64);
      high = (uint64_t)(next >> 64);
      low = (uint64_t)next;
    }
  }
  // Elements of a piece: they divide half a head (so pairs are whole pieces) and are aligned in every row that a piece is read from.  Four at
  // most: eight leave registers for three or four waves a SIMD instead of eight (the four prompts 182 us, 172 with four; fp32 rows and pages
  // 174, 161).
  const auto whole = [&](int vec) {
    const size_t n = vec * esz;
    const auto rows = [&](const void* p, int64_t stride) { return element_aligned(p, n) && stride * esz % n == 0; };
    return d_h % 2 == 0 && a.half % vec == 0 && rows(k, row_stride) && rows(v, row_stride) && (!q || (rows(q, q_stride) && rows(q_out, q_out_stride)));
  };
  const int vec = whole(4) ? 4 : whole(2) ? 2 : 1;
  PHOTON_REQUIRE((int64_t)T * 256 <= 0xffffffffll && ((int64_t)(a.H + 2 * H_kv) * a.half / 256 + 1) <= 65535, PHOTON_ERR_UNSUPPORTED,
                 "%s: T=%d rows of %d heads are too many", __func__, T, a.H + 2 * H_kv);
  (dt == PHOTON_F32 ? launch_write_t<float> : launch_write_t<bf16_t>)(a, rope, vec, cache->kv_dt, Bt, (hipStream_t)stream);
  return check_launch("paged_write_kernel");
}

extern "C" int32_t photon_paged_cache_move(const photon_paged_cache* cache, const int32_t* start, const int32_t* from, const int32_t* n, int32_t* status,
                                           int32_t Bt, int32_t T, void* stream) {
  clear_error();
  MoveArgs a;
  PHOTON_TRY(paged_pools(__func__, cache, Bt, T, &a.pool));
  PHOTON_REQUIRE(T <= PAGED_MOST_TREE, PHOTON_ERR_UNSUPPORTED, "%s: T=%d entries: at most %d move at once", __func__, T, PAGED_MOST_TREE);
  if (Bt == 0 || T == 0) return PHOTON_OK;
  PHOTON_REQUIRE(from != nullptr, PHOTON_ERR_INVALID_ARG, "%s: from is null", __func__);
  a.start = start; a.from = from; a.n = n; a.status = status; a.T = T;
  PHOTON_LAUNCH(KC_PAGED_CACHE, (hipStream_t)stream, paged_move_kernel, dim3(cache->H_kv, Bt, 2), dim3(256), (unsigned)T * a.pool.row_bytes, (hipStream_t)stream, a);
  return check_launch("paged_move_kernel");
}
