// K/V cache in 4 bits (MXFP4): rows quantised as they are written, read back, and attended over.
//
// Format (OCP microscaling): a block of 32 elements has a scale X = 2^e, e = floor(log2 max|x|) - 2 (at least -127), stored as
// e + 127, and every element is the E2M1 value nearest to x / X (ties to the even code, magnitudes above 6 become 6).  X is a
// power of two, so x / X is exact and the result is unique; a stored value has 2 significant bits and is exact in bf16.
#include "photon_mxfp4.h"

#include "photon_attn.h"
#include "photon_device.h"
#include "photon_host.h"

namespace photon {

// ------------------------------------------------------------------ rows in and out
//
// A wave takes the positions of one tile of one stream, 8 positions x 64 elements at a time ("a pass"): lane 8 r + x holds 8
// consecutive elements of position r, 4 neighbouring lanes a block.  K words go out as they are.  V words hold 8 positions of
// one element: the 8 lanes of equal x exchange nibbles (an 8 x 8 transposition in three steps).
//   d_p = 128: a pass takes half of the elements; d_p = 32: lanes x >= 4 take the next 8 positions.

constexpr int MX_WAVES = 4;      // waves (tiles) of a workgroup

template <int NB> struct MxPass {
  static constexpr int PER_TILE = NB * 4;                  // 64 positions x 32 NB elements in passes of 512
  int kk, dim;                                             // position in the tile and first of the lane's 8 elements
  __device__ __forceinline__ MxPass(int pass, int lane) {
    const int r = lane >> 3, x = lane & 7;
    if (NB == 1) { kk = pass * 16 + (x >> 2) * 8 + r; dim = (x & 3) * 8; }
    else if (NB == 2) { kk = pass * 8 + r; dim = x * 8; }
    else { kk = (pass >> 1) * 8 + r; dim = (pass & 1) * 64 + x * 8; }
  }
};

// 8 x 8 nibbles among the lanes r = 0..7 of equal x: word r, nibble j <-> word j, nibble r.  One step swaps halves at distance S.
template <int S> __device__ __forceinline__ uint32_t mx_swap_nibbles(uint32_t w, int lane) {
  constexpr uint32_t low = S == 4 ? 0x0000ffffu : S == 2 ? 0x00ff00ffu : 0x0f0f0f0fu;
  const uint32_t other = __shfl_xor(w, 8 * S);
  return (lane >> 3) & S ? (w & ~low) | ((other >> (4 * S)) & low) : (w & low) | ((other << (4 * S)) & ~low);
}
__device__ __forceinline__ uint32_t mx_transpose8(uint32_t w, int lane) {
  return mx_swap_nibbles<1>(mx_swap_nibbles<2>(mx_swap_nibbles<4>(w, lane), lane), lane);
}

// The 8 elements of a row from `dim` on, zeros past d_h.  VEC elements per access: 8 or 4 where pointer, stride and d_h are whole
// multiples of it, else 1.
template <typename T, int VEC> __device__ __forceinline__ void mx_load8(const T* row, int dim, int d_h, float (&v)[8]) {
  if constexpr (VEC == 8) {
    if (dim < d_h) {
      if constexpr (sizeof(T) == 2) Vec16<bf16_t>::load(reinterpret_cast<const bf16_t*>(row + dim), v);
      else {
        const float4_t a = *reinterpret_cast<const float4_t*>(row + dim), b = *reinterpret_cast<const float4_t*>(row + dim + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else if constexpr (VEC == 4) {
#pragma unroll
    for (int u = 0; u < 8; u += 4) {
      if (dim + u < d_h) {
        if constexpr (sizeof(T) == 2) {
          const uint2 r = *reinterpret_cast<const uint2*>(row + dim + u);
          v[u] = bf16_lo(r.x); v[u + 1] = bf16_hi(r.x); v[u + 2] = bf16_lo(r.y); v[u + 3] = bf16_hi(r.y);
        } else {
          const float4_t a = *reinterpret_cast<const float4_t*>(row + dim + u);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[u + i] = a[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[u + i] = 0.f;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = dim + i < d_h ? to_f32<T>(row[dim + i]) : 0.f;
  }
}
template <typename T, int VEC> __device__ __forceinline__ void mx_store8(T* row, int dim, int d_h, const float (&v)[8]) {
  if constexpr (VEC == 8) {
    if (dim < d_h) {
      if constexpr (sizeof(T) == 2) Vec16<bf16_t>::store(reinterpret_cast<bf16_t*>(row + dim), v);
      else {
        *reinterpret_cast<float4_t*>(row + dim) = float4_t{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<float4_t*>(row + dim + 4) = float4_t{v[4], v[5], v[6], v[7]};
      }
    }
  } else if constexpr (VEC == 4) {
#pragma unroll
    for (int u = 0; u < 8; u += 4) {
      if (dim + u < d_h) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(row + dim + u) = make_uint2(pack_bf16x2(v[u], v[u + 1]), pack_bf16x2(v[u + 2], v[u + 3]));
        else *reinterpret_cast<float4_t*>(row + dim + u) = float4_t{v[u], v[u + 1], v[u + 2], v[u + 3]};
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (dim + i < d_h) row[dim + i] = from_f32<T>(v[i]);
  }
}

// A block of 32 elements in 4 neighbouring lanes -> the lane's 8 codes and the block's scale byte.  The largest magnitude is taken
// of the bits, so that a NaN or an infinity is the largest: such a block gets the scale byte 255 and reads back as NaN.
__device__ __forceinline__ uint32_t mx_quantise8(const float (&v)[8], uint32_t& scale_byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) { const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu; top = m > top ? m : top; }
  uint32_t o = __builtin_amdgcn_update_dpp(0, top, DPP_XOR1, 0xf, 0xf, false);
  top = o > top ? o : top;
  o = __builtin_amdgcn_update_dpp(0, top, DPP_XOR2, 0xf, 0xf, false);
  top = o > top ? o : top;
  const uint32_t e = top >> 23;
  scale_byte = e == 255u ? 255u : (e > 2u ? e : 2u) - 2u;
  // The conversion takes x / X with X = 2^(exponent field - 127) of its scale operand, a field of 0 included.
  const float scale = __uint_as_float((e == 255u ? 127u : scale_byte) << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  return w;
}

// 8 codes under one scale byte -> values.
__device__ __forceinline__ void mx_values8(uint32_t w, uint32_t scale_byte, float (&v)[8]) {
  const float scale = __uint_as_float(scale_byte << 23);
  const f32x2_native a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32x2_native c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
  if (scale_byte > (uint32_t)MX_LAST_SCALE)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7fc00000u);
}

struct MxRows {                  // a stretch of rows and the positions it belongs to
  const int32_t *start, *n_new;  // [Bt] or NULL: position of row 0 (0), rows in use (T)
  int64_t row_stride;            // elements from a row to the next
  int64_t S_max;
  int T, H_kv, d_h, slots;       // slots: tiles that T rows can touch
  int64_t streams;
};

// Wave's share: stream, its tile and the positions [lo, hi) of the tile that rows in use belong to.
struct MxShare {
  int64_t stream, tile, row0;    // row0: row of position 0 of the tile
  int b, h, lo, hi;
};
__device__ __forceinline__ bool mx_share(const MxRows& a, int wave, MxShare& s, bool& outside) {
  const int64_t unit = (int64_t)blockIdx.x * MX_WAVES + wave;
  s.stream = unit / a.slots;
  outside = false;
  if (s.stream >= a.streams) return false;
  const int slot = (int)(unit - s.stream * a.slots);
  s.b = (int)(s.stream / a.H_kv);
  s.h = (int)(s.stream - (int64_t)s.b * a.H_kv);
  int64_t n = a.n_new ? a.n_new[s.b] : a.T;
  n = n < 0 ? 0 : n > a.T ? a.T : n;
  const int64_t first = a.start ? a.start[s.b] : 0;
  const int64_t begin = first < 0 ? 0 : first, end = first + n < a.S_max ? first + n : a.S_max;
  outside = n > 0 && (first < 0 || first + n > a.S_max);
  s.tile = (begin >> 6) + slot;
  const int64_t base = s.tile * MX_TILE;
  if (base >= end) return false;
  s.lo = begin > base ? (int)(begin - base) : 0;
  s.hi = end - base < MX_TILE ? (int)(end - base) : MX_TILE;
  s.row0 = (int64_t)s.b * a.T + base - first;
  return s.lo < s.hi;
}

template <typename T, int NB, int VEC>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_write_kernel(const T* __restrict__ k, const T* __restrict__ v, uint8_t* __restrict__ kc,
                                                                    uint8_t* __restrict__ vc, int32_t* __restrict__ status, MxRows a) {
  const int lane = threadIdx.x & 63;
  MxShare s;
  bool outside;
  const bool any = mx_share(a, threadIdx.x >> 6, s, outside);
  if (outside && status != nullptr && lane == 0) atomicOr(status, (int)PHOTON_STATUS_CACHE_FULL);
  if (!any) return;
  const int64_t tiles = (a.S_max + MX_TILE - 1) / MX_TILE;
  const int64_t at = (s.stream * tiles + s.tile) * mx_tile_bytes(NB * MX_BLOCK);
  kc += at;
  vc += at;
  constexpr int STEP = NB == 1 ? 16 : 8, SPLIT = NB == 4 ? 2 : 1;    // positions of a pass, passes per position
  const int first = s.lo / STEP * SPLIT, last = (s.hi + STEP - 1) / STEP * SPLIT;
  for (int pass = first; pass < last; ++pass) {
    const MxPass<NB> p(pass, lane);
    const bool ok = p.kk >= s.lo && p.kk < s.hi;
    float kv[8], vv[8];
    if (ok) {
      const int64_t row = (s.row0 + p.kk) * a.row_stride + (int64_t)s.h * a.d_h;
      mx_load8<T, VEC>(k + row, p.dim, a.d_h, kv);
      mx_load8<T, VEC>(v + row, p.dim, a.d_h, vv);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) kv[i] = vv[i] = 0.f;
    }
    uint32_t ks, vs;
    const uint32_t kw = mx_quantise8(kv, ks), vw = mx_transpose8(mx_quantise8(vv, vs), lane);
    const int block = p.dim >> 5;
    if (ok) {
      *reinterpret_cast<uint32_t*>(kc + mx_k_chunk<NB>(p.kk, block) + ((p.dim >> 3) & 3) * 4) = kw;
      if ((lane & 3) == 0) {
        kc[mx_k_scale<NB>(p.kk, block)] = (uint8_t)ks;
        vc[mx_v_scale<NB>(p.kk, block)] = (uint8_t)vs;
      }
    }
    // the lane's V word: element dim + r, the 8 positions around p.kk; those outside [lo, hi) keep what they held
    const int group = p.kk & ~7, r = lane >> 3;
    const int from = s.lo - group < 0 ? 0 : s.lo - group, to = s.hi - group > 8 ? 8 : s.hi - group;
    if (from < to) {
      uint32_t* word = reinterpret_cast<uint32_t*>(vc + mx_v_word<NB>(group, p.dim + r));
      const uint32_t mask = (to == 8 ? 0xffffffffu : (1u << (4 * to)) - 1u) & ~((1u << (4 * from)) - 1u);
      *word = mask == 0xffffffffu ? vw : (*word & ~mask) | (vw & mask);
    }
  }
}

template <typename T, int NB, int VEC>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_read_kernel(const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc, T* __restrict__ k,
                                                                   T* __restrict__ v, MxRows a) {
  const int lane = threadIdx.x & 63;
  MxShare s;
  bool outside;
  const bool any = mx_share(a, threadIdx.x >> 6, s, outside);
  if (!any) return;
  const int64_t tiles = (a.S_max + MX_TILE - 1) / MX_TILE;
  const int64_t at = (s.stream * tiles + s.tile) * mx_tile_bytes(NB * MX_BLOCK);
  kc += at;
  vc += at;
  constexpr int STEP = NB == 1 ? 16 : 8, SPLIT = NB == 4 ? 2 : 1;
  const int first = s.lo / STEP * SPLIT, last = (s.hi + STEP - 1) / STEP * SPLIT;
  for (int pass = first; pass < last; ++pass) {
    const MxPass<NB> p(pass, lane);
    const int block = p.dim >> 5;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(kc + mx_k_chunk<NB>(p.kk, block) + ((p.dim >> 3) & 3) * 4);
    const uint32_t vw = *reinterpret_cast<const uint32_t*>(vc + mx_v_word<NB>(p.kk & ~7, p.dim + (lane >> 3)));
    const uint32_t ks = kc[mx_k_scale<NB>(p.kk, block)], vs = vc[mx_v_scale<NB>(p.kk, block)];
    float kv[8], vv[8];
    mx_values8(kw, ks, kv);
    mx_values8(mx_transpose8(vw, lane), vs, vv);
    if (p.kk >= s.lo && p.kk < s.hi) {
      const int64_t row = (s.row0 + p.kk) * a.row_stride + (int64_t)s.h * a.d_h;
      mx_store8<T, VEC>(k + row, p.dim, a.d_h, kv);
      mx_store8<T, VEC>(v + row, p.dim, a.d_h, vv);
    }
  }
}

// ------------------------------------------------------------------ attention

// One wave per query: a lane per position for the scores, a lane per element for the values.
template <typename T, int NB>
__global__ __launch_bounds__(64) void mxfp4_attn_kernel(const T* __restrict__ q, int64_t q_stride, const uint8_t* __restrict__ kc,
                                                        const uint8_t* __restrict__ vc, const int32_t* __restrict__ seq_len,
                                                        const int32_t* __restrict__ n_new, T* __restrict__ out, int Tq, int H, int H_kv, int d_h,
                                                        int64_t S_max, float scale_log2e) {
  constexpr int DP = NB * MX_BLOCK;
  const int lane = threadIdx.x;
  const int h = blockIdx.x % H, t = blockIdx.x / H % Tq, b = blockIdx.x / H / Tq;
  int m = n_new ? n_new[b] : Tq;
  m = m < 0 ? 0 : m > Tq ? Tq : m;
  if (t >= m) return;
  int64_t n = seq_len[b];
  n = n < 0 ? 0 : n > S_max ? S_max : n;
  n = n - m + t + 1;
  n = n < 0 ? 0 : n;
  __shared__ float qs[DP], pb[MX_TILE][NB];
  q += ((int64_t)b * Tq + t) * q_stride + (int64_t)h * d_h;
  for (int i = lane; i < DP; i += 64) qs[i] = i < d_h ? to_f32<T>(q[i]) * scale_log2e : 0.f;
  __syncthreads();
  const int64_t tiles = (S_max + MX_TILE - 1) / MX_TILE, stream = (int64_t)b * H_kv + h / (H / H_kv);
  float top = NEG_BIG, sum = 0.f, o[2] = {0.f, 0.f};
  for (int64_t base = 0; base < n; base += MX_TILE) {
    const uint8_t* kt = kc + (stream * tiles + base / MX_TILE) * mx_tile_bytes(DP);
    const uint8_t* vt = vc + (stream * tiles + base / MX_TILE) * mx_tile_bytes(DP);
    const bool seen = base + lane < n;
    float s = 0.f;
    for (int block = 0; block < NB; ++block) {
      const uint4_t c = load16(kt + mx_k_chunk<NB>(lane, block));
      const uint32_t byte = kt[mx_k_scale<NB>(lane, block)];
      for (int j = 0; j < 4; ++j) {
        float x[8];
        mx_values8(c[j], byte, x);
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], qs[block * 32 + j * 8 + e], s);
      }
    }
    s = seen ? s : NEG_BIG;
    float mx = s;
    for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    mx = fmaxf(mx, top);
    const float old = fast_exp2(top - mx), p = seen ? fast_exp2(s - mx) : 0.f;
    top = mx;
    sum = sum * old + wave_sum(p);
    o[0] *= old;
    o[1] *= old;
    for (int block = 0; block < NB; ++block) {
      const uint32_t byte = vt[mx_v_scale<NB>(lane, block)];
      float x[8];
      mx_values8(2u, byte, x);       // 1 under this scale
      pb[lane][block] = seen ? p * x[0] : 0.f;
    }
    __syncthreads();
    for (int u = 0; u < 2; ++u) {
      const int dim = lane + 64 * u;
      if (dim >= DP) continue;
      for (int kk = 0; kk < MX_TILE; kk += 8) {
        float x[8];
        mx_values8(*reinterpret_cast<const uint32_t*>(vt + mx_v_word<NB>(kk, dim)), 127u, x);
        for (int e = 0; e < 8; ++e) o[u] = fmaf(pb[kk + e][dim >> 5], x[e], o[u]);
      }
    }
    __syncthreads();
  }
  out += (((int64_t)b * Tq + t) * H + h) * d_h;
  for (int u = 0; u < 2; ++u)
    if (lane + 64 * u < d_h) out[lane + 64 * u] = from_f32<T>(n > 0 ? o[u] / sum : 0.f);
}

}  // namespace photon

// ------------------------------------------------------------------ C ABI

using namespace photon;

namespace {

// Shapes that every entry point shares.
int32_t check_shape(const char* who, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max, photon_dtype dt) {
  PHOTON_REQUIRE(valid_dtype(dt), PHOTON_ERR_UNSUPPORTED, "%s: rows are fp32 or bf16, not dtype %d", who, (int)dt);
  PHOTON_REQUIRE(Bt >= 0 && T >= 0 && H_kv > 0 && S_max > 0, PHOTON_ERR_INVALID_ARG, "%s: Bt=%d T=%d H_kv=%d S_max=%lld invalid", who, Bt, T,
                 H_kv, (long long)S_max);
  PHOTON_REQUIRE(d_h >= 1 && d_h <= 128, PHOTON_ERR_UNSUPPORTED, "%s: d_h=%d not in [1, 128]", who, d_h);
  PHOTON_REQUIRE(S_max <= 0x7fffffff, PHOTON_ERR_UNSUPPORTED, "%s: S_max=%lld exceeds what an int32 position counts", who, (long long)S_max);
  PHOTON_REQUIRE((int64_t)Bt * H_kv <= 0x7fffffff, PHOTON_ERR_UNSUPPORTED, "%s: Bt*H_kv=%lld streams", who, (long long)Bt * H_kv);
  return PHOTON_OK;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Elements per access of rows: what pointers, stride and head size are whole multiples of.
int row_vec(const void* a, const void* b, int64_t stride, int d_h, size_t esz) {
  for (int vec = 8; vec > 1; vec -= 4) {
    const size_t bytes = vec * esz < 16 ? vec * esz : 16;
    if (d_h % vec == 0 && stride * esz % bytes == 0 && aligned(a, bytes) && aligned(b, bytes)) return vec;
  }
  return 1;
}

int32_t rows_args(const char* who, const void* k, const void* v, const void* kc, const void* vc, int64_t row_stride, const MxRows& a, photon_dtype dt) {
  const size_t esz = dtype_size(dt);
  PHOTON_REQUIRE(k && v && aligned(k, esz) && aligned(v, esz), PHOTON_ERR_INVALID_ARG, "%s: k and v must be non-null device pointers to whole elements", who);
  PHOTON_REQUIRE(kc && vc && aligned16(kc) && aligned16(vc), PHOTON_ERR_INVALID_ARG, "%s: the caches must be non-null, 16-byte aligned device pointers", who);
  PHOTON_REQUIRE(row_stride >= (int64_t)a.H_kv * a.d_h, PHOTON_ERR_INVALID_ARG, "%s: row_stride=%lld is less than a row of %d heads of %d", who,
                 (long long)row_stride, a.H_kv, a.d_h);
  const int64_t groups = (a.streams * a.slots + MX_WAVES - 1) / MX_WAVES;
  PHOTON_REQUIRE(groups <= 0x7fffffff, PHOTON_ERR_UNSUPPORTED, "%s: %lld workgroups", who, (long long)groups);
  return PHOTON_OK;
}

MxRows mx_rows(const int32_t* start, const int32_t* n_new, int64_t row_stride, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max) {
  MxRows a;
  a.start = start; a.n_new = n_new; a.row_stride = row_stride; a.S_max = S_max;
  a.T = T; a.H_kv = H_kv; a.d_h = d_h; a.slots = (int)(((int64_t)T + 62) / 64 + 1); a.streams = (int64_t)Bt * H_kv;
  return a;
}

#define MX_ROWS_CASE(kernel, T, NB, VEC, ...)                                                                      \
  PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (kernel<T, NB, VEC>), dim3((unsigned)((a.streams * a.slots + MX_WAVES - 1) / MX_WAVES)), dim3(MX_WAVES * 64), 0, st, __VA_ARGS__)
#define MX_ROWS_VEC(kernel, T, NB, ...)                                                                            \
  do {                                                                                                             \
    if (vec == 8) MX_ROWS_CASE(kernel, T, NB, 8, __VA_ARGS__);                                                     \
    else if (vec == 4) MX_ROWS_CASE(kernel, T, NB, 4, __VA_ARGS__);                                                \
    else MX_ROWS_CASE(kernel, T, NB, 1, __VA_ARGS__);                                                              \
  } while (0)
#define MX_ROWS(kernel, T, ...)                                                                                    \
  do {                                                                                                             \
    if (d_p == 32) MX_ROWS_VEC(kernel, T, 1, __VA_ARGS__);                                                         \
    else if (d_p == 64) MX_ROWS_VEC(kernel, T, 2, __VA_ARGS__);                                                    \
    else MX_ROWS_VEC(kernel, T, 4, __VA_ARGS__);                                                                   \
  } while (0)

}  // namespace

extern "C" int32_t photon_mxfp4_tile_bytes(int32_t d_h) {
  const int d_p = photon_kv_row_elems(d_h);
  return d_p == 0 ? 0 : mx_tile_bytes(d_p);
}

extern "C" size_t photon_mxfp4_cache_bytes(int32_t Bt, int32_t H_kv, int32_t d_h, int64_t S_max) {
  if (Bt <= 0 || H_kv <= 0 || S_max <= 0) return 0;
  return (size_t)Bt * H_kv * (size_t)((S_max + MX_TILE - 1) / MX_TILE) * photon_mxfp4_tile_bytes(d_h);
}

extern "C" int32_t photon_mxfp4_cache_write(const void* k, const void* v, int64_t row_stride, void* k_cache, void* v_cache, const int32_t* start,
                                            const int32_t* n_new, int32_t* status, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max,
                                            photon_dtype dt, void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const MxRows a = mx_rows(start, n_new, row_stride, Bt, T, H_kv, d_h, S_max);
  PHOTON_TRY(rows_args(__func__, k, v, k_cache, v_cache, row_stride, a, dt));
  const int d_p = photon_kv_row_elems(d_h), vec = row_vec(k, v, row_stride, d_h, dtype_size(dt));
  hipStream_t st = (hipStream_t)stream;
  if (dt == PHOTON_F32) MX_ROWS(mxfp4_write_kernel, float, (const float*)k, (const float*)v, (uint8_t*)k_cache, (uint8_t*)v_cache, status, a);
  else MX_ROWS(mxfp4_write_kernel, bf16_t, (const bf16_t*)k, (const bf16_t*)v, (uint8_t*)k_cache, (uint8_t*)v_cache, status, a);
  return check_launch("mxfp4_write_kernel");
}

extern "C" int32_t photon_mxfp4_cache_read(const void* k_cache, const void* v_cache, const int32_t* start, const int32_t* n_rows, void* k, void* v,
                                           int64_t row_stride, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max, photon_dtype dt,
                                           void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const MxRows a = mx_rows(start, n_rows, row_stride, Bt, T, H_kv, d_h, S_max);
  PHOTON_TRY(rows_args(__func__, k, v, k_cache, v_cache, row_stride, a, dt));
  const int d_p = photon_kv_row_elems(d_h), vec = row_vec(k, v, row_stride, d_h, dtype_size(dt));
  hipStream_t st = (hipStream_t)stream;
  if (dt == PHOTON_F32) MX_ROWS(mxfp4_read_kernel, float, (const uint8_t*)k_cache, (const uint8_t*)v_cache, (float*)k, (float*)v, a);
  else MX_ROWS(mxfp4_read_kernel, bf16_t, (const uint8_t*)k_cache, (const uint8_t*)v_cache, (bf16_t*)k, (bf16_t*)v, a);
  return check_launch("mxfp4_read_kernel");
}

extern "C" size_t photon_mxfp4_decode_attn_workspace_bytes(int32_t Bt, int32_t T, int32_t H, int32_t d_h, int32_t n_splits) {
  if (Bt <= 0 || T <= 0 || H <= 0 || d_h <= 0 || d_h > 128 || n_splits <= 1) return 0;
  return (size_t)Bt * T * H * n_splits * (kv_row_elems(d_h) + 2) * sizeof(float);
}

extern "C" int32_t photon_mxfp4_decode_attn_auto_splits(int32_t Bt, int32_t T, int32_t H, int32_t H_kv, int64_t S_max) {
  return 1;
}

extern "C" int32_t photon_mxfp4_decode_attn(const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const int32_t* seq_len,
                                            const int32_t* n_new, void* out, int32_t Bt, int32_t T, int32_t H, int32_t H_kv, int32_t d_h,
                                            int64_t S_max, float scale, int32_t n_splits, void* workspace, size_t workspace_bytes, photon_dtype dt,
                                            void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  PHOTON_REQUIRE(H > 0 && H % H_kv == 0, PHOTON_ERR_INVALID_ARG, "%s: H=%d query heads do not share H_kv=%d evenly", __func__, H, H_kv);
  PHOTON_REQUIRE(n_splits >= 0 && n_splits <= 1024, PHOTON_ERR_INVALID_ARG, "%s: n_splits=%d out of [0, 1024]", __func__, n_splits);
  PHOTON_REQUIRE((int64_t)Bt * H <= 0x7fffffff && (int64_t)Bt * H * (T > 0 ? T : 1) <= 0x7fffffff, PHOTON_ERR_UNSUPPORTED,
                 "%s: Bt=%d T=%d H=%d are too many queries", __func__, Bt, T, H);
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const size_t esz = dtype_size(dt);
  PHOTON_REQUIRE(q && out && aligned(q, esz) && aligned(out, esz), PHOTON_ERR_INVALID_ARG, "%s: q and out must be non-null device pointers to whole elements", __func__);
  PHOTON_REQUIRE_PTR(k_cache);
  PHOTON_REQUIRE_PTR(v_cache);
  PHOTON_REQUIRE(seq_len != nullptr, PHOTON_ERR_INVALID_ARG, "%s: seq_len is null", __func__);
  PHOTON_REQUIRE(q_stride >= (int64_t)H * d_h, PHOTON_ERR_INVALID_ARG, "%s: q_stride=%lld is less than a row of %d heads of %d", __func__,
                 (long long)q_stride, H, d_h);
  if (n_splits == 0) n_splits = photon_mxfp4_decode_attn_auto_splits(Bt, T, H, H_kv, S_max);
  if (n_splits > 1) {
    const size_t need = photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, n_splits);
    PHOTON_REQUIRE(workspace != nullptr && aligned16(workspace) && workspace_bytes >= need, PHOTON_ERR_WORKSPACE,
                   "%s: n_splits=%d needs a 16-byte aligned workspace of %zu bytes (got %zu)", __func__, n_splits, need, workspace_bytes);
  }
  hipStream_t st = (hipStream_t)stream;
  const int d_p = photon_kv_row_elems(d_h);
#define MX_ATTN(T_, NB)                                                                                                    \
  PHOTON_LAUNCH(KC_COARSE_ATTN, st, (mxfp4_attn_kernel<T_, NB>), dim3((unsigned)(Bt * T * H)), dim3(64), 0, st, (const T_*)q, q_stride, \
                (const uint8_t*)k_cache, (const uint8_t*)v_cache, seq_len, n_new, (T_*)out, T, H, H_kv, d_h, S_max, scale * LOG2E)
#define MX_ATTN_NB(T_) do { if (d_p == 32) MX_ATTN(T_, 1); else if (d_p == 64) MX_ATTN(T_, 2); else MX_ATTN(T_, 4); } while (0)
  if (dt == PHOTON_F32) MX_ATTN_NB(float); else MX_ATTN_NB(bf16_t);
  return check_launch("mxfp4_attn_kernel");
}
