// K/V cache in 4 bits (MXFP4): rows quantised as they are written, read back, and attended over.
//
// Format (OCP microscaling): a block of 32 elements has a scale X = 2^e, e = floor(log2 max|x|) - 2 (at least -127), stored as
// e + 127, and every element is the E2M1 value nearest to x / X (ties to the even code, magnitudes above 6 become 6).  X is a
// power of two, so x / X is exact and the result is unique; a stored value has 2 significant bits and is exact in bf16.
#include "photon_mxfp4.h"

#include <type_traits>

#include "photon_attn.h"
#include "photon_device.h"
#include "photon_host.h"

namespace photon {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ rows in and out
//
// A wave takes 16 positions of one stream, 8 positions x 64 elements at a time ("a pass"), all loads first.  Lane 8 r + x works on
// position r.  Of bf16 rows it loads 8 consecutive elements at once.  Of others it loads 4 elements of the pass's block 0 and 4
// of its block 1, so that 8 lanes read a row's elements side by side (4 x 8192 fp32 rows of 32 x 64 elements: 111 us, 130 with 8
// consecutive elements a lane), and neighbours exchange 4 codes: then it holds 8 consecutive elements, too.  These go out as they are
// for K.  V words hold 8 positions of one element: the 8 lanes of equal x exchange nibbles (an 8 x 8 transposition in three steps).
//   d_p = 128: a pass takes half of the elements; d_p = 32: it takes 16 positions, blocks 0 and 1 being positions r and 8 + r.
// Neighbouring workgroups take neighbouring heads of the same positions (but see launch_rows), those of one die (blocks are dealt to
// the eight dies in turn) heads that lie side by side, since heads of 52 to 60 elements share lines (4 x 8192 bf16 rows of 32 x 60
// elements: written in 190 us and read back in 148 without, in 120 and 109 with).
// Measured for four prompts of 8192 rows of 32 x 64 elements (K and V, 1.2 GB of them in turn): fp32 written in 104 us = 5.8 TB/s
// (537 MB in, 71 MB out) and read back in 128 = 4.7, in turn with each other 114 and 120; bf16 in 71 us = 4.8 and 73 = 4.7.  Without
// its stores the write takes 97 us (fp32): memory is the bound, in both directions.

constexpr int MX_WAVES = 4;      // waves of a workgroup, at most: 64 positions
constexpr int MX_STEP = 16;      // positions of a wave

template <typename T, int NB, int VEC> struct MxPass {
  static constexpr bool SPLIT = sizeof(T) == 4 || VEC < 8;
  static constexpr int LOADS = SPLIT ? 2 : 1, N = 8 / LOADS;           // loads of a pass, elements of each
  // Whether any of the positions [lo, hi) is the pass's.
  static __device__ __forceinline__ bool live(int pass, int lo, int hi) {
    const int from = NB == 1 ? 0 : NB == 2 ? 8 * pass : 8 * (pass >> 1);
    return lo < from + (NB == 1 ? 16 : 8) && hi > from;
  }
  int kk, dim;                                                         // position among the wave's 16 and first element of the lane's word
  int load_kk[LOADS], load_dim[LOADS];                                 // the same of what it loads
  __device__ __forceinline__ MxPass(int pass, int lane) {
    const int r = lane >> 3, x = lane & 7;
    const int base_kk = (NB == 1 ? 0 : NB == 2 ? pass : pass >> 1) * 8 + r, base_dim = NB == 4 ? (pass & 1) * 64 : 0;
    const int block = SPLIT ? x & 1 : x >> 2, in = (SPLIT ? x >> 1 : x & 3) * 8;
    kk = base_kk + (NB == 1 ? block * 8 : 0);
    dim = base_dim + (NB == 1 ? 0 : block * 32) + in;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      load_kk[u] = SPLIT ? base_kk + (NB == 1 ? u * 8 : 0) : kk;
      load_dim[u] = SPLIT ? base_dim + (NB == 1 ? 0 : u * 32) + x * 4 : dim;
    }
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

// N elements of a row from `dim` on, as loaded: at once where pointer, stride and d_h are whole multiples of 4 (8) elements, else
// one by one (VEC = 1).  Loads are never skipped, so that all of them are in flight: past d_h the row's last elements are loaded.
template <typename T, int N, int VEC> struct MxRaw {
  static constexpr int WORDS = N * sizeof(T) / 4;
  uint32_t w[WORDS];
  // ONCE: nothing else will read these lines, so they are read past the caches
  template <bool ONCE> __device__ __forceinline__ void load(const T* row, int dim, int d_h) {
    if constexpr (VEC == 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const T x = row[dim + i < d_h ? dim + i : d_h - 1];
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x);
        else w[i / 2] = i % 2 ? w[i / 2] | (uint32_t)x << 16 : (uint32_t)x;
      }
    } else {
      const T* from = row + (dim < d_h ? dim : d_h - N);
      if constexpr (WORDS == 4) {
        const uint4_t r = ONCE ? load16_stream(from) : load16(from);
        w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
      } else {
        const uint64_t* at = reinterpret_cast<const uint64_t*>(from);
        const uint64_t r = ONCE ? __builtin_nontemporal_load(at) : *at;
        w[0] = (uint32_t)r; w[1] = (uint32_t)(r >> 32);
      }
    }
  }
  __device__ __forceinline__ void values(int dim, int d_h, float (&v)[N]) const {      // zeros past d_h
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = sizeof(T) == 4 ? __uint_as_float(w[i % WORDS]) : i % 2 ? bf16_hi(w[i / 2 % WORDS]) : bf16_lo(w[i / 2 % WORDS]);
      v[i] = dim + i < d_h ? x : 0.f;
    }
  }
};
template <typename T, int N, int VEC> __device__ __forceinline__ void mx_store(T* row, int dim, int d_h, const float (&v)[N]) {
  if constexpr (VEC == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (dim + i < d_h) row[dim + i] = from_f32<T>(v[i]);
  } else if (dim < d_h) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4_t*>(row + dim) = float4_t{v[0], v[1], v[2], v[3]};
    else if constexpr (N == 8) Vec16<bf16_t>::store(reinterpret_cast<bf16_t*>(row + dim), v);
    else *reinterpret_cast<uint2*>(row + dim) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

template <int CTRL> __device__ __forceinline__ uint32_t mx_dpp(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, false); }

// A block of 32 elements in 32 / N neighbouring lanes -> the lane's N codes and the block's scale byte.  The largest magnitude is
// taken of the bits, so that a NaN or an infinity is the largest: such a block gets the scale byte 255 and reads back as NaN.
template <int N> __device__ __forceinline__ uint32_t mx_quantise(const float (&v)[N], uint32_t& scale_byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) { const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu; top = m > top ? m : top; }
  uint32_t o = mx_dpp<DPP_XOR1>(top);
  top = o > top ? o : top;
  o = mx_dpp<DPP_XOR2>(top);
  top = o > top ? o : top;
  if constexpr (N == 4) {
    o = mx_dpp<DPP_HALF_MIRROR>(top);
    top = o > top ? o : top;
  }
  const uint32_t e = top >> 23;
  scale_byte = e == 255u ? 255u : (e > 2u ? e : 2u) - 2u;
  // The conversion takes x / X with X = 2^(exponent field - 127) of its scale operand, a field of 0 included.
  const float scale = __uint_as_float((e == 255u ? 127u : scale_byte) << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  if constexpr (N == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  }
  return w;
}

// What a pass loaded -> the lane's word and its block's scale byte.
template <typename P, typename R> __device__ __forceinline__ uint32_t mx_word(const P& p, const R (&raw)[P::LOADS], int lane, int d_h, uint32_t& scale_byte) {
  float v[P::N];
  raw[0].values(p.load_dim[0], d_h, v);
  const uint32_t w0 = mx_quantise(v, scale_byte);
  if constexpr (!P::SPLIT) return w0;
  else {
    uint32_t s1;
    raw[1].values(p.load_dim[1], d_h, v);
    const uint32_t w1 = mx_quantise(v, s1);
    const bool odd = lane & 1;
    const uint32_t other = mx_dpp<DPP_XOR1>(odd ? w0 : w1);
    scale_byte = odd ? s1 : scale_byte;
    return odd ? other | w1 << 16 : w0 | other << 16;
  }
}

// N codes under one scale byte -> values.
template <int N> __device__ __forceinline__ void mx_values(uint32_t w, uint32_t scale_byte, float (&v)[N]) {
  const float scale = __uint_as_float(scale_byte << 23);
  const f32x2_native a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
  if constexpr (N == 8) {
    const f32x2_native c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
  }
  if (scale_byte > (uint32_t)MX_LAST_SCALE)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __uint_as_float(0x7fc00000u);
}

// The lane's word and scale byte -> the codes and scales of what its row accesses hold: mx_word's exchange backwards.
template <typename P> __device__ __forceinline__ void mx_parts(uint32_t w, uint32_t scale_byte, int lane, uint32_t (&code)[P::LOADS], uint32_t (&scale)[P::LOADS]) {
  if constexpr (!P::SPLIT) { code[0] = w; scale[0] = scale_byte; }
  else {
    const bool odd = lane & 1;
    const uint32_t other = mx_dpp<DPP_XOR1>(odd ? w & 0xffffu : w >> 16), other_scale = mx_dpp<DPP_XOR1>(scale_byte);
    code[0] = odd ? other : w & 0xffffu;
    code[1] = odd ? w >> 16 : other;
    scale[0] = odd ? other_scale : scale_byte;
    scale[1] = odd ? scale_byte : other_scale;
  }
}

struct MxRows {                  // a stretch of rows and the positions it belongs to
  const int32_t *start, *n_new;  // [Bt] or NULL: position of row 0 (0), rows in use (T)
  int64_t row_stride;            // elements from a row to the next
  int64_t S_max;
  int T, H_kv, d_h, add;         // add: to start
  bool heads_first;              // neighbouring workgroups take neighbouring heads of the same positions, else the other way round
};

// A wave's share: a step of 16 positions, and those [lo, hi) of it that rows in use belong to.
struct MxShare {
  int64_t tile, row0;            // row0: the row of position 0 of the step
  int b, h, base, lo, hi;        // base: of the step in the tile
};
// false: nothing to do.  outside: rows of this sequence have no place in the cache.
__device__ __forceinline__ bool mx_share(const MxRows& a, MxShare& s, bool& outside) {
  const unsigned of = a.heads_first ? (unsigned)a.H_kv : gridDim.x / (unsigned)a.H_kv, major = blockIdx.x / of, minor = blockIdx.x - major * of;
  const unsigned group = a.heads_first ? major : minor;
  s.b = blockIdx.y;
  s.h = !a.heads_first ? major : a.H_kv % 8 == 0 ? minor % 8 * (a.H_kv / 8) + minor / 8 : minor;
  int64_t n = a.n_new ? a.n_new[s.b] : a.T;
  n = n < 0 ? 0 : n > a.T ? a.T : n;
  const int64_t first = (a.start ? (int64_t)a.start[s.b] : 0) + a.add;
  const int64_t begin = first < 0 ? 0 : first, end = first + n < a.S_max ? first + n : a.S_max;
  outside = n > 0 && (first < 0 || first + n > a.S_max);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);           // the same in the wave: what follows is scalar
  const int64_t at = (begin / MX_STEP + (int64_t)group * (blockDim.x >> 6) + wave) * MX_STEP;
  if (at >= end) return false;
  s.tile = at / MX_TILE;
  s.base = (int)(at % MX_TILE);
  s.lo = begin > at ? (int)(begin - at) : 0;
  s.hi = end - at < MX_STEP ? (int)(end - at) : MX_STEP;
  s.row0 = (int64_t)s.b * a.T + at - first;
  return true;
}

template <typename T, int NB, int VEC, bool ONCE>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_write_kernel(const T* __restrict__ k, const T* __restrict__ v, uint8_t* __restrict__ kc,
                                                                    uint8_t* __restrict__ vc, int32_t* __restrict__ status, MxRows a) {
  const int lane = threadIdx.x & 63;
  MxShare s;
  bool outside;
  const bool any = mx_share(a, s, outside);
  if (outside && status != nullptr && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, (int)PHOTON_STATUS_CACHE_FULL);
  if (!any) return;
  const int64_t tiles = (a.S_max + MX_TILE - 1) / MX_TILE;
  const int64_t at = (((int64_t)s.b * a.H_kv + s.h) * tiles + s.tile) * mx_tile_bytes(NB * MX_BLOCK);
  kc += at;
  vc += at;
  using P = MxPass<T, NB, VEC>;
  MxRaw<T, P::N, VEC> kr[NB][P::LOADS], vr[NB][P::LOADS];
  uint32_t held[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (!P::live(i, s.lo, s.hi)) continue;
    const P p(i, lane);
#pragma unroll
    for (int u = 0; u < P::LOADS; ++u) {
      const int kk = p.load_kk[u] < s.lo ? s.lo : p.load_kk[u] < s.hi ? p.load_kk[u] : s.hi - 1;   // what other positions give is not stored
      const int64_t row = (s.row0 + kk) * a.row_stride + (int64_t)s.h * a.d_h;
      kr[i][u].template load<ONCE>(k + row, p.load_dim[u], a.d_h);
      vr[i][u].template load<ONCE>(v + row, p.load_dim[u], a.d_h);
    }
    // the lane's V word, element dim + r of the 8 positions around p.kk: those outside [lo, hi) keep what they held
    const int group = p.kk & ~7;
    held[i] = 0;
    if ((s.lo > group || s.hi < group + 8) && s.lo < group + 8 && s.hi > group)
      held[i] = *reinterpret_cast<const uint32_t*>(vc + mx_v_word<NB>(s.base + group, p.dim + (lane >> 3)));
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (!P::live(i, s.lo, s.hi)) continue;
    const P p(i, lane);
    const int kk = s.base + p.kk, block = p.dim >> 5, group = p.kk & ~7;
    uint32_t ks, vs;
    const uint32_t kw = mx_word(p, kr[i], lane, a.d_h, ks), vw = mx_transpose8(mx_word(p, vr[i], lane, a.d_h, vs), lane);
    if (p.kk >= s.lo && p.kk < s.hi) {
      *reinterpret_cast<uint32_t*>(kc + mx_k_chunk<NB>(kk, block) + ((p.dim >> 3) & 3) * 4) = kw;
      if ((p.dim & 31) == 0) {
        kc[mx_k_scale<NB>(kk, block)] = (uint8_t)ks;
        vc[mx_v_scale<NB>(kk, block)] = (uint8_t)vs;
      }
    }
    const int from = s.lo > group ? s.lo - group : 0, to = s.hi < group + 8 ? s.hi - group : 8;
    if (from < to) {
      const uint32_t mask = (to == 8 ? 0xffffffffu : (1u << (4 * to)) - 1u) & ~((1u << (4 * from)) - 1u);
      *reinterpret_cast<uint32_t*>(vc + mx_v_word<NB>(s.base + group, p.dim + (lane >> 3))) = (held[i] & ~mask) | (vw & mask);
    }
  }
}

template <typename T, int NB, int VEC>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_read_kernel(const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc, T* __restrict__ k,
                                                                   T* __restrict__ v, MxRows a) {
  const int lane = threadIdx.x & 63;
  MxShare s;
  bool outside;
  if (!mx_share(a, s, outside)) return;
  const int64_t tiles = (a.S_max + MX_TILE - 1) / MX_TILE;
  const int64_t at = (((int64_t)s.b * a.H_kv + s.h) * tiles + s.tile) * mx_tile_bytes(NB * MX_BLOCK);
  kc += at;
  vc += at;
  using P = MxPass<T, NB, VEC>;
  uint32_t kw[NB], vw[NB], ks[NB], vs[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (!P::live(i, s.lo, s.hi)) continue;
    const P p(i, lane);
    const int kk = s.base + p.kk, block = p.dim >> 5;
    kw[i] = *reinterpret_cast<const uint32_t*>(kc + mx_k_chunk<NB>(kk, block) + ((p.dim >> 3) & 3) * 4);
    vw[i] = *reinterpret_cast<const uint32_t*>(vc + mx_v_word<NB>(kk & ~7, p.dim + (lane >> 3)));
    ks[i] = kc[mx_k_scale<NB>(kk, block)];
    vs[i] = vc[mx_v_scale<NB>(kk, block)];
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (!P::live(i, s.lo, s.hi)) continue;
    const P p(i, lane);
    uint32_t kc_[P::LOADS], ks_[P::LOADS], vc_[P::LOADS], vs_[P::LOADS];
    mx_parts<P>(kw[i], ks[i], lane, kc_, ks_);
    mx_parts<P>(mx_transpose8(vw[i], lane), vs[i], lane, vc_, vs_);
#pragma unroll
    for (int u = 0; u < P::LOADS; ++u) {
      float kv[P::N], vv[P::N];
      mx_values(kc_[u], ks_[u], kv);
      mx_values(vc_[u], vs_[u], vv);
      if (p.load_kk[u] >= s.lo && p.load_kk[u] < s.hi) {
        const int64_t row = (s.row0 + p.load_kk[u]) * a.row_stride + (int64_t)s.h * a.d_h;
        mx_store<T, P::N, VEC>(k + row, p.load_dim[u], a.d_h, kv);
        mx_store<T, P::N, VEC>(v + row, p.load_dim[u], a.d_h, vv);
      }
    }
  }
}

// ------------------------------------------------------------------ few rows
//
// A wave of the kernels above uses one lane in eight where a sequence has one new row, and the instructions that it issues are
// what bounds a step's append.  Up to MX_FEW rows per sequence are taken with a lane per 8 elements of a head instead, all rows
// of 64 / (4 NB) heads by one wave: 256 sequences append one bf16 row of 32 x 52 elements in 4.4 us (7.9 with the kernel above),
// three in 5.3 (9.8), four in 6.1 (9.9) and read them back in 3.5 (5.8), 4.5 (7.6) and 5.0 (7.8); four sequences of 32 x 64 fp32
// elements one in 2.9 (3.5), four in 4.0 (3.5).  These are kernels by themselves, their rows and tiles in the chip's caches; from
// HBM 256 sequences' three rows take 5.6 and 5.0, four sequences' one 4.8 and 4.7.  The rule goes by the rows of a sequence alone: four
// of few sequences lose the half microsecond above, which shows in a graph only (a call from the host takes 6 us either way).
// V words are put together nibble by nibble, 8 of them a lane, in the one or two groups of 8 positions that the rows are in.
constexpr int MX_FEW = 4;        // rows of a sequence, at most

struct MxFew {
  int b, h, n;                   // sequence, head, rows in use that have a place
  int dim;                       // first of the lane's 8 elements
  int64_t begin, row0;           // position of the first of them, and its row
  int64_t stream;
};
template <int NB> __device__ __forceinline__ bool mx_few(const MxRows& a, MxFew& s, bool& outside) {
  constexpr int LANES = 4 * NB;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  s.b = blockIdx.y;
  s.h = (blockIdx.x * (blockDim.x >> 6) + wave) * (64 / LANES) + lane / LANES;
  s.dim = lane % LANES * 8;
  int64_t n = a.n_new ? a.n_new[s.b] : a.T;
  n = n < 0 ? 0 : n > a.T ? a.T : n;
  const int64_t first = (a.start ? (int64_t)a.start[s.b] : 0) + a.add;
  s.begin = first < 0 ? 0 : first;
  const int64_t end = first + n < a.S_max ? first + n : a.S_max;
  outside = n > 0 && (first < 0 || first + n > a.S_max);
  s.n = end > s.begin ? (int)(end - s.begin) : 0;
  s.row0 = (int64_t)s.b * a.T + s.begin - first;
  s.stream = (int64_t)s.b * a.H_kv + s.h;
  return s.n > 0;
}
// The byte of position pos's 8-position group in the stream's tiles.
template <int NB> __device__ __forceinline__ int64_t mx_few_tile(const MxRows& a, const MxFew& s, int64_t pos) {
  return (s.stream * ((a.S_max + MX_TILE - 1) / MX_TILE) + pos / MX_TILE) * mx_tile_bytes(NB * MX_BLOCK);
}

template <typename T, int NB, int VEC>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_write_few_kernel(const T* __restrict__ k, const T* __restrict__ v, uint8_t* __restrict__ kc,
                                                                        uint8_t* __restrict__ vc, int32_t* __restrict__ status, MxRows a) {
  MxFew s;
  bool outside;
  const bool any = mx_few<NB>(a, s, outside);
  if (outside && status != nullptr && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(status, (int)PHOTON_STATUS_CACHE_FULL);
  if (!any) return;
  const bool mine = s.h < a.H_kv;                          // a wave's heads past the last one load what the last one loads, and store nothing
  if (!mine) { s.stream -= s.h - (a.H_kv - 1); s.h = a.H_kv - 1; }
  MxRaw<T, 4, VEC> kr[MX_FEW][2], vr[MX_FEW][2];
#pragma unroll
  for (int t = 0; t < MX_FEW; ++t) {
    if (t >= s.n) break;
    const int64_t row = (s.row0 + t) * a.row_stride + (int64_t)s.h * a.d_h;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      kr[t][u].template load<false>(k + row, s.dim + 4 * u, a.d_h);
      vr[t][u].template load<false>(v + row, s.dim + 4 * u, a.d_h);
    }
  }
  const int in = (int)(s.begin & 7);                       // of the first group; rows from 8 - in on are in the second
  const int groups = in + s.n > 8 ? 2 : 1, block = s.dim >> 5;
  uint32_t held[2][8], word[2][8];
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int e = 0; e < 8; ++e) word[g][e] = held[g][e] = 0;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (g >= groups) break;
    const int64_t pos = s.begin + 8 * g;
    const uint8_t* tile = vc + mx_few_tile<NB>(a, s, pos);
#pragma unroll
    for (int e = 0; e < 8; ++e) held[g][e] = *reinterpret_cast<const uint32_t*>(tile + mx_v_word<NB>((int)(pos % MX_TILE) & ~7, s.dim + e));
  }
#pragma unroll
  for (int t = 0; t < MX_FEW; ++t) {
    if (t >= s.n) break;
    const int64_t pos = s.begin + t;
    const int kk = (int)(pos % MX_TILE), at = in + t;
    uint32_t ks, vs, kw, vw;
    float x[8];
    auto values = [&](const MxRaw<T, 4, VEC> (&raw)[2]) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float y[4];
        raw[u].values(s.dim + 4 * u, a.d_h, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * u + e] = y[e];
      }
    };
    values(kr[t]);
    kw = mx_quantise(x, ks);
    values(vr[t]);
    vw = mx_quantise(x, vs);
    const int64_t tile = mx_few_tile<NB>(a, s, pos);
    if (mine) {
      *reinterpret_cast<uint32_t*>(kc + tile + mx_k_chunk<NB>(kk, block) + ((s.dim >> 3) & 3) * 4) = kw;
      if ((s.dim & 31) == 0) {
        kc[tile + mx_k_scale<NB>(kk, block)] = (uint8_t)ks;
        vc[tile + mx_v_scale<NB>(kk, block)] = (uint8_t)vs;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t nibble = ((vw >> (4 * e)) & 15u) << (4 * (at & 7));
      if (at < 8) word[0][e] |= nibble;
      else word[1][e] |= nibble;
    }
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (g >= groups) break;
    const int from = g == 0 ? in : 0, to = in + s.n - 8 * g < 8 ? in + s.n - 8 * g : 8;     // of the group, never all of it
    const uint32_t mask = (to == 8 ? 0xffffffffu : (1u << (4 * to)) - 1u) & ~((1u << (4 * from)) - 1u);
    const int64_t pos = s.begin + 8 * g;
    uint8_t* tile = vc + mx_few_tile<NB>(a, s, pos);
    if (mine)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<uint32_t*>(tile + mx_v_word<NB>((int)(pos % MX_TILE) & ~7, s.dim + e)) = (held[g][e] & ~mask) | word[g][e];
  }
}

template <typename T, int NB, int VEC>
__global__ __launch_bounds__(MX_WAVES * 64) void mxfp4_read_few_kernel(const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc, T* __restrict__ k,
                                                                       T* __restrict__ v, MxRows a) {
  MxFew s;
  bool outside;
  if (!mx_few<NB>(a, s, outside) || s.h >= a.H_kv) return;
  const int in = (int)(s.begin & 7), groups = in + s.n > 8 ? 2 : 1, block = s.dim >> 5;
  uint32_t kw[MX_FEW], ks[MX_FEW], vs[MX_FEW], word[2][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) word[1][e] = 0;
#pragma unroll
  for (int t = 0; t < MX_FEW; ++t) {
    if (t >= s.n) break;
    const int64_t pos = s.begin + t, tile = mx_few_tile<NB>(a, s, pos);
    const int kk = (int)(pos % MX_TILE);
    kw[t] = *reinterpret_cast<const uint32_t*>(kc + tile + mx_k_chunk<NB>(kk, block) + ((s.dim >> 3) & 3) * 4);
    ks[t] = kc[tile + mx_k_scale<NB>(kk, block)];
    vs[t] = vc[tile + mx_v_scale<NB>(kk, block)];
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (g >= groups) break;
    const int64_t pos = s.begin + 8 * g;
    const uint8_t* tile = vc + mx_few_tile<NB>(a, s, pos);
#pragma unroll
    for (int e = 0; e < 8; ++e) word[g][e] = *reinterpret_cast<const uint32_t*>(tile + mx_v_word<NB>((int)(pos % MX_TILE) & ~7, s.dim + e));
  }
#pragma unroll
  for (int t = 0; t < MX_FEW; ++t) {
    if (t >= s.n) break;
    const int at = in + t;
    uint32_t vw = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w0 = word[0][e], w1 = word[1][e];
      vw |= (((at < 8 ? w0 : w1) >> (4 * (at & 7))) & 15u) << (4 * e);
    }
    const int64_t row = (s.row0 + t) * a.row_stride + (int64_t)s.h * a.d_h;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float kv[4], vv[4];
      mx_values(kw[t] >> (16 * u), ks[t], kv);
      mx_values(vw >> (16 * u), vs[t], vv);
      mx_store<T, 4, VEC>(k + row, s.dim + 4 * u, a.d_h, kv);
      mx_store<T, 4, VEC>(v + row, s.dim + 4 * u, a.d_h, vv);
    }
  }
}

// ------------------------------------------------------------------ attention
//
// Score and value products run on the matrix cores in bf16, in which every stored value is exact; fp32 operands (an fp32 query, a
// weight) enter as three bf16 parts of 8 bits each, which are exact too, so nothing is rounded below fp32 but a bf16 result.
//
// A wave takes 64 positions at a time: NB loads of 16 bytes a lane of K, as many of V, and the scale bytes.
//   Scores: S^T = Q K^T with the queries (or the parts of one query) as the four rows i of every row group g = 0..3 of a
//     16 x 16 x 32 MFMA and positions as columns.  A lane's K chunk is 32 elements of one position under one scale, so its
//     conversion takes the scale along, and the four MFMAs that consume it contract over all of the chunks of a column.  Which of
//     them belong to one position differs by NB: row group g has the query where the chunks belong to positions 16 g .. + 15
//     (or could), zeros elsewhere, and picks the load that holds them.  Lane l ends up with the scores of position l: softmax
//     costs one exponential per lane and query, and no lane repeats another's.
//   Values: O = (P X) V with the weights times V's scale as rows (a scale per 32 elements: one such operand per block) and the
//     elements of V as columns.  The weights change from a lane per position to operand order through LDS.  The three parts of
//     four queries (or of one) fit the sixteen rows; of eight, two do, and the third goes into the second's sums as an operand of
//     its own (sums of its own would not fit the registers: 59 spilled).
//   The reference of the exponentials is the largest score when it was last raised, which happens when one exceeds it by more
//     than MX_RAISE: the usual tile needs no maximum, and weights go up to 2^MX_RAISE.  Times V below 2^67 and summed over 2^31
//     positions that stays below 2^106.  From the first tile on that holds larger V for it (scale byte MX_LARGE and up) a wave
//     takes V in units of 2^MX_UNIT, in its slow body: below 2^103 for fp32's largest.  Results of waves and splits are means and
//     put together as such (serving and grouped heads take as long as they did without; short streams of 2 - 3 tiles 16.7 us, 16.2).
// Bound by HBM where streams are many (256 x 16 streams of 2048 positions: 573 MB in 84.5 us = 6.8 TB/s; 186 vector instructions a
// tile of 64 x 64, 16 of them MFMAs, of about 380 that the bytes leave time for), by the start and the end of a wave where they are
// few or short (4 x 32 streams of 8192 positions: 71 MB in 15.8 us with the merge, 16.8 with none of it in a cache), by the weights'
// instructions and two waves a SIMD with eight queries of 128 elements (699 a tile, 64 of them MFMAs: 143 MB in 42.3 us, four
// queries 33, one 28).
constexpr float MX_RAISE = 8.f;
constexpr float MX_LOWEST = -3.402823466e38f;    // of fp32: no finite score is below it
constexpr uint32_t MX_LARGE = 192, MX_UNIT = 64; // scale byte from which V is large, and log2 of the unit it is taken in then
constexpr int MX_ATTN_WAVES = 8;                 // of a workgroup, at most
constexpr int MX_P_PITCH = 72;                   // bf16 elements of a weight row in LDS: 64 positions, rows on different banks

template <typename T, int NB, int NQ> struct MxAttn {
  static constexpr int DP = NB * MX_BLOCK;
  static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  static constexpr int SETS = NQ == 1 ? 1 : PARTS * (NQ / 4);       // score operands: parts (one query: its parts are rows of one)
  static constexpr int B_ROWS = NQ == 1 ? 4 : 3 * NQ;               // weight rows of a block: NQ part + query (one query: its parts, and one unused)
  static constexpr int P_ROWS = B_ROWS * NB;
  static constexpr int ACC = 2 * NB;                                // column tiles of 16 elements
  // per wave: weight rows, and the staged queries or the wave's result
  static constexpr int P_BYTES = P_ROWS * MX_P_PITCH * 2;
  static constexpr int O_BYTES = NQ * (DP + 2) * 4;
  static constexpr int Q_BYTES = NQ * PARTS * DP * 2;
  static constexpr int WAVE_BYTES = ((P_BYTES > O_BYTES ? P_BYTES > Q_BYTES ? P_BYTES : Q_BYTES : O_BYTES > Q_BYTES ? O_BYTES : Q_BYTES) + 15) & ~15;
};

__device__ __forceinline__ bf16x8_t mx_operand(uint32_t w, float scale) {
  uint4_t r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return as_bf16x8(r);
}

// x = a + b + c, each with 8 significant bits (in the upper halves of the words): exact but for subnormals.
__device__ __forceinline__ void mx_split3(float x, float& a, float& b, float& c) {
  a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  const float r = x - a;
  b = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
  c = r - b;
}

// The upper PARTS * 8 bits of x as bf16 parts, `pitch` elements apart.
template <int PARTS> __device__ __forceinline__ void mx_put_parts(uint16_t* to, int pitch, float x) {
  float part[3];
  mx_split3(x, part[0], part[1], part[2]);
#pragma unroll
  for (int u = 0; u < PARTS; ++u) to[u * pitch] = (uint16_t)(__float_as_uint(part[u]) >> 16);
}

// Largest of the wave in every lane, by data-parallel moves and exchanges of rows (no trip through LDS, as in wave_sum).
__device__ __forceinline__ float mx_wave_max(float x) {
  x = fmaxf(x, dpp<DPP_XOR1>(x));
  x = fmaxf(x, dpp<DPP_XOR2>(x));
  x = fmaxf(x, dpp<DPP_HALF_MIRROR>(x));
  x = fmaxf(x, dpp<DPP_MIRROR>(x));
  typedef uint32_t uint2_native __attribute__((ext_vector_type(2)));
  const uint2_native r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint2_native h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// LDS traffic of one wave is in order; this keeps the compiler from moving it.
__device__ __forceinline__ void mx_wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

struct MxQueries {
  const int32_t *seq_len, *n_new;
  int64_t q_stride, S_max;
  int T, H, H_kv, d_h, group, groups, n_splits;    // group: query heads of a K/V head; groups: workgroups that share its T * group queries
  int add;                                         // to seq_len
  bool out_bf16;                                   // fp32 queries with bf16 results
  float scale_log2e;
};

template <typename T> __device__ __forceinline__ void mx_put(T* out, int64_t at, float y, bool bf16) {
  if (sizeof(T) == 4 && bf16) reinterpret_cast<bf16_t*>(out)[at] = from_f32<bf16_t>(y);
  else out[at] = from_f32<T>(y);
}

// x * y, not merged with what follows: the reference was rounded, too, and what a merged product keeps beyond it is an exponent of its
// own once scores pass 2^24.
__device__ __forceinline__ float mx_rounded_product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// 1 / l; 0 where nothing was seen.
__device__ __forceinline__ float mx_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Positions that count for sequence b, and its queries.
__device__ __forceinline__ void mx_sequence(const MxQueries& a, int b, int& n, int& m) {
  const int64_t all = (int64_t)a.seq_len[b] + a.add;
  n = all < 0 ? 0 : all > a.S_max ? (int)a.S_max : (int)all;                // S_max <= MX_MOST
  m = a.n_new ? a.n_new[b] : a.T;
  m = m < 0 ? 0 : m > a.T ? a.T : m;
}

template <typename T, int NB, int NQ>
__global__ __launch_bounds__(MX_ATTN_WAVES * 64) void mxfp4_attn_kernel(const T* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                                                         T* __restrict__ out, float* __restrict__ ws, MxQueries a) {
  using C = MxAttn<T, NB, NQ>;
  constexpr int DP = C::DP, SETS = C::SETS, ACC = C::ACC, PARTS = C::PARTS, TB = mx_tile_bytes(DP);
  extern __shared__ __align__(16) char mx_lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, waves = blockDim.x >> 6;
  const int c = lane & 15, kg = lane >> 4;

  const unsigned split = a.groups == 1 ? blockIdx.x : blockIdx.x / (unsigned)a.groups, chunk = blockIdx.x - split * a.groups;
  const int b = blockIdx.z, hk = blockIdx.y;

  int n, m;
  mx_sequence(a, b, n, m);
  // query i of the workgroup is row first_q + i of the stream's m * group: token row / group, head hk * group + row % group; it
  // sees seen[i] positions
  const int first_q = chunk * NQ, queries = m * a.group - first_q;           // of this workgroup, at most NQ count
  if (queries <= 0) return;
  int seen[NQ];
  int64_t q_row[NQ];
  {
    int t = a.group == 1 ? first_q : first_q / a.group, h = first_q - t * a.group;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int s = n - m + t + 1;
      seen[i] = s < 0 ? 0 : s;
      q_row[i] = ((int64_t)b * a.T + t) * a.q_stride + (int64_t)(hk * a.group + h) * a.d_h;
      if (i + 1 < queries && ++h == a.group) { h = 0; ++t; }                 // past the last query: the last one again
    }
  }
  const int hi = seen[NQ - 1], lo = seen[0];                                 // seen grows with i
  // The waves of all splits take the tiles in turn.  Splits that no tile is left for write nothing: the merge knows them.
  const int end = (int)(((unsigned)hi + MX_TILE - 1) / MX_TILE), stride = a.n_splits * waves;
  int tile = split * waves + wave;
  if (a.n_splits > 1 && (int64_t)split * waves * MX_TILE >= n) return;

  const int64_t tiles = (a.S_max + MX_TILE - 1) / MX_TILE;
  const int64_t stream = (int64_t)b * a.H_kv + hk;
  const uint8_t* kt = kc + stream * tiles * TB + lane * 16;
  const uint8_t* vt = vc + stream * tiles * TB + lane * 16;
  const uint8_t* kst = kc + stream * tiles * TB + NB * 1024 + lane * NB;
  const uint8_t* vst = vc + stream * tiles * TB + NB * 1024 + lane * NB;

  struct Tile { uint4_t k[NB], v[NB]; uint32_t ks, vs; };
  auto load_scales = [&](const uint8_t* p) -> uint32_t {
    if constexpr (NB == 1) return *p;
    else if constexpr (NB == 2) return *reinterpret_cast<const uint16_t*>(p);
    else return *reinterpret_cast<const uint32_t*>(p);
  };
  auto load = [&](int tile, Tile& x) {
    const int64_t at = (int64_t)tile * TB;
    x.ks = load_scales(kst + at);
#pragma unroll
    for (int t = 0; t < NB; ++t) x.k[t] = load16_stream(kt + at + t * 1024);
    x.vs = load_scales(vst + at);
#pragma unroll
    for (int t = 0; t < NB; ++t) x.v[t] = load16_stream(vt + at + t * 1024);
  };

  Tile cur, nxt;
  if (tile < end) load(tile, cur);

  // queries: their parts into the wave's LDS, then into the operands of the score products
  char* own = mx_lds + wave * C::WAVE_BYTES;
  bf16x8_t aq[SETS][4];
  {
    uint16_t* qs = reinterpret_cast<uint16_t*>(own);                         // [query][part][DP]
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int d0 = 0; d0 < DP; d0 += 64) {
        const int d = d0 + lane;
        if (DP < 64 && d >= DP) continue;
        uint16_t* to = qs + i * PARTS * DP + d;
        const float x = d < a.d_h ? to_f32<T>(q[q_row[i] + d]) : 0.f;
        mx_put_parts<PARTS>(to, DP, x);
      }
    mx_wave_order();
    const int g = c >> 2, i = c & 3;                                         // operand row c = 4 g + i
    const int block = NB == 1 ? 0 : NB == 2 ? kg & 1 : kg;
    const bool mine = NB == 1 ? g == kg : NB == 2 ? (g & 1) == (kg >> 1) : true;
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      // one query: row i is its part i (rows past the last part are not looked at); else part s % PARTS of query 4 (s / PARTS) + i
      const int row = NQ == 1 ? (i < PARTS ? i : 0) : ((s / PARTS) * 4 + i) * PARTS + s % PARTS;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint4_t w = *reinterpret_cast<const uint4_t*>(qs + row * DP + block * 32 + j * 8);
        if (!mine) w = uint4_t{0, 0, 0, 0};
        aq[s][j] = as_bf16x8(w);
      }
    }
  }
  mx_wave_order();                                                           // the staged queries make room for the weights

  uint16_t* pw = reinterpret_cast<uint16_t*>(own);
  const uint16_t* pr = pw + kg * 8;
  float top[NQ], sum[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) { top[i] = MX_LOWEST; sum[i] = 0.f; }
  f32x4_t acc[ACC];
#pragma unroll
  for (int t = 0; t < ACC; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // Scale bytes above MX_LAST_SCALE, or from MX_LARGE on, four at a time: the top bit of every byte that is one.
  auto bad_bytes = [](uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x03030303u) & w & 0x80808080u; };
  auto large_bytes = [](uint32_t w) { return w & (w << 1) & 0x80808080u; };
  static_assert(MX_LAST_SCALE == 252 && MX_LARGE == 192, "bad_bytes, large_bytes");
  bool large = false;                                                        // V counts in units of 2^MX_UNIT

  // SLOW: tiles that some query does not see whole, or that hold a NaN block: positions that nobody sees must not reach a sum, not
  // even times zero, and a NaN must reach its own position only, not the others of its column.  Large V, too, and all that follows it.
  auto consume = [&](auto slow_tag, int tile_at, const Tile& x) {
    constexpr bool SLOW = decltype(slow_tag)::value;
    const int base = tile_at * MX_TILE;
    float kf[NB], vf[NB];
    bool nan_here = false;
    if constexpr (SLOW) {
      if (!large && __builtin_amdgcn_ballot_w64(base + lane < hi && (large_bytes(x.vs) & ~bad_bytes(x.vs)) != 0) != 0) {
        large = true;
        const float unit = __uint_as_float((127u - MX_UNIT) << 23);
#pragma unroll
        for (int t = 0; t < ACC; ++t) acc[t] *= unit;
      }
    }
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      const uint32_t kx = (x.ks >> (8 * t)) & 255u, vx = (x.vs >> (8 * t)) & 255u;
      kf[t] = __uint_as_float(kx << 23);
      vf[t] = __uint_as_float(vx << 23);
      if constexpr (SLOW) {
        const int key = base + (t * 4 + kg) / NB * 16 + c;
        const bool bad = kx > (uint32_t)MX_LAST_SCALE;
        if (bad || key >= hi) kf[t] = 1.f;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(bad && key < hi);
#pragma unroll
        for (int u = 0; u < 4; ++u)                                          // chunks u of this load that belong to position `lane`
          if ((t * 4 + u) / NB == kg) nan_here = nan_here || ((mask >> (u * 16 + c)) & 1u);
        if (large) vf[t] = __uint_as_float((vx > MX_UNIT ? vx - MX_UNIT : 0u) << 23);
        if (vx > (uint32_t)MX_LAST_SCALE) vf[t] = __uint_as_float(0x7fc00000u);
      }
    }
    float s[NQ];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      f32x4_t d[SETS];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8_t bop = mx_operand(x.k[t][j], kf[t]);
#pragma unroll
        for (int u = 0; u < SETS; ++u)
          d[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq[u][j], bop, j == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : d[u], 0, 0, 0);
      }
      const bool pick = NB == 1 || t == 0 || (NB == 2 ? (kg >> 1) == t : kg == t);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        float y;
        if constexpr (PARTS == 1) y = d[i / 4][i % 4];
        else if constexpr (NQ == 1) y = (d[0][2] + d[0][1]) + d[0][0];
        else y = (d[i / 4 * 3 + 2][i % 4] + d[i / 4 * 3 + 1][i % 4]) + d[i / 4 * 3][i % 4];
        s[i] = pick ? y : s[i];
      }
    }
    // e: what the exponential is taken of
    float e[NQ];
    auto reduce = [&](int i) { e[i] = s[i] - top[i]; };
    float highest = MX_LOWEST;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      s[i] = mx_rounded_product(s[i], a.scale_log2e);
      if constexpr (SLOW) {
        if (nan_here) s[i] = __uint_as_float(0x7fc00000u);
        if (base + lane >= seen[i]) s[i] = MX_LOWEST;
      }
      reduce(i);
      highest = fmaxf(highest, e[i]);
    }
    if (__builtin_amdgcn_ballot_w64(highest > MX_RAISE) != 0) {
      float shrink[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const float higher = fmaxf(top[i], mx_wave_max(s[i]));
        shrink[i] = fast_exp2(top[i] - higher);
        top[i] = higher;
        sum[i] *= shrink[i];
        reduce(i);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // row 4 kg + r of the value products is of query (4 kg + r) % NQ
        const float f0 = shrink[r % NQ], f1 = shrink[(4 + r) % NQ], f = NQ == 8 && (kg & 1) ? f1 : f0;
#pragma unroll
        for (int t = 0; t < ACC; ++t) acc[t][r] *= f;
      }
    }
    float p[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      p[i] = fast_exp2(e[i]);
      if (SLOW && base + lane >= seen[i]) p[i] = 0.f;
      sum[i] += p[i];
    }
    if constexpr (NQ == 1) {
      // rows 4 block + part
      mx_wave_order();
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        float y = p[0] * vf[t];
        if (SLOW && base + lane >= seen[0]) y = 0.f;
        mx_put_parts<3>(pw + 4 * t * MX_P_PITCH + lane, MX_P_PITCH, y);
      }
      mx_wave_order();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8_t aop = as_bf16x8(*reinterpret_cast<const uint4_t*>(pr + (c % C::P_ROWS) * MX_P_PITCH + h * 32));
#pragma unroll
        for (int t = 0; t < ACC; ++t) {
          const int w = h * ACC + t;
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aop, mx_operand(x.v[w >> 2][w & 3], 1.f), acc[t], 0, 0, 0);
        }
      }
    } else {
      mx_wave_order();
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          float y = p[i] * vf[blk];
          if (SLOW && base + lane >= seen[i]) y = 0.f;
          mx_put_parts<3>(pw + (blk * C::B_ROWS + i) * MX_P_PITCH + lane, NQ * MX_P_PITCH, y);
        }
      mx_wave_order();
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int w = h * ACC + 2 * blk;
          const bf16x8_t v0 = mx_operand(x.v[w >> 2][w & 3], 1.f), v1 = mx_operand(x.v[(w + 1) >> 2][(w + 1) & 3], 1.f);
          auto weights = [&](int row) { return *reinterpret_cast<const uint4_t*>(pr + (blk * C::B_ROWS + row) * MX_P_PITCH + h * 32); };
          const bf16x8_t aop = as_bf16x8(weights(NQ == 8 || c < 12 ? c : c - 12));
          acc[2 * blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aop, v0, acc[2 * blk], 0, 0, 0);
          acc[2 * blk + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aop, v1, acc[2 * blk + 1], 0, 0, 0);
          if constexpr (NQ == 8) {                                           // two parts fill the rows: the third is added to the second's
            uint4_t third = weights(8 + c);
            if (c < 8) third = uint4_t{0, 0, 0, 0};
            acc[2 * blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(third), v0, acc[2 * blk], 0, 0, 0);
            acc[2 * blk + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(third), v1, acc[2 * blk + 1], 0, 0, 0);
          }
        }
    }
  };

  auto either = [&](const Tile& x) {
    if (tile * MX_TILE + MX_TILE > lo || large || __builtin_amdgcn_ballot_w64((bad_bytes(x.ks) | large_bytes(x.vs)) != 0) != 0)
      consume(std::true_type{}, tile, x);
    else
      consume(std::false_type{}, tile, x);
  };
  // One body: a second one for the other buffer makes the code twice as long, and a launch of some microseconds waits for code, too
  // (128k tokens, batch 4: 17.1 us, 18.6 with two).
#pragma unroll 1
  while (tile < end) {
    const int next = tile + stride;
    if (next < end) load(next, nxt);
    either(cur);
    cur = nxt;
    tile = next;
  }

  // The wave's result: sums over lanes, parts put together, into LDS.  Values are divided by the sum here, and results are put
  // together as weighted means: no sum of values leaves the range that the values are in.
  mx_wave_order();
  float* ow = reinterpret_cast<float*>(own);
  float mean[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const float l = wave_sum(sum[i]);
    if (lane == 0) { ow[i * (DP + 2)] = top[i]; ow[i * (DP + 2) + 1] = l; }
    mean[i] = mx_inverse(l) * (large ? __uint_as_float((127u + MX_UNIT) << 23) : 1.f);
  }
#pragma unroll
  for (int t = 0; t < ACC; ++t) {
    if constexpr (NQ == 1) {
      const float y = (acc[t][2] + acc[t][1]) + acc[t][0];
      if (kg == t / 2) ow[2 + 16 * t + c] = y * mean[0];
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // the parts: in row groups NQ / 4 apart
        float y = NQ == 8 || kg < 3 ? acc[t][r] : 0.f;
        y += __shfl_xor(y, 32);
        if constexpr (NQ == 4) y += __shfl_xor(y, 16);
        const float f0 = mean[r], f1 = mean[(4 + r) % NQ], f = NQ == 8 && kg ? f1 : f0;
        if (4 * kg + r < NQ) ow[(4 * kg + r) * (DP + 2) + 2 + 16 * t + c] = y * f;
      }
    }
  }
  __syncthreads();
  // The waves' results, in order.
  for (int x = tid; x < NQ * DP; x += blockDim.x) {
    const int i = x / DP, d = x % DP;
    if (i >= queries) break;
    const float* at = reinterpret_cast<const float*>(mx_lds) + i * (DP + 2);
    float w_top[MX_ATTN_WAVES], w_sum[MX_ATTN_WAVES], w_o[MX_ATTN_WAVES], mx = MX_LOWEST;
#pragma unroll
    for (int w = 0; w < MX_ATTN_WAVES; ++w) {
      const float* from = at + (w < waves ? w : 0) * (C::WAVE_BYTES / 4);
      w_top[w] = w < waves ? from[0] : MX_LOWEST;
      w_sum[w] = from[1];
      w_o[w] = from[2 + d];
      mx = fmaxf(mx, w_top[w]);
    }
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < MX_ATTN_WAVES; ++w) {
      if (w >= waves) break;
      w_sum[w] *= fast_exp2(w_top[w] - mx);
      l += w_sum[w];
    }
    const float r = mx_inverse(l);
#pragma unroll
    for (int w = 0; w < MX_ATTN_WAVES; ++w) {
      if (w >= waves) break;
      o = fmaf(w_o[w], w_sum[w] * r, o);
    }
    const int row = first_q + i, t = a.group == 1 ? row : row / a.group, h = hk * a.group + row - t * a.group;
    const int64_t to = ((int64_t)b * a.T + t) * a.H + h;
    if (a.n_splits == 1) {
      if (d < a.d_h) mx_put(out, to * a.d_h + d, o, a.out_bf16);
    } else {
      float* p = ws + (to * a.n_splits + split) * (DP + 2);
      if (d == 0) { p[0] = mx; p[1] = l; }
      p[2 + d] = o;
    }
  }
}

// The splits' results of one query, in order, eight at a time in flight.
template <typename T, int NB>
__global__ __launch_bounds__(NB * MX_BLOCK) void mxfp4_merge_kernel(const float* __restrict__ ws, T* __restrict__ out, MxQueries a, int waves) {
  constexpr int DP = NB * MX_BLOCK;
  const int h = blockIdx.x, t = blockIdx.y, b = blockIdx.z, d = threadIdx.x;
  int n, m;
  mx_sequence(a, b, n, m);
  if (t >= m) return;
  const unsigned span = waves * MX_TILE, spans = ((unsigned)n + span - 1) / span;
  const int used = spans < (unsigned)a.n_splits ? (int)spans : a.n_splits;
  const int64_t to = ((int64_t)b * a.T + t) * a.H + h;
  const float* p = ws + to * a.n_splits * (DP + 2);
  float mx = MX_LOWEST, l = 0.f, o = 0.f;                    // o: weighted mean of the splits so far, l: their weight
  for (int s0 = 0; s0 < used; s0 += 8) {
    float s_top[8], s_sum[8], s_o[8], higher = mx;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float* from = p + (s0 + u < used ? s0 + u : 0) * (DP + 2);
      s_top[u] = from[0];
      s_sum[u] = from[1];
      s_o[u] = from[2 + d];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (s0 + u >= used) s_top[u] = MX_LOWEST;
      higher = fmaxf(higher, s_top[u]);
    }
    const float before = l * fast_exp2(mx - higher);
    mx = higher;
    l = before;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (s0 + u >= used) break;
      s_sum[u] *= fast_exp2(s_top[u] - mx);
      l += s_sum[u];
    }
    const float r = mx_inverse(l);
    o *= before * r;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (s0 + u >= used) break;
      o = fmaf(s_o[u], s_sum[u] * r, o);
    }
  }
  if (d < a.d_h) mx_put(out, to * a.d_h + d, o, a.out_bf16);
}

// Queries that share what a workgroup reads.  fp32: at most 4 (the operands of 8 are 96 registers a lane: 120 spilled).
int mx_query_rows(int64_t queries, bool f32) { return queries <= 1 ? 1 : queries <= 4 || f32 ? 4 : 8; }

// One workgroup of eight waves per compute unit where streams are few, as long as a wave has four tiles: 128 streams of 128 tiles
// take 16.9 us in 2 splits, 19.9 in 1, 17.9 in 4; 16 streams of 32 tiles 7.3 us in 1, 8.2 in 2 (the merge is a launch).  Eight
// queries of 128 elements over 32 streams of 512 tiles: bf16, one workgroup for all, 42.7 us in 8 splits, 61.4 in 4; fp32, two
// workgroups, 67.2 in 8 and 60.6 in 4.
int mx_auto_splits(int Bt, int T, int H, int H_kv, int64_t S_max, bool f32) {
  const int64_t queries = (int64_t)T * (H / H_kv), rows = mx_query_rows(queries, f32);
  const int64_t groups = (int64_t)Bt * H_kv * ((queries + rows - 1) / rows), tiles = (S_max + MX_TILE - 1) / MX_TILE;
  int64_t splits = 256 / groups;
  const int64_t most = tiles / (4 * MX_ATTN_WAVES);
  splits = splits > most ? most : splits;
  return (int)(splits < 1 ? 1 : splits > 1024 ? 1024 : splits);
}

// Waves of a workgroup: eight, but not more than there are tiles, and once more waves are asked for than the chip holds, so many
// that one has eight tiles (its start and end cost as much as six): 8192 streams of 3 tiles take 17.6 us with one wave, 20.6
// with two, 52.8 with eight; 4096 streams of 32 tiles 86.2 us with four, 89.1 with two, 87.9 with eight.
int mx_waves(int64_t streams, int64_t S_max, int n_splits) {
  const int64_t tiles = (S_max + MX_TILE - 1) / MX_TILE;
  int waves = MX_ATTN_WAVES;
  while (waves > 1 && ((streams * n_splits * waves > 4096 && tiles < (int64_t)8 * waves * n_splits) || tiles <= (int64_t)waves / 2 * n_splits)) waves /= 2;
  return waves;
}

template <typename T, int NB, int NQ>
int32_t mx_launch_attn(const void* q, const void* kc, const void* vc, void* out, void* ws, const MxQueries& a, int Bt, hipStream_t st) {
  const int waves = mx_waves((int64_t)Bt * a.H_kv * a.groups, a.S_max, a.n_splits);
  const unsigned lds = waves * (MxAttn<T, NB, NQ>::WAVE_BYTES);
  PHOTON_LAUNCH(KC_COARSE_ATTN, st, (mxfp4_attn_kernel<T, NB, NQ>), dim3((unsigned)a.n_splits * (unsigned)a.groups, a.H_kv, Bt),
                dim3(waves * 64), lds, st, (const T*)q, (const uint8_t*)kc, (const uint8_t*)vc, (T*)out, (float*)ws, a);
  const int32_t rc = check_launch("mxfp4_attn_kernel");
  if (rc != PHOTON_OK || a.n_splits == 1) return rc;
  PHOTON_LAUNCH(KC_COARSE_MERGE, st, (mxfp4_merge_kernel<T, NB>), dim3(a.H, a.T, Bt), dim3(NB * MX_BLOCK), 0, st, (const float*)ws, (T*)out, a, waves);
  return check_launch("mxfp4_merge_kernel");
}

template <typename T, int NB>
int32_t mx_launch_attn_q(const void* q, const void* kc, const void* vc, void* out, void* ws, MxQueries a, int Bt, hipStream_t st) {
  const int64_t queries = (int64_t)a.T * a.group, rows = mx_query_rows(queries, sizeof(T) == 4);
  a.groups = (int)((queries + rows - 1) / rows);
  if (rows == 1) return mx_launch_attn<T, NB, 1>(q, kc, vc, out, ws, a, Bt, st);
  if constexpr (sizeof(T) == 2)
    if (rows == 8) return mx_launch_attn<T, NB, 8>(q, kc, vc, out, ws, a, Bt, st);
  return mx_launch_attn<T, NB, 4>(q, kc, vc, out, ws, a, Bt, st);
}

template <typename T>
int32_t mx_launch_attn_t(const void* q, const void* kc, const void* vc, void* out, void* ws, const MxQueries& a, int Bt, hipStream_t st) {
  switch (kv_row_elems(a.d_h)) {
    case 32: return mx_launch_attn_q<T, 1>(q, kc, vc, out, ws, a, Bt, st);
    case 64: return mx_launch_attn_q<T, 2>(q, kc, vc, out, ws, a, Bt, st);
    default: return mx_launch_attn_q<T, 4>(q, kc, vc, out, ws, a, Bt, st);
  }
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
  PHOTON_REQUIRE(S_max <= MX_MOST, PHOTON_ERR_UNSUPPORTED, "%s: S_max=%lld exceeds 2^31 - 64", who, (long long)S_max);
  PHOTON_REQUIRE(Bt <= 65535 && H_kv <= 65535, PHOTON_ERR_UNSUPPORTED, "%s: Bt=%d, H_kv=%d streams: at most 65535 each", who, Bt, H_kv);
  return PHOTON_OK;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Elements per access of rows: 8 (bf16) or 4 where pointers, stride and head size are whole multiples of it, else 1.
int row_vec(const void* a, const void* b, int64_t stride, int d_h, size_t esz) {
  const auto whole = [&](int vec) { return d_h % vec == 0 && stride % vec == 0 && aligned(a, vec * esz) && aligned(b, vec * esz); };
  return esz == 2 && whole(8) ? 8 : whole(4) ? 4 : 1;
}

// Steps of 16 positions that T rows can touch; waves of a workgroup; workgroups of a stream.
int64_t mx_row_steps(int T) { return ((int64_t)T + MX_STEP - 2) / MX_STEP + 1; }
int mx_row_waves(int T) { const int64_t n = mx_row_steps(T); return n < MX_WAVES ? (int)n : MX_WAVES; }
int64_t mx_row_groups(int T) { return (mx_row_steps(T) + mx_row_waves(T) - 1) / mx_row_waves(T); }

// Whether any of `rows` rows of `width` elements from a on, `stride` apart, shares an element with one of as many from b on.
bool rows_overlap(const void* a, const void* b, size_t esz, int64_t stride, int64_t width, int64_t rows) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  const int64_t apart = (int64_t)((x < y ? y - x : x - y) / esz), m = apart / stride, past = apart - m * stride;   // row m of the one begins `past` before the other
  return (m < rows && past < width) || (m + 1 < rows && stride - past < width);
}

int32_t rows_args(const char* who, const void* k, const void* v, const void* kc, const void* vc, int64_t row_stride, const MxRows& a, photon_dtype dt) {
  const size_t esz = dtype_size(dt);
  PHOTON_REQUIRE(k && v && aligned(k, esz) && aligned(v, esz), PHOTON_ERR_INVALID_ARG, "%s: k and v must be non-null device pointers to whole elements", who);
  PHOTON_REQUIRE(kc && vc && aligned16(kc) && aligned16(vc), PHOTON_ERR_INVALID_ARG, "%s: the caches must be non-null, 16-byte aligned device pointers", who);
  PHOTON_REQUIRE(row_stride >= (int64_t)a.H_kv * a.d_h, PHOTON_ERR_INVALID_ARG, "%s: row_stride=%lld is less than a row of %d heads of %d", who,
                 (long long)row_stride, a.H_kv, a.d_h);
  PHOTON_REQUIRE(kc != vc, PHOTON_ERR_INVALID_ARG, "%s: K and V need a cache each", who);
  PHOTON_REQUIRE(mx_row_groups(a.T) * a.H_kv <= (int64_t)0xffffffff / (MX_WAVES * 64), PHOTON_ERR_UNSUPPORTED, "%s: T=%d rows of %d heads are too many", who, a.T, a.H_kv);
  return PHOTON_OK;
}

MxRows mx_rows(const int32_t* start, const int32_t* n_new, int64_t row_stride, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max) {
  MxRows a;
  a.start = start; a.n_new = n_new; a.row_stride = row_stride; a.S_max = S_max;
  a.T = T; a.H_kv = H_kv; a.d_h = d_h; a.add = 0; a.heads_first = true;
  return a;
}

template <typename T, int NB, int VEC>
void launch_rows(bool write, const void* k, const void* v, const void* kc, const void* vc, int32_t* status, MxRows a, int Bt, hipStream_t st) {
  const dim3 grid((unsigned)(mx_row_groups(a.T) * a.H_kv), Bt), block(mx_row_waves(a.T) * 64);
  // A head's row of whole lines of 128 bytes is read past the caches (4 x 8192 rows of 32 x 64 elements: fp32 111 us, 145 through
  // them, bf16 70 and 88); where neighbours share lines that is slower (32 x 60 elements: 174 us, 167 through them, 120 and 92).
  const bool lines = a.d_h * sizeof(T) % 128 == 0 && a.row_stride * sizeof(T) % 128 == 0 && aligned(k, 128) && aligned(v, 128);
  // Read back, whole lines are written by workgroups of neighbouring positions: their tiles follow each other (bf16, 66 us instead of 76).
  a.heads_first = write || !lines;
  if (write && VEC * sizeof(T) >= 16 && lines)
    PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (mxfp4_write_kernel<T, NB, VEC, (VEC * sizeof(T) >= 16)>), grid, block, 0, st, (const T*)k, (const T*)v, (uint8_t*)kc,
                  (uint8_t*)vc, status, a);
  else if (write)
    PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (mxfp4_write_kernel<T, NB, VEC, false>), grid, block, 0, st, (const T*)k, (const T*)v, (uint8_t*)kc, (uint8_t*)vc, status, a);
  else
    PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (mxfp4_read_kernel<T, NB, VEC>), grid, block, 0, st, (const uint8_t*)kc, (const uint8_t*)vc, (T*)k, (T*)v, a);
}
template <typename T, int NB, int VEC>
void launch_few(bool write, const void* k, const void* v, const void* kc, const void* vc, int32_t* status, const MxRows& a, int Bt, hipStream_t st) {
  const int groups = (a.H_kv + 64 / (4 * NB) - 1) / (64 / (4 * NB)), waves = groups < MX_WAVES ? groups : MX_WAVES;   // of heads
  const dim3 grid((groups + waves - 1) / waves, Bt), block(waves * 64);
  if (write)
    PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (mxfp4_write_few_kernel<T, NB, VEC>), grid, block, 0, st, (const T*)k, (const T*)v, (uint8_t*)kc, (uint8_t*)vc, status, a);
  else
    PHOTON_LAUNCH(KC_MXFP4_CACHE, st, (mxfp4_read_few_kernel<T, NB, VEC>), grid, block, 0, st, (const uint8_t*)kc, (const uint8_t*)vc, (T*)k, (T*)v, a);
}
template <typename T, int NB>
void launch_rows_vec(bool write, const void* k, const void* v, const void* kc, const void* vc, int32_t* status, const MxRows& a, int Bt, hipStream_t st) {
  const int vec = row_vec(k, v, a.row_stride, a.d_h, sizeof(T));
  if (a.T <= MX_FEW) return vec > 1 ? launch_few<T, NB, 4>(write, k, v, kc, vc, status, a, Bt, st) : launch_few<T, NB, 1>(write, k, v, kc, vc, status, a, Bt, st);
  if constexpr (sizeof(T) == 2)
    if (vec == 8) return launch_rows<T, NB, 8>(write, k, v, kc, vc, status, a, Bt, st);
  if (vec == 4) return launch_rows<T, NB, 4>(write, k, v, kc, vc, status, a, Bt, st);
  launch_rows<T, NB, 1>(write, k, v, kc, vc, status, a, Bt, st);
}
template <typename T>
int32_t launch_rows_t(bool write, const void* k, const void* v, const void* kc, const void* vc, int32_t* status, const MxRows& a, int Bt, hipStream_t st) {
  switch (kv_row_elems(a.d_h)) {
    case 32: launch_rows_vec<T, 1>(write, k, v, kc, vc, status, a, Bt, st); break;
    case 64: launch_rows_vec<T, 2>(write, k, v, kc, vc, status, a, Bt, st); break;
    default: launch_rows_vec<T, 4>(write, k, v, kc, vc, status, a, Bt, st); break;
  }
  return check_launch(write ? "mxfp4_write_kernel" : "mxfp4_read_kernel");
}

}  // namespace

extern "C" int32_t photon_mxfp4_tile_bytes(int32_t d_h) {
  const int d_p = photon_kv_row_elems(d_h);
  return d_p == 0 ? 0 : mx_tile_bytes(d_p);
}

namespace photon {

size_t mx_cache_bytes(int Bt, int H_kv, int d_h, int64_t S_max) {
  return (size_t)Bt * H_kv * (size_t)((S_max + MX_TILE - 1) / MX_TILE) * photon_mxfp4_tile_bytes(d_h);
}

int32_t launch_mx_write(const float* k, const float* v, int64_t row_stride, void* kc, void* vc, const int32_t* start, int add, int Bt, int T, int H,
                        int d_h, int64_t S_max, hipStream_t st) {
  MxRows a = mx_rows(start, nullptr, row_stride, T, H, d_h, S_max);
  a.add = add;
  return launch_rows_t<float>(true, k, v, kc, vc, nullptr, a, Bt, st);
}

int32_t launch_mx_attn(const float* q, const void* kc, const void* vc, const int32_t* seq_len, int add, void* out, bool out_bf16, int Bt, int T, int H,
                       int d_h, int64_t S_max, float scale, int n_splits, void* ws, hipStream_t st) {
  MxQueries a;
  a.seq_len = seq_len; a.n_new = nullptr; a.q_stride = (int64_t)H * d_h; a.S_max = S_max;
  a.T = T; a.H = H; a.H_kv = H; a.d_h = d_h; a.group = 1; a.groups = 1; a.n_splits = n_splits; a.add = add; a.out_bf16 = out_bf16;
  a.scale_log2e = scale * LOG2E;
  return mx_launch_attn_t<float>(q, kc, vc, out, ws, a, Bt, st);
}

}  // namespace photon

extern "C" size_t photon_mxfp4_cache_bytes(int32_t Bt, int32_t H_kv, int32_t d_h, int64_t S_max) {
  if (Bt <= 0 || H_kv <= 0 || S_max <= 0) return 0;
  return mx_cache_bytes(Bt, H_kv, d_h, S_max);
}

extern "C" int32_t photon_mxfp4_cache_write(const void* k, const void* v, int64_t row_stride, void* k_cache, void* v_cache, const int32_t* start,
                                            const int32_t* n_new, int32_t* status, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max,
                                            photon_dtype dt, void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const MxRows a = mx_rows(start, n_new, row_stride, T, H_kv, d_h, S_max);
  PHOTON_TRY(rows_args(__func__, k, v, k_cache, v_cache, row_stride, a, dt));
  PHOTON_REQUIRE(!rows_overlap(k_cache, v_cache, 1, INT64_MAX, (int64_t)mx_cache_bytes(Bt, H_kv, d_h, S_max), 1), PHOTON_ERR_INVALID_ARG,
                 "%s: K and V need a cache each: these overlap", __func__);
  return (dt == PHOTON_F32 ? launch_rows_t<float> : launch_rows_t<bf16_t>)(true, k, v, k_cache, v_cache, status, a, Bt, (hipStream_t)stream);
}

extern "C" int32_t photon_mxfp4_cache_read(const void* k_cache, const void* v_cache, const int32_t* start, const int32_t* n_rows, void* k, void* v,
                                           int64_t row_stride, int32_t Bt, int32_t T, int32_t H_kv, int32_t d_h, int64_t S_max, photon_dtype dt,
                                           void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const MxRows a = mx_rows(start, n_rows, row_stride, T, H_kv, d_h, S_max);
  PHOTON_TRY(rows_args(__func__, k, v, k_cache, v_cache, row_stride, a, dt));
  PHOTON_REQUIRE(!rows_overlap(k, v, dtype_size(dt), row_stride, (int64_t)H_kv * d_h, (int64_t)Bt * T), PHOTON_ERR_INVALID_ARG,
                 "%s: k and v overlap", __func__);
  return (dt == PHOTON_F32 ? launch_rows_t<float> : launch_rows_t<bf16_t>)(false, k, v, k_cache, v_cache, nullptr, a, Bt, (hipStream_t)stream);
}

extern "C" size_t photon_mxfp4_decode_attn_workspace_bytes(int32_t Bt, int32_t T, int32_t H, int32_t d_h, int32_t n_splits) {
  if (Bt <= 0 || T <= 0 || H <= 0 || d_h <= 0 || d_h > 128 || n_splits <= 1) return 0;
  return (size_t)Bt * T * H * n_splits * (kv_row_elems(d_h) + 2) * sizeof(float);
}

extern "C" int32_t photon_mxfp4_decode_attn_auto_splits(int32_t Bt, int32_t T, int32_t H, int32_t H_kv, int64_t S_max) {
  if (Bt <= 0 || T <= 0 || H_kv <= 0 || H < H_kv || S_max <= 0) return 1;
  return mx_auto_splits(Bt, T, H, H_kv, S_max, false);       // bf16 rows: the more of the two
}

extern "C" int32_t photon_mxfp4_decode_attn(const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const int32_t* seq_len,
                                            const int32_t* n_new, void* out, int32_t Bt, int32_t T, int32_t H, int32_t H_kv, int32_t d_h,
                                            int64_t S_max, float scale, int32_t n_splits, void* workspace, size_t workspace_bytes, photon_dtype dt,
                                            void* stream) {
  clear_error();
  PHOTON_TRY(check_shape(__func__, Bt, T, H_kv, d_h, S_max, dt));
  PHOTON_REQUIRE(H > 0 && H % H_kv == 0, PHOTON_ERR_INVALID_ARG, "%s: H=%d query heads do not share H_kv=%d evenly", __func__, H, H_kv);
  PHOTON_REQUIRE(n_splits >= 0 && n_splits <= 1024, PHOTON_ERR_INVALID_ARG, "%s: n_splits=%d out of [0, 1024]", __func__, n_splits);
  PHOTON_REQUIRE(Bt <= 65535 && T <= 65535 && H <= 65535, PHOTON_ERR_UNSUPPORTED, "%s: Bt=%d, T=%d, H=%d queries: at most 65535 each", __func__, Bt, T, H);
  if (Bt == 0 || T == 0) return PHOTON_OK;
  const size_t esz = dtype_size(dt);
  PHOTON_REQUIRE(q && out && aligned(q, esz) && aligned(out, esz), PHOTON_ERR_INVALID_ARG, "%s: q and out must be non-null device pointers to whole elements", __func__);
  PHOTON_REQUIRE_PTR(k_cache);
  PHOTON_REQUIRE_PTR(v_cache);
  PHOTON_REQUIRE(seq_len != nullptr, PHOTON_ERR_INVALID_ARG, "%s: seq_len is null", __func__);
  PHOTON_REQUIRE(k_cache != v_cache, PHOTON_ERR_INVALID_ARG, "%s: K and V need a cache each", __func__);
  PHOTON_REQUIRE(((int64_t)T * (H / H_kv) / 4 + 1) * (n_splits > 1 ? n_splits : 1) <= (int64_t)0xffffffff / (MX_ATTN_WAVES * 64) && n_splits <= 1024,
                 PHOTON_ERR_UNSUPPORTED, "%s: T=%d queries of %d heads a K/V head are too many", __func__, T, H / H_kv);
  PHOTON_REQUIRE(q_stride >= (int64_t)H * d_h, PHOTON_ERR_INVALID_ARG, "%s: q_stride=%lld is less than a row of %d heads of %d", __func__,
                 (long long)q_stride, H, d_h);
  if (n_splits == 0) n_splits = mx_auto_splits(Bt, T, H, H_kv, S_max, dt == PHOTON_F32);
  if (n_splits > 1) {
    const size_t need = photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, n_splits);
    PHOTON_REQUIRE(workspace != nullptr && aligned16(workspace) && workspace_bytes >= need, PHOTON_ERR_WORKSPACE,
                   "%s: n_splits=%d needs a 16-byte aligned workspace of %zu bytes (got %zu)", __func__, n_splits, need, workspace_bytes);
  }
  MxQueries a;
  a.seq_len = seq_len; a.n_new = n_new; a.q_stride = q_stride; a.S_max = S_max;
  a.T = T; a.H = H; a.H_kv = H_kv; a.d_h = d_h; a.group = H / H_kv; a.groups = 1; a.n_splits = n_splits; a.add = 0; a.out_bf16 = false;
  a.scale_log2e = scale * LOG2E;
  if (dt == PHOTON_F32) return mx_launch_attn_t<float>(q, k_cache, v_cache, out, workspace, a, Bt, (hipStream_t)stream);
  return mx_launch_attn_t<bf16_t>(q, k_cache, v_cache, out, workspace, a, Bt, (hipStream_t)stream);
}
