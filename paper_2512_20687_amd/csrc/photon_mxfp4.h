// K/V cache in MXFP4 (OCP microscaling: 32 elements of a head's row in E2M1 under one E8M0 scale): layout and launches.
//
// A stream (b, kv head) is a row of tiles of 64 positions; a tile holds its codes, then its scale bytes:
//   K codes   a position's 32 elements of one block are 16 consecutive bytes, element e in nibble e (even ones low); chunks of
//             16 positions of a block are adjacent: the 1024 bytes that a wave loads at once are 64 (position, block) chunks,
//             each of them a lane's operand of the score MFMAs as it is
//   K scales  the byte of every lane's chunks lies at lane * NB + load
//   V codes   8 consecutive positions of one element are 4 consecutive bytes (position p in nibble p): the contraction of the
//             value MFMAs runs over positions, so a lane's operand is again what it loads
//   V scales  position by position, NB bytes each
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/photon.h"

namespace photon {

constexpr int MX_TILE = 64;      // positions of a tile
constexpr int64_t MX_MOST = (1ll << 31) - MX_TILE;   // positions of a stream: the end of its last tile is an int32, too
constexpr int MX_BLOCK = 32;     // elements under one scale
constexpr int MX_LAST_SCALE = 252;   // the writer's largest scale byte: 6 * 2^(252 - 127) is the largest power step that stays finite in fp32; bytes above it read as NaN

__host__ __device__ constexpr int mx_tile_bytes(int d_p) { return MX_TILE * (d_p / 2 + d_p / MX_BLOCK); }
__host__ __device__ constexpr int mx_codes_bytes(int d_p) { return MX_TILE * d_p / 2; }

// Byte offsets inside a tile.  kk: position in the tile.  NB = d_p / 32 blocks of a row.
template <int NB> __device__ __forceinline__ int mx_k_chunk(int kk, int block) { return ((kk >> 4) * NB + block) * 256 + (kk & 15) * 16; }
template <int NB> __device__ __forceinline__ int mx_k_scale(int kk, int block) {
  const int x = (kk >> 4) * NB + block;
  return NB * MX_TILE * 16 + ((x & 3) * 16 + (kk & 15)) * NB + (x >> 2);
}
// The word of positions 8 * (kk >> 3) .. + 7 of one element.
template <int NB> __device__ __forceinline__ int mx_v_word(int kk, int dim) {
  const int w = (kk >> 5) * 2 * NB + (dim >> 4);
  return (w >> 2) * 1024 + (((kk >> 3) & 3) * 16 + (dim & 15)) * 16 + (w & 3) * 4;
}
template <int NB> __device__ __forceinline__ int mx_v_scale(int kk, int block) { return NB * MX_TILE * 16 + kk * NB + block; }

// Launches for the decode step and the prefill: fp32 rows, H_kv = H.
size_t mx_cache_bytes(int Bt, int H_kv, int d_h, int64_t S_max);
// photon_mxfp4_cache_write of rows at positions start[b] + add + t (start NULL: add + t).
int32_t launch_mx_write(const float* k, const float* v, int64_t row_stride, void* kc, void* vc, const int32_t* start, int add, int Bt, int T, int H,
                        int d_h, int64_t S_max, hipStream_t st);
// photon_mxfp4_decode_attn with seq_len[b] + add entries; out_bf16: the fp32 results rounded to bf16.
int32_t launch_mx_attn(const float* q, const void* kc, const void* vc, const int32_t* seq_len, int add, void* out, bool out_bf16, int Bt, int T, int H,
                       int d_h, int64_t S_max, float scale, int n_splits, void* ws, hipStream_t st);
int mx_auto_splits(int Bt, int T, int H, int H_kv, int64_t S_max, bool f32);

}  // namespace photon
