"""The MXFP4 cache layout, byte by byte as include/photon.h states it (shared by the tests of the 4-bit cache)."""
import numpy as np

TILE = 64


def row_elems(d_h):
    return 32 if d_h <= 32 else 64 if d_h <= 64 else 128


def addresses(d_p, is_v):
    """(byte, shift) of the code [64, d_p] and byte of the scale [64, d_p / 32] of a tile's positions."""
    nb = d_p // 32
    kk, d, b = np.arange(TILE)[:, None], np.arange(d_p)[None], np.arange(nb)[None]
    if is_v:
        w = kk // 32 * 2 * nb + d // 16
        at = w // 4 * 1024 + (kk % 32 // 8 * 16 + d % 16) * 16 + w % 4 * 4 + kk % 8 // 2
        return at, 4 * (kk % 2) + 0 * d, 32 * d_p + kk * nb + b
    at = (kk // 16 * nb + d // 32) * 256 + kk % 16 * 16 + d % 32 // 2
    x = kk // 16 * nb + b
    return at, 4 * (d % 2) + 0 * kk, 32 * d_p + (x % 4 * 16 + kk % 16) * nb + x // 4


def unpack(cache, d_p, is_v):
    """Cache bytes [..., tiles, tile bytes] -> codes [..., positions, d_p], scale bytes [..., positions, d_p / 32]."""
    at, shift, scale = addresses(d_p, is_v)
    code = cache[..., at] >> shift & 15
    return code.reshape(cache.shape[:-2] + (-1, d_p)).astype(np.uint8), cache[..., scale].reshape(cache.shape[:-2] + (-1, d_p // 32))


def pack(codes, scales, is_v):
    """Inverse of unpack."""
    d_p = codes.shape[-1]
    at, shift, scale = addresses(d_p, is_v)
    lead, n = codes.shape[:-2], codes.shape[-2] // TILE
    out = np.zeros(lead + (n, TILE * (d_p // 2 + d_p // 32)), np.uint8)
    c = codes.reshape(lead + (n, TILE, d_p))
    for s in (0, 4):
        sel = shift == s
        out[..., at[sel]] |= c[..., sel] << s
    out[..., scale] = scales.reshape(lead + (n, TILE, d_p // 32))
    return out
