"""Rows that a 4-bit cache is read back into, and the caches that rows are written to, may lie beside each other but not share memory."""
import ctypes
import os

import numpy as np
import pytest
import torch

from util import require_gpu

P = 1 << 22                          # an address that is never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    import paper_2512_20687_amd as ph
    if not os.path.exists(ph.lib_path()):
        from paper_2512_20687_amd import build
        build.build(verbose=False)
    return ph.load_library()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("stride,apart", [
    (128, 1), (128, 127), (128, 128), (128, 128 * 5), (128, 128 * 6 - 1),    # rows without gaps: 6 rows of 128
    (384, 127), (384, 384 - 127), (384, 384 + 1), (384, 384 * 5 + 127), (384, 384 * 5 - 127), (200, 73), (200, 200 * 3 - 100),
])
def test_rows_that_share_memory_are_refused(lib, dt, stride, apart):
    esz = 2 if dt else 4
    for sign in (1, -1):
        rc = lib.photon_mxfp4_cache_read(P * 4, P * 8, None, None, P, P + sign * apart * esz, stride, 2, 3, 2, 64, 100, dt, None)
        assert rc == -1 and b"k and v overlap" in lib.photon_last_error()


@pytest.mark.parametrize("apart", [16, 2 * 2 * 2176 - 16])
def test_caches_that_share_memory_are_refused(lib, apart):
    size = lib.photon_mxfp4_cache_bytes(1, 2, 64, 100)
    assert size == 2 * 2 * 2176
    for sign in (1, -1):
        rc = lib.photon_mxfp4_cache_write(P * 4, P * 4, 128, P, P + sign * apart, None, None, None, 1, 3, 2, 64, 100, 0, None)
        assert rc == -1 and b"a cache each" in lib.photon_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_and_caches_may_touch(dtype, T):
    """K and V as columns of one matrix, as its alternate rows, and one behind the other; two caches in one piece of memory."""
    require_gpu()
    import paper_2512_20687_amd as ph
    Bt, H, d_h = 2, 2, 64
    rng = np.random.default_rng(T)
    size = ph.photon_mxfp4_cache_bytes(Bt, H, d_h, T)
    kc, vc = torch.zeros(2 * size, dtype=torch.uint8, device="cuda").view(2, Bt, H, -1, ph.photon_mxfp4_tile_bytes(d_h))
    k, v = (torch.from_numpy(rng.standard_normal((Bt, T, H, d_h)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    want = torch.empty_like(k), torch.empty_like(v)
    ph.photon_mxfp4_cache_read(kc, vc, *want)
    D = H * d_h
    behind = torch.zeros(2, Bt, T, D, dtype=dtype, device="cuda")
    columns = torch.zeros(Bt, T, 2, D, dtype=dtype, device="cuda")
    for a, b in ((behind[0], behind[1]), (columns[:, :, 0], columns[:, :, 1])):
        for x, y in ((a, b), (b, a)):
            x, y = x.unflatten(-1, (H, d_h)), y.unflatten(-1, (H, d_h))
            ph.photon_mxfp4_cache_read(kc, vc, x, y)
            assert torch.equal(x, want[0]) and torch.equal(y, want[1])
