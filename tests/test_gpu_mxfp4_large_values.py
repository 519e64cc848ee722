"""Attention over a 4-bit cache whose V is as large as fp32 values get: the result is a weighted mean of V, and finite where V is.

Bound: fp32 arithmetic on the weights, 1e-5 of sum(p |v|) as for every fp32 kernel here (scores are at most 6 and exact, a weight is
known to a few 2^-24), and half a step of a bf16 result, 2^-8 of it."""
import numpy as np
import pytest
import torch

import mxfp4_layout as lay
from oracle import photon_oracle as po
from util import require_gpu

pytestmark = pytest.mark.gpu

SHAPES = [(1, 2, 2, 64), (1, 2, 2, 32), (1, 3, 3, 100), (2, 4, 2, 64), (4, 2, 2, 128), (4, 4, 2, 64), (1, 8, 1, 128), (5, 2, 1, 32)]
MOST = float(np.finfo(np.float32).max)


def check(ph, K, V, lengths, T, H, dtype, n_splits, junk=None):
    """K, V [Bt, H_kv, n, d_h] as stored; queries that take K's first element as the score."""
    Bt, H_kv, n, d_h = K.shape
    d_p = lay.row_elems(d_h)
    values, caches = [], []
    for x, is_v in ((K, False), (V, True)):
        x = np.pad(x, [(0, 0), (0, 0), (0, -n % 64), (0, d_p - d_h)])
        codes, scales = po.mxfp4_encode(x)
        values.append(po.mxfp4_decode(codes, scales)[..., :d_h])
        if junk is not None:
            for b in range(Bt):
                scales[b, :, lengths[b]:], codes[b, :, lengths[b]:] = junk, 7
        caches.append(torch.from_numpy(lay.pack(codes, scales, is_v)).cuda())
    q = torch.zeros(Bt, T, H, d_h, dtype=dtype)
    q[..., 0] = 1
    out = torch.empty_like(q, device="cuda")
    ws = torch.empty(max(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, n_splits), 16), dtype=torch.uint8, device="cuda")
    ph.photon_mxfp4_decode_attn(q.cuda(), *caches, torch.tensor(lengths, dtype=torch.int32, device="cuda"), out, scale=1.0, n_splits=n_splits, workspace=ws)
    ref, weight = (po.mxfp4_decode_attn(q.float().numpy(), values[0], v, lengths, [T] * Bt, 1.0) for v in (values[1], np.abs(values[1])))
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    bound = 1e-5 * weight + (2.0 ** -8 * np.abs(ref) if dtype == torch.bfloat16 else 0)
    err = np.abs(got - ref)
    assert np.all(err <= bound), np.unravel_index(np.argmax(err - bound), err.shape)


@pytest.fixture(scope="module")
def ph():
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m


def scores(rng, Bt, H_kv, n, d_h, rise):
    K = np.zeros((Bt, H_kv, n, d_h))
    K[..., 0] = rise[np.arange(n) // 64 % len(rise)]
    return K


@pytest.mark.parametrize("n_splits", [1, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,H_kv,d_h", SHAPES)
def test_the_largest_values(ph, dtype, T, H, H_kv, d_h, n_splits):
    """V of both signs at fp32's largest; scores rise by less than 2^8 from tile to tile of a wave, as they may without a new maximum."""
    rng = np.random.default_rng(d_h + T)
    n, Bt = 3200, 2
    rise = np.repeat([0.0, 2.0, 4.0, 6.0], 13)                        # a wave's next tile is 8 (24) further on
    V = rng.choice([-1.0, 1.0], (Bt, H_kv, n, d_h)) * rng.uniform(0.5, 1.0, (Bt, H_kv, n, d_h)) * MOST
    check(ph, scores(rng, Bt, H_kv, n, d_h, rise), V, [n, n - 77], T, H, dtype, n_splits)


@pytest.mark.parametrize("n_splits", [1, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,H_kv,d_h", SHAPES)
def test_equal_scores_of_equal_values(ph, dtype, T, H, H_kv, d_h, n_splits):
    """The mean of thousands of equal values is that value, though their sum is not a number of fp32."""
    V = np.full((2, H_kv, 2500, d_h), MOST)
    check(ph, np.zeros((2, H_kv, 2500, d_h)), V, [2500, 1], T if T == 1 else 1, H, dtype, n_splits)


@pytest.mark.parametrize("n_splits", [1, 2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,H_kv,d_h", SHAPES)
def test_large_values_here_and_there(ph, dtype, T, H, H_kv, d_h, n_splits):
    """Magnitudes from 2^-20 to 2^127 by tile, position and block: some waves meet large values, some late, some never."""
    rng = np.random.default_rng(d_h * T)
    n, Bt = 1900, 2
    at = np.zeros((Bt, H_kv, n, (d_h + 31) // 32, 1))
    at[:, :, 700:710], at[0, :, 1300, 0], at[1, 0, n - 1] = 100, 120, 127
    V = rng.uniform(-1, 1, (Bt, H_kv, n, (d_h + 31) // 32, 32)) * 2.0 ** (at + rng.integers(-20, 1, at.shape))
    V = V.reshape(Bt, H_kv, n, -1)[..., :d_h]
    check(ph, scores(rng, Bt, H_kv, n, d_h, np.array([0.0, 3.0, 1.5, 4.0, 2.0])), V, [n, n], T, H, dtype, n_splits)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,H_kv,d_h", SHAPES)
@pytest.mark.parametrize("junk", [200, 252, 253, 255])
def test_what_nobody_sees_sets_no_unit(ph, dtype, T, H, H_kv, d_h, junk):
    """Large (and NaN) blocks behind the last entry change nothing, for values so small that another unit would lose them."""
    rng = np.random.default_rng(junk)
    V = rng.uniform(0.5, 1, (2, H_kv, 700, d_h)) * 2.0 ** -70
    check(ph, scores(rng, 2, H_kv, 700, d_h, np.array([0.0, 1.0])), V, [641, 70], T, H, dtype, 1, junk)
