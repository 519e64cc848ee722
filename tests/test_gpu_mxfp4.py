"""The 4-bit cache on the GPU: rows quantised and read back bit for bit, attention against the float64 definition.

Tolerances.  Stored values are unique (power-of-two scales, ties to even), so writing and reading compare equal.  Attention with
fp32 rows: 1e-5 of the largest value, the bar of every fp32 kernel here.  With bf16 rows the result is rounded once, half a step
(2^-8 of the value); the fp32 sums add 1e-5 as above.  The 2^-15 * sum(p |v|) that the bounds here add is more than the weights
need, which keep all of their 24 bits: tests/test_gpu_mxfp4_weights.py holds them to that."""
import math

import numpy as np
import pytest
import torch

import mxfp4_layout as lay
from oracle import photon_oracle as po
from util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ph():
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m


def rows(rng, shape, dtype, spread=3):
    """N(0, 1) rows with a magnitude of their own per (row, head), as representable in dtype (float32 numpy)."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-spread, spread + 1, shape[:-1] + (1,))
    t = torch.from_numpy(x.astype(np.float32))
    return t.to(dtype).float().numpy(), t.to(dtype).cuda()


def padded(x, d_p):
    return np.concatenate([x, np.zeros(x.shape[:-1] + (d_p - x.shape[-1],), x.dtype)], -1)


def stored(x):
    """Codes and scale bytes of rows [..., d_h]."""
    return po.mxfp4_encode(padded(x, lay.row_elems(x.shape[-1])))


# ---------------------------------------------------------------- the conversion itself

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_scale_and_every_border(ph, dtype):
    """Blocks of every binade, with the borders between neighbouring values, what lies beside them, and what saturates."""
    near = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.984375], np.float64)
    base = np.concatenate([near, near * (1 - 2.0 ** -7), near * (1 + 2.0 ** -6), [4.0, 0.0]])
    blocks = []
    for e in range(-126, 126):
        for sign in (1, -1):
            blocks.append(sign * base * 2.0 ** e)
    x = np.array(blocks)
    x = x[np.abs(x).max(1) < 3.3e38].astype(np.float32)
    t = torch.from_numpy(x).to(dtype)
    x = t.float().numpy()
    n = x.shape[0] // 4 * 4
    k = t[:n].reshape(1, n // 4, 4, 32).cuda()
    kc, vc = ph.mxfp4_cache(1, 4, 32, n // 4), ph.mxfp4_cache(1, 4, 32, n // 4)
    ph.photon_mxfp4_cache_write(k, -k, kc, vc)
    for cache, is_v, ref in ((kc, False, x), (vc, True, -x)):
        codes, scales = lay.unpack(cache.cpu().numpy(), 32, is_v)
        rc, rs = po.mxfp4_encode(ref[:n].reshape(1, n // 4, 4, 32).transpose(0, 2, 1, 3))
        np.testing.assert_array_equal(scales[:, :, : n // 4], rs)
        np.testing.assert_array_equal(po.mxfp4_decode(codes[:, :, : n // 4], rs), po.mxfp4_decode(rc, rs))
    back = torch.empty_like(k)
    ph.photon_mxfp4_cache_read(kc, vc, back, torch.empty_like(k))
    np.testing.assert_array_equal(back.float().cpu().numpy().reshape(-1, 32), po.mxfp4_round(x[:n]).astype(np.float32))


def test_subnormal_zero_and_unbounded_blocks(ph):
    x = np.zeros((8, 64), np.float32)
    x[0, :4] = [1e-45, 2.0 ** -127, -(2.0 ** -128), 2.0 ** -126]     # below the smallest scale's top binade
    x[1, :3] = [2.0 ** -125, -(2.0 ** -127), 2.0 ** -129]
    x[2, 5], x[2, 40] = np.nan, 1.0
    x[3, 40], x[3, 3] = np.inf, 2.0
    x[4, 63], x[4, 0] = -np.inf, -3.0
    x[5] = np.float32(3.4028235e38)
    x[6, ::2] = -0.0
    for dtype in (torch.float32, torch.bfloat16):
        t = torch.from_numpy(x).to(dtype)
        ref = po.mxfp4_round(t.float().numpy())
        t = t.reshape(1, 8, 1, 64).cuda()
        kc, vc = ph.mxfp4_cache(1, 1, 64, 8), ph.mxfp4_cache(1, 1, 64, 8)
        k, v = torch.empty_like(t), torch.empty_like(t)
        ph.photon_mxfp4_cache_write(t, t, kc, vc)
        ph.photon_mxfp4_cache_read(kc, vc, k, v)
        for got in (k, v):
            np.testing.assert_array_equal(got.float().cpu().numpy().reshape(8, 64), ref.astype(np.float32))


@pytest.mark.parametrize("d_h", [32, 64, 128])
def test_all_bytes_read_back(ph, d_h):
    """Caches of arbitrary bytes: every code under every scale byte."""
    rng = np.random.default_rng(d_h)
    codes = rng.integers(0, 16, (1, 2, 512, d_h)).astype(np.uint8)
    scales = np.arange(2 * 512 * (d_h // 32)).astype(np.uint8).reshape(1, 2, 512, d_h // 32)
    ref = po.mxfp4_decode(codes, np.where(scales > 252, 255, scales)).astype(np.float32).transpose(0, 2, 1, 3)
    kc, vc = (torch.from_numpy(lay.pack(codes, scales, v)).cuda() for v in (False, True))
    k, v = torch.empty(1, 512, 2, d_h, device="cuda"), torch.empty(1, 512, 2, d_h, device="cuda")
    ph.photon_mxfp4_cache_read(kc, vc, k, v)
    np.testing.assert_array_equal(k.cpu().numpy(), ref)
    np.testing.assert_array_equal(v.cpu().numpy(), ref)


# ---------------------------------------------------------------- rows in and out

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Bt,T,H,d_h,start,n_new", [
    (1, 1, 1, 64, [0], None), (1, 1, 2, 52, [63], None), (2, 1, 3, 64, [64, 7], None), (3, 2, 2, 60, [63, 5, 62], [2, 0, 1]),
    (4, 4, 5, 64, [61, 6, 0, 4], None), (3, 4, 3, 128, [5, 126, 60], [4, 3, 4]), (3, 3, 20, 20, [62, 63, 7], None), (2, 4, 17, 100, [7, 64], [1, 4]),
    (5, 2, 9, 52, [63, 7, 8, 0, 70], [2, 2, 2, 0, 1]), (2, 4, 33, 33, [61, 5], None), (2, 5, 3, 64, [60, 4], None), (2, 64, 2, 64, [0, 64], None), (2, 65, 2, 64, [63, 1], None), (2, 66, 1, 128, [63, 0], None), (2, 130, 2, 128, [3, 61], [130, 77]),
    (2, 200, 2, 32, [0, 17], [200, 1]), (2, 77, 3, 20, [55, 100], None), (1, 100, 5, 100, [31], None), (2, 33, 2, 1, [8, 15], None),
    (2, 40, 2, 33, [9, 14], [40, 39]), (1, 300, 2, 56, None, None), (2, 9, 2, 65, [0, 60], [4, 9]), (2, 17, 1, 127, [2, 120], None),
])
def test_write_places_rows_and_leaves_the_rest(ph, dtype, Bt, T, H, d_h, start, n_new):
    rng = np.random.default_rng(T * d_h)
    first, new = start or [0] * Bt, n_new or [T] * Bt
    S = max(a + T for a in first) + 3
    d_p = lay.row_elems(d_h)
    kx, k = rows(rng, (Bt, T, H, d_h), dtype)
    vx, v = rows(rng, (Bt, T, H, d_h), dtype)
    junk = rng.integers(0, 256, (2,) + tuple(ph.mxfp4_cache(Bt, H, d_h, S, device="cpu").shape)).astype(np.uint8)
    kc, vc = torch.from_numpy(junk[0]).cuda(), torch.from_numpy(junk[1]).cuda()
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ph.photon_mxfp4_cache_write(k, v, kc, vc, start=i32(start), n_new=i32(n_new), status=status)
    for cache, x, before, is_v in ((kc, kx, junk[0], False), (vc, vx, junk[1], True)):
        codes, scales = lay.unpack(before, d_p, is_v)
        new_codes, new_scales = stored(x)
        for b in range(Bt):
            at = slice(first[b], first[b] + new[b])
            codes[b, :, at] = new_codes[b, : new[b]].transpose(1, 0, 2)
            scales[b, :, at] = new_scales[b, : new[b]].transpose(1, 0, 2)
        got = lay.unpack(cache.cpu().numpy(), d_p, is_v)
        np.testing.assert_array_equal(got[1], scales)
        same = got[0] == codes                     # a zero's sign is not part of the contract
        assert np.all(same | ((got[0] | codes) == 8))
    assert int(status) == 0
    # and back: rows past n_new stay as they were
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, -7.0)
    ph.photon_mxfp4_cache_read(kc, vc, ko, vo, start=i32(start), n_rows=i32(n_new))
    for got, x, fill in ((ko, kx, 7.0), (vo, vx, -7.0)):
        ref = po.mxfp4_round(x)
        for b in range(Bt):
            ref[b, new[b]:] = fill
        np.testing.assert_array_equal(got.float().cpu().numpy(), ref.astype(np.float32))


@pytest.mark.parametrize("T", [37, 3])
@pytest.mark.parametrize("dtype,H,d_h,offset", [(torch.float32, 2, 64, 0), (torch.bfloat16, 2, 64, 0), (torch.float32, 3, 52, 0), (torch.bfloat16, 1, 52, 0),
                                                (torch.bfloat16, 2, 60, 3), (torch.float32, 2, 64, 1), (torch.bfloat16, 3, 33, 5)])
def test_rows_may_be_parts_of_a_wider_matrix(ph, dtype, H, d_h, offset, T):
    """k and v as columns of a [Bt * T, q | k | v] projection, at any alignment; the columns beside them are not touched."""
    Bt = 2
    rng = np.random.default_rng(5)
    D = H * d_h
    wide, base = rows(rng, (Bt, T, offset + 3 * D + 1), dtype)
    part = lambda t, i: t[..., offset + i * D : offset + (i + 1) * D].unflatten(-1, (H, d_h))  # noqa: E731
    kc, vc = ph.mxfp4_cache(Bt, H, d_h, T), ph.mxfp4_cache(Bt, H, d_h, T)
    ph.photon_mxfp4_cache_write(part(base, 1), part(base, 2), kc, vc)
    out = torch.full_like(base, 3.0)
    ph.photon_mxfp4_cache_read(kc, vc, part(out, 1), part(out, 2))
    ref = np.full(wide.shape, 3.0)
    for i in (1, 2):
        cols = slice(offset + i * D, offset + (i + 1) * D)
        ref[..., cols] = po.mxfp4_round(wide[..., cols].reshape(Bt, T, H, d_h)).reshape(Bt, T, D)
    np.testing.assert_array_equal(out.float().cpu().numpy(), ref.astype(np.float32))


@pytest.mark.parametrize("T", [10, 4])
def test_rows_without_a_place(ph, T):
    """Entries outside the cache are dropped and reported, the others kept; reading leaves such rows alone."""
    Bt, H, d_h, S = 4, 2, 64, 128
    rng = np.random.default_rng(8)
    kx, k = rows(rng, (Bt, T, H, d_h), torch.float32)
    first = [S - 2, -3, S, 2 ** 31 - 5]
    start = torch.tensor(first, dtype=torch.int32, device="cuda")
    kc, vc = ph.mxfp4_cache(Bt, H, d_h, S), ph.mxfp4_cache(Bt, H, d_h, S)
    status = torch.tensor([8], dtype=torch.int32, device="cuda")
    ph.photon_mxfp4_cache_write(k, k, kc, vc, start=start, status=status)
    assert int(status) == 8 | 1
    ph.photon_mxfp4_cache_write(k, k, kc.clone(), vc.clone(), start=start)           # no status word: nothing to report to
    codes, scales = stored(kx)
    for cache, is_v in ((kc, False), (vc, True)):
        got = lay.unpack(cache.cpu().numpy(), d_h, is_v)
        ref_c, ref_s = np.zeros_like(got[0]), np.zeros_like(got[1])
        for b in range(Bt):
            for t in range(T):
                if 0 <= first[b] + t < S:
                    ref_c[b, :, first[b] + t], ref_s[b, :, first[b] + t] = codes[b, t], scales[b, t]
        np.testing.assert_array_equal(got[0], ref_c)
        np.testing.assert_array_equal(got[1], ref_s)
    out = torch.full_like(k, 5.0)
    ph.photon_mxfp4_cache_read(kc, vc, out, torch.empty_like(k), start=start)
    ref = np.full(kx.shape, 5.0, np.float32)
    for b in range(Bt):
        for t in range(T):
            if 0 <= first[b] + t < S:
                ref[b, t] = po.mxfp4_round(kx[b, t])
    np.testing.assert_array_equal(out.cpu().numpy(), ref)


@pytest.mark.parametrize("T", [5, 2])
def test_counts_outside_their_range(ph, T):
    """n_new below 0 and above T count as 0 and T."""
    rng = np.random.default_rng(9)
    kx, k = rows(rng, (2, T, 1, 64), torch.float32)
    kc, vc = ph.mxfp4_cache(2, 1, 64, 64), ph.mxfp4_cache(2, 1, 64, 64)
    ph.photon_mxfp4_cache_write(k, k, kc, vc, n_new=torch.tensor([-2, 99], dtype=torch.int32, device="cuda"))
    codes, _ = lay.unpack(kc.cpu().numpy(), 64, False)
    assert not codes[0].any()
    np.testing.assert_array_equal(codes[1, 0, :T], stored(kx)[0][1, :, 0])
    assert not codes[1, 0, T:].any()


# ---------------------------------------------------------------- attention

def filled(rng, Bt, H_kv, d_h, lengths, S, junk=True):
    """Caches with N(0, 1) entries in the positions in use and arbitrary bytes (NaN scales too) behind them, and their values."""
    d_p, n = lay.row_elems(d_h), (S + 63) // 64 * 64
    values, tensors = [], []
    for is_v in (False, True):
        x = padded(rng.standard_normal((Bt, H_kv, n, d_h)), d_p)
        codes, scales = po.mxfp4_encode(x)
        values.append(po.mxfp4_decode(codes, scales)[..., :d_h])
        if junk:
            for b in range(Bt):
                codes[b, :, lengths[b]:] = rng.integers(0, 16, codes[b, :, lengths[b]:].shape)
                scales[b, :, lengths[b]:] = rng.choice([0, 3, 127, 200, 252, 254, 255], scales[b, :, lengths[b]:].shape)
        tensors.append(torch.from_numpy(lay.pack(codes, scales, is_v)).cuda())
    return values, tensors


def check_attention(ph, rng, Bt, T, H, H_kv, d_h, lengths, dtype, n_new=None, n_splits=0, scale=None, S=None, spread=1.0):
    S = S or max(max(lengths), 1)
    (kx, vx), (kc, vc) = filled(rng, Bt, H_kv, d_h, lengths, S)
    q = torch.from_numpy((rng.standard_normal((Bt, T, H, d_h)) * spread).astype(np.float32)).to(dtype)
    qx, q = q.float().numpy(), q.cuda()
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    splits = n_splits or ph.photon_mxfp4_decode_attn_auto_splits(Bt, T, H, H_kv, kc.shape[2] * 64)
    ws = torch.full((max(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, splits), 16),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((Bt, T, H, d_h), 9.0, dtype=dtype, device="cuda")
    ph.photon_mxfp4_decode_attn(q, kc, vc, i32(lengths), out, n_new=i32(n_new), n_splits=n_splits, workspace=ws, scale=scale)
    new = n_new or [T] * Bt
    sc = scale or 1 / math.sqrt(d_h)
    ref = po.mxfp4_decode_attn(qx, kx, vx, lengths, new, sc)
    got = out.float().cpu().numpy().astype(np.float64)
    for b in range(Bt):
        assert np.all(got[b, new[b]:] == 9.0)                        # rows that no query owns
        got[b, new[b]:] = 0
    assert np.isfinite(got).all()
    if dtype == torch.float32:
        bound = 1e-5 * max(np.abs(ref).max(), 1e-30)
    else:
        weight = po.mxfp4_decode_attn(qx, kx, np.abs(vx), lengths, new, sc)
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * weight + 1e-5 * np.abs(ref).max() + 1e-30
    err = np.abs(got - ref)
    assert np.all(err <= bound), (float((err / bound).max()), np.unravel_index(np.argmax(err / bound), err.shape))
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Bt,T,H,H_kv,d_h,lengths", [
    (1, 1, 1, 1, 64, [1]), (2, 1, 2, 2, 64, [0, 5]), (3, 1, 2, 2, 32, [63, 64, 65]), (2, 1, 2, 2, 128, [127, 130]), (2, 1, 3, 3, 52, [200, 1]),
    (2, 1, 2, 2, 20, [500, 33]), (2, 1, 2, 2, 60, [1000, 511]), (1, 1, 4, 4, 100, [321]), (2, 1, 2, 2, 1, [70, 2]), (1, 1, 2, 2, 127, [65]),
    (2, 1, 4, 2, 64, [100, 900]), (2, 1, 8, 2, 64, [64, 333]), (1, 1, 8, 1, 128, [700]), (2, 1, 6, 2, 32, [129, 64]), (1, 1, 16, 1, 64, [150]), (1, 1, 9, 1, 56, [77]),
    (2, 2, 2, 2, 64, [2, 300]), (2, 3, 2, 1, 52, [3, 130]), (3, 4, 2, 2, 64, [1, 4, 260]), (1, 8, 4, 1, 128, [200]), (2, 5, 4, 4, 32, [64, 68]),
    (1, 17, 2, 2, 64, [100]), (1, 70, 2, 1, 64, [70]),
])
def test_attention_matches_the_definition(ph, dtype, Bt, T, H, H_kv, d_h, lengths):
    check_attention(ph, np.random.default_rng(T * d_h + H), Bt, T, H, H_kv, d_h, lengths, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,H_kv,lengths,n_new", [
    (3, 2, 2, [10, 0, 300, 2], [3, 0, 1, 2]), (4, 4, 2, [70, 1, 64, 65], [4, 1, 2, 3]), (2, 2, 1, [1, 1, 0, 128], [2, 1, 2, 2]), (9, 2, 2, [5, 9, 63, 700], [9, 3, 7, 1]),
])
def test_attention_of_padded_batches(ph, dtype, T, H, H_kv, lengths, n_new):
    """Sequences with fewer new entries than others, with more queries than entries (rows that see nothing), and empty ones."""
    check_attention(ph, np.random.default_rng(T), 4, T, H, H_kv, 64, lengths, dtype, n_new=n_new)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_splits", [1, 2, 3, 7, 40])
@pytest.mark.parametrize("T,H,H_kv,d_h", [(1, 2, 2, 64), (2, 2, 1, 128), (5, 2, 2, 32)])
def test_attention_for_any_number_of_splits(ph, dtype, n_splits, T, H, H_kv, d_h):
    """Splits that hold nothing included."""
    check_attention(ph, np.random.default_rng(n_splits), 3, T, H, H_kv, d_h, [1100, 0, 130], dtype, n_splits=n_splits)


@pytest.mark.parametrize("dtype,spread", [(torch.float32, 0.0), (torch.float32, 8.0), (torch.bfloat16, 0.0), (torch.bfloat16, 8.0), (torch.bfloat16, 30.0)])
def test_attention_of_flat_and_sharp_scores(ph, dtype, spread):
    """Queries of zeros (the mean of the values), and scores up to some hundred, where one entry outweighs the others and the
    maximum rises along the cache.  (fp32 resolves a score of size 100 to a few 1e-6, which is what the weights are then off by.)"""
    check_attention(ph, np.random.default_rng(2), 2, 2, 4, 2, 64, [3000, 777], dtype, spread=spread)


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("order", [1, -1])
def test_scores_that_rise_or_fall_along_the_cache(ph, order, T):
    """Every tile's scores lie far above (below) those of the one before: the reference of the exponentials is raised in each."""
    d_h, n = 64, 1000
    rng = np.random.default_rng(14)
    k = rng.standard_normal((1, n, 1, d_h)) * 0.05
    k[0, ::order, 0, :32] += (np.arange(n) // 64 * 1.5)[:, None] / 32
    v = rng.standard_normal((1, n, 1, d_h))
    kc, vc = ph.mxfp4_cache(1, 1, d_h, n), ph.mxfp4_cache(1, 1, d_h, n)
    k, v = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (k, v))
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    kq, vq = (po.mxfp4_round(a.cpu().numpy()).transpose(0, 2, 1, 3) for a in (k, v))
    for dtype in (torch.float32, torch.bfloat16):
        q = torch.full((1, T, 1, d_h), 8.0, dtype=dtype, device="cuda")
        out = torch.empty_like(q)
        ph.photon_mxfp4_decode_attn(q, kc, vc, torch.tensor([n], dtype=torch.int32, device="cuda"), out, n_splits=1)
        ref = po.mxfp4_decode_attn(q.float().cpu().numpy(), kq, vq, [n], [T], 0.125)
        weight = po.mxfp4_decode_attn(q.float().cpu().numpy(), kq, np.abs(vq), [n], [T], 0.125)
        # fp32 scores of up to 30: known to 30 * 2^-23, which is what the weights are off by; bf16 as above
        bound = 1e-5 * weight if dtype == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * weight + 1e-5 * weight
        assert np.all(np.abs(out.float().cpu().numpy() - ref) <= bound)


def test_two_streams_at_once(ph):
    """Calls on two streams with caches and workspaces of their own do not meet."""
    rng = np.random.default_rng(15)
    sides = []
    for i in range(2):
        _, (kc, vc) = filled(rng, 2, 4, 64, [3000, 1500], 3000)
        q = torch.from_numpy(rng.standard_normal((2, 1, 4, 64)).astype(np.float32)).cuda()
        ws = torch.empty(ph.photon_mxfp4_decode_attn_workspace_bytes(2, 1, 4, 64, 8), dtype=torch.uint8, device="cuda")
        lens = torch.tensor([3000, 1500], dtype=torch.int32, device="cuda")
        want = torch.empty_like(q)
        ph.photon_mxfp4_decode_attn(q, kc, vc, lens, want, n_splits=8, workspace=ws)
        sides.append((torch.cuda.Stream(), q, kc, vc, lens, torch.empty_like(q), ws, want))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, q, kc, vc, lens, out, ws, _ in sides:
            with torch.cuda.stream(stream):
                ph.photon_mxfp4_decode_attn(q, kc, vc, lens, out, n_splits=8, workspace=ws)
    torch.cuda.synchronize()
    for *_, out, _, want in sides:
        assert torch.equal(out, want)


def test_attention_over_a_long_cache(ph):
    check_attention(ph, np.random.default_rng(4), 1, 1, 1, 1, 64, [100003], torch.float32)
    check_attention(ph, np.random.default_rng(4), 1, 3, 4, 1, 128, [40001], torch.bfloat16)


def test_lengths_outside_the_cache(ph):
    """Counts below 0 and above S_max count as 0 and S_max."""
    rng = np.random.default_rng(6)
    (kx, vx), (kc, vc) = filled(rng, 3, 2, 64, [128] * 3, 128)
    q = torch.from_numpy(rng.standard_normal((3, 1, 2, 64)).astype(np.float32)).cuda()
    out = torch.empty_like(q)
    ph.photon_mxfp4_decode_attn(q, kc, vc, torch.tensor([-5, 1000, 128], dtype=torch.int32, device="cuda"), out, n_splits=1)
    ref = po.mxfp4_decode_attn(q.cpu().numpy(), kx, vx, [0, 128, 128], [1] * 3, 0.125)
    assert np.abs(out.cpu().numpy() - ref).max() <= 1e-5 * np.abs(ref).max()


def test_queries_may_be_parts_of_a_wider_matrix(ph):
    rng = np.random.default_rng(7)
    for H, d_h, offset, dtype in ((2, 64, 0, torch.float32), (2, 64, 3, torch.float32), (3, 52, 1, torch.bfloat16), (4, 20, 0, torch.bfloat16)):
        (kx, vx), (kc, vc) = filled(rng, 2, H, d_h, [130, 90], 130)
        wide = torch.from_numpy(rng.standard_normal((2, 3, offset + 3 * H * d_h)).astype(np.float32)).to(dtype).cuda()
        q = wide[..., offset : offset + H * d_h].unflatten(-1, (H, d_h))
        lens = torch.tensor([130, 90], dtype=torch.int32, device="cuda")
        a, b = (torch.empty((2, 3, H, d_h), dtype=dtype, device="cuda") for _ in range(2))
        ph.photon_mxfp4_decode_attn(q, kc, vc, lens, a, n_splits=1)
        ph.photon_mxfp4_decode_attn(q.contiguous(), kc, vc, lens, b, n_splits=1)
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_h", [32, 64, 128])
def test_what_is_not_finite_stays_where_it_is(ph, dtype, d_h):
    """A NaN entry reaches exactly the queries that see it, a NaN query its own row only."""
    Bt, T, H = 2, 3, 2
    rng = np.random.default_rng(11)
    n = 150
    kx, k = rows(rng, (Bt, n, H, d_h), dtype, 0)
    vx, v = rows(rng, (Bt, n, H, d_h), dtype, 0)
    k[0, n - 2, 0, d_h - 1] = float("nan")           # seen by queries 1 and 2 of sequence 0, head 0
    v[1, n - 1, 1, 0] = float("inf")                 # query 2 of sequence 1, head 1: its first block
    kc, vc = ph.mxfp4_cache(Bt, H, d_h, n), ph.mxfp4_cache(Bt, H, d_h, n)
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    q = torch.from_numpy(rng.standard_normal((Bt, T, H, d_h)).astype(np.float32)).to(dtype).cuda()
    lens = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ph.photon_mxfp4_decode_attn(q, kc, vc, lens, out, n_splits=1)
    nan = torch.zeros(out.shape, dtype=torch.bool)
    nan[0, 1:, 0] = True
    nan[1, 2, 1, :32] = True
    assert torch.equal(torch.isnan(out).cpu(), nan)
    q[0, 0, 0, 3] = float("nan")
    again = torch.empty_like(q)
    ph.photon_mxfp4_decode_attn(q, kc, vc, lens, again, n_splits=1)
    assert torch.isnan(again[0, 0, 0]).all()
    keep = ~nan
    keep[0, 0, 0] = False
    assert torch.equal(again.cpu()[keep], out.cpu()[keep])


def test_values_of_very_different_scales(ph):
    """Blocks whose scales span 2^-60 .. 2^60 in V and 2^-40 .. 1 in K: no product leaves the range on the way."""
    rng = np.random.default_rng(12)
    Bt, H, d_h, n = 1, 2, 64, 300
    k = torch.from_numpy((rng.standard_normal((Bt, n, H, d_h)) * 2.0 ** rng.integers(-40, 1, (Bt, n, H, 1))).astype(np.float32)).cuda()
    v = torch.from_numpy((rng.standard_normal((Bt, n, H, 2, 32)) * 2.0 ** rng.integers(-60, 61, (Bt, n, H, 2, 1))).astype(np.float32)).cuda().reshape(Bt, n, H, d_h)
    kc, vc = ph.mxfp4_cache(Bt, H, d_h, n), ph.mxfp4_cache(Bt, H, d_h, n)
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    q = torch.from_numpy(rng.standard_normal((Bt, 1, H, d_h)).astype(np.float32)).cuda()
    out = torch.empty_like(q)
    ph.photon_mxfp4_decode_attn(q, kc, vc, torch.tensor([n], dtype=torch.int32, device="cuda"), out, n_splits=1)
    kq, vq = (po.mxfp4_round(t.cpu().numpy()).transpose(0, 2, 1, 3) for t in (k, v))
    ref = po.mxfp4_decode_attn(q.cpu().numpy(), kq, vq, [n], [1], 0.125)
    weight = po.mxfp4_decode_attn(q.cpu().numpy(), kq, np.abs(vq), [n], [1], 0.125)
    assert np.all(np.abs(out.cpu().numpy() - ref) <= 1e-5 * weight)


# ---------------------------------------------------------------- as they are used together

def test_decoding_with_the_cache(ph):
    """A ragged prompt, then steps of one and of three new entries, every one written and attended over; the same rows through the
    oracle.  The cache that was read back continues the same way."""
    Bt, H, H_kv, d_h, S = 3, 4, 2, 52, 256
    rng = np.random.default_rng(21)
    kc, vc = ph.mxfp4_cache(Bt, H_kv, d_h, S), ph.mxfp4_cache(Bt, H_kv, d_h, S)
    kx, vx = np.zeros((2, Bt, H_kv, S, d_h))
    lengths = torch.zeros(Bt, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for step, new in enumerate(([100, 1, 63], [1, 1, 1], [1, 0, 1], [3, 2, 1], [1, 1, 1])):
        T = max(new)
        k0, k = rows(rng, (Bt, T, H_kv, d_h), torch.float32, 0)
        v0, v = rows(rng, (Bt, T, H_kv, d_h), torch.float32, 0)
        q0, q = rows(rng, (Bt, T, H, d_h), torch.float32, 0)
        n_new = torch.tensor(new, dtype=torch.int32, device="cuda")
        ph.photon_mxfp4_cache_write(k, v, kc, vc, start=lengths, n_new=n_new, status=status)
        for b, (n, m) in enumerate(zip(lengths.tolist(), new)):
            kx[b, :, n : n + m] = po.mxfp4_round(k0[b, :m]).transpose(1, 0, 2)
            vx[b, :, n : n + m] = po.mxfp4_round(v0[b, :m]).transpose(1, 0, 2)
        lengths += n_new
        out = torch.zeros_like(q)
        ph.photon_mxfp4_decode_attn(q, kc, vc, lengths, out, n_new=n_new, n_splits=1)
        ref = po.mxfp4_decode_attn(q0, kx, vx, lengths.tolist(), new, 1 / math.sqrt(d_h))
        assert np.abs(out.cpu().numpy() - ref).max() <= 1e-5 * np.abs(ref).max(), step
    assert int(status) == 0
    n = int(lengths.max())
    k, v = torch.zeros(Bt, n, H_kv, d_h, device="cuda"), torch.zeros(Bt, n, H_kv, d_h, device="cuda")
    ph.photon_mxfp4_cache_read(kc, vc, k, v, n_rows=lengths)
    np.testing.assert_array_equal(k.cpu().numpy().transpose(0, 2, 1, 3), kx[:, :, :n].astype(np.float32))
    k2, v2 = ph.mxfp4_cache(Bt, H_kv, d_h, S), ph.mxfp4_cache(Bt, H_kv, d_h, S)
    ph.photon_mxfp4_cache_write(k, v, k2, v2, n_new=lengths)         # stored values are stored again as they are
    again = torch.zeros_like(out)
    ph.photon_mxfp4_decode_attn(q, k2, v2, lengths, again, n_new=n_new, n_splits=1)
    assert torch.equal(out, again)


def test_a_captured_step_replays(ph):
    """Append, attend and count on as one graph, on a stream of its own, replayed with other work between; then eagerly."""
    Bt, H, d_h, S, steps = 2, 3, 64, 700, 5
    rng = np.random.default_rng(22)
    lens0 = [600, 63]
    _, (kc0, vc0) = filled(rng, Bt, H, d_h, lens0, S)
    data = torch.from_numpy(rng.standard_normal((steps, 3, Bt, 1, H, d_h)).astype(np.float32)).cuda()
    n = ph.photon_mxfp4_decode_attn_auto_splits(Bt, 1, H, H, kc0.shape[2] * 64)
    n = max(n, 2)                                                    # partial results through the workspace
    ws = torch.empty(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, 1, H, d_h, n), dtype=torch.uint8, device="cuda")
    now, out = torch.empty_like(data[0]), torch.empty_like(data[0, 0])
    lens = torch.tensor(lens0, dtype=torch.int32, device="cuda")
    kc, vc = kc0.clone(), vc0.clone()

    def step():
        ph.photon_mxfp4_cache_write(now[1], now[2], kc, vc, start=lens)
        lens.add_(1)
        ph.photon_mxfp4_decode_attn(now[0], kc, vc, lens, out, n_splits=n, workspace=ws)

    now.copy_(data[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    got = []
    for run in range(2):
        lens.copy_(torch.tensor(lens0, dtype=torch.int32))
        kc.copy_(kc0)
        vc.copy_(vc0)
        outs = []
        for i in range(steps):
            now.copy_(data[i])
            if run == 0:
                graph.replay()
                torch.cuda.synchronize()
                ws.fill_(255)                                        # the workspace's contents are nobody's to keep
            else:
                step()
            outs.append(out.clone())
        got.append(torch.stack(outs))
        assert lens.tolist() == [a + steps for a in lens0]
    assert torch.equal(got[0], got[1])


def test_results_repeat_bit_for_bit(ph):
    rng = np.random.default_rng(23)
    _, (kc, vc) = filled(rng, 2, 4, 64, [3000, 2000], 3000)
    q = torch.from_numpy(rng.standard_normal((2, 4, 4, 64)).astype(np.float32)).cuda()
    lens = torch.tensor([3000, 2000], dtype=torch.int32, device="cuda")
    ws = torch.empty(ph.photon_mxfp4_decode_attn_workspace_bytes(2, 4, 4, 64, 6), dtype=torch.uint8, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    for out in (a, b):
        ph.photon_mxfp4_decode_attn(q, kc, vc, lens, out, n_splits=6, workspace=ws)
    assert torch.equal(a, b)


def test_offsets_past_32_bits(ph):
    """A cache of more than 4 GiB: the last sequence's entries are written, read and attended over where they belong."""
    Bt, H, d_h, S = 2, 1, 128, 64 * 520000
    tiles = S // 64
    kc = torch.zeros((Bt, H, tiles, 4352), dtype=torch.uint8, device="cuda")
    vc = torch.zeros_like(kc)
    assert kc.numel() > 1 << 32
    n = 200
    first = S - n
    rng = np.random.default_rng(24)
    kx, k = rows(rng, (Bt, n, H, d_h), torch.bfloat16, 0)
    vx, v = rows(rng, (Bt, n, H, d_h), torch.bfloat16, 0)
    start = torch.tensor([0, first], dtype=torch.int32, device="cuda")
    ph.photon_mxfp4_cache_write(k, v, kc, vc, start=start)
    assert int(kc[1, 0, -4:].count_nonzero()) > 0 and int(kc[1, 0, :-4].count_nonzero()) == 0
    a, b = torch.empty_like(k), torch.empty_like(v)
    ph.photon_mxfp4_cache_read(kc, vc, a, b, start=start)
    np.testing.assert_array_equal(a.float().cpu().numpy(), po.mxfp4_round(kx).astype(np.float32))
    np.testing.assert_array_equal(b.float().cpu().numpy(), po.mxfp4_round(vx).astype(np.float32))
    # the entries before them are zeros: scores 0, values 0; a query along one entry weighs that entry against S - 1 others
    q = torch.zeros(Bt, 1, H, d_h, device="cuda")
    q[1, 0, 0] = torch.from_numpy(po.mxfp4_round(kx)[1, -1, 0]).float().cuda()
    out = torch.empty_like(q)
    lens = torch.tensor([n, S], dtype=torch.int32, device="cuda")
    splits = ph.photon_mxfp4_decode_attn_auto_splits(Bt, 1, H, H, S)
    ws = torch.empty(max(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, 1, H, d_h, splits), 16), dtype=torch.uint8, device="cuda")
    ph.photon_mxfp4_decode_attn(q, kc, vc, lens, out, scale=0.25, workspace=ws)
    K, V = po.mxfp4_round(kx)[:, :, 0], po.mxfp4_round(vx)[:, :, 0]
    np.testing.assert_allclose(out[0, 0, 0].cpu().numpy(), V[0].mean(0), rtol=0, atol=1e-5 * np.abs(V[0].mean(0)).max())
    p = np.exp(0.25 * K[1] @ K[1, -1])
    ref = p @ V[1] / (p.sum() + first)
    assert np.abs(out[1, 0, 0].cpu().numpy() - ref).max() <= 1e-5 * np.abs(ref).max()


@pytest.mark.parametrize("dtype,T,n_splits,n", [(torch.float32, 1, 1, 1), (torch.float32, 1, 3, 700), (torch.float32, 4, 1, 70), (torch.float32, 4, 2, 900),
                                                (torch.bfloat16, 1, 1, 64), (torch.bfloat16, 4, 1, 70), (torch.bfloat16, 8, 2, 700), (torch.bfloat16, 8, 1, 8)])
def test_scores_near_the_lowest_number(ph, dtype, T, n_splits, n):
    """Every score about -1e37: equal keys weigh the same, and a key that is half as far away takes all of the weight."""
    rng = np.random.default_rng(n)
    H, d_h = 2, 64
    K = np.full((2, 1, H, n, d_h), -(2.0 ** 60))
    K[1, 0, :, 0] = -(2.0 ** 59)
    V = rng.standard_normal((2, 1, H, n, d_h))
    caches, values = [], []
    for x, is_v in ((K, False), (V, True)):
        x = np.concatenate([x.reshape(2, H, n, d_h), np.zeros((2, H, -n % 64, d_h))], 2)
        codes, scales = po.mxfp4_encode(x)
        values.append(po.mxfp4_decode(codes, scales))
        caches.append(torch.from_numpy(lay.pack(codes, scales, is_v)).cuda())
    q = torch.full((2, T, H, d_h), 2.0 ** 60, dtype=dtype, device="cuda")
    lens = torch.full((2,), n, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(max(ph.photon_mxfp4_decode_attn_workspace_bytes(2, T, H, d_h, n_splits), 16), dtype=torch.uint8, device="cuda")
    ph.photon_mxfp4_decode_attn(q, *caches, lens, out, n_splits=n_splits, workspace=ws, scale=0.125)
    got = out.double().cpu().numpy()
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0                # a bf16 result's rounding; 2^-15: of a weight, as above
    weight = 2.0 ** -15 if dtype == torch.bfloat16 else 0.0
    for t in range(T):
        seen = n - T + t + 1
        v = values[1][:, :, :seen]
        ref = np.stack([v[0].mean(1), v[1][:, 0]])
        bound = half * np.abs(ref) + weight * np.stack([np.abs(v[0]).mean(1), np.abs(ref[1])]) + 1e-5 * np.abs(ref).max()
        assert np.all(np.abs(got[:, t] - ref) <= bound), t
