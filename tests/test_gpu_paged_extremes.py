"""The paged attention at the ends of fp32: values and scores as large as it holds, and infinities.

Tolerances as in tests/test_gpu_paged_attn.py: relative to A = sum(p |v|), whatever its size."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from test_gpu_paged_attn import BAD_PAGE, KV, check, filled, i32, i64, trees
from test_gpu_paged_wide import Many
from util import require_gpu

pytestmark = pytest.mark.gpu
TYPES = [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.float32, "f32"), (torch.bfloat16, "f32")]
P, D_H, PAST = 32, 64, 250


@pytest.fixture(scope="module", params=["few streams", "many streams"])
def ph(request):
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m if request.param == "few streams" else Many(m, 64)


def pages_of(x, kv):
    """Entries [n, d_h] of one head as a pool, entry s in row s % P of page s / P."""
    pool = torch.zeros((-(-x.shape[0] // P), 1, P, D_H))
    pool.view(-1, D_H)[: x.shape[0]] = torch.as_tensor(x)
    return pool.to(KV[kv])


def run(ph, rows, kv, q, k, v, splits, scale=None):
    """out [T, H, d_h] in float64, and what the kernel was given: q, pools, table."""
    pools = [pages_of(x, kv) for x in (k, v)]
    table = np.arange(pools[0].shape[0], dtype=np.int32)[None]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), D_H)
    q = torch.as_tensor(q, dtype=torch.float32).to(rows)[None].cuda()
    out = torch.full_like(q, 5.0)
    ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 1, q.shape[1], q.shape[2], None, splits) + 16, dtype=torch.uint8, device="cuda")
    ph.photon_paged_attn(q, cache, i32([k.shape[0]]), out, n_splits=splits, workspace=ws, scale=scale)
    return out, q, pools, table


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 20, 40])
@pytest.mark.parametrize("at", [3, 35, 130, 249])
def test_a_large_value_under_a_score_that_rises(ph, rows, kv, T, at):
    """One entry is ahead of all others by so many powers of two in weight, and its V is 2^126, all others' 0: a row's result is 2^126
    times the entry's share, wherever the reference of the others' weights was."""
    k, v = np.zeros((PAST + T, D_H), np.float32), np.zeros((PAST + T, D_H), np.float32)
    k[at, 0] = 1
    v[at] = 2.0 ** 126
    every = [0.0, 0.5, 2.9, 5.0, 7.2, 7.9, 8.1, 15.9, 120.0]
    for rises in [[rise] for rise in every] + [every]:                # alone, and side by side: a wave's rows raise theirs together
        q = np.zeros((T, len(rises), D_H), np.float32)
        q[..., 0] = np.array(rises) * np.log(2.0)
        for splits in (1, 2):
            out, given, pools, table = run(ph, rows, kv, q, k, v, splits, scale=1.0)
            check(out, given, pools, table, [PAST + T], [T], D_H, scale=1.0)


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 40])
def test_values_that_add_up_to_the_largest(ph, rows, kv, T):
    """Scores that rise by up to 2^8 in weight from step to step, and V of up to 2^119.5: the sum over 290 entries stays below 2^128."""
    rng = np.random.default_rng(T)
    k = np.zeros((PAST + T, D_H), np.float32)
    k[:, 0] = np.arange(PAST + T) // 32 + rng.uniform(0, 1, PAST + T)
    v = (rng.uniform(0.5, 1.0, (PAST + T, D_H)) * np.where(rng.uniform(size=D_H) < 0.5, -1, 1) * 2.0 ** 119.5).astype(np.float32)
    for slopes in ([1.0], [3.0], [5.0], [5.4], [-5.4], [0.0, 1.0, 5.0, -5.4]):
        q = np.zeros((T, len(slopes), D_H), np.float32)
        q[..., 0] = np.array(slopes)
        for splits in (1, 3):
            out, given, pools, table = run(ph, rows, kv, q, k, v, splits, scale=1.0)
            check(out, given, pools, table, [PAST + T], [T], D_H, scale=1.0)


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("exponent", [-60, -100, -112])
def test_small_values(ph, rows, kv, T, exponent):
    """V of about 2^-112: as exact as elsewhere."""
    rng = np.random.default_rng(T)
    k, v = (rng.standard_normal((PAST + T, D_H)).astype(np.float32) for _ in range(2))
    q = rng.standard_normal((T, 4, D_H)).astype(np.float32)
    out, given, pools, table = run(ph, rows, kv, q, k, v * np.float32(2.0 ** exponent), 1)
    x = torch.ldexp(out.float(), torch.tensor(-exponent, device="cuda")).to(out.dtype)
    check(x, given, [pools[0], torch.ldexp(pools[1].float(), torch.tensor(-exponent)).to(pools[1].dtype)], table, [PAST + T], [T], D_H)


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T,past", [(1, 0), (1, 7), (40, 0), (1, 250), (20, 250), (40, 250)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_scores_at_the_end_of_fp32(ph, rows, kv, T, past, sign, scale):
    """Scores of 2.9e38 to 3.3e38 of either sign, in any order: finite in fp32, though not times log2 e.  The largest that a row sees takes
    all; neighbours are 2^-7 of it apart."""
    rng = np.random.default_rng(past + T)
    n = past + T
    k = np.zeros((n, D_H), np.float32)
    k[:, 0] = (1 + rng.permutation(n) % 16 / 128.0) * 2.0 ** 60
    v = rng.standard_normal((n, D_H)).astype(np.float32)
    q = np.zeros((T, 2, D_H), np.float32)
    q[..., 0] = sign * 2.9e38 / 2.0 ** 60 / scale
    for splits in (1, 2):
        out, given, pools, table = run(ph, rows, kv, q, k, v, splits, scale=scale)
        check(out, given, pools, table, [n], [T], D_H, scale=scale)


def with_unbounded(k, v, see, x, scale):
    """Row x [H, d_h]'s result where V has infinities and NaN: by their definition; elsewhere the finite one."""
    ref, size = plain.attended(x, k, np.where(np.isfinite(v), v, 0.0), see, scale)
    bad = np.where(np.isfinite(v[0][see]), 0.0, v[0][see])
    with np.errstate(invalid="ignore"):
        return ref + bad.sum(0), size


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("slope", [0.0, 1.0, 5.0, -5.0])
def test_infinities_in_values(ph, rows, kv, T, slope):
    """Infinities and NaN in V anywhere: what a row sees is in its result, with its sign, be its weight 1, 2^-80 or too small for fp32."""
    rng = np.random.default_rng(T)
    n = PAST + T
    k, v = np.zeros((n, D_H), np.float32), rng.standard_normal((n, D_H)).astype(np.float32)
    k[:, 0] = np.arange(n) // 4 * 4 / 32.0
    k[:, 1:] = 0.25 * rng.standard_normal((n, D_H - 1))
    q = rng.standard_normal((T, 3, D_H)).astype(np.float32)
    q[..., 0] = slope
    inf, nan = np.inf, np.nan
    for e, d, x in ((0, 0, inf), (7, 1, -inf), (8, 5, inf), (140, 5, inf), (20, 33, inf), (240, 33, -inf), (130, 40, nan), (131, 62, nan), (9, 62, inf),
                    (PAST - 1, 63, -inf), (n - 1, 17, inf), (PAST + T // 2, 18, -inf), (100, 24, inf), (101, 25, -inf), (199, 31, inf)):
        v[e, d] = x
    for splits in (1, 2, 12):
        out, given, pools, table = run(ph, rows, kv, q, k, v, splits)
        ks, vs = (plain.entries(plain.values(p), table[0], n, D_H) for p in pools)
        got, x = out[0].float().cpu().numpy().astype(np.float64), given[0].float().cpu().numpy()
        for t in range(T):
            ref, size = with_unbounded(ks, vs, plain.seen(n, T, t), x[t], D_H ** -0.5)
            fine = np.isfinite(ref)
            np.testing.assert_array_equal(np.where(fine, 0.0, got[t]), np.where(fine, 0.0, ref), err_msg=str((splits, t)))
            bound = 1e-5 * size.max() if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
            assert (np.abs(got[t][fine] - ref[fine]) <= np.broadcast_to(bound, ref.shape)[fine]).all(), (splits, t)


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("at", [0, 40, 130, 249, 250])
def test_infinities_in_keys(ph, rows, kv, T, at):
    """K of infinity: a query whose element there is negative does not see the entry, a positive one has no finite result.  Elements of few
    digits, whose lower parts are 0, and of many."""
    rng = np.random.default_rng(T)
    n = PAST + T
    k, v = (rng.standard_normal((n, D_H)).astype(np.float32) for _ in range(2))
    k[at, 7] = np.inf
    q = rng.standard_normal((T, 6, D_H)).astype(np.float32)
    q[..., 7] = [-1.0, -1.2345678, 1.0, 2.0 ** -60, -(2.0 ** -60), 0.0]
    for splits in (1, 2):
        out, given, pools, table = run(ph, rows, kv, q, k, v, splits)
        ks, vs = (plain.entries(plain.values(p), table[0], n, D_H) for p in pools)
        got, x = out[0].float().cpu().numpy().astype(np.float64), given[0].float().cpu().numpy()
        for t in range(T):
            with np.errstate(invalid="ignore"):
                ref, size = plain.attended(x[t], ks, vs, plain.seen(n, T, t), D_H ** -0.5)
            fine = ~np.isnan(ref)
            assert (fine.all(1) == [True, True, at > PAST + t, at > PAST + t, True, at > PAST + t]).all()
            assert np.isnan(got[t][~fine]).all()
            bound = 1e-5 * size[fine].max() if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
            assert (np.abs(got[t][fine] - ref[fine]) <= np.broadcast_to(bound, ref.shape)[fine]).all(), (splits, t)


def test_sums_that_are_too_large_stay_infinite(ph):
    """Nothing infinite in V, but a sum that fp32 does not hold: what the sum became, not a smaller number."""
    for rows, kv in TYPES:
        for T in (1, 40):
            n = PAST + T
            k, v = np.zeros((n, D_H), np.float32), np.full((n, D_H), 2.0 ** 127, np.float32)
            v[:, 1::2] = -v[:, 1::2]
            out = run(ph, rows, kv, np.zeros((T, 2, D_H)), k, v, 1)[0].float()
            assert not (out.abs() < 2.0 ** 126).any()


@pytest.mark.parametrize("rows,kv", TYPES)
@pytest.mark.parametrize("T", [1, 40])
def test_a_scale_at_the_end_of_fp32(ph, rows, kv, T):
    """scale = 3e38, whose product with log2 e is not finite, over scores of up to about 1."""
    n = PAST + T
    rng = np.random.default_rng(T)
    k, v = np.zeros((n, D_H), np.float32), rng.standard_normal((n, D_H)).astype(np.float32)
    k[:, 0] = rng.integers(-16, 17, n) / 16.0
    q = np.zeros((T, 2, D_H), np.float32)
    q[..., 0] = 2.0 ** -120
    q[:, 1, 0] = 0.0
    out, given, pools, table = run(ph, rows, kv, q, k, v, 1, scale=3e38)
    check(out, given, pools, table, [n], [T], D_H, scale=float(np.float32(3e38)))


@pytest.mark.parametrize("rows,kv", TYPES + [(torch.bfloat16, "e4m3"), (torch.float32, "e4m3")])
@pytest.mark.parametrize("T,H,H_kv", [(1, 2, 2), (1, 10, 1), (12, 4, 2), (40, 2, 1)])
def test_infinities_in_pages_trees_and_heads(ph, rows, kv, T, H, H_kv):
    """Several sequences and K/V heads, pages that are not there, a tree: what a row sees, of its own head, decides.  Unused places hold NaN."""
    rng = np.random.default_rng(10 * T + H)
    lengths = [170 + T, 90 + T, T]
    table, n_pages = plain.table_of(rng, lengths, P)
    pools = [filled(rng, n_pages, H_kv, D_H, P, kv, table, lengths) for _ in range(2)]
    for p in pools:
        p[table[0, 1]] = 255 if kv == "e4m3" else float("nan")                  # the page that goes
    wrong = table.copy()
    wrong[0, 1], wrong[1, 1] = n_pages + 3, -7
    e4m3 = kv == "e4m3"
    for b, e, h, d, x in ((0, 3, 0, 1, "inf"), (0, 100, 0, 5, "-inf"), (0, 101, H_kv - 1, 5, "inf"), (0, 160, 0, 63, "nan"), (0, 169 + T, 0, 8, "inf"), (1, 10, H_kv - 1, 9, "-inf"),
                          (1, 70, 0, 20, "inf"), (1, 89 + (T + 1) // 2, 0, 21, "-inf"), (2, T - 1, 0, 40, "inf"), (2, 0, H_kv - 1, 41, "nan")):
        pools[1][table[b, e // P], h, e % P, d] = 255 if e4m3 else float(x)
    masks = trees(rng, 3, T) if T > 1 else None
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(wrong), D_H)
    q = torch.from_numpy(rng.standard_normal((3, T, H, D_H)).astype(np.float32)).to(rows)
    values = [plain.values(p) for p in pools]
    for splits in (1, 3):
        out, status = torch.empty_like(q, device="cuda"), i32([0])
        ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 3, T, H, None, splits) + 16, dtype=torch.uint8, device="cuda")
        ph.photon_paged_attn(q.cuda(), cache, i32(lengths), out, tree=i64(masks), n_splits=splits, workspace=ws, status=status)
        assert int(status) == BAD_PAGE
        got = out.float().cpu().numpy().astype(np.float64)
        for b, n in enumerate(lengths):
            ks, vs = (plain.entries(p, table[b], n, D_H) for p in values)
            there = np.array([0 <= wrong[b, e // P] < n_pages for e in range(n)])
            for t in range(T):
                see = plain.seen(n, T, t, None if masks is None else masks[b, t]) & there
                x = q[b, t].float().numpy()
                for h in range(H):
                    kk, vv = (a[h // (H // H_kv)][None] for a in (ks, vs))
                    ref, size = with_unbounded(kk, vv, see, x[h : h + 1], D_H ** -0.5)
                    fine = np.isfinite(ref[0])
                    np.testing.assert_array_equal(np.where(fine, 0.0, got[b, t, h]), np.where(fine, 0.0, ref[0]), err_msg=str((splits, b, t, h)))
                    bound = 1e-5 * size.max() if rows == torch.float32 else 2.0 ** -8 * np.abs(ref[0]) + 2.0 ** -15 * size[0]
                    assert (np.abs(got[b, t, h][fine] - ref[0][fine]) <= np.broadcast_to(bound, ref[0].shape)[fine]).all(), (splits, b, t, h)
