"""Appending to the paged K/V cache with rotation, and moving entries within it, against the float64 definitions.

Tolerances.  V, and K without rotation, are stored as one rounding of the row: equal to torch's, bit for bit.  A rotated value is
fp32 arithmetic on fp32 cosines, |error| <= 5 * 2^-24 * (|a| + |b|) for the pair (a, b) (cosine and sine 2^-23 each, three
roundings), and one rounding to the page's type, half a step: 2^-24 (fp32), 2^-8 (bf16), 2^-4 (E4M3) of the value, and half of
E4M3's smallest step, 2^-10, below its normal range."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from util import require_gpu

pytestmark = pytest.mark.gpu
KV = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.uint8: 2.0 ** -4}
FULL, BAD_PAGE = 1, 4


@pytest.fixture(scope="module")
def ph():
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m


def i32(a):
    return None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def junk_pool(rng, ph, n_pages, H_kv, d_h, P, kv):
    like = ph.paged_pool(n_pages, H_kv, d_h, P, KV[kv], device="cpu")
    return torch.from_numpy(rng.integers(0, 256, like.numel() * like.element_size()).astype(np.uint8)).view(like.dtype).reshape(like.shape).cuda()


def bits(pool):
    return pool.cpu().view(torch.uint8).numpy()


def stored(x, dtype):
    """One rounding of rows (torch) to a page's type."""
    if dtype == torch.uint8:
        return x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.to(dtype)


def check_rotated(got, x, position, theta, dtype, saturate=False):
    """got, x [n, heads, d_h]: rows as stored and as given."""
    ref = plain.rotated(x, position, theta)
    if saturate:
        ref = np.clip(ref, -448, 448)
    pair = np.abs(x) + np.abs(np.roll(x, x.shape[-1] // 2, -1))
    bound = (5 * 2.0 ** -24 * pair if theta else 0) + HALF_STEP[dtype] * np.abs(ref) * (1 + 2.0 ** -20) + (2.0 ** -10 if dtype == torch.uint8 else 0)
    assert got.shape == ref.shape
    off = np.abs(got - ref)
    assert (off <= bound).all(), (off - bound).max()


CASES = [  # Bt, T, H, H_kv, d_h, page, start, n_new, theta
    (1, 1, 2, 2, 64, 16, [0], None, 1e4), (2, 1, 3, 1, 64, 16, [15, 16], None, 1e4), (3, 3, 4, 2, 52, 16, [30, 0, 47], [3, 0, 2], 1e4),
    (2, 5, 2, 2, 128, 32, [29, 3], [5, 4], 5e5), (2, 40, 2, 1, 56, 16, [7, 90], [40, 33], 1e4), (1, 70, 5, 5, 60, 64, None, None, 1e4),
    (2, 9, 3, 3, 2, 16, [1, 20], None, 1e4), (1, 33, 1, 1, 1, 16, [8], None, 0.0), (2, 17, 2, 2, 33, 128, [100, 5], [17, 2], 0.0), (1, 20, 7, 7, 127, 16, [3], None, 0.0),
    (2, 6, 8, 8, 20, 256, [250, 0], None, 1e4), (2, 12, 6, 3, 100, 16, [11, 40], [12, 1], 1.0), (1, 300, 4, 4, 64, 16, [5], None, 1e4), (1, 7, 2, 2, 64, 16, [9], None, 0.0),
    (4, 2, 33, 33, 32, 16, [1, 2, 3, 14], [1, 2, 2, 2], 1e4), (2, 3, 2, 1, 80, 32, [4, 31], None, 1e4), (1, 1, 64, 64, 126, 16, [17], None, 1e4),
]


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("Bt,T,H,H_kv,d_h,P,start,n_new,theta", CASES)
def test_write(ph, rows, kv, Bt, T, H, H_kv, d_h, P, start, n_new, theta):
    rng = np.random.default_rng(T * d_h + P)
    first, new = start or [0] * Bt, n_new or [T] * Bt
    table, n_pages = plain.table_of(rng, [s + T for s in first], P)
    pools = [junk_pool(rng, ph, n_pages, H_kv, d_h, P, kv) for _ in range(2)]
    before = [p.clone() for p in pools]
    k, v, q = (torch.from_numpy(rng.standard_normal((Bt, T, h, d_h)).astype(np.float32)).to(rows).cuda() for h in (H_kv, H_kv, H))
    q_out = torch.full_like(q, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = ph.PagedCache(*pools, i32(table), d_h)
    ph.photon_paged_cache_write(k, v, cache, start=i32(start), n_new=i32(n_new), q=q, q_out=q_out, rope_theta=theta, status=status)
    assert int(status) == 0
    got_q = q_out.float().cpu().numpy().astype(np.float64)
    touched = np.zeros((2, n_pages, P), bool)
    for b in range(Bt):
        m, position = new[b], first[b] + np.arange(new[b])
        check_rotated(got_q[b, :m], q[b, :m].float().cpu().numpy(), position, theta, rows)
        assert (got_q[b, m:] == 7.0).all()
        page, row = table[b][position // P], position % P
        touched[:, page, row] = True
        got_k, got_v = (p[torch.from_numpy(page).long(), :, torch.from_numpy(row).long()] for p in (pools[0].cpu(), pools[1].cpu()))
        want_v = stored(v[b, :m].cpu(), KV[kv])
        assert torch.equal(got_v[..., :d_h], want_v)
        if theta == 0:
            assert torch.equal(got_k[..., :d_h], stored(k[b, :m].cpu(), KV[kv]))
        else:
            check_rotated(plain.values(got_k)[..., :d_h], k[b, :m].float().cpu().numpy(), position, theta, KV[kv])
        for x in (got_k, got_v):
            assert not x[..., d_h:].view(torch.uint8).any()
    for pool, was, t in zip(pools, before, touched):              # everything else keeps its bits
        a, w = bits(pool).transpose(0, 2, 1, 3), bits(was).transpose(0, 2, 1, 3)
        np.testing.assert_array_equal(a[~t], w[~t])


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_h,shift", [(64, 0), (64, 1), (52, 0), (60, 2), (128, 3)])
def test_rows_of_a_projection(ph, rows, d_h, shift):
    """q, k, v as columns of one matrix, at any alignment of an element; q rotated in place."""
    rng = np.random.default_rng(d_h + shift)
    Bt, T, H, H_kv, P = 2, 11, 4, 2, 16
    width = (H + 2 * H_kv) * d_h + 5
    flat = torch.from_numpy(rng.standard_normal(Bt * T * width + shift).astype(np.float32)).to(rows).cuda()
    was = flat.clone()
    m = flat[shift:].view(Bt, T, width)
    q, k, v = (m[..., at * d_h : (at + h) * d_h].unflatten(-1, (h, d_h)) for at, h in ((0, H), (H, H_kv), (H + H_kv, H_kv)))
    q0, k0, v0 = (x.float().cpu().numpy() for x in (q, k, v))
    table, n_pages = plain.table_of(rng, [T + 3, T + 20], P)
    cache = ph.PagedCache(ph.paged_pool(n_pages, H_kv, d_h, P), ph.paged_pool(n_pages, H_kv, d_h, P), i32(table), d_h)
    ph.photon_paged_cache_write(k, v, cache, start=i32([3, 20]), q=q, q_out=q, rope_theta=1e4)
    pk, pv = plain.values(cache.k_pages), plain.values(cache.v_pages)
    for b, s in enumerate((3, 20)):
        position = s + np.arange(T)
        check_rotated(q[b].float().cpu().numpy().astype(np.float64), q0[b], position, 1e4, rows)
        check_rotated(plain.entries(pk, table[b], s + T, d_h)[:, s:].transpose(1, 0, 2), k0[b], position, 1e4, torch.bfloat16)
        np.testing.assert_array_equal(plain.entries(pv, table[b], s + T, d_h)[:, s:].transpose(1, 0, 2), torch.from_numpy(v0[b]).bfloat16().double().numpy())
    changed = (flat != was).view(-1).cpu().numpy()
    changed[shift:].reshape(Bt * T, width)[:, : H * d_h] = False
    assert not changed.any()                                       # nothing but q's columns


@pytest.mark.parametrize("theta,d_h", [(1e4, 64), (5e5, 128), (1.0, 8), (2.0, 128), (1e4, 52)])
def test_far_and_given_positions(ph, theta, d_h):
    """Positions that are not the entries' own, up to the ends of 32 bits; float64 angles are off by 2^-22 there."""
    rng = np.random.default_rng(5)
    position = np.array([[0, 1, 2, 3, 5, 100, 8191, 131071, 10 ** 6, 10 ** 7 + 1, 2 ** 31 - 1, 2 ** 31 - 77, -1, -7, -(2 ** 31), 123456789]])
    T = position.shape[1]
    k, v = (torch.from_numpy(rng.standard_normal((1, T, 1, d_h)).astype(np.float32)).cuda() for _ in range(2))
    table, n_pages = plain.table_of(rng, [T + 1], 16)
    cache = ph.PagedCache(ph.paged_pool(n_pages, 1, d_h, 16, torch.float32), ph.paged_pool(n_pages, 1, d_h, 16, torch.float32), i32(table), d_h)
    ph.photon_paged_cache_write(k, v, cache, start=i32([1]), position=i32(position), rope_theta=theta)
    got = plain.entries(plain.values(cache.k_pages), table[0], T + 1, d_h)[0, 1:]
    x = k[0, :, 0].cpu().numpy().astype(np.float64)
    ref = plain.rotated(x[:, None], position[0], theta)[:, 0]
    # the angle's own error: 2^-29 turns at the ends of 32 bits, and float64's 2^-53 of the angle
    angle = np.where(np.abs(position[0]) > 2 ** 24, 2 * np.pi * 2.0 ** -29 + np.abs(position[0]) * 2.0 ** -52, 0.0)[:, None]
    size = np.abs(x[:, : d_h // 2]) + np.abs(x[:, d_h // 2 :])
    bound = np.concatenate([size, size], 1) * (6 * 2.0 ** -24 + angle)
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) / bound).max()


def test_places_that_are_not_there(ph):
    """Entries outside the table and pages outside the pool are not written, and said; q is rotated all the same."""
    rng = np.random.default_rng(3)
    P, d_h = 16, 64
    k = torch.from_numpy(rng.standard_normal((4, 4, 2, d_h)).astype(np.float32)).cuda()
    table = i32([[0, 1], [2, 9], [3, -5], [4, 5]])
    for start, want in (([0, 0, 0, 0], 0), ([30, 0, 0, 0], FULL), ([-2, 0, 0, 0], FULL), ([0, 14, 0, 0], BAD_PAGE), ([0, 0, 14, 0], BAD_PAGE), ([0, 0, 16, 31], FULL | BAD_PAGE),
                        ([0, 0, 0, 2 ** 31 - 2], FULL), ([-(2 ** 31), 0, 0, 0], FULL)):
        pools = [ph.paged_pool(6, 2, d_h, P, torch.float32) for _ in range(2)]
        cache = ph.PagedCache(*pools, table, d_h)
        status, q_out = torch.full((1,), 16, dtype=torch.int32, device="cuda"), torch.full_like(k, 9.0)
        ph.photon_paged_cache_write(k, k, cache, start=i32(start), q=k, q_out=q_out, status=status)
        assert int(status) == 16 | want
        assert torch.equal(q_out, k)
        ref = torch.zeros_like(pools[0])
        for b, s in enumerate(start):
            for t in range(4):
                page = int(table[b, (s + t) // P]) if 0 <= s + t < 2 * P else -1
                if 0 <= page < 6:
                    ref[page, :, (s + t) % P] = k[b, t]
        assert torch.equal(pools[0], ref) and torch.equal(pools[1], ref)
        ph.photon_paged_cache_write(k, k, cache, start=i32(start))                       # without a status word
    torch.cuda.synchronize()


def test_counts_and_no_rows(ph):
    k = torch.ones((3, 2, 1, 64), device="cuda")
    for n_new, rows in (([0, 0, 0], 0), ([-3, 0, 1], 1), ([5, 2, 7], 6)):                 # counts beyond T are T
        cache = ph.PagedCache(ph.paged_pool(3, 1, 64, 16), ph.paged_pool(3, 1, 64, 16), i32([[0], [1], [2]]), 64)
        ph.photon_paged_cache_write(k, k, cache, n_new=i32(n_new))
        assert int(cache.k_pages.sum()) == rows * 64
    ph.photon_paged_cache_write(k[:, :0], k[:, :0], cache)
    empty = ph.PagedCache(ph.paged_pool(3, 1, 64, 16), ph.paged_pool(3, 1, 64, 16), torch.zeros((0, 1), dtype=torch.int32, device="cuda"), 64)
    ph.photon_paged_cache_write(k[:0], k[:0], empty)
    torch.cuda.synchronize()


def test_values_that_8_bits_do_not_hold(ph):
    x = torch.tensor([448.0, 449.0, 1e9, -1e30, float("inf"), float("-inf"), float("nan"), 2.0 ** -10, 1.5 * 2.0 ** -9, 464.0, 0.0, -0.0, 2.0 ** -9, 3e-5, 20.0, 21.0] * 4)
    for rows in (torch.float32, torch.bfloat16):
        k = x.to(rows).reshape(1, 1, 1, 64).cuda()
        cache = ph.PagedCache(ph.paged_pool(1, 1, 64, 16, torch.uint8), ph.paged_pool(1, 1, 64, 16, torch.uint8), i32([[0]]), 64)
        ph.photon_paged_cache_write(k, k, cache)
        got = cache.k_pages[0, 0, 0].view(torch.float8_e4m3fn).float().cpu()
        y = x.to(rows).float()
        want = y.clamp(-448, 448).to(torch.float8_e4m3fn).float()
        nan = torch.isnan(y)
        assert torch.isnan(got[nan]).all() and torch.equal(got[~nan], want[~nan])
    # fp32 and bf16 pages keep infinities and NaN
    for dtype in (torch.float32, torch.bfloat16):
        cache = ph.PagedCache(ph.paged_pool(1, 1, 64, 16, dtype), ph.paged_pool(1, 1, 64, 16, dtype), i32([[0]]), 64)
        ph.photon_paged_cache_write(k, k, cache)
        got, want = cache.v_pages[0, 0, 0].float().cpu(), k.to(dtype).float().cpu().reshape(64)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


# ---------------------------------------------------------------- moving

@pytest.mark.parametrize("kv,d_h", [("f32", 128), ("bf16", 64), ("e4m3", 20), ("bf16", 100)])
@pytest.mark.parametrize("Bt,T,H_kv,P,start,n", [(1, 1, 1, 16, [0], None), (3, 7, 2, 16, [12, 0, 29], [7, 0, 3]), (2, 64, 3, 16, [5, 40], None), (2, 33, 1, 64, [60, 0], [33, 20])])
def test_move(ph, kv, d_h, Bt, T, H_kv, P, start, n):
    rng = np.random.default_rng(T + d_h)
    count = n or [T] * Bt
    table, n_pages = plain.table_of(rng, [s + T + 8 for s in start], P)
    for kind in range(4):
        pools = [junk_pool(rng, ph, n_pages, H_kv, d_h, P, kv) for _ in range(2)]
        before = [p.clone() for p in pools]
        source = {0: np.sort(rng.integers(0, T + 8, (Bt, T)), 1), 1: rng.integers(0, T, (Bt, T)),                  # a path; any order, repeats
                  2: np.tile(np.arange(T)[::-1], (Bt, 1)), 3: np.tile(np.arange(T), (Bt, 1))}[kind]                # turned round; as they are
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ph.photon_paged_cache_move(ph.PagedCache(*pools, i32(table), d_h), i32(start), i32(source), n=i32(n), status=status)
        assert int(status) == 0
        for pool, was in zip(pools, before):
            want = was.clone()
            for b in range(Bt):
                for i in range(count[b]):
                    to, of = start[b] + i, start[b] + int(source[b, i])
                    want[int(table[b, to // P]), :, to % P] = was[int(table[b, of // P]), :, of % P]
            assert torch.equal(pool.view(torch.uint8), want.view(torch.uint8))


def test_moves_from_and_to_places_that_are_not_there(ph):
    table = i32([[0, 1], [2, 7]])
    for start, source, want, moved in (([0, 0], [[5], [20]], BAD_PAGE, [0]), ([0, 0], [[40], [3]], FULL, [1]), ([0, 0], [[-1], [3]], FULL, [1]), ([32, 17], [[-4], [-16]], FULL | BAD_PAGE, []),
                                       ([-1, 0], [[4], [1]], FULL, [1]), ([2 ** 31 - 1, 0], [[2 ** 31 - 1], [-(2 ** 31)]], FULL, [])):
        pools = [torch.arange(3 * 16, device="cuda", dtype=torch.float32).reshape(3, 1, 16, 1).expand(3, 1, 16, 64).contiguous() for _ in range(2)]
        ref = pools[0].clone()
        for b in moved:
            s, o = start[b], start[b] + source[b][0]
            ref[int(table[b, s // 16]), 0, s % 16] = pools[0][int(table[b, o // 16]), 0, o % 16]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ph.photon_paged_cache_move(ph.PagedCache(*pools, table, 64), i32(start), i32(source), status=status)
        assert int(status) == want
        assert torch.equal(pools[0], ref) and torch.equal(pools[1], ref)


def test_places_past_32_bits(ph):
    """Pools of more than 2^32 bytes: the last page is as good as the first."""
    d_h, P, H_kv = 128, 256, 8
    n_pages = 9000                                                  # of 512 KiB: 4.4 GiB
    pools = [torch.zeros((n_pages, H_kv, P, d_h), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = ph.PagedCache(*pools, i32([[n_pages - 1, 0]]), d_h)
    k = torch.randn((1, 6, H_kv, d_h), device="cuda").bfloat16()
    ph.photon_paged_cache_write(k, -k, cache, start=i32([253]))
    assert torch.equal(pools[0][n_pages - 1, :, 253:], k[0, :3].transpose(0, 1)) and torch.equal(pools[1][0, :, :3], -k[0, 3:].transpose(0, 1))
    ph.photon_paged_cache_move(cache, i32([251]), i32([[2, 5, 6]]))
    assert torch.equal(pools[0][n_pages - 1, :, 251:254], k[0, [0, 3, 4]].transpose(0, 1)) and torch.equal(pools[0][n_pages - 1, :, 254:], k[0, 1:3].transpose(0, 1))
    q = torch.randn((1, 1, H_kv, d_h), device="cuda").bfloat16()
    pools[0][n_pages - 1, :, :251].normal_()
    pools[1][n_pages - 1].normal_()
    out = torch.empty_like(q)
    ph.photon_paged_attn(q, cache, i32([258]), out, n_splits=1)
    ks, vs = (torch.cat([p[n_pages - 1], p[0, :, :2]], 1)[None].float().cpu().double().numpy()[0] for p in pools)
    ref, size = plain.attended(q[0, 0].float().cpu().numpy(), ks, vs, np.ones(258, bool), d_h ** -0.5)
    got = out[0, 0].float().cpu().numpy()
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size).all()
