"""Attention over the paged K/V cache against the float64 definition.

Tolerances.  Per value, with A = sum(p |v|) of its row: weights keep 17 bits (bf16 rows; error at most 2^-17 of each) or 24 (fp32
rows); scores are fp32 sums of d_h products of at most |q||k| scale, each rounding 2^-24 of it, which moves a weight by the same
part: with |s| up to about 30 here, d_h roundings in a row could add 128 * 30 * 2^-24 = 2^-12, their sum in earnest (they have either
sign) a sixteenth of that at most: 2^-16 * A.  Adding up to 4096 weights in fp32 gives less.  So 2^-15 * A (bf16 rows, of both) and
1e-5 * the largest A, the bar of every fp32 kernel here (fp32 rows); a bf16 result is rounded once, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from util import require_gpu

pytestmark = pytest.mark.gpu
KV = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}
BAD_PAGE = 4


@pytest.fixture(scope="module")
def ph():
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m


def i32(a):
    return None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def i64(a):
    return None if a is None else torch.tensor(np.asarray(a, np.int64), device="cuda")


def filled(rng, n_pages, H_kv, d_h, P, kv, table, lengths):
    """A pool with N(0, 1) entries in use, zeros in their pad columns, and NaN everywhere else."""
    d_p = 32 if d_h <= 32 else 64 if d_h <= 64 else 128
    pool = torch.full((n_pages, H_kv, P, d_p), 255, dtype=torch.uint8) if kv == "e4m3" else torch.full((n_pages, H_kv, P, d_p), float("nan"), dtype=KV[kv])
    for b, n in enumerate(lengths):
        for s in range(0, n, P):
            rows = min(P, n - s)
            x = torch.zeros((H_kv, rows, d_p))
            x[..., :d_h] = torch.from_numpy(rng.standard_normal((H_kv, rows, d_h)).astype(np.float32))
            pool[table[b, s // P], :, :rows] = x.to(torch.float8_e4m3fn).view(torch.uint8) if kv == "e4m3" else x.to(KV[kv])
    return pool


def trees(rng, Bt, T):
    out = []
    for _ in range(Bt):
        out.append(plain.tree_masks([-1] + [int(rng.integers(max(0, t - 5), t)) for t in range(1, T)])[0])
    return np.stack(out)


def check(got, q, pools, table, lengths, new, d_h, masks=None, scale=None, fill=None):
    """got, q [Bt, T, H, d_h] torch; pools torch; entries [b] x P numpy."""
    Bt, T, H, _ = q.shape
    vals = [plain.values(p) for p in pools]
    x, y = q.float().cpu().numpy(), got.float().cpu().numpy().astype(np.float64)
    scale = d_h ** -0.5 if scale is None else scale
    for b in range(Bt):
        k, v = (plain.entries(p, table[b], lengths[b], d_h) if lengths[b] else np.zeros((p.shape[1], 0, d_h)) for p in vals)
        for t in range(T):
            if t >= new[b]:
                assert fill is None or (y[b, t] == fill).all()
                continue
            ref, size = plain.attended(x[b, t], k, v, plain.seen(lengths[b], new[b], t, None if masks is None else masks[b, t]), scale)
            bound = 1e-5 * max(size.max(), 1e-30) if q.dtype == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
            off = np.abs(y[b, t] - ref)
            assert (off <= bound).all(), (b, t, (off - bound).max(), off.max())


def run(ph, rng, rows, kv, Bt, T, H, H_kv, d_h, P, lengths, new=None, tree=False, splits=0, S_max=None, width=None):
    table, n_pages = plain.table_of(rng, lengths, P, width=width)
    pools = [filled(rng, n_pages, H_kv, d_h, P, kv, table, lengths) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = torch.from_numpy(rng.standard_normal((Bt, T, H, d_h)).astype(np.float32)).to(rows).cuda()
    masks = trees(rng, Bt, T) if tree else None
    out = torch.full_like(q, 5.0)
    size = ph.photon_paged_attn_workspace_bytes(cache, Bt, T, H, S_max, splits)
    ws = torch.full((size + 16,), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ph.photon_paged_attn(q, cache, i32(lengths), out, n_new=i32(new), tree=i64(masks), n_splits=splits, workspace=ws, status=status, S_max=S_max)
    assert int(status) == 0 and (ws[size:] == 255).all()
    check(out, q, pools, table, lengths, new or [T] * Bt, d_h, masks, fill=5.0)
    return cache, q, out


CASES = [  # Bt, T, H, H_kv, d_h, page, lengths, new, tree
    (1, 1, 1, 1, 64, 16, [1], None, False), (2, 1, 2, 2, 64, 16, [17, 0], None, False), (3, 1, 4, 1, 128, 32, [33, 32, 31], None, False),
    (2, 1, 8, 2, 52, 16, [100, 63], None, False), (1, 1, 16, 1, 32, 64, [129], None, False), (2, 1, 17, 1, 60, 16, [50, 200], None, False),
    (2, 3, 4, 2, 64, 16, [40, 3], None, False), (3, 4, 3, 3, 56, 16, [64, 2, 37], [4, 3, 0], False), (2, 16, 2, 2, 128, 16, [47, 16], [16, 5], False),
    (2, 33, 2, 2, 64, 16, [70, 33], [33, 20], False), (1, 70, 2, 1, 20, 32, [150], None, False), (1, 150, 4, 2, 128, 16, [333], None, False), (2, 70, 6, 3, 64, 128, [70, 40], [70, 40], False),
    (1, 1, 1, 1, 1, 16, [5], None, False), (2, 2, 2, 1, 33, 16, [40, 15], None, False), (1, 3, 1, 1, 127, 256, [300], None, False),
    (2, 2, 2, 2, 64, 16, [20, 9], None, True), (2, 13, 4, 4, 60, 16, [60, 13], [13, 7], True), (2, 31, 4, 2, 128, 32, [31, 95], None, True), (1, 64, 2, 1, 64, 16, [200], None, True),
    (2, 64, 8, 2, 128, 64, [130, 64], [64, 33], True), (3, 9, 2, 2, 100, 16, [5, 0, 30], [9, 9, 4], True), (1, 24, 5, 1, 80, 16, [77], None, True),
]


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("Bt,T,H,H_kv,d_h,P,lengths,new,tree", CASES)
def test_attention(ph, rows, kv, Bt, T, H, H_kv, d_h, P, lengths, new, tree):
    for splits in (1, 3):
        run(ph, np.random.default_rng(T * d_h + P), rows, kv, Bt, T, H, H_kv, d_h, P, lengths, new, tree, splits)


@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("splits", [0, 1, 2, 7, 64])
@pytest.mark.parametrize("T,H,H_kv,tree", [(1, 2, 2, False), (1, 8, 1, False), (12, 4, 2, True), (40, 8, 2, False)])
def test_long_sequences_in_splits(ph, kv, splits, T, H, H_kv, tree):
    for rows in (torch.bfloat16, torch.float32):
        run(ph, np.random.default_rng(splits), rows, kv, 2, T, H, H_kv, 64, 32, [4001, 777], [T, max(1, T // 2)], tree, splits)


def test_the_same_bits_every_time(ph):
    rng = np.random.default_rng(1)
    cache, q, out = run(ph, rng, torch.bfloat16, "bf16", 2, 5, 4, 2, 64, 16, [500, 333], None, False, 4)
    ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 2, 5, 4, None, 4), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = torch.empty_like(out)
        ph.photon_paged_attn(q, cache, i32([500, 333]), again, n_splits=4, workspace=ws)
        assert torch.equal(again, out)


@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
def test_lengths_and_counts_out_of_range(ph, rows, kv):
    """Lengths beyond S_max count as S_max, below 0 as 0; counts beyond T as T; a table that is wider than needed."""
    rng = np.random.default_rng(9)
    P, d_h, H = 16, 64, 2
    table, n_pages = plain.table_of(rng, [48, 48, 20], P, width=7)
    pools = [filled(rng, n_pages, H, d_h, P, kv, table, [48, 48, 20]) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = torch.from_numpy(rng.standard_normal((3, 2, H, d_h)).astype(np.float32)).to(rows).cuda()
    out = torch.full_like(q, 5.0)
    ph.photon_paged_attn(q, cache, i32([1000, -5, 20]), out, n_new=i32([9, 2, -1]), S_max=41, n_splits=1)
    check(out, q, pools, table, [41, 0, 20], [2, 2, 0], d_h, fill=5.0)
    assert not out[1].any()


def test_masks_of_any_kind(ph):
    """Words that are no tree: rows that see nothing of their own, bits past the count, a query that does not see itself."""
    rng = np.random.default_rng(4)
    P, d_h, H, T = 16, 64, 2, 8
    lengths, new = [40, 8, 8, 6], [8, 8, 5, 8]
    masks = rng.integers(0, 2 ** 63, (4, T), dtype=np.int64)
    masks[0, 3], masks[1, 0], masks[1, 5], masks[3, 1], masks[0, 7] = 0, 0, 2, 0, -1
    for rows in (torch.float32, torch.bfloat16):
        for kv in KV:
            table, n_pages = plain.table_of(rng, lengths, P)
            pools = [filled(rng, n_pages, H, d_h, P, kv, table, lengths) for _ in range(2)]
            cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
            q = torch.from_numpy(rng.standard_normal((4, T, H, d_h)).astype(np.float32)).to(rows).cuda()
            for splits in (1, 2):
                ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 4, T, H, None, splits) + 16, dtype=torch.uint8, device="cuda")
                out = torch.full_like(q, 5.0)
                ph.photon_paged_attn(q, cache, i32(lengths), out, n_new=i32(new), tree=i64(masks), n_splits=splits, workspace=ws)
                check(out, q, pools, table, lengths, new, d_h, masks, fill=5.0)
                assert not out[1, 0].any()


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T,H,H_kv", [(9, 2, 2), (24, 4, 2), (40, 2, 1)])
def test_what_is_not_seen_may_hold_anything(ph, rows, kv, tree, T, H, H_kv):
    """Infinities and NaN in drafted entries reach the queries that see them and no other."""
    rng = np.random.default_rng(T)
    P, d_h, past = 16, 64, 21
    lengths = [past + T]
    table, n_pages = plain.table_of(rng, lengths, P)
    masks = trees(rng, 1, T) if tree else None
    q = torch.from_numpy(rng.standard_normal((1, T, H, d_h)).astype(np.float32)).to(rows).cuda()
    for what in ("v", "k"):
        pools = [filled(rng, n_pages, H_kv, d_h, P, kv, table, lengths) for _ in range(2)]
        bad = {3: (5, "nan"), T - 2: (60, "nan" if kv == "e4m3" else "inf"), T - 4: (0, "nan" if kv == "e4m3" else "-inf")}
        pool = pools[what == "v"]
        for j, (d, value) in bad.items():
            e = past + j
            pool[table[0, e // P], :, e % P, d] = 255 if kv == "e4m3" else float(value)
        cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
        clean = [p.clone() for p in pools]
        for j, (d, _) in bad.items():
            e = past + j
            clean[what == "v"][table[0, e // P], :, e % P, d] = 0
        out = torch.empty_like(q)
        ph.photon_paged_attn(q, cache, i32(lengths), out, tree=i64(masks), n_splits=1)
        got = out.float().cpu().numpy().astype(np.float64)
        x = q.float().cpu().numpy()
        k, v = (plain.entries(plain.values(p), table[0], lengths[0], d_h) for p in clean)
        for t in range(T):
            see = plain.seen(lengths[0], T, t, None if masks is None else masks[0, t])
            ref, size = plain.attended(x[0, t], k, v, see, d_h ** -0.5)
            bound = 1e-5 * size.max() if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
            touched = [j for j in bad if see[past + j]]
            if what == "v":
                fine = np.ones(d_h, bool)
                for j in touched:
                    fine[bad[j][0]] = False
                assert not np.isfinite(got[0, t][:, ~fine]).any()
                assert (np.abs(got[0, t] - ref)[:, fine] <= (bound if np.isscalar(bound) else bound[:, fine])).all(), t
            elif not touched:
                assert (np.abs(got[0, t] - ref) <= bound).all(), t
            elif any(bad[j][1] == "nan" for j in touched):
                assert np.isnan(got[0, t]).all()


def test_pages_outside_the_pool(ph):
    """Their entries are not seen, and it is said; what is there is attended to."""
    rng = np.random.default_rng(8)
    P, d_h, H = 16, 64, 2
    lengths = [70, 33]
    table, n_pages = plain.table_of(rng, lengths, P)
    for rows, kv in ((torch.float32, "f32"), (torch.bfloat16, "bf16"), (torch.bfloat16, "e4m3"), (torch.float32, "bf16")):
        pools = [filled(rng, n_pages, H, d_h, P, kv, table, lengths) for _ in range(2)]
        for p in pools:
            p[0] = 255 if kv == "e4m3" else float("nan")             # what a wrong page must not be taken for
        wrong = table.copy()
        wrong[wrong == 0] = n_pages
        wrong[0, 1], wrong[1, 2] = -1, n_pages + 7
        cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(wrong), d_h)
        q = torch.from_numpy(rng.standard_normal((2, 1, H, d_h)).astype(np.float32)).to(rows).cuda()
        for splits in (1, 2):
            out, status = torch.empty_like(q), torch.full((1,), 2, dtype=torch.int32, device="cuda")
            ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 2, 1, H, None, splits) + 16, dtype=torch.uint8, device="cuda")
            ph.photon_paged_attn(q, cache, i32(lengths), out, n_splits=splits, workspace=ws, status=status)
            assert int(status) == 2 | BAD_PAGE
            ph.photon_paged_attn(q, cache, i32(lengths), out, n_splits=splits, workspace=ws)
            for b, n in enumerate(lengths):
                see = np.array([0 <= wrong[b, e // P] < n_pages for e in range(n)])
                k, v = (plain.entries(plain.values(p), np.maximum(table[b], 0), n, d_h) for p in pools)
                ref, size = plain.attended(q[b, 0].float().cpu().numpy(), k, v, see, d_h ** -0.5)
                bound = 1e-5 * size.max() if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
                assert (np.abs(out[b, 0].float().cpu().numpy() - ref) <= bound).all()


def test_a_page_that_sequences_share(ph):
    rng = np.random.default_rng(12)
    P, d_h, H = 32, 64, 4
    table = np.array([[3, 1, 0], [3, 1, 2], [3, 4, -1]], np.int32)
    lengths = [80, 96, 40]
    pools = [torch.from_numpy(rng.standard_normal((5, 2, P, 64)).astype(np.float32)).bfloat16() for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = torch.from_numpy(rng.standard_normal((3, 2, H, d_h)).astype(np.float32)).bfloat16().cuda()
    out = torch.empty_like(q)
    ph.photon_paged_attn(q, cache, i32(lengths), out, n_splits=1)
    check(out, q, pools, table, lengths, [2, 2, 2], d_h)


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_h,shift", [(64, 1), (52, 0), (60, 3)])
def test_rows_at_any_alignment(ph, rows, d_h, shift):
    rng = np.random.default_rng(d_h)
    Bt, T, H, H_kv, P = 2, 3, 4, 2, 16
    lengths = [50, 20]
    table, n_pages = plain.table_of(rng, lengths, P)
    pools = [filled(rng, n_pages, H_kv, d_h, P, "bf16", table, lengths) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    width = H * d_h + 7
    q = torch.from_numpy(rng.standard_normal(Bt * T * width + shift).astype(np.float32)).to(rows).cuda()[shift:].view(Bt, T, width)[..., : H * d_h].unflatten(-1, (H, d_h))
    out = torch.empty(Bt * T * H * d_h + shift, dtype=rows, device="cuda")[shift:].view(Bt, T, H, d_h)
    for splits in (1, 2):
        ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, Bt, T, H, None, splits) + 16, dtype=torch.uint8, device="cuda")
        ph.photon_paged_attn(q, cache, i32(lengths), out, n_splits=splits, workspace=ws)
        check(out, q, pools, table, lengths, [T] * Bt, d_h)


@pytest.mark.parametrize("kv", ["f32", "bf16"])
def test_scores_far_from_zero(ph, kv):
    """Scores of either sign up to 10^30, rising along the sequence: softmax is a choice there, and no result is NaN."""
    for rows in (torch.float32, torch.bfloat16):
        for size in (1e3, 1e8, 1e30):
            for sign in (1.0, -1.0):
                n, d_h = 100, 64
                k = torch.zeros((7, 1, 16, d_h))
                k[..., 0] = sign * (1 + torch.arange(7 * 16).reshape(7, 1, 16) / 128.0)
                v = torch.randn((7, 1, 16, d_h), generator=torch.Generator().manual_seed(1))
                q = torch.zeros((1, 1, 1, d_h))
                q[..., 0] = size
                pools = [k.to(KV[kv]), v.to(KV[kv])]
                table = np.arange(7, dtype=np.int32)[None]
                cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
                out = torch.empty((1, 1, 1, d_h), dtype=rows, device="cuda")
                ph.photon_paged_attn(q.to(rows).cuda(), cache, i32([n]), out, n_splits=1)
                # scores are 16 apart at least; one entry takes all but e^-15, size 1e3 with a step of 1/128: e^(-0.97)
                ks, vs = (plain.entries(plain.values(p), table[0], n, d_h) for p in pools)
                ref, a = plain.attended(q[0, 0].to(rows).float().numpy(), ks, vs, np.ones(n, bool), d_h ** -0.5)
                got = out[0, 0].float().cpu().numpy()
                # a score of 10^3 / 8 is exact to 2^-24 * 250: 2^-16 of a weight
                bound = 2.0 ** -14 * a + (0 if rows == torch.float32 else 2.0 ** -8 * np.abs(ref))
                assert (np.abs(got - ref) <= bound).all(), (size, sign, np.abs(got - ref).max())


def test_streams_and_two_calls_at_once(ph):
    """Calls on two streams with a workspace each, many times; results as on one."""
    rng = np.random.default_rng(2)
    made = [run(ph, rng, torch.bfloat16, "bf16", 2, 3, 8, 2, 128, 16, [900, 411], None, False, 8) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, keep = [], []
    torch.cuda.synchronize()
    for (cache, q, want), st in zip(made, streams):
        with torch.cuda.stream(st):
            ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 2, 3, 8, None, 8), dtype=torch.uint8, device="cuda")
            lengths = i32([900, 411])
            got = [torch.empty_like(want) for _ in range(10)]
            for o in got:
                ph.photon_paged_attn(q, cache, lengths, o, n_splits=8, workspace=ws)
            outs.append(got)
            keep += [ws, lengths]
    torch.cuda.synchronize()
    for (_, _, want), got in zip(made, outs):
        for o in got:
            assert torch.equal(o, want)
