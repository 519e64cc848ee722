"""Attention over the paged K/V cache where many rows share a K/V head (with many streams of bf16 rows and pages entries go through LDS there),
and what all of its kernels have to survive: pages that are not there, far scores, large values, scales of any kind, more splits than steps.

Tolerances as in tests/test_gpu_paged_attn.py."""
import numpy as np
import pytest
import torch

import paged_plain as plain
import test_gpu_paged_attn as base
from test_gpu_paged_attn import BAD_PAGE, KV, check, filled, i32, i64, trees
from util import require_gpu

pytestmark = pytest.mark.gpu


class Many:
    """The library with every call turned into one of so many streams that workgroups take 64 rows and more: query heads are repeated until a
    stream has more than `above` rows (64: what the wide kernel takes where rows and pages are bf16), K/V heads until streams are enough.
    Equal streams have to give equal bits."""

    def __init__(self, library, above):
        self.library, self.above, self.calls = library, above, 0

    def __getattr__(self, name):
        return getattr(self.library, name)

    def photon_paged_attn(self, q, cache, seq_len, out, workspace=None, n_splits=0, **kw):
        Bt, T, H, d_h = q.shape
        H_kv = cache.H_kv
        group = H // H_kv
        copies = self.above // (T * group) + 1
        rows = T * group * copies
        streams = 512 // (Bt * H_kv * -(-rows // 32)) + 1
        assert rows > self.above and Bt * H_kv * streams * -(-rows // 32) > 512
        many = self.library.PagedCache(*(p.repeat_interleave(streams, 1) for p in (cache.k_pages, cache.v_pages)), cache.page_table, d_h)
        shape = (Bt, T, H_kv, streams, group, copies, d_h)

        def spread(x):
            return x.view(Bt, T, H_kv, 1, group, 1, d_h).expand(shape).reshape(Bt, T, -1, d_h).contiguous()

        q_many, out_many = spread(q.contiguous()), spread(out)
        if n_splits != 1:
            size = self.library.photon_paged_attn_workspace_bytes(many, Bt, T, q_many.shape[2], kw.get("S_max"), n_splits)
            workspace = torch.full((size + 16,), 255, dtype=torch.uint8, device="cuda")
        self.library.photon_paged_attn(q_many, many, seq_len, out_many, workspace=workspace, n_splits=n_splits, **kw)
        if n_splits != 1:
            assert (workspace[size:] == 255).all()
        got = out_many.view(shape)
        bits = torch.int16 if q.dtype is torch.bfloat16 else torch.int32
        assert torch.equal(got.view(bits), got[:, :, :, :1].expand(shape).contiguous().view(bits))
        self.calls += 1
        out.copy_(got[:, :, :, 0, :, self.calls % copies].reshape(out.shape))
        return out


@pytest.fixture(scope="module", params=["few streams", "many streams"])
def ph(request):
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m if request.param == "few streams" else Many(m, 64)


@pytest.fixture(scope="module", params=[16, 64])
def many(request):
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return Many(m, request.param)


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("Bt,T,H,H_kv,d_h,P,lengths,new,tree", base.CASES)
def test_attention_of_many_streams(many, rows, kv, Bt, T, H, H_kv, d_h, P, lengths, new, tree):
    for splits in (1, 3):
        base.run(many, np.random.default_rng(T * d_h + P), rows, kv, Bt, T, H, H_kv, d_h, P, lengths, new, tree, splits)


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.bfloat16, "e4m3"), (torch.float32, "f32")])
@pytest.mark.parametrize("splits", [0, 2, 7])
@pytest.mark.parametrize("T,H,H_kv,tree", [(1, 8, 1, False), (12, 4, 2, True), (40, 8, 2, False)])
def test_long_sequences_of_many_streams(many, rows, kv, splits, T, H, H_kv, tree):
    base.run(many, np.random.default_rng(splits), rows, kv, 2, T, H, H_kv, 64, 32, [4001, 777], [T, max(1, T // 2)], tree, splits)


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T,H,H_kv", [(9, 2, 2), (24, 4, 2), (40, 2, 1)])
def test_what_is_not_seen_by_many_streams(many, rows, kv, tree, T, H, H_kv):
    base.test_what_is_not_seen_may_hold_anything(many, rows, kv, tree, T, H, H_kv)


def test_masks_lengths_and_pages_of_many_streams(many):
    base.test_masks_of_any_kind(many)
    for rows in (torch.float32, torch.bfloat16):
        for kv in KV:
            base.test_lengths_and_counts_out_of_range(many, rows, kv)
    base.test_pages_outside_the_pool(many)
    base.test_scores_far_from_zero(many, "bf16")
    base.test_scores_far_from_zero(many, "f32")


def attend(ph, q, cache, lengths, splits=1, **kw):
    Bt, T, H, _ = q.shape
    out = torch.full_like(q, 5.0)
    ws = torch.full((ph.photon_paged_attn_workspace_bytes(cache, Bt, T, H, None, splits) + 16,), 255, dtype=torch.uint8, device="cuda")
    ph.photon_paged_attn(q, cache, i32(lengths), out, n_splits=splits, workspace=ws, **kw)
    return out


def queries(rng, shape, rows):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(rows).cuda()


@pytest.mark.parametrize("P", [16, 32, 64, 256])
@pytest.mark.parametrize("d_h", [20, 64, 100, 128])
@pytest.mark.parametrize("T,H,H_kv,new,tree", [(66, 2, 2, [66, 40], False), (130, 4, 2, [130, 127], False), (33, 4, 1, [33, 17], False), (64, 4, 1, [64, 35], True), (40, 8, 1, [40, 39], True)])
def test_many_rows(ph, P, d_h, T, H, H_kv, new, tree):
    """65 rows to 320, workgroups with waves that have none, entries that end inside a stage, pages smaller and larger than one."""
    rng = np.random.default_rng(P + d_h + T)
    lengths = [new[0] + 217, new[1]]
    table, n_pages = plain.table_of(rng, lengths, P)
    pools = [filled(rng, n_pages, H_kv, d_h, P, "bf16", table, lengths) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = queries(rng, (2, T, H, d_h), torch.bfloat16)
    masks = trees(rng, 2, T) if tree else None
    for splits in (1, 2, 5):
        check(attend(ph, q, cache, lengths, splits, n_new=i32(new), tree=i64(masks)), q, pools, table, lengths, new, d_h, masks, fill=5.0)


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.bfloat16, "e4m3"), (torch.float32, "f32")])
@pytest.mark.parametrize("T,H,H_kv,P", [(1, 4, 2, 16), (9, 4, 2, 32), (48, 4, 2, 16), (48, 4, 2, 64), (150, 2, 1, 64), (150, 2, 1, 16)])
def test_pages_that_are_missing_along_a_sequence(ph, rows, kv, T, H, H_kv, P):
    """Missing pages at the beginning, in the middle, among the queries' own entries: skipped, and everything behind them is seen."""
    rng = np.random.default_rng(T + P)
    d_h, n = 64, 600
    table, n_pages = plain.table_of(rng, [n], P)
    pools = [filled(rng, n_pages, H_kv, d_h, P, kv, table, [n]) for _ in range(2)]
    wrong = table.copy()
    pages = (n + P - 1) // P
    for at, page in ((0, -1), (pages // 2, n_pages), (pages // 2 + 1, 2 ** 31 - 1), (pages - 2, -(2 ** 31))):
        wrong[0, at] = page
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(wrong), d_h)
    q = queries(rng, (1, T, H, d_h), rows)
    there = np.repeat((wrong[0] >= 0) & (wrong[0] < n_pages), P)[:n]
    k, v = (plain.entries(plain.values(p), table[0], n, d_h) for p in pools)
    x = q.float().cpu().numpy()
    for splits in (1, 3):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = attend(ph, q, cache, [n], splits, status=status).float().cpu().numpy()
        assert int(status) == BAD_PAGE
        for t in range(0, T, 7):
            ref, size = plain.attended(x[0, t], k, v, plain.seen(n, T, t) & there, d_h ** -0.5)
            bound = 1e-5 * max(size.max(), 1e-30) if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
            assert (np.abs(out[0, t] - ref) <= bound).all(), t
    # no page at all: zeros
    none = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(np.full_like(table, -1)), d_h)
    assert not attend(ph, q, none, [n], 2).any()


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.float32, "f32"), (torch.bfloat16, "e4m3")])
@pytest.mark.parametrize("T", [1, 20, 70])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 2.5])
def test_scales(ph, rows, kv, T, scale):
    rng = np.random.default_rng(T)
    d_h, lengths = 32, [300]
    table, n_pages = plain.table_of(rng, lengths, 16)
    pools = [filled(rng, n_pages, 1, d_h, 16, kv, table, lengths) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = queries(rng, (1, T, 1, d_h), rows)
    for splits in (1, 3):
        check(attend(ph, q, cache, lengths, splits, scale=scale), q, pools, table, lengths, [T], d_h, scale=scale)


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.float32, "f32")])
@pytest.mark.parametrize("T", [3, 70])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_far_scores(ph, rows, kv, T, sign):
    """Scores of 10^30 of either sign that rise along the sequence: the greatest one's V, and no NaN.  Neighbours are 2^-7 of 10^30 apart."""
    n, d_h = 200, 64
    k = torch.zeros((13, 1, 16, d_h))
    k[..., 0] = sign * (1 + torch.arange(13 * 16).reshape(13, 1, 16) // 4 * 4 / 128.0)
    v = torch.randn((13, 1, 16, d_h), generator=torch.Generator().manual_seed(1)).to(KV[kv])
    q = torch.zeros((1, T, 1, d_h))
    q[..., 0] = 1e30
    table = np.arange(13, dtype=np.int32)[None]
    cache = ph.PagedCache(k.to(KV[kv]).cuda(), v.cuda(), i32(table), d_h)
    out = attend(ph, q.to(rows).cuda(), cache, [n], 1)
    ks, vs = (plain.entries(plain.values(p), table[0], n, d_h) for p in (k.to(KV[kv]), v))
    for t in (0, T - 1):
        ref, a = plain.attended(q[0, t].to(rows).float().numpy(), ks, vs, plain.seen(n, T, t), d_h ** -0.5)
        bound = 2.0 ** -14 * a + (0 if rows == torch.float32 else 2.0 ** -8 * np.abs(ref))
        assert (np.abs(out[0, t].float().cpu().numpy() - ref) <= bound).all(), t


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.float32, "f32")])
@pytest.mark.parametrize("T", [1, 17, 70])
def test_large_values(ph, rows, kv, T):
    """V whose absolute sum is near fp32's end, 150 entries of up to 2^120.8: finite, and as exact as elsewhere."""
    rng = np.random.default_rng(T)
    d_h, lengths = 64, [150]
    table, n_pages = plain.table_of(rng, lengths, 32)
    pools = [filled(rng, n_pages, 1, d_h, 32, kv, table, lengths) for _ in range(2)]
    pools[1] = (pools[1].float() * 2.0 ** 118.5).to(KV[kv])
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = queries(rng, (1, T, 1, d_h), rows)
    for splits in (1, 2):
        check(attend(ph, q, cache, lengths, splits), q, pools, table, lengths, [T], d_h)


def test_more_splits_than_steps(ph):
    rng = np.random.default_rng(3)
    lengths = [70, 1, 0]
    for rows, kv, T in ((torch.bfloat16, "bf16", 1), (torch.float32, "f32", 3), (torch.bfloat16, "bf16", 70)):
        new = [T, 1, 1]
        table, n_pages = plain.table_of(rng, [max(n, 1) for n in lengths], 16)
        pools = [filled(rng, n_pages, 2, 64, 16, kv, table, lengths) for _ in range(2)]
        cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), 64)
        q = queries(rng, (3, T, 4, 64), rows)
        for splits in (8, 9, 100, 1024):
            check(attend(ph, q, cache, lengths, splits, n_new=i32(new)), q, pools, table, lengths, new, 64, fill=5.0)


def test_a_longer_bound_changes_no_bit_of_one_split(ph):
    """S_max bounds the lengths: it chooses splits, nothing else."""
    rng = np.random.default_rng(5)
    lengths = [333, 20]
    table, n_pages = plain.table_of(rng, lengths, 16, width=64)
    pools = [filled(rng, n_pages, 2, 64, 16, "bf16", table, lengths) for _ in range(2)]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), 64)
    for T in (1, 40):
        q = queries(rng, (2, T, 4, 64), torch.bfloat16)
        new = [T, min(T, 20)]
        a, b = (attend(ph, q, cache, lengths, 1, S_max=s, n_new=i32(new)) for s in (333, 1024))
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,kv", [(torch.bfloat16, "bf16"), (torch.float32, "bf16"), (torch.float32, "f32"), (torch.bfloat16, "e4m3")])
@pytest.mark.parametrize("H", [2, 80])
@pytest.mark.parametrize("new", [1, 3])
def test_nodes_that_do_not_see_themselves(ph, rows, kv, H, new):
    """Masks of zero: the entries before the tree's, whatever the own ones hold; and nothing, where there are none before."""
    rng = np.random.default_rng(H + new)
    d_h, P = 64, 16
    for n in (new + 90, new):
        table, n_pages = plain.table_of(rng, [n], P)
        pools = [filled(rng, n_pages, 1, d_h, P, kv, table, [n]) for _ in range(2)]
        for p in pools:
            for j in range(n - new, n):
                p[int(table[0, j // P]), 0, j % P] = 255 if kv == "e4m3" else float("nan")
        cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
        q = queries(rng, (1, new, H, d_h), rows)
        masks = np.zeros((1, new), np.uint64)
        for splits in (1, 2):
            check(attend(ph, q, cache, [n], splits, tree=i64(masks)), q, pools, table, [n], [new], d_h, masks)


@pytest.mark.parametrize("rows,kv,T", [(torch.bfloat16, "bf16", 70), (torch.bfloat16, "bf16", 140), (torch.float32, "bf16", 40)])
def test_captured_calls_of_many_streams(rows, kv, T):
    """A captured call replayed with other lengths, pages and queries, eager calls in between: the eager call's bits."""
    require_gpu()
    import paper_2512_20687_amd as ph
    rng = np.random.default_rng(T)
    P, d_h, H, longest = 16, 128, 90, 400
    table, n_pages = plain.table_of(rng, [longest, longest], P)
    pools = [torch.from_numpy(rng.standard_normal((n_pages, H, P, d_h), dtype=np.float32)).to(KV[kv]).cuda() for _ in range(2)]
    pages, lengths, new = i32(table), i32([longest, 300]), i32([T, T // 2])
    cache = ph.PagedCache(pools[0], pools[1], pages, d_h)
    q = queries(rng, (2, T, H, d_h), rows)
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    sizes = ph.photon_paged_attn_workspace_bytes(cache, 2, T, H, None, 2)
    ws, other = (torch.empty(sizes, dtype=torch.uint8, device="cuda") for _ in range(2))

    def call(to, workspace):
        ph.photon_paged_attn(q, cache, lengths, to, n_new=new, n_splits=2, workspace=workspace)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(out, ws)
    for step in range(4):
        lengths.copy_(i32([longest - 37 * step, 300 - 90 * step]))
        pages.copy_(i32(table[:, ::-1].copy() if step % 2 else table))
        q.copy_(queries(rng, (2, T, H, d_h), rows))
        out.fill_(5.0)
        again.fill_(5.0)
        graph.replay()
        call(again, other)
        torch.cuda.synchronize()
        assert torch.equal(out, again) and not (out == 0).all()
