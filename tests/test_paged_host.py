"""The paged cache without a GPU: what its entry points refuse, sizes, and the plain definitions that its GPU tests compare with."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paged_plain as plain

P = 1 << 22                          # an address that is never dereferenced: validation fails first
BIG = 1 << 34                        # a second pool, far from the first


@pytest.fixture(scope="module")
def ph():
    import paper_2512_20687_amd as m
    if not os.path.exists(m.lib_path()):
        from paper_2512_20687_amd import build
        build.build(verbose=False)
    m.load_library()
    return m


def cache(ph, **change):
    from paper_2512_20687_amd import binding as b
    f = dict(k_pages=P, v_pages=BIG, page_table=P + 4, n_pages=8, page_size=16, max_pages=4, H_kv=2, d_h=64, kv_dt=1)
    f.update(change)
    return b._PagedCache(*[f[n] for n, _ in b._PagedCache._fields_])


def write(ph, c, k=P, v=P, stride=128, q=None, q_stride=0, q_out=None, out_stride=0, Bt=1, T=1, H=0, theta=0.0, dt=1):
    return ph.load_library().photon_paged_cache_write(None if c is None else ctypes.byref(c), k, v, stride, q, q_stride, q_out, out_stride, None, None,
                                                      None, None, Bt, T, H, theta, dt, None)


def attend(ph, c, q=P, q_stride=256, seq_len=P, tree=None, out=P, Bt=1, T=1, H=4, S_max=64, splits=1, ws=None, ws_bytes=0, dt=1):
    return ph.load_library().photon_paged_attn(None if c is None else ctypes.byref(c), q, q_stride, seq_len, None, tree, out, None, Bt, T, H, S_max,
                                               0.125, splits, ws, ws_bytes, dt, None)


def move(ph, c, source=P, Bt=1, T=1):
    return ph.load_library().photon_paged_cache_move(None if c is None else ctypes.byref(c), None, source, None, None, Bt, T, None)


@pytest.mark.parametrize("call", [write, attend, move])
@pytest.mark.parametrize("change,code,message", [
    (dict(kv_dt=3), -2, b"pages are fp32, bf16 or E4M3"), (dict(kv_dt=9), -2, b"dtype 9"),
    (dict(H_kv=0), -1, b"H_kv=0"), (dict(n_pages=0), -1, b"n_pages=0"), (dict(max_pages=0), -1, b"max_pages=0"),
    (dict(d_h=0), -2, b"d_h=0"), (dict(d_h=129), -2, b"d_h=129"),
    (dict(page_size=0), -2, b"page_size=0"), (dict(page_size=8), -2, b"page_size=8"), (dict(page_size=48), -2, b"page_size=48"), (dict(page_size=512), -2, b"page_size=512"),
    (dict(max_pages=1 << 27), -2, b"2^31 - 256"), (dict(k_pages=None), -1, b"pools must be"), (dict(v_pages=P + 8), -1, b"pools must be"),
    (dict(page_table=None), -1, b"page_table"), (dict(page_table=P + 2), -1, b"page_table"),
    (dict(v_pages=P), -1, b"overlap"), (dict(v_pages=P + 8 * 2 * 16 * 128 - 16), -1, b"overlap"), (dict(v_pages=P - 16), -1, b"overlap"),
])
def test_caches_that_are_refused(ph, call, change, code, message):
    assert call(ph, cache(ph, **change)) == code
    assert message in ph.load_library().photon_last_error()


@pytest.mark.parametrize("call", [write, attend, move])
def test_no_cache_and_nothing_to_do(ph, call):
    assert call(ph, None) == -1
    assert call(ph, cache(ph), Bt=0) == 0 and call(ph, cache(ph), T=0) == 0
    assert call(ph, cache(ph), Bt=-1) == -1 and call(ph, cache(ph), T=-1) == -1 and call(ph, cache(ph), Bt=65536) == -2


@pytest.mark.parametrize("args,code,message", [
    (dict(k=None), -1, b"k and v"), (dict(v=P + 1), -1, b"k and v"), (dict(stride=127), -1, b"row_stride=127"), (dict(dt=2), -2, b"dtype 2"),
    (dict(q=P), -1, b"go together"), (dict(q_out=P), -1, b"go together"), (dict(q=P, q_out=P, q_stride=256, out_stride=256), -1, b"H=0"),
    (dict(q=P, q_out=BIG, q_stride=255, out_stride=256, H=4), -1, b"q_stride=255"), (dict(q=P, q_out=BIG, q_stride=256, out_stride=255, H=4), -1, b"q_out_stride=255"),
    (dict(q=P, q_out=P, q_stride=256, out_stride=512, H=4), -1, b"in place"), (dict(q=P + 1, q_out=P, q_stride=256, out_stride=256, H=4), -1, b"whole elements"),
    (dict(theta=0.5), -1, b"rope_theta"), (dict(theta=-1.0), -1, b"rope_theta"), (dict(theta=float("nan")), -1, b"rope_theta"), (dict(theta=float("inf")), -1, b"rope_theta"),
    (dict(T=1 << 30), -2, b"too many"),
])
def test_writes_that_are_refused(ph, args, code, message):
    assert write(ph, cache(ph), **args) == code
    assert message in ph.load_library().photon_last_error()


def test_odd_heads_do_not_rotate(ph):
    assert write(ph, cache(ph, d_h=63), theta=10000.0) == -2
    assert b"odd" in ph.load_library().photon_last_error()


@pytest.mark.parametrize("args,code,message", [
    (dict(q=None), -1, b"q and out"), (dict(out=P + 1), -1, b"q and out"), (dict(seq_len=None), -1, b"seq_len"), (dict(q_stride=255), -1, b"q_stride=255"),
    (dict(H=3), -1, b"H=3"), (dict(H=0), -1, b"H=0"), (dict(S_max=0), -1, b"S_max=0"), (dict(S_max=65), -1, b"S_max=65"), (dict(splits=-1), -1, b"n_splits=-1"),
    (dict(splits=1025), -1, b"n_splits=1025"), (dict(tree=P, T=65), -2, b"tree of T=65"), (dict(T=65536), -2, b"T=65536"), (dict(dt=2), -2, b"dtype 2"),
    (dict(splits=2), -3, b"workspace of 2112 bytes"), (dict(splits=2, ws=P, ws_bytes=2111), -3, b"got 2111"), (dict(splits=2, ws=P + 8, ws_bytes=4096), -3, b"16-byte aligned"),
    (dict(T=65535, H=65534, q_stride=1 << 40, splits=1024, ws=P, ws_bytes=1 << 62), -2, b"too many workgroups"),
])
def test_attentions_that_are_refused(ph, args, code, message):
    assert attend(ph, cache(ph), **args) == code
    assert message in ph.load_library().photon_last_error()


def test_moves_that_are_refused(ph):
    assert move(ph, cache(ph), T=65) == -2 and b"T=65" in ph.load_library().photon_last_error()
    assert move(ph, cache(ph), source=None) == -1 and b"from is null" in ph.load_library().photon_last_error()


def test_workspace_bytes(ph):
    size = lambda c, *a: ph.load_library().photon_paged_attn_workspace_bytes(ctypes.byref(c), *a)  # noqa: E731
    c = cache(ph)
    assert size(c, 2, 3, 4, 64, 5) == 2 * 3 * 4 * 5 * 66 * 4 and size(cache(ph, d_h=52), 2, 3, 4, 64, 5) == 2 * 3 * 4 * 5 * 66 * 4
    assert size(c, 2, 3, 4, 64, 1) == 0 and size(c, 0, 3, 4, 64, 5) == 0 and size(c, 256, 1, 4, 64, 0) == 0
    assert size(c, 1, 1, 4, 1 << 20, 0) > 0                          # few streams, long ones: split
    assert ph.load_library().photon_paged_attn_workspace_bytes(None, 2, 3, 4, 64, 5) == 0


def test_the_binding_refuses_what_does_not_fit(ph):
    from paper_2512_20687_amd import binding as b
    pool = lambda **c: torch.zeros((4, 2, 16, 64), **c)  # noqa: E731
    table = torch.zeros((1, 4), dtype=torch.int32)
    c = b.PagedCache(pool(), pool(), table, 52)
    assert (c.H_kv, c.page_size, c.S_max, c.Bt) == (2, 16, 64, 1)
    for bad in ((pool(), pool(), table, 65), (pool(), pool(dtype=torch.bfloat16), table, 64), (pool(), pool()[:2], table, 64), (pool()[:, :, ::2], pool()[:, :, ::2], table, 64),
                (pool(), pool(), table.long(), 64), (pool(), pool(), table[0], 64), (pool(dtype=torch.float16), pool(dtype=torch.float16), table, 64)):
        with pytest.raises(b.PhotonError):
            b.PagedCache(*bad)
    k = torch.zeros(1, 3, 2, 52)
    q = torch.zeros(1, 3, 4, 52)
    for args in ((k, k[:, :2], c), (k, k.bfloat16(), c), (k[..., :50], k[..., :50], c), (k[:, :, :1], k[:, :, :1], c), (k.half(), k.half(), c), (k.expand(2, 3, 2, 52), k, c)):
        with pytest.raises(b.PhotonError):
            b.photon_paged_cache_write(*args)
    for kw in (dict(q=q), dict(q=q, q_out=q.bfloat16()), dict(q=q[:, :2], q_out=q[:, :2]), dict(position=torch.zeros(1, 3)), dict(position=torch.zeros((3, 1), dtype=torch.int32)),
               dict(start=torch.zeros(1)), dict(n_new=torch.zeros(2, dtype=torch.int32)), dict(status=torch.zeros(1)), {}):          # the last: not on a GPU
        with pytest.raises(b.PhotonError):
            b.photon_paged_cache_write(k, k, c, **kw)
    n = torch.zeros(1, dtype=torch.int32)
    for args, kw in (((q, c, None, q), {}), ((q, c, n, q[:, :2]), {}), ((q, c, n, q.bfloat16()), {}), ((q, c, n, q.transpose(1, 2).contiguous().transpose(1, 2)), {}),
                     ((q, c, n, q), dict(tree=torch.zeros((1, 3), dtype=torch.int32))), ((q, c, n, q), dict(tree=torch.zeros((1, 2), dtype=torch.int64))), ((q, c, n, q), {})):
        with pytest.raises(b.PhotonError):
            b.photon_paged_attn(*args, **kw)
    for args in ((c, n, torch.zeros((1, 3))), (c, n, torch.zeros((2, 3), dtype=torch.int32)), (c, n, torch.zeros((1, 3), dtype=torch.int32))):
        with pytest.raises(b.PhotonError):
            b.photon_paged_cache_move(*args)


def test_plain_definitions():
    """The float64 side against cases that can be told by hand."""
    x = np.arange(8.0).reshape(1, 1, 8)
    np.testing.assert_array_equal(plain.rotated(x, [0], 10000.0), x)
    r = plain.rotated(x, [1], 1.0)                                    # every pair by one radian
    np.testing.assert_allclose(r[0, 0, :4] ** 2 + r[0, 0, 4:] ** 2, x[0, 0, :4] ** 2 + x[0, 0, 4:] ** 2)
    np.testing.assert_allclose(r[0, 0, 0], -4 * np.sin(1.0))
    assert plain.seen(5, 3, 0).tolist() == [True, True, True, False, False]
    assert plain.seen(5, 3, 2, 0b101).tolist() == [True, True, True, False, True]
    assert plain.seen(2, 3, 1).tolist() == [True, False] and plain.seen(2, 3, 0).tolist() == [False, False]
    masks, depth = plain.tree_masks([-1, 0, 0, 2])
    assert masks.tolist() == [1, 3, 5, 13] and depth.tolist() == [0, 1, 1, 2]
    assert plain.tree_masks(list(range(-1, 63)))[0][63] == -1         # 64 nodes: all bits
    k = np.zeros((1, 3, 2))
    v = np.array([[[1.0, 0], [3.0, 2], [np.nan, np.inf]]])
    out, size = plain.attended(np.ones((2, 2)), k, v, np.array([True, True, False]), 1.0)
    np.testing.assert_array_equal(out, [[2, 1], [2, 1]])
    table, n = plain.table_of(np.random.default_rng(0), [17, 0, 32], 16)
    assert n == 6 and (table >= 0).sum() == 4 and table.shape == (3, 2) and len(set(table[table >= 0].tolist())) == 4
