"""The 4-bit cache without a GPU: the oracle's format pinned to its definition, the layout, what the entry points refuse."""
import ctypes
import itertools
import os

import numpy as np
import pytest
import torch

import mxfp4_layout as lay
from oracle import photon_oracle as po

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def lib():
    import paper_2512_20687_amd as ph
    if not os.path.exists(ph.lib_path()):
        from paper_2512_20687_amd import build
        build.build(verbose=False)
    return ph.load_library()


def test_e2m1_codes():
    v = po.mxfp4_decode(np.tile(np.arange(16, dtype=np.uint8), 2), np.array([127], np.uint8))
    np.testing.assert_array_equal(v[:8], MAGNITUDES)
    np.testing.assert_array_equal(v[8:16], -MAGNITUDES)
    for byte, x in ((0, 2.0 ** -127), (1, 2.0 ** -126), (254, 2.0 ** 127)):
        assert po.mxfp4_decode(np.full(32, 2, np.uint8), np.array([byte], np.uint8))[5] == x
    assert np.isnan(po.mxfp4_decode(np.zeros(32, np.uint8), np.array([255], np.uint8))).all()


def test_rounding_is_to_the_nearest_value_of_the_block():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 32)) * 2.0 ** rng.integers(-120, 120, (200, 1))
    codes, scales = po.mxfp4_encode(x)
    got = po.mxfp4_decode(codes, scales)
    for row, byte, g in zip(x, scales[:, 0], got):
        X = 2.0 ** (int(byte) - 127)
        assert 4 * X <= np.abs(row).max() < 8 * X                    # the largest value lies in the top binade, 4 .. 8
        grid = np.concatenate([-MAGNITUDES, MAGNITUDES]) * X
        for a, b in zip(np.clip(row, -6 * X, 6 * X), g):
            assert abs(a - b) == np.abs(grid - a).min()
    # ties go to the even code: the block's 4 keeps the scale at 1
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 4.0] + [0.0] * 23)
    np.testing.assert_array_equal(po.mxfp4_round(ties)[:9], [0, 1, 1, 2, 2, 4, 4, 6, 4])
    np.testing.assert_array_equal(po.mxfp4_round(-ties)[:9], [0, -1, -1, -2, -2, -4, -4, -6, -4])
    assert po.mxfp4_encode(np.full(32, 7.99))[1][0] == 127 and po.mxfp4_encode(np.full(32, 8.0))[1][0] == 128


def test_extreme_blocks():
    assert po.mxfp4_encode(np.zeros(32))[1][0] == 0 and not po.mxfp4_round(np.zeros(32)).any()
    tiny = np.zeros(32)
    tiny[3] = 2.0 ** -126                                            # below 4 * 2^-127: the scale stops at 2^-127
    assert po.mxfp4_encode(tiny)[1][0] == 0 and po.mxfp4_round(tiny)[3] == 2.0 ** -126
    assert po.mxfp4_encode(np.full(32, 3.4e38))[1][0] == 252         # the largest scale that fp32 values need
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[40] = bad
        r = po.mxfp4_round(x)
        np.testing.assert_array_equal(r[:32], 1.0)
        assert np.isnan(r[32:]).all()
    # a partial last block is its own block, filled with zeros
    x = np.arange(1.0, 53.0)
    np.testing.assert_array_equal(po.mxfp4_round(x)[32:], po.mxfp4_round(np.concatenate([x[32:], np.zeros(12)]))[:20])


@pytest.mark.parametrize("d_p,is_v", itertools.product([32, 64, 128], [False, True]))
def test_layout_is_a_bijection(d_p, is_v):
    at, shift, scale = lay.addresses(d_p, is_v)
    assert sorted((2 * at + shift // 4).ravel()) == list(range(64 * d_p))
    assert sorted(scale.ravel()) == list(range(32 * d_p, 32 * d_p + 2 * d_p))
    rng = np.random.default_rng(1)
    codes, scales = rng.integers(0, 16, (2, 128, d_p), np.uint8), rng.integers(0, 256, (2, 128, d_p // 32), np.uint8)
    back = lay.unpack(lay.pack(codes, scales, is_v), d_p, is_v)
    np.testing.assert_array_equal(back[0], codes)
    np.testing.assert_array_equal(back[1], scales)


def test_sizes(lib):
    assert [lib.photon_mxfp4_tile_bytes(d) for d in (1, 20, 32, 52, 64, 65, 128, 0, 129, -3)] == [1088, 1088, 1088, 2176, 2176, 4352, 4352, 0, 0, 0]
    assert lib.photon_mxfp4_cache_bytes(4, 32, 64, 8192) == 4 * 32 * 128 * 2176
    assert lib.photon_mxfp4_cache_bytes(1, 1, 60, 65) == 2 * 2176
    assert lib.photon_mxfp4_cache_bytes(4, 32, 128, 1 << 24) == 4 * 32 * (1 << 18) * 4352          # past 32 bits
    assert lib.photon_mxfp4_cache_bytes(0, 32, 64, 8192) == 0 and lib.photon_mxfp4_cache_bytes(4, 32, 129, 8192) == 0
    assert lib.photon_mxfp4_decode_attn_workspace_bytes(4, 2, 32, 52, 8) == 4 * 2 * 32 * 8 * 66 * 4
    assert lib.photon_mxfp4_decode_attn_workspace_bytes(4, 2, 32, 52, 1) == 0
    for shape in ((1, 1, 1, 1, 1), (4, 1, 32, 32, 8192), (256, 8, 32, 4, 2048), (1, 1, 1, 1, 1 << 30)):
        assert 1 <= lib.photon_mxfp4_decode_attn_auto_splits(*shape) <= 1024
    assert lib.photon_mxfp4_decode_attn_auto_splits(0, 1, 1, 1, 1) == 1


P, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 2)        # never dereferenced: validation fails first
Q = ctypes.c_void_p(1 << 21)
WRITE = dict(k=P, v=P, stride=128, kc=P, vc=Q, start=P, n=None, status=None, Bt=1, T=3, H=2, d=64, S=100, dt=0)
READ = dict(kc=P, vc=Q, start=P, n=None, k=P, v=P, stride=128, Bt=1, T=3, H=2, d=64, S=100, dt=0)
ATTN = dict(q=P, stride=256, kc=P, vc=Q, seq=P, n=None, out=P, Bt=1, T=3, H=4, H_kv=2, d=64, S=100, scale=0.1, splits=1, ws=None, ws_bytes=0, dt=0)


@pytest.mark.parametrize("change,code,text", [
    (dict(dt=2), -2, b"dtype 2"), (dict(dt=9), -2, b"dtype 9"), (dict(d=129, stride=999), -2, b"d_h=129"), (dict(d=0), -2, b"d_h=0"),
    (dict(Bt=-1), -1, b"Bt=-1"), (dict(T=-1), -1, b"T=-1"), (dict(H=0), -1, b"H_kv=0"), (dict(S=0), -1, b"S_max=0"),
    (dict(S=1 << 31), -2, b"S_max=2147483648"), (dict(k=None), -1, b"k and v"), (dict(v=None), -1, b"k and v"), (dict(k=ODD), -1, b"k and v"),
    (dict(vc=P), -1, b"a cache each"), (dict(kc=None), -1, b"caches"), (dict(vc=ODD), -1, b"caches"), (dict(stride=127), -1, b"row_stride=127"), (dict(stride=0), -1, b"row_stride=0"),
    (dict(Bt=1 << 16), -2, b"Bt=65536"), (dict(H=1 << 16, stride=1 << 30), -2, b"H_kv=65536"), (dict(H=60000, T=1 << 30, stride=1 << 30), -2, b"T=1073741824"),
    (dict(T=1 << 30), -2, b"T=1073741824"),
])
def test_write_and_read_refuse(lib, change, code, text):
    for fn, args in ((lib.photon_mxfp4_cache_write, WRITE), (lib.photon_mxfp4_cache_read, READ)):
        assert fn(*{**args, **change}.values(), None) == code, lib.photon_last_error()
        assert text in lib.photon_last_error()


@pytest.mark.parametrize("change,code,text", [
    (dict(dt=2), -2, b"dtype 2"), (dict(d=200, stride=999), -2, b"d_h=200"), (dict(H_kv=3), -1, b"H=4"), (dict(H=0), -1, b"H=0"), (dict(H_kv=0), -1, b"H_kv=0"),
    (dict(Bt=-2), -1, b"Bt=-2"), (dict(S=-5), -1, b"S_max=-5"), (dict(splits=-1), -1, b"n_splits=-1"), (dict(splits=1025), -1, b"n_splits=1025"),
    (dict(q=None), -1, b"q and out"), (dict(out=ODD), -1, b"q and out"), (dict(kc=ODD), -1, b"k_cache"), (dict(vc=None), -1, b"v_cache"),
    (dict(seq=None), -1, b"seq_len"), (dict(stride=255), -1, b"q_stride=255"), (dict(splits=4), -3, b"workspace"),
    (dict(splits=4, ws=P, ws_bytes=4 * 3 * 4 * 66 * 4 - 1), -3, b"workspace"), (dict(splits=4, ws=ODD, ws_bytes=1 << 20), -3, b"workspace"),
    (dict(Bt=1 << 16), -2, b"Bt=65536"), (dict(T=1 << 16), -2, b"T=65536"), (dict(H=1 << 16, stride=1 << 30), -2, b"H=65536"), (dict(vc=P), -1, b"a cache each"),
    (dict(T=65535, H=60000, H_kv=1, stride=1 << 30), -2, b"T=65535"),
])
def test_attention_refuses(lib, change, code, text):
    assert lib.photon_mxfp4_decode_attn(*{**ATTN, **change}.values(), None) == code, lib.photon_last_error()
    assert text in lib.photon_last_error()


def test_nothing_to_do_is_no_error(lib):
    for none in (dict(Bt=0), dict(T=0)):
        assert lib.photon_mxfp4_cache_write(*{**WRITE, **none, "k": None}.values(), None) == 0
        assert lib.photon_mxfp4_cache_read(*{**READ, **none, "k": None}.values(), None) == 0
        assert lib.photon_mxfp4_decode_attn(*{**ATTN, **none, "q": None}.values(), None) == 0


def test_binding_refuses(lib):
    """Argument checks of the binding that need no device: wrong shapes, types, strides, and memory that is not the device's."""
    import paper_2512_20687_amd as ph
    k = torch.zeros(2, 3, 4, 52)
    c = ph.mxfp4_cache(2, 4, 52, 100, device="cpu")
    assert c.shape == (2, 4, 2, 2176)
    i32 = torch.zeros(2, dtype=torch.int32)
    bad = [
        (k, k[:, :2], c, c), (k, k.bfloat16(), c, c), (k.half(), k.half(), c, c), (k[0], k[0], c, c),
        (k, k, c.float(), c), (k, k, c[0], c), (k, k, c[:1], c[:1]), (k, k, c[:, :2], c[:, :2]), (k, k, c, c[:, :, :1]), (k, k, c[..., :1088], c[..., :1088]),
        (k.transpose(1, 2), k.transpose(1, 2), c, c), (k, torch.zeros(2, 3, 8, 52)[:, :, :4], c, c), (torch.zeros(2, 6, 4, 52)[:, :3], torch.zeros(2, 6, 4, 52)[:, :3], c, c),
    ]
    for args in bad:
        with pytest.raises(ph.PhotonError):
            ph.photon_mxfp4_cache_write(*args)
        with pytest.raises(ph.PhotonError):
            ph.photon_mxfp4_cache_read(*args[2:], *args[:2])
    for start in (i32[:1], i32.long(), i32):                           # the last one: right in all, but not in device memory
        with pytest.raises(ph.PhotonError):
            ph.photon_mxfp4_cache_write(k, k, c, c, start=start)
    q = torch.zeros(2, 3, 8, 52)
    for args in ((q, c, c, i32, q[:, :2]), (q, c, c, i32, q.bfloat16()), (q, c, c, i32.long(), q), (q, c, c, None, q), (q[..., :20], c, c, i32, q[..., :20]),
                 (q, c, c, i32, q)):
        with pytest.raises(ph.PhotonError):
            ph.photon_mxfp4_decode_attn(*args)


def test_the_storage_type_is_accepted_where_it_is_one(lib):
    """Only a configuration's kv_dt with bf16 matrices; elsewhere it is no element type."""
    import paper_2512_20687_amd as ph
    import seeded_inputs as si
    from paper_2512_20687_amd import binding as b
    assert b.PHOTON_MXFP4 == 3
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "photon.h")).read()
    assert "PHOTON_MXFP4 = 3" in text
    assert lib.photon_coarse_decode_attn(P, P, P, P, P, 1, 2, 64, 16, 0.1, 1, None, 0, 3, None) == -2
    assert lib.photon_chunk_local_attn(P, P, P, P, 4, 4, 4, 0, 2, 64, 0.1, 3, None) == -2
    cfg = si.PhotonConfig(L=2, C=(4, 4), R=(1, 1), D=256, H=4, d_h=64, n_layers=2, d_ff=640, vocab=1024, dtype="bf16", kv_dtype="mxfp4")
    assert ph.photon_decode_step_workspace_bytes(cfg, 2, 100) > 0
    c = b._c_config(cfg)
    assert (c.dt, c.kv_dt) == (1, 3)
    c.dt = 0
    assert lib.photon_decode_step_workspace_bytes(ctypes.byref(c), 2, 100) == 0 and b"kv_dt=3" in lib.photon_last_error()
    c.dt = 1
    assert lib.photon_decode_step_workspace_bytes(ctypes.byref(c), 2, 1 << 31) == 0 and b"4-bit" in lib.photon_last_error()


def test_positions_past_the_last_whole_tile_of_31_bits_are_refused(lib):
    """Tiles end at a position that an int32 holds: S_max is at most 2^31 - 64, for the cache's calls and a step's."""
    import paper_2512_20687_amd as ph
    import seeded_inputs as si
    from paper_2512_20687_amd import binding as b
    most = (1 << 31) - 64
    c = b._c_config(si.PhotonConfig(L=2, C=(4, 4), R=(1, 1), D=256, H=4, d_h=64, n_layers=2, d_ff=640, vocab=1024, dtype="bf16", kv_dtype="mxfp4"))
    for S, ok in ((most, True), (most + 1, False), ((1 << 31) - 1, False)):
        for fn, args in ((lib.photon_mxfp4_cache_write, WRITE), (lib.photon_mxfp4_cache_read, READ), (lib.photon_mxfp4_decode_attn, ATTN)):
            assert fn(*{**args, "S": S, "T": 0}.values(), None) == (0 if ok else -2)
            assert ok or b"S_max=%d" % S in lib.photon_last_error()
        assert (lib.photon_decode_step_workspace_bytes(ctypes.byref(c), 2, S) > 0) == ok


def test_capacity_of_the_lower_levels_is_refused_too(lib):
    """A lower level's stream is a cache of its own: past 2^31 - 64 positions a hierarchical step and a prefill refuse it."""
    import paper_2512_20687_amd as ph
    import seeded_inputs as si
    from paper_2512_20687_amd import binding as b
    cfg = si.PhotonConfig(L=2, C=(4, 4), R=(1, 1), D=128, H=2, d_h=64, n_layers=1, d_ff=128, vocab=64, dtype="bf16", kv_dtype="mxfp4")
    model = ph.PhotonModel(cfg, si.make_weights(cfg, 3), device="cpu")
    at = P.value                                   # never dereferenced: there is no workspace, should the capacity pass
    state, hier = b._State(k_cache=at, v_cache=at, seq_len=at, x_top=at, carry=at, S_max=8), b._HierState()
    hier.k_cache[0] = hier.v_cache[0] = hier.seq_len[0] = at
    hier.S_cap[0] = (1 << 31) - 63
    b._register_step(lib)
    args = [ctypes.byref(x) for x in (model.c_cfg, model.c_weights, model.c_encoder_weights, state, hier)]
    assert lib.photon_hiergen_step(*args, 2, None, P, None, None) == -2, lib.photon_last_error()
    assert b"level 1" in lib.photon_last_error()
    assert lib.photon_prefill(*args, 2, P, 32, None, 0, None) == -2, lib.photon_last_error()
    assert b"level 1" in lib.photon_last_error()


def test_reading_back_needs_a_place_each(lib):
    """K and V read into the same rows would race."""
    assert lib.photon_mxfp4_cache_read(*READ.values(), None) == -1                                 # k and v are one pointer there
    assert b"k and v overlap" in lib.photon_last_error()
