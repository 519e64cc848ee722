"""Decode steps, the prefill and the hierarchical schedule on coarse caches in 4 bits (kv_dtype "mxfp4"), against the oracle with the
same storage.

Stored entries are the roundings of values that the step forms with bf16 rows upstream (a few 1e-3 off the oracle's): equal codes
but where a value lies that near to a border between two codes, which are 17 - 50 % apart (a few per cent of the elements), or a
block's largest value that near to a power of two (its scale doubles).  Either moves a value by at most half of the block's
largest: the widest step, 4 to 6 times the scale, is half of 4, the least that the largest can be."""
import numpy as np
import pytest
import torch

import mxfp4_layout as lay
import seeded_inputs as si
from oracle import photon_oracle as po
from util import TOL, dev, nerr, require_gpu

pytestmark = pytest.mark.gpu
BASE = dict(L=2, C=(4, 4), R=(1, 1), D=256, H=4, d_h=64, n_layers=2, d_ff=640, vocab=1024, dtype="bf16", kv_dtype="mxfp4")


def tiles(values, d_h, is_v):
    """Entries [..., S, d_h], representable, as cache bytes."""
    S = values.shape[-2]
    pad = [(0, 0)] * (values.ndim - 2) + [(0, -S % 64), (0, lay.row_elems(d_h) - d_h)]
    return lay.pack(*po.mxfp4_encode(np.pad(values, pad)), is_v)


def entries(cache, d_h, is_v):
    """Cache bytes (tensor) as values [..., positions, d_h]."""
    return po.mxfp4_decode(*lay.unpack(cache.cpu().numpy(), lay.row_elems(d_h), is_v))[..., :d_h]


def check_entries(got, ref):
    """Rows [..., d_h] of stored values: see above."""
    d_h = ref.shape[-1]
    pad = [(0, 0)] * (ref.ndim - 1) + [(0, -d_h % 32)]
    g, r = (np.pad(a, pad).reshape(a.shape[:-1] + (-1, 32)) for a in (got, ref))
    top = np.maximum(np.abs(g), np.abs(r)).max(-1, keepdims=True)
    assert np.all(np.abs(g - r) <= 0.5 * top * (1 + 2.0 ** -20))
    assert (got == ref).mean() >= 0.9, (got == ref).mean()


def start(cfg, Bt, S, S_max, seed, uneven=11):
    st = si.make_decode_state(cfg, Bt, S, S_max, seed=seed)
    st["seq_len"] = np.array([S - uneven * b for b in range(Bt)], np.int32)
    st["k"], st["v"] = po.mxfp4_round(st["k"]), po.mxfp4_round(st["v"])
    return st


def make_state(ph, model, st, Bt, S_max, d_h, **kw):
    return ph.PhotonState(model, Bt, S_max, k=tiles(st["k"], d_h, False), v=tiles(st["v"], d_h, True), seq_len=st["seq_len"],
                          x_top=np.asarray(st["x_top"], np.float32), carry=np.asarray(st["carry"], np.float32), **kw)


@pytest.mark.parametrize("kw,Bt", [(dict(), 3), (dict(D=832, H=16, d_h=52, d_ff=1024, R=(2, 2), n_layers=1), 2),
                                   (dict(D=256, H=2, d_h=128, n_layers=1), 2), (dict(n_layers=1), 24)])
def test_step_on_a_4bit_cache(kw, Bt):
    """Few rows and many (bf16 attention rows, projections in parts), head sizes of 52, 64 and 128."""
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**{**BASE, **kw})
    w = si.make_weights(cfg, 35)
    S, S_max = 300, 330
    st = start(cfg, Bt, S, S_max, 7)
    forced = si.make_tokens(cfg.vocab, Bt, cfg.meta_context, 9)
    ost = po.state_to_f64(st)
    s0 = ost["seq_len"].copy()
    otr = po.decode_step(cfg, po.weights_to_f64(w), ost, forced_tokens=forced)
    model = ph.PhotonModel(cfg, w)
    state = make_state(ph, model, st, Bt, S_max, cfg.d_h)
    B = cfg.meta_context
    trace = {"logits": torch.full((Bt, B, cfg.vocab), float("nan"), device="cuda"), "a_hat": torch.full((Bt, cfg.D), float("nan"), device="cuda")}
    toks = torch.full((Bt, B), -1, dtype=torch.int32, device="cuda")
    ph.photon_decode_step(model, state, toks, forced_tokens=dev(np.asarray(forced, np.int32)), trace=trace)
    torch.cuda.synchronize()
    errs = {"logits": nerr(trace["logits"], otr["logits"]), "a_hat": nerr(trace["a_hat"], otr["a_hat"]),
            "x_top": nerr(state.x_top, otr["x_top"]), "carry": nerr(state.carry, ost["carry"])}
    assert all(v <= TOL["bf16"] for v in errs.values()), errs
    for got, ref, is_v in ((state.k, ost["k"], False), (state.v, ost["v"], True)):
        g = entries(got, cfg.d_h, is_v)
        check_entries(np.stack([g[:, b, :, s0[b]] for b in range(Bt)], 1), np.stack([ref[:, b, :, s0[b]] for b in range(Bt)], 1))
        for b in range(Bt):
            np.testing.assert_array_equal(g[:, b, :, : s0[b]], ref[:, b, :, : s0[b]])      # nothing else is touched
            assert not g[:, b, :, S_max:].any()
    np.testing.assert_array_equal(state.seq_len.cpu().numpy(), s0 + 1)


def test_pipelined_and_captured_steps_are_the_same():
    """Three steps joined one by one, three pipelined ones, and three replays of a captured step: the same bits."""
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**BASE)
    w = si.make_weights(cfg, 36)
    Bt, S, S_max, steps = 2, 2100, 2120, 3
    st = start(cfg, Bt, S, S_max, 8, uneven=700)
    model = ph.PhotonModel(cfg, w)
    results = []
    for how in ("joined", "pipelined", "captured"):
        state = make_state(ph, model, st, Bt, S_max, cfg.d_h, pipeline=how == "pipelined")
        toks = [torch.full((Bt, cfg.meta_context), -1, dtype=torch.int32, device="cuda") for _ in range(steps)]
        if how == "captured":
            graph, tok = torch.cuda.CUDAGraph(), torch.empty_like(toks[0])
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                ph.photon_decode_step(model, state, tok)
            for t in toks:
                graph.replay()
                torch.cuda.synchronize()
                t.copy_(tok)
        else:
            for t in toks:
                ph.photon_decode_step(model, state, t)
            if how == "pipelined":
                ph.photon_decode_join(state)
        torch.cuda.synchronize()
        assert state.seq_len.tolist() == [S + steps, S - 700 + steps]
        results.append([state.x_top, state.k, state.v, state.carry] + toks)
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kw,Bt,T", [(dict(), 2, 16 * 90), (dict(D=832, H=16, d_h=52, d_ff=1024, R=(2, 2), n_layers=1), 1, 16 * 7)])
def test_prefill_into_a_4bit_cache_then_step(kw, Bt, T):
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**{**BASE, **kw})
    w = si.make_weights(cfg, 37)
    toks = si.make_tokens(cfg.vocab, Bt, T, 6)
    G = T // cfg.meta_context
    S_max = G + 4
    w64 = po.weights_to_f64(w)
    ost = po.prefill(cfg, w64, toks, S_max)
    model = ph.PhotonModel(cfg, w)
    state = ph.PhotonState(model, Bt, S_max)
    ph.photon_prefill(model, state, dev(np.asarray(toks, np.int32)))
    torch.cuda.synchronize()
    for got, ref, is_v in ((state.k, ost["k"], False), (state.v, ost["v"], True)):
        g = entries(got, cfg.d_h, is_v)
        check_entries(g[:, :, :, :G], ref[:, :, :, :G])
        assert not g[:, :, :, G:].any()
    assert nerr(state.x_top, ost["x_top"]) <= TOL["bf16"] and nerr(state.carry, ost["carry"]) <= TOL["bf16"]
    forced = si.make_tokens(cfg.vocab, Bt, cfg.meta_context, 9)
    otr = po.decode_step(cfg, w64, ost, forced_tokens=forced)
    out = torch.full((Bt, cfg.meta_context), -1, dtype=torch.int32, device="cuda")
    logits = torch.full((Bt, cfg.meta_context, cfg.vocab), float("nan"), device="cuda")
    ph.photon_decode_step(model, state, out, forced_tokens=dev(np.asarray(forced, np.int32)), trace={"logits": logits})
    torch.cuda.synchronize()
    assert nerr(logits, otr["logits"]) <= TOL["bf16"]
    assert nerr(state.x_top, otr["x_top"]) <= TOL["bf16"]


def test_hierarchical_step_on_4bit_caches():
    """Prefill of every level's stream and one step of the hierarchical schedule: several new units per sequence at the lower level."""
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**{**BASE, "n_layers": 1})
    w = si.make_weights(cfg, 38)
    Bt, T = 2, 16 * 40
    toks = si.make_tokens(cfg.vocab, Bt, T, 6)
    S_max = T // cfg.meta_context + 4
    w64 = po.weights_to_f64(w)
    ost = po.hier_prefill(cfg, w64, toks, S_max)
    model = ph.PhotonModel(cfg, w)
    state = ph.PhotonState(model, Bt, S_max)
    hier = ph.PhotonHierState(model, Bt, S_max)
    ph.photon_prefill(model, state, dev(np.asarray(toks, np.int32)), hier=hier)
    forced = si.make_tokens(cfg.vocab, Bt, cfg.meta_context, 9)
    otr = po.hiergen_step(cfg, w64, ost, forced_tokens=forced)
    out = torch.full((Bt, cfg.meta_context), -1, dtype=torch.int32, device="cuda")
    logits = torch.full((Bt, cfg.meta_context, cfg.vocab), float("nan"), device="cuda")
    ph.photon_hiergen_step(model, state, hier, out, forced_tokens=dev(np.asarray(forced, np.int32)), trace={"logits": logits})
    torch.cuda.synchronize()
    assert nerr(logits, otr["logits"]) <= TOL["bf16"]
    assert nerr(state.x_top, otr["x_top"]) <= TOL["bf16"]
    n = T // cfg.C[0] + cfg.C[1]
    assert hier.seq_len[0].tolist() == [n] * Bt
    for got, ref, is_v in ((hier.k[0], ost["enc_k"][0], False), (hier.v[0], ost["enc_v"][0], True)):
        check_entries(entries(got, cfg.d_h, is_v)[:, :, :, :n], ref[:, :, :, :n])
