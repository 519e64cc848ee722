"""Steps on 4-bit caches so long that the attention splits a stream: partial results in the step's workspace and their merge, with
few rows and with many (bf16 results), joined, pipelined and captured, and at the lower level of the hierarchical schedule."""
import numpy as np
import pytest
import torch

import seeded_inputs as si
from oracle import photon_oracle as po
from test_gpu_mxfp4_step import check_entries, entries, make_state, start
from util import TOL, dev, nerr, require_gpu

pytestmark = pytest.mark.gpu
SMALL = dict(L=2, C=(4, 4), R=(1, 1), D=128, H=2, d_h=64, n_layers=1, d_ff=256, vocab=256, dtype="bf16", kv_dtype="mxfp4")


def merges(ph, call):
    """Merges of partial results that the call launches."""
    torch.cuda.synchronize()
    ph.photon_profile_reset()
    ph.photon_profile_enable(True)
    call()
    torch.cuda.synchronize()
    ph.photon_profile_enable(False)
    n = ph.photon_profile_get().get("coarse_merge_kernel", (0, 0))[0]
    ph.photon_profile_reset()
    return n


@pytest.mark.parametrize("kw,Bt,S,S_max", [(dict(n_layers=2), 2, 4300, 4352), (dict(D=832, H=16, d_h=52, d_ff=1024), 1, 6200, 6300), (dict(), 20, 4300, 4352),
                                           (dict(D=128, H=1, d_h=128), 17, 4200, 4300)])
def test_step_whose_attention_is_split(kw, Bt, S, S_max):
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**{**SMALL, **kw})
    w = si.make_weights(cfg, 45)
    st = start(cfg, Bt, S, S_max, 5, uneven=S // Bt)                  # the last sequence is a short one
    forced = si.make_tokens(cfg.vocab, Bt, cfg.meta_context, 9)
    ost = po.state_to_f64(st)
    s0 = ost["seq_len"].copy()
    otr = po.decode_step(cfg, po.weights_to_f64(w), ost, forced_tokens=forced)
    model = ph.PhotonModel(cfg, w)
    state = make_state(ph, model, st, Bt, S_max, cfg.d_h)
    trace = {"logits": torch.full((Bt, cfg.meta_context, cfg.vocab), float("nan"), device="cuda")}
    toks = torch.full((Bt, cfg.meta_context), -1, dtype=torch.int32, device="cuda")
    n = merges(ph, lambda: ph.photon_decode_step(model, state, toks, forced_tokens=dev(np.asarray(forced, np.int32)), trace=trace))
    assert n == cfg.n_layers
    errs = {"logits": nerr(trace["logits"], otr["logits"]), "x_top": nerr(state.x_top, otr["x_top"]), "carry": nerr(state.carry, ost["carry"])}
    assert all(v <= TOL["bf16"] for v in errs.values()), errs
    for got, ref, is_v in ((state.k, ost["k"], False), (state.v, ost["v"], True)):
        g = entries(got, cfg.d_h, is_v)
        check_entries(np.stack([g[:, b, :, s0[b]] for b in range(Bt)], 1), np.stack([ref[:, b, :, s0[b]] for b in range(Bt)], 1))
        for b in range(Bt):
            np.testing.assert_array_equal(g[:, b, :, : s0[b]], ref[:, b, :, : s0[b]])
    np.testing.assert_array_equal(state.seq_len.cpu().numpy(), s0 + 1)


@pytest.mark.parametrize("Bt", [2, 18])
def test_split_steps_pipelined_and_captured_are_the_same(Bt):
    """Four steps joined one by one, pipelined (a second stream beside the update), and as replays with the workspace's and other eager
    work between: the same bits."""
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**SMALL)
    w = si.make_weights(cfg, 46)
    S, S_max, steps = 4300, 4352, 4
    st = start(cfg, Bt, S, S_max, 6, uneven=90)
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
        elif how == "joined":
            for t in toks:
                assert merges(ph, lambda: ph.photon_decode_step(model, state, t)) == cfg.n_layers
        else:
            for t in toks:
                ph.photon_decode_step(model, state, t)
            ph.photon_decode_join(state)
        torch.cuda.synchronize()
        results.append([state.x_top, state.k, state.v, state.carry] + toks)
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


def test_hierarchical_step_whose_lower_level_is_split():
    """Several units per sequence over a lower level's stream of 1200 entries in a cache for 4240: the top level's is not split."""
    require_gpu()
    import paper_2512_20687_amd as ph
    cfg = si.PhotonConfig(**{**SMALL, "vocab": 1024})                # partial results lie where the logits will: 8 x 1024 hold two splits of them
    w = si.make_weights(cfg, 47)
    Bt, T, S_max = 2, 16 * 300, 1060
    toks = si.make_tokens(cfg.vocab, Bt, T, 6)
    w64 = po.weights_to_f64(w)
    ost = po.hier_prefill(cfg, w64, toks, S_max)
    model = ph.PhotonModel(cfg, w)
    state, hier = ph.PhotonState(model, Bt, S_max), ph.PhotonHierState(model, Bt, S_max)
    ph.photon_prefill(model, state, dev(np.asarray(toks, np.int32)), hier=hier)
    forced = si.make_tokens(cfg.vocab, Bt, cfg.meta_context, 9)
    otr = po.hiergen_step(cfg, w64, ost, forced_tokens=forced)
    out = torch.full((Bt, cfg.meta_context), -1, dtype=torch.int32, device="cuda")
    logits = torch.full((Bt, cfg.meta_context, cfg.vocab), float("nan"), device="cuda")
    n = merges(ph, lambda: ph.photon_hiergen_step(model, state, hier, out, forced_tokens=dev(np.asarray(forced, np.int32)), trace={"logits": logits}))
    assert n == cfg.n_layers
    assert nerr(logits, otr["logits"]) <= TOL["bf16"]
    assert nerr(state.x_top, otr["x_top"]) <= TOL["bf16"]
    n = T // cfg.C[0] + cfg.C[1]
    assert hier.seq_len[0].tolist() == [n] * Bt
    for got, ref, is_v in ((hier.k[0], ost["enc_k"][0], False), (hier.v[0], ost["enc_v"][0], True)):
        check_entries(entries(got, cfg.d_h, is_v)[:, :, :, :n], ref[:, :, :, :n])
