"""How many splits a call takes by itself: one workgroup per compute unit, counted as the rows' type groups the queries (bf16 by eight,
fp32 by four)."""
import pytest
import torch

from util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,own,other", [(torch.float32, 2, 4), (torch.bfloat16, 4, 2)])
def test_splits_follow_the_workgroups_of_a_type(dtype, own, other):
    """64 streams of 128 tiles with eight queries each: 64 workgroups a split, or 128."""
    require_gpu()
    import paper_2512_20687_amd as ph
    Bt, H, H_kv, d_h, S = 8, 64, 8, 32, 8192
    g = torch.Generator(device="cuda").manual_seed(3)
    kc, vc = ph.mxfp4_cache(Bt, H_kv, d_h, S), ph.mxfp4_cache(Bt, H_kv, d_h, S)
    k, v = (torch.randn(Bt, S, H_kv, d_h, generator=g, device="cuda").bfloat16() for _ in range(2))
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    q = torch.randn(Bt, 1, H, d_h, generator=g, device="cuda").to(dtype)
    lens = torch.full((Bt,), S, dtype=torch.int32, device="cuda")
    most = ph.photon_mxfp4_decode_attn_auto_splits(Bt, 1, H, H_kv, S)
    assert most == 4
    ws = torch.empty(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, 1, H, d_h, most), dtype=torch.uint8, device="cuda")
    outs = [ph.photon_mxfp4_decode_attn(q, kc, vc, lens, torch.empty_like(q), n_splits=n, workspace=ws) for n in (0, own, other)]
    assert torch.equal(outs[0], outs[1])
    assert not torch.equal(outs[0], outs[2])
