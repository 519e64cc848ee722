"""Softmax weights of the attention over a 4-bit cache: bf16 rows round the result, not the weights.

Two entries whose values are +1 and -1 share all of the weight, their scores 0 and -a apart with a = 2^-13 .. 2^-11; the other entries
lie 2^8 below.  The result (1 - e^-a) / (1 + e^-a) is at most 2^-12, and what its own rounding (half a step, 2^-8 of it) hides is
2^-20: an error of a weight shows.  Scores are exact (one product by a power of two, scale 1).  What fp32 adds: -a log2 e is off by
2^-24 of it, the exponential by 2^-23 of itself, the two sums by 2^-24 each and the quotient by 2 * 2^-24: less than 2^-21 of
sum(p |v|) = 1 in all; factors that put waves and splits together are off by 2^-23 each, another 2^-21.  2^-19 has room for both."""
import numpy as np
import pytest
import torch

from util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_splits", [1, 2])
@pytest.mark.parametrize("d_h", [32, 52, 128])
@pytest.mark.parametrize("T,H,H_kv", [(1, 16, 16), (2, 8, 4), (4, 8, 4), (1, 9, 1), (3, 9, 3)])
def test_weights_keep_all_of_their_bits(T, H, H_kv, d_h, n_splits):
    require_gpu()
    import paper_2512_20687_amd as ph
    Bt, n = 4, 1100
    rng = np.random.default_rng(d_h * T + H)
    a = torch.from_numpy((2.0 ** rng.uniform(-13, -11, (Bt, T, H))).astype(np.float32)).bfloat16()
    q = torch.zeros(Bt, T, H, d_h, dtype=torch.bfloat16)
    q[..., 0], q[..., 1] = a, 1
    k, v = torch.zeros(Bt, n, H_kv, d_h), torch.from_numpy(rng.standard_normal((Bt, n, H_kv, d_h)).astype(np.float32))
    k[..., 1] = -256.0
    one, other = 70, 101                                              # of one tile
    k[:, one] = k[:, other] = 0
    k[:, other, :, 0] = -1
    v[:, one], v[:, other] = 1, -1
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    kc, vc = ph.mxfp4_cache(Bt, H_kv, d_h, n), ph.mxfp4_cache(Bt, H_kv, d_h, n)
    ph.photon_mxfp4_cache_write(k, v, kc, vc)
    ws = torch.empty(max(ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, n_splits), 16), dtype=torch.uint8, device="cuda")
    lens = torch.full((Bt,), n, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ph.photon_mxfp4_decode_attn(q, kc, vc, lens, out, scale=1.0, n_splits=n_splits, workspace=ws)
    ref = np.tanh(a.double().numpy() / 2)[..., None]
    err = np.abs(out.double().cpu().numpy() - ref)
    bound = 2.0 ** -8 * ref + 2.0 ** -19
    assert np.all(err <= bound), float((err / bound).max())
