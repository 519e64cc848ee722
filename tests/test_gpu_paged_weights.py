"""Weights of the paged attention keep their 24 bits, whatever rows and pages are.

Each row sees two entries whose weights are nearly alike and whose V is +1 and -1, behind or among others whose V is 0: the result is
the difference of two weights over the sum of all, some 2^-12 of their size, so that digits which a weight lost on its way into the
product with V stand out.

Tolerance.  With A = sum(p |v|): K and q have one element that is not 0, so a score is a product, rounded once, and once with log2 e:
2^-23 of at most 1; the exponential 2^-23; the parts of a weight hold all of it; waves' and splits' means and their weights take a
handful of roundings of 2^-24: less than 2^-20 * A in all.  A bf16 result is rounded once, 2^-8 of the value.  Weights of 16 or 17
bits are off by up to 2^-16."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from test_gpu_paged_attn import KV, i32
from test_gpu_paged_wide import Many
from util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["few streams", "many streams"])
def ph(request):
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m if request.param == "few streams" else Many(m, 64)


@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kv", list(KV))
@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("first,second", [(5, 9), (5, 40), (3, 230), (200, 130)])
def test_differences_of_weights(ph, rows, kv, T, first, second):
    rng = np.random.default_rng(100 * T + first)
    d_h, P, past, H = 64, 32, 250, 8
    n = past + T
    step = 2.0 ** -4 if kv == "e4m3" else 2.0 ** -8
    k, v = torch.zeros((10, 1, P, 64)), torch.zeros((10, 1, P, 64))
    k[..., 0] = -1.0
    for e, key, value in ((first, 1.0, 1.0), (second, 1.0 - step, -1.0), (77, 1.25, 0.0)):
        k[e // P, 0, e % P, 0] = key
        v[e // P, 0, e % P] = value
    pools = [x.to(torch.float8_e4m3fn).view(torch.uint8) if kv == "e4m3" else x.to(KV[kv]) for x in (k, v)]
    table = np.arange(10, dtype=np.int32)[None]
    cache = ph.PagedCache(pools[0].cuda(), pools[1].cuda(), i32(table), d_h)
    q = torch.zeros((1, T, H, d_h))
    q[..., 0] = torch.from_numpy(rng.uniform(0.2, 1.0, (1, T, H)).astype(np.float32)) * (2.0 ** -10 / step)
    q = q.to(rows)
    ks, vs = (plain.entries(plain.values(p), table[0], n, d_h) for p in pools)
    for splits in (1, 3):
        out = torch.empty_like(q, device="cuda")
        ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 1, T, H, None, splits) + 16, dtype=torch.uint8, device="cuda")
        ph.photon_paged_attn(q.cuda(), cache, i32([n]), out, scale=1.0, n_splits=splits, workspace=ws)
        got = out.float().cpu().numpy().astype(np.float64)
        for t in range(T):
            ref, size = plain.attended(q[0, t].float().numpy(), ks, vs, plain.seen(n, T, t), 1.0)
            bound = 2.0 ** -20 * size + (2.0 ** -8 * np.abs(ref) if rows == torch.bfloat16 else 0.0)
            off = np.abs(got[0, t] - ref)
            assert (off <= bound).all(), (splits, t, (off / size).max())
