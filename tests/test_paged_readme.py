"""The README's example of a paged cache, run as it stands there."""
import os
import types

import numpy as np
import pytest
import torch

import paged_plain as plain
from util import require_gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
P, D_H, H, H_KV, BT, T = 64, 128, 4, 2, 2, 5


def example():
    lines = open(README).read().splitlines()
    first = next(i for i, l in enumerate(lines) if "ph.PagedCache(" in l)
    block = []
    for line in lines[first:]:
        if not line.startswith("    "):
            break
        block.append(line.strip())
    return block


def names(device):
    i32 = dict(dtype=torch.int32, device=device)
    masks, depth = plain.tree_masks([-1, 0, 0, 2, 2])
    return dict(n_pages=8, H_kv=H_KV, d_h=D_H, T=T, page_table=torch.arange(8, **i32).view(BT, 4), lengths=torch.tensor([100, 3], **i32),
                depth=torch.tensor(depth, **i32)[None], masks=torch.tensor(np.stack([masks] * BT), device=device),
                path=torch.tensor([[0, 2, 4], [0, 1, 0]], **i32), accepted=torch.tensor([3, 2], **i32))


def test_its_pools_have_the_heads_they_are_for():
    import paper_2512_20687_amd as ph
    if not os.path.exists(ph.lib_path()):
        from paper_2512_20687_amd import build
        build.build(verbose=False)
    on_cpu = types.SimpleNamespace(PagedCache=ph.PagedCache, paged_pool=lambda *a, **k: ph.paged_pool(*a, device="cpu", **k))
    scope = dict(names("cpu"), ph=on_cpu)
    line = example()[0]
    exec(line.split("   #")[0], scope)
    cache = scope["cache"]
    assert (cache.page_size, cache.H_kv, cache.d_h, cache.S_max) == (P, H_KV, D_H, 4 * P)
    assert cache.k_pages.shape == (8, H_KV, P, D_H)


@pytest.mark.gpu
def test_it_runs():
    require_gpu()
    import paper_2512_20687_amd as ph
    scope = dict(names("cuda"), ph=ph)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((BT, T, h, D_H), generator=g, device="cuda").bfloat16() for h in (H, H_KV, H_KV))
    scope.update(q=q, k=k, v=v, out=torch.empty_like(q), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    block = example()
    assert len(block) == 4
    exec(block[0], scope)
    cache = scope["cache"]
    for pool in (cache.k_pages, cache.v_pages):
        pool.normal_(generator=g)
    was = [p.clone() for p in (cache.k_pages, cache.v_pages)]
    for line in block[1:3]:
        exec(line, scope)
    ks, vs = (plain.values(p) for p in (cache.k_pages, cache.v_pages))
    table, masks = scope["page_table"].cpu().numpy(), scope["masks"].cpu().numpy()
    for b, n in enumerate((100 + T, 3 + T)):
        kk, vv = plain.entries(ks, table[b], n, D_H), plain.entries(vs, table[b], n, D_H)
        for t in range(T):
            ref, size = plain.attended(q[b, t].float().cpu().numpy(), kk, vv, plain.seen(n, T, t, masks[b, t]), D_H ** -0.5)
            off = np.abs(scope["out"][b, t].float().cpu().numpy() - ref)
            assert (off <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size).all()
    before = cache.v_pages.clone()
    exec(block[3], scope)
    assert torch.equal(cache.v_pages[1, :, 36:39], before[1, :, [36, 38, 40]]) and torch.equal(cache.v_pages[4, :, 3:5], before[4, :, 3:5])
    assert torch.equal(cache.v_pages[0], was[1][0])
