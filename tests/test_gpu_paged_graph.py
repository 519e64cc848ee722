"""Captured calls of the paged attention, replayed with other lengths, counts, pages and queries: every replay against the float64 definition,
rows behind a sequence's count as they were.  Tolerances as in tests/test_gpu_paged_attn.py."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from test_gpu_paged_attn import KV, i32
from util import require_gpu

pytestmark = pytest.mark.gpu
FILL = 5.0


@pytest.mark.parametrize("rows,kv,T,H", [(torch.bfloat16, "bf16", 70, 90), (torch.bfloat16, "bf16", 140, 70), (torch.float32, "bf16", 40, 90), (torch.bfloat16, "e4m3", 1, 6),
                                         (torch.float32, "f32", 3, 4)])
def test_replays(rows, kv, T, H):
    require_gpu()
    import paper_2512_20687_amd as ph
    rng = np.random.default_rng(T + H)
    P, d_h, longest = 16, 128, 400
    table, n_pages = plain.table_of(rng, [longest, longest], P)
    x = [torch.from_numpy(rng.standard_normal((n_pages, H, P, d_h), dtype=np.float32)) for _ in range(2)]
    pools = [(p.to(torch.float8_e4m3fn).view(torch.uint8) if kv == "e4m3" else p.to(KV[kv])).cuda() for p in x]
    values = [plain.values(p) for p in pools]
    pages, lengths, new = i32(table), i32([longest, 300]), i32([T, T])
    cache = ph.PagedCache(pools[0], pools[1], pages, d_h)
    q = torch.zeros((2, T, H, d_h), dtype=rows, device="cuda")
    out = torch.zeros_like(q)
    ws = torch.empty(ph.photon_paged_attn_workspace_bytes(cache, 2, T, H, None, 2), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ph.photon_paged_attn(q, cache, lengths, out, n_new=new, n_splits=2, workspace=ws)
    for step in range(4):
        now, counts = [longest - 37 * step, 300 - 90 * step], [T, T - T * step // 4]
        where = table[:, ::-1].copy() if step % 2 else table
        given = torch.from_numpy(rng.standard_normal((2, T, H, d_h)).astype(np.float32)).to(rows)
        lengths.copy_(i32(now))
        new.copy_(i32(counts))
        pages.copy_(i32(where))
        q.copy_(given)
        out.fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        got = out.float().cpu().numpy().astype(np.float64)
        heads = [0, H // 2, H - 1]
        for b in range(2):
            assert (got[b, counts[b]:] == FILL).all()
            ks, vs = (plain.entries(p, where[b], now[b], d_h)[heads] for p in values)
            for t in range(counts[b]):
                ref, size = plain.attended(given[b, t, heads].float().numpy(), ks, vs, plain.seen(now[b], counts[b], t), d_h ** -0.5)
                bound = 1e-5 * max(size.max(), 1e-30) if rows == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
                assert (np.abs(got[b, t, heads] - ref) <= bound).all(), (step, b, t)
        assert (got[0, : counts[0]] != FILL).any(-1).all()                 # every head of every row was written
