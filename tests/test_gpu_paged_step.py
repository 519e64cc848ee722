"""Steps of drafted decoding over the paged cache as a program runs them: prompts are written, trees of drafted entries are written and
attended to, the accepted path is kept, and the next step goes on from it; eagerly and captured into a graph."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from util import require_gpu

pytestmark = pytest.mark.gpu
THETA = 10000.0


@pytest.fixture(scope="module")
def ph():
    require_gpu()
    import paper_2512_20687_amd as m
    m.load_library()
    return m


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Program:
    """Sequences in pages, and the same in float64: lists of rotated K and V as the pages hold them."""

    def __init__(self, ph, rng, Bt, H, H_kv, d_h, P, T, prompts, steps, dtype, kv):
        self.ph, self.rng, self.dtype = ph, rng, dtype
        self.Bt, self.H, self.H_kv, self.d_h, self.T = Bt, H, H_kv, d_h, T
        room = [n + (steps + 1) * T for n in prompts]
        table, n_pages = plain.table_of(rng, room, P)
        self.table = table
        pools = [torch.full(ph.paged_pool(n_pages, H_kv, d_h, P, kv, device="cpu").shape, 255 if kv == torch.uint8 else float("nan"), dtype=kv, device="cuda") for _ in range(2)]
        self.cache = ph.PagedCache(*pools, i32(table), d_h)
        self.seq_len = i32([0] * Bt)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(max(16, ph.photon_paged_attn_workspace_bytes(self.cache, Bt, max(T, max(prompts)), H)), dtype=torch.uint8, device="cuda")

    def rows(self, T, heads):
        return torch.from_numpy(self.rng.standard_normal((self.Bt, T, heads, self.d_h)).astype(np.float32)).to(self.dtype).cuda()

    def plain_entries(self, b, n):
        return [plain.entries(plain.values(p), self.table[b], n, self.d_h) for p in (self.cache.k_pages, self.cache.v_pages)]


def attend_plain(prog, q_rot, b, t, n, m, mask):
    k, v = prog.plain_entries(b, n)
    return plain.attended(q_rot[b, t], k, v, plain.seen(n, m, t, mask), prog.d_h ** -0.5)


def close(prog, got, ref, size):
    bound = 1e-5 * max(size.max(), 1e-30) if prog.dtype == torch.float32 else 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size
    assert (np.abs(got - ref) <= bound).all(), np.abs(got - ref).max()


@pytest.mark.parametrize("dtype,kv,d_h,H,H_kv,T", [(torch.bfloat16, torch.bfloat16, 64, 8, 2, 12), (torch.float32, torch.float32, 52, 4, 4, 7),
                                                   (torch.bfloat16, torch.uint8, 128, 4, 1, 21), (torch.float32, torch.bfloat16, 60, 2, 2, 5)])
def test_drafted_steps(ph, dtype, kv, d_h, H, H_kv, T):
    rng = np.random.default_rng(d_h)
    prompts, steps, Bt = [37, 5, 16], 4, 3
    prog = Program(ph, rng, Bt, H, H_kv, d_h, 16, T, prompts, steps, dtype, kv)
    most = max(prompts)
    # prompts, in one padded call
    k, v, q = prog.rows(most, H_kv), prog.rows(most, H_kv), prog.rows(most, H)
    q_rot, out, n_new = torch.empty_like(q), torch.full_like(q, 3.0), i32(prompts)
    ph.photon_paged_cache_write(k, v, prog.cache, n_new=n_new, q=q, q_out=q_rot, rope_theta=THETA, status=prog.status)
    prog.seq_len += n_new
    ph.photon_paged_attn(q_rot, prog.cache, prog.seq_len, out, n_new=n_new, workspace=prog.ws, status=prog.status)
    qs = q_rot.float().cpu().numpy()
    for b, n in enumerate(prompts):
        for t in (0, n // 2, n - 1):
            close(prog, out[b, t].float().cpu().numpy(), *attend_plain(prog, qs, b, t, n, n, None))
        assert (out[b, n:] == 3.0).all()
    lengths = list(prompts)
    history = [[x.copy() for x in prog.plain_entries(b, lengths[b])] for b in range(Bt)]
    for _ in range(steps):
        masks, depths = zip(*[plain.tree_masks([-1] + [int(rng.integers(max(0, t - 3), t)) for t in range(1, T)]) for _ in range(Bt)])
        k, v, q = prog.rows(T, H_kv), prog.rows(T, H_kv), prog.rows(T, H)
        q_rot, out = torch.empty_like(q), torch.empty_like(q)
        start = prog.seq_len.clone()
        position = start[:, None] + i32(np.stack(depths))
        ph.photon_paged_cache_write(k, v, prog.cache, start=start, position=position.contiguous(), q=q, q_out=q_rot, rope_theta=THETA, status=prog.status)
        ph.photon_paged_attn(q_rot, prog.cache, start + T, out, tree=torch.tensor(np.stack(masks), device="cuda"), workspace=prog.ws, status=prog.status)
        qs = q_rot.float().cpu().numpy()
        accepted = []
        for b in range(Bt):
            for t in range(T):
                close(prog, out[b, t].float().cpu().numpy(), *attend_plain(prog, qs, b, t, lengths[b] + T, T, masks[b][t]))
            node = int(rng.integers(0, T))
            accepted.append([j for j in range(T) if (int(masks[b][node]) >> j) & 1])
        drafted = [[x[:, lengths[b] :].copy() for x in prog.plain_entries(b, lengths[b] + T)] for b in range(Bt)]
        longest = max(len(p) for p in accepted)
        n_path = i32([len(p) for p in accepted])
        ph.photon_paged_cache_move(prog.cache, start, i32([p + [0] * (longest - len(p)) for p in accepted]), n=n_path, status=prog.status)
        prog.seq_len = start + n_path
        for b, path in enumerate(accepted):
            history[b] = [np.concatenate([h, d[:, path]], 1) for h, d in zip(history[b], drafted[b])]
            lengths[b] += len(path)
            for got, want in zip(prog.plain_entries(b, lengths[b]), history[b]):
                np.testing.assert_array_equal(got, want)
            # what the accepted nodes' positions are: the entries' own, so that a plain append would have left the same
            assert [int(depths[b][j]) for j in path] == list(range(len(path)))
    # one more entry each, as without drafts
    k, v, q = prog.rows(1, H_kv), prog.rows(1, H_kv), prog.rows(1, H)
    q_rot, out = torch.empty_like(q), torch.empty_like(q)
    ph.photon_paged_cache_write(k, v, prog.cache, start=prog.seq_len, q=q, q_out=q_rot, rope_theta=THETA, status=prog.status)
    ph.photon_paged_attn(q_rot, prog.cache, prog.seq_len + 1, out, workspace=prog.ws, status=prog.status)
    qs = q_rot.float().cpu().numpy()
    for b in range(Bt):
        close(prog, out[b, 0].float().cpu().numpy(), *attend_plain(prog, qs, b, 0, lengths[b] + 1, 1, None))
    assert int(prog.status) == 0


def test_captured_steps(ph):
    """A step of write, attention and move in a graph: every replay as the eager calls, lengths moving on in device memory.  Two graphs
    share the workspace, and eager work runs between the replays."""
    rng = np.random.default_rng(6)
    Bt, H, H_kv, d_h, T, P = 3, 8, 2, 64, 6, 16
    progs = [Program(ph, np.random.default_rng(7), Bt, H, H_kv, d_h, P, T, [900, 40, 333], 8, torch.bfloat16, torch.bfloat16) for _ in range(2)]
    masks = torch.tensor(np.stack([plain.tree_masks([-1, 0, 0, 1, 1, 2])[0]] * Bt), device="cuda")
    depth, path = i32([0, 1, 1, 2, 2, 2]), i32([[0, 2, 5]] * Bt)
    n_path = i32([3, 1, 2])
    k, v, q = progs[0].rows(T, H_kv), progs[0].rows(T, H_kv), progs[0].rows(T, H)

    def begin(prog):
        x = torch.randn((Bt, 900, H_kv, d_h), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
        ph.photon_paged_cache_write(x, -x, prog.cache, n_new=i32([900, 40, 333]), rope_theta=THETA)
        prog.seq_len.copy_(i32([900, 40, 333]))
        prog.q_rot, prog.out = torch.empty_like(q), torch.empty_like(q)
        prog.after = torch.empty_like(prog.seq_len)

    def step(prog, ws):
        position = (prog.seq_len[:, None] + depth).contiguous()
        torch.add(prog.seq_len, T, out=prog.after)
        ph.photon_paged_cache_write(k, v, prog.cache, start=prog.seq_len, position=position, q=q, q_out=prog.q_rot, rope_theta=THETA, status=prog.status)
        ph.photon_paged_attn(prog.q_rot, prog.cache, prog.after, prog.out, tree=masks, n_splits=3, workspace=ws, status=prog.status)
        ph.photon_paged_cache_move(prog.cache, prog.seq_len, path, n=n_path, status=prog.status)
        prog.seq_len += n_path

    ws = torch.empty(ph.photon_paged_attn_workspace_bytes(progs[0].cache, Bt, T, H, None, 3), dtype=torch.uint8, device="cuda")
    wants = []
    eager = progs[0]
    begin(eager)
    for _ in range(5):
        step(eager, ws)
        wants.append((eager.out.clone(), eager.cache.k_pages.clone(), eager.seq_len.clone()))
    side = torch.cuda.Stream()
    graphs = []
    for prog in progs:
        begin(prog)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(prog, ws)
        graphs.append(g)
    for prog in progs:                                     # the capture ran nothing: pages and lengths as begin() left them
        prog.cache.k_pages.fill_(float("nan"))
        prog.cache.v_pages.fill_(float("nan"))
        begin_out = prog.out, prog.q_rot, prog.after
        begin(prog)
        prog.out, prog.q_rot, prog.after = begin_out
    for i, (out, pages, lengths) in enumerate(wants):
        for prog, g in zip(progs, graphs):
            g.replay()
            if i % 2:
                torch.cuda.synchronize()
            assert torch.equal(prog.out, out), i
            assert torch.equal(prog.seq_len, lengths)
            got = prog.cache.k_pages
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(pages)), i
            torch.randn((64, 64), device="cuda").sum().item()
    assert int(progs[0].status) == 0 and int(progs[1].status) == 0
