"""Performance cases of the paged K/V cache: appending to it with the rotary encoding on the way, attending over it with several
queries or a drafted tree of them, and keeping a tree's accepted path.

A pool holds pages of K (and one of V): [n_pages, H_kv, page size, row elements], and a table says which page holds which stretch of
a sequence.  A case is one of three kinds:

  write   T new rows a sequence: K is rotated to its position and stored with V in the pages, q is rotated for the attention
  attend  T new queries per sequence attend over the pages; the last entries are the queries' own, seen causally or by a tree
  accept  a step's drafted rows are written behind a sequence, each at its depth in the tree, and then the entries of the
          accepted path move up to the sequence's end

With `own` the library's entry points do the work; without it elementary torch operations in 32 bits do (angles in 64), from and
to the same tensors.
"""
from __future__ import annotations

import math

import torch

DEV = "cuda"
own = False

THETA = 10000.0
# What the largest listed cases have: 4 x 8192 rows of 32 + 32 heads of 64; 256 x 2048 entries of 16 heads of 64; 512 queries of
# 32 heads of 128 behind 2 x 8191 entries; no more than a page for every 16 entries of them.
MOST_ROW_ELEMENTS = 4 * 8192 * (32 + 32) * 64
MOST_ELEMENTS = 256 * 16 * 2048 * 64
MOST_FLOPS = 4 * 2 * 512 * 32 * 8191 * 128
MOST_PAIRS = 2 * 512 * 32 * 8191


def listed():
    return [
        # One step of the 128k-token configuration: every sequence appends the entry of its newest unit.
        dict(name="append_one", kind="write", Bt=4, T=1, H=32, H_kv=32, d_h=64, S=8192, page=64, rows="f32", cache="bf16", ragged=False),
        # Serving at the paper's 600M shape (heads of 52): 256 sequences append up to three entries each.
        dict(name="append_ragged256", kind="write", Bt=256, T=3, H=32, H_kv=32, d_h=52, S=160, page=16, rows="bf16", cache="bf16", ragged=True),
        # Prompts of odd lengths into an 8-bit cache, four query heads to a K/V head.
        dict(name="write_prompts_8bit", kind="write", Bt=64, T=133, H=32, H_kv=8, d_h=128, S=200, page=32, rows="f32", cache="e4m3", ragged=True),
        # Four prompts of 128k tokens fill one layer's pages (8192 coarse entries a sequence).
        dict(name="write_prompt_128k", kind="write", Bt=4, T=8192, H=32, H_kv=32, d_h=64, S=8192, page=64, rows="bf16", cache="bf16", ragged=False),
        # One user of a small model behind 32k tokens, all in fp32.
        dict(name="attend_one_user", kind="attend", Bt=1, T=1, H=16, H_kv=16, d_h=64, S=2048, page=64, rows="f32", cache="f32", ragged=False, tree=False),
        # Serving: 256 sequences of up to 32k tokens, of all lengths, one query each.
        dict(name="attend_serving256", kind="attend", Bt=256, T=1, H=16, H_kv=16, d_h=64, S=2048, page=32, rows="f32", cache="bf16", ragged=True, tree=False),
        # Long contexts, eight query heads to a K/V head of 128, an odd length, small pages.
        dict(name="attend_grouped", kind="attend", Bt=8, T=1, H=32, H_kv=4, d_h=128, S=32749, page=16, rows="bf16", cache="bf16", ragged=False, tree=False),
        # Trees of up to 13 drafted units over 8-bit pages at the paper's 1.2B head size (60).
        dict(name="attend_tree_8bit", kind="attend", Bt=32, T=13, H=32, H_kv=32, d_h=60, S=1000, page=16, rows="bf16", cache="e4m3", ragged=True, tree=True),
        # The largest trees: 64 drafted nodes a sequence, grouped heads.
        dict(name="attend_tree64", kind="attend", Bt=16, T=64, H=32, H_kv=8, d_h=128, S=4096, page=64, rows="bf16", cache="bf16", ragged=False, tree=True),
        # A piece of 512 prompt entries behind those of the pieces before it.
        dict(name="attend_prompt_piece", kind="attend", Bt=2, T=512, H=32, H_kv=8, d_h=128, S=8191, page=64, rows="bf16", cache="bf16", ragged=False, tree=False),
        # One user's drafted tree is written and its accepted path kept.
        dict(name="accept_one_user", kind="accept", Bt=1, T=16, H=16, H_kv=16, d_h=64, S=500, page=16, rows="f32", cache="f32", ragged=False),
        # The same for 128 sequences with up to 31 nodes each.
        dict(name="accept_128", kind="accept", Bt=128, T=31, H=32, H_kv=8, d_h=128, S=300, page=32, rows="bf16", cache="bf16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "attend", "attend", "attend", "accept"])
    while True:
        d_h = rng.choice([20, 32, 48, 52, 56, 60, 64, 64, 80, 100, 128, 128])
        Bt, H_kv, G = _log_int(rng, 1, 256), _log_int(rng, 1, 32), rng.choice([1, 1, 1, 2, 4, 8])
        case = dict(kind=kind, Bt=Bt, H=H_kv * G, H_kv=H_kv, d_h=d_h, page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.5,
                    rows=rng.choice(["f32", "bf16"]), cache=rng.choice(["f32", "bf16", "bf16", "e4m3"]))
        if kind == "attend":
            how = rng.choice(["one", "one", "tree", "tree", "causal"])
            T = 1 if how == "one" else _log_int(rng, 2, 64 if how == "tree" else 1024)
            S = max(T, _log_int(rng, 1, 131072))
            case.update(T=T, S=S, tree=how == "tree")
            fits = Bt * H_kv * S * _row(d_h) <= MOST_ELEMENTS and 4 * Bt * T * H_kv * G * S * d_h <= MOST_FLOPS and Bt * T * H_kv * G * S <= MOST_PAIRS
        else:
            T = _log_int(rng, 1, 8192) if kind == "write" else _log_int(rng, 2, 64)
            S = T + rng.choice([0, rng.randint(1, 200), rng.randint(1, 4000)])
            case.update(T=T, S=S)
            fits = Bt * T * H_kv * (G + 1) * d_h <= MOST_ROW_ELEMENTS and Bt * H_kv * S * _row(d_h) <= MOST_ELEMENTS // 4
        if fits:
            return case


# ---- sizes that follow from a case ----

def _row(d_h):
    """Elements of a row of the pool: d_h rounded up to 32, 64 or 128."""
    return 32 if d_h <= 32 else 64 if d_h <= 64 else 128


def _new(case):
    """New rows of every sequence: T, or 1 .. T by turns."""
    return [1 + (b * 5 + 2) % case["T"] if case["ragged"] else case["T"] for b in range(case["Bt"])]


def _lengths(case):
    """Entries of every sequence, the new ones among them: S, or spread from S down to about S / 16; an attention's second one is empty."""
    Bt, S = case["Bt"], case["S"]
    if not case["ragged"]:
        return [S] * Bt
    new = _new(case)
    spread = [max(new[b], S - (15 * S * ((b * 11) % Bt)) // (16 * Bt)) for b in range(Bt)]
    if Bt > 1 and case["kind"] == "attend":
        spread[1] = 0
    return spread


def _tree(case):
    """(ancestors, depth) of the nodes of every sequence's tree: bit j of ancestors[b][t] is set where t or a node above it is j.
    Trees by turns are chains, binary, ternary, ..., with their nodes in order of depth."""
    masks, depths = [], []
    for b in range(case["Bt"]):
        wide, mask, depth = 1 + (b + 1) % 4, [1], [0]
        for t in range(1, case["T"]):
            above = (t - 1) // wide
            mask.append(mask[above] | (1 << t))
            depth.append(depth[above] + 1)
        masks.append(mask)
        depths.append(depth)
    return masks, depths


def _path(case):
    """The accepted nodes of every sequence: the last node in use and those above it, from the root down."""
    masks, _ = _tree(case)
    return [[j for j in range(case["T"]) if masks[b][m - 1] >> j & 1] for b, m in enumerate(_new(case))]


def _pairs(case):
    """Keys that all queries in use see, summed over queries."""
    total = 0
    masks = _tree(case)[0] if case["tree"] else None
    for b, (n, m) in enumerate(zip(_lengths(case), _new(case))):
        if n >= m:
            total += m * (n - m) + (sum(bin(masks[b][t]).count("1") for t in range(m)) if case["tree"] else m * (m + 1) // 2)
    return total


def work(case):
    esz, csz = 4 if case["rows"] == "f32" else 2, {"f32": 4, "bf16": 2, "e4m3": 1}[case["cache"]]
    H, H_kv, d_h, rows = case["H"], case["H_kv"], case["d_h"], sum(_new(case))
    if case["kind"] == "attend":
        return {"bytes": 2 * sum(_lengths(case)) * H_kv * d_h * csz + 2 * rows * H * d_h * esz, "flops": 4 * _pairs(case) * H * d_h}
    moved = sum(sum(j != i for i, j in enumerate(p)) for p in _path(case)) if case["kind"] == "accept" else 0
    return {"bytes": rows * d_h * (2 * H_kv * (esz + csz) + 2 * H * esz) + 4 * moved * H_kv * d_h * csz, "flops": 3 * rows * (H + H_kv) * d_h}


# ---- what a program has in hand ----

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _pool(g, shape, d_h, cache, filled, count):
    """A pool: zeros, or entries N(0, 1) in the places in use and all bits set elsewhere, as memory that was never written may have it."""
    storage = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}[cache]
    pool = torch.zeros(shape, dtype=storage, device=DEV)
    if not filled:
        return pool
    at_once = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
    for p in range(0, shape[0], at_once):
        part = pool[p : p + at_once]
        x = torch.randn((*part.shape[:3], d_h), generator=g, device=DEV)
        part[..., :d_h] = x.to(torch.float8_e4m3fn).view(torch.uint8) if cache == "e4m3" else x.to(storage)
        unused = torch.arange(shape[2], device=DEV) >= count[p : p + at_once, None]
        part.masked_fill_(unused[:, None, :, None], 255 if cache == "e4m3" else math.nan)
    return pool


def prepare(case, seed):
    g = _generator(seed)
    kind, Bt, T, H, H_kv, d_h, P = case["kind"], case["Bt"], case["T"], case["H"], case["H_kv"], case["d_h"], case["page"]
    rows = torch.float32 if case["rows"] == "f32" else torch.bfloat16
    int32 = dict(dtype=torch.int32, device=DEV)
    new, lengths = _new(case), _lengths(case)
    seq_len, n_new = torch.tensor(lengths, **int32), torch.tensor(new, **int32)
    # Pages in no order, as a program has handed them out; table places behind a sequence's last page hold -1; some pages are free.
    width = max(1, (case["S"] + P - 1) // P)
    held = (seq_len + P - 1) // P
    used = torch.arange(width, device=DEV) < held[:, None]
    n_used = sum((n + P - 1) // P for n in lengths)
    n_pages = n_used + 3
    order = torch.randperm(n_pages, generator=g, device=DEV)
    rank = torch.cumsum(used.flatten().long(), 0).view(Bt, width) - 1
    table = torch.where(used, order[rank.clamp(min=0)], -1).to(torch.int32)
    count = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV)
    left = (seq_len[:, None] - P * torch.arange(width, device=DEV)).clamp(0, P)
    count.scatter_(0, torch.where(used, table, n_pages).long().flatten(), left.long().flatten())
    shape = (n_pages, H_kv, P, _row(d_h))
    s = dict(kind=kind, d_h=d_h, cache=case["cache"], page_table=table, n_new=n_new if case["ragged"] else None, seq_len=seq_len,
             free=order[n_pages - 1], k_pages=_pool(g, shape, d_h, case["cache"], kind == "attend", count[:n_pages]),
             v_pages=_pool(g, shape, d_h, case["cache"], kind == "attend", count[:n_pages]),
             q=torch.randn((Bt, T, H, d_h), generator=g, device=DEV).to(rows))
    s["out"] = torch.zeros_like(s["q"])
    masks, depths = _tree(case) if kind == "accept" or case.get("tree") else (None, None)
    if kind == "attend":
        signed = lambda m: m - (1 << 64) if m >> 63 else m  # noqa: E731
        s["tree"] = torch.tensor([[signed(m) for m in row] for row in masks], dtype=torch.int64, device=DEV) if masks else None
        return s
    s["k"], s["v"] = (torch.randn((Bt, T, H_kv, d_h), generator=g, device=DEV).to(rows) for _ in range(2))
    s["start"], s["position"] = seq_len - n_new, None
    if kind == "accept":
        path = _path(case)
        most = max(len(p) for p in path)
        s["position"] = s["start"][:, None] + torch.tensor(depths, **int32)
        s["path"] = torch.tensor([p + [0] * (most - len(p)) for p in path], **int32)
        s["n_path"] = torch.tensor([len(p) for p in path], **int32)
    return s


# ---- one pass ----

def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "attend":
        return _attend(s)
    _write(s)
    if s["kind"] == "accept":
        _move(s)
    return [_as_values(s["k_pages"]), _as_values(s["v_pages"]), s["out"]]


def _as_values(pool):
    return pool.view(torch.float8_e4m3fn) if pool.dtype == torch.uint8 else pool


def _stored(x, pool):
    """fp32 values as the pool holds them."""
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if pool.dtype == torch.uint8 else x.to(pool.dtype)


def _rotated(x, cos, sin):
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _place(s, entry, used):
    """(page, row) of entries [Bt, n]; those not in use are sent to a free page."""
    P, table = s["k_pages"].shape[2], s["page_table"]
    page = torch.gather(table, 1, (entry // P).clamp(0, table.shape[1] - 1).long())
    return torch.where(used, page.long(), s["free"]), entry.long() % P


def _write(s):
    q, k, v, d_h = s["q"], s["k"], s["v"], s["d_h"]
    Bt, T = q.shape[:2]
    t = torch.arange(T, device=DEV)
    entry = s["start"][:, None] + t
    used = t < s["n_new"][:, None] if s["n_new"] is not None else (t >= 0).expand(Bt, T)
    position = entry if s["position"] is None else s["position"]
    i = torch.arange(d_h // 2, dtype=torch.float64, device=DEV)
    angle = (position.double()[..., None] * torch.pow(THETA, -2.0 * i / d_h))[:, :, None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    page, row = _place(s, entry, used)
    here = used[:, :, None, None]
    for pool, x in ((s["k_pages"], _rotated(k, cos, sin)), (s["v_pages"], v.float())):
        new = torch.where(here, _stored(x, pool), torch.zeros((), dtype=pool.dtype, device=DEV))
        pool[page, :, row, :d_h] = new
    s["out"].copy_(torch.where(here, _rotated(q, cos, sin), 0.0))


def _move(s):
    n = torch.arange(s["path"].shape[1], device=DEV)
    used = n < s["n_path"][:, None]
    page, row = _place(s, s["start"][:, None] + s["path"], used)
    to_page, to_row = _place(s, s["start"][:, None] + n.int(), used)
    for pool in (s["k_pages"], s["v_pages"]):
        kept = pool[page, :, row]
        pool[to_page, :, to_row] = torch.where(used[:, :, None, None], kept, torch.zeros((), dtype=pool.dtype, device=DEV))


def _attend(s):
    q, seq_len, d_h, P = s["q"], s["seq_len"].long(), s["d_h"], s["k_pages"].shape[2]
    Bt, T, H, _ = q.shape
    H_kv = s["k_pages"].shape[1]
    table = s["page_table"].long().clamp(min=0)
    S = table.shape[1] * P
    k, v = (_as_values(s[name][table])[..., :d_h].float().transpose(1, 2).reshape(Bt, H_kv, S, d_h) for name in ("k_pages", "v_pages"))
    position, t = torch.arange(S, device=DEV), torch.arange(T, device=DEV)
    v = torch.where((position < seq_len[:, None])[:, None, :, None], v, 0.0)
    n_new = s["n_new"].long() if s["n_new"] is not None else torch.full((Bt,), T, device=DEV)
    past = (seq_len - n_new)[:, None, None]
    if s["tree"] is None:
        seen = position <= past + t[:, None]                                                 # [Bt, T, S]
    else:
        bit = position - past
        drafted = (s["tree"][:, :, None] >> bit.clamp(0, 63)) & 1
        seen = (position < past) | ((bit >= 0) & (bit < n_new[:, None, None]) & (drafted == 1) & (position < seq_len[:, None, None]))
    seen = seen[:, None, :, None, :].expand(Bt, 1, T, H // H_kv, S).reshape(Bt, 1, T * (H // H_kv), S)
    rows = q.float().view(Bt, T, H_kv, H // H_kv, d_h).permute(0, 2, 1, 3, 4).reshape(Bt, H_kv, -1, d_h)
    score = torch.matmul(rows, k.transpose(-1, -2)) * (1.0 / math.sqrt(d_h))
    score = score.masked_fill(~seen, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / total.masked_fill(total == 0, 1.0)
    o = o.view(Bt, H_kv, T, H // H_kv, d_h).permute(0, 2, 1, 3, 4).reshape(Bt, T, H, d_h)
    s["out"].copy_(torch.where((t < n_new[:, None])[:, :, None, None], o, 0.0))
    return s["out"]


def _run_own(s):
    import paper_2512_20687_amd as ph

    if "pages" not in s:                                    # kept by a program as long as its pools and table
        s["pages"] = ph.PagedCache(s["k_pages"], s["v_pages"], s["page_table"], s["d_h"])
    if s["kind"] == "attend":
        if "workspace" not in s:                            # kept by a program for all its calls of this shape
            Bt, T, H, d_h = s["q"].shape
            size = ph.photon_paged_attn_workspace_bytes(s["pages"], Bt, T, H)
            s["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        return ph.photon_paged_attn(s["q"], s["pages"], s["seq_len"], s["out"], n_new=s["n_new"], tree=s["tree"], workspace=s["workspace"])
    ph.photon_paged_cache_write(s["k"], s["v"], s["pages"], s["start"], n_new=s["n_new"], position=s["position"], q=s["q"], q_out=s["out"],
                                rope_theta=THETA)
    if s["kind"] == "accept":
        ph.photon_paged_cache_move(s["pages"], s["start"], s["path"], n=s["n_path"])
    return [_as_values(s["k_pages"]), _as_values(s["v_pages"]), s["out"]]


# ---- the definition in 64 bits ----

def _exact_rotated(x, position):
    """Rows [n, heads, d_h] at positions [n]: each pair (i, i + d_h / 2) as a complex number times e^(i angle)."""
    half = x.shape[-1] // 2
    frequency = torch.exp(torch.arange(half, dtype=torch.float64, device=x.device) * (-math.log(THETA) / half))
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    z = z * torch.polar(torch.ones((), dtype=torch.float64, device=x.device), position.double()[:, None, None] * frequency)
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    new, lengths = _new(case), _lengths(case)
    Bt, T, H, H_kv, d_h, P = (case[n] for n in ("Bt", "T", "H", "H_kv", "d_h", "page"))
    out = torch.zeros((Bt, T, H, d_h), dtype=torch.float64, device=DEV)
    table = s["page_table"].tolist()
    if case["kind"] != "attend":
        pools = [torch.zeros(s["k_pages"].shape, dtype=torch.float64, device=DEV) for _ in range(2)]
        paths = _path(case) if case["kind"] == "accept" else None
        depths = torch.tensor(_tree(case)[1], device=DEV) if case["kind"] == "accept" else None
        for b, (n, m) in enumerate(zip(lengths, new)):
            at = torch.arange(n - m, n, device=DEV)
            position = at if depths is None else n - m + depths[b, :m]
            out[b, :m] = _exact_rotated(s["q"][b, :m], position)
            pages = torch.tensor(table[b], device=DEV)
            for pool, x in zip(pools, (_exact_rotated(s["k"][b, :m], position), s["v"][b, :m].double())):
                x = x.clamp(-448, 448) if case["cache"] == "e4m3" else x
                pool[pages[at // P], :, at % P, :d_h] = x
                if paths is not None:
                    to = at[: len(paths[b])]
                    pool[pages[to // P], :, to % P, :d_h] = x[torch.tensor(paths[b], device=DEV)]
        return [*pools, out]
    masks = _tree(case)[0] if case["tree"] else None
    for b, (n, m) in enumerate(zip(lengths, new)):
        if n == 0:
            continue
        pages = torch.tensor(table[b][: (n + P - 1) // P], device=DEV)
        k, v = (_as_values(s[c][pages]).to(torch.float32)[..., :d_h].transpose(0, 1).flatten(1, 2)[:, :n].double().repeat_interleave(H // H_kv, dim=0)
                for c in ("k_pages", "v_pages"))
        hidden = torch.zeros((m, n), dtype=torch.bool)
        hidden[:, n - m :] = torch.tensor([[not masks[b][t] >> j & 1 if masks else j > t for j in range(m)] for t in range(m)])
        score = torch.matmul(s["q"][b, :m].double().transpose(0, 1), k.transpose(1, 2)) / math.sqrt(d_h)
        weight = torch.softmax(score.masked_fill(hidden.to(DEV), -math.inf), dim=-1)
        out[b, :m] = torch.matmul(weight, v).transpose(0, 1)
    return out
