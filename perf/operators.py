"""Performance cases of the 4-bit K/V cache: writing it, reading it back, attending over it.

The cache holds K and V rows in MXFP4 (OCP microscaling: blocks of 32 elements of
a head's row in E2M1 under one power-of-two scale), laid out in tiles of 64
positions as include/photon.h describes.  A case is one of three kinds:

  write   new K/V rows [Bt, T, H_kv, d_h] go into the cache behind `start[b]`
          entries and are read back, as values, from where they went
  read    a stretch of the cache comes back as values
  attend  T new queries per sequence attend over the cache, causally, the last
          T entries being their own; H / H_kv query heads share a K/V head

With `own` the library's entry points do the work; without it elementary torch
operations in 32 bits do, from and to the same tensors.
"""
from __future__ import annotations

import math

import torch

DEV = "cuda"
own = False

TILE = 64            # positions of a cache tile
BLOCK = 32           # elements under one scale
# A cache of 256 sequences x 16 heads x 2048 positions x 64 elements, and the products of 32 heads over 8 x 32768 positions
# of 128 elements: what the largest listed cases have.
MOST_ELEMENTS = 256 * 16 * 2048 * 64
MOST_FLOPS = 4 * 8 * 32 * 32768 * 128
MOST_ROW_ELEMENTS = 4 * 8192 * 32 * 64


def listed():
    return [
        # One step of the 128k-token configuration: every sequence appends one entry a layer.
        dict(name="append_one", kind="write", Bt=4, T=1, H_kv=32, d_h=64, S=8192, dtype="f32", ragged=False),
        # Serving at the paper's 600M shape (head size 52): 256 sequences append up to three entries each, out of bf16 rows.
        dict(name="append_ragged256", kind="write", Bt=256, T=3, H_kv=32, d_h=52, S=160, dtype="bf16", ragged=True),
        # Four prompts of 128k tokens fill one layer's cache (8192 coarse entries a sequence).
        dict(name="write_prompt_128k", kind="write", Bt=4, T=8192, H_kv=32, d_h=64, S=8192, dtype="f32", ragged=False),
        # A stretch of one sequence's history, an odd number of entries, to look at or to move.
        dict(name="read_page", kind="read", Bt=1, T=333, H_kv=8, d_h=128, S=2048, dtype="bf16", ragged=False),
        # Ragged stretches at the paper's 1.2B shape (head size 60) in fp32.
        dict(name="read_ragged64", kind="read", Bt=64, T=128, H_kv=32, d_h=60, S=300, dtype="f32", ragged=True),
        # A whole layer's cache back in bf16, to continue in another precision.
        dict(name="read_128k", kind="read", Bt=4, T=8192, H_kv=32, d_h=64, S=8192, dtype="bf16", ragged=False),
        # One user of a small model behind 32k tokens.
        dict(name="attend_one_user", kind="attend", Bt=1, T=1, H=16, H_kv=16, d_h=64, S=2048, dtype="f32", ragged=False),
        # The headline configuration: 128k tokens, batch 4.
        dict(name="attend_128k", kind="attend", Bt=4, T=1, H=32, H_kv=32, d_h=64, S=8192, dtype="f32", ragged=False),
        # Serving: 256 sequences of 32k tokens.
        dict(name="attend_serving256", kind="attend", Bt=256, T=1, H=16, H_kv=16, d_h=64, S=2048, dtype="f32", ragged=False),
        # 256 short sequences of the paper's 600M shape, all of different lengths, one of them empty.
        dict(name="attend_ragged256", kind="attend", Bt=256, T=1, H=32, H_kv=32, d_h=52, S=135, dtype="bf16", ragged=True),
        # Four new units of every sequence at once, as the hierarchical schedule's lower level attends.
        dict(name="attend_units4", kind="attend", Bt=16, T=4, H=16, H_kv=16, d_h=64, S=2048, dtype="f32", ragged=True),
        # Grouped heads of 128: eight query heads share a K/V head over a long context of an odd length.
        dict(name="attend_grouped", kind="attend", Bt=8, T=1, H=32, H_kv=4, d_h=128, S=32749, dtype="bf16", ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "attend", "attend"])
    while True:
        d_h = rng.choice([20, 32, 48, 52, 56, 60, 64, 64, 80, 100, 128, 128])
        Bt, dtype, ragged = _log_int(rng, 1, 256), rng.choice(["f32", "bf16"]), rng.random() < 0.5
        if kind == "attend":
            H_kv, G, T = _log_int(rng, 1, 32), rng.choice([1, 1, 1, 2, 4, 8]), rng.choice([1, 1, 1, 1, 2, 3, 4, 8])
            S = max(T, _log_int(rng, 1, 131072))
            if Bt * H_kv * S * _row(d_h) <= MOST_ELEMENTS and 4 * Bt * H_kv * G * T * S * d_h <= MOST_FLOPS:
                return dict(kind=kind, Bt=Bt, T=T, H=H_kv * G, H_kv=H_kv, d_h=d_h, S=S, dtype=dtype, ragged=ragged)
        else:
            H_kv, T = _log_int(rng, 1, 32), _log_int(rng, 1, 8192)
            S = T + rng.choice([0, 0, rng.randint(1, 200), rng.randint(1, 4000)])
            if Bt * H_kv * T * _row(d_h) <= MOST_ROW_ELEMENTS and Bt * H_kv * S * _row(d_h) <= MOST_ELEMENTS:
                return dict(kind=kind, Bt=Bt, T=T, H_kv=H_kv, d_h=d_h, S=S, dtype=dtype, ragged=ragged)


# ---- sizes that follow from a case ----

def _row(d_h):
    """Elements of a cache row: d_h rounded up to 32, 64 or 128."""
    return 32 if d_h <= 32 else 64 if d_h <= 64 else 128


def _new(case):
    """New rows of every sequence: T, or 1 .. T by turns."""
    return [1 + (b * 5 + 2) % case["T"] if case["ragged"] else case["T"] for b in range(case["Bt"])]


def _lengths(case):
    """Entries of every sequence, the new ones among them: S, or spread from S down to about S / 2, the second one of a batch empty."""
    Bt, S = case["Bt"], case["S"]
    if not case["ragged"]:
        return [S] * Bt
    new = _new(case)
    spread = [max(new[b], S - (S * b) // (2 * Bt)) for b in range(Bt)]
    if Bt > 1 and case["kind"] == "attend":
        spread[1] = 0
    return spread


def _visible(case):
    """Keys that query t of sequence b sees, for the queries in use."""
    return [[max(0, n - m + t + 1) for t in range(m)] for n, m in zip(_lengths(case), _new(case))]


def work(case):
    blocks = math.ceil(case["d_h"] / BLOCK)
    entry = blocks * (BLOCK // 2 + 1)                       # bytes of a row in the cache
    esz = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "attend":
        keys = sum(_lengths(case))
        rows = sum(_new(case))
        pairs = sum(sum(v) for v in _visible(case))
        return {"bytes": 2 * keys * case["H_kv"] * entry + 2 * rows * case["H"] * case["d_h"] * esz,
                "flops": 4 * pairs * case["H"] * case["d_h"]}
    rows = sum(_new(case)) * case["H_kv"]
    values = 2 * rows * case["d_h"]
    if case["kind"] == "write":                             # rows in, entries out, values of the entries out
        return {"bytes": 2 * values * esz + 2 * rows * entry, "flops": 8 * values}
    return {"bytes": values * esz + 2 * rows * entry, "flops": 2 * values}


# ---- the format in plain torch ----

def _quantise(x):
    """fp32 [..., 32 n] -> (codes uint8 [..., 32 n], scale bytes uint8 [..., n])."""
    blocks = x.unflatten(-1, (-1, BLOCK))
    amax = blocks.abs().amax(-1)
    exponent = ((amax.view(torch.int32) >> 23) & 255) - 127 - 2
    exponent = exponent.clamp(min=-127)
    y = torch.ldexp(blocks.abs(), -exponent.unsqueeze(-1))
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(max=6.0)
    code = torch.where(y < 2, 2 * y, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(blocks).to(torch.uint8) << 3)
    return code.flatten(-2), (exponent + 127).to(torch.uint8)


def _scale(byte):
    f = (byte.to(torch.int32) << 23).view(torch.float32)
    f = torch.where(byte == 0, 2.0 ** -127, f)
    return torch.where(byte == 255, torch.full_like(f, math.nan), f)


def _values(code, byte):
    """(codes, scale bytes) -> fp32 values."""
    magnitude = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    table = torch.cat([magnitude, -magnitude])
    v = table[code.to(torch.int32)]
    return (v.unflatten(-1, (-1, BLOCK)) * _scale(byte).unsqueeze(-1)).flatten(-2)


def _pack(code, byte, values_first):
    """Codes [n, 64, d_p] and scale bytes [n, 64, d_p / 32] of n tiles -> tiles [n, bytes].  Nibble 2 i is the low half of byte i."""
    n, _, d_p = code.shape
    nb = d_p // BLOCK
    if values_first:     # V: [half, word of 16 dims, 8 keys, dim] -> chunks of four words, lane = (key group, dim)
        c = code.view(n, 2, 4, 8, 2 * nb, 16).permute(0, 1, 4, 2, 5, 3).reshape(n, nb, 4, 4, 16, 8).permute(0, 1, 3, 4, 2, 5)
        s = byte
    else:                # K: [16 keys, block] -> 16-byte chunks
        c = code.view(n, 4, 16, nb, BLOCK).permute(0, 1, 3, 2, 4)
        s = byte.view(n, 4, 16, nb).permute(0, 1, 3, 2).reshape(n, nb, 4, 16).permute(0, 2, 3, 1)
    c = c.reshape(n, 64 * d_p // 2, 2)
    return torch.cat([c[..., 0] | (c[..., 1] << 4), s.reshape(n, 64 * nb)], dim=1)


def _unpack(tiles, d_p, values_first):
    """Tiles [n, bytes] -> (codes [n, 64, d_p], scale bytes [n, 64, d_p / 32])."""
    n, nb = tiles.shape[0], d_p // BLOCK
    packed, s = tiles[:, : 32 * d_p], tiles[:, 32 * d_p :]
    c = torch.stack([packed & 15, packed >> 4], dim=-1)
    if values_first:
        c = c.reshape(n, nb, 4, 16, 4, 8).permute(0, 1, 4, 2, 3, 5).reshape(n, 2, 2 * nb, 4, 16, 8).permute(0, 1, 3, 5, 2, 4)
        return c.reshape(n, 64, d_p), s.reshape(n, 64, nb)
    c = c.reshape(n, 4, nb, 16, BLOCK).permute(0, 1, 3, 2, 4).reshape(n, 64, d_p)
    s = s.reshape(n, 4, 16, nb).permute(0, 3, 1, 2).reshape(n, 4, nb, 16).permute(0, 1, 3, 2)
    return c, s.reshape(n, 64, nb)


def _entries(cache, d_p, values_first):
    """Cache [Bt, H_kv, tiles, bytes] -> fp32 values [Bt, H_kv, 64 tiles, d_p]."""
    Bt, H_kv, tiles, size = cache.shape
    v = _values(*_unpack(cache.reshape(-1, size), d_p, values_first))
    return v.view(Bt, H_kv, tiles * TILE, d_p)


# ---- what a program has in hand ----

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _filled_cache(g, case, values_first):
    """Entries N(0, 1) in the positions in use; all bits set behind them, as memory that was never written may have it."""
    Bt, H_kv, S, d_h = case["Bt"], case["H_kv"], case["S"], case["d_h"]
    d_p, tiles = _row(d_h), (S + TILE - 1) // TILE
    lengths = torch.tensor(_lengths(case), device=DEV)
    cache = torch.empty((Bt, H_kv, tiles, TILE * (d_p // 2 + d_p // BLOCK)), dtype=torch.uint8, device=DEV)
    at_once = max(1, (1 << 25) // (H_kv * tiles * TILE * d_p))
    for b in range(0, Bt, at_once):
        part = cache[b : b + at_once]
        x = torch.zeros((part.shape[0] * H_kv * tiles, TILE, d_p), device=DEV)
        x[..., :d_h] = torch.randn((*x.shape[:2], d_h), generator=g, device=DEV)
        code, byte = _quantise(x)
        used = torch.arange(tiles * TILE, device=DEV) < lengths[b : b + at_once, None]
        used = used[:, None].expand(-1, H_kv, -1).reshape(-1, TILE, 1)
        part.copy_(_pack(torch.where(used, code, 15), torch.where(used, byte, 255), values_first).view_as(part))
    return cache


def prepare(case, seed):
    g = _generator(seed)
    kind, Bt, T, d_h, S = case["kind"], case["Bt"], case["T"], case["d_h"], case["S"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    new, lengths = _new(case), _lengths(case)
    d_p, tiles = _row(d_h), (S + TILE - 1) // TILE
    int32 = dict(dtype=torch.int32, device=DEV)
    s = dict(kind=kind, d_h=d_h, n_new=torch.tensor(new, **int32) if case["ragged"] else None)
    if kind == "attend":
        s.update(q=torch.randn((Bt, T, case["H"], d_h), generator=g, device=DEV).to(dtype), seq_len=torch.tensor(lengths, **int32),
                 k_cache=_filled_cache(g, case, False), v_cache=_filled_cache(g, case, True))
        s["out"] = torch.zeros_like(s["q"])
        return s
    s["start"] = torch.tensor([n - m for n, m in zip(lengths, new)], **int32)
    rows = (Bt, T, case["H_kv"], d_h)
    s["k_out"], s["v_out"] = torch.zeros(rows, dtype=dtype, device=DEV), torch.zeros(rows, dtype=dtype, device=DEV)
    if kind == "read":
        s.update(k_cache=_filled_cache(g, case, False), v_cache=_filled_cache(g, case, True))
    else:
        size = (Bt, case["H_kv"], tiles, TILE * (d_p // 2 + d_p // BLOCK))
        s.update(k=torch.randn(rows, generator=g, device=DEV).to(dtype), v=torch.randn(rows, generator=g, device=DEV).to(dtype),
                 k_cache=torch.zeros(size, dtype=torch.uint8, device=DEV), v_cache=torch.zeros(size, dtype=torch.uint8, device=DEV))
    return s


# ---- one pass ----

def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "attend":
        return _attend(s)
    k_out, v_out, n_new = s["k_out"], s["v_out"], s["n_new"]
    Bt, T, H_kv, d_h = k_out.shape
    d_p = _row(d_h)
    t = torch.arange(T, device=DEV)
    used = (t < n_new[:, None] if n_new is not None else (t >= 0).expand(Bt, T))[:, :, None, None]
    for i, (out, cache) in enumerate(((k_out, s["k_cache"]), (v_out, s["v_cache"]))):
        if s["kind"] == "write":
            x = torch.nn.functional.pad((s["k"], s["v"])[i].float(), (0, d_p - d_h))
            got = _values(*_quantise(x))[..., :d_h]
        else:
            at = (s["start"].long()[:, None] + t).clamp(max=cache.shape[2] * TILE - 1)
            got = _entries(cache, d_p, i == 1)[torch.arange(Bt, device=DEV)[:, None], :, at][..., :d_h]
        out.copy_(torch.where(used, got, 0.0))
    return [k_out, v_out]


def _attend(s):
    q, seq_len, n_new = s["q"], s["seq_len"].long(), s["n_new"]
    Bt, T, H, d_h = q.shape
    d_p, H_kv = _row(d_h), s["k_cache"].shape[1]
    k, v = _entries(s["k_cache"], d_p, False), _entries(s["v_cache"], d_p, True)
    S = k.shape[2]
    position, t = torch.arange(S, device=DEV), torch.arange(T, device=DEV)
    v = torch.where((position < seq_len[:, None])[:, None, :, None], v, 0.0)
    n_new = n_new.long() if n_new is not None else torch.full((Bt,), T, device=DEV)
    last = seq_len[:, None] - n_new[:, None] + t                                             # [Bt, T]: the last key a query sees
    seen = (position <= last[:, :, None])[:, None, :, None, :].expand(Bt, 1, T, H // H_kv, S).reshape(Bt, 1, T * (H // H_kv), S)
    rows = q.float().view(Bt, T, H_kv, H // H_kv, d_h).permute(0, 2, 1, 3, 4).reshape(Bt, H_kv, -1, d_h)
    score = torch.matmul(rows, k[..., :d_h].transpose(-1, -2)) * (1.0 / math.sqrt(d_h))
    score = score.masked_fill(~seen, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v[..., :d_h]) / total.masked_fill(total == 0, 1.0)
    o = o.view(Bt, H_kv, T, H // H_kv, d_h).permute(0, 2, 1, 3, 4).reshape(Bt, T, H, d_h)
    s["out"].copy_(torch.where((t < n_new[:, None])[:, :, None, None], o, 0.0))
    return s["out"]


def _run_own(s):
    import paper_2512_20687_amd as ph

    if s["kind"] == "attend":
        if "workspace" not in s:                            # kept by a program for all its calls of this shape
            Bt, T, H, d_h = s["q"].shape
            H_kv, tiles = s["k_cache"].shape[1:3]
            n = ph.photon_mxfp4_decode_attn_auto_splits(Bt, T, H, H_kv, tiles * TILE)
            size = ph.photon_mxfp4_decode_attn_workspace_bytes(Bt, T, H, d_h, n)
            s["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
        return ph.photon_mxfp4_decode_attn(s["q"], s["k_cache"], s["v_cache"], s["seq_len"], s["out"], n_new=s["n_new"], workspace=s["workspace"])
    if s["kind"] == "write":
        ph.photon_mxfp4_cache_write(s["k"], s["v"], s["k_cache"], s["v_cache"], start=s["start"], n_new=s["n_new"])
    ph.photon_mxfp4_cache_read(s["k_cache"], s["v_cache"], s["k_out"], s["v_out"], start=s["start"], n_rows=s["n_new"])
    return [s["k_out"], s["v_out"]]


# ---- the definition in 64 bits ----

def _exact_rows(x):
    """What the format makes of rows [..., d_h]: the nearest of the fifteen values of a block, halves to the even code."""
    d_h = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -d_h % BLOCK))
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    _, e = torch.frexp(blocks.abs().amax(-1, keepdim=True))                                # amax in [2^(e-1), 2^e)
    scale = torch.pow(2.0, (e - 3).double().clamp(min=-127))
    y = (blocks / scale).abs().contiguous()
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    below, above = torch.bucketize(y, border), torch.bucketize(y, border, right=True)      # they differ on a border only
    code = torch.where(below % 2 == 0, below, above)
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)[code]
    return (value * scale * torch.where(blocks < 0, -1.0, 1.0)).reshape(x.shape)[..., :d_h]


def _exact_entries(cache, d_h, values_first):
    """Cache of one sequence [H_kv, tiles, bytes] -> values [H_kv, positions, d_h], every byte looked up by its address."""
    d_p = _row(d_h)
    nb = d_p // BLOCK
    key = torch.arange(TILE, device=cache.device)[:, None]
    e = torch.arange(d_h, device=cache.device)[None, :]
    if values_first:
        word = (key // 32) * 2 * nb + e // 16
        at = (word // 4) * 1024 + ((key % 32) // 8 * 16 + e % 16) * 16 + (word % 4) * 4 + (key % 8) // 2
        shift = 4 * (key % 2) + 0 * e
        at_scale = key * nb + e // BLOCK
    else:
        chunk = (key // 16) * nb + e // BLOCK
        at = chunk * 256 + (key % 16) * 16 + (e % BLOCK) // 2
        shift = 4 * (e % 2) + 0 * key
        at_scale = (chunk % 4 * 16 + key % 16) * nb + chunk // 4
    code = (cache[..., at].long() >> shift) & 15
    size, exponent = code % 2, (code % 8) // 2
    value = torch.where(exponent == 0, 0.5 * size, (1 + 0.5 * size) * torch.pow(2.0, (exponent - 1).double()))
    value = torch.where(code >= 8, -value, value)
    byte = cache[..., 32 * d_p + at_scale].long()
    value = value * torch.pow(2.0, (byte - 127).double())
    return torch.where(byte == 255, math.nan, value).reshape(cache.shape[0], -1, d_h)


def exact(case, seed):
    s = prepare(case, seed)
    new = _new(case)
    if case["kind"] == "write":
        got = [_exact_rows(s["k"]), _exact_rows(s["v"])]
        for x in got:
            for b, m in enumerate(new):
                x[b, m:] = 0
        return got
    Bt, T, d_h, H_kv = case["Bt"], case["T"], case["d_h"], case["H_kv"]
    lengths = _lengths(case)
    if case["kind"] == "read":
        got = [torch.zeros((Bt, T, H_kv, d_h), dtype=torch.float64, device=DEV) for _ in range(2)]
        for b, (n, m) in enumerate(zip(lengths, new)):
            got[0][b, :m] = _exact_entries(s["k_cache"][b], d_h, False)[:, n - m : n].transpose(0, 1)
            got[1][b, :m] = _exact_entries(s["v_cache"][b], d_h, True)[:, n - m : n].transpose(0, 1)
        return got
    out = torch.zeros((Bt, T, case["H"], d_h), dtype=torch.float64, device=DEV)
    group = case["H"] // H_kv
    for b, seen in enumerate(_visible(case)):
        k, v = (_exact_entries(s[c][b], d_h, c == "v_cache").repeat_interleave(group, dim=0) for c in ("k_cache", "v_cache"))
        for t, n in enumerate(seen):
            if n > 0:
                score = (k[:, :n] * s["q"][b, t].double()[:, None, :]).sum(-1) / math.sqrt(d_h)
                weight = torch.softmax(score, dim=-1)
                out[b, t] = (weight[:, :, None] * v[:, :n]).sum(1)
    return out
