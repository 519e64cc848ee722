"""Rows appended at the end of 32 bits: their entries are not there, and yet q is rotated to start + t.

Tolerance as in tests/test_gpu_paged_cache.py: 6 * 2^-24 of |a| + |b| for a pair, and the angle's own error at such positions, 2^-27 turns and
float64's 2^-52 of it."""
import numpy as np
import pytest
import torch

import paged_plain as plain
from util import require_gpu

pytestmark = pytest.mark.gpu
FULL = 1


@pytest.mark.parametrize("T", [6, 70])
@pytest.mark.parametrize("d_h", [64, 52])
def test_rows_behind_the_last_position_of_32_bits(T, d_h):
    require_gpu()
    import paper_2512_20687_amd as ph
    rng = np.random.default_rng(T)
    starts = [2 ** 31 - 3, 2 ** 31 - 1, 2 ** 31 - T, -(2 ** 31), -2]
    Bt = len(starts)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q, k = (torch.from_numpy(rng.standard_normal((Bt, T, h, d_h)).astype(np.float32)).cuda() for h in (3, 1))
    pools = [ph.paged_pool(2 * Bt, 1, d_h, 64, torch.float32) for _ in range(2)]
    cache = ph.PagedCache(*pools, i32(np.arange(2 * Bt).reshape(Bt, 2)), d_h)
    out, status = torch.full_like(q, 9.0), i32([0])
    ph.photon_paged_cache_write(k, k, cache, start=i32(starts), q=q, q_out=out, rope_theta=1e4, status=status)
    assert int(status) == FULL
    for b, start in enumerate(starts):
        x = q[b].cpu().numpy().astype(np.float64)
        position = start + np.arange(T, dtype=np.int64)
        size = np.abs(x) + np.abs(np.roll(x, d_h // 2, -1))
        angle = 2 * np.pi * 2.0 ** -27 + np.abs(position)[:, None, None] * 2.0 ** -52
        off = np.abs(out[b].cpu().numpy() - plain.rotated(x, position, 1e4))
        assert (off <= size * (6 * 2.0 ** -24 + angle)).all(), (b, (off / size).max())
    for b in range(Bt - 1):
        assert not pools[0][2 * b : 2 * b + 2].any()                       # the last sequence's rows from entry 0 on are there
    np.testing.assert_array_equal(pools[1][2 * Bt - 2, 0, : min(64, T - 2), :d_h].cpu().numpy(), k[-1, 2 : min(66, T), 0].cpu().numpy())
