"""The time-outs of the prompt attention: keys that never come.  The block drains its copies and matrix instructions, fills
with NaN what it can not compute and what it has taken over, frees its tensor memory and returns; other blocks do not notice."""
import time

import pytest
import torch

from paper_2404_14469_b200 import binding as sk
from test_gpu_prefill import _draw

pytestmark = pytest.mark.gpu


def _units(lens, Hq, Hkv):
    """Rows [(tokens, heads)] of every work unit, in the launch's order (lengths descending)."""
    pack = 1
    while pack < 64 and (Hq // Hkv) % (2 * pack) == 0:
        pack *= 2
    tile = 128 // pack
    split = sum(-(-n // tile) for n in lens) * (Hq // pack) <= torch.cuda.get_device_properties(0).multi_processor_count
    tile *= 1 if split else 2
    units, at = [], 0
    for n in lens:
        for block in reversed(range(-(-n // tile))):
            for head in range(0, Hq, pack):
                units.append((slice(at + block * tile, at + min(block * tile + tile, n)), slice(head, head + pack)))
        at += n
    return units, split


@pytest.mark.parametrize("lens,Hq,Hkv,d,which,few", [
    ([500], 4, 2, 64, (0, 5, 15), True),                # few query tiles: a unit per block, keys in two halves
    ([300, 129, 7], 8, 2, 128, (0, 3, -1), True),
    ([100], 1, 1, 128, (0,), True),
    ([3000], 32, 8, 128, (0, 100, 147, 148, 300, -1), False),
    ([900, 700, 650, 1], 64, 16, 64, (0, 77, 200, -1, -3), False),
    ([6000], 16, 16, 64, (3, 200, -1), False),
])
def test_keys_that_never_come(lens, Hq, Hkv, d, which, few):
    T, W = sum(lens), 1
    q, k, v = _draw(T, T, Hq, Hkv, d, T)
    want = sk.snapkv_prefill_attention(q, k, v, lens, window=W)
    units, split = _units(lens, Hq, Hkv)
    assert split == few
    for unit in which:
        unit %= len(units)
        was = sk.snapkv_set_wait_limit_ns(20_000_000)
        try:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            out, lse, obs = sk.snapkv_selftest_lost_keys(q, k, v, lens, unit, window=W)
            torch.cuda.synchronize()
            took = time.perf_counter() - t0
        finally:
            sk.snapkv_set_wait_limit_ns(was)
        assert 0.015 < took < 1.0, took
        bad = torch.isnan(lse)
        assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
        assert torch.equal(out[~bad], want[0][~bad]) and torch.equal(lse[~bad], want[1][~bad])
        ends = torch.tensor(lens).cumsum(0).cuda() - 1
        assert torch.equal(torch.nan_to_num(obs[..., 0]), torch.nan_to_num(lse[ends]))
        # whole units: the one that was asked for, and two more at most
        hit = [i for i, rows in enumerate(units) if bad[rows].any()]
        assert unit in hit and len(hit) <= (1 if split else 3), hit
        assert sum(bad[units[i]].numel() for i in hit) == int(bad.sum())
        # and the context is as good as before
        again = sk.snapkv_prefill_attention(q, k, v, lens, window=W)
        assert all(torch.equal(x, y) for x, y in zip(again, want))


def test_a_unit_that_is_not_there():
    q, k, v = _draw(200, 200, 4, 2, 128, 3)
    want = sk.snapkv_prefill_attention(q, k, v, [200])
    got = sk.snapkv_selftest_lost_keys(q, k, v, [200], 10 ** 6)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
