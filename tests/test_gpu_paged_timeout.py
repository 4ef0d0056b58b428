"""The time-outs of the paged decode: partial results that come when they have been given up.  Every wait is bounded and the
context stays usable; what was given up is NaN, and the workspace holds nothing that a later call could take for its own."""
import time

import pytest
import torch

from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu

FLAG_BYTES = 2 * 192 * 8


def _case(lens, Hq, Hc, d, page=64):
    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    B, per = len(lens), max(-(-max(lens) // page), 1)
    return (rand(B, Hq, d), rand(B * per, Hc, page, d), rand(B * per, Hc, page, d),
            torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per),
            torch.tensor(lens, dtype=torch.int32, device="cuda"))


class _Limit:
    def __enter__(self):
        torch.cuda.synchronize()
        self.was = sk.snapkv_set_wait_limit_ns(20_000_000)

    def __exit__(self, *_):
        sk.snapkv_set_wait_limit_ns(self.was)


def _check_late(got, want, lens, Hc):
    """NaN in whole (sequence, cache head, up to 8 query heads) units, everything else as it should be."""
    (out, lse), (B, Hq) = got, want[1].shape
    bad = torch.isnan(lse)
    assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
    assert torch.equal(out[~bad], want[0][~bad]) and torch.equal(lse[~bad], want[1][~bad])
    for unit in bad.view(B, Hc, Hq // Hc).split(8, -1):
        assert torch.equal(unit.any(-1), unit.all(-1))
    return int(bad.sum())


@pytest.mark.parametrize("lens,Hq,Hc,d,shared", [
    ([20000], 8, 2, 128, True),                   # two units over all blocks
    ([150000], 2, 1, 64, True),                   # one
    ([777], 32, 8, 128, True),
    ([3000, 1, 0, 500, 9000], 20, 2, 128, True),  # more than 8 query heads per cache head; no rows
    ([7], 2, 2, 128, False),                      # one block has all there is
])
def test_partials_that_come_too_late(lens, Hq, Hc, d, shared):
    case = _case(lens, Hq, Hc, d)
    want = sk.snapkv_decode_paged(*case)
    ws = torch.zeros_like(want[2])
    with _Limit():
        t0 = time.perf_counter()
        got = sk.snapkv_selftest_late_partials(*case, ws)
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
    assert took < 2.0 and (took > 0.015 or not shared)
    assert (_check_late(got, want, lens, Hc) > 0) == shared
    assert not ws[:FLAG_BYTES].any()              # neither a number nor the mark of giving it up
    again = sk.snapkv_decode_paged(*case, ws)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    assert not ws[:FLAG_BYTES].any()


def test_a_replayed_graph_never_takes_the_partials_of_an_earlier_replay():
    case = _case([30000, 5000], 8, 2, 128)
    want = sk.snapkv_decode_paged(*case)
    ws = torch.full_like(want[2], 255)            # whatever was in it
    with _Limit():
        sk.snapkv_selftest_late_partials(*case, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = sk.snapkv_selftest_late_partials(*case, ws)
    bad = None
    for scale in (1.0, 0.5, 2.0, 1.0):
        case[0].mul_(scale)
        want = sk.snapkv_decode_paged(*case)
        g.replay()
        torch.cuda.synchronize()
        assert _check_late(got, want, [30000, 5000], 2) > 0
        assert bad is None or torch.equal(bad, torch.isnan(got[1]))
        bad = torch.isnan(got[1])
    # the workspace is as good as before
    again = sk.snapkv_decode_paged(*case, ws)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


@pytest.mark.parametrize("lens,Hq,Hc,d", [([20000], 8, 2, 128), ([300, 0, 5, 4000], 20, 2, 64), ([1] * 30, 1, 1, 128)])
def test_rows_that_never_come(lens, Hq, Hc, d):
    case = _case(lens, Hq, Hc, d)
    want = sk.snapkv_decode_paged(*case)
    ws = torch.full_like(want[2], 255)
    with _Limit():
        t0 = time.perf_counter()
        out, lse = sk.snapkv_selftest_lost_rows(*case, ws)
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
    assert 0.015 < took < 2.0
    some = torch.tensor(lens, device="cuda") > 0
    assert torch.isnan(out[some]).all() and torch.isnan(lse[some]).all()
    assert not out[~some].any() and (lse[~some] == -float("inf")).all()
    again = sk.snapkv_decode_paged(*case, ws)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
