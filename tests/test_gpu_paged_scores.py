"""Attention over a paged cache where scores are far from zero or overflow to minus infinity.  Two elements of the queries
and keys are not zero and their products' sum is a number of fp32, so that the scores are exact."""
import math

import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu

PAGE = 64


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _case(lens, Hq, Hc, d, q0, k0, k1, seed=3):
    """q [B, Hq, d] = (q0 of the head, 1, 0, ...), rows (k0(row), k1(row), 0, ...), pages in reverse order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, per = len(lens), -(-max(lens) // PAGE)
    table = torch.arange(B * per - 1, -1, -1, dtype=torch.int32, device="cuda").view(B, per)
    q = torch.zeros(B, Hq, d, device="cuda")
    q[:, :, 0], q[:, :, 1] = q0(torch.arange(Hq, device="cuda")), 1.0
    row = torch.arange(per * PAGE, device="cuda")
    k = torch.zeros(B, per, Hc, PAGE, d, device="cuda")
    k[..., 0], k[..., 1] = (x(row).view(1, per, 1, PAGE).expand(B, per, Hc, PAGE) for x in (k0, k1))
    pool = k.new_empty(B * per, Hc, PAGE, d)
    pool[table.long().flatten()] = k.view(B * per, Hc, PAGE, d)
    v = torch.randn(B * per, Hc, PAGE, d, generator=g, device="cuda").to(torch.bfloat16)
    assert torch.equal(k[..., 1].to(torch.bfloat16).float(), k[..., 1])
    return q.to(torch.bfloat16), pool.to(torch.bfloat16), v, table


def _check(q, k, v, table, lens, out, lse):
    B, Hq, d = q.shape
    for b, n in enumerate(lens):
        keys, values = (plain64.read_paged(x, table[b].tolist(), n).double() for x in (k, v))
        for h in range(Hq):
            kh, vh = keys[:, h // (Hq // k.shape[1])], values[:, h // (Hq // k.shape[1])]
            s = kh @ q[b, h].double() / math.sqrt(d)
            top = s.max()
            p = torch.exp(s - top)
            ref, scale, rlse = p @ vh / p.sum(), p @ vh.abs() / p.sum(), top + p.sum().log()
            err, tol = (out[b, h].double() - ref).abs(), plain64.fp32_tolerance(scale, torch.zeros_like(rlse), d)
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            # the scale, the sum of reference and logarithm, ln 2 and the result: half a step of 2^-24 each
            assert (lse[b, h].double() - rlse).abs() <= 2.0 ** -19 + rlse.abs() * 2.0 ** -22, (b, h)


LENS = [[5], [100], [777], [20000, 3, 800], [1300] * 40]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hc", [(2, 1), (4, 1), (8, 1), (12, 4)])
@pytest.mark.parametrize("lens", LENS)
def test_a_head_whose_first_scores_are_minus_infinity(lens, Hq, Hc, d):
    # even heads: -2^200 in the first rows, beyond fp32; odd heads see a few units, rising
    hidden = min(lens) // 2 if len(lens) == 1 else 1
    for few in {hidden, max(lens) - 1}:
        q, k, v, table = _case(lens, Hq, Hc, d, lambda h: torch.where(h % 2 == 0, 2.0 ** 100, 0.0),
                               lambda r: torch.where(r < few, -2.0 ** 100, 0.0), lambda r: (r % 300) / 4 // 8)
        some = [b for b, n in enumerate(lens) if n > few]
        out, lse, _ = sk.snapkv_decode_paged(q, k, v, table, _i32(lens))
        _check(q[some], k, v, table[some], [lens[b] for b in some], out[some], lse[some])
        for b in set(range(len(lens))) - set(some):     # even heads whose scores are all so: as without rows
            assert not out[b, ::2].any() and (lse[b, ::2] == -math.inf).all()
            if Hc == 1:
                _check(q[b:b + 1, 1::2], k, v, table[b:b + 1], [lens[b]], out[b:b + 1, 1::2], lse[b:b + 1, 1::2])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hc", [(2, 1), (8, 2), (5, 1)])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("what", ["all far below", "first half far below", "all far above"])
def test_scores_far_from_zero(what, lens, Hq, Hc, d):
    k0 = {"all far below": lambda r: torch.full_like(r, -2.0 ** 60, dtype=torch.float32),
          "first half far below": lambda r: torch.where(r < max(lens) // 2, -2.0 ** 60, 0.0),
          "all far above": lambda r: torch.full_like(r, 2.0 ** 60, dtype=torch.float32)}[what]
    q, k, v, table = _case(lens, Hq, Hc, d, lambda h: torch.full_like(h, 2.0 ** 60, dtype=torch.float32), k0,
                           lambda r: torch.zeros_like(r, dtype=torch.float32))
    out, lse, _ = sk.snapkv_decode_paged(q, k, v, table, _i32(lens))
    _check(q, k, v, table, lens, out, lse)
