"""The reference that the prompt attention's weights are taken against, where a row's scores are far from zero or far from
its first ones.  Queries and keys have two elements apart from zero, the products' sum is a number of fp32, so the scores
are exact and the tolerances hold no error of theirs."""
import math

import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu

FORMS = [(4, 2, 64), (2, 1, 128), (32, 8, 128), (64, 16, 64)]   # with 700 tokens: two of few query tiles, two of many
N = 700


def _two(Hq, Hkv, d, q0, k0, k1):
    """Queries (q0, 1, 0, ...), keys (k0, k1, 0, ...) and random values."""
    g = torch.Generator(device="cuda").manual_seed(77)
    q, k = torch.zeros(N, Hq, d, device="cuda"), torch.zeros(N, Hkv, d, device="cuda")
    q[:, :, 0], q[:, :, 1] = q0.cuda()[:, None], 1.0
    k[:, :, 0], k[:, :, 1] = k0.cuda()[:, None], k1.cuda()[:, None]
    v = torch.randn(N, Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    qb, kb = q.to(torch.bfloat16), k.to(torch.bfloat16)
    assert torch.equal(kb[:, 0, 1].float(), k[:, 0, 1]) and torch.equal(qb.float(), q)
    return qb, kb, v


def _check(q, k, v, out, lse, n_before):
    # (64 bits relative to the largest score: a log-sum-exp of 1e36 has no room for the logarithm of the sum)
    n, Hq, d = q.shape
    ref, rlse, scale = torch.zeros(n, Hq, d).cuda().double(), torch.zeros(n, Hq).cuda().double(), torch.zeros(n, Hq, d).cuda().double()
    see = torch.arange(k.shape[0], device="cuda")[None] <= n_before + torch.arange(n, device="cuda")[:, None]
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // k.shape[1])].double(), v[:, h // (Hq // k.shape[1])].double()
        s = (q[:, h].double() @ kh.T / math.sqrt(d)).masked_fill(~see, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        ref[:, h], scale[:, h], rlse[:, h] = p @ vh / total, p @ vh.abs() / total, (top + total.log())[:, 0]
    mag = torch.zeros_like(rlse)
    err = (out.double() - ref).abs()
    tol = plain64.bf16_tolerance(ref, scale, mag, d)
    assert (err <= tol).all(), float((err / tol).max())
    # the scale, the sum of reference and logarithm, ln 2 and the result: half a step of 2^-24 each
    err, tol = (lse.double() - rlse).abs(), 2.0 ** -19 + rlse.abs() * 2.0 ** -22
    assert (err <= tol).all(), float((err / tol).max())


J = torch.arange(N)
ONE = torch.ones(N)


def _case(name):
    """q0 [N], k0 [N], k1 [N] on the CPU."""
    first = J < 32
    steps = 8.0 * (J % 7)
    if name == "first keys at -1e11":
        return ONE, torch.where(first, -1e11, 0.0), torch.where(first, 0.0, 1600.0 + steps)
    if name == "first keys at -1e12":
        return ONE, torch.where(first, -1e12, 0.0), torch.where(first, 0.0, -2000.0 + steps)
    if name == "first keys at -1e37":
        return ONE, torch.where(first, -1e37, 0.0), torch.where(first, 0.0, 1600.0 + steps)
    if name in ("all at 2^30", "all at -2^30", "all at 2^37"):
        q0 = 2.0 ** (22 if "37" in name else 15) * ONE
        step = 128.0 * 128.0 if "37" in name else 128.0       # one step of fp32 at that size
        return q0, (-1.0 if "-" in name else 1.0) * 2.0 ** 15 * ONE, step * (J % 5)
    if name == "slowly rising at 2^22":
        return 2.0 ** 10 * ONE, 2.0 ** 12 * ONE, 4.0 * (J % 9) + 32.0 * (J // 100)
    if name == "rows of every size":
        q0 = torch.tensor([2.0 ** 15, 1.0, -2.0 ** 15, 0.0, 2.0 ** 9])[J % 5]
        return q0, 2.0 ** 15 * ONE, 128.0 * (J % 5)
    if name == "from far below to near":
        return 2.0 ** 15 * ONE, torch.where(J < 100, -2.0 ** 15, 0.0), 128.0 * (J % 5)
    if name == "from near to far above":
        return 2.0 ** 15 * ONE, torch.where(J < 100, 0.0, 2.0 ** 15), 128.0 * (J % 5)
    if name == "from far to farther, and back":
        return 2.0 ** 15 * ONE, torch.where(J < 100, 2.0 ** 15, torch.where(J < 500, 2.0 ** 16, 0.0)), 256.0 * (J % 5)
    raise KeyError(name)


@pytest.mark.parametrize("Hq,Hkv,d", FORMS)
@pytest.mark.parametrize("name", [
    "first keys at -1e11", "first keys at -1e12", "first keys at -1e37", "all at 2^30", "all at -2^30", "all at 2^37",
    "slowly rising at 2^22", "rows of every size", "from far below to near", "from near to far above",
    "from far to farther, and back"])
def test_scores_far_from_zero_or_from_the_first_ones(name, Hq, Hkv, d):
    q, k, v = _two(Hq, Hkv, d, *_case(name))
    out, lse, obs = sk.snapkv_prefill_attention(q, k, v, [N], window=16)
    _check(q, k, v, out, lse, 0)
    assert torch.equal(obs[0], lse[N - 16:].t())
    # and as a chunk behind the other keys, whose first tile every row sees whole
    out, lse, _ = sk.snapkv_prefill_attention(q[-90:], k, v, [90], [N])
    _check(q[-90:], k, v, out, lse, N - 90)


@pytest.mark.parametrize("Hq,Hkv,d", FORMS)
@pytest.mark.parametrize("hidden", [1, 31, 32, 64, 128, 130, 300])
@pytest.mark.parametrize("later", [4992.0, -4992.0, 0.0])
def test_scores_of_minus_infinity_weigh_nothing(later, hidden, Hq, Hkv, d):
    # a padding mask written into the keys, then logits beyond what one exponential spans
    few = J < hidden
    q, k, v = _two(Hq, Hkv, d, ONE, torch.where(few, -math.inf, 0.0), torch.where(few, 0.0, later + 32.0 * (J % 7)))
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [N])
    _check(q[hidden:], k[hidden:], v[hidden:], out[hidden:], lse[hidden:], 0)
    # rows whose keys are all so: as rows without a key
    assert not out[:hidden].any() and (lse[:hidden] == -math.inf).all()


@pytest.mark.parametrize("Hq,Hkv,d", FORMS)
def test_scores_of_plus_infinity_and_nan_give_nan(Hq, Hkv, d):
    for x in (math.inf, math.nan):
        for at in (0, 40, 200, 500):
            q, k, v = _two(Hq, Hkv, d, ONE, torch.where(J == at, x, 0.0), 8.0 * (J % 7))
            out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [N])
            assert torch.isnan(out[at:].float()).all() and torch.isnan(lse[at:]).all()
            if at:
                _check(q[:at], k[:at], v[:at], out[:at], lse[:at], 0)
