"""How exact the paged decode is: three bf16 terms per probability, and sums of the matrix instructions that are flushed
into rounded ones.  The scores are exact (two elements of queries and keys are not zero), so that the bounds are tight
enough to tell; either measure left out fails here."""
import math

import pytest
import torch

from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a step of fp32 next to 1; an operand that is cut loses up to 2 U


def _exact(scores, v):
    """scores [n], v [n, d] in 64 bits: the attention's output and sum_j p_j |v_j|."""
    p = torch.softmax(scores, 0)
    return p @ v, p @ v.abs()


@pytest.mark.parametrize("Hq", [1, 4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_probabilities_keep_24_bits(d, Hq):
    # three rows a sequence, logits below 0.7 (1 in the log2 domain)
    B, n, page = 400, 3, 16
    g = torch.Generator(device="cuda").manual_seed(d + Hq)
    q, k = torch.zeros(B, Hq, d, device="cuda"), torch.zeros(B, 1, page, d, device="cuda")
    q[:, :, 0] = 1 + torch.arange(Hq, device="cuda") % 3      # scores of one number and of a few bits
    k[:, 0, :, 0] = torch.randint(-127, 128, (B, page), generator=g, device="cuda") / 128.0
    v = torch.randn(B, 1, page, d, generator=g, device="cuda")
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None]
    out, _, _ = sk.snapkv_decode_paged(q, k, v, table, torch.full((B,), n, dtype=torch.int32, device="cuda"))
    # a weight: its exponent (scale and product, 1.5 U of at most 1; difference, 1 U of at most 2; ln 2), ex2 4 U, the terms 1 U
    # the output: four addends that may be cut 8 U, the sum of the weights 3 U, the quotient 3 U
    tol = (0.7 * 3.5 + 4 + 1 + 8 + 3 + 3) * U
    for b in range(B):
        for h in range(Hq):
            ref, scale = _exact(k[b, 0, :n].double() @ q[b, h].double() / math.sqrt(d), v[b, 0, :n].double())
            assert ((out[b, h].double() - ref).abs() <= tol * scale).all(), (b, h, float(((out[b, h].double() - ref).abs() / scale).max() / U))


@pytest.mark.parametrize("d,rows", [(64, 32), (128, 16)])
def test_long_sums_are_rounded_not_cut(d, rows):
    # more sequences than warps, all over the same 131072 rows: thousands of tiles for a warp; positive values, so that
    # what is cut off adds up
    B, n, page = 1300, 131072, 256
    g = torch.Generator(device="cuda").manual_seed(d)
    q, k = torch.zeros(B, 1, d, device="cuda"), torch.zeros(n // page, 1, page, d, device="cuda")
    q[:, :, 0] = 1
    k[..., 0] = torch.randint(-127, 128, k.shape[:3], generator=g, device="cuda") / 128.0
    v = 1 + torch.rand(n // page, 1, page, d, generator=g, device="cuda")
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(B, 1)
    out, _, _ = sk.snapkv_decode_paged(q, k, v, table, torch.full((B,), n, dtype=torch.int32, device="cuda"))
    ref, scale = _exact(k.view(n, d).double() @ q[0, 0].double() / math.sqrt(d), v.view(n, d).double())
    # between two flushes 8 tiles, an instruction per 16 rows with 17 addends that may be cut; then a rounding per flush;
    # the weights as above, their sum (cut nowhere) with a rounding per 16 rows and lane
    flushes = n // (8 * rows)
    tol = (8 * (rows // 16) * 17 * 2 + flushes + n // 16 / 8 + 16) * U
    assert ((out[:, 0].double() - ref).abs() <= tol * scale).all(), float(((out[:, 0].double() - ref).abs() / scale).max() / U)
