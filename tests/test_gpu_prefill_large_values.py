"""Values near the end of the number range in the prompt attention.  What is summed before the division by the softmax's
sum is at most (Lk + 64) max|v|, as with a running maximum but for the 64: as long as this is a number, so is the result."""
import pytest
import torch

from paper_2404_14469_b200 import binding as sk
from test_gpu_prefill import _check, _draw

pytestmark = pytest.mark.gpu

N = 900          # (N + 64) max|v| < 2^10 * 2^116 < 2^128


@pytest.mark.parametrize("Hq,Hkv,d", [(2, 1, 128), (4, 2, 64), (32, 8, 128), (64, 16, 64)])   # few query tiles, and many
@pytest.mark.parametrize("logits", ["level", "17 above the first keys", "rising", "one far key per tile"])
@pytest.mark.parametrize("signs", [False, True])
def test_sums_stay_in_range(logits, signs, Hq, Hkv, d):
    q, k, v = _draw(N, N, Hq, Hkv, d, 23, 0.25)
    u = torch.zeros(d, device="cuda")
    u[0] = 1.0
    j = torch.arange(N, device="cuda")
    add = {"level": 0.0 * j, "17 above the first keys": torch.where(j < 32, 0.0, 17.0), "rising": j / 20.0,
           "one far key per tile": torch.where(j % 128 == 77, 17.0, 0.0)}[logits]
    q[:, :, 0], k[:, :, 0] = 4.0, (add * d ** 0.5 / 4.0)[:, None].to(torch.bfloat16)
    v = (1.0 + v.float().abs().clamp(max=0.99)) * (torch.where(v < 0, -1.0, 1.0) if signs else 1.0) * 2.0 ** 115
    v = v.to(torch.bfloat16)
    assert v.abs().max() <= 2.0 ** 116
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [N])
    assert torch.isfinite(out).all()
    _check(q, k, v, out, lse, 0)
    # behind the other keys, where the chains are longest
    out, lse, _ = sk.snapkv_prefill_attention(q[-7:], k, v, [7], [N])
    _check(q[-7:], k, v, out, lse, N - 7)
