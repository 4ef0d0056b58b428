"""A prompt alone and in batches: the other sequences decide how the work is split, so the order of the sums may change with
them, the result only by what that order may do."""
import pytest
import torch

from paper_2404_14469_b200 import binding as sk
from test_gpu_prefill import _check, _draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (16, 16, 64)])
def test_a_prompt_alone_and_among_others(Hq, Hkv, d):
    lens = [130] + [400] * 12
    q, k, v = _draw(sum(lens), sum(lens), Hq, Hkv, d, 4)
    n = lens[0]
    alone, lse, _ = sk.snapkv_prefill_attention(q[:n], k[:n], v[:n], [n])
    among = sk.snapkv_prefill_attention(q, k, v, lens)
    for out, e in ((alone, lse), (among[0][:n], among[1][:n])):
        _check(q[:n], k[:n], v[:n], out, e, 0)
    # the same number of tiles of each form: the same bits, whoever the others are
    other = [130] + [200] * 24
    again = sk.snapkv_prefill_attention(q, k, v, other)
    assert torch.equal(again[0][:n], among[0][:n]) and torch.equal(again[1][:n], among[1][:n])
    two = sk.snapkv_prefill_attention(q[:n + 50], k[:n + 50], v[:n + 50], [n, 50])
    assert torch.equal(two[0][:n], alone) and torch.equal(two[1][:n], lse)
