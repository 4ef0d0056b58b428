"""The prompt's attention at its limits: wide groups, halves of fused rows, long contexts for few queries, offsets
beyond 32 bits."""
import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk
from test_gpu_prefill import _check, _draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,n", [(64, 1, 128, 70), (128, 1, 64, 9), (128, 2, 128, 33), (48, 1, 64, 50)])
def test_wide_groups(Hq, Hkv, d, n):
    q, k, v = _draw(n, n + 200, Hq, Hkv, d, Hq)
    out, lse, obs = sk.snapkv_prefill_attention(q, k, v, [n], [n + 200], window=9)
    _check(q, k, v, out, lse, 200)
    assert torch.equal(obs[0], lse[n - 9:].t())


def test_keys_and_values_as_halves_of_the_same_rows():
    q, k, v = _draw(300, 300, 4, 2, 64, 3)
    want = sk.snapkv_prefill_attention(q, k, v, [300])
    kv = torch.cat((k, v), -1)
    got = sk.snapkv_prefill_attention(q, kv[..., :64], kv[..., 64:], [300])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n,m", [(1, 100000), (3, 70001), (200, 30000)])
def test_few_queries_behind_a_long_context(n, m):
    q, k, v = _draw(n, m, 4, 2, 128, n, 2.0)
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [n], [m])
    _check(q, k, v, out, lse, m - n)


def test_tokens_whose_offsets_pass_32_bits():
    T, Hq, Hkv, d, n = 530000, 32, 2, 128, 300        # 2.2e9 elements of q and of the output
    q = torch.zeros(T, Hq, d, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    qs, k, v = _draw(n, n, Hq, Hkv, d, 5)
    start = T - n - 7
    q[start:start + n] = qs
    _, lse, _ = sk.snapkv_prefill_attention(q, k, v, [n], q_starts=[start], out=out)
    _check(qs, k, v, out[start:start + n], lse[start:start + n], 0)
    assert not out[start + n:].any() and not out[:start].any()
    del q, out, lse
    # and of the keys
    k2 = torch.zeros(2 ** 31 // (Hkv * d) + 2000, Hkv, d, dtype=torch.bfloat16, device="cuda")
    start = k2.shape[0] - n - 5
    k2[start:start + n] = k
    got = sk.snapkv_prefill_attention(qs, k2, k2, [n], k_starts=[start])
    want = sk.snapkv_prefill_attention(qs, k, k, [n])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_large_values_are_not_lost_to_the_reference():
    # logits that rise from tile to tile, values far from 1
    q, k, v = _draw(600, 600, 2, 1, 128, 8)
    u = torch.randn(128, device="cuda")
    u /= u.norm()
    q = (q + 8 * u).to(torch.bfloat16)
    k = (k + torch.linspace(0, 120, 600, device="cuda")[:, None, None] * u).to(torch.bfloat16)
    for size in (1e15, 1e-25):
        big = (v.float() * size).to(torch.bfloat16)
        out, lse, _ = sk.snapkv_prefill_attention(q, k, big, [600])
        ref, rlse, scale, mag = plain64.attention(q, k, big, 0)
        assert ((out.double() - ref).abs() <= plain64.bf16_tolerance(ref, scale, mag, 128)).all()
