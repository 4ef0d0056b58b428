"""Pins for the plain 64-bit statements that the prompt attention and paged-cache kernels are tested
against: the framework's own routines, closed forms, planted mistakes.  CPU only."""
import math

import pytest
import torch

import plain64


def _qkv(n, m, Hq, Hkv, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(torch.bfloat16) for s in ((n, Hq, d), (m, Hkv, d), (m, Hkv, d))]


@pytest.mark.parametrize("n,m", [(1, 1), (5, 5), (3, 9), (7, 4)])
def test_attention_matches_the_frameworks_routine(n, m):
    q, k, v = _qkv(n, m, 4, 2, 16)
    out, lse, _, _ = plain64.attention(q, k, v, m - n)
    mask = torch.ones(n, m).tril(m - n).bool()
    rep = lambda x: x.double().repeat_interleave(2, 1).transpose(0, 1)
    some = mask.any(1)
    ref = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1)[:, some], rep(k), rep(v),
                                                           attn_mask=mask[some])
    assert torch.allclose(out[some], ref.transpose(0, 1), rtol=1e-12, atol=1e-14)
    assert not out[~some].any() and torch.isinf(lse[~some]).all()


def test_attention_in_closed_form():
    # equal logits: the mean of what is seen, and its count
    q, k, v = _qkv(4, 6, 1, 1, 8, 1)
    out, lse, scale, mag = plain64.attention(torch.zeros_like(q), k, v, 2)
    for i in range(4):
        assert torch.allclose(out[i, 0], v[:3 + i, 0].double().mean(0)) and math.isclose(lse[i, 0], math.log(3 + i))
    assert torch.allclose(scale[3, 0], v[:, 0].double().abs().mean(0)) and not mag.any()


def test_masked_rows_cannot_reach_a_result():
    q, k, v = _qkv(4, 4, 2, 1, 8, 2)
    want = plain64.attention(q[:2], k[:2], v[:2], 0)
    k[2:], v[2:] = 77.0, -5.0
    got = plain64.attention(q, k, v, 0)
    assert all(torch.allclose(x[:2], y, rtol=1e-12) for x, y in zip(got, want))
    k[0] = 0  # a visible one can
    assert not torch.allclose(plain64.attention(q, k, v, 0)[0][:2], want[0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_unit_numbers(interleaved):
    x = torch.randn(5, 2, 16, generator=torch.Generator().manual_seed(3))
    pos, f = torch.tensor([0, 1, 17, 100000, 2 ** 30]), 10000.0 ** -(torch.arange(4) / 4.0)
    y, size = plain64.rotate(x, pos, f, interleaved)
    z = torch.polar(torch.ones(5, 4, dtype=torch.float64), pos.double()[:, None] * f.double())[:, None]
    a, b = (x[..., 0:8:2], x[..., 1:8:2]) if interleaved else (x[..., :4], x[..., 4:8])
    w = torch.complex(a.double(), b.double()) * z
    got = (y[..., 0:8:2], y[..., 1:8:2]) if interleaved else (y[..., :4], y[..., 4:8])
    assert torch.allclose(got[0], w.real) and torch.allclose(got[1], w.imag)
    assert torch.equal(y[..., 8:], x[..., 8:].double()) and torch.equal(y[0], x[0].double())
    # an inner product of two turned heads depends on the distance of their positions alone
    s = lambda p: (plain64.rotate(x[:1], torch.tensor([p]), f, interleaved)[0] *
                   plain64.rotate(x[1:2], torch.tensor([p + 5]), f, interleaved)[0]).sum()
    assert math.isclose(s(0), s(1000), rel_tol=1e-9)


def test_paged_rows():
    pool = torch.arange(3 * 2 * 4 * 5).float().view(3, 2, 4, 5)
    got = plain64.read_paged(pool, [2, 0, 9], 10)
    assert torch.equal(got[5], pool[0, :, 1]) and torch.equal(got[3], pool[2, :, 3]) and not got[8:].any()
    rows = torch.full((3, 2, 5), -1.0)
    k, v = plain64.append_paged(rows, rows * 2, pool, pool, torch.tensor([[2, 0, 9]]), [3], [0], [3])
    assert (k[2, :, 3] == -1).all() and (k[0, :, :2] == -1).all() and (v[0, :, :2] == -2).all()
    assert (k != pool).sum() == 30                      # nothing else
    k, _ = plain64.append_paged(rows, rows, pool, pool, torch.tensor([[2, 0, 9]]), [7], [0], [3])
    assert (k != pool).sum() == 10                      # the rows on the page outside the pool are dropped
