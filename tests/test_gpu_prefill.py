"""The prompt's attention on the GPU against plain 64-bit attention, element by element."""
import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu


def _draw(n, m, Hq, Hkv, d, seed, q_scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return [x.to(torch.bfloat16) for x in (q_scale * rand(n, Hq, d), rand(m, Hkv, d), rand(m, Hkv, d))]


def _check(q, k, v, out, lse, n_before):
    ref, rlse, scale, mag = plain64.attention(q, k, v, n_before)
    d = q.shape[2]
    err, tol = (out.double() - ref).abs(), plain64.bf16_tolerance(ref, scale, mag, d)
    assert (err <= tol).all(), float((err / tol).max())
    some = torch.isfinite(rlse)
    assert torch.equal(torch.isfinite(lse), some) and (lse[~some] < 0).all() and not out[~some].any()
    err, tol = (lse.double() - rlse).abs()[some], plain64.lse_tolerance(rlse, mag, d)[some]
    assert (err <= tol).all(), float((err / tol).max())


def _starts(lens):
    return [sum(lens[:b]) for b in range(len(lens))]


def _run(lens, k_lens, Hq, Hkv, d, seed=0, q_scale=1.0, window=0):
    q, k, v = _draw(sum(lens), sum(k_lens), Hq, Hkv, d, seed, q_scale)
    out, lse, obs = sk.snapkv_prefill_attention(q, k, v, lens, k_lens, window)
    for b, (q0, n, k0, m) in enumerate(zip(_starts(lens), lens, _starts(k_lens), k_lens)):
        _check(q[q0:q0 + n], k[k0:k0 + m], v[k0:k0 + m], out[q0:q0 + n], lse[q0:q0 + n], m - n)
        if window:
            assert torch.equal(obs[b], lse[q0 + n - window:q0 + n].t())
    return q, k, v, out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 127, 128, 129, 255, 256, 257, 640, 1000])
def test_one_prompt(n, d):
    _run([n], [n], 4, 2, d, n)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (6, 2), (7, 7), (8, 1), (5, 1), (12, 2), (16, 1), (32, 8), (130, 1)])
def test_head_groups(Hq, Hkv):
    _run([70, 201], [70, 201], Hq, Hkv, 128, Hq)
    _run([97], [300], Hq, Hkv, 64, Hq)


@pytest.mark.parametrize("lens,k_lens", [
    ([1], [1000]), ([5], [513]), ([128], [129]), ([200], [4097]), ([300], [700]),  # chunks behind earlier keys
    ([300, 1], [1, 300]), ([129, 64, 7], [128, 0, 3]),                             # queries that see nothing
    ([0, 5, 0, 300], [9, 5, 0, 300]),                                              # nothing to ask, nothing to see
    ([17, 1, 255, 33, 512, 2, 1, 640], [17, 1, 255, 33, 512, 2, 1, 640]),
])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 128), (2, 2, 64)])
def test_packed_sequences_and_chunks(lens, k_lens, Hq, Hkv, d):
    _run(lens, k_lens, Hq, Hkv, d, sum(lens), window=0 if 0 in lens else min(min(lens), 32))


def test_more_sequences_than_a_launch_takes():
    lens = [1 + 37 * i % 200 for i in range(75)]
    _run(lens, [n + i % 3 * 50 for i, n in enumerate(lens)], 4, 2, 128, 3, window=1)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 4, 4)])
def test_a_long_prompt(d, Hq, Hkv):
    _run([5003], [5003], Hq, Hkv, d, 11, window=32)


@pytest.mark.parametrize("q_scale", [0.0, 8.0, 30.0])
def test_large_logits_and_none(q_scale):
    _run([700], [700], 4, 2, 128, 5, q_scale)


def test_rising_and_falling_maxima():
    # keys whose logits rise along the sequence, so that the running maximum moves at every step; and fall
    for sign in (1, -1):
        q, k, v = _draw(600, 600, 2, 1, 128, 9)
        u = torch.randn(128, device="cuda")
        u /= u.norm()
        ramp = torch.linspace(0, 60 * sign, 600, device="cuda")
        q = (q + 6 * u).to(torch.bfloat16)
        k = (k + ramp[:, None, None] * u).to(torch.bfloat16)
        out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [600])
        _check(q, k, v, out, lse, 0)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 2, 1), (64, 4, 2), (128, 1, 1)])
@pytest.mark.parametrize("places", ["every tile", "one key", "few rows"])
def test_maxima_that_rise_far(d, Hq, Hkv, places):
    # by more than fp32 exponentials of one reference can bridge: rows have to take new ones on the way
    n = 900
    q, k, v = _draw(n, n, Hq, Hkv, d, 19)
    u = torch.randn(d, device="cuda")
    u /= u.norm()
    size = torch.full((n,), 30.0, device="cuda")
    ramp = torch.linspace(0, 600, n, device="cuda")
    if places == "one key":    # in the second half of a tile; later tiles fall back
        ramp = torch.zeros(n, device="cuda")
        ramp[[200, 333, 500]] = torch.tensor([90.0, 200.0, 600.0], device="cuda")
    if places == "few rows":
        size = torch.where(torch.arange(n, device="cuda") % 37 == 5, 40.0, 0.0)
    q = (q + size[:, None, None] * u).to(torch.bfloat16)
    k = (k + ramp[:, None, None] * u).to(torch.bfloat16)
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [n])
    _check(q, k, v, out, lse, 0)
    again = sk.snapkv_prefill_attention(q, k, v, [n])
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    # and those that fall as far
    k = k.flip(0)
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [n])
    _check(q, k, v, out, lse, 0)


def test_the_same_bits_every_run_and_in_every_batch():
    q, k, v, out, lse = _run([700, 130], [700, 130], 8, 2, 128, 4)
    again = sk.snapkv_prefill_attention(q, k, v, [700, 130])
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    alone = sk.snapkv_prefill_attention(q[700:], k[700:], v[700:], [130])
    assert torch.equal(alone[0], out[700:]) and torch.equal(alone[1], lse[700:])


@pytest.mark.parametrize("what", ["fused", "heads first", "padded"])
def test_layouts(what):
    lens, Hq, Hkv, d = [200, 77], 8, 2, 128
    T = sum(lens)
    q, k, v = _draw(T, T, Hq, Hkv, d, 21)
    want = sk.snapkv_prefill_attention(q, k, v, lens, window=16)
    if what == "fused":
        f = torch.cat((q, k, v), 1)
        got = sk.snapkv_prefill_attention(f[:, :Hq], f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:], lens, window=16)
    elif what == "heads first":
        t = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
        got = sk.snapkv_prefill_attention(t(q), t(k), t(v), lens, window=16)
    else:  # [B, 256] with NaN behind each sequence; rows of no sequence stay as they were
        pad = lambda x: torch.cat([torch.cat((x[a:a + n], torch.full((256 - n, *x.shape[1:]), float("nan"), device="cuda",
                                                                     dtype=x.dtype))) for a, n in zip(_starts(lens), lens)])
        mark = torch.full((512, Hq, d), 7.0, device="cuda", dtype=torch.bfloat16)
        out, lse, obs = sk.snapkv_prefill_attention(pad(q), pad(k), pad(v), lens, window=16, q_starts=[0, 256],
                                                    k_starts=[0, 256], out=mark)
        assert out.data_ptr() == mark.data_ptr() and (out[200:256] == 7).all() and (out[333:] == 7).all()
        assert torch.isinf(lse[200:256]).all() and torch.isinf(lse[333:]).all()
        got = [torch.cat((x[:200], x[256:333])) for x in (out, lse)] + [obs]
        fresh, _, none = sk.snapkv_prefill_attention(pad(q), pad(k), pad(v), lens, q_starts=[0, 256], k_starts=[0, 256])
        assert none is None and not fresh[200:256].any() and not fresh[333:].any() and torch.equal(fresh[:200], out[:200])
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_sequences_may_share_keys_and_their_neighbours_values_do_not_reach_them():
    q, k, v = _draw(100, 400, 4, 2, 128, 31)
    out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [60, 40], [300, 200], k_starts=[0, 0])
    _check(q[:60], k[:300], v[:300], out[:60], lse[:60], 240)
    _check(q[60:], k[:200], v[:200], out[60:], lse[60:], 160)
    v[200:], k[200:] = float("inf"), float("nan")
    again = sk.snapkv_prefill_attention(q[60:], k, v, [40], [200])
    assert torch.equal(again[0], out[60:]) and torch.equal(again[1], lse[60:])


def test_masked_keys_may_hold_anything():
    # a later key's infinity or NaN does not reach the queries in front of it (its value's may, as documented)
    q, k, v = _draw(300, 300, 2, 1, 128, 41)
    want = sk.snapkv_prefill_attention(q, k, v, [300])
    for x in (float("nan"), float("inf"), torch.finfo(torch.bfloat16).min):
        k[290:] = x
        got = sk.snapkv_prefill_attention(q, k, v, [300])
        assert torch.equal(got[0][:290], want[0][:290]) and torch.equal(got[1][:290], want[1][:290])


def test_stream_and_graph():
    q, k, v = _draw(333, 333, 8, 2, 128, 51)
    want = sk.snapkv_prefill_attention(q, k, v, [333], window=32)
    s = torch.cuda.Stream()
    out = torch.empty_like(want[0])
    with torch.cuda.stream(s):
        sk.snapkv_prefill_attention(q, k, v, [333], window=32, out=out)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got = sk.snapkv_prefill_attention(q, k, v, [333], window=32, out=out)
    s.synchronize()
    q.mul_(0.5)
    out.zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    want = sk.snapkv_prefill_attention(q, k, v, [333], window=32)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_refusals():
    q, k, v = _draw(40, 50, 4, 2, 128, 61)
    for bad in [lambda: sk.snapkv_prefill_attention(q, k, v, [41]),                  # beyond the tokens
                lambda: sk.snapkv_prefill_attention(q, k, v, [40], [51]),
                lambda: sk.snapkv_prefill_attention(q, k, v, [20, 20], q_starts=[0, 10]),
                lambda: sk.snapkv_prefill_attention(q, k, v, [20, 20], [20]),
                lambda: sk.snapkv_prefill_attention(q, k, v, [40], window=41),
                lambda: sk.snapkv_prefill_attention(q, k, v, []),
                lambda: sk.snapkv_prefill_attention(q, k, v, [2 ** 33]),
                lambda: sk.snapkv_prefill_attention(q, k, v, [-1]),
                lambda: sk.snapkv_prefill_attention(q.float(), k, v, [40]),
                lambda: sk.snapkv_prefill_attention(q, k, v[:, :1], [40]),
                lambda: sk.snapkv_prefill_attention(q[:, :3], k, v, [40]),
                lambda: sk.snapkv_prefill_attention(q[..., :64], k, v, [40]),
                lambda: sk.snapkv_prefill_attention(q.transpose(1, 2), k, v, [40]),
                lambda: sk.snapkv_prefill_attention(q.cpu(), k, v, [40]),
                lambda: sk.snapkv_prefill_attention(q, k, v, [40], out=q[:20])]:
        with pytest.raises(sk.SnapKVError):
            bad()
