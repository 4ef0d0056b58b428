"""The prompt's attention has two forms, for fewer query tiles than SMs and for more; the same hard cases with enough
heads for the second one."""
import pytest
import torch

from paper_2404_14469_b200 import binding as sk
from test_gpu_prefill import _check, _draw, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d", [(64, 16, 128), (32, 32, 64), (48, 16, 128), (40, 8, 64)])
@pytest.mark.parametrize("lens,k_lens", [
    ([700, 1, 300], [700, 1, 300]),                 # packed prompts
    ([513], [900]), ([257, 640], [1500, 640]),      # chunks behind earlier keys
    ([900, 300, 128], [200, 0, 127]),               # queries that see nothing
    ([640, 0, 129, 255], [640, 7, 129, 255]),
])
def test_many_query_tiles(Hq, Hkv, d, lens, k_lens):
    _run(lens, k_lens, Hq, Hkv, d, sum(lens), window=0 if 0 in lens else 1)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (32, 32)])
@pytest.mark.parametrize("places", ["every tile", "one key", "few rows"])
def test_maxima_that_rise_far_in_many_tiles(Hq, Hkv, places):
    n, d = 900, 128
    q, k, v = _draw(n, n, Hq, Hkv, d, 19)
    u = torch.randn(d, device="cuda")
    u /= u.norm()
    size = torch.full((n,), 30.0, device="cuda")
    ramp = torch.linspace(0, 600, n, device="cuda")
    if places == "one key":
        ramp = torch.zeros(n, device="cuda")
        ramp[[200, 333, 500]] = torch.tensor([90.0, 200.0, 600.0], device="cuda")
    if places == "few rows":
        size = torch.where(torch.arange(n, device="cuda") % 37 == 5, 40.0, 0.0)
    q = (q + size[:, None, None] * u).to(torch.bfloat16)
    k = (k + ramp[:, None, None] * u).to(torch.bfloat16)
    for keys in (k, k.flip(0)):
        out, lse, _ = sk.snapkv_prefill_attention(q, keys, v, [n])
        _check(q, keys, v, out, lse, 0)
        again = sk.snapkv_prefill_attention(q, keys, v, [n])
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_neighbours_and_masked_keys_in_many_tiles():
    q, k, v = _draw(800, 1000, 32, 8, 128, 7)
    want = sk.snapkv_prefill_attention(q, k, v, [500, 300], [500, 300])
    k[800:], v[800:] = float("nan"), float("inf")   # behind the last sequence
    k[790:800] = float("nan")                       # seen by its last ten queries alone
    got = sk.snapkv_prefill_attention(q, k, v, [500, 300], [500, 300])
    assert torch.equal(got[0][:790], want[0][:790]) and torch.equal(got[1][:790], want[1][:790])
    assert torch.isnan(got[1][790:]).all()


@pytest.mark.parametrize("n", [100, 1000])
def test_graphs_of_both_forms(n):
    q, k, v = _draw(n, n, 32, 8, 128, n)
    sk.snapkv_prefill_attention(q, k, v, [n])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse, _ = sk.snapkv_prefill_attention(q, k, v, [n])
    for scale in (0.5, 2.0):
        q.mul_(scale)
        for _ in range(5):
            g.replay()
        want = sk.snapkv_prefill_attention(q, k, v, [n])
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
