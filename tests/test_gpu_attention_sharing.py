"""The prompt attention and the paged cache's calls beside one another: on streams, threads and graphs."""
import threading

import pytest
import torch

from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _case(seed, B=3, Hq=8, Hkv=2, d=128, page=32, rows=700):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    per = -(-(rows + 1) // page)
    return dict(q=rand(B, 1, Hq, d), k=rand(B, 1, Hkv, d), v=rand(B, 1, Hkv, d), kp=rand(B * per, Hkv, page, d),
                vp=rand(B * per, Hkv, page, d), table=torch.arange(B * per, device="cuda", dtype=torch.int32).view(B, per),
                lens=_i32([rows - 7 * b for b in range(B)]), freq=(10000.0 ** -(torch.arange(0, d, 2) / d)).float().cuda(),
                pq=rand(500, Hq, d), pk=rand(500, Hkv, d), pv=rand(500, Hkv, d))


def _step(c, ws=None):
    qr = sk.snapkv_append_paged(c["k"], c["v"], c["kp"], c["vp"], c["table"], c["lens"], inv_freq=c["freq"], q=c["q"])
    out, lse, ws = sk.snapkv_decode_paged(qr[:, 0], c["kp"], c["vp"], c["table"], c["lens"] + 1, ws)
    a, e, _ = sk.snapkv_prefill_attention(c["pq"], c["pk"], c["pv"], [300, 200])
    return [qr, out, lse, a, e], ws


def _same(x, y):
    return all(torch.equal(a, b) for a, b in zip(x, y))


def test_calls_on_two_streams_at_once():
    cases = [_case(s, rows=4000) for s in (1, 2)]
    want = [_step(c)[0] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(_step(c)[0])
        torch.cuda.synchronize()
        assert all(_same(g, w) for g, w in zip(got, want))


def test_threads_whose_first_calls_these_are():
    cases = [_case(s) for s in range(6)]
    want = [_step(c)[0] for c in cases]
    torch.cuda.synchronize()
    got, gate = [None] * len(cases), threading.Barrier(len(cases))

    def work(i):
        gate.wait()
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = _step(cases[i])[0]
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert all(g is not None and _same(g, w) for g, w in zip(got, want))


def test_two_graphs_share_a_workspace_and_are_replayed_in_turn():
    a, b = _case(3, rows=5000), _case(4, B=5, rows=90)
    want = [_step(a)[0], _step(b)[0]]
    ws = _step(a)[1]
    ws.fill_(255)  # whatever was in it
    graphs, outs = [], []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_step(c, ws)[0])
        graphs.append(g)
    for i in (0, 1, 0, 0, 1, 1, 0):
        for o in outs[i]:
            o.fill_(7)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert _same(outs[i], want[i])
    # and a plain call between replays
    assert _same(_step(a, ws)[0], want[0])
    graphs[1].replay()
    torch.cuda.synchronize()
    assert _same(outs[1], want[1])


def test_one_graph_replayed_many_times_back_to_back():
    c = _case(5, rows=9000)
    want, ws = _step(c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _step(c, ws)[0]
    for _ in range(300):
        g.replay()
    torch.cuda.synchronize()
    assert _same(out, want)


def test_calls_right_behind_the_kernels_that_make_their_inputs():
    # no waiting between producers and consumers: what a call reads is what the stream's last kernel wrote
    c = _case(6, rows=3000)
    want = _step(c)[0]
    for _ in range(50):
        k, v, q = (torch.empty_like(c[x]).fill_(3.0) for x in "kvq")
        k.copy_(c["k"]), v.copy_(c["v"]), q.copy_(c["q"])
        lens = (c["lens"].float() * 2).to(torch.int32) // 2
        assert _same(_step(dict(c, k=k, v=v, q=q, lens=lens))[0], want)


def test_decode_with_nan_in_one_query_head_leaves_the_others():
    c = _case(7)
    q = c["q"][:, 0].contiguous()
    want = sk.snapkv_decode_paged(q, c["kp"], c["vp"], c["table"], c["lens"])
    bad = q.clone()
    bad[1, 5] = float("nan")
    got = sk.snapkv_decode_paged(bad, c["kp"], c["vp"], c["table"], c["lens"])
    keep = torch.ones(3, 8, dtype=torch.bool, device="cuda")
    keep[1, 5] = False
    assert torch.isnan(got[0][1, 5]).all() and torch.isnan(got[1][1, 5])
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])


def test_prefill_with_nan_in_one_query_leaves_the_others():
    c = _case(8)
    want = sk.snapkv_prefill_attention(c["pq"], c["pk"], c["pv"], [500])
    bad = c["pq"].clone()
    bad[77, 3] = float("nan")
    got = sk.snapkv_prefill_attention(bad, c["pk"], c["pv"], [500])
    keep = torch.ones(500, 8, dtype=torch.bool, device="cuda")
    keep[77, 3] = False
    assert torch.isnan(got[0][77, 3].float()).all() and torch.isnan(got[1][77, 3])
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])
