"""The calls of a generation run together: the prompts' attention hands its normalisers to the compression,
the compressed caches go into pages, and tokens are appended and attend to them."""
import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("expanded", [False, True])
def test_prompt_to_tokens(expanded):
    lens, Hq, Hkv, d, W, budget, page, steps = [700, 333], 8, 2, 128, 32, 160, 128, 5
    B, T, g = len(lens), sum(lens), torch.Generator(device="cuda").manual_seed(17)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    starts = [0, lens[0]]
    freq = (10000.0 ** -(torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")

    # the prompts into a paged cache, turned by their positions, and the queries with them
    Hc = Hq if expanded else Hkv
    per = -(-max(lens) // page)
    new_pool = lambda heads: torch.full((2 * B * per, heads, page, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    k_pool, v_pool = new_pool(Hkv), new_pool(Hkv)
    table = torch.randperm(2 * B * per, generator=torch.Generator().manual_seed(1))[:B * per].view(B, per).to(torch.int32).cuda()
    q, k, v = 2 * rand(T, Hq, d), rand(T, Hkv, d), rand(T, Hkv, d)
    q = sk.snapkv_append_paged(k, v, k_pool, v_pool, table, i32([0, 0]), i32([0, lens[0], T]), None, freq, q=q)
    k = torch.cat([plain64.read_paged(k_pool, table[b].tolist(), n) for b, n in enumerate(lens)])

    # the prompts' attention, and with its normalisers the same selection as with recomputed ones
    out, lse, lse_obs = sk.snapkv_prefill_attention(q, k, v, lens, window=W)
    q_obs = torch.stack([q[s + n - W:s + n].transpose(0, 1) for s, n in zip(starts, lens)]).contiguous()
    if expanded:
        ck, cv, idx, ws = sk.snapkv_compress_paged(q_obs, k_pool, v_pool, table, max(lens), 7, sk.POOL_MAX, budget,
                                                   seq_lens=lens, lse_obs=lse_obs)
        _, _, idx2, _ = sk.snapkv_compress_paged(q_obs, k_pool, v_pool, table, max(lens), 7, sk.POOL_MAX, budget,
                                                 seq_lens=lens)
    else:
        one = lambda b, n, obs: sk.snapkv_compress_grouped(
            q_obs[b:b + 1], k[starts[b]:starts[b] + n].transpose(0, 1)[None], v[starts[b]:starts[b] + n].transpose(0, 1)[None],
            7, sk.POOL_MAX, budget, lse_obs=obs)
        both = [one(b, n, lse_obs[b:b + 1]) for b, n in enumerate(lens)]
        ck, cv, idx = (torch.cat([x[i] for x in both]) for i in range(3))
        ws = both[0][3]
        idx2 = torch.cat([one(b, n, None)[2] for b, n in enumerate(lens)])
    assert sk.snapkv_device_status(ws) == (sk.OK, 0)
    assert (idx != idx2).float().mean() < 0.02  # near ties alone

    # the compressed caches into pages of their own, with room for the tokens to come
    per = -(-(budget + steps) // page)
    ck_pool, cv_pool = new_pool(Hc), new_pool(Hc)
    table = torch.randperm(2 * B * per, generator=torch.Generator().manual_seed(2))[:B * per].view(B, per).to(torch.int32).cuda()
    sk.snapkv_append_paged(ck.transpose(1, 2), cv.transpose(1, 2), ck_pool, cv_pool, table, i32([0, 0]))
    for b in range(B):
        assert torch.equal(plain64.read_paged(ck_pool, table[b].tolist(), budget), ck[b].transpose(0, 1))
        assert torch.equal(plain64.read_paged(cv_pool, table[b].tolist(), budget), cv[b].transpose(0, 1))

    # a step as a captured graph, its lengths and positions on the device
    q1, k1, v1 = rand(B, 1, Hq, d), rand(B, 1, Hkv, d), rand(B, 1, Hkv, d)
    rows, pos = i32([budget] * B), i32(lens)

    def step(ws=None):
        qr = sk.snapkv_append_paged(k1, v1, ck_pool, cv_pool, table, rows, None, pos, freq, q=q1)
        now = rows + 1
        return qr, *sk.snapkv_decode_paged(qr[:, 0], ck_pool, cv_pool, table, now, ws)

    ws = step()[3]  # (writes the rows that the first replay writes again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qr, out, lse, _ = step(ws)
    hist_k = [plain64.read_paged(ck_pool, table[b].tolist(), budget) for b in range(B)]
    hist_v = [plain64.read_paged(cv_pool, table[b].tolist(), budget) for b in range(B)]
    for _ in range(steps):
        for x in (q1, k1, v1):
            x.copy_(rand(*x.shape))
        graph.replay()
        kr, size = plain64.rotate(k1[:, 0], pos, freq, False)
        tol = plain64.rotate_tolerance(kr, size)
        for b in range(B):
            n = int(rows[b])
            got = plain64.read_paged(ck_pool, table[b].tolist(), n + 1)
            rep = lambda x: x.repeat_interleave(Hc // Hkv, 0)
            assert torch.equal(got[:n], hist_k[b]) and ((got[n].double() - rep(kr[b])).abs() <= rep(tol[b])).all()
            hist_k[b] = got
            hist_v[b] = torch.cat((hist_v[b], rep(v1[b, 0])[None]))
            ref, rlse, scale, mag = plain64.attention(qr[b], hist_k[b], hist_v[b], n)
            assert ((out[b:b + 1].double() - ref).abs() <= plain64.fp32_tolerance(scale, mag, d)).all()
            assert ((lse[b:b + 1].double() - rlse).abs() <= plain64.lse_tolerance(rlse, mag, d)).all()
        rows += 1
        pos += 1
