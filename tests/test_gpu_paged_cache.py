"""The paged cache of the generation steps on the GPU, appending to it and attending to it, against plain
64-bit statements."""
import pytest
import torch

import plain64
from paper_2404_14469_b200 import binding as sk

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _bf16(g, *s):
    return torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(lens, heads, page, d, seed, spare=0, layout="heads"):
    """Pools with a random page order, NaN in every row that no sequence has."""
    g = _gen(seed)
    per = max(-(-max(lens) // page) + spare, 1)
    pages = len(lens) * per + 2
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:len(lens) * per]
    table = order.view(len(lens), per).to(torch.int32).cuda()
    shape = (pages, heads, page, d) if layout == "heads" else (pages, page, heads, d)
    k, v = _bf16(g, *shape), _bf16(g, *shape)
    if layout != "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        for p in range(-(-n // page)):
            used[int(table[b, p]), :min(page, n - p * page)] = True
    k.masked_fill_(~used[:, None, :, None], NAN)
    v.masked_fill_(~used[:, None, :, None], NAN)
    return k, v, table


def _check_decode(q, k, v, table, lens, out, lse):
    ref, rlse, scale, mag = plain64.decode_paged(q, k, v, table, lens)
    d = q.shape[2]
    err, tol = (out.double() - ref).abs(), plain64.fp32_tolerance(scale, mag, d)
    assert (err <= tol).all(), float((err / tol).max())
    some = torch.isfinite(rlse)
    assert torch.equal(torch.isfinite(lse), some) and (lse[~some] < 0).all() and not out[~some].any()
    err, tol = (lse.double() - rlse).abs()[some], plain64.lse_tolerance(rlse, mag, d)[some]
    assert (err <= tol).all(), float((err / tol).max())


def _decode(lens, Hq, Hc, page, d, seed=0, layout="heads", q_scale=1.0):
    k, v, table = _cache(lens, Hc, page, d, seed, layout=layout)
    q = (q_scale * _bf16(_gen(seed + 1), len(lens), Hq, d)).to(torch.bfloat16)
    out, lse, ws = sk.snapkv_decode_paged(q, k, v, table, _i32(lens))
    _check_decode(q, k, v, table, lens, out, lse)
    return q, k, v, table, out, lse, ws


# ------------------------------------------------------------------------------------------ decode
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 100, 128, 129, 1000, 4099])
def test_decode_lengths(n, d):
    _decode([n], 4, 2, 32, d, n)


@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("d,layout", [(64, "heads"), (128, "heads"), (128, "rows"), (64, "rows")])
def test_decode_pages_and_layouts(page, d, layout):
    _decode([1, 700, 255, 16, 300], 8, 2, page, d, page, layout)


@pytest.mark.parametrize("Hq,Hc", [(1, 1), (3, 1), (6, 2), (7, 7), (8, 1), (9, 1), (17, 1), (32, 8), (40, 2)])
def test_decode_head_groups(Hq, Hc):
    _decode([333, 50], Hq, Hc, 64, 128, Hq)
    _decode([333, 50], Hq, Hc, 16, 64, Hq)


@pytest.mark.parametrize("lens", [[0], [0, 0, 0], [5, 0, 2000, 0, 1], [3000] + [1] * 40, [7] * 150,
                                  [1 + 113 * i % 977 for i in range(90)]])
def test_decode_ragged_batches(lens):
    _decode(lens, 4, 2, 32, 128, len(lens))


@pytest.mark.parametrize("B,Hq,Hc,n", [(1, 1, 1, 40000), (1, 32, 8, 20000), (5, 8, 8, 9001), (1, 2, 1, 150000)])
def test_decode_long_caches_are_split_and_joined(B, Hq, Hc, n):
    _decode([n - 77 * b for b in range(B)], Hq, Hc, 128, 128, n)


@pytest.mark.parametrize("q_scale", [0.0, 10.0, 40.0])
def test_decode_large_logits_and_none(q_scale):
    _decode([900, 3], 4, 2, 64, 128, 5, q_scale=q_scale)


def test_decode_the_same_bits_every_run_with_one_workspace():
    q, k, v, table, out, lse, ws = _decode([4000, 17, 900], 8, 2, 64, 128, 8)
    ws.fill_(255)  # whatever was in it
    again = sk.snapkv_decode_paged(q, k, v, table, _i32([4000, 17, 900]), ws)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse) and again[2] is ws
    assert sk.snapkv_decode_paged(q, k, v, table, _i32([4000, 17, 900]), ws, want_lse=False)[1] is None


def test_decode_agrees_with_the_dense_call():
    B, Hq, Hc, rows, d = 2, 8, 2, 640, 128
    g = _gen(3)
    q, k, v = _bf16(g, B, Hq, d), _bf16(g, B, Hc, rows, d), _bf16(g, B, Hc, rows, d)
    want = sk.snapkv_decode_attention(q, k, v)
    # the dense cache is a pool of B pages of `rows` rows
    got = sk.snapkv_decode_paged(q, k, v, _i32([[0], [1]]), _i32([rows, rows]))
    assert torch.allclose(got[0], want[0], rtol=0, atol=1e-5) and torch.allclose(got[1], want[1], rtol=0, atol=1e-5)


def test_decode_lengths_and_tables_out_of_range():
    k, v, table = _cache([64, 64, 64], 2, 16, 64, 4)
    q = _bf16(_gen(5), 3, 4, 64)
    table[0, 1], table[0, 2], table[1, 0] = -1, k.shape[0], 2 ** 30     # read as zeros
    lens = [64, 1000, -5]                                               # clamped: 64 and 0
    out, lse, _ = sk.snapkv_decode_paged(q, k, v, table, _i32(lens))
    _check_decode(q, k, v, table, lens, out, lse)


def test_decode_graph_follows_the_lengths():
    lens = _i32([100, 500])
    k, v, table = _cache([600, 600], 2, 64, 128, 6)
    q = _bf16(_gen(7), 2, 8, 128)
    ws = sk.snapkv_decode_paged(q, k, v, table, lens)[2]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse, _ = sk.snapkv_decode_paged(q, k, v, table, lens, ws)
    for now in ([100, 500], [101, 600], [600, 1], [0, 64]):
        lens.copy_(_i32(now))
        g.replay()
        _check_decode(q, k, v, table, now, out, lse)


def test_decode_rows_beyond_32_bit_offsets():
    # a pool of more than 2^31 elements: the sequence's pages are its last ones
    pages, page, d = 2 ** 31 // (128 * 128) + 40, 128, 128
    k = torch.zeros(pages, 1, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = _gen(11)
    k[-5:], v[-5:] = _bf16(g, 5, 1, page, d), _bf16(g, 5, 1, page, d)
    table, q = _i32([[pages - 1, pages - 3, pages - 5]]), _bf16(g, 1, 4, d)
    out, lse, _ = sk.snapkv_decode_paged(q, k, v, table, _i32([300]))
    _check_decode(q, k, v, table, [300], out, lse)
    new = _bf16(g, 1, 1, d)
    sk.snapkv_append_paged(new, new, k, v, table, _i32([300]), _i32([0, 1]))
    assert torch.equal(k[pages - 5, 0, 44], new[0, 0]) and torch.equal(v[pages - 5, 0, 44], new[0, 0])


def test_decode_refusals():
    k, v, table = _cache([64], 2, 16, 64, 9)
    q, lens = _bf16(_gen(1), 1, 4, 64), _i32([64])
    for bad in [lambda: sk.snapkv_decode_paged(q, k, v, table, lens.long()),
                lambda: sk.snapkv_decode_paged(q, k, v, table, _i32([64, 64])),
                lambda: sk.snapkv_decode_paged(q, k, v, table.long(), lens),
                lambda: sk.snapkv_decode_paged(q, k, v, table[0], lens),
                lambda: sk.snapkv_decode_paged(q, k, v[:, :1], table, lens),
                lambda: sk.snapkv_decode_paged(q[:, :3], k, v, table, lens),
                lambda: sk.snapkv_decode_paged(q, k[:, :, :8], v[:, :, :8], table, lens),
                lambda: sk.snapkv_decode_paged(q[:, ::2], k, v, table, lens),
                lambda: sk.snapkv_decode_paged(q.cpu(), k, v, table, lens),
                lambda: sk.snapkv_decode_paged(q, k, v, table, lens.cpu()),
                lambda: sk.snapkv_decode_paged(q, k.transpose(2, 3), v.transpose(2, 3), table, lens)]:
        with pytest.raises(sk.SnapKVError):
            bad()


# ------------------------------------------------------------------------------------------ append
def _expect(k_new, v_new, k_pool, v_pool, table, cache_lens, counts, turn=None):
    """The pools that a call must leave, and the tolerance of K (None: the same bits)."""
    reps, starts = k_pool.shape[1] // k_new.shape[1], [sum(counts[:b]) for b in range(len(counts))]
    kr, size = (k_new.double(), None) if turn is None else plain64.rotate(k_new, *turn)
    rep = lambda x: x.repeat_interleave(reps, 1)
    args = (table, cache_lens, starts, counts)
    k, v = plain64.append_paged(rep(kr), rep(v_new).double(), k_pool.double(), v_pool.double(), *args)
    if size is None:
        return k, v, None
    zero = torch.zeros_like(k_pool, dtype=torch.float64)
    tol, _ = plain64.append_paged(rep(plain64.rotate_tolerance(kr, size)), rep(v_new).double(), zero, zero, *args)
    return k, v, tol


def _check_append(k, v, want):
    ref, vref, tol = want
    assert torch.equal(torch.nan_to_num(v.double(), 1e30), torch.nan_to_num(vref, 1e30))
    err = (torch.nan_to_num(k.double(), 1e30) - torch.nan_to_num(ref, 1e30)).abs()
    assert (err <= (0 if tol is None else tol)).all()


FREQ = lambda rot, base=10000.0: (base ** -(torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (128, 16), (64, 32), (128, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,Hc,page", [(4, 2, 2, 32), (6, 2, 6, 7), (1, 1, 1, 128)])
def test_append_with_rotation(d, rot, interleaved, Hq, Hkv, Hc, page):
    counts, before = [1, 40, 0, 3, 100], [0, 31, 5, 64, 27]
    lens = [a + b for a, b in zip(counts, before)]
    k_pool, v_pool, table = _cache(lens, Hc, page, d, rot, spare=1)
    g = _gen(rot + Hq)
    T = sum(counts)
    f = _bf16(g, T, Hq + 2 * Hkv, d)
    q, k, v = f[:, :Hq], f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:]
    pos = torch.randint(0, 400000, (T,), generator=g, device="cuda", dtype=torch.int32)
    freq = FREQ(rot)
    want = _expect(k, v, k_pool, v_pool, table, before, counts, (pos, freq, interleaved))
    cu = _i32([sum(counts[:b]) for b in range(6)])
    got = sk.snapkv_append_paged(k, v, k_pool, v_pool, table, _i32(before), cu, pos, freq, interleaved, q)
    _check_append(k_pool, v_pool, want)
    ref, size = plain64.rotate(q, pos, freq, interleaved)
    assert ((got.double() - ref).abs() <= plain64.rotate_tolerance(ref, size)).all()


@pytest.mark.parametrize("d,rot,interleaved,Hq,Hkv,Hc,counts", [
    (128, 128, False, 6, 2, 6, [5000, 1, 0, 777]),      # many tokens: several share a block
    (64, 32, True, 3, 1, 1, [13, 6001]),
    (128, 96, True, 4, 4, 4, [2, 3] * 1100),            # more sequences than one probe of a warp tells apart
    (64, 64, False, 2, 2, 2, [1] * 40 + [0] * 5 + [7]),
    (128, 64, False, 33, 3, 33, [1, 2]),                # more heads than a block takes at a time
])
def test_append_many_tokens_and_sequences(d, rot, interleaved, Hq, Hkv, Hc, counts):
    page = 16
    before = [3 * b % 20 for b in range(len(counts))]
    k_pool, v_pool, table = _cache([x + n for x, n in zip(before, counts)], Hc, page, d, rot)
    g = _gen(rot + Hq)
    T = sum(counts)
    f = _bf16(g, T, Hq + 2 * Hkv, d)
    q, k, v = f[:, :Hq], f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:]
    pos = torch.randint(0, 400000, (T,), generator=g, device="cuda", dtype=torch.int32)
    starts = torch.cumsum(torch.tensor([0] + counts), 0)
    b = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts))
    slot = torch.tensor(before)[b] + torch.arange(T) - starts[b]
    where = (table.long()[b.cuda(), (slot // page).cuda()], slice(None), (slot % page).cuda())
    kr, size = plain64.rotate(k, pos, FREQ(rot), interleaved)
    rep = lambda x: x.repeat_interleave(Hc // Hkv, 1)
    want_k, want_v, tol = k_pool.double(), v_pool.clone(), torch.zeros_like(k_pool, dtype=torch.float64)
    want_k[where], want_v[where], tol[where] = rep(kr), rep(v), rep(plain64.rotate_tolerance(kr, size))
    got = sk.snapkv_append_paged(k, v, k_pool, v_pool, table, _i32(before), starts.to(torch.int32).cuda(), pos, FREQ(rot),
                                 interleaved, q)
    assert torch.equal(torch.nan_to_num(v_pool, 1e30), torch.nan_to_num(want_v, 1e30))
    err = (torch.nan_to_num(k_pool.double(), 1e30) - torch.nan_to_num(want_k, 1e30)).abs()
    assert (err <= tol).all()
    ref, size = plain64.rotate(q, pos, FREQ(rot), interleaved)
    assert ((got.double() - ref).abs() <= plain64.rotate_tolerance(ref, size)).all()


@pytest.mark.parametrize("Hc,n", [(2, 1), (2, 50), (8, 33)])
def test_append_dense_batches_at_their_cache_rows(Hc, n):
    B, Hq, Hkv, d, page, before = 3, 8, 2, 128, 64, [0, 100, 63]
    k_pool, v_pool, table = _cache([x + n for x in before], Hc, page, d, n, layout="rows")
    g = _gen(n)
    k, v, q = _bf16(g, B, n, Hkv, d), _bf16(g, B, Hkv, n, d).transpose(1, 2), _bf16(g, B, n, Hq, d)
    pos = torch.cat([torch.arange(x, x + n) for x in before]).cuda()
    turn = (pos, FREQ(d), False)
    want = _expect(k.flatten(0, 1), v.flatten(0, 1), k_pool, v_pool, table, before, [n] * B, turn)
    out = torch.empty_like(q)
    got = sk.snapkv_append_paged(k, v, k_pool, v_pool, table, _i32(before), inv_freq=FREQ(d), q=q, q_out=out)
    assert got is out
    _check_append(k_pool, v_pool, want)
    ref, size = plain64.rotate(q.flatten(0, 1), *turn)
    assert ((got.flatten(0, 1).double() - ref).abs() <= plain64.rotate_tolerance(ref, size)).all()


def test_append_copies_bits_without_rotation_and_leaves_all_else():
    # any bit pattern, NaN payloads among them, from a dense compressed cache [B, H, rows, d]
    B, H, rows, d, page = 2, 4, 100, 128, 32
    k_pool, v_pool, table = _cache([rows] * B, H, page, d, 1, spare=1)
    g = _gen(2)
    k, v = (torch.randint(-2 ** 15, 2 ** 15, (B, H, rows, d), generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
            for _ in "kv")
    ints = lambda x: x.view(torch.int16)
    want = [ints(p.clone()) for p in (k_pool, v_pool)]
    for b in range(B):
        for r in range(rows):
            for w, x in zip(want, (k, v)):
                w[int(table[b, r // page]), :, r % page] = ints(x)[b, :, r]
    assert sk.snapkv_append_paged(k.transpose(1, 2), v.transpose(1, 2), k_pool, v_pool, table, _i32([0, 0])) is None
    assert torch.equal(ints(k_pool), want[0]) and torch.equal(ints(v_pool), want[1])


def test_append_skips_padding_and_rows_without_a_place():
    d, page = 64, 16
    k_pool, v_pool, table = _cache([32, 32, 32], 1, page, d, 3)
    table[1, 1], table[2, 0] = -1, k_pool.shape[0]
    counts, before = [6, 20, 20], [30, 3, 0]  # beyond the table; onto pages outside the pool
    g = _gen(4)
    T = sum(counts) + 9
    k, v, q = _bf16(g, T, 1, d), _bf16(g, T, 1, d), _bf16(g, T, 2, d)
    want = _expect(k, v, k_pool, v_pool, table, before, counts)
    out = torch.full_like(q, 7.0)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    sk.snapkv_append_paged(k, v, k_pool, v_pool, table, _i32(before), _i32([0, 6, 26, 46]), pos, FREQ(d), q=q, q_out=out)
    _check_append(k_pool, v_pool, want)                          # (position 0: not turned)
    assert torch.equal(out[:46], q[:46]) and (out[46:] == 7).all()
    before = [-3, 0, 0]                                          # in front of the cache: dropped, too
    want = _expect(k, v, k_pool, v_pool, table, before, counts)
    sk.snapkv_append_paged(k, v, k_pool, v_pool, table, _i32(before), _i32([0, 6, 26, 46]))
    _check_append(k_pool, v_pool, want)


def test_append_far_positions_keep_their_angle():
    pos = _i32([2 ** 31 - 1, 2 ** 30 + 1, 380000, 0])
    k = _bf16(_gen(5), 4, 1, 128)
    k_pool, v_pool, table = _cache([4], 1, 16, 128, 5)
    want = _expect(k, k, k_pool, v_pool, table, [0], [4], (pos, FREQ(128), False))
    sk.snapkv_append_paged(k, k, k_pool, v_pool, table, _i32([0]), _i32([0, 4]), pos, FREQ(128))
    _check_append(k_pool, v_pool, want)


def test_append_refusals():
    k_pool, v_pool, table = _cache([32, 32], 4, 16, 64, 3)
    g = _gen(4)
    k, v, q = _bf16(g, 6, 2, 64), _bf16(g, 6, 2, 64), _bf16(g, 6, 4, 64)
    lens, cu, f = _i32([0, 0]), _i32([0, 3, 6]), FREQ(64)
    pos = torch.zeros(6, dtype=torch.int32, device="cuda")
    A = sk.snapkv_append_paged
    for bad in [lambda: A(k, v, k_pool, v_pool, table, lens),                      # packed without cu_tokens
                lambda: A(k, v[:5], k_pool, v_pool, table, lens, cu),
                lambda: A(k, v, k_pool, v_pool[:, :2], table, lens, cu),
                lambda: A(k, v, k_pool[:, :3], v_pool[:, :3], table, lens, cu),    # heads do not divide
                lambda: A(k, v, k_pool, v_pool, table, lens, cu[:2]),
                lambda: A(k, v, k_pool, v_pool, table, lens.long(), cu),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos[:5], f),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos.long(), f),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, f.double()),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, FREQ(80)),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, FREQ(24)),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, q=q),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, f, q=q[:5]),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, f, q=q, q_out=q[:, :2]),
                lambda: A(k, v, k_pool, v_pool, table, lens, cu, pos, f, q_out=q),
                lambda: A(k.cpu(), v, k_pool, v_pool, table, lens, cu),
                lambda: A(k, v, k_pool.cpu(), v_pool, table, lens, cu),
                lambda: A(k.float(), v, k_pool, v_pool, table, lens, cu)]:
        with pytest.raises(sk.SnapKVError):
            bad()
