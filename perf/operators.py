"""Cases for the operators around the compression step: the prompt's attention before it, and the
paged cache that generated tokens are appended to and attend to after it.

listed()   the cases; draw(rng): one more of the same ranges
prepare    inputs of a case from a seed, on the GPU
run        one pass: the library's calls with `own`, else the same in elementary torch operations
work       bytes and operations that a pass cannot do without
exact      the same outputs from the definitions, in 64 bits
"""
from __future__ import annotations

import math
import random

import torch

own = False

MHA, GQA, TINY = (32, 32, 128), (32, 8, 128), (4, 4, 64)
ROPE_BASE = 1000000.0


# ------------------------------------------------------------------------------------------ cases
def _prefill(name, B, heads, Lmin, Lmax, context=0, window=0):
    Hq, Hkv, d = heads
    return {"name": name, "kind": "prefill", "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "Lmin": Lmin, "Lmax": Lmax,
            "context": context, "window": window}


def _decode(name, B, heads, Lmin, Lmax, page):
    Hq, Hc, d = heads
    return {"name": name, "kind": "decode", "B": B, "Hq": Hq, "Hc": Hc, "d": d, "Lmin": Lmin, "Lmax": Lmax,
            "page": page}


def _append(name, B, heads, Hc, Lmin, Lmax, page, rotate, rot=128, interleaved=False, behind=0):
    Hq, Hkv, d = heads
    return {"name": name, "kind": "append", "B": B, "Hq": Hq, "Hkv": Hkv, "Hc": Hc, "d": d, "Lmin": Lmin,
            "Lmax": Lmax, "page": page, "rotate": rotate, "rot": rot, "interleaved": interleaved, "behind": behind}


def listed():
    return [
        # the smallest configuration: one prompt of a toy model, launch latency
        _prefill("prefill-tiny-1k", 1, TINY, 1024, 1024, 0, 32),
        # a serving batch: eight prompts of 200 to 4000 tokens, packed
        _prefill("prefill-mixed-8", 8, GQA, 200, 4000, 0, 32),
        # a chunk of a long prompt against the keys that the chunks before it left
        _prefill("prefill-chunk-2k-of-32k", 1, GQA, 2048, 2048, 30720, 32),
        # a 7B MHA model's prompt of 16K tokens
        _prefill("prefill-mha-16k", 1, MHA, 16384, 16384, 0, 32),
        # the largest: one 32K prompt with grouped heads
        _prefill("prefill-gqa-32k", 1, GQA, 32768, 32768, 0, 32),
        # one chat turn, a short cache: latency
        _decode("decode-one-777", 1, GQA, 777, 777, 64),
        # a serving batch of very different lengths
        _decode("decode-ragged-64", 64, GQA, 30, 8000, 64),
        # the compressed caches of sixteen sequences, one selection per query head, with some
        # generated tokens behind the 4096 kept rows
        _decode("decode-expanded-16", 16, MHA, 4100, 4400, 128),
        # one long prompt that was not compressed
        _decode("decode-one-128k", 1, GQA, 131071, 131071, 256),
        # a generation step of 64 sequences: rotate the queries and keys, one row per sequence
        _append("append-step-64", 64, GQA, 8, 1, 1, 64, True, behind=4000),
        # the prompts of a serving batch into the cache
        _append("append-prompts-8", 8, GQA, 8, 1000, 8000, 128, True),
        # the compressed caches of four sequences (one selection per query head) into pages
        _append("append-import-4", 4, MHA, 32, 4096, 4096, 128, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(("prefill", "decode", "append"))
    d = rng.choice((64, 128, 128))
    Hkv = rng.choice((1, 2, 4, 8, 8))
    Hq = Hkv * rng.choice((1, 2, 3, 4, 8))
    if kind == "prefill":
        B = rng.choice((1, 1, 2, 5, 11))
        while True:
            Lmax = _log_int(rng, 20, 24000)
            context = rng.choice((0, 0, _log_int(rng, 1, 20000)))
            if B * Hq * Lmax * (Lmax + 2 * context) < 32 * 1.6e8 and B * (Lmax + context) < 60000:
                break
        Lmin = min(Lmax, _log_int(rng, 1, Lmax))
        return {"kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "Lmin": Lmin, "Lmax": Lmax, "context": context,
                "window": rng.choice((0, min(Lmin, 32)))}
    if kind == "decode":
        Hc = rng.choice((Hkv, Hkv, Hq))
        while True:
            B, Lmax = _log_int(rng, 1, 100), _log_int(rng, 5, 120000)
            if B * Lmax * Hc < 4.0e6:
                break
        return {"kind": kind, "B": B, "Hq": Hq, "Hc": Hc, "d": d, "Lmin": _log_int(rng, 1, Lmax), "Lmax": Lmax,
                "page": rng.choice((16, 32, 64, 128, 256))}
    rotate = rng.random() < 0.75
    Hc = rng.choice((Hkv, Hkv, Hq))
    B = _log_int(rng, 1, 64)
    while True:
        Lmax = rng.choice((1, _log_int(rng, 1, 10000)))
        if B * Lmax * (Hc + Hq) < 2.0e6:
            break
    return {"kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "Hc": Hc, "d": d, "Lmin": _log_int(rng, 1, Lmax), "Lmax": Lmax,
            "page": rng.choice((16, 64, 128, 256)), "rotate": rotate, "rot": rng.choice((d, d, d // 2)),
            "interleaved": rng.random() < 0.3, "behind": rng.choice((0, _log_int(rng, 1, 4000)))}


def _lens(case):
    """The batch's lengths, spread over the logarithm between Lmin and Lmax (both occur)."""
    B, lo, hi = case["B"], case["Lmin"], case["Lmax"]
    rng = random.Random("%d-%d-%d" % (B, lo, hi))
    lens = [hi, lo][:B] + [_log_int(rng, lo, hi) for _ in range(B - 2)]
    rng.shuffle(lens)
    return lens


# ----------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _starts(lens):
    at, out = 0, []
    for n in lens:
        out.append(at)
        at += n
    return out


def _pages(case, lens, seed):
    """A page table with the pages of all sequences in random order, and how many pages the pool has."""
    page = case["page"]
    per_seq = max(-(-max(lens) // page), 1)
    total = sum(-(-n // page) for n in lens)
    order = list(range(total + 3))
    random.Random(seed).shuffle(order)
    table = [[0] * per_seq for _ in lens]
    at = 0
    for row, n in zip(table, lens):
        need = -(-n // page)
        row[:need] = order[at:at + need]
        at += need
    return torch.tensor(table, dtype=torch.int32, device="cuda"), total + 3


def prepare(case, seed):
    g, kind, d, lens = _gen(seed), case["kind"], case["d"], _lens(case)
    s = {"case": case, "lens": lens}
    if kind == "prefill":
        Hq, Hkv, context = case["Hq"], case["Hkv"], case["context"]
        T = sum(lens)
        # queries and keys share a direction per KV head, as the heads of trained models do
        u = torch.randn(Hkv, d, generator=g, device="cuda")
        u = u / u.norm(dim=-1, keepdim=True)
        uq = u.repeat_interleave(Hq // Hkv, 0)
        if context == 0:  # slices of one fused projection's output
            qkv = _normal(g, T, Hq + 2 * Hkv, d)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            q = _normal(g, T, Hq, d)
            k, v = _normal(g, T + context * len(lens), Hkv, d), _normal(g, T + context * len(lens), Hkv, d)
        q.mul_(2).add_((4 * uq).to(torch.bfloat16))
        k[::97].add_((3 * u).to(torch.bfloat16))
        s.update(q=q, k=k, v=v, k_lens=[n + context for n in lens])
    elif kind == "decode":
        B, Hq, Hc = case["B"], case["Hq"], case["Hc"]
        s["table"], pages = _pages(case, lens, seed)
        s["k_pool"], s["v_pool"] = _normal(g, pages, Hc, case["page"], d), _normal(g, pages, Hc, case["page"], d)
        s["q"] = _normal(g, B, Hq, d) * 2
        s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["workspace"] = None
    else:
        B, Hq, Hkv, Hc, behind = case["B"], case["Hq"], case["Hkv"], case["Hc"], case["behind"]
        s["table"], pages = _pages(case, [n + behind for n in lens], seed)
        s["k_pool"], s["v_pool"] = _normal(g, pages, Hc, case["page"], d), _normal(g, pages, Hc, case["page"], d)
        s["cache_lens"] = torch.full((B,), behind, dtype=torch.int32, device="cuda")
        if not case["rotate"] and len(set(lens)) == 1:  # dense caches [B, H, rows, d], as the compression leaves them
            s["k"], s["v"] = (_normal(g, B, Hkv, lens[0], d).transpose(1, 2) for _ in "kv")
            s["cu"] = None
        else:
            T = sum(lens)
            qkv = _normal(g, T, Hq + 2 * Hkv, d)
            s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            s["cu"] = torch.tensor(_starts(lens) + [T], dtype=torch.int32, device="cuda")
        s["positions"] = s["inv_freq"] = None
        if case["rotate"]:
            # the tokens' positions in the text: cache rows that compression dropped count on
            at = random.Random(seed)
            first = [behind + at.randrange(1, 100000) if behind else 0 for _ in lens]
            s["positions"] = torch.cat([torch.arange(p, p + n) for p, n in zip(first, lens)]).to(torch.int32).cuda()
            r = torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"]
            s["inv_freq"] = (ROPE_BASE ** -r).float().cuda()
    return s


# ------------------------------------------------------------------------- the operators, plainly
def _attend(q, k, v, n_before, real):
    """q [n, Hq, d]; k, v [m, Hkv, d]; query i sees keys j <= n_before + i.  (out, lse), in `real`."""
    n, Hq, d = q.shape
    m, Hkv, _ = k.shape
    g = Hq // Hkv
    kr, vr = k.to(real).permute(1, 2, 0), v.to(real).permute(1, 0, 2)  # [Hkv, d, m], [Hkv, m, d]
    outs, lses = [], []
    step = max(1, int(1.0e9 // (Hq * max(m, 1))))  # query rows at a time: the logits stay within a few GB
    for i in range(0, n, step):
        c = min(step, n - i)
        see = max(min(m, n_before + i + c), 0)
        rows = q[i:i + c].to(real).reshape(c, Hkv, g, d).permute(1, 2, 0, 3).reshape(Hkv, g * c, d)
        x = (rows @ kr[:, :, :see]) * (1.0 / math.sqrt(d))
        hidden = torch.arange(see, device=q.device)[None] > torch.arange(i, i + c, device=q.device)[:, None] + n_before
        x = x.view(Hkv, g, c, see).masked_fill_(hidden, -math.inf).view(Hkv, g * c, see)
        top = x.amax(-1, keepdim=True) if see else torch.full((Hkv, g * c, 1), -math.inf, device=q.device, dtype=real)
        x = x.sub_(top.clamp(min=-1e30)).exp_()
        total = x.sum(-1, keepdim=True)
        o = (x @ vr[:, :see]) / total.clamp(min=1e-300 if real == torch.float64 else 1e-38)
        outs.append(o.view(Hkv, g, c, d).permute(2, 0, 1, 3).reshape(c, Hq, d))
        lses.append((top + total.log()).view(Hkv, g, c).permute(2, 0, 1).reshape(c, Hq))
    return torch.cat(outs), torch.cat(lses)


def _prefill_plain(s, real):
    W, outs, lses, seen = s["case"]["window"], [], [], []
    for q0, n, k0, m in zip(_starts(s["lens"]), s["lens"], _starts(s["k_lens"]), s["k_lens"]):
        o, e = _attend(s["q"][q0:q0 + n], s["k"][k0:k0 + m], s["v"][k0:k0 + m], m - n, real)
        outs.append(o)
        lses.append(e)
        if W:
            seen.append(e[n - W:].t())
    got = [torch.cat(outs), torch.cat(lses)]
    return got + ([torch.stack(seen)] if W else [])


def _decode_plain(s):
    q, table, lens = s["q"], s["table"].long(), s["seq_lens"]
    B, Hq, d = q.shape
    Hc, page = s["k_pool"].shape[1:3]
    most = table.shape[1] * page
    k = s["k_pool"][table].float().permute(0, 2, 1, 3, 4).reshape(B, Hc, most, d)
    x = (q.float().view(B, Hc, Hq // Hc, d) @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    del k
    hidden = torch.arange(most, device=q.device)[None, :] >= lens[:, None]
    x = x.masked_fill(hidden[:, None, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - top.clamp(min=-1e30)).exp()
    total = p.sum(-1, keepdim=True)
    v = s["v_pool"][table].float().permute(0, 2, 1, 3, 4).reshape(B, Hc, most, d)
    v = v.masked_fill(hidden[:, None, :, None], 0)
    out = (p @ v) / total.clamp(min=1e-38)
    return [out.view(B, Hq, d), (top + total.log()).view(B, Hq)]


def _rotated(x, positions, inv_freq, interleaved, real):
    """x [T, H, d] turned by its positions; angles in 64 bits."""
    half = inv_freq.numel()
    angle = positions.double()[:, None] * inv_freq.double()
    c, sn = angle.cos().to(real)[:, None], angle.sin().to(real)[:, None]
    x = x.to(real)
    turn, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if interleaved else (turn[..., :half], turn[..., half:])
    y = (a * c - b * sn, a * sn + b * c)
    y = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat((y, rest), -1)


def _append_plain(s, real):
    """The rows, the page and the row in it of every token, and the turned queries."""
    k, v, cu = s["k"], s["v"], s["cu"]
    if cu is None:
        B, n = k.shape[:2]
        k, v = k.reshape(B * n, *k.shape[2:]), v.reshape(B * n, *v.shape[2:])
        cu = torch.arange(B + 1, device=k.device, dtype=torch.int32) * n
    T = k.shape[0]
    t = torch.arange(T, device=k.device)
    b = torch.searchsorted(cu[1:].long(), t, right=True)
    slot = s["cache_lens"][b].long() + t - cu[b].long()
    Hc, page = s["k_pool"].shape[1:3]
    where = (s["table"][b, slot // page].long(), slot % page)
    q = None
    if s["inv_freq"] is not None:
        turn = (s["positions"], s["inv_freq"], s["case"]["interleaved"], real)
        k, q = _rotated(k, *turn), _rotated(s["q"], *turn)
    reps = Hc // k.shape[1]
    return k.repeat_interleave(reps, 1), v.repeat_interleave(reps, 1), where, q


# -------------------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2404_14469_b200 import binding as sk
        if kind == "prefill":
            out, lse, lse_obs = sk.snapkv_prefill_attention(s["q"], s["k"], s["v"], s["lens"], s["k_lens"],
                                                            window=s["case"]["window"])
            return [out, lse] + ([lse_obs] if lse_obs is not None else [])
        if kind == "decode":
            out, lse, s["workspace"] = sk.snapkv_decode_paged(s["q"], s["k_pool"], s["v_pool"], s["table"],
                                                              s["seq_lens"], s["workspace"])
            return [out, lse]
        q = sk.snapkv_append_paged(s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["cache_lens"], s["cu"],
                                   s["positions"], s["inv_freq"], s["case"]["interleaved"],
                                   s["q"] if s["inv_freq"] is not None else None)
        return [s["k_pool"], s["v_pool"]] + ([q] if q is not None else [])
    if kind == "prefill":
        out, *lse = _prefill_plain(s, torch.float32)
        return [out.to(torch.bfloat16)] + lse
    if kind == "decode":
        return _decode_plain(s)
    k, v, (pages, rows), q = _append_plain(s, torch.float32)
    s["k_pool"][pages, :, rows] = k.to(torch.bfloat16)
    s["v_pool"][pages, :, rows] = v.to(torch.bfloat16)
    return [s["k_pool"], s["v_pool"]] + ([q.to(torch.bfloat16)] if q is not None else [])


def work(case):
    kind, d, lens = case["kind"], case["d"], _lens(case)
    if kind == "prefill":
        T, c = sum(lens), case["context"]
        pairs = sum(n * c + n * (n + 1) // 2 for n in lens)
        rows = 2 * T * case["Hq"] + 2 * (T + c * len(lens)) * case["Hkv"]
        return {"bytes": 2 * d * rows + 4 * case["Hq"] * (T + case["window"] * len(lens)),
                "flops": 4 * d * case["Hq"] * pairs}
    if kind == "decode":
        pages = sum(-(-n // case["page"]) for n in lens)
        return {"bytes": 4 * d * case["Hc"] * sum(lens) + case["B"] * case["Hq"] * (6 * d + 4) + 4 * (pages + case["B"]),
                "flops": 4 * d * case["Hq"] * sum(lens)}
    T = sum(lens)
    rows = 2 * case["Hkv"] + 2 * case["Hc"] + (2 * case["Hq"] if case["rotate"] else 0)
    turned = (case["Hkv"] + case["Hq"]) * case["rot"] * 3 if case["rotate"] else 0
    return {"bytes": T * (2 * d * rows + (4 if case["rotate"] else 0)), "flops": T * turned}


# ------------------------------------------------------------------------------- in 64 bits, apart
def exact(case, seed):
    s = prepare(case, seed)
    kind, d = case["kind"], case["d"]
    if kind == "prefill":
        g, W = case["Hq"] // case["Hkv"], case["window"]
        outs, lses = [], []
        at = after = 0
        for n, m in zip(s["lens"], s["k_lens"]):
            o = torch.empty(n, case["Hq"], d, dtype=torch.float64, device="cuda")
            e = torch.empty(n, case["Hq"], dtype=torch.float64, device="cuda")
            for h in range(case["Hq"]):
                kh = s["k"][after:after + m, h // g].double()
                vh = s["v"][after:after + m, h // g].double()
                for i in range(0, n, 4096):
                    qi = s["q"][at + i:at + min(i + 4096, n), h].double()
                    last = m - n + i + torch.arange(len(qi), device="cuda")
                    z = torch.einsum("id,jd->ij", qi, kh) / d ** 0.5
                    z = torch.where(torch.arange(m, device="cuda")[None] <= last[:, None], z, -torch.inf)
                    e[i:i + len(qi), h] = torch.logsumexp(z, -1)
                    o[i:i + len(qi), h] = torch.softmax(z, -1) @ vh
            outs.append(o)
            lses.append(e)
            at, after = at + n, after + m
        got = [torch.cat(outs), torch.cat(lses)]
        return got + ([torch.stack([e[-W:].t() for e in lses])] if W else [])
    if kind == "decode":
        g, page = case["Hq"] // case["Hc"], case["page"]
        out = torch.empty(case["B"], case["Hq"], d, dtype=torch.float64, device="cuda")
        lse = torch.empty(case["B"], case["Hq"], dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["lens"]):
            ids = s["table"][b, :-(-n // page)].long()
            k = s["k_pool"][ids].double().transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(g, 0)
            v = s["v_pool"][ids].double().transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(g, 0)
            z = torch.einsum("hd,hjd->hj", s["q"][b].double(), k) / d ** 0.5
            lse[b] = torch.logsumexp(z, -1)
            out[b] = torch.einsum("hj,hjd->hd", torch.softmax(z, -1), v)
        return [out, lse]
    # a token at a time would take minutes: by sequence, the rows of each written one behind the other
    kp, vp = s["k_pool"].double(), s["v_pool"].double()
    k, v = s["k"].double(), s["v"].double()
    if s["cu"] is None:
        k, v = k.flatten(0, 1), v.flatten(0, 1)
    q = s["q"].double() if case["rotate"] else None
    if case["rotate"]:
        z = torch.exp(1j * s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]  # unit numbers
        r = case["rot"]

        def turned(x):
            x = x.clone()
            if case["interleaved"]:
                w = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * z
                x[..., 0:r:2], x[..., 1:r:2] = w.real, w.imag
            else:
                w = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * z
                x[..., :r // 2], x[..., r // 2:r] = w.real, w.imag
            return x
        k, q = turned(k), turned(q)
    reps, at = case["Hc"] // case["Hkv"], 0
    for b, n in enumerate(s["lens"]):
        slots = case["behind"] + torch.arange(n, device="cuda")
        ids = s["table"][b].long()[slots // case["page"]]
        kp[ids, :, slots % case["page"]] = k[at:at + n].repeat_interleave(reps, 1)
        vp[ids, :, slots % case["page"]] = v[at:at + n].repeat_interleave(reps, 1)
        at += n
    return [kp, vp] + ([q] if q is not None else [])
