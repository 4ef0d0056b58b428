"""Refusals of the prompt attention and the paged-cache calls: all on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2404_14469_b200 import binding as sk
from paper_2404_14469_b200 import build as sk_build

FAKE = 0x1000  # aligned, never dereferenced
OK, INV, UNS, WSP = 0, 1, 2, 3
I32, I64 = lambda *x: (ctypes.c_int32 * len(x))(*x), lambda *x: (ctypes.c_int64 * len(x))(*x)


@pytest.fixture(scope="module")
def L():
    sk_build.build()
    return sk.lib()


def test_prefill_attention_rejects_bad_arguments(L):
    def call(q=FAKE, k=FAKE, v=FAKE, qs=None, ks=None, vs=None, ql=I32(5, 7), kl=None, q0=None, k0=None, B=2, Hq=4,
             Hkv=2, d=128, W=0, out=FAKE, lse=None, obs=None):
        return L.snapkv_prefill_attention(q, k, v, qs, ks, vs, ql, kl, q0, k0, B, Hq, Hkv, d, W, out, lse, obs, None)

    for bad in [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(ql=None), dict(B=0), dict(Hq=5),
                dict(Hkv=0), dict(d=0), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(lse=FAKE + 2), dict(W=-1),
                dict(W=4), dict(obs=FAKE), dict(W=6, obs=FAKE),               # a window longer than a sequence
                dict(ql=I32(5, -1)), dict(kl=I32(5, -1)),
                dict(q0=I64(0, 4)), dict(q0=I64(-1, 9)), dict(q0=I64(7, 0)),  # overlap, negative, descending
                dict(k0=I64(0, -1)), dict(k0=I64(0, 1 << 32)),
                dict(qs=I64(4 * 128, 100)), dict(ks=I64(2 * 128 + 4, 128)), dict(vs=I64(64, 128)),
                dict(qs=I64(1 << 39, 128)), dict(ks=I64(-256, 128))]:
        assert call(**bad) == INV, bad
    for bad in [dict(d=96), dict(d=256), dict(W=129, ql=I32(200, 200), obs=FAKE)]:
        assert call(**bad) == UNS, bad
    assert call(ql=I32(0, 0)) == OK  # nothing to do: nothing is launched


def test_append_paged_rejects_bad_arguments(L):
    st, pool = I64(8, 4 * 128, 128), I64(4 * 64 * 128, 64 * 128, 128)

    def call(k=FAKE, v=FAKE, ks=st, vs=st, cu=FAKE, lens=FAKE, pos=FAKE, freq=FAKE, rot=128, inter=0, q=FAKE, qs=st,
             qo=FAKE, kp=FAKE, vp=FAKE, kps=pool, vps=pool, table=FAKE, pps=4, page=64, pages=9, B=2, T=7, Hq=8, Hkv=4,
             Hc=4, d=128):
        return L.snapkv_append_paged(k, v, ks, vs, cu, lens, pos, freq, rot, inter, q, qs, qo, kp, vp, kps, vps, table,
                                     pps, page, pages, B, T, Hq, Hkv, Hc, d, None)

    for bad in [dict(k=None), dict(v=None), dict(lens=None), dict(kp=None), dict(vp=None), dict(table=None),
                dict(freq=None), dict(qo=None), dict(qs=None), dict(ks=None), dict(vps=None), dict(B=0), dict(T=-1),
                dict(Hkv=0), dict(Hc=6), dict(Hc=2), dict(pps=0), dict(page=0), dict(pages=0), dict(cu=None),
                dict(rot=7), dict(rot=0), dict(rot=130), dict(k=FAKE + 2), dict(q=FAKE + 8), dict(kp=FAKE + 8),
                dict(cu=FAKE + 1), dict(freq=FAKE + 2), dict(ks=I64(8, 500, 128)), dict(vs=I64(8, 64, 128)),
                dict(qs=I64(8, 1024, 64)), dict(kps=I64(1024, 100, 128)), dict(vps=I64(1024, 128, 64)), dict(Hq=0)]:
        assert call(**bad) == INV, bad
    for bad in [dict(d=96), dict(rot=24)]:
        assert call(**bad) == UNS, bad
    assert call(T=0) == OK and call(T=0, cu=None) == OK


def test_decode_paged_rejects_bad_arguments(L):
    st = I64(4 * 64 * 128, 64 * 128, 128)

    def call(q=FAKE, k=FAKE, v=FAKE, ks=st, vs=st, table=FAKE, pps=4, page=64, pages=9, lens=FAKE, B=2, Hq=8, Hc=4, d=128,
             out=FAKE, lse=None, ws=FAKE, wsb=1 << 30):
        return L.snapkv_decode_paged(q, k, v, ks, vs, table, pps, page, pages, lens, B, Hq, Hc, d, out, lse, ws, wsb, None)

    for bad in [dict(q=None), dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(out=None), dict(ks=None),
                dict(B=0), dict(Hq=6), dict(Hc=0), dict(pps=0), dict(page=0), dict(page=24), dict(pages=0),
                dict(q=FAKE + 2), dict(k=FAKE + 8), dict(out=FAKE + 2), dict(lse=FAKE + 1), dict(lens=FAKE + 2),
                dict(ks=I64(1024, 100, 128)), dict(vs=I64(1024, 1024, 64)), dict(vs=I64(0, 1024, 128))]:
        assert call(**bad) == INV, bad
    for bad in [dict(d=96), dict(B=9000), dict(pps=1 << 28)]:
        assert call(**bad) == UNS, bad
    for bad in [dict(ws=None), dict(ws=FAKE + 16), dict(wsb=16)]:
        assert call(**bad) == WSP, bad
    assert sk.lib().snapkv_decode_paged_workspace_size(2, 8, 4, 128) > 0
    for bad in [(0, 8, 4, 128), (2, 6, 4, 128), (2, 8, 4, 96), (2, 8, 0, 128)]:
        assert sk.lib().snapkv_decode_paged_workspace_size(*bad) == 0


def test_the_binding_refuses_what_is_not_on_the_gpu(L):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pool, i = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(sk.SnapKVError):
        sk.snapkv_prefill_attention(x, x, x, [4])
    with pytest.raises(sk.SnapKVError):
        sk.snapkv_append_paged(x, x, pool, pool, i[None], i[:1], i)
    with pytest.raises(sk.SnapKVError):
        sk.snapkv_decode_paged(x, pool, pool, i[None], i)
