"""The self-tests of the prompt attention's and the paged decode's time-outs take and refuse what the calls do."""
import ctypes

import pytest

from paper_2404_14469_b200 import binding as sk
from paper_2404_14469_b200 import build as sk_build

FAKE = 0x1000
INV, UNS, WSP = 1, 2, 3
I32, I64 = lambda *x: (ctypes.c_int32 * len(x))(*x), lambda *x: (ctypes.c_int64 * len(x))(*x)


@pytest.fixture(scope="module")
def L():
    sk_build.build()
    return sk.lib()


def test_lost_keys(L):
    def call(unit=0, q=FAKE, B=2, Hq=4, d=128, ql=I32(5, 7)):
        return L.snapkv_selftest_lost_keys(q, FAKE, FAKE, None, None, None, ql, None, None, None, B, Hq, 2, d, 0, FAKE, None,
                                           None, unit, None)
    assert [call(unit=-1), call(q=None), call(B=0), call(Hq=5), call(d=96)] == [INV, INV, INV, INV, UNS]
    assert call(ql=I32(0, 0)) == 0


@pytest.mark.parametrize("name", ["snapkv_selftest_late_partials", "snapkv_selftest_lost_rows"])
def test_paged(L, name):
    pool = I64(4 * 64 * 128, 64 * 128, 128)

    def call(q=FAKE, page=64, B=2, Hq=8, Hc=4, d=128, ws=FAKE, bytes_=1 << 30):
        return getattr(L, name)(q, FAKE, FAKE, pool, pool, FAKE, 4, page, 9, FAKE, B, Hq, Hc, d, FAKE, None, ws, bytes_, None)
    assert [call(q=None), call(page=40), call(B=0), call(Hc=3), call(d=96)] == [INV, INV, INV, INV, UNS]
    assert [call(ws=None), call(ws=FAKE + 64), call(bytes_=4096)] == [WSP] * 3
