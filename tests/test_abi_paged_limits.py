"""Sizes that the paged calls and the prompt attention refuse: offsets and counts that would leave 32 bits."""
import ctypes

from paper_2404_14469_b200 import binding as sk

FAKE = 0x1000
I32, I64 = lambda *x: (ctypes.c_int32 * len(x))(*x), lambda *x: (ctypes.c_int64 * len(x))(*x)


def test_tables_of_more_rows_than_an_int_counts():
    L, st, pool = sk.lib(), I64(8, 512, 128), I64(4 * 64 * 128, 64 * 128, 128)
    append = lambda pps, page: L.snapkv_append_paged(FAKE, FAKE, st, st, FAKE, FAKE, None, None, 0, 0, None, None, None, FAKE,
                                                     FAKE, pool, pool, FAKE, pps, page, 9, 2, 0, 8, 4, 4, 128, None)
    assert append(1 << 20, 1 << 10) == 0 and append(1 << 20, 1 << 11) == 2 and append(1 << 30, 2) == 2


def test_prompts_beyond_the_last_token():
    L = sk.lib()
    call = lambda ql, q0=None, k0=None, out=FAKE: L.snapkv_prefill_attention(
        FAKE, FAKE, FAKE, None, None, None, ql, None, q0, k0, 1, 4, 2, 128, 0, out, None, None, None)
    assert call(I32(5), I64((1 << 30) - 4)) == 1 and call(I32(5), I64(0), I64(1 << 30)) == 1
    assert call(I32((1 << 30) + 1)) == 1
    assert call(I32(5), out=FAKE + 16) == 1          # the output is written 32 bytes at a time
    assert call(I32(0), I64(1 << 30)) == 0
