"""Sizes and choices that 32 bits do not hold are refused, not wrapped (no GPU needed)."""
import ctypes

import pytest

import paper_2609_30846_gb300 as ip

FAR = (2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 32 + 16, 2 ** 70, -2 ** 31 - 1, -2 ** 32 + 1)
P = ctypes.c_void_p
FAKE, WS = P(1 << 20), P(1 << 21)


@pytest.mark.parametrize("far", FAR)
def test_python_calls(far):
    for i in range(5):
        args = [1, 1, 8, 8, 64]
        args[i] = far
        with pytest.raises(ip.IpError):
            ip.kv4_attention_workspace_bytes(*args)
    with pytest.raises(ip.IpError):
        ip.kv4_page_bytes(far)
    with pytest.raises(ip.IpError):
        ip.kv4_page_bytes(16, far)


@pytest.mark.parametrize("far", FAR)
def test_entry_points(far):
    lib = ip.load()
    st = (ctypes.c_longlong * 3)(1024, 128, 128)
    calls = (
        (lib.ip_quantize_rows_i8, [FAKE, 2, 4, 100, 112, FAKE, 112, FAKE, None], (1, 3)),
        (lib.ip_linear_scaled_i8, [FAKE, 112, FAKE, FAKE, 112, FAKE, None, 0, 4, 100, 50, FAKE, 50, 2, WS, 256, None],
         (7, 9, 10, 13)),
        (lib.ip_kv4_append, [FAKE, FAKE, 1, st, st, FAKE, None, 2, 3, 8, 128, FAKE, 4, FAKE, 9, 32, WS, 256, None],
         (2, 7, 8, 9, 10, 12, 15)),
        (lib.ip_kv4_read, [FAKE, 9, 32, FAKE, 4, FAKE, None, 2, 3, 8, 128, FAKE, FAKE, 0, WS, 256, None],
         (2, 4, 7, 8, 9, 10, 13)),
        (lib.ip_kv4_attention, [FAKE, 2, st, FAKE, None, 1, 0.1, 2, 3, 8, 2, 128, 64, FAKE, 4, FAKE, 9, 32, FAKE, WS,
                                1 << 24, None], (1, 5, 7, 8, 9, 10, 11, 12, 14, 17)))
    for fn, args, ints in calls:
        for i in ints:
            a = list(args)
            a[i] = far
            if fn in (lib.ip_quantize_rows_i8, lib.ip_linear_scaled_i8):      # rows as long as the size asks
                a = [2 ** 40 - 16 if j in ((4, 6) if fn is lib.ip_quantize_rows_i8 else (1, 4, 12)) else x
                     for j, x in enumerate(a)]
                if fn is lib.ip_linear_scaled_i8:
                    a[12] = 1 << 31
            assert fn(*a) in (-2, -4, -7), (i, far)      # shape, unsupported, parameter: before any launch
