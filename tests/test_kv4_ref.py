"""The numpy restatement of the 4-bit cache that the GPU tests compare with, itself pinned:
scales and codes against rational arithmetic, bytes against a decoder written apart, the
attention against closed forms."""
from fractions import Fraction

import numpy as np

import kv4_ref as ref


def nearest_even(x):
    f = x.numerator // x.denominator
    r = x - f
    return f + (1 if r > Fraction(1, 2) or (r == Fraction(1, 2) and f % 2) else 0)


def test_scales_and_codes_are_the_nearest():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 128)).astype(np.float32) * 2.0 ** rng.integers(-30, 30, (40, 1))
    x[0] = 0
    x[1] = np.tile([7.0, 3.5, 0.5, 1.5, 2.5, -0.5, -6.5, 0.25], 16)       # s = 1: ties
    x[2, :32] = np.float32(7 * (1 + 2.0 ** -8))                           # a scale between two bf16 values
    c, s = ref.quant(x)
    for i in range(x.shape[0]):
        for g in range(4):
            part = [Fraction(float(v)) for v in x[i, 32 * g:32 * g + 32]]
            top = max(abs(v) for v in part) / 7
            if top == 0:
                assert s[i, g] == 0 and not c[i, 32 * g:32 * g + 32].any()
                continue
            e = 0
            while top >= 256 * Fraction(2) ** e:
                e += 1
            while top < 128 * Fraction(2) ** e:
                e -= 1
            sc = nearest_even(top / Fraction(2) ** e) * Fraction(2) ** e
            assert Fraction(float(s[i, g])) == sc
            for d in range(32):
                n = nearest_even(abs(part[d]) / sc)
                assert abs(c[i, 32 * g + d]) == min(n, 7)
                assert c[i, 32 * g + d] * part[d] >= 0


def test_bytes_decode_to_the_values():
    x = np.random.default_rng(1).standard_normal((5, 128))
    for byte, name in ((ref.K_BYTE, "k"), (ref.V_BYTE, "v")):
        codes, scales = ref.rows_bytes(x, byte)
        seen = set()
        out = np.zeros_like(x)
        for d in range(128):
            g, r = divmod(d, 32)
            at = 16 * (r // 8) + 4 * g + (r % 8) // 2 if name == "k" else 8 * (r // 4) + 2 * g + (r % 4) // 2
            seen.add((at, d % 2))
            u = codes[:, at] >> 4 if d % 2 else codes[:, at] & 15
            s = (scales[:, 2 * g:2 * g + 2].copy().view(np.uint16)[:, 0].astype(np.uint32) << 16).view(np.float32)
            out[:, d] = (u.astype(np.int64) - 8) * s.astype(np.float64)
        assert len(seen) == 128
        np.testing.assert_array_equal(out, ref.values(x))


def test_not_finite_groups():
    x = np.ones((1, 128))
    x[0, 40] = np.inf
    v = ref.values(x)
    assert np.isnan(v[0, 32:64]).all() and np.isfinite(v[0, :32]).all() and np.isfinite(v[0, 64:]).all()


def test_attention_closed_forms():
    rng = np.random.default_rng(2)
    ks, vs = [np.zeros((9, 1, 128))], [rng.standard_normal((9, 1, 128))]
    q = rng.standard_normal((1, 4, 2, 128))
    out, bound = ref.attention(q, ks, vs, [4], True, 0.1)       # equal scores: means of what is seen
    v = ref.values(vs[0])[:, 0]
    for t in range(4):
        np.testing.assert_allclose(out[0, t, 1], v[:6 + t].mean(0), atol=1e-12)
    out, _ = ref.attention(q, [k[:2] for k in ks], [x[:2] for x in vs], [4], True, 0.1)
    assert not out[0, :2].any() and np.allclose(out[0, 2, 0], v[0])
