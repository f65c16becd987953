"""The 4-bit rows' reference against what is known of the formats (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")

import fp4_ref as ref


def test_grids():
    assert len(ref.E2M1) == 8 and len(ref.E4M3) == 127 and ref.E4M3[-1] == 448 and ref.E4M3[8] == 2.0 ** -6
    assert list(ref.E4M3) == sorted(set(ref.E4M3))
    b = torch.arange(127, dtype=torch.uint8)
    assert b.view(torch.float8_e4m3fn).double().tolist() == list(ref.E4M3)


def test_nearest_is_even_between_two():
    y = torch.tensor([0.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.0], dtype=torch.float64)
    assert [ref.E2M1[i] for i in ref.nearest(y, ref.E2M1)] == [0, 0, .5, 1, 1, 2, 2, 4, 4, 6, 6]
    x = (torch.rand(4000, generator=torch.Generator().manual_seed(1)) * 500).clamp(max=448)
    got = torch.tensor(ref.E4M3, dtype=torch.float64)[ref.nearest(x.double(), ref.E4M3)]
    assert torch.equal(got, x.to(torch.float8_e4m3fn).double())


def test_bytes_and_values_are_inverse():
    g = torch.Generator().manual_seed(2)
    for M, d in ((1, 1), (3, 17), (130, 100), (33, 64)):
        c, sb, r = ref.quantize(torch.randn(M, d, generator=g) * 3)
        q, blocks = ref.bytes_of(c, sb)
        v = ref.values(q, blocks, r, d)
        s = torch.tensor(ref.E4M3, dtype=torch.float64)[sb.long()].repeat_interleave(16, 1)[:, :d]
        want = torch.tensor(ref.E2M1, dtype=torch.float64)[(c & 7).long()] * torch.where(c > 7, -1.0, 1.0) * s * r[:, None]
        assert torch.equal(v, want)
        assert ref.untouched(blocks, M).sum() == (blocks.shape[0] * 128 - M) * 4 * blocks.shape[1]


def test_error_of_a_value():
    # a code is off by at most a quarter of 6 s r / 3 (the step from 4 to 6 is 2, half of it 1, of 6), the
    # scale rounds by 2^-4 at most
    x = torch.randn(50, 160, generator=torch.Generator().manual_seed(3))
    c, sb, r = ref.quantize(x)
    v = ref.values(*ref.bytes_of(c, sb), r, 160)
    top = x.double().unflatten(1, (-1, 16)).abs().amax(-1).repeat_interleave(16, 1)
    assert ((v - x.double()).abs() <= top / 6 * (1 + 2.0 ** -4) + 1e-12).all()
