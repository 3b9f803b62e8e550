"""The check of what a cache of 4 bits holds lets the float32 steps through and nothing else (no GPU is needed)."""
import pytest

torch = pytest.importorskip("torch")

import fourbit_ref as R  # noqa: E402
import held_ref  # noqa: E402


def _made(g, seed=0):
    x = torch.randn(40, 3, 64, generator=torch.Generator().manual_seed(seed)) * g
    code, s8 = R.quantise32(x, g)
    return x, code, s8


@pytest.mark.parametrize("g", [1.0, 0.37, 2.0 ** 30, 1e-9])
def test_the_float32_steps_pass(g):
    x, code, s8 = _made(g)
    held_ref.check(held_ref.dequantise32(code, s8, g), x, float(torch.tensor(g, dtype=torch.float32)))


def test_zeros_pass_only_where_they_are_right():
    x, _, _ = _made(1.0)
    assert not bool(held_ref.fits(torch.zeros_like(x), x, 1.0).any())
    small = x * 2.0 ** -14  # below half of the least scale
    assert bool(held_ref.fits(torch.zeros_like(x), small, 1.0).all())


@pytest.mark.parametrize("by", [2.0, 0.5, -1.0])
def test_a_wrong_scale_or_sign_fails(by):
    x, code, s8 = _made(1.0)
    assert not bool(held_ref.fits(held_ref.dequantise32(code, s8, 1.0) * by, x, 1.0).any())


def test_one_scale_beside_the_right_one_fails():
    """All 16 requantised with the next larger scale."""
    x, _, s8 = _made(1.0)
    s = (s8 + 1).view(torch.float8_e4m3fn).float()[..., None]
    e2m1 = torch.tensor(R.E2M1)
    y = (x.unflatten(-1, (-1, 16)) / s)
    got = (e2m1[(y.abs()[..., None] - e2m1).abs().argmin(-1)] * y.sign() * s).flatten(-2)
    assert not bool(held_ref.fits(got, x, 1.0).any())


def test_one_code_beside_the_right_one_fails():
    x, code, s8 = _made(1.0)
    other = code.clone()
    other[..., 5::16] = code[..., 5::16] ^ 1
    got = held_ref.fits(held_ref.dequantise32(other, s8, 1.0), x, 1.0)
    assert not bool(got.any())
