"""What a cache of 4 bits may hold of a value, in 64 bits: fourbit_ref's check, where a turn counts only if a scale is left for it.
(There, a group held as zeros fits always: once no scale is left the turn takes the first one, which is 0.)"""
import torch

import fourbit_ref as R


def fits(got, x, g):
    """Which groups of 16 (..., d / 16) of `got` are what a correct quantisation of x holds: the scale nearest to max / 6 g and
    values nearest to x, or as near as float32's quotients can tell (2^-22 of the value)."""
    got, x = got.double().unflatten(-1, (-1, 16)), x.double().unflatten(-1, (-1, 16))
    grid = torch.tensor(R.E4M3[:-1], dtype=torch.float64, device=x.device)
    e2m1 = torch.tensor(R.E2M1, dtype=torch.float64, device=x.device)
    want = x.abs().amax(-1) / (6 * g)
    near = (want[..., None] - grid).abs()
    allowed = near <= near.amin(-1, keepdim=True) + 2.0 ** -22 * want[..., None]  # one scale, or two neighbours
    ok = torch.zeros(want.shape, dtype=torch.bool, device=x.device)
    for _ in range(2):
        left = allowed.any(-1)
        pick = allowed.to(torch.int8).argmax(-1)
        allowed.scatter_(-1, pick[..., None], False)
        value = e2m1 * (grid[pick] * g)[..., None, None]
        off = (x.abs()[..., None] - value).abs().amin(-1)
        nearest = (x - got).abs() <= off + 2.0 ** -22 * x.abs() + 1e-45
        held = (got.abs()[..., None] - value).abs().amin(-1) <= 2.0 ** -22 * got.abs()
        ok |= left & (nearest & held).all(-1)
    return ok


def check(got, x, g):
    bad = ~fits(got, x, g)
    assert not bool(bad.any()), bad.nonzero()[:4].tolist()


def dequantise32(code, s8, g):
    """What codes [..., d] and scale bytes [..., d / 16] hold, in float32 steps."""
    x = torch.tensor(R.E2M1)[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
    x = x.unflatten(-1, (-1, 16)) * s8.view(torch.float8_e4m3fn).float()[..., None]  # (exact)
    return (x * torch.tensor(g, dtype=torch.float32)).flatten(-2)
