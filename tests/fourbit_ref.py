"""Plain forms of the rotation and of the cache that holds 4.5 bits a value, for their tests: 64-bit torch, and the
quantisation once more in float32 steps, which has to be met bit for bit."""
import math

import torch

import cache_ref

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
# float8 of 4 exponent and 3 mantissa bits: 0 .. 0x7e, then NaN
E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1] + [math.nan]


def table(positions, dim, base=10000.0):
    rate = base ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def turn(x, positions, tab, interleaved):
    """x [rows, heads, d] -> (turned in 64 bits, |x1 cos| + |x2 sin| of each result, which its roundings scale with)."""
    x, tab, dim = x.double(), tab.double(), tab.shape[1]
    y, size = x.clone(), torch.zeros_like(x)
    for i in range(dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
        c, s = tab[positions.long(), i][:, None], tab[positions.long(), dim // 2 + i][:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = (x[..., a] * c).abs() + (x[..., b] * s).abs()
        size[..., b] = (x[..., b] * c).abs() + (x[..., a] * s).abs()
    return y, size


def step(dtype):
    """Half of the distance between two values of a type below its normal range, where it does not shrink with them any more:
    a result there is off by that much.  (float16: values below 2^-14 are multiples of 2^-24, so 2^-25.)"""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def check_turned(got, x, positions, tab, interleaved):
    """Two products and a sum in float32, each off by 2^-24 of at most `size`, and one rounding to the type."""
    y, size = turn(x, positions, tab, interleaved)
    half = torch.finfo(got.dtype).eps / 2
    far = (got.double() - y).abs() > half * y.abs() + 2.0 ** -22 * size + 1e-30 + step(got.dtype)
    assert not bool(far.any()), far.nonzero()[:4].tolist()


def check_attention(got, want, dtype, d, keys, where="", largest=0.0):
    """cache_ref's tolerance, and half of a step below the normal range for the one rounding of the output.  Held values are
    often exactly 0: where the heaviest keys' are, the mean of |v| that the tolerance goes by says nothing of the light ones.
    A weight that falls below float16's normal range is off by at most 2^-31 of the largest (its step there is 2^-24, half of it
    2^-25; the largest weight is 2^7 or more), so the output by at most that for each key, times the `largest` |v|."""
    o, a, s = want
    off = (got.double() - o).abs()
    far = off > cache_ref.tolerance(o, a, s, dtype, d, keys) + step(dtype) + keys * 2.0 ** -31 * largest
    assert not bool(far.any()) and bool(torch.isfinite(got).all()), (where, int(far.sum()), far.nonzero()[:4].tolist(), float(off.max()))


def turn32(x, positions, tab, interleaved):
    """The same in float32, an operation at a time."""
    x, dim = x.float(), tab.shape[1]
    c, s = tab[positions.long()][:, None, : dim // 2], tab[positions.long()][:, None, dim // 2:]
    a, b = (x[..., 0:dim:2], x[..., 1:dim:2]) if interleaved else (x[..., : dim // 2], x[..., dim // 2: dim])
    y1, y2 = a * c - b * s, b * c + a * s
    y = torch.stack([y1, y2], -1).flatten(-2) if interleaved else torch.cat([y1, y2], -1)
    return torch.cat([y, x[..., dim:]], -1)


def quantise32(x, g):
    """float32 [..., d] on the host -> codes [..., d] and scale bytes [..., d / 16], in float32 steps."""
    groups = x.unflatten(-1, (-1, 16))
    g = torch.tensor(g, dtype=torch.float32)
    s8 = (groups.abs().amax(-1) / (g * 6)).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = s8.float()[..., None]
    y = torch.where(s == 0, torch.zeros(()), groups / (s * g))
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for edge, even_above in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += ((a >= edge) if even_above else (a > edge)).to(torch.uint8)
    return (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2), s8.view(torch.uint8)


def write(cache, slot, head, kc, ks, vc, vs):
    """One token's codes and scales of one head (host tensors) into the host's copy of the cache."""
    d = kc.shape[0]
    bs = cache.shape[2] * 16
    page, t = cache[slot // bs, head, slot % bs // 16], slot % 16
    for i in range(d):
        at, up = i // 32 * 256 + t * 16 + i % 32 // 2, i % 2 * 4
        page[at] = (int(page[at]) & ~(15 << up)) | int(kc[i]) << up
        at, up = 9 * d + i * 8 + t // 2, t % 2 * 4
        page[at] = (int(page[at]) & ~(15 << up)) | int(vc[i]) << up
    for j in range(d // 16):
        page[8 * d + t * (d // 16) + j] = ks[j]
        page[17 * d + j * 16 + t] = vs[j]


def read(cache, slots, head, g, values):
    """What the cache holds of `slots` of one head: [n, d] in 64 bits, without the cache's scale rounded in."""
    d, bs = cache.shape[3] // 18, cache.shape[2] * 16
    dev = cache.device
    slots = slots.long().to(dev)
    page, t = cache[slots // bs, head, slots % bs // 16].long(), (slots % 16)[:, None]
    dim = torch.arange(d, device=dev)[None, :]
    if values:
        at, up, sc = 9 * d + dim * 8 + t // 2, t % 2 * 4 + 0 * dim, 17 * d + dim // 16 * 16 + t
    else:
        at, up, sc = dim // 32 * 256 + t * 16 + dim % 32 // 2, dim % 2 * 4 + 0 * t, 8 * d + t * (d // 16) + dim // 16
    code, scale = page.gather(1, at) >> up & 15, page.gather(1, sc)
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device=dev)
    e4m3 = torch.tensor(E4M3, dtype=torch.float64, device=dev)
    x = e2m1[code & 7] * torch.where(code >= 8, -1.0, 1.0).double()
    return x * e4m3[scale & 127] * torch.where(scale >= 128, -1.0, 1.0).double() * g


def check_held(got, x, g):
    """got is what a correct quantisation of x (64 bits, [..., d]) holds: the scale nearest to max / 6 g and values nearest to
    x, or as near as float32's quotients can tell (2^-22 of the value)."""
    got, x = got.double().unflatten(-1, (-1, 16)), x.double().unflatten(-1, (-1, 16))
    grid = torch.tensor(E4M3[:-1], dtype=torch.float64, device=x.device)
    want = x.abs().amax(-1) / (6 * g)
    near = (want[..., None] - grid).abs()
    best = near.amin(-1, keepdim=True)
    allowed = near <= best + 2.0 ** -22 * want[..., None]  # scales that may have been taken
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    fits = torch.zeros(want.shape, dtype=torch.bool, device=x.device)
    for _ in range(2):  # (two neighbours at the most)
        pick = allowed.to(torch.int8).argmax(-1)
        allowed.scatter_(-1, pick[..., None], False)
        s = (grid[pick] * g)[..., None]
        value = (e2m1 * s[..., None] if s.dim() else e2m1 * s)
        off = (x.abs()[..., None] - value).abs().amin(-1)
        mine = (x - got).abs()
        fits |= ((mine <= off + 2.0 ** -22 * x.abs() + 1e-45) & ((got.abs()[..., None] - value).abs().amin(-1) <= 2.0 ** -22 * got.abs())).all(-1)
    assert bool(fits.all()), (~fits).nonzero()[:4].tolist()
