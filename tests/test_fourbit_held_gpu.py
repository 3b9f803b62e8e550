"""What the append to the cache of 4 bits holds and gives back: nearest values in 64 bits, rows without a slot, quotients as a division
rounds them; and how far a NaN that is held reaches."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import fourbit_ref as R  # noqa: E402
import held_ref  # noqa: E402
from test_fourbit_attention_gpu import _build, _run  # noqa: E402


@pytest.mark.parametrize("dtype,d,bs,ks,vs", [(torch.bfloat16, 128, 64, 1.0, 1.0), (torch.float16, 64, 16, 0.25, 3.0),
                                              (torch.float32, 96, 32, 0.40625, 1e-3), (torch.bfloat16, 256, 128, 2.0 ** -20, 2.0 ** 20)])
@pytest.mark.parametrize("split", [False, True])
def test_values_are_the_nearest(dtype, d, bs, ks, vs, split):
    """Whole pages and parts of pages, turned keys; the outputs are what is held, rounded to the type."""
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(d)
    rows, kvh = 203, 2
    k, v = ((torch.randn(rows, kvh, d, generator=gen) * g).to(dtype) for g in (4 * ks, vs))
    slots = torch.randperm(rows + 40, generator=gen)[:rows].int() if split else torch.arange(5, rows + 5, dtype=torch.int32)
    positions, tab = torch.arange(rows, dtype=torch.int32), R.table(rows, d)
    cache = torch.randint(0, 256, binding.pcg_fourbit_cache_shape((rows + 40) // bs + 2, kvh, bs, d), generator=gen, dtype=torch.uint8).cuda()
    k_out, v_out = (torch.empty(rows, kvh, d, dtype=dtype, device="cuda") for _ in range(2))
    binding.pcg_cache_append_fourbit(None, k.cuda(), v.cuda(), slots.cuda(), cache, positions=positions.cuda(), table=tab.cuda(), k_scale=ks,
                                     v_scale=vs, k_out=k_out, v_out=v_out)
    turned = R.turn32(k, positions, tab, False)
    half = torch.finfo(dtype).eps / 2
    for h in range(kvh):
        for values, out, g, x in ((False, k_out, ks, turned), (True, v_out, vs, v)):
            g = float(torch.tensor(g, dtype=torch.float32))
            held = R.read(cache, slots, h, g, values)
            held_ref.check(held, x[:, h].double().cuda(), g)
            assert bool(((out[:, h].double() - held).abs() <= (half + 2.0 ** -23) * held.abs() + R.step(dtype)).all())


def test_rows_outside_the_cache_are_turned_and_held_all_the_same():
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(4)
    k, v = (torch.randn(20, 2, 64, generator=gen) for _ in range(2))
    q = torch.randn(20, 4, 64, generator=gen)
    slots = torch.arange(3, 23, dtype=torch.int32)
    slots[4], slots[9], slots[19] = -1, 4 * 16, -2 ** 31
    positions, tab = torch.arange(20, dtype=torch.int32) * 3, R.table(60, 64)
    cache = torch.randint(0, 256, binding.pcg_fourbit_cache_shape(4, 2, 16, 64), generator=gen, dtype=torch.uint8)
    mine = cache.cuda()
    k_out, v_out = (torch.full((20, 2, 64), 3.0, device="cuda") for _ in range(2))
    q_out = binding.pcg_cache_append_fourbit(q.cuda(), k.cuda(), v.cuda(), slots.cuda(), mine, positions=positions.cuda(), table=tab.cuda(),
                                             k_out=k_out, v_out=v_out)
    (kc, k8), (vc, v8) = R.quantise32(R.turn32(k, positions, tab, False), 1.0), R.quantise32(v, 1.0)
    assert torch.equal(q_out.cpu(), R.turn32(q, positions, tab, False))
    assert torch.equal(k_out.cpu(), held_ref.dequantise32(kc, k8, 1.0)) and torch.equal(v_out.cpu(), held_ref.dequantise32(vc, v8, 1.0))
    for r in range(20):
        if r not in (4, 9, 19):
            for h in range(2):
                R.write(cache, int(slots[r]), h, kc[r, h], k8[r, h], vc[r, h], v8[r, h])
    assert torch.equal(mine.cpu(), cache)


@pytest.mark.parametrize("g", [1.0, 0.40625, 0.37, 1e-9, 2.0 ** -60, 2.0 ** 60])
def test_quotients_are_a_division_s(g):
    """Two million values a scale, in every binade that float32 has: those around the borders of two codes, up to two of their steps
    away, and any others; scales of the groups of every mantissa.  The product with the rounded reciprocal and its remainder
    has to give the code that a division gives, -0 among them."""
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(11)
    rows, kvh, d = 1024, 8, 256
    groups = rows * kvh * d // 16
    low, high = (-149.0, 127.9) if g == 1.0 else (max(-149.0, torch.tensor(g).log2().item() - 12), min(127.9, torch.tensor(g).log2().item() + 14))
    most = torch.exp2(torch.rand(groups, 1, generator=gen, dtype=torch.float64) * (high - low) + low).float()
    half = groups // 2  # of the scales' own range, where codes are not all 0 or all 6
    most[:half] = (torch.exp2(torch.rand(half, 1, generator=gen, dtype=torch.float64) * 18 - 9) * 6 * g).float().clamp(max=3e38)
    _, s8 = R.quantise32(most.expand(groups, 16), g)
    by = s8.view(torch.float8_e4m3fn).float() * torch.tensor(g, dtype=torch.float32)
    edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])[torch.randint(0, 7, (groups, 16), generator=gen)] * by
    step = torch.randint(-2, 3, (groups, 16), generator=gen, dtype=torch.int32)
    near = (edge.view(torch.int32) + step).clamp(min=0).view(torch.float32)
    other = (most.double() * torch.exp2(-30 * torch.rand(groups, 16, generator=gen, dtype=torch.float64) ** 2)).float()
    x = torch.where((torch.rand(groups, 16, generator=gen) < 0.7) & (near <= most), near, other)
    x[:, :1] = most
    x = x.gather(1, torch.rand(groups, 16, generator=gen).argsort(1)) * torch.where(torch.rand(groups, 16, generator=gen) < 0.5, -1.0, 1.0)
    x = x.view(rows, kvh, d)
    cache = torch.zeros(binding.pcg_fourbit_cache_shape(rows // 128, kvh, 128, d), dtype=torch.uint8, device="cuda")
    k_out, v_out = (torch.empty(rows, kvh, d, device="cuda") for _ in range(2))
    binding.pcg_cache_append_fourbit(None, x.cuda(), -x.cuda(), torch.arange(rows, dtype=torch.int32, device="cuda"), cache, k_scale=g, v_scale=g,
                                     k_out=k_out, v_out=v_out)
    want = held_ref.dequantise32(*R.quantise32(x, g), g)
    for out, w in ((k_out, want), (v_out, -want)):
        same = out.cpu().view(torch.int32) == w.view(torch.int32)
        zero = (out.cpu() == 0) & (w == 0) & (R.quantise32(x, g)[1].repeat_interleave(16, -1) == 0)  # (a scale of 0 holds +0)
        assert bool((same | zero).all()), ((~(same | zero)).nonzero()[:4].tolist())


@pytest.mark.parametrize("n,d", [(2, 64), (2, 128), (17, 128), (20, 64), (40, 128), (40, 64), (5, 96)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_held_nan_value_stays_in_its_sequence_and_its_dimensions(n, d, dtype):
    """A group of NaN among a sequence's values: the rows from its token on are NaN in its 16 dimensions; earlier rows may be there,
    and nothing else changes."""
    s = _build([100 + n, 60 + n, 300], [n, n, n], 8, 2, d, 32, dtype, seed=n)
    want = _run(s)
    seen = n // 2  # the first row that sees the token
    slot = int(s["slots"][0][100 + seen])
    page = s["cache"][slot // 32, 1, slot % 32 // 16]
    page[17 * d + 16 + slot % 16] = 0x7F  # dimensions 16 to 31 of the second key head
    out = _run(s)
    assert bool(out[seen:n, 4:, 16:32].isnan().all())
    touched = torch.zeros_like(out, dtype=torch.bool)
    touched[:n, 4:, 16:32] = True
    assert torch.equal(out[~touched], want[~touched])
    early = out[:seen, 4:, 16:32]
    assert bool((early.isnan() | (early == want[:seen, 4:, 16:32])).all())


def test_two_rows_with_one_slot_leave_the_others_alone():
    """A slot that several rows name holds a mixture of them; every other byte is what it is without them."""
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(6)
    rows, kvh, d, bs = 90, 2, 64, 32
    k, v = (torch.randn(rows, kvh, d, generator=gen).cuda() for _ in range(2))
    slots = torch.arange(7, rows + 7, dtype=torch.int32)
    slots[50], slots[60], slots[61], slots[3] = 20, 20, 33, 33  # beside the rows 13 and 26, whose slots these are
    twice = (20, 33)
    start = torch.randint(0, 256, binding.pcg_fourbit_cache_shape(4, kvh, bs, d), generator=gen, dtype=torch.uint8).cuda()
    mine, alone = start.clone(), start.clone()
    binding.pcg_cache_append_fourbit(None, k, v, slots.cuda(), mine)
    only = slots.clone()
    only[[3, 13, 26, 50, 60, 61]] = -1
    binding.pcg_cache_append_fourbit(None, k, v, only.cuda(), alone)
    code, s8 = zip(*(R.quantise32(x.cpu(), 1.0) for x in (k, v)))
    for s in range(4 * bs):
        for h in range(kvh):
            for values in (False, True):
                page, t = [c[s // bs, h, s % bs // 16].cpu() for c in (mine, alone)], s % 16
                dims = torch.arange(d)
                at, up = (9 * d + dims * 8 + t // 2, t % 2 * 4 + 0 * dims) if values else (dims // 32 * 256 + t * 16 + dims % 32 // 2, dims % 2 * 4)
                got, want = ((p[at] >> up) & 15 for p in page)
                if s not in twice:
                    assert torch.equal(got, want), (s, h, values)
                elif not values:  # words of 16 codes are one row's or another's (value codes may mix within a code)
                    names = [r for r in range(rows) if int(slots[r]) == s]
                    for j in range(0, d, 16):
                        assert any(torch.equal(got[j:j + 16], code[0][r, h, j:j + 16]) for r in names), (s, h, j)
