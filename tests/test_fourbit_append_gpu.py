"""The append to the cache of 4 bits: bit for bit against float32 steps, and against what a correct quantisation may hold;
orders of slots, parts of pages, neighbours, special values."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import fourbit_ref as R  # noqa: E402


def _slots(kind, rows, bs, gen):
    """(slots, n_blocks)"""
    n_blocks = rows // bs + 4
    total = n_blocks * bs
    if kind == "shuffled":  # rows of one page anywhere
        return torch.randperm(total, generator=gen)[:rows].to(torch.int32), n_blocks
    at = torch.arange(rows)
    if kind == "reversed":
        return (rows + 5 - at).to(torch.int32), n_blocks
    if kind == "chunks":  # sequences of 1 to 19 rows, each somewhere
        got, used = [], 3
        order = torch.randperm(n_blocks * 8, generator=gen).tolist()
        n_blocks = n_blocks * 8
        while len(got) < rows:
            n = min(int(torch.randint(1, 20, (1,), generator=gen)), rows - len(got))
            start = int(torch.randint(0, 16, (1,), generator=gen))
            block = [order.pop() for _ in range((start + n + bs - 1) // bs)]
            got += [block[(start + i) // bs] * bs + (start + i) % bs for i in range(n)]
        return torch.tensor(got, dtype=torch.int32), n_blocks
    return (at + {"whole": 16, "odd": 7}[kind]).to(torch.int32), n_blocks


CASES = [
    # (rows, q_heads, kv_heads, d, dim, interleaved, block_size, dtype, slots, k_scale, v_scale)
    (1, 4, 2, 64, 64, 0, 16, torch.bfloat16, "odd", 1.0, 1.0),
    (16, 4, 2, 64, 64, 1, 16, torch.float16, "whole", 0.25, 3.0),
    (50, 8, 2, 128, 128, 0, 32, torch.bfloat16, "odd", 1.0, 1.0),
    (70, 8, 2, 128, 64, 0, 64, torch.bfloat16, "chunks", 0.37, 1.0),
    (45, 3, 3, 96, 96, 1, 16, torch.float32, "shuffled", 1.0, 1.0),
    (33, 2, 1, 256, 128, 0, 128, torch.float16, "reversed", 1.0, 2.0 ** -20),
    (40, 1, 1, 32, 32, 0, 256, torch.float32, "chunks", 2.0 ** 30, 1e-9),
    (64, 0, 4, 160, 0, 0, 16, torch.bfloat16, "whole", 1.0, 1.0),
    (21, 0, 2, 64, 0, 0, 16, torch.float32, "shuffled", 0.1, 10.0),
]


def _call(k, v, slots, cache, q=None, positions=None, tab=None, inter=False, ks=1.0, vs=1.0, held=True, **kw):
    from paper_2511_13732_b200 import binding

    k_out, v_out = (torch.zeros_like(t.contiguous()) for t in (k, v)) if held else (None, None)
    got = binding.pcg_cache_append_fourbit(q, k, v, slots, cache, positions=positions, table=tab, interleaved=inter, k_scale=ks, v_scale=vs,
                                           k_out=k_out, v_out=v_out, **kw)
    return got, k_out, v_out


@pytest.mark.parametrize("rows,qh,kvh,d,dim,inter,bs,dtype,kind,ks,vs", CASES)
def test_append(rows, qh, kvh, d, dim, inter, bs, dtype, kind, ks, vs):
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(rows)
    fused = torch.randn((rows, qh + 2 * kvh, d), generator=gen).to(dtype).cuda()
    fused[:, qh:qh + kvh] *= 5 * ks
    fused[:, qh + kvh:] *= vs
    q, k, v = (fused[:, :qh] if dim else None), fused[:, qh:qh + kvh], fused[:, qh + kvh:]
    slots, n_blocks = _slots(kind, rows, bs, gen)
    cache = torch.randint(0, 256, binding.pcg_fourbit_cache_shape(n_blocks, kvh, bs, d), generator=gen, dtype=torch.uint8)
    positions, tab = (torch.randint(0, 900, (rows,), generator=gen, dtype=torch.int32), R.table(900, dim)) if dim else (None, None)
    mine = cache.cuda()
    got, k_out, v_out = _call(k, v, slots.cuda(), mine, q, positions.cuda() if dim else None, tab.cuda() if dim else None, bool(inter), ks, vs)
    # the cache's bytes, neighbours among them, in float32 steps on the host
    kt = R.turn32(k.cpu(), positions, tab, inter) if dim else k.cpu().float()
    (kc, k8), (vc, v8) = R.quantise32(kt, ks), R.quantise32(v.cpu().float(), vs)
    for r in range(rows):
        for h in range(kvh):
            R.write(cache, int(slots[r]), h, kc[r, h], k8[r, h], vc[r, h], v8[r, h])
    assert torch.equal(mine.cpu(), cache)
    if dim:
        R.check_turned(got, q, positions.cuda(), tab.cuda(), inter)
    # what is held, in 64 bits: nearest values, and the outputs are what the cache holds, rounded
    g32 = [float(torch.tensor(g, dtype=torch.float32)) for g in (ks, vs)]
    half = torch.finfo(dtype).eps / 2
    for h in range(kvh):
        for values, out, g, x in ((False, k_out, g32[0], kt[:, h].double().cuda()), (True, v_out, g32[1], v[:, h].double())):
            held = R.read(mine, slots, h, g, values)
            R.check_held(held, x, g)
            assert bool(((out[:, h].double() - held).abs() <= (half + 2.0 ** -23) * held.abs() + R.step(dtype)).all())


def test_ties_go_to_the_even_value_and_large_ones_to_the_largest():
    """A scale of exactly 1 (the largest of the 16 is 6) and values in the middle of two."""
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    even = [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    x = torch.tensor([6.0] + ties + [-t for t in ties] + [-6.0], dtype=torch.float32)
    want = torch.tensor([6.0] + even + [-t for t in even] + [-6.0], dtype=torch.float32)
    x, want = (torch.cat([t, t * 32]).view(1, 1, 32).cuda() for t in (x, want))
    cache = torch.zeros(2, 1, 1, 18 * 32, dtype=torch.uint8, device="cuda")
    _, k_out, v_out = _call(x, x, torch.tensor([5], dtype=torch.int32, device="cuda"), cache)
    assert torch.equal(k_out, want) and torch.equal(v_out, want)
    # the scale's own ties: 17 / 16 is in the middle of 1 and 9 / 8, 19 / 16 of 9 / 8 and 10 / 8
    for top, held in ((6 * 17 / 16, 6.0), (6 * 19 / 16, 6 * 1.25), (1e6, 6 * 448.0), (6 * 2.0 ** -10, 0.0), (6.1 * 2.0 ** -10, 3 * 2.0 ** -9)):
        x = torch.full((1, 1, 32), top, device="cuda")
        _, k_out, v_out = _call(x, -x, torch.tensor([5], dtype=torch.int32, device="cuda"), cache)
        assert bool((k_out == held).all()) and bool((v_out == -held).all()), (top, k_out)


def test_infinite_values_zeros_and_nan():
    x = torch.randn(6, 2, 64, device="cuda")
    x[1] = 0.0
    x[2, 0, 5], x[2, 1, 40] = float("inf"), float("-inf")
    x[3, 1, 17] = float("nan")
    x[4] = 1e-30
    cache = torch.zeros(2, 2, 1, 18 * 64, dtype=torch.uint8, device="cuda")
    _, k_out, v_out = _call(x, x, torch.arange(6, dtype=torch.int32, device="cuda"), cache)
    assert torch.equal(k_out.isnan(), v_out.isnan())
    assert not bool(k_out[1].any()) and not bool(k_out[4].any())
    assert k_out[2, 0, 5] == 2688 and k_out[2, 1, 40] == -2688 and bool((k_out[2, 0, :5] == 0).all())
    nan = k_out.isnan().cpu()
    want = torch.zeros_like(nan)
    want[3, 1, 16:32] = True
    assert torch.equal(nan, want)
    for h in range(2):
        held = R.read(cache, torch.arange(6), h, 1.0, False)
        assert torch.equal(held.isnan().cpu(), want[:, h]) and torch.equal(held.nan_to_num().float(), k_out[:, h].nan_to_num())


def test_rows_without_a_slot_or_a_position():
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn(20, 2, 64, generator=gen).cuda() for _ in range(2))
    q = torch.randn(20, 4, 64, generator=gen).cuda()
    slots = torch.arange(3, 23, dtype=torch.int32)
    slots[4], slots[9] = -1, 4 * 16
    positions = torch.arange(20, dtype=torch.int32)
    positions[7], positions[12] = -1, 30
    tab = R.table(30, 64)
    cache = torch.randint(0, 256, binding.pcg_fourbit_cache_shape(4, 2, 16, 64), generator=gen, dtype=torch.uint8)
    mine = cache.cuda()
    q_out = torch.full_like(q, 3.0)
    k_out, v_out = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    binding.pcg_cache_append_fourbit(q, k, v, slots.cuda(), mine, positions=positions.cuda(), table=tab.cuda(), q_out=q_out, k_out=k_out,
                                     v_out=v_out)
    safe = positions.clamp(0, 29)
    kt = R.turn32(k.cpu(), safe, tab, 0)
    (kc, k8), (vc, v8) = R.quantise32(kt, 1.0), R.quantise32(v.cpu(), 1.0)
    for r in range(20):
        if r in (4, 9, 7, 12):
            continue
        for h in range(2):
            R.write(cache, int(slots[r]), h, kc[r, h], k8[r, h], vc[r, h], v8[r, h])
    for h in range(2):  # row 12's key has no angle: NaN; its value has its place
        R.write(cache, int(slots[12]), h, kc[12, h] * 0, torch.full_like(k8[12, h], 0x7F), vc[12, h], v8[12, h])
    at = mine.cpu()
    t = int(slots[12]) % 16
    for h in range(2):  # the codes beside a scale of NaN are of no matter
        for c in range(2):
            at[int(slots[12]) // 16, h, 0, c * 256 + t * 16: c * 256 + t * 16 + 16] = 0
    assert torch.equal(at, cache)
    for r in (4, 9):
        assert not bool((q_out[r] == 3.0).any()) and torch.equal(v_out[r, 0], R.read(mine, slots[5:6], 0, 1.0, True)[0].float()) is False
        R.check_held(v_out[r], v[r], 1.0)
    assert bool((q_out[7] == 3.0).all()) and bool((k_out[7] == 3.0).all()) and bool((v_out[7] == 3.0).all())
    assert bool(q_out[12].isnan().all()) and bool(k_out[12].isnan().all()) and not bool(v_out[12].isnan().any())


def test_many_rows_in_whole_and_split_pages():
    """A batch of prompts of odd lengths, and the same rows in another order: the same cache."""
    from paper_2511_13732_b200 import binding

    gen = torch.Generator().manual_seed(8)
    lens, kvh, d, bs = [100, 1, 37, 16, 333, 15, 17], 2, 128, 64
    rows = sum(lens)
    blocks = iter(torch.randperm(60, generator=gen).tolist())
    slots = []
    for n in lens:
        mine = [next(blocks) for _ in range((n + bs - 1) // bs)]
        slots += [mine[i // bs] * bs + i % bs for i in range(n)]
    slots = torch.tensor(slots, dtype=torch.int32)
    k, v = (torch.randn(rows, kvh, d, generator=gen).bfloat16().cuda() for _ in range(2))
    start = torch.randint(0, 256, binding.pcg_fourbit_cache_shape(60, kvh, bs, d), generator=gen, dtype=torch.uint8).cuda()
    one, other = start.clone(), start.clone()
    _, k_out, v_out = _call(k, v, slots.cuda(), one)
    p = torch.randperm(rows, generator=gen)
    _call(k[p.cuda()], v[p.cuda()], slots[p].cuda(), other, held=False)
    assert torch.equal(one, other)
    for h in range(kvh):
        assert torch.equal(R.read(one, slots, h, 1.0, False).to(k.dtype), k_out[:, h])
        assert torch.equal(R.read(one, slots, h, 1.0, True).to(v.dtype), v_out[:, h])
    R.check_held(v_out, v, 1.0)
