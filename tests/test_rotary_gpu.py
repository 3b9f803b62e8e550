"""The append with position rotation against 64-bit rotation: types, head layouts, both orders of pairs, partial rotation,
strides, rows without a slot or a position, in place."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import fourbit_ref as R  # noqa: E402

CASES = [
    # (rows, q_heads, kv_heads, d, dim, interleaved, block_size, dtype)
    (1, 4, 2, 64, 64, 0, 16, torch.bfloat16),
    (5, 12, 4, 64, 64, 0, 16, torch.float32),
    (17, 8, 1, 128, 128, 1, 32, torch.float16),
    (33, 28, 4, 128, 128, 0, 64, torch.bfloat16),
    (7, 3, 3, 80, 80, 0, 16, torch.bfloat16),
    (7, 6, 2, 80, 48, 1, 16, torch.float16),
    (9, 5, 5, 96, 32, 0, 256, torch.float32),
    (6, 2, 1, 256, 256, 0, 128, torch.bfloat16),
    (4, 1, 1, 16, 16, 1, 16, torch.float16),
    (3, 40, 40, 24, 16, 0, 16, torch.bfloat16),
    (2, 71, 1, 64, 32, 1, 16, torch.float32),
]


def _inputs(rows, qh, kvh, d, dim, bs, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    fused = torch.randn((rows, qh + 2 * kvh, d), generator=g).to(dtype).cuda()
    n_blocks = rows // bs + 3
    slots = torch.randperm(n_blocks * bs, generator=g)[:rows].to(torch.int32)
    positions = torch.randint(0, 5000, (rows,), generator=g, dtype=torch.int32)
    tab = R.table(5000, dim).cuda()
    caches = [torch.full((n_blocks, kvh, bs, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    return fused[:, :qh], fused[:, qh:qh + kvh], fused[:, qh + kvh:], slots.cuda(), positions.cuda(), tab, caches


def _rows_of(cache, slots):
    bs = cache.shape[2]
    return cache[slots.long() // bs, :, slots.long() % bs]


@pytest.mark.parametrize("rows,qh,kvh,d,dim,inter,bs,dtype", CASES)
def test_append_with_rotation(rows, qh, kvh, d, dim, inter, bs, dtype):
    from paper_2511_13732_b200 import binding

    q, k, v, slots, positions, tab, (kc, vc) = _inputs(rows, qh, kvh, d, dim, bs, dtype)
    k_out = torch.zeros(rows, kvh, d, dtype=dtype, device="cuda")
    got = binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, interleaved=bool(inter), k_out=k_out)
    R.check_turned(got, q, positions, tab, inter)
    R.check_turned(k_out, k, positions, tab, inter)
    assert torch.equal(_rows_of(kc, slots), k_out) and torch.equal(_rows_of(vc, slots), v)
    if dim < d:
        assert torch.equal(got[..., dim:], q[..., dim:])
    other = torch.ones(kc.shape[0] * bs, dtype=torch.bool, device="cuda")
    other[slots.long()] = False
    rest = torch.arange(kc.shape[0] * bs, device="cuda")[other]
    for c in (kc, vc):
        assert bool((_rows_of(c, rest) == 7.0).all())
    # once more without queries: the same cache
    kc2, vc2 = torch.full_like(kc, 7.0), torch.full_like(vc, 7.0)
    assert binding.pcg_cache_append_rotary(None, k, v, slots, positions, tab, kc2, vc2, interleaved=bool(inter)) is None
    assert torch.equal(kc, kc2) and torch.equal(vc, vc2)


def test_rows_without_a_slot_or_a_position():
    from paper_2511_13732_b200 import binding

    q, k, v, slots, positions, tab, (kc, vc) = _inputs(8, 4, 2, 64, 64, 16, torch.bfloat16)
    slots[1] = -1
    slots[2] = kc.shape[0] * 16
    positions[3] = -1
    positions[4] = -2 ** 31
    positions[5] = 5000
    q_out, k_out = torch.full_like(q.contiguous(), 3.0), torch.full_like(k.contiguous(), 3.0)
    binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, q_out=q_out, k_out=k_out)
    for r in (0, 1, 2, 6, 7):
        one = slice(r, r + 1)
        R.check_turned(q_out[one], q[one], positions[one], tab, 0)
        R.check_turned(k_out[one], k[one], positions[one], tab, 0)
    for r in (3, 4):
        assert bool((q_out[r] == 3.0).all()) and bool((k_out[r] == 3.0).all())
        assert bool((_rows_of(kc, slots[r:r + 1]) == 7.0).all())
    assert bool(q_out[5].isnan().all()) and bool(k_out[5].isnan().all()) and bool(_rows_of(kc, slots[5:6]).isnan().all())
    assert torch.equal(_rows_of(vc, slots[5:6])[0], v[5])
    written = [r for r in (0, 5, 6, 7)]
    assert int((kc != 7.0).any(-1).sum()) <= len(written) * 2 and int((vc != 7.0).any(-1).sum()) <= len(written) * 2


@pytest.mark.parametrize("inter", [0, 1])
def test_in_place_of_a_fused_projection(inter):
    from paper_2511_13732_b200 import binding

    q, k, v, slots, positions, tab, (kc, vc) = _inputs(37, 8, 2, 128, 64, 32, torch.bfloat16)
    kc2, vc2 = kc.clone(), vc.clone()
    k_out = torch.empty_like(k.contiguous())
    want = binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, interleaved=bool(inter), k_out=k_out)
    vv = v.clone()
    got = binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc2, vc2, interleaved=bool(inter), q_out=q, k_out=k)
    assert got is q and torch.equal(q, want) and torch.equal(k, k_out) and torch.equal(v, vv)
    assert torch.equal(kc, kc2) and torch.equal(vc, vc2)


def test_far_positions_and_a_cache_beyond_32_bits_of_elements():
    """Row numbers times elements pass 2^31: a pool of 20 GB, whose last slots are written."""
    from paper_2511_13732_b200 import binding

    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("too little memory")
    n_blocks, kvh, bs, d = 40000, 8, 64, 128
    kc = torch.empty((n_blocks, kvh, bs, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    assert kc.numel() > 2 ** 31
    q, k, v, slots, positions, tab, _ = _inputs(40, 16, kvh, d, d, 64, torch.bfloat16)
    slots = torch.arange(n_blocks * bs - 40, n_blocks * bs, dtype=torch.int32, device="cuda")
    tab = R.table(300000, d).cuda()
    positions = torch.arange(300000 - 40, 300000, dtype=torch.int32, device="cuda")
    got = binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc)
    R.check_turned(got, q, positions, tab, 0)
    R.check_turned(_rows_of(kc, slots), k, positions, tab, 0)
    assert torch.equal(_rows_of(vc, slots), v)


def test_captured_and_replayed_with_new_positions():
    from paper_2511_13732_b200 import binding

    q, k, v, slots, positions, tab, (kc, vc) = _inputs(12, 4, 2, 64, 64, 16, torch.float16)
    q_out = torch.empty_like(q.contiguous())
    binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, q_out=q_out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, q_out=q_out)
    for seed in (1, 2):
        new = torch.randint(0, 5000, (12,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
        positions.copy_(new)
        graph.replay()
        R.check_turned(q_out, q, positions, tab, 0)
        R.check_turned(_rows_of(kc, slots), k, positions, tab, 0)
