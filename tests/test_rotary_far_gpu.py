"""The append with rotation at the end of a pool that just passes 2^31 elements (two caches of 4.3 GB, and little else)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import fourbit_ref as R  # noqa: E402


@pytest.mark.parametrize("inter", [False, True])
def test_the_last_slots_of_a_pool_beyond_32_bits_of_elements(inter):
    from paper_2511_13732_b200 import binding

    if torch.cuda.mem_get_info()[0] < 10 << 30:
        pytest.skip("too little memory")
    kvh, bs, d, rows = 8, 64, 128, 70
    n_blocks = 2 ** 31 // (kvh * bs * d) + 3
    kc = torch.empty((n_blocks, kvh, bs, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    assert kc.numel() > 2 ** 31 and kc[-2:].data_ptr() - kc.data_ptr() > 2 ** 32
    kc[-3:], vc[-3:] = 7.0, 7.0
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(rows, h, d, generator=gen, device="cuda").bfloat16() for h in (16, kvh, kvh))
    at = torch.arange(rows, dtype=torch.int32, device="cuda")
    slots, positions, tab = (n_blocks * bs - rows + at).int(), 40000 - rows + at, R.table(40000, d).cuda()
    got = binding.pcg_cache_append_rotary(q, k, v, slots, positions, tab, kc, vc, interleaved=inter)
    R.check_turned(got, q, positions, tab, inter)
    held = [c[slots.long() // bs, :, slots.long() % bs] for c in (kc, vc)]
    R.check_turned(held[0], k, positions, tab, inter)
    assert torch.equal(held[1], v)
    before = torch.arange((n_blocks - 3) * bs, n_blocks * bs - rows, device="cuda")
    for c in (kc, vc):  # neighbours as they were
        assert bool((c[before // bs, :, before % bs] == 7.0).all())
