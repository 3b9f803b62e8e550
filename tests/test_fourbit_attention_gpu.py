"""Attention over the cache of 4 bits against 64-bit attention over what the cache holds."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import cache_ref  # noqa: E402
import fourbit_ref as R  # noqa: E402


def _build(lens, news, qh, kvh, d, bs, dtype, ks=1.0, vs=1.0, seed=0, q_size=1.0, pad_rows=0, gap=0):
    """A cache of sequences whose kv_len are `lens`, filled by the library's own append; bytes behind the last tokens are
    random, their scales NaN."""
    from paper_2511_13732_b200 import binding

    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = len(lens)
    blocks = [(n + bs - 1) // bs for n in lens]
    max_blocks, n_blocks = max(max(blocks, default=0), 1) + 1, sum(blocks) + 2
    perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, max_blocks), -7, dtype=torch.int32, device="cuda")
    at, slots = 0, []
    for b in range(B):
        table[b, :blocks[b]] = perm[at:at + blocks[b]]
        at += blocks[b]
        p = torch.arange(lens[b], device="cuda")
        slots.append(table[b].long()[p // bs] * bs + p % bs)
    cache = torch.full(binding.pcg_fourbit_cache_shape(n_blocks, kvh, bs, d), 0x7F, dtype=torch.uint8, device="cuda")
    all_slots = torch.cat(slots).to(torch.int32) if slots else torch.zeros(0, dtype=torch.int32, device="cuda")
    k = torch.randn((all_slots.shape[0], kvh, d), generator=gen, device="cuda") * ks
    v = torch.randn((all_slots.shape[0], kvh, d), generator=gen, device="cuda") * vs
    if all_slots.shape[0]:
        binding.pcg_cache_append_fourbit(None, k, v, all_slots, cache, k_scale=ks, v_scale=vs)
    rows = gap + sum(news) + pad_rows
    q = (torch.randn((rows, qh, d), generator=gen, device="cuda") * q_size).to(dtype)
    start = torch.zeros(B + 1, dtype=torch.int32)
    start[1:] = torch.tensor(news).cumsum(0)
    return dict(q=q, start=(start + gap).cuda(), kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table, cache=cache,
                slots=slots, lens=lens, news=news, ks=ks, vs=vs)


def _run(s, **kw):
    from paper_2511_13732_b200 import binding

    return binding.pcg_cache_attention_fourbit(s["q"], s["start"], s["kv_len"], s["table"], s["cache"], k_scale=s["ks"], v_scale=s["vs"], **kw)


def _check(s, out, scale=None):
    q, start = s["q"], s["start"].tolist()
    d, kvh = q.shape[2], s["cache"].shape[1]
    g = [float(torch.tensor(x, dtype=torch.float32)) for x in (s["ks"], s["vs"])]
    for b, (L, n) in enumerate(zip(s["lens"], s["news"])):
        if n == 0:
            continue
        k, v = (torch.stack([R.read(s["cache"], s["slots"][b], h, g[i], bool(i)) for h in range(kvh)], 1) for i in range(2))
        lim = torch.arange(n, device="cuda") + L - n + 1
        lo = start[b]
        want = cache_ref.attention(q[lo:lo + n], k, v, lim, d ** -0.5 if scale is None else scale)
        R.check_attention(out[lo:lo + n], want, q.dtype, d, max(L, 1), b, largest=float(v.abs().max()) if L else 0.0)


SHAPES = [(4, 1, 64), (8, 2, 128), (12, 4, 64), (7, 1, 128), (16, 1, 64), (3, 3, 128), (48, 1, 128), (64, 1, 64), (6, 2, 96), (4, 4, 32),
          (5, 1, 256), (2, 1, 160), (2, 2, 192), (1, 1, 224)]


@pytest.mark.parametrize("qh,kvh,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_heads_and_types(qh, kvh, d, dtype):
    s = _build([40, 1, 150, 17, 128], [3, 1, 9, 0, 17], qh, kvh, d, 32, dtype)
    _check(s, _run(s))


@pytest.mark.parametrize("bs", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_block_sizes_and_edges_of_tiles(bs, d):
    lens = [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 383, 384, 385, 520]
    s = _build(lens, [1] * len(lens), 8, 2, d, bs, torch.bfloat16, seed=bs)
    _check(s, _run(s))


@pytest.mark.parametrize("qh,kvh", [(8, 2), (4, 4), (14, 2), (16, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_of_many_lengths(qh, kvh, d):
    news = [1, 2, 5, 8, 11, 12, 13, 17, 24, 25, 48, 49, 96, 97, 130]
    lens = [n + c for n, c in zip(news, [0, 200, 3, 0, 64, 127, 500, 300, 0, 1, 17, 260, 31, 0, 300])]
    s = _build(lens, news, qh, kvh, d, 16, torch.float16, ks=0.25, vs=2.0)
    _check(s, _run(s))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_contexts_are_shared_between_blocks(dtype):
    s = _build([20011, 5, 3000], [1, 5, 17], 8, 2, 128, 64, dtype)
    _check(s, _run(s))
    s = _build([33000], [2], 4, 1, 64, 256, dtype)
    _check(s, _run(s))


def test_a_long_chunk():
    s = _build([1500, 700], [700, 700], 8, 2, 128, 64, torch.bfloat16)
    _check(s, _run(s))


@pytest.mark.parametrize("d", [64, 96, 128])
def test_rows_that_see_nothing_and_rows_of_no_sequence(d):
    """More new rows than keys: the first ones see none.  Rows before the first sequence and behind the last stay."""
    s = _build([3, 0, 40, 0], [8, 2, 5, 0], 8, 2, d, 16, torch.bfloat16, gap=2, pad_rows=5)
    out = torch.full_like(s["q"], 9.0)
    _run(s, out=out)
    _check(s, out)
    assert bool((out[:2] == 9.0).all()) and bool((out[17:] == 9.0).all())
    assert not bool(out[2:7].any()) and not bool(out[10:12].any())


@pytest.mark.parametrize("d", [64, 160, 128])
def test_blocks_outside_the_pool_stand_for_zeros(d):
    s = _build([70, 200], [4, 20], 8, 2, d, 16, torch.float16)
    s["table"][0, 1], s["table"][1, 5], s["table"][1, 0] = -1, s["cache"].shape[0], 2 ** 31 - 1
    out = _run(s)
    zero = torch.zeros(1, *s["cache"].shape[1:], dtype=torch.uint8, device="cuda")
    s["cache"] = torch.cat([s["cache"], zero])
    n = s["cache"].shape[0] - 1
    for b, j in ((0, 1), (1, 5), (1, 0)):
        s["slots"][b][j * 16:(j + 1) * 16] = n * 16 + torch.arange(16, device="cuda")
    _check(s, out)


@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scores_far_apart(d, dtype):
    """Queries so large that the softmax picks one key, after the reference has moved many times; and scores far below 0."""
    s = _build([700, 300, 64], [3, 20, 1], 8, 2, d, 32, dtype, q_size=60.0)
    _check(s, _run(s))
    s = _build([700, 300, 64], [3, 20, 1], 8, 2, d, 32, dtype, q_size=1e-3)
    _check(s, _run(s))
    _check(s, _run(s, scale=3.0), scale=3.0)


def test_bfloat16_queries_of_any_size():
    """Sizes that float16 does not have, in one tile; each row has its own."""
    for d in (64, 128):
        s = _build([200, 90], [4, 9], 8, 2, d, 32, torch.bfloat16)
        size = 10.0 ** torch.linspace(-30, 4, s["q"].shape[0] * 8, device="cuda").view(-1, 8, 1)
        s["q"] = (s["q"].float() * size).bfloat16()
        _check(s, _run(s, scale=1e-4), scale=1e-4)
        s["q"] = (s["q"].float() * 1e30).bfloat16()
        _check(s, _run(s, scale=1e-34), scale=1e-34)


@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_with_infinite_and_nan_queries(d, dtype):
    s = _build([300, 40], [6, 30], 4, 2, d, 32, dtype)
    for r, h, x in ((1, 2, math.inf), (3, 0, math.nan), (20, 1, -math.inf)):
        s["q"][r, h, 7] = x
    out = _run(s)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    for r, h in ((1, 2), (3, 0), (20, 1)):
        assert bool(out[r, h].isnan().all())
        bad[r, h] = True
    s["q"][bad.cuda()] = 0
    got = _run(s)
    got[~bad.cuda()] = out[~bad.cuda()]
    _check(s, got)


@pytest.mark.parametrize("d", [64, 128])
def test_held_nan_reaches_the_rows_that_see_it_only(d):
    """A group of NaN among a sequence's keys: rows from its token on are NaN, the others and other sequences as before."""
    s = _build([100, 60], [20, 20], 4, 1, d, 32, torch.bfloat16)
    want = _run(s)
    slot = int(s["slots"][0][90])
    page = s["cache"][slot // 32, 0, slot % 32 // 16]
    page[8 * d + slot % 16 * (d // 16) + 1] = 0x7F
    out = _run(s)
    assert bool(out[10:20].isnan().all()) and torch.equal(out[:10], want[:10]) and torch.equal(out[20:], want[20:])


def test_results_do_not_change_from_run_to_run_or_with_a_used_workspace():
    from paper_2511_13732_b200 import binding

    s = _build([5000, 700, 30, 3000], [1, 17, 17, 60], 8, 2, 128, 16, torch.bfloat16)
    need = binding.pcg_attention_workspace_bytes(4, 8, 2, 128, 1)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    one = _run(s, workspace=ws)
    for _ in range(3):
        assert torch.equal(one, _run(s, workspace=ws))
    _check(s, one)


def test_lengths_are_clamped_to_the_table_and_rows_to_the_batch():
    s = _build([64, 40], [2, 3], 8, 2, 64, 32, torch.bfloat16)
    s["table"] = s["table"][:, :2].contiguous()
    s["kv_len"][0] = 100000  # the table holds 64
    _check(s, _run(s))
    s["start"][2] = 99  # rows end at 5
    _check(s, _run(s))


def test_strided_queries_and_unaligned_outputs():
    s = _build([300, 129, 40], [5, 17, 30], 8, 2, 128, 64, torch.bfloat16)
    rows = s["q"].shape[0]
    wide = torch.randn(rows, 20, 128, device="cuda").bfloat16()
    wide[:, 3:11] = s["q"]
    want = _run(s)
    s["q"] = wide[:, 3:11]
    buf = torch.zeros(rows * 8 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    out = buf[8:].view(rows, 8, 128)
    assert out.data_ptr() % 32 == 16
    _run(s, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("B,n", [(600, 1), (300, 4), (2000, 1)])
def test_many_sequences(B, n):
    gen = torch.Generator().manual_seed(B)
    lens = (torch.randint(0, 90, (B,), generator=gen) + n).tolist()
    s = _build(lens, [n] * B, 4, 1, 64, 16, torch.float16)
    _check(s, _run(s))


def test_the_largest_batch():
    B = 16384
    s = _build([1] * B, [1] * B, 2, 1, 64, 16, torch.bfloat16)
    out = _run(s)
    for b in (0, 1, 8191, B - 1):
        v = R.read(s["cache"], s["slots"][b], 0, 1.0, True)
        assert torch.equal(out[b], v.expand(2, 64).to(out.dtype))


def test_captured_and_replayed_on_another_stream():
    s = _build([500, 40], [17, 5], 8, 2, 128, 32, torch.bfloat16)
    out = torch.empty_like(s["q"])
    _run(s, out=out)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(s, out=out)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _run(s, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_a_cache_beyond_32_bits_of_bytes():
    """Blocks at the end of a pool of 7 GB."""
    from paper_2511_13732_b200 import binding

    s = _build([300], [5], 8, 2, 128, 64, torch.bfloat16)
    n = 1500000 // 4
    big = torch.empty(binding.pcg_fourbit_cache_shape(n, 2, 64, 128), dtype=torch.uint8, device="cuda")
    assert big.numel() > 2 ** 32
    small = s["cache"].shape[0]
    big[n - small:] = s["cache"]
    want = _run(s)
    s["cache"], s["table"] = big, torch.where(s["table"] >= 0, s["table"] + n - small, s["table"])
    assert torch.equal(_run(s), want)
