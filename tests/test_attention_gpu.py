"""pcg_cache_attention and pcg_prompt_attention against 64-bit attention, on the GPU."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Paged:
    """Sequences with `lens` = [(tokens cached before, new tokens)] in a shuffled paged cache.  Everything that attention
    may not use holds NaN (cache) or arbitrary numbers (block table)."""

    def __init__(self, lens, qh, kvh, d, bs, dtype, seed=0, lead=0, tail=0, short=0, spread=1.5):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        rng = random.Random(seed)
        self.lens, self.bs, self.dtype, self.d, self.qh, self.kvh = lens, bs, dtype, d, qh, kvh
        used = [-(-(c + n - short) // bs) if c + n - short > 0 else 0 for c, n in lens]
        n_blocks = sum(used) + 2
        ids = list(range(n_blocks))
        rng.shuffle(ids)
        width = max(max(used), 1) + 1
        table = [[rng.choice([-1, 2 ** 31 - 1, n_blocks]) for _ in range(width)] for _ in lens]
        rnd = lambda *s: torch.randn(s, generator=self.g, device="cuda")  # noqa: E731
        self.kc, self.vc = (torch.full((n_blocks, kvh, bs, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        self.k, self.v, start, kv_len = [], [], [lead], []
        for b, (c, n) in enumerate(lens):
            L = max(c + n - short, 0)
            k, v = rnd(L, kvh, d).to(dtype), rnd(L, kvh, d).to(dtype)
            for j in range(used[b]):
                table[b][j] = ids.pop()
                part = slice(j * bs, min(L, (j + 1) * bs))
                w = part.stop - part.start
                self.kc[table[b][j], :, :w] = k[part].transpose(0, 1)
                self.vc[table[b][j], :, :w] = v[part].transpose(0, 1)
            self.k.append(k), self.v.append(v), kv_len.append(c + n - short), start.append(start[-1] + n)
        self.q = (rnd(start[-1] + tail, qh, d) * spread).to(dtype)
        self.start, self.kv_len, self.table = _ints(start), _ints(kv_len), _ints(table)
        self.short = short

    def run(self, **kw):
        from paper_2511_13732_b200 import binding

        return binding.pcg_cache_attention(self.q, self.start, self.kv_len, self.table, self.kc, self.vc, **kw)

    def check(self, got, scale=None):
        import cache_ref

        start = self.start.tolist()
        for b, (c, n) in enumerate(self.lens):
            lim = [max(c - self.short + i + 1, 0) for i in range(n)]
            if n == 0:
                continue
            rows = slice(start[b], start[b + 1])
            want = cache_ref.attention(self.q[rows], self.k[b], self.v[b], lim, self.d ** -0.5 if scale is None else scale)
            cache_ref.check(got[rows], want, self.dtype, self.d, c + n, (b, c, n))


HEADS = [(1, 1), (4, 4), (8, 2), (32, 8), (12, 4), (7, 1), (28, 4), (40, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_single_tokens(dtype, d, heads):
    lens = [(0, 1), (1, 1), (15, 1), (16, 1), (63, 1), (127, 1), (128, 1), (129, 1), (300, 1), (1000, 1)]
    s = Paged(lens, *heads, d, 16, dtype, seed=1)
    s.check(s.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bs", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_drafted_chunks_over_every_block_size(dtype, bs, d):
    lens = [(0, 5), (1, 17), (250, 9), (511, 5), (128 - 5, 5), (700, 2), (33, 1), (0, 0), (90, 0), (256, 16)]
    s = Paged(lens, 8, 2, d, bs, dtype, seed=2)
    s.check(s.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(8, 2), (4, 4), (28, 4), (40, 2), (3, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_of_prompts(dtype, heads, d):
    lens = [(0, 300), (100, 129), (513, 64), (1000, 33), (5, 257), (0, 1), (31, 32)]
    s = Paged(lens, *heads, d, 32, dtype, seed=3)
    s.check(s.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 40, 72, 80, 96, 192, 256])
def test_other_head_dimensions(dtype, d):
    s = Paged([(0, 3), (77, 5), (200, 1), (0, 140)], 6, 2, d, 16, dtype, seed=4)
    s.check(s.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128, 96])
def test_rows_that_see_nothing_are_zero(dtype, d):
    s = Paged([(0, 5), (2, 9), (0, 300), (40, 3)], 8, 2, d, 16, dtype, seed=5, short=4)
    got = s.run(out=torch.full_like(s.q, 7.0))
    s.check(got)
    assert not got[:4].any() and not got[5:7].any()
    s.kv_len = _ints([-7, 0, 0, -2 ** 31])  # lengths below zero are zero
    assert not s.run(out=torch.full_like(s.q, 7.0)).any()


@pytest.mark.parametrize("d", [64, 128, 48])
def test_rows_of_no_sequence_are_left_as_they_were(d):
    s = Paged([(9, 4), (0, 0), (150, 20)], 8, 2, d, 64, torch.bfloat16, seed=6, lead=3, tail=6)
    got = s.run(out=torch.full_like(s.q, 7.0))
    assert bool((got[:3] == 7).all()) and bool((got[-6:] == 7).all())
    s.check(got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 32])
def test_used_entries_outside_the_cache_are_zeros(dtype, d):
    s = Paged([(100, 5), (300, 1), (64, 150)], 8, 2, d, 64, dtype, seed=7)
    for b, j in ((0, 1), (1, 0), (1, 4), (2, 2)):
        s.table[b, j] = random.Random(b).choice([-1, -2 ** 31, s.kc.shape[0], 2 ** 31 - 1])
        s.k[b][64 * j: 64 * j + 64] = 0
        s.v[b][64 * j: 64 * j + 64] = 0
    s.check(s.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_flat_and_steep_scores_and_scales(dtype, spread):
    s = Paged([(500, 5), (3, 1), (10, 200)], 8, 2, 64, 16, dtype, seed=8, spread=spread)
    s.check(s.run())
    s.check(s.run(scale=0.01), scale=0.01)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_grow_along_the_keys(d):
    """Each block of keys outdoes the last by far: the running reference moves in every tile."""
    s = Paged([(1500, 3), (700, 200)], 8, 2, d, 64, torch.bfloat16, seed=9)
    for b, (c, n) in enumerate(s.lens):
        s.q[:, :, 0] = 4.0
        s.k[b][:, :, 0] = (torch.arange(c + n, device="cuda") // 32).float()[:, None].to(s.dtype)
        for j in range(-(-(c + n) // 64)):
            w = min(64, c + n - 64 * j)
            s.kc[s.table[b, j], :, :w] = s.k[b][64 * j: 64 * j + w].transpose(0, 1)
    s.check(s.run())


@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16), (128, torch.float16), (64, torch.float32)])
def test_infinite_and_undefined_scores(d, dtype):
    """A score of -inf weighs nothing; a row of them, of +inf or of NaN is NaN, as its softmax is; others are untouched."""
    s = Paged([(200, 1), (200, 1), (200, 1), (200, 1)], 2, 2, d, 64, dtype, seed=10)
    s.q[:, :, 0] = 1.0
    kc = s.kc.clone()
    kc[s.table[0, 1], 0, 5, 0] = float("-inf")  # one score
    for j in range(4):
        kc[s.table[1, j], 0, :, 0] = float("-inf")  # all scores of one head
    kc[s.table[2, 0], 1, 3, 0] = float("inf")
    kc[s.table[3, 2], 1, 3, 0] = float("nan")
    want = s.run()
    s.kc = kc
    got = s.run()
    assert bool(torch.isnan(got[1, 0]).all()) and bool(torch.isnan(got[2, 1]).all()) and bool(torch.isnan(got[3, 1]).all())
    for r, h in ((0, 1), (1, 1), (2, 0), (3, 0)):
        assert torch.equal(got[r, h], want[r, h])
    s.k[0][69, 0, 0] = float("-inf")
    import cache_ref

    o, a, m = cache_ref.attention(s.q[:1, :1], s.k[0][:, :1], s.v[0][:, :1], [201], d ** -0.5)
    m = torch.full_like(m, 40.0)
    cache_ref.check(got[:1, :1], (o, a, m), dtype, d, 201)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [80, 24, 256, 64, 128])
@pytest.mark.parametrize("lo,hi", [(0, 32), (32, 64), (200, 201), (192, 201), (0, 201)])
def test_undefined_scores_next_to_each_other(dtype, d, lo, hi):
    """A row that sees a score that is NaN is NaN, however many of its neighbours are; the other head is untouched."""
    s = Paged([(200, 1), (200, 1)], 2, 2, d, 64, dtype, seed=13)
    want = s.run()
    for p in range(lo, hi):
        s.kc[s.table[0, p // 64], 0, p % 64, d - 1] = float("nan")
    got = s.run()
    assert bool(torch.isnan(got[0, 0]).all()) and torch.equal(got[0, 1], want[0, 1]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,n", [(1, 1), (3, 5), (70, 17), (2, 200), (300, 1)])
def test_results_do_not_depend_on_the_run(dtype, B, n):
    rng = random.Random(B)
    s = Paged([(rng.randint(0, 2500 if B < 50 else 400), n) for _ in range(B)], 16, 4, 64, 32, dtype, seed=11)
    first = s.run()
    s.check(first)
    ws = torch.empty(1, dtype=torch.uint8)
    from paper_2511_13732_b200 import binding

    ws = torch.full((binding.pcg_attention_workspace_bytes(B, 16, 4, 64, binding.dtype_code(s.q)),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        assert torch.equal(first, s.run(workspace=ws))


def test_one_very_long_sequence():
    s = Paged([(60000, 3)], 8, 2, 128, 128, torch.bfloat16, seed=12)
    s.check(s.run())


def test_offsets_past_32_bits():
    from paper_2511_13732_b200 import binding
    import cache_ref

    n_blocks, kvh, bs, d = 70000, 8, 64, 128  # 4.6e9 elements each
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    kc, vc = (torch.empty((n_blocks, kvh, bs, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    blocks = [69999, 3, 66000]
    for j in blocks:
        kc[j].normal_(), vc[j].normal_()
    q = torch.randn((4, 16, d), device="cuda").bfloat16()
    got = binding.pcg_cache_attention(q, _ints([0, 4]), _ints([190]), _ints([blocks]), kc, vc)
    k, v = (c[blocks].transpose(1, 2).reshape(-1, kvh, d)[:190] for c in (kc, vc))
    cache_ref.check(got, cache_ref.attention(q, k, v, [187, 188, 189, 190], d ** -0.5), torch.bfloat16, d, 190)


# ---- whole prompts -------------------------------------------------------------------------------------------------
def _prompt(lens, qh, kvh, d, dtype, seed=0, lead=0, tail=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    start = [lead]
    for n in lens:
        start.append(start[-1] + n)
    fused = torch.randn((start[-1] + tail, qh + 2 * kvh, d), generator=g, device="cuda").to(dtype)
    return fused[:, :qh], fused[:, qh:qh + kvh], fused[:, qh + kvh:], start


def _check_prompt(got, q, k, v, start, dtype):
    import cache_ref

    for lo, hi in zip(start, start[1:]):
        if hi > lo:
            want = cache_ref.attention(q[lo:hi], k[lo:hi], v[lo:hi], list(range(1, hi - lo + 1)), q.shape[2] ** -0.5)
            cache_ref.check(got[lo:hi], want, dtype, q.shape[2], hi - lo, (lo, hi))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128, 24])
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (5, 5), (28, 4), (40, 2)])
def test_packed_prompts(dtype, d, heads):
    from paper_2511_13732_b200 import binding

    lens = [1, 2, 0, 127, 128, 129, 31, 300, 0, 64, 513]
    q, k, v, start = _prompt(lens, *heads, d, dtype, seed=20)
    _check_prompt(binding.pcg_prompt_attention(q, k, v, _ints(start)), q, k, v, start, dtype)
    _check_prompt(binding.pcg_prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), _ints(start)), q, k, v, start, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_long_prompt_and_a_single_token(dtype):
    from paper_2511_13732_b200 import binding

    for lens in ([2500], [1]):
        q, k, v, start = _prompt(lens, 8, 2, 128, dtype, seed=21)
        _check_prompt(binding.pcg_prompt_attention(q, k, v, _ints(start)), q, k, v, start, dtype)


@pytest.mark.parametrize("d", [64, 128, 16])
def test_neighbours_and_padding_of_a_prompt_are_not_used(d):
    """What lies before, between and behind the prompts' rows is NaN, and other prompts hold NaN: none of it is seen."""
    from paper_2511_13732_b200 import binding

    lens = [70, 1, 200, 90]
    q, k, v, start = _prompt(lens, 8, 2, d, torch.bfloat16, seed=22, lead=5, tail=9)
    for t in (q, k, v):
        t[:5] = float("nan")
        t[-9:] = float("nan")
        t[start[2]:start[3]] = float("nan")  # the whole third prompt
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    got = binding.pcg_prompt_attention(q, k, v, _ints(start), out=out)
    assert bool((got[:5] == 7).all()) and bool((got[-9:] == 7).all()) and bool(torch.isnan(got[start[2]:start[3]]).all())
    for i in (0, 1, 3):
        _check_prompt(got, q, k, v, start[i:i + 2], torch.bfloat16)


@pytest.mark.parametrize("d", [64, 16])
def test_row_starts_outside_the_rows_are_cut(d):
    from paper_2511_13732_b200 import binding

    q, k, v, _ = _prompt([150], 8, 2, d, torch.bfloat16, seed=23)
    got = binding.pcg_prompt_attention(q, k, v, _ints([-5, 40, 10 ** 6, 2 ** 31 - 1]))
    _check_prompt(got, q, k, v, [0, 40, 150], torch.bfloat16)


# ---- streams, graphs -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [1, 5, 200])
def test_a_captured_call_replays_on_new_inputs(n):
    a, b = (Paged([(300 + i, n), (20, n), (900, n)], 8, 2, 64, 32, torch.bfloat16, seed=30 + i) for i in range(2))
    from paper_2511_13732_b200 import binding

    ws = torch.empty(binding.pcg_attention_workspace_bytes(3, 8, 2, 64, binding.PCG_BF16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(a.q)
    a.run(out=out, workspace=ws)
    q, table, kv_len = a.q.clone(), a.table.clone(), a.kv_len.clone()
    n_blocks = max(a.kc.shape[0], b.kc.shape[0])
    kc, vc = (torch.zeros((n_blocks,) + a.kc.shape[1:], dtype=a.kc.dtype, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.pcg_cache_attention(q, a.start, kv_len, table, kc, vc, out=out, workspace=ws)
    for s in (b, a, b):
        q.copy_(s.q), table.copy_(s.table), kv_len.copy_(s.kv_len)
        kc[: s.kc.shape[0]], vc[: s.vc.shape[0]] = s.kc, s.vc
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        s.check(out)


def test_two_streams_with_their_own_workspaces():
    sets = [Paged([(700 + 90 * i, 5), (40, 60)], 8, 2, 128, 64, torch.bfloat16, seed=40 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                outs[i].append(s.run(stream=streams[i]))
    torch.cuda.synchronize()
    for s, got in zip(sets, outs):
        s.check(got[0])
        assert all(torch.equal(got[0], x) for x in got)


# ---- what the documentation allows and a model seldom does -----------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128, 40])
def test_outputs_and_queries_on_any_16_byte_boundary(dtype, d):
    s = Paged([(300, 5), (70, 1), (0, 150)], 8, 2, d, 32, dtype, seed=50)
    want = s.run()
    step = 16 // want.element_size()
    room = torch.zeros(want.numel() + 2 * step, dtype=dtype, device="cuda")
    out = room[step: step + want.numel()].view(want.shape)
    wide = torch.zeros((s.q.shape[0], s.q.shape[1] * d + step), dtype=dtype, device="cuda")  # rows 16 bytes apart from dense
    q = wide[:, step:].unflatten(1, (s.q.shape[1], d))
    q.copy_(s.q)
    s.q = q
    assert torch.equal(s.run(out=out), want)
    assert not room[:step].any() and not room[step + want.numel():].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_beyond_the_table_are_cut(dtype):
    import cache_ref

    s = Paged([(100, 5), (40, 3)], 4, 2, 64, 16, dtype, seed=51)
    width = s.table.shape[1] * 16
    s.kv_len = _ints([2 ** 31 - 1, width + 1])
    got = s.run()
    for b, n in ((0, 5), (1, 3)):
        k, v = torch.zeros((width, 2, 64), dtype=dtype, device="cuda"), torch.zeros((width, 2, 64), dtype=dtype, device="cuda")
        blocks = s.table[b].tolist()
        used = [j for j in range(len(blocks)) if 0 <= blocks[j] < s.kc.shape[0]]
        s.kc.nan_to_num_(0.0), s.vc.nan_to_num_(0.0)
        for j in used:
            k[16 * j: 16 * j + 16], v[16 * j: 16 * j + 16] = s.kc[blocks[j]].transpose(0, 1), s.vc[blocks[j]].transpose(0, 1)
        rows = slice(0, 5) if b == 0 else slice(5, 8)
        got = s.run()
        cache_ref.check(got[rows], cache_ref.attention(s.q[rows], k, v, [width - n + i + 1 for i in range(n)], 0.125), dtype, 64, width)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_batch(dtype, d):
    """16384 sequences of one token: each row is its own value; the next size is refused."""
    from paper_2511_13732_b200 import binding

    B = 16384
    q, k, v = (torch.randn((B, h, d), device="cuda").to(dtype) for h in (4, 2, 2))
    start = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    got = binding.pcg_prompt_attention(q, k, v, start)
    assert torch.equal(got, v.repeat_interleave(2, 1))
    kc, vc = (torch.zeros((B, 2, 16, d), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.randperm(B, device="cuda").to(torch.int32)[:, None].contiguous()
    binding.pcg_cache_append(k, v, table[:, 0] * 16, kc, vc)
    got = binding.pcg_cache_attention(q, start, torch.ones(B, dtype=torch.int32, device="cuda"), table, kc, vc)
    assert torch.equal(got, v.repeat_interleave(2, 1))
    with pytest.raises(binding.PcgError):
        binding.pcg_prompt_attention(q, k, v, torch.arange(B + 2, dtype=torch.int32, device="cuda").clamp(max=B))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
def test_mixed_batches_of_tokens_chunks_and_prompts(dtype, d):
    """Items with one row tile and with two in one call, in any order: the ring's stages mean different things to them."""
    rng = random.Random(d)
    for seed in range(6):
        lens = [(rng.choice([0, 3, 63, 64, 65, 500, 1300]), rng.choice([0, 1, 1, 2, 5, 17, 31, 32, 33, 64, 65, 96, 200, 400]))
                for _ in range(rng.randint(1, 40))]
        s = Paged(lens, 8, 2, d, rng.choice([16, 64, 256]), dtype, seed=60 + seed)
        s.check(s.run())


@pytest.mark.parametrize("heads", [(128, 1), (100, 1), (64, 2), (6, 2), (5, 1), (96, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_and_odd_heads_a_key_head(heads, dtype):
    s = Paged([(70, 1), (10, 4), (0, 9), (300, 2)], *heads, 64, 16, dtype, seed=70)
    s.check(s.run())


def test_calls_that_share_a_workspace_in_one_stream():
    """Back to back, of different sizes and types, without a wait between them."""
    from paper_2511_13732_b200 import binding

    sets = [Paged([(900, 5), (20, 1)], 8, 2, 128, 32, torch.bfloat16, seed=80), Paged([(0, 400), (50, 3)], 8, 2, 64, 16, torch.float16, seed=81),
            Paged([(333, 17)] * 5, 8, 2, 64, 16, torch.float32, seed=82)]
    ws = torch.empty(max(binding.pcg_attention_workspace_bytes(9, 8, 2, d, 0) for d in (64, 128)), dtype=torch.uint8, device="cuda")
    want = [s.run() for s in sets]
    torch.cuda.synchronize()
    outs = [[s.run(workspace=ws) for s in sets] for _ in range(8)]
    torch.cuda.synchronize()
    for s, w, got in zip(sets, want, zip(*outs)):
        s.check(w)
        assert all(torch.equal(w, x) for x in got)
