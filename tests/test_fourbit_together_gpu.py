"""The append to the cache of 4 bits and the attention over it as they are used together: batches that mix single tokens and
long chunks, large groups of heads, several calls at a time, captured rounds."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import fourbit_ref as R  # noqa: E402
from test_fourbit_attention_gpu import _build, _check, _run  # noqa: E402


@pytest.mark.parametrize("qh,kvh", [(8, 2), (2, 2), (3, 1), (8, 1), (12, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_chunk_among_single_tokens(qh, kvh, d):
    """Few rows a sequence on average, but one has many."""
    news = [1] * 40 + [130] + [1] * 40 + [0] * 40 + [2]
    lens = [30 + 7 * i % 400 for i in range(40)] + [333] + [5 + 11 * i for i in range(40)] + [64] * 40 + [4000]
    s = _build(lens, news, qh, kvh, d, 16, torch.bfloat16)
    _check(s, _run(s))


@pytest.mark.parametrize("d", [64, 128])
def test_a_single_token_among_chunks(d):
    s = _build([90, 3000, 17, 500, 0], [40, 1, 17, 1, 0], 8, 2, d, 32, torch.float16, ks=0.5, vs=3.0)
    _check(s, _run(s))


@pytest.mark.parametrize("G,n", [(1, 25), (1, 32), (2, 16), (3, 9), (4, 7), (4, 8), (5, 5), (5, 6), (9, 3), (13, 2), (16, 2), (28, 1), (8, 4)])
@pytest.mark.parametrize("d", [64, 128])
def test_around_a_tile_of_few_rows(G, n, d):
    s = _build([n, 129, 40, 700, 64 + n], [n, n, 0, n, n], 2 * G, 2, d, 16, torch.bfloat16)
    _check(s, _run(s))
    s = _build([n, 129, 700, 64 + n], [n, n, n, n], 2 * G, 2, d, 64, torch.float16)
    _check(s, _run(s))


@pytest.mark.parametrize("G,n", [(128, 1), (100, 1), (64, 2), (33, 3), (5, 24), (1, 128), (1, 100), (3, 86), (128, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_around_one_row_tile(G, n, d):
    """Items of one row tile, long ones cut between blocks, and the first that have two."""
    s = _build([3000, 77 + n, 640, n], [n] * 4, G, 1, d, 32, torch.bfloat16, seed=G)
    _check(s, _run(s))
    s = _build([300, 77 + n, 1, 2500], [n, 0, 1, 2 * n - 1], 2 * G, 2, d, 16, torch.float16, ks=2.0, vs=0.5, seed=n)
    _check(s, _run(s))


@pytest.mark.parametrize("G", [25, 33, 49, 100, 127, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_large_groups_of_heads(G, d, dtype):
    s = _build([40, 1, 150, 300], [3, 1, 9, 1], 2 * G, 2, d, 32, dtype)
    _check(s, _run(s))


def test_calls_on_several_streams_at_once():
    cases = [_build([9000, 300, 40], [1, 2, 1], 8, 2, 128, 16, torch.bfloat16, seed=1),
             _build([3000, 300, 400], [60, 17, 40], 8, 2, 128, 64, torch.bfloat16, seed=2),
             _build([3000, 700], [1, 1], 4, 4, 64, 32, torch.float16, seed=3)]
    want = [_run(s) for s in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[] for _ in cases]
    for _ in range(5):
        for i, s in enumerate(cases):
            got[i].append(_run(s, stream=streams[i]))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)
    for s, w in zip(cases, want):
        _check(s, w)


@pytest.mark.parametrize("n", [1, 30])
def test_captured_rounds_follow_lengths_on_the_device(n):
    """One graph of an append and the attention, replayed while lengths, slots, positions and inputs change; a second graph that
    shares the workspace is replayed in between."""
    from paper_2511_13732_b200 import binding

    B, qh, kvh, d, bs, ks = 3, 8, 2, 128, 16, 0.5
    gen = torch.Generator(device="cuda").manual_seed(n)
    max_blocks = 24
    table = torch.randperm(B * max_blocks, generator=gen, device="cuda").to(torch.int32).view(B, max_blocks)
    cache = torch.full(binding.pcg_fourbit_cache_shape(B * max_blocks, kvh, bs, d), 0x7F, dtype=torch.uint8, device="cuda")
    tab = R.table(400, d).cuda()
    rows = B * n
    fused = torch.zeros(rows, qh + 2 * kvh, d, dtype=torch.bfloat16, device="cuda")
    q, k, v = fused[:, :qh], fused[:, qh:qh + kvh], fused[:, qh + kvh:]
    slots, positions = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    start = torch.arange(0, rows + 1, n, dtype=torch.int32, device="cuda")
    kv_len = torch.full((B,), n, dtype=torch.int32, device="cuda")
    ws = torch.empty(binding.pcg_attention_workspace_bytes(B, qh, kvh, d, 1), dtype=torch.uint8, device="cuda")
    q_out = torch.empty(rows, qh, d, dtype=torch.bfloat16, device="cuda")
    out, other = torch.empty_like(q_out), _build([500, 40, 77], [17, 5, 1], qh, kvh, d, 32, torch.bfloat16)
    other_out = torch.empty_like(other["q"])

    def go():
        binding.pcg_cache_append_fourbit(q, k, v, slots, cache, positions=positions, table=tab, k_scale=ks, q_out=q_out)
        binding.pcg_cache_attention_fourbit(q_out, start, kv_len, table, cache, k_scale=ks, out=out, workspace=ws)

    want_other = _run(other)
    slots.fill_(-1)
    go()
    _run(other, out=other_out, workspace=ws)
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    with torch.cuda.graph(second):
        _run(other, out=other_out, workspace=ws)
    held = [0, 5, 40]
    for b, L in enumerate(held):  # what is there before
        p = torch.arange(L, device="cuda")
        x = torch.randn(L, kvh, d, generator=gen, device="cuda")
        if L:
            binding.pcg_cache_append_fourbit(None, x, x, (table[b].long()[p // bs] * bs + p % bs).int(), cache, k_scale=ks)
    for turn in range(4):
        fused.copy_(torch.randn(fused.shape, generator=gen, device="cuda"))
        p = torch.cat([torch.arange(L, L + n, device="cuda") for L in held])
        slots.copy_(table.long().repeat_interleave(n, 0)[torch.arange(rows, device="cuda"), p // bs] * bs + p % bs)
        positions.copy_(p)
        held = [L + n for L in held]
        kv_len.copy_(torch.tensor(held))
        graph.replay()
        other_out.zero_()
        second.replay()
        R.check_turned(q_out, q, positions, tab, False)
        at = [table[b].long()[torch.arange(L, device="cuda") // bs] * bs + torch.arange(L, device="cuda") % bs for b, L in enumerate(held)]
        _check(dict(q=q_out, start=start, cache=cache, slots=at, lens=held, news=[n] * B, ks=ks, vs=1.0), out)
        assert torch.equal(other_out, want_other)


def test_the_order_of_the_batch():
    """A sequence's result does not depend on what stands beside it, nor on the order of the batch, beyond the rounding of
    sums that are cut elsewhere: each against the formula."""
    lens, news = [700, 33, 129, 2500, 64], [5, 3, 17, 2, 1]
    s = _build(lens, news, 8, 2, 128, 16, torch.bfloat16)
    _check(s, _run(s))
    order = [3, 0, 4, 2, 1]
    start = s["start"].tolist()
    t = dict(s, q=torch.cat([s["q"][start[b]:start[b + 1]] for b in order]), lens=[lens[b] for b in order], news=[news[b] for b in order],
             slots=[s["slots"][b] for b in order], kv_len=s["kv_len"][order], table=s["table"][order].contiguous())
    t["start"] = torch.tensor([0] + [news[b] for b in order]).cumsum(0).int().cuda()
    _check(t, _run(t))
