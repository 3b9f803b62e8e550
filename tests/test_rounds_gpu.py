"""Decoding rounds end to end: plan, append, attention and verification of a small model, against a model that keeps
every sequence's tokens in a list and attends in 64 bits."""
import random

import numpy as np
import pytest

from paper_2511_13732_b200 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,qh,kvh,d,bs", [(torch.bfloat16, 8, 2, 64, 16), (torch.float16, 4, 4, 128, 32), (torch.float32, 6, 2, 64, 16)])
def test_rounds_follow_the_tokens(dtype, qh, kvh, d, bs):
    from gpu_util import make_handle
    from paper_2511_13732_b200.rounds import DecodeRounds
    import cache_ref

    V, M, B, K, layers = 512, 64, 6, 4, 2
    rng = random.Random(5)
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cfg = W.scaled(W.CONFIGS["C1"], V=V, M=M, B=B, K=K)
    handle = make_handle(W.make_groups(cfg))
    width = (qh + 2 * kvh) * d
    embed = rnd(V, 96)
    weight = [rnd(96, width) * 0.15 for _ in range(layers)]
    head = rnd(qh * d, V)
    state = DecodeRounds(B, layers, 90, bs, kvh, d, 24, dtype=dtype)
    state.k_cache.fill_(float("nan")), state.v_cache.fill_(float("nan"))  # as fresh memory may be
    kept = [[] for _ in range(B)]  # committed tokens of each sequence

    def project(tokens, layer):
        x = embed[torch.tensor(tokens, device="cuda")] @ weight[layer]
        x = x.view(-1, qh + 2 * kvh, d).to(dtype)
        return x[:, :qh], x[:, qh:qh + kvh], x[:, qh + kvh:]

    def run(chunks, fresh=False):
        """The round's attention outputs of the last layer, checked layer by layer against the kept lists."""
        rows = [t for c in chunks for t in c]
        plan = state.begin(_ints([len(c) if c is not None else -1 for c in chunks]), len(rows) + 3)
        assert plan.flags.tolist() == [0] * B
        start = plan.row_start.tolist()
        positions = plan.positions.tolist()
        for b, c in enumerate(chunks):
            assert positions[start[b]:start[b + 1]] == list(range(len(kept[b]), len(kept[b]) + len(c)))
        padded = rows + [0, 0, 0]
        for layer in range(layers):
            q, k, v = project(padded, layer)
            out = state.attend(layer, q, k, v, fresh=fresh)
            for b, c in enumerate(chunks):
                if not c:
                    continue
                _, ck, cv = project(kept[b] + c, layer)
                lim = [len(kept[b]) + i + 1 for i in range(len(c))]
                at = slice(start[b], start[b + 1])
                cache_ref.check(out[at], cache_ref.attention(q[at], ck, cv, lim, d ** -0.5), dtype, d, lim[-1], (b, layer))
        return out, start

    prompts = [[rng.randrange(V) for _ in range(rng.randint(1, 150))] for _ in range(B)]
    run(prompts, fresh=True)
    state.keep_all()
    kept = [list(p) for p in prompts]
    run([[rng.randrange(V)] if b % 2 else [] for b in range(B)][:B])  # single tokens for some, nothing for the others
    last = [c for c in state.plan.row_start.tolist()]
    assert last[-1] == B // 2
    # what that round fed is dropped again: verification of nothing
    state._end(torch.full((B,), -1, dtype=torch.int32, device="cuda"))
    token = [p[-1] for p in prompts]
    accepted = []
    for r in range(5):
        drafts = [[rng.randrange(V) for _ in range(K)] for _ in range(B)]
        out, start = run([[token[b]] + drafts[b] for b in range(B)])
        target = (out[: B * (K + 1)].float().reshape(B, K + 1, -1) @ head).contiguous()
        draft = target[:, :K] + 0.5 * rnd(B, K, V)
        if r % 2:
            draft = target[:, :K].clone()  # all drafts are accepted
        uniforms = torch.rand((B, K + 1, 2), generator=g, device="cuda")
        n, tokens, _, flags = state.verify(target, draft.contiguous(), _ints(drafts), handle, uniforms)
        n, tokens = n.tolist(), tokens.tolist()
        accepted += n
        for b in range(B):
            kept[b] = kept[b] + [token[b]] + drafts[b][: n[b]]
            token[b] = tokens[b][n[b]]
    assert max(accepted) == K and min(accepted) < K
    # two sequences finish, a third is given the blocks
    plan = state.begin(_ints([-1, -1] + [0] * (B - 2)), 4)
    assert plan.held.tolist()[:2] == [0, 0] and plan.kv_len.tolist()[:2] == [0, 0]
    state.keep_all()
    kept[0], kept[1] = [], []
    fresh = [rng.randrange(V) for _ in range(70)]
    run([fresh, [], [token[2]], [], [], []])


def test_rounds_refuse_calls_out_of_order():
    from paper_2511_13732_b200.rounds import DecodeRounds

    s = DecodeRounds(2, 1, 8, 16, 1, 64, 4)
    with pytest.raises(RuntimeError):
        s.attend(0, None, None, None)
    with pytest.raises(RuntimeError):
        s.keep_all()
    s.begin(_ints([1, 1]), 2)
    with pytest.raises(RuntimeError):
        s.begin(_ints([1, 1]), 2)
    with pytest.raises(ValueError):
        DecodeRounds(0, 1, 8, 16, 1, 64, 4)


def test_a_sequence_without_blocks_waits_for_a_later_round():
    from paper_2511_13732_b200 import binding
    from paper_2511_13732_b200.rounds import DecodeRounds

    s = DecodeRounds(3, 1, 4, 16, 2, 64, 4)
    q = torch.randn(80, 4, 64, device="cuda").bfloat16()
    kv = torch.randn(2, 80, 2, 64, device="cuda").bfloat16()
    plan = s.begin(_ints([20, 40, 10]), 80)
    assert plan.flags.tolist() == [0, binding.FLAG_NO_BLOCKS, binding.FLAG_NO_BLOCKS]
    out = s.attend(0, q, kv[0], kv[1], out=torch.full_like(q, 5.0))
    assert not out[20:70].any() and bool((out[70:] == 5).all()) and bool(torch.isfinite(out[:20]).all())
    s.keep_all()
    plan = s.begin(_ints([-1, 40, 10]), 80)  # the first has finished: its blocks are free in the next round
    assert plan.flags.tolist() == [0, binding.FLAG_NO_BLOCKS, binding.FLAG_NO_BLOCKS] and plan.cached_len.tolist() == [0, 0, 0]
    s.keep_all()
    plan = s.begin(_ints([0, 40, 10]), 80)
    assert plan.flags.tolist() == [0, 0, 0] and plan.kv_len.tolist() == [0, 40, 10]


def test_a_captured_round_replays():
    """Plan, append and attention of one round in a graph, replayed with other lengths and rows in the same buffers."""
    from paper_2511_13732_b200 import binding
    import cache_ref

    B, bs, rows = 3, 16, 12
    kc, vc = (torch.zeros((40, 2, bs, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cached, accept, new, held = _ints([100, 30, 0]), _ints([1, 3, -1]), _ints([4, 4, 4]), _ints([8, 4, 0])
    table = torch.full((B, 12), -1, dtype=torch.int32, device="cuda")
    table[0, :8], table[1, :4] = torch.arange(8), torch.arange(8, 12)
    ring, state = torch.arange(40, dtype=torch.int32, device="cuda"), _ints([12, 28])
    q, k, v = (torch.randn((rows, h, 64), device="cuda").bfloat16() for h in (4, 2, 2))
    ws = torch.empty(binding.pcg_attention_workspace_bytes(B, 4, 2, 64, binding.PCG_BF16), dtype=torch.uint8, device="cuda")

    def step(plan=None, out=None):
        plan = binding.pcg_cache_plan(cached, new, held, table, ring, state, bs, rows, accept_len=accept, out=plan)
        binding.pcg_cache_append(k, v, plan.slots, kc, vc)
        return plan, binding.pcg_cache_attention(q, plan.row_start, plan.kv_len, table, kc, vc, out=out, workspace=ws)

    plan, out = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(plan, out)
    for lens in ([100, 30, 0], [90, 33, 0], [60, 45, 0]):
        kc.normal_(), vc.normal_(), q.normal_(), k.normal_(), v.normal_()
        cached.copy_(_ints(lens))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        kv = plan.kv_len.tolist()
        assert kv == [lens[0] + 6, lens[1] + 8, lens[2] + 4]
        t = table.tolist()
        for b in range(B):
            at = slice(4 * b, 4 * b + 4)
            keys, values = (torch.cat([c[j].transpose(0, 1) for j in t[b][: -(-kv[b] // bs)]])[: kv[b]] for c in (kc, vc))
            assert torch.equal(keys[-4:], k[at]) and torch.equal(values[-4:], v[at])
            lim = [kv[b] - 3 + i for i in range(4)]
            cache_ref.check(out[at], cache_ref.attention(q[at], keys, values, lim, 0.125), torch.bfloat16, 64, kv[b])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_prompt_joins_a_round_of_drafts(dtype):
    """A prompt, a short prompt, a single token and full drafts in one round, whose cache the next rounds attend over.
    Slots that hold nothing that stays are NaN."""
    from gpu_util import make_handle
    from paper_2511_13732_b200.rounds import DecodeRounds
    import cache_ref

    V, B, K, qh, kvh, d = 512, 5, 4, 4, 2, 64
    handle = make_handle(W.make_groups(W.scaled(W.CONFIGS["C1"], V=V, M=64, B=B, K=K)))
    g = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    state = DecodeRounds(B, 1, 80, 16, kvh, d, 24, dtype=dtype)
    state.k_cache.fill_(float("nan")), state.v_cache.fill_(float("nan"))
    kept = [[torch.empty((0, kvh, d), dtype=dtype, device="cuda")] * 2 for _ in range(B)]

    def run(lens):
        """Checks the round against what was kept of the rounds before; its keys and values."""
        n = sum(lens)
        q, k, v = (rnd(n, h, d).to(dtype) for h in (qh, kvh, kvh))
        plan = state.begin(_ints(lens), n)
        assert plan.flags.tolist() == [0] * B and plan.cached_len.tolist() == [x[0].shape[0] for x in kept]
        out = state.attend(0, q, k, v)
        parts = []
        for b, (lo, hi) in enumerate(zip(plan.row_start.tolist(), plan.row_start.tolist()[1:])):
            kv = [torch.cat([old, new[lo:hi]]) for old, new in zip(kept[b], (k, v))]
            parts.append(kv)
            lim = [kept[b][0].shape[0] + i + 1 for i in range(hi - lo)]
            if lim:
                cache_ref.check(out[lo:hi], cache_ref.attention(q[lo:hi], *kv, lim, d ** -0.5), dtype, d, lim[-1], b)
        return parts

    def verify(lens, parts, whole, all_accepted):
        target = rnd(B, K + 1, V)
        draft = target[:, :K].clone() if all_accepted else rnd(B, K, V)
        mask = torch.tensor(whole, device="cuda") if any(whole) else None
        accept = state.verify(target, draft, torch.randint(0, V, (B, K), generator=g, device="cuda").to(torch.int32), handle,
                              torch.rand((B, K + 1, 2), generator=g, device="cuda"), whole=mask)[0].tolist()
        assert not all_accepted or accept == [K] * B
        for b, n in enumerate(lens):
            m = n if whole[b] or n > K + 1 else min(accept[b] + 1, n)
            kept[b] = [x[: kept[b][0].shape[0] + m] for x in parts[b]]

    for lens, whole, all_accepted in (([40, 3, 5, 5, 70], [True, True, False, False, False], True), ([5, 1, 130, 2, 5], [False] * 5, True),
                                      ([5, 5, 5, 3, 0], [False, False, False, True, False], False), ([5, 5, 1, 5, 9], [False] * 5, False),
                                      ([5] * 5, [False] * 5, True)):
        verify(lens, run(lens), whole, all_accepted)
