"""Decoding rounds with positions and with a cache of 4 bits, against a model that keeps every sequence's tokens in a list,
turns and quantises them in float32 steps and attends in 64 bits."""
import random

import pytest

from paper_2511_13732_b200 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import cache_ref  # noqa: E402
import fourbit_ref as R  # noqa: E402


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _held(x, g):
    code, s8 = R.quantise32(x.float().cpu(), g)
    magnitude = torch.tensor(R.E2M1)[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
    return (magnitude.unflatten(-1, (-1, 16)) * s8.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2).double().cuda() * g


CASES = [
    # (dtype, q_heads, kv_heads, d, turned dimensions or 0, interleaved, fourbit, block_size)
    (torch.bfloat16, 8, 2, 128, 128, False, False, 32),
    (torch.float16, 6, 2, 64, 32, True, False, 16),
    (torch.bfloat16, 8, 2, 128, 128, False, True, 64),
    (torch.float16, 4, 4, 64, 64, True, True, 16),
    (torch.float32, 6, 2, 96, 64, False, True, 32),
    (torch.bfloat16, 4, 1, 64, 0, False, True, 16),
]


@pytest.mark.parametrize("dtype,qh,kvh,d,dim,inter,four,bs", CASES)
def test_rounds_follow_the_tokens(dtype, qh, kvh, d, dim, inter, four, bs):
    from gpu_util import make_handle
    from paper_2511_13732_b200.rounds import DecodeRounds

    V, M, B, K, layers, ks, vs = 512, 64, 5, 4, 2, 0.5, 0.375
    rng = random.Random(5)
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cfg = W.scaled(W.CONFIGS["C1"], V=V, M=M, B=B, K=K)
    handle = make_handle(W.make_groups(cfg))
    embed = rnd(V, 96)
    made = [(embed @ (rnd(96, (qh + 2 * kvh) * d) * 0.15)).view(-1, qh + 2 * kvh, d).to(dtype) for _ in range(layers)]
    head = rnd(qh * d, V)
    tab = R.table(400, dim).cuda() if dim else None
    kw = dict(fourbit=True, k_scale=ks, v_scale=vs) if four else {}
    state = DecodeRounds(B, layers, 90, bs, kvh, d, 24, dtype=dtype, rotary=tab, interleaved=inter, **kw)
    if four:
        state.cache.fill_(0x7F)
    else:
        state.k_cache.fill_(float("nan")), state.v_cache.fill_(float("nan"))
    kept = [[] for _ in range(B)]

    def project(tokens, layer):
        x = made[layer][torch.tensor(tokens, device="cuda")]
        return x[:, :qh], x[:, qh:qh + kvh], x[:, qh + kvh:]

    def run(chunks, fresh=False):
        rows = [t for c in chunks for t in c]
        plan = state.begin(_ints([len(c) for c in chunks]), len(rows) + 3)
        assert plan.flags.tolist() == [0] * B
        start = plan.row_start.tolist()
        for layer in range(layers):
            q, k, v = project(rows + [0, 0, 0], layer)
            out = state.attend(layer, q, k, v, fresh=fresh)
            for b, c in enumerate(chunks):
                if not c:
                    continue
                tokens, n = kept[b] + c, len(kept[b])
                qq, kk, vv = project(tokens, layer)
                if dim:
                    at = torch.arange(len(tokens), device="cuda")
                    qq = R.turn32(qq, at, tab, inter).to(dtype)
                    kk = R.turn32(kk, at, tab, inter)
                if four:
                    kk, vv = _held(kk, ks), _held(vv, vs)
                    if fresh:
                        kk, vv = kk.to(dtype), vv.to(dtype)
                else:
                    kk = kk.to(dtype)
                lim = [n + i + 1 for i in range(len(c))]
                R.check_attention(out[start[b]:start[b + 1]], cache_ref.attention(qq[n:], kk, vv, lim, d ** -0.5), dtype, d, lim[-1], (b, layer))
        return out

    prompts = [[rng.randrange(V) for _ in range(rng.randint(1, 150))] for _ in range(B)]
    run(prompts, fresh=True)
    state.keep_all()
    kept = [list(p) for p in prompts]
    token = [p[-1] for p in prompts]
    for r in range(3):
        drafts = [[rng.randrange(V) for _ in range(K)] for _ in range(B)]
        out = run([[token[b]] + drafts[b] for b in range(B)])
        target = (out[: B * (K + 1)].float().reshape(B, K + 1, -1) @ head).contiguous()
        draft = target[:, :K].clone() if r % 2 else target[:, :K] + 0.5 * rnd(B, K, V)
        uniforms = torch.rand((B, K + 1, 2), generator=g, device="cuda")
        n, tokens, _, _ = state.verify(target, draft.contiguous(), _ints(drafts), handle, uniforms)
        n, tokens = n.tolist(), tokens.tolist()
        for b in range(B):
            kept[b] = kept[b] + [token[b]] + drafts[b][: n[b]]
            token[b] = tokens[b][n[b]]
    # a chunk of a prompt behind what is cached, and single tokens
    run([[rng.randrange(V) for _ in range(60 if b == 2 else 1)] for b in range(B)])


@pytest.mark.parametrize("four", [False, True])
def test_a_round_on_a_given_stream(four):
    from paper_2511_13732_b200.rounds import DecodeRounds

    tab = R.table(100, 64).cuda()
    q, k, v = (torch.randn(20, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    results = []
    for side in (None, torch.cuda.Stream()):
        s = DecodeRounds(2, 1, 8, 16, 2, 64, 4, rotary=tab, fourbit=four)
        lens = _ints([15, 5])
        if side is not None:
            side.wait_stream(torch.cuda.current_stream())
        s.begin(lens, 20, stream=side)
        results.append(s.attend(0, q, k, v, fresh=True, stream=side))
        s.keep_all(stream=side)
        s.begin(_ints([1, 3]), 4)
        results.append(s.attend(0, q[:4], k[:4], v[:4]))
        torch.cuda.synchronize()
    assert torch.equal(results[0], results[2]) and torch.equal(results[1], results[3])
