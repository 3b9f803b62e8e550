"""Calls on a given stream that is not the current one: whose memory they use, and until when."""
import pytest

from paper_2511_13732_b200 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture
def recorder(monkeypatch):
    from gpu_util import Recorder
    from paper_2511_13732_b200 import binding

    r = Recorder(binding.load())
    monkeypatch.setattr(binding, "_lib", r)
    return r


class Calls:
    """One call of each kind, on tensors of its own.  `own`: the argument of the library's call that holds the buffer which
    the binding allocates for itself, or the first output."""

    own = dict(verify=13, thinning=16, group_probs=5, plan=12, cache_attention=12, prompt_attention=15)

    def __init__(self, name):
        from gpu_util import logits_to_device, make_handle

        self.name = name
        if name in ("verify", "thinning", "group_probs"):
            cfg = W.scaled(W.CONFIGS["C1"], V=2000, M=100, B=4, K=4)
            bt = W.make_batch(cfg)
            self.handle = make_handle(W.make_groups(cfg))
            t = dict(target=logits_to_device(bt.target_logits), draft=logits_to_device(bt.draft_logits),
                     tokens=torch.from_numpy(bt.draft_tokens).cuda(), uniforms=torch.from_numpy(bt.uniforms).cuda())
            if name == "thinning":
                t["thin"] = torch.rand((4, 9, 3), device="cuda")
            if name == "group_probs":
                t = dict(logits=t["target"][0].clone())
        else:
            g = torch.Generator(device="cuda").manual_seed(1)
            rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
            t = dict(q=rnd(70, 8, 64), k=rnd(70, 2, 64), v=rnd(70, 2, 64), start=_ints([0, 30, 70]), kv_len=_ints([300, 90]),
                     table=_ints([[0, 1, 2, 3, 4], [6, 5, 7, 8, 9]]), kc=rnd(10, 2, 64, 64), vc=rnd(10, 2, 64, 64),
                     cached=_ints([270, 50]), new=_ints([30, 40]), held=_ints([5, 1]), ring=_ints(list(range(10))),
                     state=_ints([0, 4]), slots=_ints(list(range(70))))
            names = dict(plan="cached new held table ring state", append="k v slots kc vc", cache_attention="q start kv_len table kc vc",
                         prompt_attention="q k v start")
            t = {n: t[n] for n in names[name].split()}
        self.tensors = t

    def __call__(self, **kw):
        from paper_2511_13732_b200 import binding

        t = list(self.tensors.values())
        if self.name == "verify":
            return binding.pcg_verify(*t[:3], self.handle, *t[3:], **kw)
        if self.name == "thinning":
            return binding.pcg_verify_thinning(*t[:3], self.handle, *t[3:], **kw)
        if self.name == "group_probs":
            return binding.pcg_group_probs(*t, self.handle, **kw)
        if self.name == "plan":
            return binding.pcg_cache_plan(*t, 64, 70, **kw)
        return getattr(binding, "pcg_" + ("cache_append" if self.name == "append" else self.name))(*t, **kw)


@pytest.mark.parametrize("name", list(Calls.own))
def test_two_given_streams_get_buffers_of_their_own(name, recorder):
    """Neither another stream's call nor the current stream's next tensor is given a buffer that a call's stream has yet to
    use.  (Nothing is launched.)"""
    call = Calls(name)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    at = []
    for s in streams:
        call(stream=s)
        at.append(recorder.calls[-1][Calls.own[name]])
    call()  # on the current stream
    at.append(recorder.calls[-1][Calls.own[name]])
    assert len(set(at)) == 3


@pytest.mark.parametrize("name", list(Calls.own) + ["append"])
def test_tensors_of_a_call_are_kept_until_its_stream_is_done(name, recorder):
    """A caller may drop its tensors when the call returns, as it may on the current stream.  (Nothing is launched but a
    delay on the call's stream.)"""
    call = Calls(name)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)  # half a second
    call(stream=side)
    for n in list(call.tensors):
        t = call.tensors.pop(n)
        at, shape, dtype = t.data_ptr(), t.shape, t.dtype
        del t
        assert torch.empty(shape, dtype=dtype, device="cuda").data_ptr() != at, n
    assert not side.query()  # the delay had not ended meanwhile
    side.synchronize()


@pytest.mark.parametrize("name", ["cache_attention", "prompt_attention", "verify"])
def test_calls_on_two_given_streams_do_not_disturb_each_other(name):
    calls = [Calls(name) for _ in range(2)]
    for x in calls[1].tensors.values():
        if x.is_floating_point() and x.dim() > 2 and name != "verify":
            x.mul_(0.5)
    first = [c() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, c in enumerate(calls):
            got[i].append(c(stream=streams[i]))
            torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda")  # the current stream goes on meanwhile
    torch.cuda.synchronize()
    for want, outs in zip(first, got):
        for o in outs:
            for a, b in zip(want if isinstance(want, tuple) else [want], o if isinstance(o, tuple) else [o]):
                assert torch.equal(a, b)


# ---- decoding rounds ---------------------------------------------------------------------------------------------------
def test_a_round_ends_behind_the_stream_that_it_ran_on(recorder):
    """Nothing is launched but a delay on the round's stream, which the end of the round has to wait for."""
    from paper_2511_13732_b200.rounds import DecodeRounds

    state = DecodeRounds(2, 1, 8, 16, 1, 64, 4)
    side = torch.cuda.Stream()
    state.begin(_ints([3, 4]), 7)
    state.keep_all()  # loads the kernels of torch that it uses
    new = _ints([3, 4])
    torch.cuda.synchronize()
    state.begin(new, 7, stream=side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)  # half a second
    state.keep_all()
    end = torch.cuda.Event()
    end.record()
    while not end.query() and not side.query():
        pass
    assert side.query()
    side.synchronize()


@pytest.mark.parametrize("plan", ["one stream", "streams in turn"])
def test_rounds_on_given_streams_follow_rounds_on_the_current_one(plan):
    from gpu_util import logits_to_device, make_handle
    from paper_2511_13732_b200.rounds import DecodeRounds

    B, K, V = 4, 4, 2000
    cfg = W.scaled(W.CONFIGS["C1"], V=V, M=100, B=B, K=K)
    bt, handle = W.make_batch(cfg), make_handle(W.make_groups(cfg))
    target, draft = logits_to_device(bt.target_logits), logits_to_device(bt.draft_logits)
    tokens = torch.from_numpy(bt.draft_tokens).cuda()
    g = torch.Generator(device="cuda").manual_seed(5)
    sides = [torch.cuda.Stream() for _ in range(2)]
    pick = iter(range(10 ** 6))

    def stream(on):
        """A stream for the next call, which starts late."""
        if not on:
            return None
        s = sides[0] if plan == "one stream" else [sides[0], None, sides[1]][next(pick) % 3]
        with torch.cuda.stream(s):
            torch.cuda._sleep(4_000_000)
        return s

    states = [DecodeRounds(B, 2, 60, 16, 2, 64, 12) for _ in range(2)]
    lens = _ints([40, 7, 1, 90])
    rows = [torch.randn((n, 8, 64), generator=g, device="cuda").bfloat16() for n in (138, 138, 20, 20, 20, 20, 20, 20)]
    us = [torch.rand((B, K + 1, 2), generator=g, device="cuda") for _ in range(3)]
    drafts = _ints([K + 1] * B)
    torch.cuda.synchronize()
    got = []
    for on, state in enumerate(states):
        outs = []

        def round_(new_len, n, qs):
            p = state.begin(new_len, n, stream=stream(on))
            return [*p] + [state.attend(i, q, q[:, :2], q[:, 2:4], stream=stream(on)) for i, q in enumerate(qs)]

        outs += round_(lens, 138, rows[:2])
        state.keep_all(stream=stream(on))
        for r in range(3):
            outs += round_(drafts, 20, rows[2 + 2 * r: 4 + 2 * r])
            outs += state.verify(target, draft, tokens, handle, us[r], stream=stream(on))
        outs += round_(drafts, 20, rows[2:4])
        got.append(outs)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.equal(a, b), i
    assert got[0][-10].tolist() != [40, 7, 1, 90]  # (the cached lengths of the last round)


@pytest.mark.parametrize("given", [False, True])
def test_the_attention_of_a_round_is_captured_and_replayed(given):
    """The layers of a round in a graph (on the capturing stream, or on one forked from it), between eager begins and ends."""
    from paper_2511_13732_b200.rounds import DecodeRounds

    g = torch.Generator(device="cuda").manual_seed(8)
    lens = [_ints([40, 7, 30]), _ints([5, 5, 5])]
    q = [torch.randn((n, 8, 64), generator=g, device="cuda").bfloat16() for n in (77, 15)]
    side = torch.cuda.Stream()
    got = []
    for captured in (False, True):
        state, outs = DecodeRounds(3, 2, 30, 16, 2, 64, 8), []
        for i in range(2):
            state.begin(lens[i], q[i].shape[0])
            out = [torch.empty_like(q[i]) for _ in range(2)]

            def layers(stream=None):
                for layer in range(2):
                    state.attend(layer, q[i], q[i][:, :2], q[i][:, 2:4], out=out[layer], stream=stream)

            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    if given:
                        side.wait_stream(torch.cuda.current_stream())
                    layers(side if given else None)
                    if given:
                        torch.cuda.current_stream().wait_stream(side)
                graph.replay()
            else:
                layers()
            outs += [o.clone() for o in out]
            state.keep_all()
        outs += [*state.begin(lens[1], 15)]
        got.append(outs)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.equal(a, b), i
