"""What the binding of the cache and attention calls refuses of CUDA tensors.  It hands raw addresses to the kernels, so a
tensor that is too short, of another type or elsewhere has to be refused here.  The library is replaced by one that launches
nothing: a check that is missing shows as a call that goes through."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _rows(n, heads, d=64, dtype=torch.bfloat16):
    return torch.zeros((n, heads, d), dtype=dtype, device="cuda")


def _cache(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


@pytest.fixture
def recorder(monkeypatch):
    from gpu_util import Recorder
    from paper_2511_13732_b200 import binding

    r = Recorder(binding.load())
    monkeypatch.setattr(binding, "_lib", r)
    return r


def _append_args():
    return dict(k=_rows(3, 2), v=_rows(3, 2), slots=_ints(3), kc=_cache(4, 2, 16, 64), vc=_cache(4, 2, 16, 64))


def _attention_args():
    return dict(q=_rows(3, 4), start=_ints(3), kv=_ints(2), table=_ints(2, 8), kc=_cache(4, 2, 16, 64), vc=_cache(4, 2, 16, 64))


def _prompt_args():
    return dict(q=_rows(3, 4), k=_rows(3, 2), v=_rows(3, 2), start=_ints(3))


def _plan_args():
    return dict(cached=_ints(2), new=_ints(2), held=_ints(2), table=_ints(2, 8), ring=_ints(16), state=_ints(2))


def _calls():
    from paper_2511_13732_b200 import binding

    return dict(append=(_append_args, lambda a, **kw: binding.pcg_cache_append(*a, **kw)),
                attention=(_attention_args, lambda a, **kw: binding.pcg_cache_attention(*a, **kw)),
                prompt=(_prompt_args, lambda a, **kw: binding.pcg_prompt_attention(*a, **kw)),
                plan=(_plan_args, lambda a, **kw: binding.pcg_cache_plan(*a, 16, 4, **kw)))


INTS = "expected a contiguous int32 tensor"
CACHES = "k_cache and v_cache must be contiguous"
# (call, argument, what stands in its place, the refusal)
BAD = [
    ("append", "k", lambda t: t.cpu(), "current device"),
    ("append", "k", lambda t: t.float(), "k must be"),
    ("append", "k", lambda t: t[0], "k must be"),
    ("append", "k", lambda t: _rows(3, 2, 128)[:, :, ::2], "k: a token's heads must be dense"),
    ("append", "k", lambda t: _rows(3, 4)[:, ::2], "k: a token's heads must be dense"),
    ("append", "k", lambda t: _rows(2, 2), "k and v must be"),
    ("append", "k", lambda t: _rows(3, 1), "k and v must be"),
    ("append", "v", lambda t: t.cpu(), "v must be"),
    ("append", "v", lambda t: t.half(), "v must be"),
    ("append", "v", lambda t: _rows(2, 2), "k and v must be"),
    ("append", "v", lambda t: _rows(3, 2, 32), "k and v must be"),
    ("append", "slots", lambda t: t[:2], INTS),
    ("append", "slots", lambda t: t.long(), INTS),
    ("append", "slots", lambda t: t.cpu(), INTS),
    ("append", "slots", lambda t: _ints(6)[::2], INTS),
    ("append", "slots", lambda t: _ints(3, 1), INTS),
    ("append", "kc", lambda t: t.cpu(), CACHES),
    ("append", "kc", lambda t: t[:3], CACHES),
    ("append", "kc", lambda t: t.float(), CACHES),
    ("append", "vc", lambda t: t.cpu(), CACHES),
    ("append", "vc", lambda t: t[0], CACHES),
    ("append", "vc", lambda t: _cache(4, 16, 2, 64).transpose(1, 2), CACHES),
    ("attention", "q", lambda t: t.cpu(), "current device"),
    ("attention", "q", lambda t: t.float(), "q must be"),
    ("attention", "q", lambda t: t[0], "q must be"),
    ("attention", "q", lambda t: _rows(3, 4, 128)[:, :, ::2], "q: a token's heads must be dense"),
    ("attention", "q", lambda t: _rows(4, 3).transpose(0, 1), "q: a token's heads must be dense"),
    ("attention", "q", lambda t: _rows(3, 4, 128), "cache's head_dim"),
    ("attention", "start", lambda t: _ints(3, 1), "row_start"),
    ("attention", "start", lambda t: t[:2], INTS),
    ("attention", "start", lambda t: t.cpu(), INTS),
    ("attention", "start", lambda t: t.long(), INTS),
    ("attention", "kv", lambda t: _ints(3), INTS),
    ("attention", "kv", lambda t: t[:1], INTS),
    ("attention", "kv", lambda t: t.long(), INTS),
    ("attention", "kv", lambda t: t.cpu(), INTS),
    ("attention", "table", lambda t: _ints(3, 8), INTS),
    ("attention", "table", lambda t: _ints(2, 16)[:, ::2], INTS),
    ("attention", "table", lambda t: _ints(16), "block_table be"),
    ("attention", "table", lambda t: t.cpu(), INTS),
    ("attention", "table", lambda t: t.long(), INTS),
    ("attention", "kc", lambda t: t.transpose(1, 2), CACHES),
    ("attention", "kc", lambda t: t.cpu(), CACHES),
    ("attention", "vc", lambda t: t.float(), CACHES),
    ("attention", "vc", lambda t: t[:2], CACHES),
    ("prompt", "q", lambda t: t.cpu(), "current device"),
    ("prompt", "q", lambda t: _rows(2, 4), "with q's rows"),
    ("prompt", "q", lambda t: _rows(3, 4, 128)[:, :, ::2], "q: a token's heads must be dense"),
    ("prompt", "k", lambda t: t[:2], "with q's rows"),
    ("prompt", "k", lambda t: t.float(), "k must be"),
    ("prompt", "k", lambda t: t.cpu(), "k must be"),
    ("prompt", "k", lambda t: _rows(3, 2, 32), "with q's rows"),
    ("prompt", "v", lambda t: t[:2], "with q's rows"),
    ("prompt", "v", lambda t: _rows(3, 1), "with q's rows"),
    ("prompt", "v", lambda t: t.cpu(), "v must be"),
    ("prompt", "v", lambda t: _rows(3, 4)[:, ::2], "v: a token's heads must be dense"),
    ("prompt", "start", lambda t: t[:0], "row_start"),
    ("prompt", "start", lambda t: _ints(3, 1), "row_start"),
    ("prompt", "start", lambda t: t.long(), INTS),
    ("prompt", "start", lambda t: t.cpu(), INTS),
    ("prompt", "start", lambda t: _ints(6)[::2], INTS),
    ("plan", "cached", lambda t: t.cpu(), "current device"),
    ("plan", "cached", lambda t: _ints(3), INTS),
    ("plan", "cached", lambda t: _ints(2, 1), INTS),
    ("plan", "new", lambda t: _ints(3), INTS),
    ("plan", "new", lambda t: t.long(), INTS),
    ("plan", "new", lambda t: t.cpu(), INTS),
    ("plan", "held", lambda t: t[:1], INTS),
    ("plan", "held", lambda t: t.cpu(), INTS),
    ("plan", "table", lambda t: _ints(16), "block_table must be"),
    ("plan", "table", lambda t: _ints(3, 8), INTS),
    ("plan", "table", lambda t: _ints(2, 16)[:, ::2], INTS),
    ("plan", "table", lambda t: t.cpu(), INTS),
    ("plan", "ring", lambda t: _ints(4, 4), "free_ring"),
    ("plan", "ring", lambda t: _ints(32)[::2], INTS),
    ("plan", "ring", lambda t: t.cpu(), INTS),
    ("plan", "state", lambda t: t[:1], INTS),
    ("plan", "state", lambda t: t.cpu(), INTS),
]


@pytest.mark.parametrize("call", ["append", "attention", "prompt", "plan"])
def test_the_arguments_that_the_refusals_start_from_are_good(call, recorder):
    args, make = _calls()[call]
    make(args().values())
    assert len(recorder.calls) == 1


@pytest.mark.parametrize("call,name,bad,text", BAD, ids=[f"{c}-{n}-{i}" for i, (c, n, _, _) in enumerate(BAD)])
def test_a_tensor_of_another_shape_type_or_place_is_refused(call, name, bad, text, recorder):
    args, make = _calls()[call]
    a = args()
    a[name] = bad(a[name])
    with pytest.raises(ValueError, match=text):
        make(a.values())
    assert not recorder.calls


@pytest.mark.parametrize("call", ["attention", "prompt"])
@pytest.mark.parametrize("bad", [lambda: _rows(2, 4), lambda: _rows(3, 4, dtype=torch.float16), lambda: _rows(3, 8)[:, ::2], lambda: _rows(3, 4).cpu()])
def test_a_given_output_is_checked(call, bad, recorder):
    args, make = _calls()[call]
    with pytest.raises(ValueError, match="out must be contiguous"):
        make(args().values(), out=bad())
    assert not recorder.calls


@pytest.mark.parametrize("call", ["attention", "prompt"])
@pytest.mark.parametrize("bad", [lambda: torch.zeros(1 << 20, dtype=torch.uint8), lambda: _ints(64)[::2]])
def test_a_given_workspace_is_checked(call, bad, recorder):
    args, make = _calls()[call]
    with pytest.raises(ValueError, match="workspace must be contiguous"):
        make(args().values(), workspace=bad())
    assert not recorder.calls


@pytest.mark.parametrize("field,bad", [("cached_len", (3,)), ("kv_len", (1,)), ("held", (2, 1)), ("row_start", (2,)), ("slots", (3,)),
                                       ("positions", (5,)), ("ring_state", (1,)), ("flags", (3,))])
def test_given_outputs_of_a_plan_are_checked(field, bad, recorder):
    from paper_2511_13732_b200 import binding

    args, make = _calls()["plan"]
    out = binding.CachePlan(_ints(2), _ints(2), _ints(2), _ints(3), _ints(4), _ints(4), _ints(2), _ints(2))
    make(args().values(), out=out)
    assert len(recorder.calls) == 1
    for t in (_ints(*bad), getattr(out, field).long(), getattr(out, field).cpu()):
        with pytest.raises(ValueError, match=INTS):
            make(args().values(), out=out._replace(**{field: t}))
    with pytest.raises(ValueError, match=INTS):
        make(args().values(), accept_len=_ints(3))
    assert len(recorder.calls) == 1


def test_rows_that_repeat_one_token_are_refused():
    from paper_2511_13732_b200 import binding

    a = _prompt_args()
    for name in ("q", "k", "v"):
        with pytest.raises(binding.PcgError, match="stride"):
            binding.pcg_prompt_attention(*dict(a, **{name: a[name][:1].expand(3, -1, -1)}).values())
