"""What the binding of the calls that rotate by position and of those on the cache of 4 bits refuses of CUDA tensors.  It
hands raw addresses to the kernels, so a tensor that is too short, of another type or elsewhere has to be refused here.  The
library is replaced by one that launches nothing: a check that is missing shows as a call that goes through."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _rows(n, heads, d=64, dtype=torch.bfloat16):
    return torch.zeros((n, heads, d), dtype=dtype, device="cuda")


def _cache(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


def _bytes(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device="cuda")


@pytest.fixture
def recorder(monkeypatch):
    from gpu_util import Recorder
    from paper_2511_13732_b200 import binding

    r = Recorder(binding.load())
    monkeypatch.setattr(binding, "_lib", r)
    return r


def _turned():
    return dict(q=_rows(3, 4), k=_rows(3, 2), v=_rows(3, 2), slots=_ints(3), positions=_ints(3), table=torch.zeros(9, 32, device="cuda"))


def _rotary_args():
    return dict(_turned(), k_cache=_cache(4, 2, 16, 64), v_cache=_cache(4, 2, 16, 64), q_out=_rows(3, 4), k_out=_rows(3, 2))


def _fourbit_args():
    return dict(_turned(), cache=_bytes(4, 2, 1, 18 * 64), q_out=_rows(3, 4), k_out=_rows(3, 2), v_out=_rows(3, 2))


def _attention_args():
    return dict(q=_rows(3, 4), row_start=_ints(3), kv_len=_ints(2), block_table=_ints(2, 8), cache=_bytes(4, 2, 1, 18 * 64),
                out=_rows(3, 4), workspace=_bytes(1 << 20))


def _calls():
    from paper_2511_13732_b200 import binding

    return dict(rotary=(_rotary_args, binding.pcg_cache_append_rotary), fourbit=(_fourbit_args, binding.pcg_cache_append_fourbit),
                attention=(_attention_args, binding.pcg_cache_attention_fourbit))


INTS, CACHES, TABLE = "expected a contiguous int32 tensor", "k_cache and v_cache must be contiguous", "table must be"
FOUR, HELD = "cache must be a contiguous uint8 tensor", "must be contiguous, of k's shape"
TURNED = [
    ("q", lambda t: t.cpu(), "q must be"),
    ("q", lambda t: t.float(), "q must be"),
    ("q", lambda t: t[:2], "q must have"),
    ("q", lambda t: _rows(3, 4, 32), "q must have"),
    ("q", lambda t: _rows(3, 8)[:, ::2], "heads must be dense"),
    ("q", lambda t: None, "q_out without q"),
    ("k", lambda t: t.cpu(), "current device"),
    ("k", lambda t: t[0], "k must be"),
    ("k", lambda t: _rows(3, 2, 128)[:, :, ::2], "heads must be dense"),
    ("k", lambda t: _rows(3, 1), "k and v must be"),
    ("v", lambda t: t.half(), "v must be"),
    ("v", lambda t: _rows(2, 2), "k and v must be"),
    ("slots", lambda t: t[:2], INTS),
    ("slots", lambda t: t.long(), INTS),
    ("slots", lambda t: _ints(6)[::2], INTS),
    ("positions", lambda t: t[:2], INTS),
    ("positions", lambda t: t.float(), INTS),
    ("positions", lambda t: t.cpu(), INTS),
    ("table", lambda t: t.cpu(), TABLE),
    ("table", lambda t: t.half(), TABLE),
    ("table", lambda t: t[0], TABLE),
    ("table", lambda t: t.t(), TABLE),
    ("q_out", lambda t: t[:2], "q_out must be"),
    ("q_out", lambda t: t.float(), "q_out must be"),
    ("q_out", lambda t: _rows(3, 8)[:, ::2], "heads must be dense"),
    ("k_out", lambda t: t[:2], "must be"),
    ("k_out", lambda t: t.float(), "must be"),
    ("k_out", lambda t: t.cpu(), "must be"),
]
OF_FOUR = [
    ("cache", lambda t: t.cpu(), FOUR),
    ("cache", lambda t: t.to(torch.int8), FOUR),
    ("cache", lambda t: t[0], FOUR),
    ("cache", lambda t: _bytes(4, 2, 2, 18 * 64)[:, :, ::2], FOUR),
    ("cache", lambda t: _bytes(4, 2, 1, 18 * 64 + 1), FOUR),
]
BAD = ([("rotary", *bad) for bad in TURNED] + [("fourbit", *bad) for bad in TURNED + OF_FOUR] + [("attention", *bad) for bad in OF_FOUR] + [
    ("rotary", "k", lambda t: t.float(), "k must be"),
    ("rotary", "k_cache", lambda t: t[:3], CACHES),
    ("rotary", "v_cache", lambda t: t.cpu(), CACHES),
    ("fourbit", "cache", lambda t: _bytes(4, 1, 1, 18 * 64), "k and v must be"),
    ("fourbit", "cache", lambda t: _bytes(4, 2, 1, 18 * 128), "k and v must be"),
    ("fourbit", "table", lambda t: None, "go together"),
    ("fourbit", "positions", lambda t: None, "go together"),
    ("fourbit", "k_out", lambda t: _rows(3, 4)[:, :2], HELD),
    ("fourbit", "v_out", lambda t: t[:2], HELD),
    ("fourbit", "v_out", lambda t: t.half(), HELD),
    ("fourbit", "v_out", lambda t: t.cpu(), HELD),
    ("attention", "q", lambda t: t.cpu(), "current device"),
    ("attention", "q", lambda t: t[0], "q must be"),
    ("attention", "q", lambda t: _rows(3, 4, 32), "q must have the cache's head_dim"),
    ("attention", "q", lambda t: _rows(3, 8)[:, ::2], "heads must be dense"),
    ("attention", "row_start", lambda t: t[:2], INTS),
    ("attention", "row_start", lambda t: t.long(), INTS),
    ("attention", "kv_len", lambda t: _ints(3), INTS),
    ("attention", "kv_len", lambda t: t.cpu(), INTS),
    ("attention", "block_table", lambda t: t[0], "block_table be"),
    ("attention", "block_table", lambda t: _ints(2, 16)[:, ::2], INTS),
    ("attention", "block_table", lambda t: t.long(), INTS),
    ("attention", "out", lambda t: t[:2], "out must be"),
    ("attention", "out", lambda t: t.float(), "out must be"),
    ("attention", "workspace", lambda t: t.cpu(), "workspace must be"),
    ("attention", "workspace", lambda t: t[::2], "workspace must be"),
])


@pytest.mark.parametrize("call,name,change,text", BAD)
def test_a_bad_tensor_is_refused(recorder, call, name, change, text):
    make, run = _calls()[call]
    args = make()
    args[name] = change(args[name])
    with pytest.raises(ValueError, match=text):
        run(**args)
    assert recorder.calls == []


@pytest.mark.parametrize("call", ["rotary", "fourbit", "attention"])
def test_good_tensors_are_not(recorder, call):
    make, run = _calls()[call]
    run(**make())
    assert len(recorder.calls) == 1


def test_a_short_workspace_is_refused():
    from paper_2511_13732_b200 import binding

    args = _attention_args()
    args["workspace"] = args["workspace"][:64]
    with pytest.raises(binding.PcgError, match="workspace"):
        binding.pcg_cache_attention_fourbit(**args)
