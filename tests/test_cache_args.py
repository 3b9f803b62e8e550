"""What the cache's and the attention's entry points refuse, before anything is launched (no GPU is needed)."""
import ctypes

import pytest

from paper_2511_13732_b200 import binding

P = 4096  # stands for an aligned device address: nothing below gets as far as looking at it
INVALID, UNSUPPORTED, WORKSPACE = 1, 3, 4


def _cache(**kw):
    f = dict(n_blocks=8, block_size=16, kv_heads=2, head_dim=64, dtype=1, k=P, v=P)
    f.update(kw)
    return binding._Cache(*f.values())


BAD_CACHES = [dict(n_blocks=0), dict(block_size=8), dict(block_size=48), dict(block_size=512), dict(kv_heads=0), dict(kv_heads=1025),
              dict(head_dim=0), dict(head_dim=68), dict(head_dim=264), dict(dtype=3), dict(k=None), dict(v=P + 8),
              dict(n_blocks=1 << 27)]


def _plan(**kw):
    a = dict(B=4, cached=P, accept=P, new=P, held=P, bs=16, max_blocks=8, table=P, ring=P, ring_size=64, state=P, rows=20,
             o_cached=2 * P, o_kv=3 * P, o_held=4 * P, o_start=P, o_slots=P, o_pos=P, o_state=5 * P, o_flags=P, stream=None)
    a.update(kw)
    return binding.load().pcg_cache_plan(*a.values())


@pytest.mark.parametrize("bad", [dict(B=-1), dict(rows=-1), dict(ring_size=0), dict(max_blocks=0), dict(bs=24), dict(bs=8),
                                 dict(max_blocks=1 << 27), dict(cached=None), dict(new=None), dict(held=None), dict(table=None),
                                 dict(ring=None), dict(state=None), dict(o_cached=None), dict(o_kv=None), dict(o_held=None),
                                 dict(o_start=None), dict(o_slots=None), dict(o_state=None), dict(o_cached=P), dict(o_held=P),
                                 dict(o_state=P), dict(o_kv=P)])
def test_plan_refusals(bad):
    assert _plan(**bad) == INVALID
    assert "pcg_cache_plan" in binding.load().pcg_last_error().decode()


def test_plan_refuses_more_sequences_than_it_is_built_for():
    assert _plan(B=16385) == UNSUPPORTED


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_a_bad_cache_is_refused_everywhere(bad):
    lib, c = binding.load(), _cache(**bad)
    assert lib.pcg_cache_append(P, 128, P, 128, 4, P, ctypes.byref(c), None) == INVALID
    assert lib.pcg_cache_attention(P, 256, 4, 4, P, P, P, 2, 8, ctypes.byref(c), 0.1, P, P, 1 << 30, None) == INVALID


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k=P + 2), dict(ks=120), dict(vs=132), dict(vs=-128), dict(rows=-1),
                                 dict(slots=None)])
def test_append_refusals(bad):
    a = dict(k=P, ks=128, v=P, vs=128, rows=4, slots=P)
    a.update(bad)
    assert binding.load().pcg_cache_append(*a.values(), ctypes.byref(_cache()), None) == INVALID


def test_append_of_nothing_is_a_no_op():
    assert binding.load().pcg_cache_append(None, 0, None, 0, 0, None, ctypes.byref(_cache()), None) == 0
    assert binding.load().pcg_cache_append(P, 128, P, 128, 4, P, None, None) == INVALID


def _attend(**kw):
    a = dict(q=P, stride=256, rows=4, q_heads=4, start=P, kv=P, table=P, B=2, max_blocks=8, cache=ctypes.byref(_cache()), scale=0.1,
             out=P, ws=P, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return binding.load().pcg_cache_attention(*a.values())


def _prompt(**kw):
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, dtype=1, rows=4, q_heads=4, kv_heads=2, d=64, start=P, B=2, scale=0.1, out=P, ws=P,
             ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return binding.load().pcg_prompt_attention(*a.values())


BOTH = [dict(q=None), dict(q=P + 8), dict(rows=-1), dict(B=-1), dict(q_heads=3), dict(q_heads=0), dict(start=None), dict(out=None),
        dict(out=P + 4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))]


@pytest.mark.parametrize("bad", BOTH + [dict(kv=None), dict(table=None), dict(max_blocks=0), dict(max_blocks=1 << 28), dict(max_blocks=134217727), dict(stride=248),
                                        dict(stride=260)])
def test_cache_attention_refusals(bad):
    assert _attend(**bad) == INVALID


@pytest.mark.parametrize("bad", BOTH + [dict(k=None), dict(v=P + 8), dict(ks=64), dict(vs=129), dict(dtype=5), dict(d=12), dict(d=512),
                                        dict(kv_heads=0), dict(kv_heads=-2), dict(qs=1)])
def test_prompt_attention_refusals(bad):
    assert _prompt(**bad) == INVALID


def test_attention_limits_and_workspace():
    one = _cache(kv_heads=1)
    assert _attend(q_heads=129, stride=129 * 64, cache=ctypes.byref(one)) == UNSUPPORTED
    assert _attend(B=16385) == UNSUPPORTED and _prompt(B=16385) == UNSUPPORTED
    need = binding.load().pcg_attention_workspace_bytes(2, 4, 2, 64, 1)
    assert need >= 256 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1)):
        assert _attend(**bad) == WORKSPACE and _prompt(**bad) == WORKSPACE


def test_attention_of_nothing_is_a_no_op():
    assert _attend(rows=0, q=None, out=None, ws=None) == 0 and _prompt(rows=0, q=None, out=None, ws=None) == 0
    assert _attend(B=0) == 0 and _prompt(B=0) == 0


def test_the_binding_checks_shapes_and_places():
    import torch

    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    kc = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):  # host tensors
        binding.pcg_cache_append(q[:, :2], q[:, 2:], i(3), kc, kc.clone())
    for bad in (dict(q=q.float()), dict(q=q[:, :, ::2]), dict(q=q[0]), dict(q=q.transpose(0, 1)), dict(start=i(3, 1)), dict(kv=i(3)),
                dict(kv=i(2).long()), dict(table=i(3, 8)), dict(table=i(2, 16)[:, ::2]), dict(v=kc.float()), dict(k=kc.transpose(1, 2))):
        a = dict(q=q, start=i(3), kv=i(2), table=i(2, 8), k=kc, v=kc)
        a.update(bad)
        with pytest.raises(ValueError):
            binding.pcg_cache_attention(*a.values(), out=torch.empty_like(q), workspace=torch.empty(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        binding.pcg_prompt_attention(q, q[:, :2], q[:2, :2], i(3), out=torch.empty_like(q), workspace=i(1))
    with pytest.raises(ValueError):
        binding.pcg_cache_plan(i(2), i(3), i(2), i(2, 8), i(16), i(2), 16, 4)
