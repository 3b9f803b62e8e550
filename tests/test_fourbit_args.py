"""What the entry points with positions and with a cache of 4 bits refuse, before anything is launched (no GPU is needed)."""
import ctypes

import pytest

from paper_2511_13732_b200 import binding

P = 4096  # stands for an aligned device address: nothing below gets as far as looking at it
INVALID, UNSUPPORTED, WORKSPACE = 1, 3, 4


def _ref(struct, base, kw):
    base.update(kw)
    return ctypes.byref(struct(*base.values()))


def _cache(**kw):
    return _ref(binding._Cache, dict(n_blocks=8, block_size=16, kv_heads=2, head_dim=64, dtype=1, k=P, v=P), kw)


def _four(**kw):
    return _ref(binding._FourbitCache, dict(n_blocks=8, block_size=16, kv_heads=2, head_dim=64, k_scale=1.0, v_scale=1.0, data=P), kw)


def _rotary(**kw):
    return _ref(binding._Rotary, dict(dim=64, interleaved=0, positions=100, table=P), kw)


def _append_rotary(**kw):
    a = dict(q=P, qs=256, q_heads=4, k=P, ks=128, v=P, vs=128, rows=4, slots=P, positions=P, rotary=_rotary(), cache=_cache(), q_out=2 * P,
             qos=256, k_out=None, kos=0, stream=None)
    a.update(kw)
    return binding.load().pcg_cache_append_rotary(*a.values())


def _append_fourbit(**kw):
    a = dict(q=P, qs=256, q_heads=4, k=P, ks=128, v=P, vs=128, dtype=1, rows=4, slots=P, positions=P, rotary=_rotary(), cache=_four(),
             q_out=2 * P, qos=256, k_out=None, v_out=None, stream=None)
    a.update(kw)
    return binding.load().pcg_cache_append_fourbit(*a.values())


def _attend(**kw):
    a = dict(q=P, stride=256, dtype=1, rows=4, q_heads=4, start=P, kv=P, table=P, B=2, max_blocks=8, cache=_four(), scale=0.1, out=P, ws=P,
             ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return binding.load().pcg_cache_attention_fourbit(*a.values())


ROTARIES = [dict(dim=0), dict(dim=-32), dict(dim=72), dict(dim=128), dict(interleaved=2), dict(positions=0), dict(table=None), dict(table=P + 4)]
APPENDS = [dict(q=None), dict(q_out=None), dict(q_heads=0), dict(q_heads=-1), dict(q=P + 8), dict(q_out=P + 2), dict(qs=248), dict(qos=260),
           dict(q_out=P, qos=512), dict(k=None), dict(v=None), dict(k=P + 2), dict(ks=120), dict(vs=-128), dict(rows=-1), dict(slots=None),
           dict(positions=None), dict(rotary=None)]


@pytest.mark.parametrize("bad", ROTARIES)
def test_a_bad_rotation_is_refused(bad):
    for call in (_append_rotary, _append_fourbit):
        assert call(rotary=_rotary(**bad)) == INVALID
        assert "rotation" in binding.load().pcg_last_error().decode()
    assert _append_fourbit(rotary=_rotary(dim=48)) == INVALID  # whole groups of 16 on either side of a pair


@pytest.mark.parametrize("bad", APPENDS + [dict(k_out=P + 8, kos=128), dict(k_out=2 * P, kos=64), dict(k_out=P, kos=256), dict(cache=None),
                                           dict(cache=_cache(head_dim=68)), dict(cache=_cache(k=None))])
def test_append_with_rotation_refusals(bad):
    assert _append_rotary(**bad) == INVALID


@pytest.mark.parametrize("bad", APPENDS + [dict(k_out=P + 8), dict(v_out=P + 4), dict(dtype=3), dict(cache=None)])
def test_append_fourbit_refusals(bad):
    assert _append_fourbit(**bad) == INVALID
    assert "pcg_cache_append_fourbit" in binding.load().pcg_last_error().decode()


@pytest.mark.parametrize("bad", [dict(n_blocks=0), dict(block_size=8), dict(block_size=48), dict(block_size=512), dict(kv_heads=0),
                                 dict(kv_heads=1025), dict(head_dim=0), dict(head_dim=80), dict(head_dim=288), dict(data=None), dict(data=P + 8),
                                 dict(n_blocks=1 << 27), dict(k_scale=0.0), dict(k_scale=-1.0), dict(v_scale=float("nan")),
                                 dict(v_scale=float("inf")), dict(k_scale=1e-30), dict(v_scale=1e30)])
def test_a_bad_fourbit_cache_is_refused(bad):
    assert _append_fourbit(cache=_four(**bad)) == INVALID
    assert _attend(cache=_four(**bad)) == INVALID


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=P + 8), dict(rows=-1), dict(B=-1), dict(q_heads=3), dict(q_heads=0), dict(start=None),
                                 dict(out=None), dict(out=P + 4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(scale=1e38, cache=_four(k_scale=2.0 ** 40)), dict(kv=None), dict(table=None),
                                 dict(max_blocks=0), dict(max_blocks=1 << 28), dict(max_blocks=134217727), dict(stride=248), dict(stride=260),
                                 dict(dtype=7), dict(cache=None)])
def test_attention_fourbit_refusals(bad):
    assert _attend(**bad) == INVALID


def test_limits_and_workspace():
    assert _attend(q_heads=129, stride=129 * 64, cache=_four(kv_heads=1)) == UNSUPPORTED
    assert _attend(B=16385) == UNSUPPORTED
    need = binding.load().pcg_attention_workspace_bytes(2, 4, 2, 64, 1)
    for bad in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1)):
        assert _attend(**bad) == WORKSPACE
    assert _append_fourbit(rows=2147483647, k=P, cache=_four(kv_heads=1024), ks=1024 * 64, vs=1024 * 64) == UNSUPPORTED


def test_calls_of_nothing_are_no_ops():
    assert _append_rotary(rows=0, k=None, v=None, slots=None, positions=None) == 0
    assert _append_fourbit(rows=0, k=None, v=None, slots=None, positions=None) == 0
    assert _attend(rows=0, q=None, out=None, ws=None) == 0 and _attend(B=0) == 0
    assert _append_fourbit(rows=0, rotary=None, q=None, q_out=None, q_heads=0) == 0


def test_the_binding_checks_shapes_and_places():
    import torch

    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    cache = torch.zeros(binding.pcg_fourbit_cache_shape(4, 2, 32, 64), dtype=torch.uint8)
    assert cache.shape == (4, 2, 2, 1152)
    kc, tab = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(10, 64)
    for call in (lambda: binding.pcg_cache_append_rotary(None, k, k, i(3), i(3), tab, kc, kc.clone()),
                 lambda: binding.pcg_cache_append_fourbit(None, k, k, i(3), cache),
                 lambda: binding.pcg_cache_attention_fourbit(k, i(3), i(2), i(2, 8), cache)):
        with pytest.raises(ValueError, match="current device"):  # host tensors
            call()
