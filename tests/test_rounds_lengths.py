"""What stays cached from round to round, followed on the CPU: the plan is the tests' plain loop, the verification a list of
accept lengths."""
import pytest

torch = pytest.importorskip("torch")


def _ints(x):
    return torch.tensor(x, dtype=torch.int32)


@pytest.fixture
def rounds(monkeypatch):
    """A maker of states in host memory, and the accept lengths that the next verification returns."""
    from paper_2511_13732_b200 import binding
    from paper_2511_13732_b200.rounds import DecodeRounds
    import cache_ref

    def plan(cached_len, new_len, held, block_table, free_ring, ring_state, block_size, rows, accept_len=None, stream=None):
        out, table, ring = cache_ref.plan(cached_len.tolist(), accept_len.tolist(), new_len.tolist(), held.tolist(), block_table.tolist(),
                                          free_ring.tolist(), ring_state.tolist(), block_size, rows)
        block_table.copy_(_ints(table)), free_ring.copy_(_ints(ring))
        return binding.CachePlan(**{k: _ints(v) for k, v in out.items()})

    accepts = []
    monkeypatch.setattr(binding, "pcg_cache_plan", plan)
    monkeypatch.setattr(binding, "pcg_verify", lambda target, draft, *a, **kw: (_ints(accepts.pop(0)), None, None, None))
    return lambda B, n_blocks=64, max_blocks=32: DecodeRounds(B, 1, n_blocks, 16, 1, 8, max_blocks, device="cpu"), accepts


def _verify(state, B, K, **kw):
    return state.verify(torch.zeros(B, K + 1, 1), torch.zeros(B, K, 1), torch.zeros(B, K, dtype=torch.int32), None, None, **kw)


def test_a_round_of_prompts_short_and_full_drafts_ends_with_what_was_fed(rounds):
    """K = 4: a prompt stays whole, a chunk keeps its first token and the accepted ones of the drafts that it has."""
    make, accepts = rounds
    s = make(7)
    s.begin(_ints([200, 5, 1, 3, 6, 0, -1]), 300)
    accepts.append([2, 3, 4, 4, 0, 4, 4])
    _verify(s, 7, 4)
    p = s.begin(_ints([5] * 7), 300)
    assert p.cached_len.tolist() == [200, 4, 1, 3, 6, 0, 0]
    assert p.positions.tolist()[:5] == [200, 201, 202, 203, 204]
    accepts.append([4, 0, 2, 1, 4, 3, 0])
    _verify(s, 7, 4)
    p = s.begin(_ints([1] * 7), 300)
    assert p.cached_len.tolist() == [205, 5, 4, 5, 11, 4, 1]


def test_sequences_named_whole_keep_all_of_a_short_chunk(rounds):
    make, accepts = rounds
    s = make(4)
    s.begin(_ints([3, 5, 5, 2]), 20)
    accepts.append([0, 0, 0, 0])
    _verify(s, 4, 4, whole=torch.tensor([True, False, True, False]))
    assert s.begin(_ints([1] * 4), 20).cached_len.tolist() == [3, 1, 5, 1]
    s.keep_all()
    s.begin(_ints([5] * 4), 20)
    with pytest.raises(ValueError, match="whole"):
        _verify(s, 4, 4, whole=torch.tensor([True]))
    with pytest.raises(ValueError, match="batch"):
        _verify(s, 1, 4)
    accepts.append([1] * 4)
    _verify(s, 4, 4)  # refused calls leave the round as it was
    assert s.begin(_ints([1] * 4), 20).cached_len.tolist() == [6, 4, 8, 4]


def test_a_flagged_sequence_keeps_nothing_of_its_chunk(rounds):
    make, accepts = rounds
    s = make(3, n_blocks=4)
    p = s.begin(_ints([40, 20, 5]), 100)
    assert p.flags.tolist() == [0, 16, 16]
    accepts.append([1, 4, 4])
    _verify(s, 3, 4, whole=torch.tensor([False, True, True]))
    assert s.begin(_ints([0] * 3), 100).cached_len.tolist() == [40, 0, 0]


@pytest.mark.parametrize("verified", [True, False])
def test_a_buffer_of_chunk_lengths_may_be_refilled_at_once(rounds, verified):
    make, accepts = rounds
    s = make(3)
    new = _ints([20, 5, 0])
    s.begin(new, 30)
    new.copy_(_ints([-1, 1, 5]))  # the next round's
    if verified:
        accepts.append([0, 3, 2])
        _verify(s, 3, 4)
    else:
        s.keep_all()
    assert s.begin(_ints([1] * 3), 30).cached_len.tolist() == [20, 4 if verified else 5, 0]


def test_attention_of_other_rows_than_the_round_has_is_refused(rounds):
    make, _ = rounds
    s = make(2)
    s.begin(_ints([3, 4]), 9)
    rows = lambda n, heads: torch.zeros(n, heads, 8, dtype=torch.bfloat16)  # noqa: E731
    for q, k in ((7, 9), (9, 7), (10, 9), (0, 0)):
        with pytest.raises(ValueError, match="9 rows"):
            s.attend(0, rows(q, 2), rows(k, 1), rows(k, 1))
