"""pcg_cache_plan and pcg_cache_append against plain loops, on the GPU."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _state(B, bs, rng, max_blocks=40, most_new=30, spare=2.0, finished=0.1, fresh=0.2, accept=True, dirty=False):
    """A round's inputs: what is held covers what was cached and the last chunk, now and then with a block to spare."""
    cached, acc, new, held = [], [], [], []
    for _ in range(B):
        c, last = rng.randint(0, (max_blocks - 4) * bs - most_new), rng.randint(1, most_new)
        a, n = rng.randint(0, last - 1), rng.choice([0, 1, rng.randint(1, most_new)])
        h = -(-(c + last) // bs) + rng.randint(0, 1)
        if rng.random() < fresh:
            c, a, h, n = 0, -1, 0, rng.randint(1, 4 * most_new)
        elif rng.random() < finished:
            n = -rng.randint(1, 5)
        cached.append(c), acc.append(a), new.append(n), held.append(h)
    total = sum(held)
    ids = list(range(total + int(spare * B) + 1))
    rng.shuffle(ids)
    table = [[-1] * max_blocks for _ in range(B)]
    for b in range(B):
        for j in range(held[b]):
            table[b][j] = ids.pop()
    N = total + len(ids)
    head = rng.randrange(N)
    ring = [-5] * N
    for i, x in enumerate(ids):
        ring[(head + i) % N] = x
    return dict(cached_len=cached, accept_len=acc if accept else None, new_len=new, held=held, block_table=table, free_ring=ring,
                ring_state=[head, len(ids)], block_size=bs)


def _run(st, rows, repeat=1):
    from paper_2511_13732_b200 import binding

    d = {k: (None if v is None else v if k == "block_size" else _ints(v)) for k, v in st.items()}
    if not st["cached_len"]:
        d["block_table"] = torch.zeros((0, 8), dtype=torch.int32, device="cuda")
    for _ in range(repeat):
        p = binding.pcg_cache_plan(d["cached_len"], d["new_len"], d["held"], d["block_table"], d["free_ring"], d["ring_state"],
                                   d["block_size"], rows, accept_len=d["accept_len"])
    torch.cuda.synchronize()
    return p, d


def _compare(st, rows, repeat=1):
    import cache_ref

    want, table, ring = cache_ref.plan(rows=rows, **st)
    got, d = _run(st, rows, repeat)
    for name, w in want.items():
        assert getattr(got, name).tolist() == w, name
    assert d["block_table"].tolist() == table and d["free_ring"].tolist() == ring


@pytest.mark.parametrize("B,bs", [(1, 16), (2, 256), (3, 64), (31, 16), (256, 64), (513, 32), (1500, 16), (16384, 16)])
@pytest.mark.parametrize("accept", [True, False])
def test_plan_matches_the_loops(B, bs, accept):
    rng = random.Random(B * 7 + bs + accept)
    st = _state(B, bs, rng, accept=accept, max_blocks=40 if B < 5000 else 12)
    total = sum(max(n, 0) for n in st["new_len"])
    for rows in (total, total + 17, max(0, total - 40)):
        _compare(st, rows, repeat=2)


@pytest.mark.parametrize("spare", [0.0, 0.3])
def test_plan_denies_in_order_when_blocks_run_out(spare):
    import cache_ref

    st = _state(200, 16, random.Random(3), spare=spare)
    rows = sum(max(n, 0) for n in st["new_len"])
    flags = cache_ref.plan(rows=rows, **st)[0]["flags"]
    assert flags.count(cache_ref.NO_BLOCKS) > 5 and flags.count(0) > 5
    _compare(st, rows)


def test_plan_flags_sequences_beyond_the_table_and_clamps_lengths():
    st = _state(64, 16, random.Random(9), max_blocks=40)
    st["new_len"][5] = 5000  # more than the table holds
    st["cached_len"][7], st["accept_len"][7], st["held"][7] = -30, -1, 0
    rows = sum(max(n, 0) for n in st["new_len"])
    _compare(st, rows)
    st["new_len"][5] = 2 ** 31 - 1  # its rows do not fit either
    _compare(st, 400)


def test_plan_of_an_empty_batch_and_of_finished_sequences_only():
    _compare(dict(cached_len=[], accept_len=[], new_len=[], held=[], block_table=[], free_ring=[3, 1, 2], ring_state=[2, 2],
                  block_size=16), 5)
    st = _state(40, 32, random.Random(2))
    st["new_len"] = [-1] * 40
    _compare(st, 0)
    _compare(st, 3)


def test_released_blocks_never_overrun_the_ring():
    st = _state(20, 16, random.Random(4))
    st["new_len"] = [-1] * 20
    st["free_ring"] = st["free_ring"][:50]  # smaller than the pool: a caller's mistake, entries are dropped
    st["ring_state"] = [7, 10]
    _compare(st, 4)


@pytest.mark.parametrize("B,room,seed", [(2, 2, 0), (20, 0, 1), (20, 7, 2), (300, 40, 3)])
def test_what_a_full_ring_drops_is_not_counted_as_free(B, room, seed):
    """The call releases more than the ring has room for, and takes blocks as well: no block is then both held and free."""
    from paper_2511_13732_b200 import binding

    rng = random.Random(seed)
    bs, max_blocks = 16, 8
    held = [rng.randint(1, 5) for _ in range(B)]
    new = [-1 if b % 2 == 0 else rng.randint(0, 16) for b in range(B)]
    cached = [bs * h for h in held]  # full: a new token needs a block
    ids = list(range(sum(held) + B + room))
    rng.shuffle(ids)
    table = [[ids.pop() for _ in range(h)] + [-1] * (max_blocks - h) for h in held]
    free = [ids.pop() for _ in range(B)]  # enough for every sequence
    N, head = len(free) + room, rng.randrange(len(free) + room)
    ring = [-7] * N
    for i, x in enumerate(free):
        ring[(head + i) % N] = x
    taken = sum(1 for n in new if n > 0)
    released = [x for b in range(B) if new[b] < 0 for x in table[b][: held[b]]]
    assert taken > 0 and len(released) > room
    d_table, d_ring = _ints(table), _ints(ring)
    p = binding.pcg_cache_plan(_ints(cached), _ints(new), _ints(held), d_table, d_ring, _ints([head, len(free)]), bs, 16 * B)
    at, count = p.ring_state.tolist()
    assert p.flags.tolist() == [0] * B and count == len(free) - taken + room
    now = [d_ring.tolist()[(at + i) % N] for i in range(count)]
    assert now == free[taken:] + released[:room]
    owned = [x for row, h in zip(d_table.tolist(), p.held.tolist()) for x in row[:h]]
    assert not set(owned) & set(now)


def test_a_plan_feeds_the_next_one():
    """Forty rounds by swapping two sets of tensors: no block is ever in two hands, none is lost."""
    from paper_2511_13732_b200 import binding

    rng = random.Random(11)
    B, bs, n_blocks, max_blocks, rows = 24, 16, 150, 12, 24 * 40
    z = lambda: torch.zeros(B, dtype=torch.int32, device="cuda")  # noqa: E731
    cached, held, table = z(), z(), torch.full((B, max_blocks), -1, dtype=torch.int32, device="cuda")
    ring, state = torch.arange(n_blocks, dtype=torch.int32, device="cuda"), _ints([0, n_blocks])
    accept = _ints([-1] * B)
    live = [False] * B
    for _ in range(40):
        new = []
        for b in range(B):
            if live[b] and rng.random() < 0.15:
                new.append(-1)
                live[b] = False
            else:
                new.append(rng.randint(1, 40) if not live[b] else 5)
                live[b] = True
        p = binding.pcg_cache_plan(cached, _ints(new), held, table, ring, state, bs, rows, accept_len=accept)
        h, t = p.held.tolist(), table.tolist()
        owned = [x for b in range(B) for x in t[b][: h[b]]]
        head, count = p.ring_state.tolist()
        free = [ring.tolist()[(head + i) % n_blocks] for i in range(count)]
        assert sorted(owned + free) == list(range(n_blocks))
        slots = [s for s in p.slots.tolist() if s >= 0]
        assert len(set(slots)) == len(slots) and set(s // bs for s in slots) <= set(owned)
        flags = p.flags.tolist()
        for b in range(B):
            if flags[b]:
                live[b] = live[b] and h[b] > 0
        accept = _ints([-1 if flags[b] or new[b] < 1 else rng.randint(0, new[b] - 1) for b in range(B)])
        cached, held, state = p.cached_len, p.held, p.ring_state


# ---- append ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,heads,d,bs", [(1, 1, 8, 16), (5, 4, 64, 16), (33, 3, 40, 32), (700, 8, 128, 64), (257, 5, 256, 256)])
def test_append_writes_the_slots_and_nothing_else(dtype, rows, heads, d, bs):
    from paper_2511_13732_b200 import binding

    g = torch.Generator(device="cuda").manual_seed(rows + d)
    n_blocks = rows // bs + 3
    kc, vc = (torch.randn((n_blocks, heads, bs, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    fused = torch.randn((rows, 2 * heads + 3, d), generator=g, device="cuda").to(dtype)
    k, v = fused[:, 1: heads + 1], fused[:, heads + 2: 2 * heads + 2]
    if rows > 1:
        fused[1] = float("nan")  # copied as they are
    slots = torch.randperm(n_blocks * bs, generator=g, device="cuda")[:rows].to(torch.int32)
    slots[rows // 2::7] = -1
    if rows > 4:
        slots[3] = n_blocks * bs  # behind the cache
        slots[4] = -2 ** 31
    wk, wv = kc.clone(), vc.clone()
    for r, s in enumerate(slots.tolist()):
        if 0 <= s < n_blocks * bs:
            wk[s // bs, :, s % bs], wv[s // bs, :, s % bs] = k[r], v[r]
    binding.pcg_cache_append(k, v, slots, kc, vc)
    torch.cuda.synchronize()
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    assert torch.equal(kc.view(bits), wk.view(bits)) and torch.equal(vc.view(bits), wv.view(bits))


def test_append_reaches_offsets_past_32_bits():
    from paper_2511_13732_b200 import binding

    n_blocks, heads, bs, d = 70000, 8, 64, 128  # 4.6e9 elements each
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    kc, vc = (torch.empty((n_blocks, heads, bs, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.randn((2, heads, d), device="cuda").bfloat16() for _ in range(2))
    slots = [n_blocks * bs - 1, 40000 * bs + 5]
    for s in slots:
        kc[s // bs, :, s % bs] = vc[s // bs, :, s % bs] = 0
    binding.pcg_cache_append(k, v, _ints(slots), kc, vc)
    for r, s in enumerate(slots):
        assert torch.equal(kc[s // bs, :, s % bs], k[r]) and torch.equal(vc[s // bs, :, s % bs], v[r])


def test_plan_and_append_on_another_stream():
    from paper_2511_13732_b200 import binding
    import cache_ref

    side = torch.cuda.Stream()
    st = _state(50, 16, random.Random(6))
    rows = sum(max(n, 0) for n in st["new_len"])
    want, table, _ = cache_ref.plan(rows=rows, **st)
    d = {k: (v if k == "block_size" else _ints(v)) for k, v in st.items()}
    kc, vc = (torch.zeros((len(st["free_ring"]), 2, 16, 64), device="cuda") for _ in range(2))
    k = torch.randn((rows, 2, 64), device="cuda")
    torch.cuda.synchronize()
    p = binding.pcg_cache_plan(d["cached_len"], d["new_len"], d["held"], d["block_table"], d["free_ring"], d["ring_state"], 16, rows,
                               accept_len=d["accept_len"], stream=side)
    binding.pcg_cache_append(k, -k, p.slots, kc, vc, stream=side)
    side.synchronize()
    assert p.slots.tolist() == want["slots"] and d["block_table"].tolist() == table
    for r, s in enumerate(want["slots"]):
        if s >= 0:
            assert torch.equal(kc[s // 16, :, s % 16], k[r]) and torch.equal(vc[s // 16, :, s % 16], -k[r])


def test_plan_into_given_tensors_without_flags_and_positions():
    from paper_2511_13732_b200 import binding
    import cache_ref

    st = _state(9, 32, random.Random(8))
    rows = sum(max(n, 0) for n in st["new_len"])
    want = cache_ref.plan(rows=rows, **st)[0]
    d = {k: (v if k == "block_size" else _ints(v)) for k, v in st.items()}
    e = lambda n: torch.full((n,), -9, dtype=torch.int32, device="cuda")  # noqa: E731
    out = binding.CachePlan(e(9), e(9), e(9), e(10), e(rows), None, e(2), None)
    got = binding.pcg_cache_plan(d["cached_len"], d["new_len"], d["held"], d["block_table"], d["free_ring"], d["ring_state"], 32, rows,
                                 accept_len=d["accept_len"], out=out)
    assert got is out and got.slots.tolist() == want["slots"] and got.held.tolist() == want["held"]
    with pytest.raises(binding.PcgError):  # outputs that are inputs
        binding.pcg_cache_plan(d["cached_len"], d["new_len"], d["held"], d["block_table"], d["free_ring"], d["ring_state"], 32, rows,
                               accept_len=d["accept_len"], out=out._replace(held=d["held"]))
