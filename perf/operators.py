"""Cases of the cache and attention operators: what a decoding round runs before its drafted tokens are verified.

A round feeds each sequence its last token and its drafted tokens (K + 1 rows).  ``plan`` turns the accept lengths of the
last verification and the lengths of the new chunks into block tables, slots and positions; ``append`` writes the chunk's
keys and values to the paged cache; ``attend`` is the attention of the chunk over the cache (single tokens, drafted chunks
and chunks of a prompt); ``prompt`` is the causal attention of whole prompts, packed one after the other.

Key/value cache: ``[n_blocks, kv_heads, block_size, head_dim]`` for keys and for values; slot s is row s % block_size of
block s // block_size.  Block tables are ``[B, max_blocks]``; what they hold behind a sequence's blocks is arbitrary, and
so is what the cache holds behind a sequence's last token (here: NaN, as fresh memory may).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one sequence, one lookahead of four: the smallest round, where only latency counts
        dict(name="plan_b1_k4", op="plan", B=1, k=4, ctx=1000, bs=64, mix=0),
        # 256 sequences with sixteen drafted tokens: the round of the largest verification workload
        dict(name="plan_b256_k16", op="plan", B=256, k=16, ctx=4000, bs=64, mix=0),
        # a large server's batch: most sequences decode, some bring prompts, some have finished, some find no block
        dict(name="plan_b3001_mixed", op="plan", B=3001, k=8, ctx=2500, bs=16, mix=1),
        # the keys and values of one drafted chunk, small draft model
        dict(name="append_r5_f32", op="append", rows=5, kvh=4, d=64, bs=16, dtype="f32"),
        # prompts entering the cache of one layer, rows taken out of the fused projection
        dict(name="append_r33001_bf16", op="append", rows=33001, kvh=8, d=128, bs=64, dtype="bf16"),
        # one token a sequence, ragged contexts: plain decoding
        dict(name="attend_b64_n1_bf16", op="attend", B=64, n=1, ctx=8000, qh=32, kvh=8, d=128, bs=64, dtype="bf16", ragged=1),
        # sixteen drafted tokens and the last one over 256 contexts: the largest verification workload's round
        dict(name="attend_b256_n17_bf16", op="attend", B=256, n=17, ctx=2000, qh=32, kvh=8, d=128, bs=64, dtype="bf16", ragged=1),
        # the small float32 model's round of eight drafted tokens
        dict(name="attend_b16_n9_f32", op="attend", B=16, n=9, ctx=700, qh=12, kvh=4, d=64, bs=16, dtype="f32", ragged=1),
        # one sequence drafting four tokens: latency of a single stream
        dict(name="attend_b1_n5_bf16", op="attend", B=1, n=5, ctx=3001, qh=32, kvh=8, d=128, bs=32, dtype="bf16", ragged=0),
        # chunks of long prompts over what is cached of them already
        dict(name="attend_b2_n2048_f16", op="attend", B=2, n=2048, ctx=16000, qh=32, kvh=8, d=128, bs=128, dtype="f16", ragged=0),
        # a batch of spoken prompts of different lengths, draft model's heads
        dict(name="prompt_b16_l1500_f16", op="prompt", B=16, len=1500, qh=16, kvh=4, d=64, dtype="f16", ragged=1),
        # one long prompt
        dict(name="prompt_b1_l8192_bf16", op="prompt", B=1, len=8192, qh=32, kvh=8, d=128, dtype="bf16", ragged=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attend", "attend", "attend", "prompt", "prompt"])
    if op == "plan":
        return dict(op=op, B=_log(rng, 1, 3000), k=rng.randint(0, 16), ctx=_log(rng, 20, 4000),
                    bs=rng.choice([16, 32, 64, 128]), mix=rng.randint(0, 1))
    heads = rng.choice([(32, 8), (16, 4), (16, 16), (12, 4), (28, 4), (16, 2), (8, 1)])
    d = rng.choice([64, 128])
    if op == "append":
        return dict(op=op, rows=_log(rng, 1, 30000), kvh=heads[1], d=d, bs=rng.choice([16, 32, 64, 128]),
                    dtype=rng.choice(["bf16", "f16", "f32"]))
    if op == "prompt":
        length = _log(rng, 1, 6000)
        B = max(1, min(32, _log(rng, 1, 32), 12000 // length))
        return dict(op=op, B=B, len=length, qh=heads[0], kvh=heads[1], d=d, dtype=rng.choice(["bf16", "f16"]),
                    ragged=rng.randint(0, 1))
    dtype = rng.choice(["bf16", "f16", "bf16", "f16", "f32"])
    case = dict(op=op, qh=heads[0], kvh=heads[1], d=d, bs=rng.choice([16, 32, 64, 128]), dtype=dtype, ragged=rng.randint(0, 1))
    kind = rng.choice(["token", "draft", "draft", "chunk"])
    if dtype == "f32":  # the small models' type
        return dict(case, B=_log(rng, 1, 16), n=1 if kind == "token" else rng.randint(2, 17), ctx=_log(rng, 16, 1500))
    if kind == "chunk":
        n = _log(rng, 18, 2000)
        B = max(1, min(_log(rng, 1, 8), 4000 // n))
        return dict(case, B=B, n=n, ctx=_log(rng, 16, 12000))
    ctx = _log(rng, 16, 12000)
    return dict(case, B=max(1, min(_log(rng, 1, 256), 400000 // ctx)), n=1 if kind == "token" else rng.randint(2, 17), ctx=ctx)


def _spread(count, most, ragged):
    """Lengths up to `most`: all of them the largest, or spread evenly between an eighth of it and all of it."""
    lo = max(1, most // 8) if ragged and count > 1 else most
    return torch.linspace(lo, most, count, dtype=torch.float64).round().to(torch.int64)


def _lengths(count, most, ragged, gen):
    """_spread's lengths in an order of the seed's, so that every seed's tensors have the same shapes."""
    return _spread(count, most, ragged)[torch.randperm(count, generator=gen)].to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    cuda = torch.Generator(device="cuda").manual_seed(seed)

    def ints(lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=gen, dtype=torch.int32)

    def normal(*shape, dtype):
        return torch.randn(shape, generator=cuda, device="cuda", dtype=dtype)

    op = case["op"]
    if op == "plan":
        B, bs = case["B"], case["bs"]
        cached = _lengths(B, case["ctx"], 1, gen)
        new = torch.full((B,), case["k"] + 1, dtype=torch.int32)
        accept = ints(0, case["k"] + 1, B)
        # blocks held from the last round, whose chunk was as long as this one's
        held = (cached + case["k"] + 1 + bs - 1) // bs
        if case["mix"]:  # a tenth brings prompts, a twentieth has finished
            kind = torch.randperm(B, generator=gen)
            fresh, done = kind < B // 10, kind >= B - B // 20
            new[fresh] = _lengths(B // 10, 700, 1, gen)
            new[done] = -1
            cached[fresh] = held[fresh] = 0
            accept[fresh] = -1
        max_blocks = (case["ctx"] + 2 * (case["k"] + 1) + 700 + bs - 1) // bs
        n_blocks = B * max_blocks
        perm = torch.randperm(n_blocks, generator=gen, dtype=torch.int32)
        table = torch.full((B, max_blocks), -1, dtype=torch.int32)
        at = torch.arange(max_blocks)[None, :] < held[:, None]
        table[at] = perm[: int(held.sum())]
        free = min(n_blocks - int(held.sum()), 64 + 2 * B)  # the mixed batch's prompts do not all find their blocks
        head = int(ints(0, n_blocks, 1))
        ring = torch.full((n_blocks,), -1, dtype=torch.int32)
        ring[(head + torch.arange(free)) % n_blocks] = perm[n_blocks - free:]
        rows = int(new.clamp(min=0).sum())
        state = torch.tensor([head, free], dtype=torch.int32)
        return dict(case, cached_len=cached.cuda(), new_len=new.cuda(), accept_len=accept.cuda(), held=held.cuda(),
                    block_table=table.cuda(), free_ring=ring.cuda(), ring_state=state.cuda(), rows=rows)
    dtype, kvh, d = DTYPES[case["dtype"]], case["kvh"], case["d"]
    if op == "append":
        rows, bs = case["rows"], case["bs"]
        n_blocks = (rows + rows // 4 + bs - 1) // bs + 2
        slots = torch.randperm(n_blocks * bs, generator=cuda, device="cuda")[:rows].sort().values
        # the blocks of a sequence lie anywhere in the cache; inside a block the tokens follow one another
        order = torch.randperm(n_blocks, generator=cuda, device="cuda")
        slots = (order[slots // bs] * bs + slots % bs).to(torch.int32)
        fused = normal(rows, 4 * kvh, d, dtype=dtype)  # queries, keys and values of one projection
        cache = [torch.zeros((n_blocks, kvh, bs, d), dtype=dtype, device="cuda") for _ in range(2)]
        return dict(case, k=fused[:, 2 * kvh:3 * kvh], v=fused[:, 3 * kvh:], slots=slots, k_cache=cache[0], v_cache=cache[1])
    qh, B = case["qh"], case["B"]
    if op == "prompt":
        lens = _lengths(B, case["len"], case["ragged"], gen)
        start = torch.zeros(B + 1, dtype=torch.int32)
        start[1:] = lens.cumsum(0)
        fused = normal(int(start[-1]), qh + 2 * kvh, d, dtype=dtype)
        fused[:, :qh] *= 1.5
        return dict(case, q=fused[:, :qh], k=fused[:, qh:qh + kvh], v=fused[:, qh + kvh:], row_start=start.cuda(),
                    most=int(lens.max()))
    n, bs = case["n"], case["bs"]
    before = _lengths(B, case["ctx"], case["ragged"], gen)
    # drafted chunks have one length; chunks of prompts end where the prompt does
    new = _lengths(B, n, 1, gen) if case["ragged"] and n > 17 else torch.full((B,), n, dtype=torch.int32)
    kv_len = before + new
    start = torch.zeros(B + 1, dtype=torch.int32)
    start[1:] = new.cumsum(0)
    used = (kv_len + bs - 1) // bs
    max_blocks, total = int(used.max()) + 1, int(used.sum())
    n_blocks = total + 3
    perm = torch.randperm(n_blocks, generator=gen, dtype=torch.int32)
    table = torch.full((B, max_blocks), -1, dtype=torch.int32)
    table[torch.arange(max_blocks)[None, :] < used[:, None]] = perm[:total]
    table, kv_len = table.cuda(), kv_len.cuda()
    k_cache, v_cache = normal(n_blocks, kvh, bs, d, dtype=dtype), normal(n_blocks, kvh, bs, d, dtype=dtype)
    at = torch.arange(max_blocks * bs, device="cuda")
    slot = table.long().repeat_interleave(bs, 1) * bs + at % bs
    written = torch.zeros(n_blocks * bs, dtype=torch.bool, device="cuda")
    written[slot[at[None, :] < kv_len[:, None]]] = True
    for c in (k_cache, v_cache):
        c.masked_fill_(~written.view(n_blocks, 1, bs, 1), math.nan)
    q = normal(int(start[-1]), qh, d, dtype=dtype) * 1.5
    return dict(case, q=q, row_start=start.cuda(), kv_len=kv_len, block_table=table, k_cache=k_cache, v_cache=v_cache,
                most=int(new.max()))


def _plan(s):
    B, bs, rows = s["B"], s["bs"], s["rows"]
    table, ring = s["block_table"], s["free_ring"]
    size, max_blocks = ring.shape[0], table.shape[1]
    head, count = s["ring_state"][0].long(), s["ring_state"][1].long()
    done = s["new_len"] < 0
    held = s["held"].long()
    base = torch.where(done, 0, s["cached_len"].long() + s["accept_len"].long() + 1)
    new = s["new_len"].long().clamp(min=0)
    end = new.cumsum(0)
    begin = end - new
    blocks = (base + new + bs - 1) // bs
    full = (end > rows) & (new > 0)
    long_ = blocks > max_blocks
    need = torch.where(done | full | long_, 0, (blocks - held).clamp(min=0))
    upto = need.cumsum(0)
    short = (need > 0) & (upto > count)
    denied = full | long_ | short
    need_ok = torch.where(short, 0, need)
    first = upto - need
    freed = torch.where(done, held, 0)
    freed_at = freed.cumsum(0) - freed
    j = torch.arange(max_blocks, device=table.device)[None, :]
    fresh = (j >= held[:, None]) & (j < (held + need_ok)[:, None])
    new_table = torch.where(fresh, ring[(head + first[:, None] + j - held[:, None]) % size], table)
    # released blocks go behind the ring's tail, every other entry keeps its value
    where = torch.where(j < freed[:, None], (head + count + freed_at[:, None] + j) % size, size)
    new_ring = torch.cat([ring, ring[:1]]).scatter(0, where.reshape(-1), table.reshape(-1))[:size]
    r = torch.arange(rows, device=table.device)
    b = torch.searchsorted(end, r, right=True)
    bb = b.clamp(max=B - 1)
    pos = base[bb] + r - begin[bb]
    ok = (b < B) & ~denied[bb]
    block = new_table[bb, (pos // bs).clamp(0, max_blocks - 1)].long()
    slots = torch.where(ok, block * bs + pos % bs, -1)
    positions = torch.where(ok, pos, -1)
    kv_len = torch.where(done | denied, 0, base + new)
    start = torch.cat([end.new_zeros(1), end.clamp(max=rows)])
    state = torch.stack([(head + need_ok.sum()) % size, count - need_ok.sum() + freed.sum()])
    flags = 16 * short + 32 * long_ + 64 * full
    out = [base, kv_len, torch.where(done, 0, held + need_ok), start, slots, positions, state, flags]
    return [t.to(torch.int32) for t in out] + [new_table, new_ring]


def _softmax_rows(scores, seen):
    """Softmax over the last axis of the places that are seen; a row that sees nothing is zero."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total)


def _attention(q, k, v, row_start, kv_len, most):
    """q [T, qh, d]; k, v [B, kvh, S, d] in 32 bits; attention of the packed rows, each over its own sequence."""
    T, qh, d = q.shape
    B, kvh, S, _ = k.shape
    n = (row_start[1:] - row_start[:-1]).long()
    i = torch.arange(most, device=q.device)
    at = (row_start[:-1].long()[:, None] + i).clamp(max=T - 1)
    qp = q.float()[at].view(B, most, kvh, qh // kvh, d).permute(0, 2, 3, 1, 4).reshape(B, kvh, -1, d)
    scores = torch.matmul(qp, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    limit = (kv_len.long() - n)[:, None] + i + 1  # [B, most]
    seen = torch.arange(S, device=q.device) < limit[:, :, None]  # [B, most, S]
    p = _softmax_rows(scores.view(B, kvh, qh // kvh, most, S), seen[:, None, None])
    known = torch.arange(S, device=q.device) < kv_len.long()[:, None]
    o = torch.matmul(p.view(B, kvh, -1, S), torch.where(known[:, None, :, None], v, 0.0))
    o = o.view(B, kvh, qh // kvh, most, d).permute(0, 3, 1, 2, 4).reshape(B, most, qh, d)
    r = torch.arange(T, device=q.device)
    b = torch.searchsorted(row_start[1:].contiguous(), r.to(torch.int32), right=True)
    return o[b, r - row_start[b]].to(q.dtype)


def run(s):
    op = s["op"]
    if own:
        from paper_2511_13732_b200 import binding

        if op == "plan":
            plan = binding.pcg_cache_plan(s["cached_len"], s["new_len"], s["held"], s["block_table"], s["free_ring"],
                                          s["ring_state"], s["bs"], s["rows"], accept_len=s["accept_len"])
            return list(plan) + [s["block_table"], s["free_ring"]]
        if op == "append":
            binding.pcg_cache_append(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
            return [s["k_cache"], s["v_cache"]]
        if op == "attend":
            return binding.pcg_cache_attention(s["q"], s["row_start"], s["kv_len"], s["block_table"], s["k_cache"], s["v_cache"])
        return binding.pcg_prompt_attention(s["q"], s["k"], s["v"], s["row_start"])
    if op == "plan":
        return _plan(s)
    if op == "append":
        bs = s["bs"]
        block, row = s["slots"].long() // bs, s["slots"].long() % bs
        s["k_cache"][block, :, row] = s["k"]
        s["v_cache"][block, :, row] = s["v"]
        return [s["k_cache"], s["v_cache"]]
    if op == "attend":
        B, kvh, bs, d = s["B"], s["kvh"], s["bs"], s["d"]
        table = s["block_table"].long().clamp(min=0)

        def pages(c):
            return c[table].permute(0, 2, 1, 3, 4).reshape(B, kvh, -1, d).float()

        return _attention(s["q"], pages(s["k_cache"]), pages(s["v_cache"]), s["row_start"], s["kv_len"], s["most"])
    start, most = s["row_start"], s["most"]
    n = start[1:] - start[:-1]
    at = (start[:-1].long()[:, None] + torch.arange(most, device=start.device)).clamp(max=s["q"].shape[0] - 1)
    k, v = (t.float()[at].permute(0, 2, 1, 3) for t in (s["k"], s["v"]))
    return _attention(s["q"], k, v, start, n, most)


def _pairs(case):
    """(rows, keys and values read, pairs of row and key) of an attention case."""
    if case["op"] == "prompt":
        n = _spread(case["B"], case["len"], case["ragged"])
        return int(n.sum()), int(n.sum()), int((n * (n + 1) // 2).sum())
    n = _spread(case["B"], case["n"], case["ragged"] and case["n"] > 17).double()
    ctx = _spread(case["B"], case["ctx"], case["ragged"]).double()
    # which context goes with which chunk is the seed's: the mean over all orders
    return int(n.sum()), int((n + ctx).sum()), float(n.sum() * ctx.mean() + (n * (n + 1) / 2).sum())


def work(case):
    op = case["op"]
    if op == "plan":
        # lengths in and out, the table's new entries (about one a chunk), slots and positions
        B = case["B"]
        chunk = B - B // 10 - B // 20 if case["mix"] else B
        rows = chunk * (case["k"] + 1) + (int(_spread(B // 10, 700, 1).sum()) if case["mix"] else 0)
        return {"bytes": 4 * (9 * B + 2 * rows) + 8 * (rows // case["bs"] + 1), "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    if op == "append":
        return {"bytes": case["rows"] * (4 * case["kvh"] * case["d"] * size + 4), "flops": 0}
    rows, keys, pairs = _pairs(case)
    return {"bytes": size * case["d"] * (2 * rows * case["qh"] + 2 * keys * case["kvh"]),
            "flops": 4 * case["qh"] * case["d"] * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return None  # whole numbers
    if op == "append":
        made = []
        for new, old in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            rows = old.double().transpose(1, 2).reshape(-1, case["kvh"], case["d"])
            rows[s["slots"].long()] = new.double()
            made.append(rows.view(-1, case["bs"], case["kvh"], case["d"]).transpose(1, 2).contiguous())
        return made
    start = s["row_start"].tolist()
    G = case["qh"] // case["kvh"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        lo, hi = start[b], start[b + 1]
        n = hi - lo
        if op == "prompt":
            k, v, L = s["k"][lo:hi].double(), s["v"][lo:hi].double(), n
        else:
            L = int(s["kv_len"][b])
            blocks = s["block_table"][b, :(L + case["bs"] - 1) // case["bs"]].long()
            k, v = (c[blocks].double().transpose(1, 2).reshape(-1, case["kvh"], case["d"])[:L] for c in (s["k_cache"], s["v_cache"]))
        behind = torch.arange(L, device="cuda")[None, :] > (torch.arange(n, device="cuda") + L - n)[:, None]
        for h in range(case["qh"]):
            w = (s["q"][lo:hi, h].double() @ k[:, h // G].T) / math.sqrt(case["d"])
            w[behind] = -math.inf
            out[lo:hi, h] = torch.softmax(w, 1) @ v[:, h // G]
    return out
