"""Plain forms of the cache and attention operators for their tests: Python loops over lists, and 64-bit torch."""
import torch

NO_BLOCKS, TOO_LONG, NO_ROWS = 16, 32, 64


def plan(cached_len, accept_len, new_len, held, block_table, free_ring, ring_state, block_size, rows):
    """Lists in, dict of lists out; block_table and free_ring come back as copies."""
    B, max_blocks, N = len(cached_len), len(block_table[0]) if block_table else 0, len(free_ring)
    table, ring = [list(r) for r in block_table], list(free_ring)
    head, count = ring_state
    out = {k: [] for k in ("cached_len", "kv_len", "held", "flags")}
    out["row_start"], out["slots"], out["positions"] = [0], [-1] * rows, [-1] * rows
    at = asked = taken = freed = 0
    for b in range(B):
        if new_len[b] < 0:
            for i in range(held[b]):
                if count + freed < N:
                    ring[(head + count + freed) % N] = block_table[b][i]
                freed += 1
            for k in ("cached_len", "kv_len", "held", "flags"):
                out[k].append(0)
            out["row_start"].append(min(at, rows))
            continue
        c = max(0, cached_len[b] + (accept_len[b] + 1 if accept_len is not None else 0))
        n = new_len[b]
        blocks = -(-(c + n) // block_size)
        flag = NO_ROWS if n > 0 and at + n > rows else TOO_LONG if blocks > max_blocks else 0
        if not flag and blocks > held[b]:
            asked += blocks - held[b]
            if asked > count:
                flag = NO_BLOCKS
            else:
                for j in range(held[b], blocks):
                    table[b][j] = free_ring[(head + taken) % N]
                    taken += 1
        if not flag:
            for i in range(n):
                p = c + i
                out["slots"][at + i] = table[b][p // block_size] * block_size + p % block_size
                out["positions"][at + i] = p
        out["cached_len"].append(c)
        out["kv_len"].append(0 if flag else c + n)
        out["held"].append(held[b] if flag else max(held[b], blocks))
        out["flags"].append(flag)
        at += n
        out["row_start"].append(min(at, rows))
    out["ring_state"] = [(head + taken) % N, min(count - taken + freed, N)]
    return out, table, ring


def attention(q, k, v, lim, scale):
    """One sequence in 64 bits: q [n, qh, d], k and v [L, kvh, d], lim [n] -> (o, a, s): the output [n, qh, d], the
    weighted mean of |v| and the largest sum of |q k| of a score that a row sees [n, qh], which rounding scales with."""
    q, k, v = q.double(), k.double(), v.double()
    n, qh, d = q.shape
    L, kvh, _ = k.shape
    G = qh // kvh
    o, a, m = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((n, qh), dtype=torch.float64, device=q.device)
    if L == 0:
        return o, a, m
    hidden = torch.arange(L, device=q.device)[None, :] >= torch.as_tensor(lim, device=q.device)[:, None]
    empty = hidden.all(1)
    for h in range(qh):
        s = (q[:, h] @ k[:, h // G].T) * scale
        p = torch.softmax(s.masked_fill(hidden, float("-inf")), 1)
        p[empty] = 0
        o[:, h], a[:, h] = p @ v[:, h // G], p @ v[:, h // G].abs()
        m[:, h] = ((q[:, h].abs() @ k[:, h // G].abs().T) * scale).masked_fill(hidden, 0).amax(1)
    return o, a, m


def tolerance(o, a, s, dtype, d, keys):
    """How far a value may be off.  The output is rounded once: eps / 2 of it.  In the 16-bit types each weight is
    rounded once more before it meets its value (eps / 2 of the weighted mean of |v|), float16's weights below its
    normal range to 2^-31 of the largest.  A score is a sum of d products in 32 bits: each of its d additions, and the
    scale, the reference's subtraction and the power of two behind it, is off by at most 2^-23 of the sum of |q k|; that
    is a relative error of the weight, and another of the sum that it is divided by.  Powers of two: 2^-21, and 2^-16
    where weights are rounded to 16 bits; the running sums of weighted values: 2^-24 for each of the keys, which are
    summed in parts of at least 16."""
    half = torch.finfo(dtype).eps / 2
    weights = 2 * ((d + 4) * 2.0 ** -23 * s.unsqueeze(-1) + 2.0 ** (-21 if dtype == torch.float32 else -16)) + keys / 16 * 2.0 ** -23
    if dtype != torch.float32:
        weights = weights + half + keys * 2.0 ** -31
    return (half * o.abs() + weights * a) * 1.01 + 1e-30


def check(got, want, dtype, d, keys, where=""):
    o, a, s = want
    off = (got.double() - o).abs()
    far = off > tolerance(o, a, s, dtype, d, keys)
    assert not bool(far.any()) and bool(torch.isfinite(got).all()), (
        where, int(far.sum()), far.nonzero()[:4].tolist(), float(off.max()))
