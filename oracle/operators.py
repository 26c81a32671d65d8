"""Operators (foreign functions) of a combinator program, node at a time, in 64 bits (test infrastructure, CPU only).

Plain loops over requests, tokens and heads, written from the definitions in the C header.  fp16 arrays are numpy
float16, bf16 arrays the uint16 patterns of their values.
"""
import numpy as np

F64 = np.float64

KINDS = ("block_table", "slot_map", "put_rows", "paged_attention", "penalize")


class Reported(ValueError):
    """The data hold a number outside its range: what the library reports as ACC_ERR_INDEX_RANGE."""


def widen(a, dtype):
    """Values in 64 bits."""
    if dtype == "bf16":
        return (a.astype(np.uint32) << 16).view(np.float32).astype(F64)
    return a.astype(F64)


def narrow(x, dtype):
    """The nearest value of the type, ties to even."""
    if dtype == "bf16":
        with np.errstate(over="ignore"):
            f = x.astype(np.float32)
        bits = f.view(np.uint32).astype(np.uint64)
        # (two roundings: through fp32, whose error is 2^-16 of bf16's; the tests' tolerances count it)
        up = (bits + 0x7FFF + ((bits >> 16) & 1)) >> 16
        return np.where(np.isnan(f), 0x7FC0, up).astype(np.uint16)
    with np.errstate(over="ignore"):
        return x.astype(np.float16 if dtype == "f16" else np.float32)


def _signed(a):
    return a.reshape(-1).view(np.int32).astype(np.int64).reshape(a.shape)


def _blocks(length, block):
    return -(-max(int(length), 0) // block)


def block_table(nd, xs):
    block, (R, W) = int(nd.iparam[0]), nd.shape
    lens, free = _signed(xs[0]), _signed(xs[1])
    old_lens = _signed(xs[2]) if len(xs) == 4 else np.zeros(R, np.int64)
    old = _signed(xs[3]) if len(xs) == 4 else np.full((R, W), -1, np.int64)
    out = np.full((R, W), -1, np.int64)
    bad = bool((lens < 0).any() or (old_lens < 0).any())
    used = 0
    for r in range(R):
        had, has = _blocks(old_lens[r], block), _blocks(lens[r], block)
        bad |= has > W
        for j in range(min(had, has, W)):
            out[r, j] = old[r, j]
        for j in range(had, has):
            k = used + j - had
            if k >= free.size:
                bad = True
                break
            if j < W:
                out[r, j] = free[k]
        used += max(has - had, 0)
    return out, bad


def slot_map(nd, xs):
    block, T = int(nd.iparam[0]), nd.shape[0]
    table, lens, off = _signed(xs[0]), _signed(xs[1]), _signed(xs[2])
    W = table.shape[1]
    out = np.full(T, -1, np.int64)
    bad = False
    for r in range(lens.size):
        for t in range(max(int(off[r]), 0), min(int(off[r + 1]), T)):
            p = int(lens[r]) - (int(off[r + 1]) - t)
            page = int(table[r, p // block]) if 0 <= p < W * block else -1
            slot = page * block + p % block
            if page < 0 or slot >= 1 << 31:
                bad = True
            else:
                out[t] = slot
    return out, bad


def put_rows(nd, xs):
    dest, slots, rows = xs[0].copy(), _signed(xs[1]), xs[2]
    bad = False
    for t, s in enumerate(slots):
        if s >= dest.shape[0]:
            bad = True
        elif s >= 0:
            dest[s] = rows[t]
    return dest, bad


def attended_slots(nd, table_row, length, slots):
    """(slots of the tokens that a request attends to, whether something about it is reported)."""
    block, window = int(nd.iparam[0]), int(nd.iparam[2]) if len(nd.iparam) > 2 else 0
    n = int(length)
    bad = n < 0 or n > table_row.size * block
    n = min(max(n, 0), table_row.size * block)
    lo = max(0, n - window) if window > 0 else 0
    out = []
    for p in range(lo, n):
        page = int(table_row[p // block])
        slot = page * block + p % block
        if page < 0 or slot >= slots:
            bad = True
        else:
            out.append(slot)
    return out, bad


def paged_attention(nd, xs):
    """(result in 64 bits, weighted mean of |V| per element, reported)."""
    D = int(nd.iparam[1])
    scale = float(nd.fparam[0])
    q, k, v = (widen(x, nd.dtype) for x in xs[:3])
    table, lens = _signed(xs[3]), _signed(xs[4])
    B, hq, hk = q.shape[0], q.shape[1] // D, k.shape[1] // D
    q, k, v = q.reshape(B, hq, D), k.reshape(-1, hk, D), v.reshape(-1, hk, D)
    out, scale_of = np.zeros((B, hq, D)), np.zeros((B, hq, D))
    bad = False
    for b in range(B):
        slots, wrong = attended_slots(nd, table[b], lens[b], k.shape[0])
        bad |= wrong
        if not slots:
            continue
        for h in range(hq):
            g = h // (hq // hk)
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (k[slots, g] @ q[b, h])
                w = np.exp(s - s.max())
                w = w / w.sum()
                out[b, h] = w @ v[slots, g]
                scale_of[b, h] = w @ np.abs(v[slots, g])
    return out.reshape(B, -1), scale_of.reshape(B, -1), bad


def penalize(nd, xs):
    """(result in 64 bits, sum of the magnitudes that were added up, reported)."""
    x = widen(xs[0], nd.dtype)
    mag = np.abs(x)
    tokens, params, ids, bias, mask = _signed(xs[1]), xs[2].astype(F64), _signed(xs[3]), xs[4].astype(F64), xs[5]
    B, V = x.shape
    bad = bool((tokens >= V).any() or (ids >= V).any())
    for b in range(B):
        rep, freq, pres, prompt = params[b]
        first = int(min(max(prompt, 0), tokens.shape[1]))
        seen, count = set(), {}
        for i, t in enumerate(tokens[b]):
            if 0 <= t < V:
                seen.add(int(t))
                if i >= first:
                    count[int(t)] = count.get(int(t), 0) + 1
        with np.errstate(divide="ignore", invalid="ignore"):
            for t in seen:
                x[b, t] = x[b, t] / rep if x[b, t] > 0 else x[b, t] * rep
                mag[b, t] = abs(x[b, t])
            for t, c in count.items():
                x[b, t] = x[b, t] - freq * c - pres
                mag[b, t] += abs(freq * c) + abs(pres)
            for t, add in zip(ids[b], bias[b]):
                if 0 <= t < V:
                    x[b, t] += add
                    mag[b, t] += abs(add)
        if mask.shape[1]:
            v = np.arange(V)
            x[b, (mask[b, v // 32] >> (v % 32).astype(np.uint32)) & 1 == 0] = -np.inf
    return x, mag, bad


def evaluate(nd, xs, res=None, i=None, strict=True):
    """The node's array in its own type; with strict, data that the library reports raise Reported."""
    if nd.kind in ("block_table", "slot_map"):
        out, bad = (block_table if nd.kind == "block_table" else slot_map)(nd, xs)
        out = (out & 0xFFFFFFFF).astype(np.uint32)
    elif nd.kind == "put_rows":
        out, bad = put_rows(nd, xs)
    else:
        exact, scale, bad = (paged_attention if nd.kind == "paged_attention" else penalize)(nd, xs)
        if res is not None:
            res.exact[i], res.abs_sum[i] = exact, scale
        out = narrow(exact, nd.dtype)
    if bad and strict:
        raise Reported(f"{nd.kind}: a number outside its range")
    return out
