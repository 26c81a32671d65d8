"""What is timed: the operators of a decode step, as a user's program runs them -- a program of one or two nodes is
built, planned and bound once, then `Graph.run(FUSED)` is called on it step after step.

  tables      block tables and slot maps from request lengths: every request keeps a row of block numbers, new blocks
              come from a free list, and every new token learns its slot in the cache
  append      rows of new keys and values put into the cache at those slots, in place
  attention   one new token per request over its paged keys and values
  penalties   penalties for tokens seen before, biases and a grammar mask on rows of logits

Sizes go from a single request, where a call's latency is all that counts, to caches several times the L2.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}

# ---- the cases -----------------------------------------------------------------------------------


def listed():
    return [
        # One step of a small batch: every request grows by one token, few need a new block.  The smallest call.
        {"name": "tables_step_16", "op": "tables", "requests": 16, "longest": 2000, "block": 16, "new": 1, "fresh": False},
        # The same for a large batch with long tables.
        {"name": "tables_step_1000", "op": "tables", "requests": 1000, "longest": 60000, "block": 16, "new": 1, "fresh": False},
        # Prompts of very unequal lengths are admitted at once: tables from nothing, slots of every token.
        {"name": "tables_prompts_517", "op": "tables", "requests": 517, "longest": 20011, "block": 32, "new": 0, "fresh": True},
        # The new keys and values of one step's batch, some rows of it padding.
        {"name": "append_step_96", "op": "append", "tokens": 96, "padding": 7, "cols": 1024, "slots": 1 << 16, "dtype": "bf16"},
        # Those of a chunk of prompts, with rows of a width that is a multiple of nothing much.
        {"name": "append_prompt_12001", "op": "append", "tokens": 12001, "padding": 100, "cols": 1000, "slots": 30000, "dtype": "f32"},
        # One conversation, a few hundred tokens: what counts is the latency.
        {"name": "attention_one_700", "op": "attention", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "longest": 700, "block": 16, "window": 0, "dtype": "bf16"},
        # A few very long documents: few rows, so that the work has to be split over the length.
        {"name": "attention_long_3", "op": "attention", "batch": 3, "q_heads": 16, "kv_heads": 2, "head_dim": 128,
         "longest": 200000, "block": 64, "window": 0, "dtype": "bf16"},
        # A full server: ragged lengths, grouped heads.
        {"name": "attention_batch_128", "op": "attention", "batch": 128, "q_heads": 64, "kv_heads": 8, "head_dim": 128,
         "longest": 24000, "block": 16, "window": 0, "dtype": "bf16"},
        # Heads of their own, another width, a sliding window, half precision.
        {"name": "attention_window_31", "op": "attention", "batch": 31, "q_heads": 20, "kv_heads": 20, "head_dim": 80,
         "longest": 9001, "block": 24, "window": 4096, "dtype": "f16"},
        # The framework's own type.
        {"name": "attention_f32_40", "op": "attention", "batch": 40, "q_heads": 32, "kv_heads": 8, "head_dim": 64,
         "longest": 5000, "block": 32, "window": 0, "dtype": "f32"},
        # One conversation's logits: latency again.
        {"name": "penalties_one_32003", "op": "penalties", "batch": 1, "vocabulary": 32003, "history": 600, "biases": 10,
         "mask": True, "dtype": "f32"},
        # A server's batch with long histories.
        {"name": "penalties_batch_256", "op": "penalties", "batch": 256, "vocabulary": 131072, "history": 4096, "biases": 64,
         "mask": True, "dtype": "bf16"},
    ]


def _size(rng, lo, hi):
    """An integer between lo and hi, even over the logarithm; every third one is a multiple of 16, the others as they fall."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 1 / 3:
        v -= v % 16
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["tables", "append", "attention", "attention", "attention", "penalties"])
    if op == "tables":
        fresh = rng.random() < 0.5
        return {"op": op, "requests": _size(rng, 1, 4000), "longest": _size(rng, 16, 30000), "block": rng.choice([8, 16, 24, 32, 64, 128]),
                "new": 0 if fresh else rng.choice([1, 1, 4]), "fresh": fresh}
    if op == "append":
        tokens, cols = _size(rng, 1, 16000), rng.choice([64, 128, 256, 512, 1000, 1024, 1333, 2048])
        return {"op": op, "tokens": tokens, "padding": rng.choice([0, tokens // 9]), "cols": cols,
                "slots": max(2 * tokens, (1 << 24) // cols), "dtype": rng.choice(["f32", "f16", "bf16"])}
    if op == "attention":
        kv = rng.choice([1, 2, 4, 8, 8, 16, 20])
        group = rng.choice([1, 2, 4, 5, 7, 8, 16]) if kv <= 8 else rng.choice([1, 2])
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        batch = _size(rng, 1, 300)
        longest = _size(rng, 16, max(64, min(200000, (1 << 31) // (batch * kv * dim * SIZE[dtype]))))
        return {"op": op, "batch": batch, "q_heads": kv * group, "kv_heads": kv, "head_dim": dim, "longest": longest,
                "block": rng.choice([8, 16, 16, 24, 32, 64, 128]), "window": rng.choice([0, 0, 0, _size(rng, 64, 4096)]), "dtype": dtype}
    batch, vocabulary = _size(rng, 1, 256), _size(rng, 1000, 131072)
    return {"op": op, "batch": batch, "vocabulary": vocabulary, "history": _size(rng, 1, 6000), "biases": rng.choice([0, 0, 5, 64, 300]),
            "mask": rng.random() < 0.5, "dtype": rng.choice(["f32", "f32", "bf16", "f16"])}


# ---- inputs -----------------------------------------------------------------------------------------


def _lengths(case, rows):
    """Request lengths: the same for every seed (so that the work is the case's), in an order that the seed shuffles.
    One is the longest, the others spread over one and a half orders of magnitude below."""
    rng = random.Random("%d/%d" % (rows, case["longest"]))
    low = max(1.0, case["longest"] / 30)
    lens = [case["longest"]] + [int(math.exp(rng.uniform(math.log(low), math.log(case["longest"])))) for _ in range(rows - 1)]
    return np.array([max(1, v) for v in lens], dtype=np.int64)


def _i32(values):
    return torch.as_tensor(np.ascontiguousarray(values, dtype=np.int32), device="cuda")


def _tables_data(case, seed):
    rng = np.random.default_rng(seed)
    b, R = case["block"], case["requests"]
    lens = _lengths(case, R)
    rng.shuffle(lens)
    old = np.zeros(R, np.int64) if case["fresh"] else np.maximum(lens - case["new"], 0)
    need_old, need = -(-old // b), -(-lens // b)
    W = -(-case["longest"] // b)
    pool = rng.permutation(int(need.sum()) + 64)                       # every block of the cache, in some order of use
    table = np.full((R, W), -1, np.int64)
    at = np.arange(W)[None, :]
    first = np.concatenate([[0], np.cumsum(need_old)[:-1]])
    held = at < need_old[:, None]
    table[held] = pool[(first[:, None] + at)[held]]
    free = pool[int(need_old.sum()):]
    off = np.concatenate([[0], np.cumsum(lens - old)])
    T = int(off[-1]) + (0 if case["fresh"] else 3)                     # a batch is padded to some size
    return {"lens": lens, "old_lens": old, "old": table, "free": free, "off": off, "T": T, "W": W}


def _attention_lengths(case):
    return _lengths(case, case["batch"])


def _attended(case):
    lens = _attention_lengths(case)
    return int(np.minimum(lens, case["window"]).sum() if case["window"] else lens.sum())


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _data(case, seed):
    op = case["op"]
    if op == "tables":
        d = _tables_data(case, seed)
        return {k: _i32(d[k]) for k in ("lens", "old_lens", "old", "free", "off")} | {"T": d["T"], "W": d["W"]}
    gen = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, device="cuda", dtype=dtype, generator=gen)
    if op == "append":
        S, T, C = case["slots"], case["tokens"], case["cols"]
        slots = torch.randperm(S, device="cuda", generator=gen)[:T].to(torch.int32)
        if case["padding"]:
            slots[T - case["padding"]:] = -1
        # one row more than the cache has: where a program without a check for padding may send it
        return {"keys": normal(S + 1, C), "values": normal(S + 1, C), "slots": slots, "k": normal(T, C), "v": normal(T, C)}
    if op == "attention":
        rng = np.random.default_rng(seed)
        b, B = case["block"], case["batch"]
        lens = _attention_lengths(case)
        rng.shuffle(lens)
        need = -(-lens // b)
        W = int(need.max())
        blocks = int(need.sum()) + 8
        pool = rng.permutation(blocks)
        table = np.full((B, W), -1, np.int64)
        at = np.arange(W)[None, :]
        held = at < need[:, None]
        table[held] = pool[((np.cumsum(need) - need)[:, None] + at)[held]]
        q = normal(B, case["q_heads"] * case["head_dim"])
        keys = normal(blocks * b, case["kv_heads"] * case["head_dim"])
        values = normal(blocks * b, case["kv_heads"] * case["head_dim"])
        return {"q": q, "keys": keys, "values": values, "table": _i32(table), "lens": _i32(lens)}
    B, V, L, K = case["batch"], case["vocabulary"], case["history"], case["biases"]
    uniform = lambda *shape: torch.rand(*shape, device="cuda", generator=gen)
    logits = (4 * torch.randn(B, V, device="cuda", generator=gen)).to(dtype)
    tokens = (V * uniform(B, L) ** 3).to(torch.int32).clamp_(max=V - 1)          # some tokens far more often than others
    length = (uniform(B, 1) * (L + 1)).to(torch.int32)
    tokens = torch.where(torch.arange(L, device="cuda")[None, :] < length, tokens, -1).to(torch.int32)
    params = torch.stack([1 + 0.3 * uniform(B), 0.5 * uniform(B), 0.5 * uniform(B), (uniform(B) * length[:, 0]).floor()], dim=1).contiguous()
    start = torch.randint(0, V, (B, 1), device="cuda", generator=gen)
    step = 1 + V // max(K, 1) // 2
    bias_ids = ((start + step * torch.arange(K, device="cuda")[None, :]) % V).to(torch.int32)
    bias = 10 * uniform(B, K) - 5
    words = -(-V // 32) if case["mask"] else 0
    mask = torch.randint(-(1 << 31), 1 << 31, (B, words), device="cuda", generator=gen, dtype=torch.int64).to(torch.int32)
    return {"logits": logits, "tokens": tokens, "params": params, "bias_ids": bias_ids.contiguous(), "bias": bias, "mask": mask}


def prepare(case, seed):
    state = {"case": case, "data": _data(case, seed)}
    if own:
        _bind(state)
    return state


# ---- the framework's operators ------------------------------------------------------------------------


def _bind(state):
    """The handle that a program keeps: the nodes, a clustering, the buffers, a workspace."""
    import workloads as W
    from paper_2407_13585_b200 import binding as B
    case, d = state["case"], state["data"]
    op = case["op"]
    into = {}
    if op == "tables":
        prog = W.block_tables(case["requests"], d["W"], d["free"].numel(), d["T"], case["block"], grow=not case["fresh"])
        arrays = {k: d[k] for k in (("lens", "free", "off") if case["fresh"] else ("lens", "free", "old_lens", "old", "off"))}
    elif op == "append":
        prog = W.append_rows(case["slots"], case["cols"], case["tokens"], case["dtype"])
        S = case["slots"]
        arrays = {"keys": d["keys"][:S], "values": d["values"][:S], "slots": d["slots"], "k": d["k"], "v": d["v"]}
        into = {"new_keys": arrays["keys"], "new_values": arrays["values"]}               # in place
    elif op == "attention":
        prog = W.paged_attention(case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"], d["keys"].shape[0], case["block"],
                                 d["table"].shape[1], case["dtype"], scale=case["head_dim"] ** -0.5, window=case["window"])
        arrays = d
    else:
        prog = W.penalized_logits(case["batch"], case["vocabulary"], case["history"], case["biases"], case["mask"], case["dtype"])
        arrays = d
    g = B.Graph(prog.nodes, prog.outputs)
    g.plan("enumerate", "bytes")
    for name, t in arrays.items():
        g.bind(prog.id(name), t)
    outs = []
    for o in prog.outputs:
        nd = prog.nodes[o]
        t = into.get(nd.name)
        if t is None:
            t = torch.empty(nd.shape, dtype=DTYPES.get(nd.dtype, torch.int32), device="cuda")
        g.bind(o, t)
        outs.append(t)
    g.ensure_workspace(B.FUSED)
    state.update(graph=g, outs=outs, fused=B.FUSED)


# ---- the plain forms ------------------------------------------------------------------------------------


def _plain_tables(case, d):
    b = case["block"]
    lens, free = d["lens"].long(), d["free"]
    old = torch.zeros_like(lens) if case["fresh"] else d["old_lens"].long()
    need, need_old = (lens + b - 1) // b, (old + b - 1) // b
    take = (need - need_old).clamp(min=0)
    base = take.cumsum(0) - take
    j = torch.arange(d["W"], device=lens.device)[None, :]
    fresh = free[(base[:, None] + j - need_old[:, None]).clamp(0, free.numel() - 1)]
    kept = fresh if case["fresh"] else d["old"]
    minus = torch.full_like(fresh, -1)
    table = torch.where(j < need[:, None], torch.where(j < need_old[:, None], kept, fresh), minus)
    off = d["off"].long()
    T, R = d["T"], lens.numel()
    t = torch.arange(T, device=lens.device)
    row = torch.zeros(T + 1, dtype=torch.long, device=lens.device).index_add_(0, off[1:], torch.ones_like(off[1:])).cumsum(0)[:T]
    inside = row < R
    row = row.clamp(max=R - 1)
    p = (lens[row] - (off[row + 1] - t)).clamp(min=0)
    slots = torch.where(inside, table[row, (p // b).clamp(max=d["W"] - 1)].long() * b + p % b, -1).to(torch.int32)
    return [table, slots]


def _plain_append(case, d):
    S = case["slots"]
    at = torch.where(d["slots"] < 0, S, d["slots"]).long()
    d["keys"][at] = d["k"]
    d["values"][at] = d["v"]
    return [d["keys"][:S], d["values"][:S]]


def _plain_attention(case, d):
    B, Hk, D, b = case["batch"], case["kv_heads"], case["head_dim"], case["block"]
    G = case["q_heads"] // Hk
    W = d["table"].shape[1]
    n = W * b
    t = torch.arange(n, device="cuda")
    out = torch.empty(B, Hk, G, D, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 29) // (n * Hk * D))                            # a few requests at a time, so that the copies fit
    for lo in range(0, B, step):
        hi = min(B, lo + step)
        lens = d["lens"][lo:hi].long()
        slot = d["table"][lo:hi].long().clamp(min=0)[:, t // b] * b + t % b
        k = d["keys"][slot].view(hi - lo, n, Hk, D).float()
        q = d["q"][lo:hi].view(hi - lo, Hk, G, D).float()
        s = torch.einsum("bhgd,bnhd->bhgn", q, k) * D ** -0.5
        del k
        valid = t[None, :] < lens[:, None]
        if case["window"]:
            valid = valid & (t[None, :] >= lens[:, None] - case["window"])
        s = torch.where(valid[:, None, None, :], s, -math.inf)
        p = (s - s.amax(-1, keepdim=True)).exp()
        p = p / p.sum(-1, keepdim=True)
        v = d["values"][slot].view(hi - lo, n, Hk, D).float()
        out[lo:hi] = torch.einsum("bhgn,bnhd->bhgd", p, v)
        del v
    return [out.view(B, -1).to(DTYPES[case["dtype"]])]


def _plain_penalties(case, d):
    B, V, L = case["batch"], case["vocabulary"], case["history"]
    x = d["logits"].float()
    at = torch.where(d["tokens"] < 0, V, d["tokens"]).long()
    rep, freq, pres, prompt = (d["params"][:, k:k + 1] for k in range(4))
    later = (torch.arange(L, device="cuda")[None, :] >= prompt).float()
    seen = torch.zeros(B, V + 1, device="cuda").scatter_(1, at, 1.0)[:, :V] > 0
    count = torch.zeros(B, V + 1, device="cuda").scatter_add_(1, at, later)[:, :V]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * count
    x = x - pres * (count > 0)
    if case["biases"]:
        ids = torch.where(d["bias_ids"] < 0, V, d["bias_ids"]).long()
        x = x + torch.zeros(B, V + 1, device="cuda").scatter_add_(1, ids, d["bias"])[:, :V]
    if case["mask"]:
        bits = (d["mask"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.view(B, -1)[:, :V] != 0, x, -math.inf)
    return [x.to(DTYPES[case["dtype"]])]


_PLAIN = {"tables": _plain_tables, "append": _plain_append, "attention": _plain_attention, "penalties": _plain_penalties}


def run(state):
    if "graph" in state:
        state["graph"].run(state["fused"], finish=False)
        return state["outs"]
    return _PLAIN[state["case"]["op"]](state["case"], state["data"])


# ---- what a pass cannot do without ---------------------------------------------------------------------


def work(case):
    """Every input that the path needs read once, every output written once."""
    op = case["op"]
    if op == "tables":
        R, b, W = case["requests"], case["block"], -(-case["longest"] // case["block"])
        lens = _lengths(case, R)
        need = int((-(-lens // b)).sum())
        fresh = case["fresh"]
        new = int(lens.sum()) if fresh else int(np.minimum(lens, case["new"]).sum())
        # lengths, offsets, the entries that a row has (from the free list or the old table), the new table, the slots
        return {"bytes": 4 * (R * (1 if fresh else 2) + R + 1 + need + R * W + new), "flops": R * W + 4 * new}
    e = SIZE[case["dtype"]]
    if op == "append":
        T = case["tokens"] - case["padding"]
        return {"bytes": 4 * case["tokens"] + 2 * 2 * T * case["cols"] * e, "flops": 0}
    if op == "attention":
        B, n = case["batch"], _attended(case)
        row = case["kv_heads"] * case["head_dim"] * e
        return {"bytes": 2 * n * row + 4 * (n // case["block"] + B) + 2 * B * case["q_heads"] * case["head_dim"] * e,
                "flops": 4 * n * case["q_heads"] * case["head_dim"]}
    B, V = case["batch"], case["vocabulary"]
    words = -(-V // 32) if case["mask"] else 0
    return {"bytes": 2 * B * V * e + 4 * B * (case["history"] + 4 + 2 * case["biases"] + words), "flops": 6 * B * V}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return _exact_tables(case, seed)
    if op == "append":
        d = _data(case, seed)
        slots = d["slots"].cpu().numpy()
        keys, values = d["keys"][:case["slots"]].double(), d["values"][:case["slots"]].double()
        rows = torch.as_tensor(np.flatnonzero(slots >= 0), device="cuda")
        where = torch.as_tensor(slots[slots >= 0].astype(np.int64), device="cuda")
        return [keys.index_copy(0, where, d["k"].double()[rows]), values.index_copy(0, where, d["v"].double()[rows])]
    if op == "attention":
        return _exact_attention(case, seed)
    return _exact_penalties(case, seed)


def _exact_tables(case, seed):
    d = _tables_data(case, seed)
    b, free, used = case["block"], d["free"], 0
    table = np.full((case["requests"], d["W"]), -1, np.int64)
    slots = np.full(d["T"], -1, np.int64)
    at = 0
    for r in range(case["requests"]):
        had, has = -(-int(d["old_lens"][r]) // b), -(-int(d["lens"][r]) // b)
        table[r, :had] = d["old"][r, :had]
        table[r, had:has] = free[used:used + has - had]
        used += has - had
        p = np.arange(int(d["old_lens"][r]), int(d["lens"][r]))
        slots[at:at + p.size] = table[r, p // b] * b + p % b
        at += p.size
    return [torch.as_tensor(table.astype(np.int32)), torch.as_tensor(slots.astype(np.int32))]


def _exact_attention(case, seed):
    d = _data(case, seed)
    B, Hk, D, b = case["batch"], case["kv_heads"], case["head_dim"], case["block"]
    G = case["q_heads"] // Hk
    lens, table = d["lens"].cpu().numpy(), d["table"].cpu().numpy()
    out = torch.zeros(B, Hk, G, D, dtype=torch.float64, device="cuda")
    q = d["q"].double().view(B, Hk, G, D)
    for r in range(B):
        n = int(lens[r])
        lo = max(0, n - case["window"]) if case["window"] else 0
        p = np.arange(lo, n)
        slot = torch.as_tensor(table[r, p // b].astype(np.int64) * b + p % b, device="cuda")
        k = d["keys"][slot].view(-1, Hk, D)
        v = d["values"][slot].view(-1, Hk, D)
        for h in range(Hk):                                             # head by head: 64-bit copies of one head at a time
            s = (k[:, h].double() @ q[r, h].T) / math.sqrt(D)
            w = torch.exp(s - s.max(0).values)
            out[r, h] = (w.T @ v[:, h].double()) / w.sum(0)[:, None]
    return [out.view(B, -1)]


def _exact_penalties(case, seed):
    d = _data(case, seed)
    if d["logits"].numel() > 1 << 25:
        return None
    x = d["logits"].double().cpu().numpy()
    tokens, params = d["tokens"].cpu().numpy(), d["params"].double().cpu().numpy()
    ids, bias, mask = d["bias_ids"].cpu().numpy(), d["bias"].double().cpu().numpy(), d["mask"].cpu().numpy().view(np.uint32)
    for r in range(case["batch"]):
        rep, freq, pres, prompt = params[r]
        have = np.unique(tokens[r][tokens[r] >= 0])
        x[r, have] = np.where(x[r, have] > 0, x[r, have] / rep, x[r, have] * rep)
        later, times = np.unique(tokens[r][int(prompt):][tokens[r][int(prompt):] >= 0], return_counts=True)
        x[r, later] -= freq * times + pres
        np.add.at(x[r], ids[r][ids[r] >= 0], bias[r][ids[r] >= 0])
        if case["mask"]:
            bit = np.unpackbits(mask[r].view(np.uint8), bitorder="little")[:case["vocabulary"]]
            x[r, bit == 0] = -math.inf
    return [torch.as_tensor(x)]
