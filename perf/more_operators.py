"""Attention of sequences that share a prefix, and a cache that keeps the rows of most attention weight: their calls,
their plain forms and their results in 64 bits.

attn     louiskv.shared_prefix_attn: the queries of the last tokens of every sequence over the rows that all sequences
         share and the sequence's own ones, under one softmax.  Optionally each own row's weight, summed over the
         queries, is added to an accumulator; with no prefix this is the attention of a cache of bounded size.
weights  louiskv.attn_weights: the weight that a prompt's (last) queries give to each key, added to an accumulator,
         from the keys and the logs of the softmax denominators.
evict    louiskv.evict_rows: the n_keep rows of largest accumulated weight (the first positions and the recent ones are
         always kept) into a smaller cache.
store    louiskv.store_evict: new rows enter a cache of bounded size, the lightest rows leave for them.

A slice is one (sequence, layer, KV head), sequences outermost; a prefix slice one (layer, KV head).  Query t of n_q
sees the first n_own - n_q + t + 1 own rows, and the whole prefix.  Of n rows m = min(n, n_keep) stay: all that are
protected, then the heaviest; of equal weights the lower row leaves.  Kept rows below m stay where they are, the k-th
row below m that leaves is replaced by the k-th kept row from m on.
"""
import math

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases

def _attn(name, seqs, layers, kv_heads, q_heads, prefix, own_rows, own_least, queries=1, weights=False, ragged=False,
          dtype="bf16"):
    return {"name": name, "kind": "attn", "seqs": seqs, "layers": layers, "kv_heads": kv_heads, "q_heads": q_heads,
            "prefix": prefix, "own_rows": own_rows, "own_least": own_least, "queries": queries, "weights": weights,
            "ragged": ragged, "dtype": dtype}


def _weights(name, kv_heads, q_heads, keys, queries, dtype="bf16"):
    return {"name": name, "kind": "weights", "kv_heads": kv_heads, "q_heads": q_heads, "keys": keys,
            "queries": queries, "dtype": dtype}


def _evict(name, slices, rows, least, keep, first, recent, dtype="bf16"):
    return {"name": name, "kind": "evict", "slices": slices, "rows": rows, "least": least, "keep": keep,
            "first": first, "recent": recent, "dtype": dtype}


def _store(name, slices, budget, least, first, recent, new=1, dtype="bf16"):
    return {"name": name, "kind": "store", "slices": slices, "budget": budget, "least": least, "first": first,
            "recent": recent, "new": new, "dtype": dtype}


def listed():
    return [
        # one layer of four samples of a 32K prompt, some 500 tokens into their answers
        _attn("attn-prefix-b4", 4, 1, 8, 32, 32768, 640, 300),
        # one layer of 64 samples of a 32K prompt at different points of answers of up to 1024 tokens
        _attn("attn-prefix-b64", 64, 1, 8, 32, 32768, 1024, 1),
        # questions of up to 300 tokens about one document: their last 77, for eight at once
        _attn("attn-prefix-chunk", 8, 1, 8, 32, 20011, 300, 77, queries=77),
        # float32, eight heads to a KV head, three tokens at a time, a prefix that was cut down to ragged lengths
        _attn("attn-prefix-f32-g8", 3, 2, 4, 32, 5003, 257, 2, queries=3, ragged=True, dtype="f32"),
        # a layer of one sequence over its cache of 2048 rows, weights accumulated: latency
        _attn("attn-bounded", 1, 1, 8, 32, 0, 2048, 2048, weights=True),
        # every layer of four sequences over caches of 2048 rows
        _attn("attn-bounded-all-b4", 4, 32, 8, 32, 0, 2048, 1500, weights=True),
        # the last 64 queries of one layer's 32K prompt decide which of its rows stay
        _weights("weights-last-64", 8, 32, 32768, 64),
        # all queries of one layer's 32K prompt
        _weights("weights-layer-32k", 8, 32, 32768, 32768),
        # eight layers' prompts of 32K tokens down to 2048 rows each
        _evict("evict-prompt-32k", 64, 32768, 32768, 2048, 4, 128),
        # short ragged prompts, some of which fit whole, in float32
        _evict("evict-ragged-f32", 24, 1501, 200, 777, 1, 33, dtype="f32"),
        # one layer's step: the lightest row leaves for the new one
        _store("store-layer", 8, 2048, 2048, 4, 128),
        # every layer of four sequences, a chunk of five tokens each, some caches not yet full
        _store("store-all-b4", 1024, 2048, 1900, 4, 128, new=5),
    ]


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "weights", "evict", "store"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    kv = rng.choice([1, 2, 4, 8, 8, 8])
    g = rng.choice([1, 2, 3, 4, 4, 4, 7, 8])
    if kind == "attn":
        weights = rng.random() < 0.5
        prefix = 0 if weights and rng.random() < 0.6 else _log_int(rng, 1, 32768)
        rows = _log_int(rng, 1, 4096)
        queries = 1 if rng.random() < 0.7 else min(rows, _log_int(rng, 1, 128))
        seqs = _log_int(rng, 1, 64)
        # rows read and products within the largest listed cases, a quarter of that in float32
        part = 4 if dtype == "f32" else 1
        most = (1 << 21) // part
        seqs = max(1, min(seqs, most // (kv * rows)))
        pairs = (1 << 28) // part
        while seqs > 1 and seqs * g * queries * kv * (prefix + rows) > pairs:
            seqs //= 2
        queries = max(1, min(queries, pairs // (seqs * g * kv * (prefix + rows))))
        layers = _log_int(rng, 1, max(1, min(32, most // (kv * (prefix + seqs * rows)),
                                             pairs // (seqs * g * queries * kv * (prefix + rows)))))
        return _unnamed(_attn("", seqs, layers, kv, kv * g, prefix, rows, rng.randint(queries, rows), queries, weights,
                              rng.random() < 0.5, dtype))
    if kind == "weights":
        keys = _log_int(rng, 1, 32768)
        queries = keys if rng.random() < 0.4 else min(keys, _log_int(rng, 1, 4096))
        most = 32768 * 32768 * 16 // (16 if dtype == "f32" else 1)
        queries = min(queries, max(1, most // (keys * kv * g)))
        return _unnamed(_weights("", kv, kv * g, keys, queries, dtype))
    if kind == "evict":
        rows = _log_int(rng, 1, 40000)
        most = (1 << 21) // (2 if dtype == "f32" else 1)
        keep = _log_int(rng, 1, rows)
        first = rng.randint(0, min(8, keep))
        return _unnamed(_evict("", _log_int(rng, 1, max(1, min(1024, most // rows))), rows, rng.randint(1, rows), keep,
                               first, rng.randint(0, min(256, keep - first)), dtype))
    budget = _log_int(rng, 2, 8192)
    new = 1 if rng.random() < 0.5 else _log_int(rng, 1, max(1, min(64, budget // 2)))
    first = rng.randint(0, min(8, budget - new))
    most = (1 << 21) // (2 if dtype == "f32" else 1)
    return _unnamed(_store("", _log_int(rng, 1, max(1, min(1024, most // budget))), budget,
                           rng.randint(0, budget), first, rng.randint(0, min(256, budget - new - first)), new, dtype))


# ------------------------------------------------------------------- inputs

def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + tag) & ((1 << 62) - 1))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    """Whole numbers from lo to hi, both included."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _some(slices, n):
    """Slices taken at a time so that their float32 rows stay within a quarter of a GiB."""
    step = max(1, (1 << 19) // max(1, n))
    return [(i, min(slices, i + step)) for i in range(0, slices, step)]


def _keys(g, slices, n, dtype):
    """Keys that drift as a text does, four channels eight times the others'."""
    out = torch.empty(slices, n, D, dtype=dtype, device="cuda")
    topics = max(1, n // 48)
    pos = torch.arange(n, device="cuda")
    for a, b in _some(slices, n):
        c = _randn(g, b - a, topics, D)
        z = torch.randint(0, topics, (b - a, n), generator=g, device="cuda")
        stay = _rand(g, b - a, n) < 0.9
        stay[:, :1] = False
        last = torch.where(stay, torch.zeros_like(z), pos.expand_as(z)).cummax(1).values
        k = 0.3 * _randn(g, b - a, n, D)
        k += torch.gather(c, 1, z.gather(1, last).unsqueeze(-1).expand(-1, -1, D))
        k[..., :4] *= 8.0
        out[a:b] = k
    return out


def _values(g, slices, n, dtype):
    out = torch.empty(slices, n, D, dtype=dtype, device="cuda")
    for a, b in _some(slices, n):
        out[a:b] = _randn(g, b - a, n, D)
    return out


def _gathered(g, slices, n):
    """Accumulated weights: a few rows hold most of the mass, one in twenty was never attended."""
    w = 0.05 * torch.exp(2.0 * _randn(g, slices, n))
    return w.masked_fill(_rand(g, slices, n) < 0.05, 0.0)


def _queries(g, keys, per, n_q, dtype):
    """Queries [slices][per][n_q][d] that look for a row of their slice: a key and noise."""
    s, n = keys.shape[:2]
    at = torch.randint(0, n, (s, per * n_q), generator=g, device="cuda")
    k = torch.gather(keys, 1, at.unsqueeze(-1).expand(-1, -1, D)).float()
    return (0.4 * k + _randn(g, s, per * n_q, D)).reshape(s, per, n_q, D).to(dtype)


def _prepare_attn(case, seed):
    g = _gen(seed, 1)
    dt, kv, n_q = DTYPES[case["dtype"]], case["kv_heads"], case["queries"]
    sp = case["layers"] * kv
    s = case["seqs"] * sp
    groups, per = case["seqs"] * case["layers"], case["q_heads"] // kv
    st = {"kv_heads": kv, "n_prefix": None, "k_prefix": None, "v_prefix": None}
    st["k_own"], st["v_own"] = _keys(g, s, case["own_rows"], dt), _values(g, s, case["own_rows"], dt)
    # one length for the slices of a sequence
    n = _randint(g, case["own_least"], case["own_rows"], case["seqs"], 1)
    st["n_own"] = n.expand(-1, sp).reshape(-1).contiguous()
    look = st["k_own"]
    if case["prefix"]:
        st["k_prefix"], st["v_prefix"] = _keys(g, sp, case["prefix"], dt), _values(g, sp, case["prefix"], dt)
        if case["ragged"]:
            st["n_prefix"] = _randint(g, case["prefix"] // 2, case["prefix"], sp)
        look = st["k_prefix"].repeat(case["seqs"], 1, 1) if case["prefix"] <= 4096 else None
    if look is None:       # a copy of a long prefix for every sequence would not fit: rows of its first part
        look = st["k_prefix"][:, :4096].repeat(case["seqs"], 1, 1)
    st["q"] = _queries(g, look, per, n_q, dt).reshape(groups, case["q_heads"], n_q, D)
    st["out"] = torch.zeros_like(st["q"])
    st["lse"] = torch.zeros(st["q"].shape[:3], device="cuda")
    st["weights"] = _gathered(g, s, case["own_rows"]) if case["weights"] else None
    return st


def _prepare_weights(case, seed):
    g = _gen(seed, 2)
    dt, kv, n_q, n = DTYPES[case["dtype"]], case["kv_heads"], case["queries"], case["keys"]
    per = case["q_heads"] // kv
    keys = _keys(g, kv, n, dt)
    q = _queries(g, keys, per, n_q, dt)
    lse = torch.empty(kv, per, n_q, device="cuda")
    for i in range(kv):      # a part of a head at a time: all scores of a prompt would not fit
        k = keys[i].float().t().contiguous()
        for j in range(per):
            for a, b, seen, hidden in _causal(n_q, n):
                x = torch.matmul(q[i, j, a:b].float(), k[:, :seen]) * SCALE
                lse[i, j, a:b] = torch.logsumexp(x.masked_fill(hidden, -math.inf), -1)
    return {"kv_heads": kv, "q": q.reshape(1, case["q_heads"], n_q, D), "keys": keys,
            "lse": lse.reshape(1, case["q_heads"], n_q), "weights": torch.zeros(kv, n, device="cuda")}


def _causal(n_q, n):
    """Parts of the last n_q tokens of n: (first, end, keys that the part's last query sees, those hidden from each)."""
    step = max(1, (1 << 26) // n)
    for a in range(0, n_q, step):
        b = min(n_q, a + step)
        seen = n - n_q + b
        row = n - n_q + torch.arange(a, b, device="cuda")
        yield a, b, seen, torch.arange(seen, device="cuda") > row[:, None]


def _prepare_evict(case, seed):
    g = _gen(seed, 3)
    dt, s, n, keep = DTYPES[case["dtype"]], case["slices"], case["rows"], case["keep"]
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"keep": keep, "first": case["first"], "recent": case["recent"], "weights": _gathered(g, s, n),
            "n_rows": _randint(g, case["least"], n, s), "k": _keys(g, s, n, dt), "v": _values(g, s, n, dt),
            "k_to": torch.zeros(s, keep, D, dtype=dt, device="cuda"),
            "v_to": torch.zeros(s, keep, D, dtype=dt, device="cuda"), "weights_to": torch.zeros(s, keep, device="cuda"),
            "pos_to": torch.zeros(s, keep, **i32), "n_to": torch.zeros(s, **i32)}


def _prepare_store(case, seed):
    g = _gen(seed, 4)
    dt, s, n, new = DTYPES[case["dtype"]], case["slices"], case["budget"], case["new"]
    n_rows = _randint(g, case["least"], n, s)
    n_seen = torch.where(n_rows == n, n_rows + _randint(g, 0, 5000, s), n_rows)
    # the rows hold some of the positions so far, the recent ones among them, in no order
    at = torch.arange(n, device="cuda", dtype=torch.int32).expand(s, n)
    gap = (n_seen - n_rows)[:, None]
    pos = torch.where(at < case["first"], at, at + gap)
    old = at < (n_rows - case["recent"])[:, None]
    pos = torch.where(old & (at >= case["first"]), at + (gap * _rand(g, s, 1)).to(torch.int32), pos)
    mix = torch.where(at < n_rows[:, None], _rand(g, s, n), 1.0 + at).argsort(1)
    k_new, v_new = _keys(g, s, new, dt), _values(g, s, new, dt)
    return {"budget": n, "first": case["first"], "recent": case["recent"], "k_new": k_new, "v_new": v_new,
            "k": _keys(g, s, n, dt), "v": _values(g, s, n, dt), "weights": _gathered(g, s, n),
            "pos": pos.gather(1, mix).contiguous(), "n_rows": n_rows, "n_seen": n_seen}


def prepare(case, seed):
    return {"kind": case["kind"], **{"attn": _prepare_attn, "weights": _prepare_weights, "evict": _prepare_evict,
                                     "store": _prepare_store}[case["kind"]](case, seed)}


# ------------------------------------------------------------------- plain forms

def _plain_attn(st):
    q, k_own, kv = st["q"], st["k_own"], st["kv_heads"]
    n_q, per = q.shape[2], q.shape[1] // kv
    s, rows = k_own.shape[:2]
    sp = s if st["k_prefix"] is None else st["k_prefix"].shape[0]
    seqs, m = s // sp, per * n_q
    qs = q.reshape(seqs, sp, m, D)
    out, lse = torch.empty(seqs, sp, m, D, device="cuda"), torch.empty(seqs, sp, m, device="cuda")
    weights = None if st["weights"] is None else st["weights"].view(seqs, sp, rows)
    t = torch.arange(n_q, device="cuda").repeat(per)
    at = torch.arange(rows, device="cuda")
    p_rows = 0 if st["k_prefix"] is None else st["k_prefix"].shape[1]
    # some prefix slices at a time: float32 rows and scores of all would not fit three times over
    step = max(1, (1 << 27) // max(1, seqs * (m + D) * rows + p_rows * (seqs * m + D)))
    for i in range(0, sp, step):
        j = slice(i, min(sp, i + step))
        c = j.stop - j.start
        x = qs[:, j].float()
        n = st["n_own"].view(seqs, sp)[:, j]
        ko = k_own.view(seqs, sp, rows, D)[:, j].float()
        vo = st["v_own"].view(seqs, sp, rows, D)[:, j].float()
        xo = torch.matmul(x, ko.transpose(2, 3).contiguous()) * SCALE
        live = at < (n[..., None] - n_q + t + 1)[..., None]
        xo = xo.masked_fill(~live, -math.inf)
        top = xo.amax(-1, keepdim=True)
        if p_rows:
            xp = torch.matmul(x.transpose(0, 1).reshape(c, seqs * m, D),
                              st["k_prefix"][j].float().transpose(1, 2).contiguous()) * SCALE
            if st["n_prefix"] is not None:
                gone = torch.arange(p_rows, device="cuda") >= st["n_prefix"][j][:, None]
                xp = xp.masked_fill(gone[:, None], -math.inf)
            xp = xp.view(c, seqs, m, p_rows).transpose(0, 1)
            top = torch.maximum(top, xp.amax(-1, keepdim=True))
        base = torch.where(top == -math.inf, torch.zeros_like(top), top)
        eo = torch.exp(xo - base)
        total = eo.sum(-1, keepdim=True)
        o = torch.matmul(eo, vo)
        if p_rows:
            ep = torch.exp(xp - base)
            total = total + ep.sum(-1, keepdim=True)
            o = o + torch.matmul(ep.transpose(0, 1).reshape(c, seqs * m, p_rows),
                                 st["v_prefix"][j].float()).view(c, seqs, m, D).transpose(0, 1)
        safe = torch.where(total > 0, total, torch.ones_like(total))
        out[:, j] = o / safe
        lse[:, j] = (base + torch.log(total)).squeeze(-1)
        if weights is not None:
            weights[:, j] += (eo / safe).sum(2)
    st["out"][:] = out.reshape(q.shape).to(q.dtype)
    st["lse"][:] = lse.reshape(q.shape[:3])


def _plain_weights(st):
    kv, n = st["keys"].shape[:2]
    n_q = st["q"].shape[2]
    q = st["q"].reshape(kv, -1, n_q, D)
    lse = st["lse"].reshape(kv, -1, n_q)
    for i in range(kv):
        k = st["keys"][i].float().t().contiguous()
        total = torch.zeros(n, device="cuda", dtype=torch.float64)     # sums over a whole prompt's queries
        for j in range(q.shape[1]):
            for a, b, seen, hidden in _causal(n_q, n):
                x = torch.matmul(q[i, j, a:b].float(), k[:, :seen]) * SCALE - lse[i, j, a:b, None]
                total[:seen] += torch.exp(x).masked_fill(hidden, 0.0).sum(0, dtype=torch.float64)
        st["weights"][i] = (st["weights"][i].double() + total).float()


def _kept(weights, pos, n_rows, n_seen, n_keep, first, recent):
    """For the rows of smaller caches the row that each is taken from [slices][max rows], and how many there are."""
    s, n = weights.shape
    at = torch.arange(n, device="cuda")
    live = at < n_rows[:, None]
    safe = (pos < first) | (pos >= (n_seen - recent)[:, None])
    key = weights.masked_fill(safe, math.inf).masked_fill(~live, -math.inf)
    # largest first, of equal ones the higher row
    order = n - 1 - key.flip(1).sort(dim=1, descending=True, stable=True).indices
    m = torch.minimum(n_rows, n_keep).long()
    kept = torch.zeros(s, n, dtype=torch.bool, device="cuda").scatter_(1, order, at < m[:, None])
    hole = ~kept & (at < m[:, None])
    late = kept & (at >= m[:, None])
    movers = torch.where(late, at, n).sort(1).values             # the kept rows from m on, ascending
    rank = (hole.cumsum(1) - 1).clamp(min=0)
    return torch.where(hole, movers.gather(1, rank), at), m


def _plain_evict(st):
    s, n = st["weights"].shape
    pos = torch.arange(n, device="cuda", dtype=torch.int32).expand(s, n)
    src, m = _kept(st["weights"], pos, st["n_rows"], st["n_rows"], torch.full_like(st["n_rows"], st["keep"]),
                   st["first"], st["recent"])
    src = src[:, :st["keep"]]
    live = torch.arange(src.shape[1], device="cuda") < m[:, None]
    src = torch.where(live, src, torch.zeros_like(src))
    rows = src.unsqueeze(-1).expand(-1, -1, D)
    st["k_to"][:] = torch.where(live.unsqueeze(-1), torch.gather(st["k"], 1, rows), st["k_to"])
    st["v_to"][:] = torch.where(live.unsqueeze(-1), torch.gather(st["v"], 1, rows), st["v_to"])
    st["weights_to"][:] = torch.where(live, torch.gather(st["weights"], 1, src), st["weights_to"])
    st["pos_to"][:] = torch.where(live, torch.gather(pos, 1, src), st["pos_to"])
    st["n_to"][:] = m.to(torch.int32)


def _plain_store(st):
    s, new = st["k_new"].shape[:2]
    n = st["weights"].shape[1]
    src, m = _kept(st["weights"], st["pos"], st["n_rows"], st["n_seen"],
                   torch.full_like(st["n_rows"], st["budget"] - new), st["first"], st["recent"])
    src = torch.where(torch.arange(n, device="cuda") < m[:, None], src, torch.arange(n, device="cuda"))
    fresh = m[:, None] + torch.arange(new, device="cuda")
    # only rows that change are written: at most as many as leave
    changed = src != torch.arange(n, device="cuda")
    most = min(n, max(1, new + max(0, n - st["budget"])))
    at = changed.to(torch.int8).sort(dim=1, descending=True, stable=True).indices[:, :most]
    take = src.gather(1, at)
    for name, x in (("k", st["k_new"]), ("v", st["v_new"])):
        moved = torch.gather(st[name], 1, take.unsqueeze(-1).expand(-1, -1, D))
        st[name].scatter_(1, at.unsqueeze(-1).expand(-1, -1, D), moved)
        st[name].scatter_(1, fresh.unsqueeze(-1).expand(-1, -1, D), x)
    st["weights"].scatter_(1, at, torch.gather(st["weights"], 1, take))
    st["weights"].scatter_(1, fresh, 0.0)
    st["pos"].scatter_(1, at, torch.gather(st["pos"], 1, take))
    st["pos"].scatter_(1, fresh, st["n_seen"][:, None] + torch.arange(new, device="cuda", dtype=torch.int32))
    st["n_rows"][:] = (m + new).to(torch.int32)
    st["n_seen"] += new


# ------------------------------------------------------------------- one pass

def run(state):
    st = state
    if own:
        from paper_2510_11292_amd import louiskv as L
    if st["kind"] == "attn":
        if own:
            L.shared_prefix_attn(st["q"], st["kv_heads"], st["k_prefix"], st["v_prefix"], st["n_prefix"], st["k_own"],
                                 st["v_own"], st["n_own"], st["out"], st["lse"], weights=st["weights"])
        else:
            _plain_attn(st)
        return {k: st[k] for k in ("out", "lse", "weights") if st[k] is not None}
    if st["kind"] == "weights":
        if own:
            L.attn_weights(st["q"], st["kv_heads"], st["keys"], None, st["lse"], st["weights"])
        else:
            _plain_weights(st)
        return {"weights": st["weights"]}
    if st["kind"] == "evict":
        if own:
            L.evict_rows(st["weights"], None, st["n_rows"], None, st["keep"], st["first"], st["recent"], st["k"],
                         st["v"], st["k_to"], st["v_to"], st["weights_to"], st["pos_to"], st["n_to"])
        else:
            _plain_evict(st)
        return {k: st[k] for k in ("k_to", "v_to", "weights_to", "pos_to", "n_to")}
    if own:
        L.store_evict(st["k_new"], st["v_new"], st["k"], st["v"], st["weights"], st["pos"], st["n_rows"],
                      st["n_seen"], st["budget"], st["first"], st["recent"])
    else:
        _plain_store(st)
    return {k: st[k] for k in ("k", "v", "weights", "pos", "n_rows", "n_seen")}


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    row = 2 * D * size                       # a key and its value
    if case["kind"] == "attn":
        sp = case["layers"] * case["kv_heads"]
        s, m = case["seqs"] * sp, case["q_heads"] // case["kv_heads"] * case["queries"]
        n = (case["own_least"] + case["own_rows"]) / 2
        p = case["prefix"] * (0.75 if case["ragged"] else 1)
        pairs = s * m * (p + n - (case["queries"] - 1) / 2)
        return {"bytes": sp * p * row + s * n * (row + (8 if case["weights"] else 0)) + s * m * (2 * D * size + 4),
                "flops": 4 * D * pairs}
    if case["kind"] == "weights":
        n, n_q, kv = case["keys"], case["queries"], case["kv_heads"]
        pairs = case["q_heads"] * (n_q * (n - n_q) + n_q * (n_q + 1) / 2)
        return {"bytes": kv * n * (D * size + 8) + case["q_heads"] * n_q * (D * size + 4), "flops": 2 * D * pairs}
    if case["kind"] == "evict":
        n = (case["least"] + case["rows"]) / 2
        kept = min(n, case["keep"])
        return {"bytes": case["slices"] * (4 * n + kept * (2 * row + 8)), "flops": 0}
    n = (case["least"] + case["budget"]) / 2
    # weights and positions are read, the new rows written, and as many moved as leave
    return {"bytes": case["slices"] * (8 * n + case["new"] * (2 * row + 8) + max(0, n + case["new"] - case["budget"])
                                       * (2 * row + 16)), "flops": 0}


# ------------------------------------------------------------------- 64 bits

def _exact_attn(case, st):
    kv, n_q = case["kv_heads"], case["queries"]
    per, s = case["q_heads"] // kv, st["k_own"].shape[0]
    q = st["q"].double().reshape(s, per, n_q, D)
    out, lse = torch.zeros_like(q), torch.full((s, per, n_q), -math.inf, dtype=torch.float64, device="cuda")
    weights = None if st["weights"] is None else st["weights"].double()
    lengths = st["n_own"].tolist()
    sp = case["layers"] * kv
    p_len = [0] * sp if not case["prefix"] else \
        [case["prefix"]] * sp if st["n_prefix"] is None else st["n_prefix"].tolist()
    prefix = {}
    for i in sorted(range(s), key=lambda i: i % sp):
        c, n = i % sp, lengths[i]
        if c not in prefix:
            prefix = {c: [st[x][c, :p_len[c]].double() if p_len[c] else torch.zeros(0, D, dtype=torch.float64,
                                                                                   device="cuda")
                          for x in ("k_prefix", "v_prefix")]}
        k = torch.cat((prefix[c][0], st["k_own"][i, :n].double()))
        v = torch.cat((prefix[c][1], st["v_own"][i, :n].double()))
        x = torch.matmul(q[i], k.t()) / math.sqrt(D)
        last = p_len[c] + n - n_q + torch.arange(n_q, device="cuda")
        x = torch.where(torch.arange(len(k), device="cuda") <= last[:, None], x, torch.full_like(x, -math.inf))
        e = torch.logsumexp(x, -1)
        p = torch.exp(x - torch.where(torch.isinf(e), torch.zeros_like(e), e).unsqueeze(-1))
        out[i], lse[i] = torch.matmul(p, v), e
        if weights is not None:
            weights[i, :n] += p[..., p_len[c]:].sum((0, 1))
    r = {"out": out.reshape(st["q"].shape), "lse": lse.reshape(st["q"].shape[:3])}
    return r if weights is None else {**r, "weights": weights}


def _exact_weights(case, st):
    kv, n, n_q = case["kv_heads"], case["keys"], case["queries"]
    q, lse = st["q"].reshape(kv, -1, n_q, D), st["lse"].reshape(kv, -1, n_q)
    weights = st["weights"].double()
    step = max(1, (1 << 25) // n)
    for i in range(kv):
        k = st["keys"][i].double().t().contiguous()
        for j in range(q.shape[1]):
            for b in range(n_q, 0, -step):
                a, seen = max(0, b - step), n - n_q + b
                e = torch.exp(torch.matmul(q[i, j, a:b].double() / math.sqrt(D), k[:, :seen])
                              - lse[i, j, a:b, None].double())
                weights[i, :seen] += torch.tril(e, diagonal=n - n_q + a).sum(0)
    return {"weights": weights}


def _rows_that_stay(w, pos, n, n_seen, keep, first, recent):
    """Rows 0 .. m - 1 of the smaller cache as the rows that they are taken from, a slice's weights on the host."""
    m = min(n, keep)
    safe = (pos[:n] < first) | (pos[:n] >= n_seen - recent)
    # the last key decides first: protected rows, then weights, then row numbers, largest last
    order = np.lexsort((np.arange(n), w[:n], safe))
    stay = np.sort(order[n - m:])
    src = np.arange(m)
    src[np.setdiff1d(src, stay)] = stay[stay >= m]
    return src


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(case, st)
    if case["kind"] == "weights":
        return _exact_weights(case, st)
    w, n_rows = st["weights"].double().cpu().numpy(), st["n_rows"].tolist()
    if case["kind"] == "evict":
        # the rows come as they are: 64-bit copies of all would not fit beside each other
        out = {k: st[k].clone() for k in ("k_to", "v_to", "weights_to", "pos_to", "n_to")}
        for i, n in enumerate(n_rows):
            src = _rows_that_stay(w[i], np.arange(n), n, n, case["keep"], case["first"], case["recent"])
            at = torch.from_numpy(src).cuda()
            for to, x in (("k_to", st["k"][i]), ("v_to", st["v"][i]), ("weights_to", st["weights"][i])):
                out[to][i, :len(at)] = x[at]
            out["pos_to"][i, :len(at)] = at.to(torch.int32)
            out["n_to"][i] = len(at)
        return out
    out = {k: st[k].clone() for k in ("k", "v", "weights", "pos", "n_rows", "n_seen")}
    pos, seen, new = st["pos"].cpu().numpy(), st["n_seen"].tolist(), case["new"]
    for i, n in enumerate(n_rows):
        src = _rows_that_stay(w[i], pos[i], n, seen[i], case["budget"] - new, case["first"], case["recent"])
        m = len(src)
        to = np.flatnonzero(src != np.arange(m))
        a, b = torch.from_numpy(to).cuda(), torch.from_numpy(src[to]).cuda()
        for x in ("k", "v", "weights", "pos"):
            out[x][i, a] = st[x][i, b]
        out["k"][i, m:m + new], out["v"][i, m:m + new] = st["k_new"][i], st["v_new"][i]
        out["weights"][i, m:m + new] = 0.0
        out["pos"][i, m:m + new] = seen[i] + torch.arange(new, device="cuda", dtype=torch.int32)
        out["n_rows"][i], out["n_seen"][i] = m + new, seen[i] + new
    return out
