"""The cache that keeps the rows of most attention weight: rows that stay, their moves and new rows, exact."""
import numpy as np
import pytest
import torch

from oracle import prefix as op

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"
I32 = dict(dtype=torch.int32, device=DEV)


def L():
    from paper_2510_11292_amd import louiskv
    return louiskv


def bits(t):
    """A tensor's bytes, so that NaN compares."""
    return t.contiguous().view(torch.uint8)


def weights_of(kind, rng, s, n):
    w = np.exp(2 * rng.standard_normal((s, n))).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 4, (s, n)).astype(np.float32)
        w[w == 3] = 0.0
        w[rng.random((s, n)) < 0.1] = -0.0
    elif kind == "bad":
        for v in (np.nan, np.inf, -np.inf, -1.5, 0.0, 1e-42):
            w[rng.random((s, n)) < 0.12] = v
        w.view(np.uint32)[rng.random((s, n)) < 0.05] = 0xffffffff      # another NaN
    elif kind == "same":
        w[:] = 0.25
    return w


class Cache:
    def __init__(self, s, rows, dtype, kind="any", seed=0, least=0, spread=True):
        rng = np.random.default_rng(seed + rows)
        gen = torch.Generator(device=DEV).manual_seed(rows + seed)
        self.s, self.rows = s, rows
        self.k, self.v = (torch.randn(s, rows, 128, generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))
        self.n = rng.integers(least, rows + 1, s)
        self.n[0] = rows
        self.seen = self.n + (rng.integers(0, 50, s) if spread else 0)
        self.pos = np.full((s, rows), -7, dtype=np.int32)
        for i in range(s):
            self.pos[i, :self.n[i]] = rng.permutation(rng.choice(self.seen[i], self.n[i], replace=False)) if self.n[i] else []
        self.w = weights_of(kind, rng, s, rows)
        self.gpu()

    def gpu(self):
        self.wt, self.pt = torch.from_numpy(self.w).to(DEV), torch.from_numpy(self.pos).to(DEV)
        self.nt = torch.from_numpy(self.n.astype(np.int32)).to(DEV)
        self.st = torch.from_numpy(self.seen.astype(np.int32)).to(DEV)


EVICT = [  # slices, rows, keep, rows_to, first, recent
    (1, 1, 1, 1, 0, 0), (2, 5, 3, 3, 1, 1), (3, 64, 64, 70, 4, 16), (5, 300, 129, 129, 0, 64), (4, 1000, 7, 20, 3, 4),
    (2, 2049, 1024, 1024, 4, 128), (3, 777, 900, 1000, 4, 32), (70, 90, 33, 33, 2, 5), (2, 40000, 2048, 2048, 4, 128),
    (1, 70001, 69000, 69000, 1, 1000), (2, 33000, 32500, 32501, 0, 0),
]


@pytest.mark.parametrize("kind", ["any", "ties", "bad", "same"])
@pytest.mark.parametrize("case", EVICT, ids=["-".join(map(str, c)) for c in EVICT])
def test_eviction(kind, case):
    s, rows, keep, rows_to, first, recent = case
    for dtype in ("bf16", "f32") if rows < 3000 else ("bf16",):
        for with_pos in (True, False):
            c = Cache(s, rows, dtype, kind)
            if not with_pos:
                c.pos = np.tile(np.arange(rows, dtype=np.int32), (s, 1))
            dt = DT[dtype]
            k_to, v_to = (torch.full((s, rows_to, 128), 7.0, dtype=dt, device=DEV) for _ in range(2))
            w_to, p_to = torch.full((s, rows_to), 7.0, device=DEV), torch.full((s, rows_to), -9, **I32)
            n_to = torch.full((s,), -9, **I32)
            print(case, kind, dtype, with_pos, flush=True)
            L().evict_rows(c.wt, c.pt if with_pos else None, c.nt, c.st if with_pos else None, keep, first, recent, c.k,
                           c.v, k_to, v_to, w_to, p_to, n_to)
            # the same in place
            ki, vi, wi, ni = c.k.clone(), c.v.clone(), c.wt.clone(), c.nt.clone()
            pi = c.pt.clone() if with_pos else torch.full((s, rows), -9, **I32)
            in_place = keep <= rows
            if in_place:
                L().evict_rows(wi, pi if with_pos else None, ni, c.st if with_pos else None, keep, first, recent, ki, vi, ki,
                               vi, wi, pi, ni)
            for i in range(s):
                n = int(c.n[i])
                src = op.rows_that_stay(c.w[i], c.pos[i], n, int(c.seen[i]) if with_pos else n, keep, first, recent)
                m, at = len(src), torch.tensor(src, dtype=torch.long, device=DEV)
                assert int(n_to[i]) == m == min(n, keep)
                want_pos = torch.from_numpy(c.pos[i]).to(DEV)[at]
                for got, x in ((k_to, c.k), (v_to, c.v), (w_to, c.wt)):
                    assert torch.equal(bits(got[i, :m]), bits(x[i][at])), i
                    assert (got[i, m:] == 7).all()
                assert torch.equal(p_to[i, :m], want_pos) and (p_to[i, m:] == -9).all()
                if in_place:
                    assert int(ni[i]) == m
                    for got, x in ((ki, c.k), (vi, c.v), (wi, c.wt)):
                        assert torch.equal(bits(got[i, :m]), bits(x[i][at])), i
                        assert torch.equal(bits(got[i, m:]), bits(x[i, m:]))
                    assert torch.equal(pi[i, :m], want_pos)
                    assert torch.equal(pi[i, m:], c.pt[i, m:]) if with_pos else (pi[i, m:] == -9).all()


def test_all_rows_without_lengths_and_optional_outputs():
    c = Cache(2, 100, "bf16")
    k_to, v_to = torch.zeros(2, 30, 128, device=DEV).bfloat16(), torch.zeros(2, 30, 128, device=DEV).bfloat16()
    n_to = torch.zeros(2, **I32)
    L().evict_rows(c.wt, None, None, None, 30, 1, 2, c.k, c.v, k_to, v_to, None, None, n_to)
    assert n_to.tolist() == [30, 30]
    for i in range(2):
        src = op.rows_that_stay(c.w[i], list(range(100)), 100, 100, 30, 1, 2)
        assert torch.equal(k_to[i], c.k[i][src]) and torch.equal(v_to[i], c.v[i][src])


def test_more_protected_rows_than_are_kept():
    """Positions that repeat can protect more rows than fit: the higher ones stay."""
    c = Cache(1, 50, "f32", least=50)
    c.pt.fill_(3)
    n_to = torch.zeros(1, **I32)
    k = c.k.clone()
    L().evict_rows(c.wt, c.pt, None, c.st, 10, 9, 0, c.k, c.v, c.k, c.v, c.wt, c.pt, n_to)
    assert torch.equal(c.k[0, :10], k[0, 40:]) and int(n_to) == 10


STORE = [  # slices, rows, budget, new, first, recent
    (1, 1, 1, 1, 0, 0), (2, 3, 2, 1, 0, 1), (3, 70, 64, 1, 4, 16), (4, 300, 300, 5, 1, 40), (2, 20, 9, 9, 0, 0),
    (5, 1000, 777, 64, 4, 128), (2, 2048, 2048, 1, 4, 128), (1, 9000, 8192, 33, 2, 100), (2, 40000, 40000, 1, 4, 128),
    (1, 40001, 39000, 7, 4, 128), (600, 40, 33, 2, 1, 3),
]


@pytest.mark.parametrize("kind", ["any", "ties", "bad"])
@pytest.mark.parametrize("case", STORE, ids=["-".join(map(str, c)) for c in STORE])
def test_store(kind, case):
    s, rows, budget, new, first, recent = case
    for dtype in ("bf16", "f32") if rows < 3000 else ("bf16",):
        c = Cache(s, rows, dtype, kind, seed=3)       # some caches hold more rows than the budget, some fewer
        gen = torch.Generator(device=DEV).manual_seed(1)
        for step in range(3):
            kn, vn = (torch.randn(s, new, 128, generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))
            before = [x.clone() for x in (c.k, c.v, c.wt, c.pt)]
            print(case, kind, dtype, step, flush=True)
            L().store_evict(kn if new > 1 or step else kn[:, 0].contiguous(), vn if new > 1 or step else vn[:, 0].contiguous(),
                            c.k, c.v, c.wt, c.pt, c.nt, c.st, budget, first, recent)
            for i in range(s):
                n, seen = int(c.n[i]), int(c.seen[i])
                src = op.rows_that_stay(c.w[i], c.pos[i], n, seen, budget - new, first, recent)
                m, at = len(src), torch.tensor(src, dtype=torch.long, device=DEV)
                pos = torch.arange(seen, seen + new, **I32)
                for got, x, y in ((c.k, before[0], kn[i]), (c.v, before[1], vn[i]), (c.wt, before[2], torch.zeros(new, device=DEV)),
                                  (c.pt, before[3], pos)):
                    assert torch.equal(bits(got[i, :m]), bits(x[i][at])), (i, step)
                    assert torch.equal(bits(got[i, m:m + new]), bits(y))
                    assert torch.equal(bits(got[i, m + new:]), bits(x[i, m + new:]))
                c.n[i], c.seen[i] = m + new, seen + new
            assert torch.equal(c.nt.cpu(), torch.from_numpy(c.n.astype(np.int32)))
            assert torch.equal(c.st.cpu(), torch.from_numpy(c.seen.astype(np.int32)))
            c.w, c.pos = c.wt.cpu().numpy(), c.pt.cpu().numpy()


def test_long_buffers():
    """Rows past two gigabytes."""
    s, rows = 300, 40000
    k = torch.zeros(s, rows, 128, dtype=torch.bfloat16, device=DEV)
    k[-1] = torch.randn(rows, 128, device=DEV)
    w, pos = torch.rand(s, rows, device=DEV), torch.arange(rows, **I32).expand(s, rows).contiguous()
    k_to, v_to = torch.zeros(s, 64, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(s, 64, 128, dtype=torch.bfloat16, device=DEV)
    n = torch.zeros(s, **I32)
    L().evict_rows(w, None, None, None, 64, 1, 2, k, k.clone(), k_to, v_to, None, None, n)
    src = op.rows_that_stay(w[-1].tolist(), list(range(rows)), rows, rows, 64, 1, 2)
    assert torch.equal(k_to[-1], k[-1][src]) and torch.equal(v_to[-1], k[-1][src])
    n_rows, seen = torch.full((s,), rows, **I32), torch.full((s,), rows, **I32)
    new = torch.randn(s, 128, device=DEV).bfloat16()
    ref, v = k[-1].clone(), k.clone()
    L().store_evict(new, new, k, v, w, pos, n_rows, seen, rows, 1, 2)
    gone = int(torch.nonzero(pos[-1] == rows - 1)[0])        # where the last row went
    ref[gone], ref[-1] = ref[rows - 1].clone(), new[-1]
    assert torch.equal(k[-1], ref) and torch.equal(v[-1], ref)


def test_replayed_store_enters_the_next_token():
    """The counts are on the device: every replay of a captured store and attention is the next step."""
    l = L()
    s, rows, budget, kv, g = 4, 40, 33, 2, 4

    def state():
        return dict(k=torch.zeros(s, rows, 128, device=DEV).bfloat16(), v=torch.zeros(s, rows, 128, device=DEV).bfloat16(),
                    w=torch.zeros(s, rows, device=DEV), pos=torch.zeros(s, rows, **I32), n=torch.zeros(s, **I32),
                    seen=torch.zeros(s, **I32), new=torch.zeros(s, 128, device=DEV).bfloat16(),
                    q=torch.zeros(2, kv * g, 128, device=DEV).bfloat16(), out=torch.zeros(2, kv * g, 128, device=DEV).bfloat16())

    def step(x, stream=None):
        l.store_evict(x["new"], x["new"], x["k"], x["v"], x["w"], x["pos"], x["n"], x["seen"], budget, 1, 4, stream=stream)
        l.shared_prefix_attn(x["q"], kv, None, None, None, x["k"], x["v"], x["n"], x["out"], weights=x["w"], stream=stream)
    eager, captured, other = state(), state(), state()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(captured)
    for t in range(60):
        new, q = torch.randn(s, 128, device=DEV).bfloat16(), torch.randn(2, kv * g, 128, device=DEV).bfloat16()
        for x in (eager, captured, other):
            x["new"].copy_(new)
            x["q"].copy_(q)
        torch.cuda.synchronize()
        step(eager)
        step(other, side)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(bits(eager[name]), bits(captured[name])) and torch.equal(bits(eager[name]), bits(other[name])), (t, name)
        assert (eager["n"] == min(t + 1, budget)).all() and (eager["seen"] == t + 1).all()
    pos = eager["pos"][:, :budget]
    for i in range(s):
        held = set(pos[i].tolist())
        assert len(held) == budget and 0 in held and set(range(56, 60)) <= held


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_branches_with_bounded_caches_together(dtype):
    """A prompt that is cut down to its heaviest rows, shared by three sequences whose own caches evict: every step
    against plain attention over the rows that the rules leave."""
    l, dt = L(), DT[dtype]
    kv, g, n, keep, seqs, budget, first, recent = 2, 4, 200, 90, 3, 24, 1, 6
    s = seqs * kv
    gen = torch.Generator(device=DEV).manual_seed(5)

    def rnd(*shape):
        return torch.randn(*shape, generator=gen, device=DEV).to(dt)
    keys, values, q = rnd(kv, n, 128), rnd(kv, n, 128), rnd(1, kv * g, n, 128)
    out, lse = torch.zeros_like(q), torch.zeros(1, kv * g, n, device=DEV)
    w = torch.zeros(kv, n, device=DEV)
    l.shared_prefix_attn(q, kv, None, None, None, keys, values, None, out, lse, weights=w)
    w2 = torch.zeros_like(w)
    l.attn_weights(q, kv, keys, None, lse, w2)
    assert (w - w2).abs().max() <= 1e-4 * w.max() and abs(float(w.double().sum()) / (kv * g * n) - 1) < 1e-4
    kp, vp, n_p = torch.zeros(kv, keep, 128, device=DEV, dtype=dt), torch.zeros(kv, keep, 128, device=DEV, dtype=dt), torch.zeros(kv, **I32)
    l.evict_rows(w2, None, None, None, keep, 4, 16, keys, values, kp, vp, None, None, n_p)
    stay = [op.rows_that_stay(w2[i].tolist(), list(range(n)), n, n, keep, 4, 16) for i in range(kv)]
    ko, vo = torch.zeros(s, budget, 128, device=DEV, dtype=dt), torch.zeros(s, budget, 128, device=DEV, dtype=dt)
    wo, pos, rows, seen = torch.zeros(s, budget, device=DEV), torch.zeros(s, budget, **I32), torch.zeros(s, **I32), torch.zeros(s, **I32)
    history = []
    o = torch.zeros(seqs, kv * g, 128, device=DEV, dtype=torch.float32)
    acc = [dict() for _ in range(s)]                    # position -> accumulated weight, kept by hand
    for t in range(45):
        qt, kt, vt = rnd(seqs, kv * g, 128), rnd(s, 128), rnd(s, 128)
        history.append((kt, vt))
        before = [sorted(pos[i, :int(rows[i])].tolist()) for i in range(s)]
        l.store_evict(kt, vt, ko, vo, wo, pos, rows, seen, budget, first, recent)
        l.shared_prefix_attn(qt, kv, kp, vp, n_p, ko, vo, rows, o, weights=wo)
        for i in range(s):
            held = pos[i, :int(rows[i])].tolist()
            gone = set(before[i]) - set(held)
            assert len(gone) == (t >= budget) and held[-1] == t
            for x in gone:      # the lightest that is not protected; weights that are nearly equal may go either way
                free = [v for p_, v in acc[i].items() if first <= p_ < t - recent]
                assert first <= x < t - recent and acc[i].pop(x) <= min(free) * (1 + 1e-2) + 1e-6
            c = i % kv
            k = torch.cat([keys[c][stay[c]]] + [history[p_][0][i:i + 1] for p_ in held]).double()
            v = torch.cat([values[c][stay[c]]] + [history[p_][1][i:i + 1] for p_ in held]).double()
            qi = qt.view(s, g, 128)[i].double()
            p = torch.softmax(qi @ k.t().contiguous() * 128 ** -0.5, -1)
            # the weights' rounding to bfloat16 (2^-8 of each), float32 else
            tol = (2.0 ** -8 if dtype == "bf16" else 1e-5) * (p @ v.abs())
            assert ((o.view(s, g, 128)[i].double() - p @ v).abs() <= tol + 1e-5).all(), (t, i)
            for j, p_ in enumerate(held):
                acc[i][p_] = acc[i].get(p_, 0.0) + float(p[:, keep + j].sum())
            got = torch.tensor([acc[i][p_] for p_ in held], device=DEV)
            assert (wo[i, :len(held)] - got).abs().max() < 1e-4, (t, i)


def lightest(w, pos, seen, first, recent, k):
    """The k rows of least weight of each slice of unprotected rows, in ascending order (weights all different)."""
    safe = (pos < first) | (pos >= seen[:, None] - recent)
    return torch.topk(w.masked_fill(safe, float("inf")), k, dim=1, largest=False).indices.sort(1).values


def test_a_store_to_all_layers_of_many_branches():
    """16384 slices (64 branches of 32 layers and 8 KV heads) of 2048 rows: their caches are full, one row of each leaves."""
    s, rows = 16384, 2048
    gen = torch.Generator(device=DEV).manual_seed(11)
    k = torch.zeros(s, rows, 128, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    k[:, :, 0] = torch.arange(rows, device=DEV) % 256
    k[:, :, 1] = torch.arange(rows, device=DEV) // 256
    v[:, :, 5] = k[:, :, 0] + 1
    w = torch.rand(s, rows, generator=gen, device=DEV)
    pos = torch.arange(rows, **I32).expand(s, -1).contiguous()
    n, seen = torch.full((s,), rows, **I32), torch.full((s,), rows, **I32)
    gone = lightest(w, pos, seen, 4, 128, 1)[:, 0]
    kn, vn = torch.full((s, 128), 3.0, device=DEV).bfloat16(), torch.full((s, 128), 4.0, device=DEV).bfloat16()
    L().store_evict(kn, vn, k, v, w, pos, n, seen, rows, 4, 128)
    assert (n == rows).all() and (seen == rows + 1).all()
    # the last row takes the place of the one that leaves, the new one comes behind
    want = torch.arange(rows, device=DEV).expand(s, -1).clone()
    want[torch.arange(s, device=DEV), gone] = rows - 1
    want[:, rows - 1] = rows
    assert torch.equal(pos.long(), want) and (w[:, -1] == 0).all()
    held = want[:, :-1]
    assert torch.equal(k[:, :-1, 0].long(), held % 256) and torch.equal(k[:, :-1, 1].long(), held // 256)
    assert torch.equal(v[:, :-1, 5].long(), held % 256 + 1)
    assert (k[:, -1] == 3).all() and (v[:, -1] == 4).all()


def test_eviction_of_a_few_rows_of_many_long_slices():
    """1024 slices of 32768 rows, of which all but 5 stay: some million blocks move rows."""
    s, rows, keep = 1024, 32768, 32763
    gen = torch.Generator(device=DEV).manual_seed(12)
    k = torch.zeros(s, rows, 128, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    k[:, :, 0] = torch.arange(rows, device=DEV) % 256
    v[:, :, 7] = torch.arange(rows, device=DEV) // 256
    w = torch.stack([torch.randperm(rows, generator=gen, device=DEV) for _ in range(s)]).float()
    pos = torch.arange(rows, **I32).expand(s, -1).contiguous()
    n = torch.full((s,), rows, **I32)
    gone = lightest(w, pos, n, 4, 128, 5)                  # none of the last 128 rows leaves
    L().evict_rows(w, pos, n, n.clone(), keep, 4, 128, k, v, k, v, w, pos, n)
    assert (n == keep).all()
    want = torch.arange(keep, device=DEV).expand(s, -1).clone()
    want.scatter_(1, gone, torch.arange(keep, rows, device=DEV).expand(s, -1).contiguous())
    assert torch.equal(pos[:, :keep].long(), want)
    assert torch.equal(k[:, :keep, 0].long(), want % 256) and torch.equal(v[:, :keep, 7].long(), want // 256)
