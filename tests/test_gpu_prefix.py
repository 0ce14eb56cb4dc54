"""Attention over a shared prefix and own rows, and the weight that queries give to keys, against the float64 oracle.

Weights: a softmax weight exp(x - lse) is off by the fractions that attn_bounds states for x and for lse; both in
base 2 another 2^-24 of their size each, and the exponential two steps.  N of them are added up in float32 to what was
there: N 2^-24 of the sum at most, and one rounding of the result.
"""
import numpy as np
import pytest
import torch

from attn_bounds import U, attention_bounds, check_attention
from oracle import blocks as ob
from oracle import prefix as op

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"
SCALE = 128 ** -0.5


def L():
    from paper_2510_11292_amd import louiskv
    return louiskv


def n64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def weight_tolerance(before, added, size, lse, n_rows, n_queries):
    """size: largest sum |q k| * scale of the keys; lse: largest |lse| of the queries that see them; n_rows: that a
    query's own softmax runs over."""
    frac = 3 * 140 * U * size + (3 * n_rows + 48) * U + 8 * U * lse + n_queries * U
    return frac * added + 2 * U * (np.abs(before) + added) + 1e-37


class Problem:
    """Sequences over a prefix: kv KV heads of g query heads, rows behind the lengths NaN."""

    def __init__(self, seqs, layers, kv, g, n_q, prefix, rows, dtype, seed=0, ragged=True, weights=True):
        gen = torch.Generator(device=DEV).manual_seed(seed + 7 * rows + prefix)
        rng = np.random.default_rng(seed + rows)
        self.seqs, self.kv, self.g, self.n_q, self.dt = seqs, kv, g, n_q, DT[dtype]
        self.sp, self.s = layers * kv, seqs * layers * kv
        self.q = (2 * torch.randn(seqs * layers, kv * g, n_q, 128, generator=gen, device=DEV)).to(self.dt)

        def buf(s, n):
            return torch.randn(s, n, 128, generator=gen, device=DEV).to(self.dt)
        self.kp, self.vp = (buf(self.sp, prefix), buf(self.sp, prefix)) if prefix else (None, None)
        self.ko, self.vo = (buf(self.s, rows), buf(self.s, rows)) if rows else (None, None)
        self.n_p = self.n_o = None
        self.len_p, self.len_o = np.full(self.sp, prefix), np.full(self.s, rows)
        if ragged and prefix:
            self.len_p = rng.integers(0, prefix + 1, self.sp)
            self.len_p[rng.integers(0, self.sp)] = prefix
            self.n_p = torch.from_numpy(self.len_p.astype(np.int32)).to(DEV)
        if ragged and rows:
            self.len_o = rng.integers(0, rows + 1, self.s)
            self.len_o[-1], self.len_o[0] = rows, min(rows, n_q // 2)
            self.n_o = torch.from_numpy(self.len_o.astype(np.int32)).to(DEV)
        for n, *bufs in ((self.len_p, self.kp, self.vp), (self.len_o, self.ko, self.vo)):
            for b in bufs:
                for i in range(len(n) if b is not None else 0):
                    b[i, int(n[i]):] = float("nan")
        self.w = torch.rand(self.s, rows, generator=gen, device=DEV) if weights and rows else None

    def run(self, odt=None, weights="own", **kw):
        out = torch.full(self.q.shape, 7.0, dtype=odt or self.dt, device=DEV)
        lse = torch.full(self.q.shape[:3], 7.0, device=DEV)
        w = self.w.clone() if weights == "own" and self.w is not None else None
        L().shared_prefix_attn(self.q, self.kv, self.kp, self.vp, self.n_p, self.ko, self.vo, self.n_o, out, lse,
                               weights=w, **kw)
        return out, lse, w

    def rows_of(self, i):
        """(keys, values, see [queries of a head][keys], prefix rows) of slice i."""
        p, n = int(self.len_p[i % self.sp]), int(self.len_o[i])
        none = np.zeros((0, 128))
        k = np.concatenate([n64(self.kp[i % self.sp, :p]) if p else none, n64(self.ko[i, :n]) if n else none])
        v = np.concatenate([n64(self.vp[i % self.sp, :p]) if p else none, n64(self.vo[i, :n]) if n else none])
        return k, v, np.arange(p + n)[None] <= p + n - self.n_q + np.arange(self.n_q)[:, None], p

    def check(self, out, lse, w, slices=None):
        on, ln = n64(out).reshape(self.s, self.g, self.n_q, 128), n64(lse).reshape(self.s, self.g, self.n_q)
        q = n64(self.q).reshape(on.shape)
        worst = 0.0
        for i in range(self.s) if slices is None else slices:
            k, v, see, p = self.rows_of(i)
            see[:, :p] = True
            added, size, top = np.zeros(len(k)), np.zeros(len(k)), 0.0
            for j in range(self.g):
                want = ob.masked_attention(q[i, j], k, v, see, SCALE)
                worst = max(worst, check_attention(on[i, j], ln[i, j], want, self.dt == torch.bfloat16,
                                                   out.dtype == torch.bfloat16, len(k)))
                a, b = op.row_weights(q[i, j], k, see, want[1], SCALE)
                added, size = added + a, np.maximum(size, b)
                top = max([top] + list(np.abs(want[1][np.isfinite(want[1])])))
            if w is not None:
                n, before = len(k) - p, n64(self.w[i])
                got = n64(w[i])
                tol = weight_tolerance(before[:n], added[p:], max([0.0] + list(size)), top, len(k), self.g * self.n_q)
                err = np.abs(got[:n] - before[:n] - added[p:])
                assert (err <= tol).all(), f"weights of slice {i}: {(err / tol).max():.3g} of the bound"
                worst = max([worst] + list(err / tol))
                assert np.array_equal(got[n:], before[n:]), "weights behind the last row"
        return worst


ATTN = [  # seqs, layers, kv, g, n_q, prefix, rows
    (1, 1, 1, 1, 1, 0, 1), (1, 1, 1, 1, 1, 1, 0), (1, 1, 2, 4, 1, 0, 300), (3, 1, 2, 4, 1, 200, 70), (5, 2, 1, 3, 1, 65, 33),
    (2, 1, 2, 8, 3, 129, 64), (4, 1, 1, 7, 5, 31, 40), (2, 1, 1, 2, 40, 500, 90), (1, 1, 2, 4, 70, 0, 200),
    (3, 1, 1, 5, 33, 96, 31), (9, 1, 1, 8, 1, 1000, 17), (20, 1, 1, 4, 1, 700, 5), (2, 3, 2, 1, 2, 64, 2),
    (70, 1, 1, 4, 1, 333, 60), (1, 2, 1, 6, 1, 4000, 1500), (2, 1, 1, 4, 130, 130, 257),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ATTN, ids=["-".join(map(str, c)) for c in ATTN])
def test_attention(dtype, case):
    for ragged in (False, True):
        p = Problem(*case, dtype, ragged=ragged)
        for odt in {p.dt, torch.float32}:
            print(f"{case} {dtype} -> {odt}, ragged {ragged}", flush=True)
            out, lse, w = p.run(odt)
            print(f"  largest error {p.check(out, lse, w):.3f} of the bound", flush=True)
        plain, lse2, _ = p.run(odt, weights=None)       # the same attention without weights
        assert torch.equal(plain, out) and torch.equal(lse2, lse)


MANY = [  # enough queries for every way to cut a call; the first and last slices are checked
    (64, 1, 8, 4, 1, 3000, 500), (8, 1, 8, 4, 77, 1200, 300), (4, 32, 8, 4, 1, 300, 200), (33, 1, 2, 8, 3, 5000, 100),
    (1, 1, 8, 4, 700, 0, 900), (130, 2, 8, 1, 1, 64, 33), (16, 1, 2, 4, 1, 9000, 40), (2, 1, 1, 8, 500, 800, 501),
    (4, 32, 8, 4, 1, 0, 300), (64, 16, 1, 3, 2, 0, 1500), (130, 8, 1, 8, 6, 0, 90),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", MANY, ids=["-".join(map(str, c)) for c in MANY])
def test_attention_of_many_rows(dtype, case):
    p = Problem(*case, dtype, seed=1)
    out, lse, w = p.run()
    worst = p.check(out, lse, w, sorted({0, 1, p.s // 2, p.s - 1} & set(range(p.s))))
    print(f"{case} {dtype}: largest error {worst:.3f} of the bound", flush=True)


def test_one_token_without_its_dimension():
    p = Problem(3, 1, 2, 4, 1, 100, 50, "bf16")
    out, lse, w = p.run()
    flat, lse3, w3 = torch.zeros(3, 8, 128, device=DEV, dtype=p.dt), torch.zeros(3, 8, device=DEV), p.w.clone()
    L().shared_prefix_attn(p.q[:, :, 0].contiguous(), 2, p.kp, p.vp, p.n_p, p.ko, p.vo, p.n_o, flat, lse3, weights=w3)
    assert torch.equal(flat, out[:, :, 0]) and torch.equal(lse3, lse[:, :, 0]) and torch.equal(w3, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_to_see(dtype):
    """No row at all, or none that a query sees: 0, lse -inf, no weight added."""
    for case in ((2, 1, 1, 4, 1, 0, 0), (2, 1, 1, 4, 3, 0, 20), (2, 1, 2, 4, 1, 40, 20)):
        p = Problem(*case, dtype, ragged=True)
        if p.n_o is not None:
            p.n_o.zero_()
        if p.n_p is not None:
            p.n_p.zero_()
        out, lse, w = p.run()
        assert (out == 0).all() and torch.isneginf(lse).all() and (w is None or torch.equal(w, p.w))


@pytest.mark.parametrize("case", [(4, 1, 2, 4, 1, 300, 60), (20, 1, 1, 4, 1, 300, 60), (70, 1, 1, 2, 3, 200, 40)])
def test_a_padded_sequence_changes_no_other(case):
    """Queries and own rows of a sequence that holds nothing may be NaN: the others' results stay, bit for bit."""
    for dtype in DT:
        p = Problem(*case, dtype, ragged=False)
        p.n_o = torch.full((p.s,), case[6], dtype=torch.int32, device=DEV)
        ref = p.run()
        per = p.s // case[0]
        p.q[1], p.ko[per:2 * per], p.vo[per:2 * per] = float("nan"), float("nan"), float("inf")
        p.n_o[per:2 * per] = 0
        got = p.run()
        others = torch.arange(case[0], device=DEV) != 1
        assert torch.equal(got[0][others], ref[0][others]) and torch.equal(got[1][others], ref[1][others])
        keep = torch.arange(p.s, device=DEV) // per != 1
        assert torch.equal(got[2][keep], ref[2][keep]) and torch.equal(got[2][~keep], p.w[~keep])


def test_lengths_are_clamped():
    p = Problem(2, 1, 2, 4, 1, 70, 50, "bf16", ragged=False)
    ref = p.run()
    p.n_p = torch.tensor([71, 1 << 30], dtype=torch.int32, device=DEV)
    p.n_o = torch.tensor([51, 1 << 30, 50, (1 << 31) - 1], dtype=torch.int32, device=DEV)
    for x, y in zip(p.run(), ref):
        assert torch.equal(x, y)
    p.n_p.fill_(-3)
    p.n_o.fill_(-(1 << 31))
    out, lse, w = p.run()
    assert (out == 0).all() and torch.isneginf(lse).all() and torch.equal(w, p.w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(2, 1, 1, 4, 40, 70, 100), (1, 1, 1, 8, 90, 0, 200), (40, 1, 1, 8, 5, 33, 60),
                                  (1, 1, 1, 2, 6, 0, 64)])
def test_later_rows_do_not_reach_a_query(dtype, case):
    """Keys and values behind a query may be NaN or infinite: its result does not change by a bit."""
    seqs, _, _, g, n_q, _, rows = case
    p = Problem(*case, dtype, ragged=False)
    ref, ref_lse, _ = p.run(torch.float32)
    assert not torch.isnan(ref).any()
    first = rows - n_q                       # the row of query 0
    for t, bad in ((1, float("nan")), (n_q // 2, float("inf")), (n_q - 1, -float("inf"))):
        for which in ("k", "v", "kv"):
            ko, vo = p.ko.clone(), p.vo.clone()
            if "k" in which:
                ko[:, first + t:, ::3] = bad
            if "v" in which:
                vo[:, first + t:, 5:90] = bad
            p.ko, ko = ko, p.ko
            p.vo, vo = vo, p.vo
            out, lse, w = p.run(torch.float32)
            p.ko, p.vo = ko, vo
            assert torch.equal(out[:, :, :t], ref[:, :, :t]) and torch.equal(lse[:, :, :t], ref_lse[:, :, :t]), (t, which)
            if which == "v":
                assert not torch.isfinite(out[:, :, t:, 5:90]).any()
                assert torch.equal(out[..., 90:], ref[..., 90:]) and torch.equal(lse, ref_lse)
                assert torch.isfinite(w).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("prefix,rows", [(40, 0), (0, 40), (64, 33), (333, 1), (1500, 700)])
def test_values_that_are_not_finite(dtype, bad, prefix, rows):
    """An infinite or NaN value of the last row that is held reaches every query in its own channel alone."""
    p = Problem(2, 1, 1, 4, 1, prefix, rows, dtype, ragged=False)
    ref = p.run(torch.float32)[0]
    last = p.vo if rows else p.vp
    last[:, -1, 17] = bad
    out, lse, w = p.run(torch.float32)
    want = torch.full_like(out[..., 17], bad)
    assert torch.equal(torch.isnan(out[..., 17]), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out[..., 17], nan=1.0), torch.nan_to_num(want, nan=1.0))
    others = torch.arange(128, device=DEV) != 17
    assert torch.equal(out[..., others], ref[..., others]) and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,g,n_q,prefix,rows", [
    (2, 4, 1, 64, 0), (1, 4, 1, 0, 64), (1, 1, 1, 0, 96), (2, 4, 1, 1536, 700), (16, 1, 1, 320, 32), (4, 2, 2, 200, 130),
    (5, 4, 1, 320, 64), (1, 8, 3, 0, 256), (1, 8, 9, 0, 320), (40, 4, 1, 640, 64), (3, 4, 20, 256, 96)])
def test_infinite_values_wherever_they_stand(dtype, seqs, g, n_q, prefix, rows):
    """An infinity of any row that a query sees is its result, of both signs NaN, in that channel alone."""
    p = Problem(seqs, 1, 1, g, n_q, prefix, rows, dtype, ragged=False)
    ref, ref_lse, ref_w = p.run(torch.float32)
    inf = float("inf")
    for values, n, hidden in ((p.vp, prefix, 0), (p.vo, rows, n_q - 1)):      # all queries see the rows before the hidden ones
        last = n - hidden - 1
        for at in sorted({0, 5, 31, 32, 63, n // 2, last - 1, last} & set(range(last + 1))):
            keep = values[0, at].clone()
            other = values[0, last - at].clone()
            values[0, at, 3], values[0, at, 77] = inf, -inf
            values[0, at, 100], values[0, last - at, 100] = inf, -inf          # twice the same row: -inf
            out, lse, w = p.run(torch.float32)
            values[0, last - at], values[0, at] = other, keep
            seen = out if values is p.vp else out[:1]
            assert (seen[..., 3] == inf).all() and (seen[..., 77] == -inf).all(), at
            assert (torch.isneginf if 2 * at == last else torch.isnan)(seen[..., 100]).all(), at
            same = torch.ones_like(out, dtype=torch.bool)
            same[:len(seen)][..., [3, 77, 100]] = False
            assert torch.equal(out[same], ref[same]) and torch.equal(lse, ref_lse), at
            assert w is None or torch.equal(w, ref_w)


@pytest.mark.parametrize("seqs,kv,g,n_q,prefix,rows", [
    (1, 2, 4, 1, 0, 300), (4, 2, 4, 1, 3000, 500), (1, 1, 1, 1, 64, 0), (8, 1, 4, 1, 2000, 100), (5, 2, 4, 1, 700, 33),
    (3, 1, 8, 1, 900, 40), (2, 1, 8, 2, 333, 64), (1, 2, 8, 4, 0, 1500), (1, 1, 6, 5, 0, 70), (17, 1, 1, 1, 128, 1)])
def test_bf16_attention_keeps_its_weights_beyond_bf16(seqs, kv, g, n_q, prefix, rows):
    """Up to 32 queries of the same rows: weights meet the values as two bfloat16.  What the second rounding leaves is
    2^-8 of at most 2^-8 of a weight, so a float32 result is off by 2^-16 of the weighted mean of |v| beside the float32
    roundings."""
    p = Problem(seqs, 1, kv, g, n_q, prefix, rows, "bf16")
    out, lse, _ = p.run(torch.float32)
    on, ln, q = n64(out).reshape(p.s, g, n_q, 128), n64(lse).reshape(p.s, g, n_q), n64(p.q).reshape(p.s, g, n_q, 128)
    worst = 0.0
    for i in range(p.s):
        k, v, see, n = p.rows_of(i)
        see[:, :n] = True
        for j in range(g):
            o, e, mass, size = ob.masked_attention(q[i, j], k, v, see, SCALE)
            tol, tol_lse = attention_bounds(o, mass, e, size, len(k), False, False)
            tol = tol + 2.0 ** -16 * mass
            err = np.abs(on[i, j] - o)
            assert (err <= tol).all(), f"slice {i}: {(err / tol).max():.3g} of the bound"
            worst = max(worst, (err / tol).max())
            live = np.isfinite(e)
            assert (np.abs(ln[i, j][live] - e[live]) <= tol_lse[live]).all() and np.array_equal(np.isneginf(ln[i, j]), ~live)
    print(f"  largest error {worst:.3f} of the bound", flush=True)


def test_scores_of_minus_infinity_weigh_nothing():
    p = Problem(1, 1, 1, 2, 1, 30, 40, "bf16", ragged=False)
    p.q.fill_(1.0)
    p.kp.fill_(-float("inf"))
    p.ko[:, :39] = -float("inf")
    p.ko[:, 39] = 0.0
    out, lse, w = p.run(torch.float32)
    assert torch.allclose(out, p.vo[0, 39].float().expand_as(out), rtol=2.0 ** -8) and (lse == 0).all()
    assert torch.equal(w[0, :39], p.w[0, :39]) and abs(float(w[0, 39] - p.w[0, 39]) - 2) < 1e-5
    p.ko.fill_(-float("inf"))
    out, lse, w = p.run(torch.float32)
    assert (out == 0).all() and torch.isneginf(lse).all() and torch.equal(w, p.w)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    for dtype in DT:
        p = Problem(3, 1, 1, 4, 2, 90, 70, dtype, ragged=False)
        out, lse, _ = p.run(torch.float32, weights=None, scale=scale)
        q = p.q.double().view(3, 8, 128)
        k = torch.cat((p.kp.double().expand(3, -1, -1), p.ko.double()), 1)
        v = torch.cat((p.vp.double().expand(3, -1, -1), p.vo.double()), 1)
        x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(3, 4, 2, 160) * scale
        x[:, :, 0, -1] = -float("inf")
        ref = torch.bmm(x.softmax(-1).view(3, 8, 160), v).view(3, 4, 2, 128)
        # weights rounded to bfloat16 (2^-8), or float32 logits of up to 3 * 1500 (140 2^-24 of it twice)
        tol = (2.0 ** -8 if dtype == "bf16" else 0.0) + 280 * U * abs(scale) * 1500 + 1e-4
        assert (out.double() - ref).abs().max() < tol * v.abs().max()
        assert (lse.double() - x.logsumexp(-1)).abs().max() < 140 * U * abs(scale) * 1500 + 1e-4


def test_rows_past_two_gigabytes():
    """Offsets of a slice's rows need 64 bits."""
    rows, s = 60000, 300
    kv = torch.zeros(s, rows, 128, dtype=torch.bfloat16, device=DEV)        # 4.6 GB
    kv[-1] = torch.randn(rows, 128, device=DEV)
    q = torch.randn(1, s, 1, 128, device=DEV).bfloat16()
    n_o = torch.full((s,), 5, dtype=torch.int32, device=DEV)
    n_o[-1] = rows - 3
    out, w, lse = torch.zeros_like(q), torch.zeros(s, rows, device=DEV), torch.zeros(1, s, 1, device=DEV)
    L().shared_prefix_attn(q, s, None, None, None, kv, kv, n_o, out, lse, weights=w)
    x = kv[-1, :rows - 3].float() @ q[0, -1, 0].float() * SCALE
    p = x.softmax(0)
    # a bfloat16 result of weights that are bfloat16: 2^-8 twice, of values up to 5
    assert (out[0, -1, 0].float() - p @ kv[-1, :rows - 3].float()).abs().max() < 5 * 2.0 ** -7
    assert (w[-1, :rows - 3] - p).abs().max() < 1e-4 * p.max() and (w[-1, rows - 3:] == 0).all() and (out[0, :-1] == 0).all()
    w2 = torch.zeros_like(w)
    L().attn_weights(q, s, kv, n_o, lse, w2)
    assert (w2 - w).abs().max() < 1e-4 * w.max()
    # the same rows as a prefix: one slice of many rows
    long = kv.view(1, -1, 128)[:, -9_000_000:]
    out2, q2 = torch.zeros(2, 1, 1, 128, device=DEV), q[:, -1:].expand(2, -1, -1, -1).contiguous()
    n_p = torch.tensor([long.shape[1] - 3], dtype=torch.int32, device=DEV)
    L().shared_prefix_attn(q2, 1, long, long, n_p, None, None, None, out2)
    y = torch.cat((x, torch.zeros(1, device=DEV)))
    zero = np.log(long.shape[1] - rows)                                     # rows of zeros: a logit of 0 each
    y[-1] = zero
    ref = y.softmax(0)[:-1] @ kv[-1, :rows - 3].float()
    assert (out2 - ref).abs().max() < 2.0 ** -7 * ref.abs().max() + 1e-5


def test_replayed_graph_and_two_streams():
    l = L()
    p = Problem(3, 1, 2, 4, 1, 600, 300, "bf16")
    size = l.shared_prefix_attn_workspace_size(p.s, p.sp, p.g, p.n_q, 600, 300, True)

    def state():
        return dict(q=p.q.clone(), n=p.n_o.clone(), out=torch.zeros_like(p.q), lse=torch.zeros(p.q.shape[:3], device=DEV),
                    w=p.w.clone(), w2=p.w.clone(), ws=torch.empty(max(size, 1), dtype=torch.uint8, device=DEV))

    def one(x, stream=None):
        l.shared_prefix_attn(x["q"], p.kv, p.kp, p.vp, p.n_p, p.ko, p.vo, x["n"], x["out"], x["lse"], weights=x["w"],
                             workspace=x["ws"], stream=stream)
        l.attn_weights(x["q"], p.kv, p.ko, x["n"], x["lse"], x["w2"], stream=stream)
    eager, captured, other = state(), state(), state()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            one(captured)
    for i in range(4):
        new = torch.randn(p.q.shape, device=DEV).bfloat16()
        for x in (eager, captured, other):
            x["q"].copy_(new)
            x["n"].copy_((p.n_o - i).clamp(min=0))
        torch.cuda.synchronize()
        one(eager)
        one(other, side)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("out", "lse", "w", "w2"):
            assert torch.equal(eager[n], captured[n]) and torch.equal(eager[n], other[n]), (i, n)


# ------------------------------------------------------------------- weights from an lse

WEIGHTS = [  # groups, kv, g, n_q, keys
    (1, 1, 1, 1, 1), (1, 2, 4, 1, 3000), (2, 1, 8, 5, 70), (1, 1, 3, 33, 33), (1, 2, 4, 64, 1000), (3, 2, 7, 20, 257),
    (1, 1, 4, 300, 300), (1, 1, 8, 129, 600), (2, 4, 1, 2, 2048), (1, 1, 2, 700, 1111), (1, 8, 4, 64, 5000), (40, 8, 2, 7, 90),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", WEIGHTS, ids=["-".join(map(str, c)) for c in WEIGHTS])
def test_weights(dtype, case):
    groups, kv, g, n_q, rows = case
    s = groups * kv
    gen = torch.Generator(device=DEV).manual_seed(rows)
    rng = np.random.default_rng(rows)
    q = (2 * torch.randn(groups, kv * g, n_q, 128, generator=gen, device=DEV)).to(DT[dtype])
    keys = torch.randn(s, rows, 128, generator=gen, device=DEV).to(DT[dtype])
    for ragged in (False, True):
        n = rng.integers(0, rows + 1, s) if ragged else np.full(s, rows)
        n[-1] = rows
        for i in range(s):
            keys[i, int(n[i]):] = float("nan")
        n_k = torch.from_numpy(n.astype(np.int32)).to(DEV) if ragged else None
        lse = torch.randn(groups, kv * g, n_q, generator=gen, device=DEV) + 8
        lse[:, :, ::5] = -float("inf")                  # queries that add nothing
        if n_q > 1:
            lse[:, :, 1] = 7.5
        before = torch.rand(s, rows, generator=gen, device=DEV)
        w = before.clone()
        print(f"{case} {dtype}, ragged {ragged}", flush=True)
        L().attn_weights(q, kv, keys, n_k, lse, w)
        qn, ln, got = n64(q).reshape(s, g, n_q, 128), n64(lse).reshape(s, g, n_q), n64(w)
        for i in {0, s // 2, s - 1}:
            k, b = n64(keys[i, :n[i]]), n64(before[i])
            see = np.arange(n[i])[None] <= n[i] - n_q + np.arange(n_q)[:, None]
            added, size = np.zeros(n[i]), np.zeros(n[i])
            for j in range(g):
                x, y = op.row_weights(qn[i, j], k, see, ln[i, j], SCALE)
                added, size = added + x, np.maximum(size, y)
            tol = weight_tolerance(b[:n[i]], added, size, 12.0, 0, g * n_q)
            err = np.abs(got[i, :n[i]] - b[:n[i]] - added)
            assert (err <= tol).all(), f"slice {i}: {(err / tol).max():.3g} of the bound"
            assert np.array_equal(got[i, n[i]:], b[n[i]:])


def test_weights_with_bad_keys_and_lse():
    """A NaN key or lse makes the weights that it enters NaN, a key behind a query none of that query's."""
    for dtype in DT:
        q = torch.randn(1, 2, 10, 128, device=DEV).to(DT[dtype])
        keys = torch.randn(1, 40, 128, device=DEV).to(DT[dtype])
        lse = torch.full((1, 2, 10), 5.0, device=DEV)
        ref = torch.zeros(1, 40, device=DEV)
        L().attn_weights(q, 1, keys, None, lse, ref)
        keys[0, 33, 7] = float("nan")
        w = torch.zeros(1, 40, device=DEV)
        L().attn_weights(q, 1, keys, None, lse, w)
        others = torch.arange(40, device=DEV) != 33
        assert torch.isnan(w[0, 33]) and torch.equal(w[0, others], ref[0, others])
        keys[0, 33, 7] = 0.0
        lse[0, 1, 4] = float("nan")                      # the query of row 34 sees the rows up to it
        w.zero_()
        L().attn_weights(q, 1, keys, None, lse, w)
        assert torch.isnan(w[0, :35]).all() and torch.isfinite(w[0, 35:]).all()


def test_attention_then_weights_equal_the_attention_with_weights():
    for dtype, case in (("bf16", (2, 1, 2, 4, 3, 300, 500)), ("f32", (2, 1, 2, 4, 3, 300, 500)), ("bf16", (1, 1, 1, 8, 60, 0, 400))):
        p = Problem(*case, dtype)
        p.w.zero_()
        out, lse, w = p.run()
        w2 = torch.zeros_like(w)
        L().attn_weights(p.q, p.kv, p.ko, p.n_o, lse, w2)
        # the same formula with the same lse: float32 products, exponentials and sums of the two
        assert (w - w2).abs().max() <= 1e-4 * w.max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_many_slices_a_block_each(dtype):
    """Two blocks a CU, whose waves join their sums at their own times: the same weights every time."""
    p = Problem(64, 2, 4, 4, 2, 0, 230, dtype)
    runs = [p.run() for _ in range(4)]
    for x in runs[1:]:
        for a, b in zip(x, runs[0]):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    p.check(*runs[0], slices=range(0, p.s, 13))
