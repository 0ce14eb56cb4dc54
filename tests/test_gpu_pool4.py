"""The 4-bit pool on the GPU against its float64 oracle: bytes exact, dense reads
exact, stores in lockstep with the calls that keep the pool in full precision,
attention within the bounds of tests/attn_bounds.py."""
import numpy as np
import pytest
import torch

from attn_bounds import attention_bounds, check_attention
from oracle import blocks as ob
from oracle import pool4 as o4

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


def L():
    from paper_2510_11292_amd import louiskv
    return louiskv


def n64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows_with_corners(rng, n, dt):
    """Rows of every magnitude; the first ones hold ties, zeros, subnormals, extremes and blocks that are not finite."""
    x = rng.standard_normal((n, 128)) * 2.0 ** rng.integers(-20, 20, (n, 4)).repeat(32, 1)
    tie = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -5.0, 6.5, -7.0, 0.0, -0.0, 6.0])
    for i, row in enumerate([np.tile(tie, 8), np.zeros(128), np.tile(tie, 8) * 2.0 ** -125, np.tile(tie, 8) * 2.0 ** -133,
                             np.tile(tie, 8) * 2.0 ** 124][:n]):
        x[i] = row
    if n > 8:
        x[5, 7], x[6, 127], x[7, 64], x[8, 32:64] = np.inf, np.nan, -np.inf, 3.3e38
    return torch.from_numpy(x).to(torch.float32).to(dt)


def pool_of(rng, s, rows):
    codes = torch.from_numpy(rng.integers(0, 256, (s, rows, 128), dtype=np.uint8))
    scales = torch.from_numpy(rng.integers(124, 129, (s, rows, 8), dtype=np.uint8))
    return codes, scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,extra,order", [(1, 0, "perm"), (31, 2, "none"), (33, 0, "perm"), (300, 7, "perm"),
                                           (64, 0, "wild")])
def test_pack_writes_the_oracles_bytes(dtype, n, extra, order):
    rng = np.random.default_rng(n)
    s = 3
    k = torch.stack([rows_with_corners(rng, n, DT[dtype]) for _ in range(s)])
    v = torch.stack([rows_with_corners(rng, n, DT[dtype]).flip(0) for _ in range(s)])
    perm = np.stack([rng.permutation(n) for _ in range(s)]).astype(np.int32)
    if order == "wild":     # entries outside the prompt are clamped into it
        perm[:, ::3] -= 40
        perm[:, 1::3] += 40
    at = np.tile(np.arange(n), (s, 1)) if order == "none" else np.clip(perm, 0, n - 1)
    codes = torch.full((s, n + extra, 128), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((s, n + extra, 8), 0x5A, dtype=torch.uint8, device=DEV)
    L().pack_pool_q4(k.to(DEV), v.to(DEV), None if order == "none" else torch.from_numpy(perm).to(DEV), codes, scales)
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    for i in range(s):
        want = o4.pack_bytes(*o4.quantise(n64(k[i])[at[i]]), *o4.quantise(n64(v[i])[at[i]]))
        np.testing.assert_array_equal(scales[i, :n], want[1])
        np.testing.assert_array_equal(codes[i, :n], want[0])
    assert (codes[:, n:] == 0xA5).all() and (scales[:, n:] == 0x5A).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("listed", [True, False])
def test_gather_reads_exact_values(dtype, listed):
    rng = np.random.default_rng(3)
    s, rows, n = 4, 300, 101
    codes = torch.from_numpy(rng.integers(0, 256, (s, rows, 128), dtype=np.uint8))
    scales = torch.from_numpy(rng.integers(2, 253, (s, rows, 8), dtype=np.uint8))
    scales[:, ::9, 3] = 255
    sel = rng.integers(-5, rows + 5, (s, n)).astype(np.int32)
    sel[:, 1] = sel[:, 0]
    n_sel = np.array([0, 1, 77, 500], dtype=np.int32)
    kb = torch.full((s, n, 128), 9.0, dtype=DT[dtype], device=DEV)
    vb = torch.full((s, n, 128), 9.0, dtype=DT[dtype], device=DEV)
    L().gather_rows_q4(codes.to(DEV), scales.to(DEV), torch.from_numpy(sel).to(DEV) if listed else None,
                       torch.from_numpy(n_sel).to(DEV) if listed else None, kb, vb)
    for i in range(s):
        m = min(int(n_sel[i]), n) if listed else n
        at = np.clip(sel[i, :m], 0, rows - 1) if listed else np.arange(n)
        k, v = o4.values(codes[i].numpy()[at], scales[i].numpy()[at])
        for got, want in ((kb, k), (vb, v)):
            np.testing.assert_array_equal(n64(got[i, :m]), want.astype(np.float32).astype(np.float64))
            assert (n64(got[i, m:]) == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,seg", [(32, 8), (20, 5), (4, 4), (1, 1), (128, 32)])
def test_fixed_segment_store_in_lockstep(dtype, window, seg):
    """Window, units and means equal louiskv.segment_output's bit for bit, the pool the quantised rows of its pool."""
    l = L()
    dt, s, c, prompt, steps = DT[dtype], 5, 3, 7, window + 3 * seg + 2
    g = torch.Generator(device=DEV).manual_seed(1)
    cap, rows = c + 4 + steps // seg, prompt + steps
    mk = lambda: dict(k_local=torch.zeros(s, window, 128, dtype=dt, device=DEV),
                      v_local=torch.zeros(s, window, 128, dtype=dt, device=DEV),
                      reps=torch.zeros(s, cap, 128, device=DEV),
                      unit_start=torch.zeros(s, cap, dtype=torch.int32, device=DEV),
                      unit_size=torch.zeros(s, cap, dtype=torch.int32, device=DEV))
    a, b = mk(), mk()
    kp = torch.zeros(s, rows, 128, dtype=dt, device=DEV)
    vp = torch.zeros_like(kp)
    codes = torch.zeros(s, rows, 128, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(s, rows, 8, dtype=torch.uint8, device=DEV)
    for t in range(steps):
        k = (3 * torch.randn(s, 128, generator=g, device=DEV)).to(dt)
        v = torch.randn(s, 128, generator=g, device=DEV).to(dt)
        l.segment_output(k, v, a["k_local"], a["v_local"], t, seg, a["reps"], a["unit_start"], a["unit_size"], c, kp, vp,
                         prompt)
        l.segment_output_q4(k, v, b["k_local"], b["v_local"], t, seg, b["reps"], b["unit_start"], b["unit_size"], c,
                            codes, scales, prompt)
        for n in a:
            assert torch.equal(a[n], b[n]), (t, n)
    ev = l.window_info(steps - 1, window, seg)[1] * seg
    assert ev > 0
    want_c, want_s = torch.zeros_like(codes), torch.zeros_like(scales)
    tc, ts = want_c[:, :ev].contiguous(), want_s[:, :ev].contiguous()
    l.pack_pool_q4(kp[:, prompt:prompt + ev].contiguous(), vp[:, prompt:prompt + ev].contiguous(), None, tc, ts)
    want_c[:, prompt:prompt + ev], want_s[:, prompt:prompt + ev] = tc, ts
    assert torch.equal(codes, want_c) and torch.equal(scales, want_s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap_short", [False, True])
def test_boundary_segment_store_in_lockstep(dtype, cap_short):
    l = L()
    dt, kv, groups, c, prompt, steps, window, seg = DT[dtype], 2, 3, 3, 7, 150, 24, 9
    s = kv * groups
    cap, rows = (c + 5 if cap_short else c + steps), prompt + steps
    rng = np.random.default_rng(4)
    g = torch.Generator(device=DEV).manual_seed(2)
    mk = lambda: dict(k_local=torch.zeros(s, window, 128, dtype=dt, device=DEV),
                      v_local=torch.zeros(s, window, 128, dtype=dt, device=DEV),
                      reps=torch.zeros(s, cap, 128, device=DEV),
                      unit_start=torch.zeros(s, cap, dtype=torch.int32, device=DEV),
                      unit_size=torch.zeros(s, cap, dtype=torch.int32, device=DEV),
                      state=torch.zeros(s, l.segment_state_ints(window), dtype=torch.int32, device=DEV))
    a, b = mk(), mk()
    kp = torch.zeros(s, rows, 128, dtype=dt, device=DEV)
    vp = torch.zeros_like(kp)
    codes = torch.zeros(s, rows, 128, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(s, rows, 8, dtype=torch.uint8, device=DEV)
    for x in (a, b):
        l.segment_state_init(x["state"], window, c)
    for t in range(steps):
        k, v = ((2 * torch.randn(s, 128, generator=g, device=DEV)).to(dt) for _ in range(2))
        fire = torch.from_numpy((rng.random(groups) < 0.2).astype(np.uint8)).to(DEV)
        l.segment_output_boundary(k, v, a["k_local"], a["v_local"], t, seg, fire, a["state"], a["reps"], a["unit_start"],
                                  a["unit_size"], c, kv, kp, vp, prompt)
        l.segment_output_boundary_q4(k, v, b["k_local"], b["v_local"], t, seg, fire, b["state"], b["reps"],
                                     b["unit_start"], b["unit_size"], c, kv, codes, scales, prompt)
        for n in a:
            assert torch.equal(a[n], b[n]), (t, n)
    wc, ws = torch.zeros(s, rows, 128, dtype=torch.uint8, device=DEV), torch.zeros(s, rows, 8, dtype=torch.uint8, device=DEV)
    l.pack_pool_q4(kp, vp, None, wc, ws)
    stored = torch.from_numpy(np.zeros((s, rows), dtype=bool))
    for i in range(s):
        for u in range(c, int(b["state"][i, 0])):
            st, n = int(b["unit_start"][i, u]), int(b["unit_size"][i, u])
            stored[i, st:st + n] = True
    m = stored.to(DEV)
    assert m.any() and torch.equal(codes[m], wc[m]) and torch.equal(scales[m], ws[m])
    assert (codes[~m] == 0).all() and (scales[~m] == 0).all()
    assert bool((b["state"][:, 4] != 0).all()) == cap_short


def attn_want(codes, scales, rows, kl, vl, q, scale):
    k, v = o4.values(codes[rows], scales[rows])
    k, v = np.concatenate([k, kl]), np.concatenate([v, vl])
    return ob.masked_attention(q, k, v, np.ones((q.shape[0], len(k)), dtype=bool), scale)


ATTN = [  # groups, kv heads, g, pool rows, budget, window, local start, local rows
    (1, 1, 4, 1, 1, 1, 0, 0), (1, 2, 1, 40, 3, 8, 7, 8), (1, 8, 4, 500, 333, 128, 100, 100), (2, 3, 2, 700, 64, 32, 5, 0),
    (1, 2, 8, 5000, 4100, 64, 63, 64), (3, 8, 4, 200, 0, 16, 2, 11), (40, 8, 4, 300, 129, 128, 0, 128),
    (1, 1, 8, 3000, 2999, 1, 0, 1), (70, 8, 2, 90, 90, 40, 39, 17), (1, 4, 4, 9000, 8200, 128, 3, 125),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ATTN, ids=[f"{c[0]}x{c[1]}x{c[2]}-{c[4]}+{c[7]}" for c in ATTN])
def test_attention_over_listed_rows(dtype, case):
    groups, kv, g, rows, budget, window, start, local = case
    s, dt = groups * kv, DT[dtype]
    rng = np.random.default_rng(budget + g)
    codes, scales = pool_of(rng, s, rows)
    sel = rng.integers(0, rows, (s, max(budget, 1))).astype(np.int32)
    n_sel = rng.integers(0, budget + 1, s).astype(np.int32)
    n_sel[0] = budget
    if s > 1:
        n_sel[-1] = 0
    if budget > 2:
        sel[:, 2] = sel[:, 0]                       # a row listed twice counts twice
    if budget > 40:
        sel[:, 30], sel[:, 31] = -7, rows + 9       # clamped into the pool
    used = np.zeros((s, rows), dtype=bool)
    for i in range(s):
        used[i, np.clip(sel[i, :n_sel[i]], 0, rows - 1)] = True
    scales[torch.from_numpy(~used)] = 255           # rows that no list holds are NaN
    sel[np.arange(sel.shape[1])[None] >= n_sel[:, None]] = 1 << 30
    q = torch.from_numpy(rng.standard_normal((groups, kv * g, 128)) * 2).to(dt)
    kl, vl = (torch.from_numpy(rng.standard_normal((s, window, 128))).to(dt) for _ in range(2))
    ring = [(start + i) % window for i in range(local)]
    dead = [i for i in range(window) if i not in ring]
    kl[:, dead], vl[:, dead] = float("nan"), float("nan")
    for odt in (dt, torch.float32):
        out = torch.full((groups, kv * g, 128), 7.0, dtype=odt, device=DEV)
        lse = torch.full((groups, kv * g), 7.0, device=DEV)
        L().sparse_decode_attn_rows_q4(q.to(DEV), kv, codes.to(DEV), scales.to(DEV),
                                       torch.from_numpy(sel[:, :budget].copy()).to(DEV), torch.from_numpy(n_sel).to(DEV),
                                       kl.to(DEV), vl.to(DEV), start, local, out, lse)
        got, got_lse = n64(out).reshape(s, g, 128), n64(lse).reshape(s, g)
        worst = 0.0
        for i in range(s):
            at = np.clip(sel[i, :n_sel[i]], 0, rows - 1)
            want = attn_want(codes[i].numpy(), scales[i].numpy(), at, n64(kl[i, ring]), n64(vl[i, ring]),
                             n64(q).reshape(s, g, 128)[i], 128 ** -0.5)
            worst = max(worst, check_attention(got[i], got_lse[i], want, dtype == "bf16", odt == torch.bfloat16,
                                               len(at) + local))
        print(f"{dtype} -> {odt}: largest error {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_values_that_are_not_finite(dtype):
    """A NaN block reaches exactly the heads and channels that the formula gives it; scores of -inf weigh nothing."""
    rng = np.random.default_rng(8)
    s, g, rows, budget, dt = 3, 4, 64, 50, DT[dtype]
    codes, scales = pool_of(rng, s, rows)
    sel = np.stack([rng.permutation(rows)[:budget] for _ in range(s)]).astype(np.int32)
    scales[0, sel[0, 17], 5] = 255       # a value block: 32 channels
    scales[1, sel[1, 49], 2] = 255       # a key block: everything
    q = torch.ones(1, s * g, 128, dtype=dt)
    kl = torch.zeros(s, 4, 128, dtype=dt)
    vl = torch.ones(s, 4, 128, dtype=dt)
    kl[2, 1] = -float("inf")
    out, lse = torch.zeros(1, s * g, 128, device=DEV), torch.zeros(1, s * g, device=DEV)
    n_sel = torch.tensor([budget, budget, 0], dtype=torch.int32, device=DEV)
    L().sparse_decode_attn_rows_q4(q.to(DEV), s, codes.to(DEV), scales.to(DEV), torch.from_numpy(sel).to(DEV), n_sel,
                                   kl.to(DEV), vl.to(DEV), 0, 2, out, lse)
    o = n64(out).reshape(s, g, 128)
    assert np.isnan(o[0][:, 32:64]).all() and np.isfinite(np.delete(o[0], range(32, 64), 1)).all()
    assert np.isnan(o[1]).all()
    np.testing.assert_array_equal(o[2], np.ones((g, 128)))     # the key of -inf weighs 0, the other 1
    # and a slice whose every score is -inf has no weight at all
    n_sel.zero_()
    L().sparse_decode_attn_rows_q4(q.to(DEV), s, codes.to(DEV), scales.to(DEV), torch.from_numpy(sel).to(DEV), n_sel,
                                   kl.to(DEV), vl.to(DEV), 1, 1, out, lse)
    assert (n64(out).reshape(s, g, 128)[2] == 0).all() and np.isneginf(n64(lse).reshape(s, g)[2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_local", [1, 15, 31, 33, 45, 64])
@pytest.mark.parametrize("budget", [0, 37, 700])
def test_infinite_window_values(dtype, n_local, budget):
    """An infinity among the window's values gives its channel an infinity wherever it stands, in the newest row too,
    which a last tile that it does not fill repeats; other channels keep their bits."""
    rng = np.random.default_rng(n_local + budget)
    s, g, rows, window, start, dt = 3, 4, 800, 64, 21, DT[dtype]
    codes, scales = (x.to(DEV) for x in pool_of(rng, s, rows))
    sel = torch.from_numpy(rng.integers(0, rows, (s, budget)).astype(np.int32)).to(DEV)
    n_sel = torch.full((s,), budget, dtype=torch.int32, device=DEV)
    # scores stay within a few units: no weight is lost beside another
    q = torch.from_numpy(0.1 * rng.standard_normal((1, s * g, 128))).to(dt).to(DEV)
    kl, vl = (torch.from_numpy(rng.standard_normal((s, window, 128))).to(dt).to(DEV) for _ in range(2))

    def attend(v):
        out, lse = torch.zeros(1, s * g, 128, device=DEV), torch.zeros(1, s * g, device=DEV)
        L().sparse_decode_attn_rows_q4(q, s, codes, scales, sel, n_sel, kl, v, start, n_local, out, lse)
        return out.view(s, g, 128), lse
    ref, ref_lse = attend(vl)
    assert torch.isfinite(ref).all()
    for at in {0, n_local // 2, n_local - 1}:
        slot, bad = (start + at) % window, vl.clone()
        bad[1, slot, 3], bad[1, slot, 77], bad[2, slot, 127] = float("inf"), -float("inf"), float("nan")
        out, lse = attend(bad)
        assert (out[1, :, 3] == float("inf")).all() and (out[1, :, 77] == -float("inf")).all(), at
        assert torch.isnan(out[2, :, 127]).all()
        keep = torch.ones(s, 128, dtype=torch.bool, device=DEV)
        keep[1, 3] = keep[1, 77] = keep[2, 127] = False
        keep = keep[:, None].expand(s, g, 128)
        assert torch.equal(out[keep], ref[keep]) and torch.equal(lse, ref_lse), at


@pytest.mark.parametrize("groups,kv,g,budget,local", [(1, 2, 1, 900, 50), (2, 3, 2, 64, 128), (1, 8, 4, 2048, 100),
                                                      (40, 8, 4, 129, 128), (2, 2, 8, 333, 17), (1, 1, 8, 0, 40)])
def test_bf16_attention_keeps_its_weights_beyond_bf16(groups, kv, g, budget, local):
    """Weights enter the sum of values as two bfloat16: what the second rounding leaves is 2^-8 of at most 2^-8 of a
    weight, so a float32 result is off by 2^-16 of the weighted mean of |v| beside the float32 roundings."""
    s, rows, window, start = groups * kv, 2500, 128, 77
    rng = np.random.default_rng(budget + g)
    codes, scales = pool_of(rng, s, rows)
    sel = rng.integers(0, rows, (s, budget)).astype(np.int32)
    n_sel = np.full(s, budget, dtype=np.int32)
    q = torch.from_numpy(rng.standard_normal((groups, kv * g, 128))).bfloat16()
    kl, vl = (torch.from_numpy(rng.standard_normal((s, window, 128))).bfloat16() for _ in range(2))
    out, lse = torch.zeros(groups, kv * g, 128, device=DEV), torch.zeros(groups, kv * g, device=DEV)
    L().sparse_decode_attn_rows_q4(q.to(DEV), kv, codes.to(DEV), scales.to(DEV), torch.from_numpy(sel).to(DEV),
                                   torch.from_numpy(n_sel).to(DEV), kl.to(DEV), vl.to(DEV), start, local, out, lse)
    ring = [(start + i) % window for i in range(local)]
    for i in range(s):
        o, e, mass, size = attn_want(codes[i].numpy(), scales[i].numpy(), sel[i], n64(kl[i, ring]), n64(vl[i, ring]),
                                     n64(q).reshape(s, g, 128)[i], 128 ** -0.5)
        tol, tol_lse = attention_bounds(o, mass, e, size, budget + local, False, False)
        assert np.all(np.abs(n64(out).reshape(s, g, 128)[i] - o) <= tol + 2.0 ** -16 * mass), i
        assert np.all(np.abs(n64(lse).reshape(s, g)[i] - e) <= tol_lse), i


@pytest.mark.parametrize("bits", [0x7fc00000, 0x7fffffff, -1, 0x7f800001, -0x7fffff])
@pytest.mark.parametrize("budget", [1, 900])     # one block a slice and several, whose merge rounds
def test_a_nan_of_any_bits_stays_one_in_a_bf16_output(bits, budget):
    s, g, rng = 2, 4, np.random.default_rng(2)
    codes, scales = (x.to(DEV) for x in pool_of(rng, s, 50))
    nan = torch.tensor([bits], dtype=torch.int32, device=DEV).view(torch.float32)
    q = torch.randn(1, s * g, 128, device=DEV)
    loc = torch.randn(s, 16, 128, device=DEV)
    loc.view(torch.int32)[1, 7, 5] = nan.view(torch.int32)[0]
    sel = torch.from_numpy(rng.integers(0, 50, (s, budget)).astype(np.int32)).to(DEV)
    n_sel = torch.full((s,), budget, dtype=torch.int32, device=DEV)
    kl = torch.randn(s, 16, 128, device=DEV)
    out = torch.zeros(1, s * g, 128, dtype=torch.bfloat16, device=DEV)
    L().sparse_decode_attn_rows_q4(q, s, codes, scales, sel, n_sel, kl, loc, 0, 16, out)
    want = torch.zeros(s, g, 128, dtype=torch.bool, device=DEV)
    want[1, :, 5] = True
    assert torch.equal(torch.isnan(out.view(s, g, 128)), want)


def test_attention_with_per_slice_windows():
    l = L()
    rng = np.random.default_rng(9)
    groups, kv, g, rows, budget, window, n_tok = 2, 2, 4, 300, 200, 16, 45
    s = groups * kv
    codes, scales = pool_of(rng, s, rows)
    state = torch.zeros(s, l.segment_state_ints(window), dtype=torch.int32)
    first = [45 - 16, 45 - 3, 45, 30]
    state[:, 1] = torch.tensor(first)
    sel = torch.from_numpy(rng.integers(0, rows, (s, budget)).astype(np.int32))
    n_sel = torch.tensor([0, 200, 3, 150], dtype=torch.int32)
    q = torch.from_numpy(rng.standard_normal((groups, kv * g, 128))).bfloat16()
    kl, vl = (torch.from_numpy(rng.standard_normal((s, window, 128))).bfloat16() for _ in range(2))
    out, lse = torch.zeros(groups, kv * g, 128, device=DEV), torch.zeros(groups, kv * g, device=DEV)
    l.sparse_decode_attn_rows_q4_seg(q.to(DEV), kv, codes.to(DEV), scales.to(DEV), sel.to(DEV), n_sel.to(DEV), kl.to(DEV),
                                     vl.to(DEV), state.to(DEV), n_tok, out, lse)
    for i in range(s):
        ring = [t % window for t in range(first[i], n_tok)]
        want = attn_want(codes[i].numpy(), scales[i].numpy(), sel[i, :n_sel[i]].numpy(), n64(kl[i, ring]), n64(vl[i, ring]),
                         n64(q).reshape(s, g, 128)[i], 128 ** -0.5)
        check_attention(n64(out).reshape(s, g, 128)[i], n64(lse).reshape(s, g)[i], want, True, False, 300)


def test_attention_offsets_past_32_bits():
    """A pool whose bytes pass 2^32: the last slice's rows are the ones read."""
    rows, s = 1 << 23, 5
    codes = torch.zeros(s, rows, 128, dtype=torch.uint8, device=DEV)
    scales = torch.full((s, rows, 8), 127, dtype=torch.uint8, device=DEV)
    assert codes.numel() > 1 << 32
    codes[4, rows - 3, 64:] = 0x22          # 1.0
    codes[4, 5, 64:] = 0x44                 # 2.0
    codes[3, rows - 1, 64:] = 0x77          # 6.0
    sel = torch.zeros(s, 2, dtype=torch.int32, device=DEV)
    sel[4] = torch.tensor([rows - 3, 5])
    sel[3] = rows - 1
    n_sel = torch.full((s,), 2, dtype=torch.int32, device=DEV)
    for dt in (torch.bfloat16, torch.float32):
        q = torch.ones(1, s, 128, dtype=dt, device=DEV)
        loc = torch.zeros(s, 1, 128, dtype=dt, device=DEV)
        out = torch.zeros(1, s, 128, device=DEV)
        L().sparse_decode_attn_rows_q4(q, s, codes, scales, sel, n_sel, loc, loc, 0, 0, out)
        assert (out[0, 4] == 1.5).all() and (out[0, 3] == 6.0).all() and (out[0, 0] == 0).all()
        kb, vb = (torch.zeros(s, 2, 128, dtype=dt, device=DEV) for _ in range(2))
        L().gather_rows_q4(codes, scales, sel, n_sel, kb, vb)
        assert (vb[4, 0] == 1).all() and (vb[4, 1] == 2).all() and (vb[3] == 6).all()


def test_two_streams_and_a_replayed_graph():
    """Calls on two streams with a workspace each, and store + attention captured once and replayed."""
    l = L()
    rng = np.random.default_rng(11)
    s, g, rows, budget, window = 8, 4, 600, 500, 32
    codes, scales = (x.to(DEV) for x in pool_of(rng, s, rows))
    sel = torch.from_numpy(rng.integers(0, rows, (s, budget)).astype(np.int32)).to(DEV)
    n_sel = torch.full((s,), budget, dtype=torch.int32, device=DEV)
    kl, vl = (torch.randn(s, window, 128, device=DEV).bfloat16() for _ in range(2))
    size = l.sparse_decode_attn_rows_q4_workspace_size(s, g, budget, window)
    assert size > 0
    qs = [torch.randn(1, s * g, 128, device=DEV).bfloat16() for _ in range(2)]
    ref = []
    for q in qs:
        o = torch.zeros_like(q)
        l.sparse_decode_attn_rows_q4(q, s, codes, scales, sel, n_sel, kl, vl, 3, 20, o)
        ref.append(o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [torch.zeros_like(q) for q in qs]
    for _ in range(20):
        for i in range(2):
            l.sparse_decode_attn_rows_q4(qs[i], s, codes, scales, sel, n_sel, kl, vl, 3, 20, outs[i], workspace=ws[i],
                                         stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))

    def one(x):
        l.segment_output_q4(x["kn"], x["vn"], x["kl"], x["vl"], 40, 8, x["reps"], x["st"], x["sz"], 2, x["codes"],
                            x["scales"], 100)
        l.sparse_decode_attn_rows_q4(qs[0], s, x["codes"], x["scales"], sel, n_sel, x["kl"], x["vl"], 8, 25, x["out"],
                                     workspace=ws[0])

    def fresh():
        torch.manual_seed(5)
        return dict(kn=torch.randn(s, 128, device=DEV).bfloat16(), vn=torch.randn(s, 128, device=DEV).bfloat16(),
                    kl=kl.clone(), vl=vl.clone(), reps=torch.zeros(s, 9, 128, device=DEV),
                    st=torch.zeros(s, 9, dtype=torch.int32, device=DEV), sz=torch.zeros(s, 9, dtype=torch.int32, device=DEV),
                    codes=codes.clone(), scales=scales.clone(), out=torch.zeros_like(qs[0]))
    eager, cap = fresh(), fresh()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            one(cap)
    for i in range(4):
        kn = torch.randn(s, 128, device=DEV).bfloat16()
        for x in (eager, cap):
            x["kn"].copy_(kn)
        one(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eager[n], cap[n]) for n in eager), i


def test_a_workspace_of_the_call_is_memory_of_its_stream():
    """Without a workspace the call takes one that the caller's stream does not reuse while it runs."""
    l, size = L(), 3 << 20
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        ws, n = l._ws_bytes(None, DEV, size, stream)
        at = ws.data_ptr()
        assert n == size and torch.cuda.current_stream() != side
        del ws
        other = torch.empty(size, dtype=torch.uint8, device=DEV)
        assert other.data_ptr() != at
        del other
    rng = np.random.default_rng(12)
    s, g, budget = 2, 4, 700
    codes, scales = (x.to(DEV) for x in pool_of(rng, s, 800))
    sel = torch.from_numpy(rng.integers(0, 800, (s, budget)).astype(np.int32)).to(DEV)
    n_sel = torch.full((s,), budget, dtype=torch.int32, device=DEV)
    q = torch.randn(1, s * g, 128, device=DEV).bfloat16()
    loc = torch.randn(s, 16, 128, device=DEV).bfloat16()
    assert l.sparse_decode_attn_rows_q4_workspace_size(s, g, budget, 16) > 0
    outs = [torch.zeros_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    for out, stream in zip(outs, (None, side, side.cuda_stream)):
        l.sparse_decode_attn_rows_q4(q, s, codes, scales, sel, n_sel, loc, loc, 0, 16, out, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    with pytest.raises(l.LouisKVError, match="aligned"):     # a view that starts in the middle of 16 bytes
        odd = torch.zeros(s * g * 128 + 4, device=DEV, dtype=torch.bfloat16)[4:].view(1, s * g, 128)
        l.sparse_decode_attn_rows_q4(odd, s, codes, scales, sel, n_sel, loc, loc, 0, 16, outs[0])
