"""The engine over a 4-bit pool, and its prompt attention.

Selections depend on index vectors and queries alone, so an engine with
pool_bits=4 must make those of a full-precision one bit for bit; its attention
is checked against the float64 oracle over the values its pool stands for."""
import numpy as np
import pytest
import torch

import synth
from attn_bounds import U, check_attention
from oracle import blocks as ob
from oracle import pool4 as o4

pytestmark = pytest.mark.gpu
DEV = "cuda"


def n64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def engines(dtype, n_groups=2, **kw):
    from paper_2510_11292_amd.engine import LouisKVEngine, config_from_workload
    wl = synth.get_workload("tiny-4k" if dtype == torch.float32 else "li-so-32k").replace(
        prompt_len=600, n_clusters=20, gen_len=150, budget=200, window=32, seg_len=8)
    data = synth.make_slices(wl, DEV, groups=[(0, i) for i in range(n_groups)] if dtype == torch.bfloat16 else [(0, 0)])
    cfg = config_from_workload(wl, n_groups=n_groups if dtype == torch.bfloat16 else 1, **kw)
    mk = lambda **k: LouisKVEngine(cfg, dtype, DEV, fused_step=False, **k)
    return wl, data, mk


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kw", [dict(), dict(segments="boundary"), dict(index="pages"),
                                dict(trigger="stride", stride=5)], ids=["fixed", "boundary", "pages", "stride"])
def test_decode_loop_over_a_4_bit_pool(dtype, kw):
    wl, data, mk = engines(dtype, **kw)
    full, four = mk(), mk(pool_bits=4)
    for e in (full, four):
        e.prefill(data.prompt_keys, data.prompt_values, data.init_idx)
    c = full.cfg
    P = c.prompt_len
    # the pool is the other engine's, quantised (rows 0..P-1; generated rows as they leave the window)
    def same_rows(lo, hi):
        from paper_2510_11292_amd import louiskv as L
        k, v = full.k_pool[:, lo:hi].contiguous(), full.v_pool[:, lo:hi].contiguous()
        cc = torch.zeros(k.shape[0], hi - lo, 128, dtype=torch.uint8, device=DEV)
        cs = torch.zeros(k.shape[0], hi - lo, 8, dtype=torch.uint8, device=DEV)
        L.pack_pool_q4(k, v, None, cc, cs)
        assert torch.equal(cc, four.codes[:, lo:hi]) and torch.equal(cs, four.scales[:, lo:hi])
    same_rows(0, P)
    H, g = c.n_kv_heads, c.n_q_heads // c.n_kv_heads
    checked = 0
    for t in range(wl.gen_len):
        args = (data.queries[t], data.gen_keys[t], data.gen_values[t])
        full.step(*args)
        four.step(*args)
        for n in ("fire", "reps", "unit_start", "unit_size", "n_sel", "n_sel_units", "k_local", "v_local", "q_ref"):
            assert torch.equal(getattr(full, n), getattr(four, n)), (t, n)
        if full.seg_state is not None:
            assert torch.equal(full.seg_state, four.seg_state)
        live = torch.arange(c.budget, device=DEV)[None] < four.n_sel[:, None]
        assert torch.equal(full.sel_rows[live], four.sel_rows[live])
        if t % 29 and t != wl.gen_len - 1:
            continue
        codes, scales, rows = four.codes.cpu().numpy(), four.scales.cpu().numpy(), four.sel_rows.cpu().numpy()
        n_sel, out, lse = four.n_sel.cpu().numpy(), n64(four.out), n64(four.lse)
        for s in range(0, c.n_slices, 3):
            first = (int(four.seg_state[s, 1]) if four.seg_state is not None
                     else 0 if t < c.window else ((t - c.window) // c.seg_len + 1) * c.seg_len)
            ring = [j % c.window for j in range(first, t + 1)]
            k, v = o4.values(codes[s, rows[s, :n_sel[s]]], scales[s, rows[s, :n_sel[s]]])
            k = np.concatenate([k, n64(four.k_local[s, ring])])
            v = np.concatenate([v, n64(four.v_local[s, ring])])
            q = n64(data.queries[t]).reshape(-1, g, 128)[s]
            want = ob.masked_attention(q, k, v, np.ones((g, len(k)), dtype=bool), 128 ** -0.5)
            check_attention(out.reshape(-1, g, 128)[s], lse.reshape(-1, g)[s], want, dtype == torch.bfloat16,
                            dtype == torch.bfloat16, len(k))
            checked += 1
    assert checked > 10
    if not kw:
        same_rows(P, P + full.n_units_before(wl.gen_len) * c.seg_len - c.n_clusters * c.seg_len)


def test_layer_by_layer_and_replayed_graph():
    wl, data, mk = engines(torch.bfloat16)
    a, b = mk(pool_bits=4), mk(pool_bits=4)
    for e in (a, b):
        e.prefill(data.prompt_keys, data.prompt_values, data.init_idx)
    top = max(data.prompt_values.abs().max().item(), data.gen_values.abs().max().item()) * 1.25   # held values round up
    for t in range(60):
        a.step(data.queries[t], data.gen_keys[t], data.gen_values[t])
        b.step_layer_by_layer(data.queries[t], data.gen_keys[t], data.gen_values[t])
        assert torch.equal(a.n_sel, b.n_sel) and torch.equal(a.k_local, b.k_local)
        # each is within 2^-8 (mean |v| + |o|) of the formula (tests/attn_bounds.py), both at most max |v|
        assert (a.out.float() - b.out.float()).abs().max() <= 2.0 ** -6 * top
    assert torch.equal(a.codes[:, :600 + 24], b.codes[:, :600 + 24])
    # steps 0..39 (evictions among them) as one graph, replayed after fresh prefills
    cap = mk(pool_bits=4)
    cap.prefill(data.prompt_keys, data.prompt_values, data.init_idx)
    outs = torch.zeros(40, *cap.out.shape, dtype=cap.out.dtype, device=DEV)

    def loop(e, o):
        e.t = 0
        for t in range(40):
            e.step(data.queries[t], data.gen_keys[t], data.gen_values[t])
            o[t].copy_(e.out)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        loop(cap, outs)
    for _ in range(3):
        eager = mk(pool_bits=4)
        eager.prefill(data.prompt_keys, data.prompt_values, data.init_idx)
        ref = torch.zeros_like(outs)
        loop(eager, ref)
        torch.cuda.synchronize()
        cap.prefill(data.prompt_keys, data.prompt_values, data.init_idx)
        outs.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs, ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_attention(dtype):
    """Whole and in chunks; with every block taken it is dense causal attention."""
    wl, data, mk = engines(dtype)
    eng = mk(pool_bits=4)
    c = eng.cfg
    n, G, H, g = c.prompt_len, c.n_groups, c.n_kv_heads, c.n_q_heads // c.n_kv_heads
    gen = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(G, c.n_q_heads, n, 128, generator=gen, device=DEV).to(dtype)
    keys, values = data.prompt_keys, data.prompt_values
    see = np.tril(np.ones((n, n), dtype=bool))
    dense = eng.prompt_attention(q, keys, values, n_top=100)
    for s in range(0, c.n_slices, 5):
        for j in (0, g - 1):
            want = ob.masked_attention(n64(q).reshape(-1, g, n, 128)[s, j], n64(keys[s]), n64(values[s]), see, 128 ** -0.5)
            check_attention(n64(dense).reshape(-1, g, n, 128)[s, j], None, want, dtype == torch.bfloat16,
                            dtype == torch.bfloat16, n)
    # tiles and blocks of a chunk at a multiple of both are the whole prompt's
    sparse = eng.prompt_attention(q, keys, values, block_len=32, q_block=32, n_top=4, n_recent=1)
    for a, b in ((0, 320), (320, 600)):
        part = eng.prompt_attention(q[:, :, a:b].contiguous(), keys[:, :b].contiguous(), values[:, :b].contiguous(), a,
                                    block_len=32, q_block=32, n_top=4, n_recent=1)
        # two results, each as far from the formula as tests/attn_bounds.py allows with mean |v| at most max |v|
        size = max((q.reshape(-1, g * n, 128)[s].float().abs() @ keys[s].float().abs().T).max().item()
                   for s in range(c.n_slices)) * 128 ** -0.5
        tol = 2 * (280 * U * size + (3 * n + 32) * U) * values.abs().max().item()
        tol += 2.0 ** -6 * values.abs().max().item() if dtype == torch.bfloat16 else 0.0
        assert (part.float() - sparse[:, :, a:b].float()).abs().max() <= tol
    assert (sparse.float() - dense.float()).abs().max() > tol
    with pytest.raises(ValueError):
        eng.prompt_attention(q, keys, values, block_len=48)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_attention_over_a_buffer_that_is_still_filling(dtype):
    """Rows behind the queries, here NaN and infinities, change nothing: chunks and tokens read one whole buffer."""
    wl, data, mk = engines(dtype)
    eng = mk(pool_bits=4)
    c = eng.cfg
    gen = torch.Generator(device=DEV).manual_seed(5)
    q = torch.randn(c.n_groups, c.n_q_heads, c.prompt_len, 128, generator=gen, device=DEV).to(dtype)
    kw = dict(block_len=32, q_block=32, n_top=4, n_recent=1)
    for a, b in ((320, 451), (451, 452), (500, 600)):
        keys, values = data.prompt_keys.clone(), data.prompt_values.clone()
        keys[:, b:], values[:, b:] = float("nan"), float("inf")
        qc = q[:, :, a:b].contiguous()
        short = eng.prompt_attention(qc, keys[:, :b].contiguous(), values[:, :b].contiguous(), a, **kw)
        assert torch.isfinite(short).all() and torch.equal(eng.prompt_attention(qc, keys, values, a, **kw), short), (a, b)
