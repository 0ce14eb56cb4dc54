"""Shared prefixes and bounded caches without a GPU: the oracle's rules, and what the calls refuse before any launch."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import blocks as ob
from oracle import prefix as op

P = ctypes.c_void_p
NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
D16, ODD = P(4096), P(4104)


@pytest.fixture(scope="module")
def lib():
    from paper_2510_11292_amd import louiskv
    return louiskv.load_library()


def refused(fn, base, table):
    for change, want in table:
        args = list(base)
        for i, v in change.items():
            args[i] = v
        got = fn(*args)
        assert got == want, f"{change}: {got}, expected {want}"


# ------------------------------------------------------------------- the oracle

def test_weights_are_the_columns_of_the_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((6, 8)), rng.standard_normal((11, 8)), rng.standard_normal((11, 3))
    see = np.arange(11)[None] <= 4 + np.arange(6)[:, None]
    see[2] = False
    out, lse, _, _ = ob.masked_attention(q, k, v, see, 0.3)
    w, size = op.row_weights(q, k, see, lse, 0.3)
    x = np.where(see, q @ k.T * 0.3, -np.inf)
    rows = [0, 1, 3, 4, 5]
    p = np.exp(x[rows]) / np.exp(x[rows]).sum(1, keepdims=True)
    np.testing.assert_allclose(w, p.sum(0), rtol=1e-12)
    np.testing.assert_allclose(p @ v, out[rows], rtol=1e-12)
    assert abs(w.sum() - 5) < 1e-12 and (size >= 0).all()


def test_rows_that_stay_by_hand():
    pos = list(range(6))
    # row 0 is protected (first), 5 (recent); of 1..4 the two lightest leave: 2 and 4
    assert op.rows_that_stay([0.0, 3.0, 1.0, 2.0, 0.5, 0.0], pos, 6, 6, 4, 1, 1) == [0, 1, 5, 3]
    # equal weights: the lower rows leave
    assert op.rows_that_stay([1.0] * 6, pos, 6, 6, 3, 0, 0) == [3, 4, 5]
    assert op.rows_that_stay([1.0] * 6, pos, 6, 6, 3, 1, 0) == [0, 4, 5]
    nan = float("nan")
    assert op.rows_that_stay([nan, -np.inf, 0.0, nan], pos, 4, 4, 2, 0, 0) == [2, 1]
    assert op.rows_that_stay([-0.0, 0.0], pos, 2, 2, 1, 0, 0) == [1]
    # fewer rows than fit: all stay where they are; none kept
    assert op.rows_that_stay([1.0, 2.0], pos, 2, 2, 5, 0, 1) == [0, 1]
    assert op.rows_that_stay([1.0, 2.0], pos, 2, 2, 0, 0, 0) == []
    # positions, not rows, are protected
    assert op.rows_that_stay([5.0, 1.0, 1.0, 9.0], [7, 9, 0, 8], 4, 10, 2, 1, 1) == [2, 1]


# ------------------------------------------------------------------- refusals

def test_attention_refuses(lib):
    size = lib.louiskv_shared_prefix_attn_workspace_size
    ws = size(32, 8, 4, 1, 128, 4096, 600, 1)
    assert ws > 0 and size(0, 8, 4, 1, 128, 4096, 600, 1) == size(32, 8, 9, 1, 128, 4096, 600, 1) == 0
    assert size(32, 8, 4, 0, 128, 4096, 600, 1) == size(32, 5, 4, 1, 128, 4096, 600, 1) == size(32, 8, 4, 1, 128, -1, 600, 1) == 0
    assert size(32, 8, 4, 1, 128, 4096, (1 << 30) + 1, 1) == size(1 << 62, 8, 4, 1, 128, 4096, 600, 1) == 0
    #       q    dt S   kv g  nq d    scale kp   vp  Sp rows  np   ko   vo   rows no  w    out odt lse ws   bytes
    base = [D16, 1, 32, 8, 4, 1, 128, 0.1, D16, D16, 8, 4096, None, D16, D16, 600, D16, D16, D16, 1, None, D16, ws, None]
    refused(lib.louiskv_shared_prefix_attn, base, [
        ({0: None}, NULL), ({18: None}, NULL), ({8: None}, NULL), ({9: None}, NULL), ({13: None}, NULL), ({14: None}, NULL),
        ({1: 2}, DTYPE), ({19: -1}, DTYPE), ({6: 64}, UNSUPPORTED), ({4: 0}, UNSUPPORTED), ({4: 9}, UNSUPPORTED),
        ({2: 0}, SHAPE), ({2: 33}, SHAPE), ({3: 0}, SHAPE), ({3: 5}, SHAPE), ({5: 0}, SHAPE), ({5: 1 << 30}, SHAPE),
        ({2: 1 << 40}, SHAPE), ({10: 0}, SHAPE), ({10: 4}, SHAPE), ({10: 24}, SHAPE), ({11: -1}, SHAPE),
        ({11: (1 << 30) + 1}, SHAPE), ({15: -1}, SHAPE), ({15: (1 << 30) + 1}, SHAPE),
        ({0: ODD}, UNSUPPORTED), ({8: ODD}, UNSUPPORTED), ({9: ODD}, UNSUPPORTED), ({13: ODD}, UNSUPPORTED),
        ({14: ODD}, UNSUPPORTED), ({18: ODD}, UNSUPPORTED), ({21: None}, WORKSPACE), ({21: ODD}, WORKSPACE),
        ({22: ws - 1}, WORKSPACE)])


def test_weights_refuse(lib):
    size = lib.louiskv_attn_weights_workspace_size
    assert size(0, 4, 64, 128, 4096) == size(8, 9, 64, 128, 4096) == size(8, 4, 0, 128, 4096) == size(8, 4, 64, 128, -1) == 0
    ws = size(8, 4, 64, 128, 4096)
    #       q    dt S  kv g  nq  d    scale keys rows n    lse  w    ws   bytes
    base = [D16, 1, 8, 8, 4, 64, 128, 0.1, D16, 4096, D16, D16, D16, D16, ws, None]
    refused(lib.louiskv_attn_weights, base, [
        ({0: None}, NULL), ({8: None}, NULL), ({11: None}, NULL), ({12: None}, NULL), ({1: 7}, DTYPE),
        ({6: 256}, UNSUPPORTED), ({4: 12}, UNSUPPORTED), ({2: 12}, SHAPE), ({5: 0}, SHAPE), ({9: 0}, SHAPE),
        ({9: (1 << 30) + 1}, SHAPE), ({0: ODD}, UNSUPPORTED), ({8: ODD}, UNSUPPORTED)]
        + ([({13: None}, WORKSPACE), ({14: ws - 1}, WORKSPACE)] if ws else []))


def test_eviction_refuses(lib):
    size = lib.louiskv_evict_rows_workspace_size
    ws = size(8, 4096, 512)
    assert ws > 0 and size(0, 4096, 512) == size(8, 0, 512) == size(8, 4096, 0) == size(1 << 62, 4096, 512) == 0
    a = [P(1 << 30 | i << 26) for i in range(1, 12)]        # buffers far from each other
    #       w     pos  n     seen  dt S  d    rows  keep fst rec k     v     k_to  v_to  w_to  p_to  to   n_to  ws    bytes
    base = [a[0], a[1], a[2], a[3], 1, 8, 128, 4096, 512, 4, 64, a[4], a[5], a[6], a[7], a[8], a[9], 600, a[10], D16, ws, None]
    refused(lib.louiskv_evict_rows, base, [
        ({0: None}, NULL), ({11: None}, NULL), ({12: None}, NULL), ({13: None}, NULL), ({14: None}, NULL), ({18: None}, NULL),
        ({1: None}, NULL), ({3: None}, NULL), ({4: 4}, DTYPE), ({6: 64}, UNSUPPORTED), ({5: 0}, SHAPE), ({7: 0}, SHAPE),
        ({7: (1 << 30) + 1}, SHAPE), ({8: 0}, SHAPE), ({8: 601}, SHAPE), ({9: -1}, SHAPE), ({10: -1}, SHAPE),
        ({9: 449}, SHAPE), ({10: (1 << 31) - 1}, SHAPE), ({5: 1 << 23}, SHAPE), ({11: P((1 << 30) + 8)}, UNSUPPORTED),
        # a part of another buffer, the same buffer with another number of rows, another input's buffer
        ({13: P(a[4].value + 4096)}, SHAPE), ({13: a[4]}, SHAPE), ({13: a[5]}, SHAPE), ({14: a[6]}, SHAPE),
        ({15: a[4]}, SHAPE), ({18: a[3]}, SHAPE), ({18: a[8]}, SHAPE),
        ({19: None}, WORKSPACE), ({19: ODD}, WORKSPACE), ({20: ws - 1}, WORKSPACE)])


def test_store_refuses(lib):
    size = lib.louiskv_store_evict_workspace_size
    assert size(0, 600, 1, 512) == size(8, 600, 0, 512) == size(8, 600, 1, 601) == size(8, 600, 9, 8) == 0
    ws = size(8, 600, 3, 512)
    #       kn   vn   dt S  new d    k    v    w    pos  n    seen rows bud  fst rec ws  bytes
    base = [D16, D16, 1, 8, 3, 128, D16, D16, D16, D16, D16, D16, 600, 512, 4, 64, D16, ws, None]
    refused(lib.louiskv_store_evict, base, [
        *[({i: None}, NULL) for i in (0, 1, 6, 7, 8, 9, 10, 11)], ({2: -1}, DTYPE), ({5: 96}, UNSUPPORTED), ({3: 0}, SHAPE),
        ({4: 0}, SHAPE), ({4: 513}, SHAPE), ({13: 601}, SHAPE), ({13: 2}, SHAPE), ({12: (1 << 30) + 1}, SHAPE),
        ({14: 446}, SHAPE), ({15: 506}, SHAPE), ({14: -1}, SHAPE), ({15: -1}, SHAPE), ({0: ODD}, UNSUPPORTED),
        ({7: ODD}, UNSUPPORTED)] + ([({16: None}, WORKSPACE), ({17: ws - 1}, WORKSPACE)] if ws else []))
    a = [P(1 << 30 | i << 26) for i in range(1, 9)]         # buffers far from each other, but for one
    base = [a[0], a[1], 1, 8, 3, 128, *a[2:8], 600, 512, 4, 64, D16, max(ws, 1), None]
    refused(lib.louiskv_store_evict, base, [
        ({0: P(a[2].value + 256)}, SHAPE), ({1: a[3]}, SHAPE), ({7: P(a[2].value + 4096)}, SHAPE), ({9: a[4]}, SHAPE),
        ({11: a[6]}, SHAPE), ({10: a[5]}, SHAPE), ({8: a[1]}, SHAPE)])


def test_calls_too_large_for_a_launch_are_refused_before_any(lib):
    # 2^20 slices of 4096 own rows: as many blocks fit, the weights' do not
    many = [D16, 1, 1 << 20, 8, 4, 16, 128, 0.1, None, None, 0, 0, None, D16, D16, 4096, None, None, D16, 1, None, D16,
            1 << 62, None]
    refused(lib.louiskv_shared_prefix_attn, many, [({5: 8, 15: 1 << 20, 17: D16}, SHAPE), ({17: D16, 5: 8, 2: 1 << 23}, SHAPE)])
    refused(lib.louiskv_attn_weights, [D16, 1, 1 << 20, 8, 4, 8, 128, 0.1, D16, 1 << 20, None, D16, D16, D16, 1 << 62, None],
            [({5: 8, 2: 1 << 23}, SHAPE), ({2: 1 << 16, 5: 128, 9: 1 << 30}, SHAPE)])


def test_python_calls_refuse_sizes_types_and_host_memory():
    from paper_2510_11292_amd import louiskv as L
    i32 = dict(dtype=torch.int32)
    q, kp, ko, out = torch.zeros(3, 4, 2, 128), torch.zeros(2, 9, 128), torch.zeros(6, 5, 128), torch.zeros(3, 4, 2, 128)
    n_p, n_o, w, lse = torch.zeros(2, **i32), torch.zeros(6, **i32), torch.zeros(6, 5), torch.zeros(3, 4, 2)
    pos, ws = torch.zeros(6, 5, **i32), torch.zeros(1 << 16, dtype=torch.uint8)

    def attn(q=q, kp=kp, vp=kp, n_p=n_p, ko=ko, vo=ko, n_o=n_o, out=out, lse=lse, w=w):
        L.shared_prefix_attn(q, 2, kp, vp, n_p, ko, vo, n_o, out, lse, weights=w, workspace=ws, stream=0)

    def weights(keys=ko, n=n_o, lse=lse, w=w):
        L.attn_weights(q, 2, keys, n, lse, w, workspace=ws, stream=0)

    def evict(w=w, pos=pos, n=n_o, seen=n_o, v=ko, to=ko, w_to=w, pos_to=pos, n_to=n_o):
        L.evict_rows(w, pos, n, seen, 3, 1, 1, ko, v, to, ko, w_to, pos_to, n_to, workspace=ws, stream=0)

    def store(new=ko[:, :1], v_new=ko[:, :1], v=ko, w=w, pos=pos, n=n_o, seen=n_o):
        L.store_evict(new.contiguous(), v_new, ko, v, w, pos, n, seen, 4, 1, 1, workspace=ws, stream=0)
    for call, kw in ((attn, dict(vp=kp[:, :8])), (attn, dict(n_p=n_p[:1])), (attn, dict(vo=ko[:5])), (attn, dict(ko=ko[:5])),
                     (attn, dict(n_o=n_o[:5])), (attn, dict(out=out[:, :3])), (attn, dict(lse=lse[0])),
                     (attn, dict(w=w[:, :4])), (weights, dict(keys=ko[:4])), (weights, dict(n=n_o[:1])),
                     (weights, dict(lse=lse[:2])), (weights, dict(w=w[:, :3])), (evict, dict(w=w[:1])), (evict, dict(pos=pos[:1])),
                     (evict, dict(v=ko[:5])), (evict, dict(n=n_o[:1])), (evict, dict(seen=n_o[:1])), (evict, dict(w_to=w[:1])),
                     (evict, dict(pos_to=pos[:1])), (evict, dict(n_to=n_o[:1])), (evict, dict(to=ko[:, :4])),
                     (store, dict(v_new=ko[:, :2])), (store, dict(v=ko[:5])), (store, dict(w=w[:5])), (store, dict(pos=pos[:5])),
                     (store, dict(n=n_o[:5])), (store, dict(seen=n_o[:5]))):
        with pytest.raises(ValueError, match="expected"):
            call(**kw)
    for call, kw in ((attn, dict(n_o=n_o.long())), (attn, dict(n_p=n_p.float())), (attn, dict(kp=kp.bfloat16())),
                     (attn, dict(w=w.double())), (weights, dict(n=n_o.long())), (weights, dict(w=w.bfloat16())),
                     (weights, dict(lse=lse.double())), (evict, dict(pos=pos.long())), (evict, dict(w=w.bfloat16())),
                     (evict, dict(n_to=n_o.long())), (store, dict(v_new=ko[:, :1].bfloat16())), (store, dict(n=n_o.long()))):
        with pytest.raises(TypeError, match="expected"):
            call(**kw)
    with pytest.raises(ValueError, match="multiple"):
        attn(q=torch.zeros(3, 3, 2, 128), out=torch.zeros(3, 3, 2, 128), lse=None)
    for kw in (dict(kp=None), dict(kp=None, vp=None), dict(ko=None, vo=None), dict(ko=None, vo=None, w=None)):
        with pytest.raises(ValueError, match="None"):
            attn(**kw)
    with pytest.raises(ValueError, match="queries"):
        attn(q=q[0, 0])
    for call in (attn, weights, evict, store):      # every size is right: host memory is what is left
        with pytest.raises(ValueError, match="current device|contiguous"):
            call()
    with pytest.raises(TypeError, match="dtype"):
        h = torch.float16
        L.shared_prefix_attn(q.to(h), 2, kp.to(h), kp.to(h), None, None, None, None, out, stream=0)


def test_a_step_that_is_refused_stores_nothing(monkeypatch):
    """Queries that do not fit the new rows are refused before those enter the caches."""
    from paper_2510_11292_amd import engine
    from paper_2510_11292_amd.engine import BranchConfig, BranchEngine
    e = BranchEngine(BranchConfig(n_branches=2, n_layers=1, n_kv_heads=2, n_q_heads=4, prompt_len=5, budget=16, n_first=1,
                                  n_recent=2, n_new=3), torch.float32, "cpu")
    k = torch.zeros(4, 128)
    with pytest.raises(RuntimeError, match="prefill"):
        e.step(torch.zeros(2, 4, 128), k, k)
    e.prefill(torch.zeros(2, 5, 128), torch.zeros(2, 5, 128))
    q = torch.zeros(2, 4, 128)
    stores = []

    class Recorder:
        def store_evict(self, *a, **kw):
            stores.append(a)
    monkeypatch.setattr(engine, "L", Recorder())
    k3 = torch.zeros(4, 3, 128)
    for bad, rows in ((torch.zeros(2, 4, 2, 128), k), (torch.zeros(2, 4, 2, 128), k3), (q, k3), (q[:1], k), (q[:, :2], k),
                      (q[..., :64], k), (q.bfloat16(), k), (torch.zeros(2, 128, 4).transpose(1, 2), k), (q[0], k),
                      (torch.zeros(2, 4, 4, 128), torch.zeros(4, 4, 128))):
        with pytest.raises(ValueError):
            e.step(bad, rows, rows)
    for out in (torch.zeros(2, 4, 1, 128), torch.zeros(2, 128, 4).transpose(1, 2)):
        with pytest.raises(ValueError, match="out"):
            e.step(q, k, k, out)
    assert not stores and e.n_seen.eq(0).all()
    for heads in (18, 0):
        with pytest.raises(ValueError, match="positive"):
            BranchEngine(BranchConfig(n_branches=1, n_layers=1, n_kv_heads=2, n_q_heads=heads, prompt_len=5, budget=200),
                         torch.float32, "cpu")


def test_a_prompt_is_copied_to_the_engine_s_rows():
    """A captured step reads the addresses of its capture: they stay, and hold the last prompt."""
    from paper_2510_11292_amd.engine import BranchConfig, BranchEngine
    e = BranchEngine(BranchConfig(n_branches=2, n_layers=3, n_kv_heads=2, n_q_heads=4, prompt_len=5, budget=16, n_first=1,
                                  n_recent=2), torch.float32, "cpu")
    places = set()
    for i in range(2):
        keys, values = torch.randn(6, 5, 128), torch.randn(5, 6, 128).transpose(0, 1)
        e.n_rows.fill_(7)
        e.prefill(keys, values)
        places.add((e.k_prefix.data_ptr(), e.v_prefix.data_ptr()))
        assert torch.equal(e.k_prefix, keys) and torch.equal(e.v_prefix, values) and e.v_prefix.is_contiguous()
        assert (e.n_rows == 0).all() and e.k_prefix.data_ptr() != keys.data_ptr()
    assert len(places) == 1
    e.k_prefix.normal_()                        # the caller may fill them in place
    keys = e.k_prefix.clone()
    e.prefill(e.k_prefix, e.v_prefix)
    assert torch.equal(e.k_prefix, keys) and torch.equal(e.v_prefix, values)
    e.prefill(keys.clone().requires_grad_(), values)      # a model's keys: the engine holds none of their graph
    assert torch.equal(e.k_prefix, keys) and not e.k_prefix.requires_grad
    for k, v in ((keys.bfloat16(), values), (keys, values.double()), (keys[:, :4], values), (keys, values[:5])):
        with pytest.raises(ValueError, match="expected"):
            e.prefill(k, v)
    assert torch.equal(e.k_prefix, keys)
    cut = BranchEngine(BranchConfig(n_branches=2, n_layers=3, n_kv_heads=2, n_q_heads=4, prompt_len=50, budget=16, n_first=1,
                                    n_recent=2, prefix_budget=9), torch.float32, "cpu")
    x = torch.zeros(12, 128)
    with pytest.raises(RuntimeError, match="prefill"):
        cut.step(torch.zeros(6, 4, 128), x, x)


def test_a_step_stores_nothing_that_its_attention_would_refuse(monkeypatch):
    """Queries and results of another type, place or alignment are refused before the new rows enter the caches."""
    from paper_2510_11292_amd import engine
    from paper_2510_11292_amd.engine import BranchConfig, BranchEngine
    cfg = BranchConfig(n_branches=2, n_layers=1, n_kv_heads=2, n_q_heads=4, prompt_len=5, budget=16, n_first=1, n_recent=2)
    e = BranchEngine(cfg, torch.float32, "cpu")
    e.prefill(torch.zeros(2, 5, 128), torch.zeros(2, 5, 128))
    q, k = torch.zeros(2, 4, 128), torch.zeros(4, 128)
    calls = []

    class Recorder:
        def store_evict(self, *a, **kw):
            calls.append("store")

        def shared_prefix_attn(self, *a, **kw):
            calls.append("attn")
    monkeypatch.setattr(engine, "L", Recorder())

    def odd(x):                                 # the same, 4 bytes off a 16-byte boundary
        y = torch.zeros(x.numel() + 8)
        at = next(i for i in range(8) if (y.data_ptr() + 4 * i) % 16 == 4)
        return y[at:at + x.numel()].view(x.shape)
    for bad in (odd(q), q.to("meta")):
        with pytest.raises(ValueError, match="q "):
            e.step(bad, k, k)
    for out in (q.half(), q.double(), q.int(), odd(q), q.to("meta")):
        with pytest.raises(ValueError, match="out "):
            e.step(q, k, k, out)
    assert not calls
    for out in (None, torch.zeros_like(q), q.bfloat16()):
        got = e.step(q, k, k, out)
        assert got is (e.out if out is None else out) and calls == ["store", "attn"]
        calls.clear()
    monkeypatch.undo()
    for types in ((torch.float16, None), (torch.float32, torch.float16), (torch.float64, torch.float32)):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            BranchEngine(cfg, types[0], "cpu", out_dtype=types[1])


def test_sizes_that_fit_the_card_are_not_refused(lib):
    """64 branches of 256 (layer, KV head) slices with caches of 2048 rows, 1024 slices of 32768 rows kept, and the most
    slices: what is refused is a buffer's alignment or the missing workspace, which are looked at behind the sizes."""
    a = [P(1 << 30 | i << 26) for i in range(1, 12)]

    def store(s, new, rows, k):
        return lib.louiskv_store_evict(a[0], a[1], 1, s, new, 128, k, a[3], a[4], a[5], a[6], a[7], rows, rows, 4, 64, None, 0,
                                       None)

    def evict(s, rows, keep):
        far = [P(i << 50) for i in range(1, 12)]
        return lib.louiskv_evict_rows(far[0], far[1], far[2], far[3], 1, s, 128, rows, keep, 4, 64, far[4], far[5], far[6],
                                      far[7], far[8], far[9], keep, far[10], None, 0, None)
    for s, new, rows in ((16384, 1, 2048), (16384, 64, 2048), (1024, 1, 32768), (1 << 20, 1, 300), ((1 << 22) - 1, 1, 70)):
        assert store(s, new, rows, ODD) == UNSUPPORTED, (s, new, rows)
        assert lib.louiskv_store_evict_workspace_size(s, rows, new, rows) == 0          # one launch
    for s, new, rows in ((16384, 100, 2048), (1024, 1, 40000), (8192, 1, 40000)):
        size = lib.louiskv_store_evict_workspace_size(s, rows, new, rows)
        assert size >= s * (rows - new) * 4 and store(s, new, rows, ODD) == UNSUPPORTED, (s, new, rows)
    for s, rows, keep in ((16384, 32768, 2048), (1024, 40000, 32768), (16383, 32768, 32767), ((1 << 22) - 1, 70, 70)):
        size = lib.louiskv_evict_rows_workspace_size(s, rows, keep)
        assert size >= s * keep * 4 and evict(s, rows, keep) == WORKSPACE, (s, rows, keep)
    # more blocks than a launch holds: refused, and no workspace
    for s, rows, keep in ((16384, 32768, 32767), (1 << 22, 4096, 100), (1 << 20, 4096, 513), (1 << 14, 1 << 20, 1 << 20)):
        assert lib.louiskv_evict_rows_workspace_size(s, rows, keep) == 0 and evict(s, rows, keep) == SHAPE, (s, rows, keep)
    assert lib.louiskv_store_evict_workspace_size(1 << 20, 1 << 20, 100, 1 << 20) == 0
    assert store(1 << 22, 1, 4096, ODD) == store(16384, 1, 32769, ODD) == SHAPE and store(1 << 20, 100, 1 << 20, ODD) == SHAPE
    # the attention of as many slices, whose workspace is 0 where the call is refused
    size = lib.louiskv_shared_prefix_attn_workspace_size
    attn = [D16, 1, (1 << 22) - 1, 1, 4, 1, 128, 0.1, D16, D16, (1 << 22) - 1, 9, None, D16, D16, 70, None, D16, D16, 1, None,
            None, 0, None]
    assert size(attn[2], attn[2], 4, 1, 128, 9, 70, 1) > 0
    refused(lib.louiskv_shared_prefix_attn, attn, [({}, WORKSPACE)])
    assert size(1 << 20, 1, 4, 8, 128, 0, 1 << 20, 1) == size(1 << 20, 1, 4, 16, 128, 0, 1 << 20, 1) == 0
    assert lib.louiskv_attn_weights_workspace_size(1 << 16, 4, 128, 128, 1 << 30) == 0


def test_an_engine_that_no_step_fits_is_refused():
    from paper_2510_11292_amd.engine import BranchConfig, BranchEngine
    base = dict(n_branches=64, n_layers=32, n_kv_heads=8, n_q_heads=64, prompt_len=1 << 17, budget=2048)
    BranchEngine(BranchConfig(n_new=256, **base), torch.bfloat16, "meta")
    with pytest.raises(ValueError, match="too many"):
        BranchEngine(BranchConfig(n_new=257, **base), torch.bfloat16, "meta")
    with pytest.raises(ValueError, match="too many"):
        BranchEngine(BranchConfig(**{**base, "n_branches": 1 << 16}), torch.bfloat16, "meta")


def test_a_prefix_of_no_rows_is_refused():
    from paper_2510_11292_amd.engine import BranchConfig, BranchEngine
    for budget in (0, -1):
        with pytest.raises(ValueError, match="prefix_budget"):
            BranchEngine(BranchConfig(n_branches=2, n_layers=1, n_kv_heads=2, n_q_heads=4, prompt_len=5, budget=16, n_first=0,
                                      n_recent=0, prefix_budget=budget), torch.float32, "cpu")
