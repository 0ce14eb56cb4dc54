"""The 4-bit pool and the prompt's block calls without a GPU: the oracle's format
against facts that do not retype it, and the refusals of every entry point,
which return before any launch."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import blocks as ob
from oracle import pool4 as o4

P = ctypes.c_void_p
OK, NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    from paper_2510_11292_amd import louiskv
    if not os.path.exists(louiskv.LIB_PATH):
        pytest.fail("liblouiskv.so is not built")
    return louiskv.load_library()


def test_levels_and_nibbles_round_trip():
    rng = np.random.default_rng(0)
    codes = rng.integers(0, 256, (5, 128), dtype=np.uint8)
    scales = rng.integers(100, 150, (5, 8), dtype=np.uint8)
    k, v = o4.values(codes, scales)
    assert k[0, 0] == (-1.0 if codes[0, 0] & 8 else 1.0) * o4.LEVELS[codes[0, 0] & 7] * 2.0 ** (int(scales[0, 0]) - 127)
    assert v[4, 127] == ((-1.0 if codes[4, 127] & 128 else 1.0) * o4.LEVELS[(codes[4, 127] >> 4) & 7]
                         * 2.0 ** (int(scales[4, 7]) - 127))
    # what the values quantise to stands for the same values: a fixed point
    for x in (k, v):
        c, s = o4.quantise(x)
        b, sc = o4.pack_bytes(c, s, c, s)
        np.testing.assert_array_equal(o4.values(b, sc)[0], x)


def test_quantisation_is_nearest_and_within_a_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 128)) * 2.0 ** rng.integers(-30, 30, (40, 1))
    c, s = o4.quantise(x)
    held = o4.values(*o4.pack_bytes(c, s, c, s))[0]
    unit = np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=1)
    assert np.all(np.abs(held - x) <= unit)
    grid = np.concatenate([-o4.LEVELS, o4.LEVELS])
    best = np.abs(x[..., None] - grid * unit[..., None]).min(-1)
    np.testing.assert_array_equal(np.abs(held - x), best)
    top = np.abs(x).reshape(40, 4, 32).max(-1)
    assert np.all(top <= 7 * 2.0 ** (s.astype(float) - 127)) and np.all(top > 3.5 * 2.0 ** (s.astype(float) - 127))


def test_ties_extremes_and_blocks_that_are_not_finite():
    x = np.zeros((4, 128))
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -5.0, 6.5, 4.999, -7.0, 0.0, 1.0, 6.0]
    x[1, 3], x[1, 40] = np.inf, np.nan
    x[2, :3] = [2.0 ** -133, 2.0 ** -126, 2.0 ** -125]
    x[3, 0] = 3.3e38
    c, s = o4.quantise(x)
    held = o4.values(*o4.pack_bytes(c, s, c, s))[0]
    np.testing.assert_array_equal(held[0, :16], [0, 1, 1, 2, 2, 4, 4, 6, 0, -4, 6, 4, -6, 0, 1, 6])
    assert np.isnan(held[1, :64]).all() and (held[1, 64:] == 0).all()
    assert s[2, 0] == 2 and list(held[2, :3]) == [0.0, 2.0 ** -126, 2.0 ** -125]
    assert s[3, 0] == 252 and held[3, 0] == 6 * 2.0 ** 125


def test_oracle_selection_and_attention():
    rng = np.random.default_rng(2)
    reps = rng.standard_normal((20, 8))
    q = rng.standard_normal((6, 8))
    got = ob.tile_blocks(q, reps, 16 * 18 + 3, 16 * 19 + 2, 16, 1, 2, 3)
    assert got[0] == 0 and got[-4:] == [16, 17, 18, 19] and len(got) == 8
    score = q.sum(0) @ reps.T
    assert set(got[1:4]) == set(1 + np.argsort(-score[1:16])[:3])
    assert ob.tile_blocks(q, reps, 0, 5, 16, 1, 2, 3) == [0]
    assert ob.tile_blocks(q, np.ones((9, 8)), 16 * 8, 16 * 8, 16, 0, 0, 2) == [0, 1, 8]   # equal scores: the lower block
    k, v, qq = rng.standard_normal((9, 8)), rng.standard_normal((9, 8)), rng.standard_normal((3, 8))
    see = rng.random((3, 9)) < 0.5
    see[1] = False
    see[0, 0] = see[2, 1] = True
    out, lse, _, _ = ob.masked_attention(qq, k, v, see, 0.3)
    t = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (qq, k, v)),
                                                         attn_mask=torch.from_numpy(see)[None], scale=0.3)[0].numpy()
    np.testing.assert_allclose(out[[0, 2]], t[[0, 2]], rtol=1e-12)
    assert np.isneginf(lse[1]) and (out[1] == 0).all()


# ------------------------------------------------------------------- refusals

def _statuses(fn, base, table):
    for change, want in table:
        args = list(base)
        for i, v in change.items():
            args[i] = v
        got = fn(*args)
        assert got == want, f"{change}: {got}, expected {want}"


D16 = P(4096)


def test_pack_and_gather_refuse(lib):
    base = [D16, D16, 1, 2, 64, 128, None, D16, D16, 64, None]
    _statuses(lib.louiskv_pack_pool_q4, base, [
        ({0: None}, NULL), ({1: None}, NULL), ({7: None}, NULL), ({8: None}, NULL), ({2: 2}, DTYPE),
        ({5: 64}, UNSUPPORTED), ({3: 0}, SHAPE), ({4: 0}, SHAPE), ({9: 63}, SHAPE), ({9: (1 << 24) + 1}, SHAPE),
        ({7: P(4104)}, UNSUPPORTED), ({8: P(4100)}, UNSUPPORTED)])
    base = [D16, D16, 2, 64, 128, None, None, 64, D16, D16, 1, None]
    _statuses(lib.louiskv_gather_rows_q4, base, [
        ({0: None}, NULL), ({9: None}, NULL), ({10: 5}, DTYPE), ({4: 96}, UNSUPPORTED), ({2: 0}, SHAPE),
        ({7: 0}, SHAPE), ({7: 65}, SHAPE), ({3: 0}, SHAPE), ({0: P(4100)}, UNSUPPORTED)])


def test_segment_stores_refuse(lib):
    #       k_new v_new dt S  d    kl   vl  win step seg reps st  size cap nc codes scales rows prompt
    base = [D16, D16, 1, 8, 128, D16, D16, 64, 64, 32, D16, D16, D16, 10, 9, D16, D16, 132, 100, None]
    _statuses(lib.louiskv_segment_output_q4, base, [
        ({0: None}, NULL), ({6: None}, NULL), ({10: None}, NULL), ({15: None}, NULL), ({16: None}, NULL),
        ({2: 9}, DTYPE), ({4: 64}, UNSUPPORTED), ({3: 0}, SHAPE), ({7: 60}, SHAPE), ({8: -1}, SHAPE),
        ({13: 9}, SHAPE), ({14: -1}, SHAPE), ({17: 131}, SHAPE), ({18: -1}, SHAPE), ({15: P(4097)}, UNSUPPORTED)])
    #       k_new v_new dt S kv d    kl   vl  win step max fire state reps st size cap nc codes scales rows prompt
    base = [D16, D16, 1, 8, 8, 128, D16, D16, 64, 0, 16, None, D16, D16, D16, D16, 20, 10, D16, D16, 200, 100, None]
    _statuses(lib.louiskv_segment_output_boundary_q4, base, [
        ({0: None}, NULL), ({12: None}, NULL), ({13: None}, NULL), ({18: None}, NULL), ({2: -1}, DTYPE),
        ({5: 64}, UNSUPPORTED), ({4: 3}, SHAPE), ({8: 1}, SHAPE), ({10: 64}, SHAPE), ({9: -2}, SHAPE), ({17: 0}, SHAPE),
        ({17: 21}, SHAPE), ({20: 99}, SHAPE), ({21: -1}, SHAPE), ({20: 0}, SHAPE)])


def test_attention_refuses(lib):
    ws = lib.louiskv_sparse_decode_attn_rows_q4_workspace_size(8, 4, 128, 2048, 128)
    assert ws > 0 and lib.louiskv_sparse_decode_attn_rows_q4_workspace_size(4096, 4, 128, 2048, 128) == 0
    assert lib.louiskv_sparse_decode_attn_rows_q4_workspace_size(0, 4, 128, 2048, 128) == 0
    #       q  dt S kv g  d   scale codes scales rows sel n_sel budget kl vl win start n out odt lse ws bytes
    base = [D16, 1, 8, 8, 4, 128, 0.1, D16, D16, 4096, D16, D16, 2048, D16, D16, 128, 0, 128, D16, 1, None, D16, ws, None]
    table = [
        ({0: None}, NULL), ({7: None}, NULL), ({8: None}, NULL), ({10: None}, NULL), ({11: None}, NULL),
        ({13: None}, NULL), ({18: None}, NULL), ({1: 3}, DTYPE), ({19: 2}, DTYPE), ({5: 64}, UNSUPPORTED),
        ({4: 3}, UNSUPPORTED), ({4: 16}, UNSUPPORTED), ({3: 3}, SHAPE), ({9: 0}, SHAPE), ({9: 1 << 25}, SHAPE),
        ({12: -1}, SHAPE), ({17: 129}, SHAPE), ({16: 128}, SHAPE), ({21: None}, WORKSPACE), ({22: ws - 1}, WORKSPACE)]
    _statuses(lib.louiskv_sparse_decode_attn_rows_q4, base, table)
    seg = base[:16] + [D16, 5] + base[18:]
    _statuses(lib.louiskv_sparse_decode_attn_rows_q4_seg, seg, [
        ({16: None}, NULL), ({13: None}, NULL), ({14: None}, NULL), ({15: 1}, SHAPE), ({17: 0}, SHAPE),
        ({22: ws - 1}, WORKSPACE)])


def test_block_calls_refuse(lib):
    cap = lib.louiskv_retrieve_blocks_cap
    assert cap(32768, 64, 64, 1, 4, 24) == 1 + 4 + 24 + 2
    assert cap(100, 64, 64, 1, 4, 24) == 2 and cap(4096, 1, 16, 0, 0, 0) == 1
    assert cap(0, 64, 64, 1, 4, 24) == cap(100, 129, 64, 1, 4, 24) == cap(100, 64, 48, 1, 4, 24) == 0
    assert cap(100, 64, 64, -1, 4, 24) == cap(100, 0, 64, 1, 4, 24) == 0
    big = (1 << 31) - 1
    assert cap(big, 128, 16, big, big, big) == -(-big // 16)
    #       q  dt S kv g nq  d  reps cap keys start tile block first recent top sel cap n_sel
    base = [D16, 1, 8, 8, 4, 500, 128, D16, 32, 2000, 1500, 64, 64, 1, 2, 4, D16, 9, D16, None]
    _statuses(lib.louiskv_retrieve_blocks, base, [
        ({0: None}, NULL), ({7: None}, NULL), ({16: None}, NULL), ({18: None}, NULL), ({1: 2}, DTYPE),
        ({6: 64}, UNSUPPORTED), ({4: 9}, UNSUPPORTED), ({4: 0}, UNSUPPORTED), ({11: 0}, UNSUPPORTED),
        ({11: 129}, UNSUPPORTED), ({12: 48}, UNSUPPORTED), ({3: 5}, SHAPE), ({5: 0}, SHAPE), ({9: 0}, SHAPE),
        ({10: -1}, SHAPE), ({10: 1501}, SHAPE), ({8: 31}, SHAPE), ({17: 8}, SHAPE), ({13: -1}, SHAPE), ({14: -1}, SHAPE),
        ({15: -1}, SHAPE), ({9: 200000, 12: 16, 8: 20000, 17: 100}, SHAPE)])
    #       q  dt S kv g nq  d  scale k v rows keys start tile block sel cap n_sel out odt lse ws bytes
    base = [D16, 1, 8, 8, 4, 500, 128, 0.1, D16, D16, 2000, 2000, 1500, 64, 64, D16, 9, D16, D16, 1, None, None, 0, None]
    _statuses(lib.louiskv_sparse_prefill_attn, base, [
        ({0: None}, NULL), ({8: None}, NULL), ({9: None}, NULL), ({15: None}, NULL), ({17: None}, NULL),
        ({18: None}, NULL), ({1: 2}, DTYPE), ({19: 2}, DTYPE), ({6: 64}, UNSUPPORTED), ({4: 3}, UNSUPPORTED),
        ({13: 0}, UNSUPPORTED), ({14: 512}, UNSUPPORTED), ({3: 5}, SHAPE), ({10: 1999}, SHAPE), ({16: 0}, SHAPE),
        ({12: 1501}, SHAPE)])


def test_python_calls_check_shapes():
    from paper_2510_11292_amd import louiskv as L
    k = torch.zeros(2, 10, 128)
    with pytest.raises(ValueError, match="4-bit pool"):
        L.pack_pool_q4(k, k, None, torch.zeros(2, 10, 64, dtype=torch.uint8), torch.zeros(2, 10, 8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="4-bit pool"):
        L.gather_rows_q4(torch.zeros(2, 10, 128, dtype=torch.uint8), torch.zeros(2, 9, 8, dtype=torch.uint8), None, None, k, k)
    q = torch.zeros(1, 4, 100, 128)
    sel, n = torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="lists"):
        L.retrieve_blocks(q, 2, torch.zeros(2, 8, 128), 100, 0, 64, 16, 0, 0, 1, sel, n)
    with pytest.raises(ValueError, match="lists"):
        L.sparse_prefill_attn(q, 2, k, k, 100, 0, 64, 16, sel, n, q)
    good = torch.zeros(2, 2, 4, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="lists"):
        L.sparse_prefill_attn(q, 2, k, k, 10, 0, 64, 16, good[0].long(), good[1], q)
    with pytest.raises(ValueError, match="expected"):
        L.sparse_prefill_attn(q, 2, k, k[:1], 10, 0, 64, 16, *good, q)
    with pytest.raises(TypeError, match="differ in dtype"):
        L.sparse_prefill_attn(q, 2, k, k.bfloat16(), 10, 0, 64, 16, *good, q)
    with pytest.raises(TypeError, match="differ in dtype"):
        L.pack_pool_q4(k, k.bfloat16(), None, torch.zeros(2, 10, 128, dtype=torch.uint8),
                       torch.zeros(2, 10, 8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="contiguous"):
        c = torch.zeros(2, 10, 256, dtype=torch.uint8)[..., :128]
        L.pack_pool_q4(k, k, None, c, torch.zeros(2, 10, 8, dtype=torch.uint8))


def test_unaligned_buffers_and_sizes_behind_the_index_range_are_refused(lib):
    odd, ws = P(4104), 1 << 20
    base = [D16, D16, 1, 2, 64, 128, None, D16, D16, 64, None]
    _statuses(lib.louiskv_pack_pool_q4, base, [({0: odd}, UNSUPPORTED), ({1: odd}, UNSUPPORTED)])
    base = [D16, D16, 2, 64, 128, None, None, 64, D16, D16, 1, None]
    _statuses(lib.louiskv_gather_rows_q4, base, [({8: odd}, UNSUPPORTED), ({9: odd}, UNSUPPORTED)])
    base = [D16, D16, 1, 8, 128, D16, D16, 64, 64, 32, D16, D16, D16, 10, 9, D16, D16, 132, 100, None]
    _statuses(lib.louiskv_segment_output_q4, base,
              [({i: odd}, UNSUPPORTED) for i in (0, 1, 5, 6)] + [({3: 1 << 23}, SHAPE)])
    base = [D16, D16, 1, 8, 8, 128, D16, D16, 64, 0, 16, None, D16, D16, D16, D16, 20, 10, D16, D16, 200, 100, None]
    _statuses(lib.louiskv_segment_output_boundary_q4, base,
              [({i: odd}, UNSUPPORTED) for i in (0, 1, 6, 7)] + [({3: 1 << 23}, SHAPE)])
    base = [D16, 1, 8, 8, 4, 128, 0.1, D16, D16, 4096, D16, D16, 2048, D16, D16, 128, 0, 128, D16, 1, None, D16, ws, None]
    _statuses(lib.louiskv_sparse_decode_attn_rows_q4, base,
              [({i: odd}, UNSUPPORTED) for i in (0, 13, 14)] + [({21: odd}, WORKSPACE), ({3: 1 << 23}, SHAPE),
                                                                ({12: 1 << 25}, SHAPE), ({15: (1 << 31) - 1}, SHAPE)])
    base = [D16, 1, 8, 8, 4, 500, 128, D16, 32, 2000, 1500, 64, 64, 1, 2, 4, D16, 9, D16, None]
    _statuses(lib.louiskv_retrieve_blocks, base, [
        ({0: odd}, UNSUPPORTED), ({7: odd}, UNSUPPORTED), ({9: (1 << 30) + 1}, SHAPE), ({2: 1 << 20}, SHAPE)])
    size = lib.louiskv_sparse_prefill_attn_workspace_size(8, 4, 64, 128, 64, 64, 9)
    assert size > 0
    base = [D16, 1, 8, 8, 4, 64, 128, 0.1, D16, D16, 2000, 2000, 1500, 64, 64, D16, 9, D16, D16, 1, None, D16, size, None]
    _statuses(lib.louiskv_sparse_prefill_attn, base, [({i: odd}, UNSUPPORTED) for i in (0, 8, 9, 18)] + [
        ({21: odd}, WORKSPACE), ({22: size - 1}, WORKSPACE), ({16: (1 << 24) + 1}, SHAPE),
        ({10: 1 << 31, 11: (1 << 30) + 1}, SHAPE), ({2: 1 << 23}, SHAPE)])


def test_workspace_sizes_of_what_the_calls_refuse_are_zero(lib):
    size, big = lib.louiskv_sparse_prefill_attn_workspace_size, (1 << 31) - 1
    assert size(8, 8, 64, 128, 64, 64, 9) > 0 and size(8, 8, 64, 128, 64, 64, big) > 0
    assert size(8, big, 64, 128, 64, 64, 9) == size(1 << 62, 4, 64, 128, 64, 64, 9) == size(8, 4, 64, 128, 129, 64, 9) == 0
    size = lib.louiskv_sparse_decode_attn_rows_q4_workspace_size
    assert size(8, 8, 128, big, 128) > 0 and size(8, big, 128, 64, 128) == size(1 << 62, 4, 128, 64, 128) == 0


def test_python_calls_refuse_sizes_types_and_host_memory():
    from paper_2510_11292_amd import louiskv as L
    i32, u8 = dict(dtype=torch.int32), dict(dtype=torch.uint8)
    k, loc = torch.zeros(2, 10, 128), torch.zeros(2, 4, 128)
    pool = torch.zeros(2, 10, 128, **u8), torch.zeros(2, 10, 8, **u8)
    perm, sel, n_sel = torch.zeros(2, 10, **i32), torch.zeros(2, 5, **i32), torch.zeros(2, **i32)
    q, out, ws = torch.zeros(1, 4, 128), torch.zeros(1, 4, 128), torch.zeros(1 << 20, **u8)
    new, reps, table = torch.zeros(2, 128), torch.zeros(2, 6, 128), torch.zeros(2, 6, **i32)

    def pack(values=k, perm=perm):
        L.pack_pool_q4(k, values, perm, *pool, stream=0)

    def gather(sel=perm, n=n_sel, v=k):
        L.gather_rows_q4(*pool, sel, n, k, v, stream=0)

    def store(v_new=new, v_local=loc, start=table):
        L.segment_output_q4(new, v_new, loc, v_local, 0, 2, reps, start, table, 3, *pool, stream=0)

    def bound(state=torch.zeros(2, 12, **i32), size=table):
        L.segment_output_boundary_q4(new, new, loc, loc, 0, 2, None, state, reps, table, size, 3, 2, stream=0)

    def attn(q=q, out=out, lse=None, sel=sel, n=n_sel, loc=loc):
        L.sparse_decode_attn_rows_q4(q, 2, *pool, sel, n, loc, loc, 0, 4, out, lse, workspace=ws, stream=0)

    def seg(out=out, n=n_sel):
        L.sparse_decode_attn_rows_q4_seg(q, 2, *pool, sel, n, loc, loc, torch.zeros(2, 12, **i32), 3, out, workspace=ws,
                                         stream=0)
    qp, lists = torch.zeros(1, 4, 7, 128), (torch.zeros(2, 1, 3, **i32), torch.zeros(2, 1, **i32))

    def blocks(q=qp, reps=reps):
        L.retrieve_blocks(q, 2, reps, 10, 3, 16, 16, 1, 1, 1, *lists, stream=0)

    def prompt(q=qp, values=k, out=qp, lse=None):
        L.sparse_prefill_attn(q, 2, k, values, 10, 3, 16, 16, *lists, out, lse, workspace=ws, stream=0)
    for call, kw in ((pack, dict(values=k[:, :9])), (pack, dict(perm=perm[:1])), (gather, dict(sel=perm[:, :9])),
                     (gather, dict(n=n_sel[:1])), (gather, dict(v=k[:, :9])), (store, dict(v_new=new[:1])),
                     (store, dict(v_local=loc[:, :3])), (store, dict(start=table[:, :5])), (bound, dict(size=table[:1])),
                     (attn, dict(out=out[:, :3])), (attn, dict(lse=out[..., 0][:, :3])), (attn, dict(sel=sel[:1])),
                     (attn, dict(n=n_sel[:1])), (attn, dict(loc=loc[:1])), (seg, dict(n=n_sel[:1])),
                     (blocks, dict(reps=reps[:1])), (prompt, dict(values=k[:, :9])), (prompt, dict(out=qp[:, :3])),
                     (prompt, dict(lse=qp[..., :3, 0]))):
        with pytest.raises(ValueError, match="expected"):
            call(**kw)
    for call, kw in ((pack, dict(perm=perm.long())), (gather, dict(sel=perm.long())), (gather, dict(n=n_sel.float())),
                     (store, dict(start=table.long())), (bound, dict(state=torch.zeros(2, 12))),
                     (attn, dict(sel=sel.long())), (seg, dict(n=n_sel.long()))):
        with pytest.raises(TypeError, match="int32"):
            call(**kw)
    for call in (attn, blocks, prompt):
        with pytest.raises(ValueError, match="multiple"):
            call(**({"q": q[:, :3], "out": out[:, :3]} if call is attn else {"q": qp[:, :3].contiguous()}
                    | ({"out": qp[:, :3]} if call is prompt else {})))
    for call in (pack, gather, store, bound, attn, seg, blocks, prompt):   # every size is right: host memory is what is left
        with pytest.raises(ValueError, match="current device"):
            call()


def test_boundary_store_checks_the_groups_decisions():
    """fire holds a byte for each group: fewer would be read past their end, wider numbers as the wrong bytes."""
    from paper_2510_11292_amd import louiskv as L
    i32, u8 = dict(dtype=torch.int32), dict(dtype=torch.uint8)
    new, loc, reps, table = torch.zeros(6, 128), torch.zeros(6, 4, 128), torch.zeros(6, 6, 128), torch.zeros(6, 6, **i32)

    def store(fire):
        L.segment_output_boundary_q4(new, new, loc, loc, 0, 2, fire, torch.zeros(6, 12, **i32), reps, table, table, 3, 2,
                                     stream=0)
    for n in (0, 2, 4, 6):
        with pytest.raises(ValueError, match="fire.*expected"):
            store(torch.zeros(n, **u8))
    with pytest.raises(ValueError, match="fire.*expected"):
        store(torch.zeros(3, 1, **u8))
    for dtype in (torch.int32, torch.float32, torch.int8):
        with pytest.raises(TypeError, match="fire.*uint8"):
            store(torch.zeros(3, dtype=dtype))
    for fire in (None, torch.zeros(3, **u8), torch.zeros(3, dtype=torch.bool)):   # host memory is what is left to refuse
        with pytest.raises(ValueError, match="current device"):
            store(fire)


def test_engine_refuses_what_a_4_bit_pool_is_not_built_for():
    from paper_2510_11292_amd.engine import EngineConfig, LouisKVEngine
    cfg = EngineConfig(n_slices=2, n_kv_heads=2, n_q_heads=8, prompt_len=64, n_clusters=4, n_iters=1, gen_len=8,
                       seg_len=4, budget=16, window=8, tau=0.9)
    for kw in (dict(pool_bits=8), dict(pool_bits=4, pool_on_host=True), dict(pool_bits=4, zero_copy=False),
               dict(pool_bits=4, fused_step=True), dict(pool_bits=4, cache_rows=64), dict(pool_bits=4, prefill_chunk=1),
               dict(pool_bits=4, delta=True)):
        with pytest.raises(ValueError, match="4-bit pool|pool_bits"):
            LouisKVEngine(cfg, torch.bfloat16, "cpu", **kw)


def test_prompt_attention_refuses_its_sizes():
    from paper_2510_11292_amd.engine import EngineConfig, LouisKVEngine
    cfg = EngineConfig(n_slices=2, n_kv_heads=2, n_q_heads=8, prompt_len=64, n_clusters=4, n_iters=1, gen_len=8,
                       seg_len=4, budget=16, window=8, tau=0.9)
    eng = LouisKVEngine(cfg, torch.float32, "cpu")
    q, k = torch.zeros(1, 8, 64, 128), torch.zeros(2, 64, 128)
    for kw in (dict(block_len=0), dict(block_len=-64), dict(block_len=48), dict(q_block=0), dict(q_block=129),
               dict(n_first=-1), dict(n_recent=-1), dict(n_top=-1)):
        with pytest.raises(ValueError, match="block_len="):
            eng.prompt_attention(q, k, k, **kw)
    with pytest.raises(ValueError, match="block_len="):
        eng.prompt_attention(q, k[:, :0], k[:, :0])


def test_numbers_that_an_argument_cannot_hold_are_refused():
    """Cut to 32 bits, a token count of 2^32 + 100 would be one of 100."""
    from paper_2510_11292_amd import louiskv as L
    big = 1 << 32
    assert L.retrieve_blocks_cap((1 << 31) - 1, 64, 64, 1, 4, 24) == 31
    for args in ((big + 100, 64, 64, 1, 4, 24), (100, 64, big + 64, 1, 4, 24), (100, 64, 64, 1, 4, 1 << 31),
                 (-big + 100, 64, 64, 1, 4, 24)):
        with pytest.raises(OverflowError, match="32-bit"):
            L.retrieve_blocks_cap(*args)
    q, k = torch.zeros(1, 4, 7, 128), torch.zeros(2, 10, 128)
    lists = torch.zeros(2, 1, 3, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(OverflowError, match="32-bit"):
        L.sparse_prefill_attn(q, 2, k, k, big + 10, 3, 16, 16, *lists, q, workspace=k, stream=0)
    with pytest.raises(OverflowError, match="32-bit"):
        L.sparse_prefill_attn(q, 2, k, k, 10, big + 3, 16, 16, *lists, q, workspace=k, stream=0)
    assert L.sparse_decode_attn_rows_q4_workspace_size(big + 8, 4, 100, 10) == 0     # 64 bits there: more slices than fit
