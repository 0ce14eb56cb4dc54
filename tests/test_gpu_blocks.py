"""The prompt's block selection and block-sparse attention on the GPU against the
float64 oracle."""
import numpy as np
import pytest
import torch

from attn_bounds import check_attention
from oracle import blocks as ob

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


def L():
    from paper_2510_11292_amd import louiskv
    return louiskv


def n64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def page_reps(keys, block):
    s, n, d = keys.shape
    nb = -(-n // block)
    reps = torch.zeros(s, nb, d, device=keys.device)
    st = torch.zeros(s, nb, dtype=torch.int32, device=keys.device)
    L().page_prefill(keys, block, reps, st, torch.zeros_like(st))
    return reps


SELECT = [  # groups, kv, g, n_q, n_k, tile, block, first, recent, top
    (1, 1, 1, 1, 1, 1, 16, 0, 0, 1), (1, 2, 4, 1, 5000, 1, 16, 1, 2, 30), (2, 2, 4, 300, 300, 64, 64, 1, 1, 1),
    (1, 2, 8, 77, 3001, 7, 16, 0, 0, 5), (1, 1, 2, 513, 4097, 128, 32, 2, 3, 20), (1, 3, 3, 130, 2000, 100, 128, 0, 4, 2),
    (1, 1, 4, 257, 2570, 16, 16, 5, 0, 0), (1, 1, 1, 40, 131072, 64, 16, 1, 1, 64), (1, 2, 4, 700, 700, 33, 256, 0, 0, 9),
    (1, 1, 4, 64, 90000, 64, 16, 0, 0, 3000),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SELECT, ids=[f"{c[3]}of{c[4]}t{c[5]}b{c[6]}" for c in SELECT])
def test_selection(dtype, case):
    groups, kv, g, n_q, n_k, tile, block, first, recent, top = case
    l, s = L(), groups * kv
    gen = torch.Generator(device=DEV).manual_seed(n_k + tile)
    q = torch.randn(groups, kv * g, n_q, 128, generator=gen, device=DEV).to(DT[dtype])
    nb = -(-n_k // block)
    reps = torch.randn(s, nb + 3, 128, generator=gen, device=DEV)
    if nb > 12:
        reps[:, 3:11:2] = reps[:, 4:5]      # equal scores: the lower block goes first
        reps[0, 6] = float("nan")           # and a NaN comes last
        reps[0, 8] = 0.0
    tiles, cap = -(-n_q // tile), l.retrieve_blocks_cap(n_k, tile, block, first, recent, top)
    sel = torch.full((s, tiles, cap + 2), -9, dtype=torch.int32, device=DEV)
    n = torch.full((s, tiles), -9, dtype=torch.int32, device=DEV)
    l.retrieve_blocks(q, kv, reps, n_k, n_k - n_q, tile, block, first, recent, top, sel, n)
    sel, n = sel.cpu().numpy(), n.cpu().numpy()
    qn, rn = n64(q).reshape(s, g, n_q, 128), n64(reps)
    for i in range(s):
        for t in range(tiles):
            a, b = t * tile, min((t + 1) * tile, n_q)
            p0 = n_k - n_q + a
            want = ob.tile_blocks(qn[i, :, a:b].reshape(-1, 128), rn[i], p0, n_k - n_q + b - 1, block, first, recent, top)
            assert list(sel[i, t, :n[i, t]]) == want, (i, t)
            assert (sel[i, t, n[i, t]:] == -9).all() and len(want) <= cap


ATTN = [  # groups, kv, g, n_q, n_k, tile, block, cap
    (1, 1, 1, 1, 1, 1, 16, 1), (1, 2, 4, 1, 3000, 1, 16, 40), (1, 1, 8, 5, 700, 2, 64, 6), (2, 2, 4, 200, 200, 64, 64, 4),
    (1, 2, 2, 77, 777, 7, 16, 9), (1, 1, 4, 300, 1111, 128, 32, 12), (1, 1, 8, 130, 500, 100, 128, 4),
    (1, 2, 4, 33, 2048, 16, 256, 3), (1, 1, 4, 150, 4000, 64, 64, 31), (1, 1, 2, 250, 1000, 128, 16, 20),
    (1, 3, 1, 65, 640, 33, 16, 17), (1, 1, 8, 260, 600, 128, 64, 7), (1, 1, 1, 140, 900, 128, 32, 6),
]


def lists_for(rng, s, n_q, n_k, tile, block, cap, wild):
    tiles, nb = -(-n_q // tile), -(-n_k // block)
    sel = np.full((s, tiles, cap), 1 << 30, dtype=np.int32)
    n = np.zeros((s, tiles), dtype=np.int32)
    for i in range(s):
        for t in range(tiles):
            hi = (n_k - n_q + min((t + 1) * tile, n_q) - 1) // block
            k = min(cap, hi + 1)
            pick = rng.permutation(hi + 1)[:k]
            if wild and k > 1 and rng.random() < 0.5:
                pick[-1] = pick[0]                       # a block listed twice counts twice
            if wild and rng.random() < 0.3:
                pick[0] = rng.choice([-5, nb, nb + 7, nb - 1])   # clamped; a block behind every query weighs nothing
            n[i, t] = 0 if wild and rng.random() < 0.15 else k
            sel[i, t, :k] = pick
    return sel, n


def run_attn(q, kv, keys, values, n_k, tile, block, sel, n, odt, **kw):
    out = torch.full(q.shape, 7.0, dtype=odt, device=DEV)
    lse = torch.full(q.shape[:3], 7.0, device=DEV)
    L().sparse_prefill_attn(q, kv, keys, values, n_k, n_k - q.shape[2], tile, block, torch.from_numpy(sel).to(DEV),
                            torch.from_numpy(n).to(DEV), out, lse, **kw)
    return out, lse


def check_against_oracle(q, kv, keys, values, n_k, tile, block, sel, n, out, lse, bf16_in):
    groups, hq, n_q, _ = q.shape
    s, g, nb = groups * kv, hq // kv, -(-n_k // block)
    qn, kn, vn = n64(q).reshape(s, g, n_q, 128), n64(keys), n64(values)
    on, ln = n64(out).reshape(s, g, n_q, 128), n64(lse).reshape(s, g, n_q)
    worst = 0.0
    for i in range(s):
        for t in range(sel.shape[1]):
            a, b = t * tile, min((t + 1) * tile, n_q)
            blocks = np.clip(sel[i, t, :n[i, t]], 0, nb - 1)
            key = (blocks[:, None] * block + np.arange(block)).reshape(-1)
            key = key[key < n_k]
            see = key[None] <= n_k - n_q + np.arange(a, b)[:, None]
            for j in range(g):
                want = ob.masked_attention(qn[i, j, a:b], kn[i, key], vn[i, key], see, 128 ** -0.5)
                worst = max(worst, check_attention(on[i, j, a:b], ln[i, j, a:b], want, bf16_in,
                                                   out.dtype == torch.bfloat16, len(key)))
    return worst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ATTN, ids=[f"{c[2]}x{c[3]}of{c[4]}t{c[5]}b{c[6]}" for c in ATTN])
def test_attention(dtype, case):
    groups, kv, g, n_q, n_k, tile, block, cap = case
    s, dt = groups * kv, DT[dtype]
    rng = np.random.default_rng(n_q + tile)
    gen = torch.Generator(device=DEV).manual_seed(n_k)
    q = (2 * torch.randn(groups, kv * g, n_q, 128, generator=gen, device=DEV)).to(dt)
    keys, values = (torch.randn(s, n_k + 5, 128, generator=gen, device=DEV).to(dt) for _ in range(2))
    keys[:, n_k:], values[:, n_k:] = float("nan"), float("nan")     # rows behind the last key
    for wild in (False, True):
        sel, n = lists_for(rng, s, n_q, n_k, tile, block, cap, wild)
        for odt in {dt, torch.float32}:
            out, lse = run_attn(q, kv, keys, values, n_k, tile, block, sel, n, odt)
            worst = check_against_oracle(q, kv, keys, values, n_k, tile, block, sel, n, out, lse, dtype == "bf16")
            print(f"{case} {dtype} -> {odt}, wild {wild}: largest error {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile,block,g", [(16, 64, 4), (64, 64, 4), (1, 16, 2), (128, 32, 8), (5, 128, 1)])
def test_later_keys_do_not_reach_a_query(dtype, tile, block, g):
    """Keys and values behind a query may be NaN or infinite: its result does not change by a bit."""
    dt, n = DT[dtype], 200
    gen = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(1, g, n, 128, generator=gen, device=DEV).to(dt)
    keys, values = (torch.randn(1, n, 128, generator=gen, device=DEV).to(dt) for _ in range(2))
    nb, tiles = -(-n // block), -(-n // tile)
    sel = np.tile(np.arange(nb, dtype=np.int32), (1, tiles, 1))
    cnt = np.full((1, tiles), nb, dtype=np.int32)
    ref, ref_lse = run_attn(q, 1, keys, values, n, tile, block, sel, cnt, torch.float32)
    assert not torch.isnan(ref).any()
    for at, bad in ((60, float("nan")), (111, float("inf")), (130, -float("inf"))):
        for which in ("k", "v", "kv"):
            k2, v2 = keys.clone(), values.clone()
            if "k" in which:
                k2[:, at:, ::3] = bad
            if "v" in which:
                v2[:, at:at + 40, 5:90] = bad
            out, lse = run_attn(q, 1, k2, v2, n, tile, block, sel, cnt, torch.float32)
            assert torch.equal(out[:, :, :at], ref[:, :, :at]), (at, bad, which)
            assert torch.equal(lse[:, :, :at], ref_lse[:, :, :at])
            if which == "v":        # the queries that see them get what the formula says, the other channels are whole
                assert not torch.isfinite(out[:, :, at:, 5:90]).any()
                assert torch.equal(out[..., 90:], ref[..., 90:]) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("bits", [0x7fc00000, 0x7fffffff, -1, 0x7f800001])
@pytest.mark.parametrize("n", [40, 600])     # whole lists, and lists in parts, whose merge rounds
def test_a_nan_of_any_bits_stays_one_in_a_bf16_output(bits, n):
    q, keys, values = torch.randn(1, 4, 40, 128, device=DEV), torch.randn(1, n, 128, device=DEV), torch.randn(1, n, 128, device=DEV)
    values.view(torch.int32)[0, 7, 5] = torch.tensor(bits, dtype=torch.int32)
    nb = -(-n // 16)
    out, _ = run_attn(q, 1, keys, values, n, 64, 16, np.arange(nb, dtype=np.int32).reshape(1, 1, nb),
                      np.full((1, 1), nb, dtype=np.int32), torch.bfloat16)
    want = torch.zeros(1, 4, 40, 128, dtype=torch.bool, device=DEV)
    want[..., max(0, 7 - (n - 40)):, 5] = True
    assert torch.equal(torch.isnan(out), want)


def test_scores_of_minus_infinity_weigh_nothing():
    q = torch.ones(1, 2, 40, 128, device=DEV).bfloat16()
    keys = torch.zeros(1, 40, 128, device=DEV).bfloat16()
    values = torch.arange(40, device=DEV).view(1, 40, 1).expand(1, 40, 128).contiguous().bfloat16()
    keys[:, :30] = -float("inf")
    sel, n = np.arange(3, dtype=np.int32).reshape(1, 1, 3), np.full((1, 1), 3, dtype=np.int32)
    out, lse = run_attn(q, 1, keys, values, 40, 64, 16, sel, n, torch.float32)
    assert (out[:, :, :30] == 0).all() and torch.isneginf(lse[:, :, :30]).all()
    for i in range(30, 40):
        assert torch.allclose(out[0, :, i], torch.full((2, 128), (30 + i) / 2, device=DEV), rtol=2.0 ** -8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_selection_attention_together(dtype):
    """page_prefill, retrieve_blocks and sparse_prefill_attn as a prompt uses them, in two chunks; with every block
    taken it is dense causal attention."""
    l, dt = L(), DT[dtype]
    kv, g, n, cut, tile, block = 2, 4, 900, 611, 32, 32
    gen = torch.Generator(device=DEV).manual_seed(7)
    q = torch.randn(1, kv * g, n, 128, generator=gen, device=DEV).to(dt)
    keys, values = (torch.randn(kv, n, 128, generator=gen, device=DEV).to(dt) for _ in range(2))
    for top in (3, 1000):
        for a, b in ((0, cut), (cut, n)):
            reps = page_reps(keys[:, :b].contiguous(), block)
            cap, tiles = l.retrieve_blocks_cap(b, tile, block, 1, 1, top), -(-(b - a) // tile)
            sel = torch.zeros(kv, tiles, cap, dtype=torch.int32, device=DEV)
            cnt = torch.zeros(kv, tiles, dtype=torch.int32, device=DEV)
            qc = q[:, :, a:b].contiguous()
            out, lse = torch.zeros(1, kv * g, b - a, 128, device=DEV), torch.zeros(1, kv * g, b - a, device=DEV)
            l.retrieve_blocks(qc, kv, reps, b, a, tile, block, 1, 1, top, sel, cnt)
            l.sparse_prefill_attn(qc, kv, keys, values, b, a, tile, block, sel, cnt, out, lse)
            check_against_oracle(qc, kv, keys, values, b, tile, block, sel.cpu().numpy(), cnt.cpu().numpy(), out, lse,
                                 dtype == "bf16")
            if top == 1000:
                x = q[0, :, a:b].double().view(kv, g, b - a, 128) @ keys[:, None, :b].double().transpose(2, 3).contiguous()
                x = x * 128 ** -0.5
                x.masked_fill_(torch.arange(b, device=DEV) > torch.arange(a, b, device=DEV)[:, None], -float("inf"))
                ref = (x.softmax(-1) @ values[:, None, :b].double()).view(1, kv * g, b - a, 128)
                tol = 2.0 ** -6 if dtype == "bf16" else 1e-5
                assert (out.double() - ref).abs().max() < tol * values.abs().max()


def test_replayed_graph_and_two_streams():
    l = L()
    kv, g, n_q, n_k, tile, block, top = 2, 4, 24, 3000, 8, 16, 40
    gen = torch.Generator(device=DEV).manual_seed(9)
    q = torch.randn(1, kv * g, n_q, 128, generator=gen, device=DEV).bfloat16()
    keys, values = (torch.randn(kv, n_k, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    reps = page_reps(keys, block)
    cap, tiles = l.retrieve_blocks_cap(n_k, tile, block, 1, 2, top), -(-n_q // tile)
    size = l.sparse_prefill_attn_workspace_size(kv, g, n_q, tile, block, cap)

    def state():
        return dict(q=q.clone(), sel=torch.zeros(kv, tiles, cap, dtype=torch.int32, device=DEV),
                    n=torch.zeros(kv, tiles, dtype=torch.int32, device=DEV), out=torch.zeros_like(q),
                    lse=torch.zeros(1, kv * g, n_q, device=DEV), ws=torch.empty(max(size, 1), dtype=torch.uint8, device=DEV))

    def one(x, stream=None):
        l.retrieve_blocks(x["q"], kv, reps, n_k, n_k - n_q, tile, block, 1, 2, top, x["sel"], x["n"], stream=stream)
        l.sparse_prefill_attn(x["q"], kv, keys, values, n_k, n_k - n_q, tile, block, x["sel"], x["n"], x["out"], x["lse"],
                              workspace=x["ws"], stream=stream)
    eager, cap_, other = state(), state(), state()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            one(cap_)
    for i in range(4):
        new = torch.randn(q.shape, generator=gen, device=DEV).bfloat16()
        for x in (eager, cap_, other):
            x["q"].copy_(new)
        torch.cuda.synchronize()
        one(eager)
        one(other, side)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("sel", "n", "out", "lse"):
            assert torch.equal(eager[n], cap_[n]) and torch.equal(eager[n], other[n]), (i, n)


MANY = [  # enough tiles for blocks of 256 and 128 rows; groups, kv, g, n_q, n_k, tile, block, cap
    (16, 8, 4, 130, 400, 64, 32, 9), (40, 4, 8, 70, 300, 33, 16, 8), (64, 2, 8, 40, 333, 16, 64, 5),
    (160, 1, 1, 200, 200, 128, 128, 2), (130, 1, 8, 130, 500, 128, 64, 7),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", MANY, ids=[f"{c[0] * c[1]}x{c[2]}x{c[3]}t{c[5]}b{c[6]}" for c in MANY])
def test_attention_of_many_tiles(dtype, case):
    groups, kv, g, n_q, n_k, tile, block, cap = case
    s, dt = groups * kv, DT[dtype]
    rng = np.random.default_rng(n_k)
    gen = torch.Generator(device=DEV).manual_seed(n_q)
    q = (2 * torch.randn(groups, kv * g, n_q, 128, generator=gen, device=DEV)).to(dt)
    keys, values = (torch.randn(s, n_k, 128, generator=gen, device=DEV).to(dt) for _ in range(2))
    sel, n = lists_for(rng, s, n_q, n_k, tile, block, cap, True)
    out, lse = run_attn(q, kv, keys, values, n_k, tile, block, sel, n, dt)
    for i in (0, groups // 2, groups - 1):
        a, b = slice(i, i + 1), slice(i * kv, (i + 1) * kv)
        worst = check_against_oracle(q[a], kv, keys[b], values[b], n_k, tile, block, sel[b], n[b], out[a], lse[a],
                                     dtype == "bf16")
        print(f"{case} {dtype}, group {i}: largest error {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile,g", [(64, 4), (128, 8), (32, 4)])
def test_later_keys_do_not_reach_a_query_of_many_tiles(dtype, tile, g):
    """As above where the blocks take more rows: 150 sequences, one of them with bad keys behind its queries."""
    dt, n, groups, block = DT[dtype], 200, 150, 32
    gen = torch.Generator(device=DEV).manual_seed(4)
    q = torch.randn(groups, g, n, 128, generator=gen, device=DEV).to(dt)
    keys, values = (torch.randn(groups, n, 128, generator=gen, device=DEV).to(dt) for _ in range(2))
    nb, tiles = -(-n // block), -(-n // tile)
    sel = np.tile(np.arange(nb, dtype=np.int32), (groups, tiles, 1))
    cnt = np.full((groups, tiles), nb, dtype=np.int32)
    ref, ref_lse = run_attn(q, 1, keys, values, n, tile, block, sel, cnt, torch.float32)
    assert not torch.isnan(ref).any()
    for at, bad in ((77, float("nan")), (130, -float("inf"))):
        k2, v2 = keys.clone(), values.clone()
        k2[70, at + 40:], v2[70, at:at + 40, 5:90] = bad, bad
        out, lse = run_attn(q, 1, k2, v2, n, tile, block, sel, cnt, torch.float32)
        assert torch.equal(out[70, :, :at], ref[70, :, :at]) and torch.equal(lse[70, :, :at], ref_lse[70, :, :at])
        assert not torch.isfinite(out[70, :, at:at + 40, 5:90]).any()
        assert torch.equal(out[70, :, :at + 40, 90:], ref[70, :, :at + 40, 90:])
        others = torch.arange(groups, device=DEV) != 70
        assert torch.equal(out[others], ref[others]) and torch.equal(lse[others], ref_lse[others])
