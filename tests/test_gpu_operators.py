"""The operators of a step over drafted tokens against their plain forms in 64 bits (tests/operator_forms.py).

Tolerances, u = 2^-24 half a step of fp32, v = torch.finfo(bfloat16).eps / 2 = 2^-8 half a step of bf16:
  projections  2e-6 (32 u) of the sum of absolute products: products of bf16 are exact in fp32, the running sums of a few thousand terms stay far
               below that sum, and each addition is off by u of the running sum.  fp32 operands add u a product
  rotation     an angle in turns rounded to fp32 is off by 2^-26, 2 pi times that is 1.6 u; sine and cosine 2 u, three products and sums 3 u:
               8 u of (|a| + |b|) amplitude, and half a step of the output's type
  attention    a score is off by e = (head_dim / 8) u sum |q k| scale (partial sums of eight and more), its exponential by that and 2 u |score log2 e|, the
               sum and the result by twice that, with the weights of the second product in 16 bits or more (2^-16); and half a step of the output
  draws        equal wherever the decision in fp64 is further than 1e-9 of the mass from a border
"""
import math
import random

import numpy as np
import pytest
import torch

from tests import operator_forms as F

pytestmark = pytest.mark.gpu
torch.set_grad_enabled(False)
U32, HALF = 2.0 ** -24, {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, FP = torch.bfloat16, torch.float32


def _randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(dtype)


# ---- projections with an adapter per row ---------------------------------------------------------------------------------


def _lora_inputs(dtype, m, n, k, r, ads, seed=0, kind="mixed"):
    g = torch.Generator().manual_seed(seed)
    ids = {"mixed": lambda: torch.randint(-1, ads, (m,), generator=g), "none": lambda: torch.full((m,), -1), "one": lambda: torch.full((m,), ads - 1),
           "out": lambda: torch.randint(-2 ** 31, 2 ** 31 - 1, (m,), generator=g), "runs": lambda: torch.arange(m) * ads // m}[kind]().int()
    return (_randn(g, (m, k), dtype), _randn(g, (n, k), dtype, 0.05), _randn(g, (ads, r, k), dtype, 0.1), _randn(g, (ads, n, r), dtype, 0.3), ids,
            torch.rand(ads, generator=g) * 4)


def _lora_check(args, accumulate=False, seed=1):
    import paper_2410_12513_amd as P
    A, W = args[:2]
    m, n = A.shape[0], W.shape[0]
    C0 = torch.randn((m, n), generator=torch.Generator().manual_seed(seed))
    C = C0.cuda() if accumulate else torch.full((m, n), float("nan"), device="cuda")
    P.op_gemm_nt_lora(*[t.cuda() for t in args], C, accumulate=accumulate)
    ref, size = F.lora(*args)
    if accumulate:
        ref, size = ref + C0.double(), size + C0.double().abs()
    err = (C.cpu().double() - ref).abs()
    assert bool((err <= 2e-6 * size + 1e-30).all()), float((err / size).max())
    return C


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m,n,k,r,ads", [(1, 1, 8, 1, 1), (1, 130, 4096, 8, 3), (2, 64, 72, 3, 2), (16, 512, 1032, 8, 16), (17, 257, 264, 16, 4), (33, 688, 256, 5, 7),
                                         (64, 100, 2056, 64, 2), (65, 333, 520, 33, 5), (129, 1000, 136, 17, 32), (250, 300, 1416, 12, 8), (300, 520, 2048, 64, 3)])
def test_lora_projection(dtype, m, n, k, r, ads):
    _lora_check(_lora_inputs(dtype, m, n, k, r, ads))
    _lora_check(_lora_inputs(dtype, m, n, k, r, ads, seed=3), accumulate=True)


@pytest.mark.parametrize("m", [5, 40, 200, 700])
@pytest.mark.parametrize("kind", ["none", "one", "out", "runs"])
def test_lora_adapters_of_rows(m, kind):
    _lora_check(_lora_inputs(BF, m, 260, 512, 8, 6, seed=m, kind=kind))


def test_lora_of_long_prompts():
    _lora_check(_lora_inputs(BF, 1030, 1300, 1160, 8, 4, kind="runs"))
    _lora_check(_lora_inputs(BF, 2049, 520, 264, 24, 32))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m,n,k,r,ads", [(100, 130, 4096, 7, 3), (130, 600, 2056, 24, 5), (64, 3000, 128, 40, 2), (40, 64, 8, 64, 1)])
def test_lora_slices_of_the_contraction(dtype, m, n, k, r, ads):
    """Few tiles and a long contraction: slices of it, added in order (and what is cut into slices without need)."""
    _lora_check(_lora_inputs(dtype, m, n, k, r, ads, seed=4))
    _lora_check(_lora_inputs(dtype, m, n, k, r, ads, seed=5, kind="runs"), accumulate=True)


@pytest.mark.parametrize("kind,r", [("runs", 8), ("mixed", 19)])
def test_lora_large_tiles(kind, r):
    _lora_check(_lora_inputs(BF, 4000, 4001, 136, r, 6, seed=6, kind=kind), accumulate=kind == "runs")


def test_lora_last_ranks_of_the_last_adapter():
    """Ranks that fill no chunk, at the very end of Lb: the array ends a page, nothing behind it may be read into the result."""
    import paper_2410_12513_amd as P
    for r in (1, 3, 9, 13):
        for m in (4, 50, 300):
            A, W, La, Lb, ids, scale = _lora_inputs(BF, m, 70, 64, r, 2, seed=r, kind="one")
            big = torch.full((Lb.numel() + 64,), float("nan"), dtype=BF, device="cuda")
            big[:Lb.numel()] = Lb.cuda().flatten()
            C = torch.empty((m, 70), device="cuda")
            P.op_gemm_nt_lora(A.cuda(), W.cuda(), La.cuda(), big[:Lb.numel()].view(Lb.shape), ids.cuda(), scale.cuda(), C)
            ref, size = F.lora(A, W, La, Lb, ids, scale)
            assert bool(((C.cpu().double() - ref).abs() <= 2e-6 * size).all())


def test_lora_rows_do_not_depend_on_their_neighbours_adapters():
    """Infinities in an adapter stay with its own rows, and no adapter reads a row that is not its."""
    import paper_2410_12513_amd as P
    for m in (7, 90, 300):
        A, W, La, Lb, ids, scale = _lora_inputs(BF, m, 200, 256, 8, 3, seed=m)
        plain = torch.empty((m, 200), device="cuda")
        P.op_gemm_nt_lora(*[t.cuda() for t in (A, W, La, Lb, ids, scale)], plain)
        La[1], Lb[1, ::2] = float("inf"), float("nan")
        C = torch.empty((m, 200), device="cuda")
        P.op_gemm_nt_lora(*[t.cuda() for t in (A, W, La, Lb, ids, scale)], C)
        mine = ids == 1
        assert torch.equal(C.cpu()[~mine], plain.cpu()[~mine])
        assert not bool(torch.isfinite(C.cpu()[mine]).all())


@pytest.mark.parametrize("m", [7, 60, 90, 300])
def test_lora_first_products_at_the_end_of_the_range(m):
    """T between the largest bf16 number and the largest fp32 one is finite; T beyond is an infinity, of its sign in every column."""
    import paper_2410_12513_amd as P
    A, W, La, Lb = torch.zeros((m, 64), dtype=BF), torch.ones((130, 64), dtype=BF), torch.zeros((2, 5, 64), dtype=BF), torch.ones((2, 130, 5), dtype=BF)
    A[:, :2] = 1
    La[:, 0, 0], La[0, 0, 1], La[1, 0, 1] = torch.finfo(BF).max, 2.0 ** 119, 2.0 ** 127
    Lb *= 2.0 ** -20
    Lb[:, ::3] *= -1
    ids = (torch.arange(m) % 2).int()
    C = torch.empty((m, 130), device="cuda")
    P.op_gemm_nt_lora(*[t.cuda() for t in (A, W, La, Lb, ids, torch.ones(2))], C)
    ref, size = F.lora(A, W, La, Lb, ids, torch.ones(2))
    assert float(F.lora(A, W, La, Lb.sign(), ids, torch.ones(2))[0].abs().max()) > torch.finfo(FP).max
    C = C.cpu().double()
    assert bool(((C - ref).abs() <= 2e-6 * size)[ids == 0].all())
    assert torch.equal(C[ids == 1], (ref.sign() * float("inf"))[ids == 1])


def test_lora_merged_weights_give_the_same(dtype=FP):
    """One task for all rows: what first_lora_merge puts into the matrix."""
    import paper_2410_12513_amd as P
    A, W, La, Lb, ids, scale = _lora_inputs(dtype, 40, 96, 128, 8, 1, kind="one")
    C, M = torch.empty((40, 96), device="cuda"), torch.empty((40, 96), device="cuda")
    P.op_gemm_nt_lora(*[t.cuda() for t in (A, W, La, Lb, ids, scale)], C)
    Wm = W.cuda()
    P.lora_merge(Wm, La[0].cuda(), Lb[0].cuda(), float(scale[0]))
    P.op_gemm_nt(A.cuda(), Wm, M)
    _, size = F.lora(A, W, La, Lb, ids, scale)
    assert bool(((C - M).abs().cpu().double() <= 4e-6 * size).all())


# ---- rotary positions ----------------------------------------------------------------------------------------------------


def _rope_check(dtype, rows, heads, hd, rot, layout, scaling="none", packed=None, inplace=False, inverse=False, amplitude=1.0, base=10000.0, positions=None, seed=0):
    import paper_2410_12513_amd as P
    g = torch.Generator().manual_seed(seed)
    packed = packed or heads
    buf = _randn(g, (rows, packed, hd), dtype)
    pos = torch.randint(0, 200000, (rows,), generator=g).int() if positions is None else positions
    kw = dict(factor=8.0, low=1.0, high=4.0, original_len=8192)
    dev = buf.cuda()
    x = dev[:, packed - heads:]
    y = x if inplace else torch.full((rows, heads, hd), float("nan"), dtype=dtype, device="cuda")
    P.op_rope(x, pos.cuda(), y, rot_dim=rot, layout=layout, base=base, scaling=scaling, inverse=inverse, amplitude=amplitude, **kw)
    ref = F.rope(buf[:, packed - heads:], pos, rot, layout, F.rope_frequencies(rot, base, scaling, **kw), amplitude, inverse)
    i = torch.arange(rot // 2)
    ia, ib = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + rot // 2)
    s = buf[:, packed - heads:].double().abs()
    both = s[..., ia] + s[..., ib]                       # |a| + |b| of a pair
    mag = torch.zeros_like(s)
    mag[..., ia], mag[..., ib] = both, both
    err = (y.cpu().double() - ref).abs()
    assert bool((err <= 8 * U32 * abs(amplitude) * mag + HALF[dtype] * ref.abs()).all()), float(err.max())
    if rot < hd:
        assert torch.equal(y.cpu()[..., rot:], buf[:, packed - heads:, rot:])        # passed through, bit for bit
    if packed > heads:
        assert torch.equal(dev.cpu()[:, :packed - heads], buf[:, :packed - heads])   # the neighbours stay as they were


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,hd,rot", [(1, 1, 2, 2), (1, 40, 128, 128), (3, 5, 64, 64), (70, 7, 128, 64), (33, 3, 64, 22), (9, 2, 256, 256), (5, 3, 66, 6),
                                               (257, 16, 128, 32), (4, 2, 80, 80), (2, 3, 7, 4)])
def test_rope(dtype, layout, rows, heads, hd, rot):
    _rope_check(dtype, rows, heads, hd, rot, layout)
    _rope_check(dtype, rows, heads, hd, rot, layout, packed=heads + 1, inplace=True, seed=1)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("scaling", ["none", "linear", "bands"])
def test_rope_scalings_and_the_way_back(dtype, scaling):
    _rope_check(dtype, 65, 4, 128, 128, "half", scaling, base=500000.0)
    _rope_check(dtype, 65, 4, 128, 96, "interleaved", scaling, inverse=True, amplitude=1.25, packed=6)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_of_long_prompts(dtype, layout):
    _rope_check(dtype, 8195, 2, 64, 48, layout, packed=3, inplace=True)


def test_rope_positions_of_any_size():
    edge = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1048577, 123456789], dtype=torch.int32)
    _rope_check(FP, 7, 2, 64, 64, "half", positions=edge)


def test_rope_gradient_against_the_formula_and_differences():
    """<dy, R x> has the gradient R^T dy: what the inverse turn gives, and what differences of the inner product along random directions give."""
    import paper_2410_12513_amd as P
    g = torch.Generator().manual_seed(5)
    x, dy, d = (_randn(g, (11, 3, 64), FP) for _ in range(3))
    pos = torch.randint(0, 5000, (11,), generator=g).int().cuda()
    kw = dict(rot_dim=48, layout="interleaved", scaling="bands", factor=4.0, amplitude=1.5)
    def turn(t, inverse=False):
        y = torch.empty_like(t, device="cuda")
        P.op_rope(t.cuda(), pos, y, inverse=inverse, **kw)
        return y.cpu().double()
    grad = turn(dy, inverse=True)
    ref = F.rope(dy, pos.cpu(), 48, "interleaved", F.rope_frequencies(48, 10000.0, "bands", 4.0), 1.5, True)
    assert float((grad - ref).abs().max()) <= 1.5 * 16 * U32 * 4
    step = 0.5                                              # linear: a large step loses nothing
    diff = ((turn(x + step * d) - turn(x - step * d)) * dy.double()).sum() / (2 * step)
    assert abs(float(diff - (grad * d.double()).sum())) <= 1e-3


# ---- attention of drafted tokens -----------------------------------------------------------------------------------------


def _tree_inputs(dtype, lens, nodes, hq, hkv, hd, seed=0, masks="tree", spare=2, max_pages=None, qstd=1.5):
    g = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    N, most = sum(nodes), max(max(nodes), 1)
    pages = [-(-x // 16) for x in lens]
    n_pages, width = sum(pages) + spare, max(1, max(pages)) if max_pages is None else max_pages
    pool = _randn(g, (n_pages, 2, hkv, 16, hd), dtype)
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = torch.full((len(lens), width), 2 ** 30, dtype=torch.int32), 0       # unused entries: no page
    for b, c in enumerate(pages):
        for i in range(c):
            table[b, i] = order[at + i]
        for p in range(lens[b], 16 * c):                  # slots past the end hold what was there before
            pool[order[at + c - 1], :, :, p % 16] = float("nan") if p % 2 else float("inf")
        at += c
    words = -(-most // 64)
    rows = []
    for c in nodes:
        seen = []
        for i in range(c):
            parent = rng.randint(max(-1, i - 3), i - 1)
            seen.append({"tree": (seen[parent] if parent >= 0 else 0) | 1 << i, "none": 0, "all": (1 << c) - 1, "some": rng.getrandbits(c) if rng.random() < 0.7 else 0}[masks]
                        if masks != "chain" else 0)
        rows += [[(s >> 64 * w & (1 << 64) - 1) - ((s >> 64 * w + 63 & 1) << 64) for w in range(words)] for s in seen]
    offs = [0]
    for c in nodes:
        offs.append(offs[-1] + c)
    return dict(q=_randn(g, (N, hq, hd), dtype, qstd), k=_randn(g, (N, hkv, hd), dtype), v=_randn(g, (N, hkv, hd), dtype), pool=pool, table=table,
                lens=torch.tensor(lens, dtype=torch.int32), offs=torch.tensor(offs, dtype=torch.int32),
                mask=None if masks == "chain" else torch.tensor(rows, dtype=torch.int64).reshape(N, words))


def _tree_run(t, max_nodes=None, max_len=None, scale=None, stream=None, workspace=None):
    import paper_2410_12513_amd as P
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    nodes = [int(b - a) for a, b in zip(t["offs"][:-1], t["offs"][1:])]
    out, lse = torch.full_like(d["q"], 7.0), torch.full(d["q"].shape[:2], 7.0, device="cuda")
    P.op_tree_attn(d["q"], d["k"], d["v"], d["pool"], d["table"], d["lens"], d["offs"], out, max(nodes) if max_nodes is None else max_nodes,
                   int(t["lens"].max()) if max_len is None else max_len, mask=d["mask"], scale=scale, lse=lse, stream=stream, workspace=workspace)
    return out, lse


def _tree_compare(t, out, lse, scale=None, **kw):
    q = t["q"]
    hd, scale = q.shape[2], q.shape[2] ** -0.5 if scale is None else scale
    ref, rlse, mag, size = F.tree_attention(q, t["k"], t["v"], t["pool"], t["table"], t["lens"], t["offs"], t["mask"], scale, **kw)
    out, lse = out.cpu().double(), lse.cpu().double()
    done = ~torch.isnan(rlse)
    assert bool((out[~done] == 7.0).all()) and bool((lse[~done] == 7.0).all())       # rows of nobody stay as they were
    empty = done & (rlse == -math.inf)
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    e = (hd / 8) * U32 * size + 4 * U32 * (size + 1)
    full = done & ~empty
    err = (out - ref).abs()[full]
    assert bool((err <= (HALF[q.dtype] * ref.abs() + (2 * e[..., None] + 2.0 ** -16 + 8 * U32) * mag)[full]).all()), float(err.max())
    lerr = (lse - rlse).abs()[full]
    assert bool((lerr <= (2 * e + 8 * U32 + 2 * U32 * rlse.abs())[full]).all()), float(lerr.max())


HEADS = [(32, 8, 128), (4, 4, 64), (5, 1, 64), (16, 2, 128), (3, 3, 128)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("lens,nodes", [([40], [1]), ([0], [1]), ([1], [3]), ([15, 16, 17, 0], [2, 1, 4, 3]), ([129, 64, 300], [9, 0, 17]), ([63, 0, 1, 260], [33, 5, 8, 1])])
def test_tree_attention(dtype, hq, hkv, hd, lens, nodes):
    t = _tree_inputs(dtype, lens, nodes, hq, hkv, hd, seed=sum(lens) + hq)
    _tree_compare(t, *_tree_run(t))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("masks", ["chain", "none", "all", "some"])
@pytest.mark.parametrize("lens,nodes", [([0, 20], [5, 70]), ([31, 0, 0], [64, 65, 130])])
def test_tree_masks(dtype, masks, lens, nodes):
    t = _tree_inputs(dtype, lens, nodes, 4, 2, 64, seed=len(masks), masks=masks)
    _tree_compare(t, *_tree_run(t))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
def test_tree_attention_over_long_caches(dtype, hd):
    t = _tree_inputs(dtype, [5000, 1, 2300], [2, 3, 1], 2, 1, hd, seed=9)
    _tree_compare(t, *_tree_run(t))
    t = _tree_inputs(dtype, [9001], [3], 8, 2, hd, seed=10, qstd=4.0)
    _tree_compare(t, *_tree_run(t))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("batch", [2, 64, 65])
@pytest.mark.parametrize("hq,hkv,hd", [(5, 1, 64), (6, 2, 128)])
def test_tree_sequences_of_very_different_lengths(dtype, batch, hq, hkv, hd):
    rng = random.Random(batch)
    lens, nodes = [rng.choice([0, 1, 17, 130, 260]) for _ in range(batch)], [rng.choice([0, 1, 1, 3, 14]) for _ in range(batch)]
    lens[batch // 2], lens[-1], nodes[batch // 2], nodes[-1] = 3333, 1500, 2, 40
    for kw in ({}, {"max_len": 2000, "max_nodes": 9}):
        t = _tree_inputs(dtype, lens, nodes, hq, hkv, hd, seed=batch)
        _tree_compare(t, *_tree_run(t, **kw), **kw)


def test_tree_more_splits_of_the_largest_size_than_places():
    """Two sequences whose splits of 8192 keys are more than the chip takes at once; all of their pages are the same few."""
    t = _tree_inputs(BF, [0, 0], [1, 2], 32, 32, 64, seed=8)
    g = torch.Generator().manual_seed(8)
    t["pool"], t["table"], t["lens"] = _randn(g, (64, 2, 32, 16, 64), BF), torch.randint(0, 64, (2, 4375), generator=g).int(), torch.tensor([70000, 69003], dtype=torch.int32)
    _tree_compare(t, *_tree_run(t))


def test_tree_splits_of_the_largest_size():
    """So many heads that a sequence is cut into splits of the largest size only; the others are short."""
    t = _tree_inputs(BF, [8300, 0, 3, 17, 5, 1, 40, 16], [1, 1, 2, 1, 0, 1, 1, 1], 64, 64, 64, seed=12)
    _tree_compare(t, *_tree_run(t))


def test_tree_pages_far_into_a_large_cache():
    """Pages whose elements lie past 2^31."""
    import paper_2410_12513_amd as P
    t = _tree_inputs(BF, [100, 33], [5, 2], 32, 8, 128, seed=14)
    n, per = t["pool"].shape[0], t["pool"][0].numel()
    far = 2 ** 31 // per + 9
    big = torch.empty((far + n, *t["pool"].shape[1:]), dtype=BF, device="cuda")
    big[far:] = t["pool"].cuda()
    d = {k: v.cuda() for k, v in t.items() if k != "pool"}
    table = torch.where(d["table"] < n, d["table"] + far, d["table"])
    out, lse = torch.full_like(d["q"], 7.0), torch.full(d["q"].shape[:2], 7.0, device="cuda")
    P.op_tree_attn(d["q"], d["k"], d["v"], big, table, d["lens"], d["offs"], out, 5, 100, mask=d["mask"], lse=lse)
    _tree_compare(t, out, lse)


def test_tree_sequences_that_share_pages():
    t = _tree_inputs(BF, [64, 64, 50], [3, 2, 4], 8, 2, 64, seed=15)
    t["table"][1] = t["table"][0]
    t["table"][2, :3] = t["table"][0, 0]
    t["pool"] = torch.nan_to_num(t["pool"].float(), 0, 0, 0).to(BF)
    _tree_compare(t, *_tree_run(t))


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_tree_scales(scale):
    for dtype in (BF, FP):
        t = _tree_inputs(dtype, [40, 9], [3, 6], 4, 2, 64, seed=16, masks="some")
        _tree_compare(t, *_tree_run(t, scale=scale), scale=scale)


def test_tree_masks_of_infinite_scores():
    """Keys of the largest values: scores beyond 32 bits of some nodes are infinite, and only their own rows feel it."""
    t = _tree_inputs(FP, [20], [6], 2, 1, 64, seed=17)
    t["k"][2] = 3e38
    t["mask"][:, 0] &= ~(1 << 2)
    out, lse = _tree_run(t)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    _tree_compare({**t, "k": t["k"].clamp(max=3.0)}, out, lse)


def test_tree_bounds_shorter_than_the_sequences():
    """max_len, max_nodes and the page table's width cut what the device's numbers say; rows past max_nodes stay as they were."""
    t = _tree_inputs(BF, [100, 40], [9, 4], 4, 2, 64, seed=3)
    _tree_compare(t, *_tree_run(t, max_nodes=5, max_len=33), max_nodes=5, max_len=33)
    t["lens"] = torch.tensor([10 ** 9, -5], dtype=torch.int32)
    t["table"] = t["table"][:, :4].contiguous()
    _tree_compare(t, *_tree_run(t, max_len=2 ** 20), max_len=2 ** 20)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_tree_pages_that_do_not_exist_are_not_seen(dtype):
    t = _tree_inputs(dtype, [100, 90, 30], [3, 2, 2], 4, 2, 128, seed=4)
    t["table"][0, 2], t["table"][0, 5], t["table"][1, 0], t["table"][2, 0], t["table"][2, 1] = -1, 2 ** 31 - 1, t["pool"].shape[0], -7, -2 ** 31
    _tree_compare(t, *_tree_run(t))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_tree_unseen_nodes_may_hold_anything(dtype):
    t = _tree_inputs(dtype, [50, 7], [40, 6], 4, 2, 64, seed=6, masks="tree")
    bad = [3, 17, 41]
    for j in bad:                                          # nobody but itself and its children see a node: cut it out of all masks
        o0, b = (0, j) if j < 40 else (40, j - 40)
        rows = slice(0, 40) if j < 40 else slice(40, 46)
        t["mask"][rows, 0] &= ~(1 << b)
        t["k"][j], t["v"][j] = float("nan"), float("inf") if j % 2 else float("nan")
    out, lse = _tree_run(t)
    clean = {**t, "k": torch.nan_to_num(t["k"], 0, 0, 0), "v": torch.nan_to_num(t["v"], 0, 0, 0)}
    _tree_compare(clean, out, lse)


def test_tree_without_a_cache():
    import paper_2410_12513_amd as P
    t = _tree_inputs(BF, [0], [6], 4, 2, 64)
    d = {k: v.cuda() for k, v in t.items()}
    out, lse = torch.full_like(d["q"], 7.0), torch.full(d["q"].shape[:2], 7.0, device="cuda")
    P.op_tree_attn(d["q"], d["k"], d["v"], None, None, d["lens"], d["offs"], out, 6, 0, mask=d["mask"], lse=lse)
    _tree_compare(t, out, lse)


@pytest.mark.parametrize("model", ["mini_bf16", "tiny"])
def test_tree_attention_over_the_cache_of_a_context(model):
    """The pages, tables and lengths of live sequences, in a shuffled page order, before and after decode steps."""
    import paper_2410_12513_amd as P
    from synth import CONFIGS, make_prompt, make_router, make_weights
    from synth.generators import to_device
    desc = CONFIGS[model]
    dtype, hq, hkv, hd = (BF if desc.dtype == "bf16" else FP), desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    ctx = P.FirstContext(desc, to_device(make_weights(desc, 5), "cuda"), make_router(desc, 5).cuda(), max_batch=3, max_seq_len=96)
    with pytest.raises(P.FirstError) as e:                   # no live sequence
        one = torch.zeros(1, hq, hd, dtype=dtype, device="cuda")
        ctx.tree_attn(0, one, torch.zeros(1, hkv, hd, dtype=dtype, device="cuda"), torch.zeros(1, hkv, hd, dtype=dtype, device="cuda"),
                      torch.zeros(1, dtype=torch.int32, device="cuda"), one.clone(), 1)
    assert e.value.code == -2
    order = list(range(ctx.num_pages()))
    random.Random(3).shuffle(order)
    ctx.set_page_order(order)
    lens = [40, 16, 1]
    ctx.prefill_route(torch.cat([make_prompt(desc.vocab, n, 60 + n) for n in lens]).cuda(), lens)
    for b in range(3):
        ctx.set_mask(b, [1] * desc.n_layers)
    t = _tree_inputs(dtype, [0, 0, 0], [5, 1, 3], hq, hkv, hd, seed=18)
    d = {k: t[k].cuda() for k in ("q", "k", "v", "offs", "mask")}
    tok = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    for step in range(3):
        layer = desc.n_layers - 1 if step else 0
        out, lse = torch.full_like(d["q"], 7.0), torch.full(d["q"].shape[:2], 7.0, device="cuda")
        ctx.tree_attn(layer, d["q"], d["k"], d["v"], d["offs"], out, 5, mask=d["mask"], lse=lse)
        ctx.sync()
        now = [ctx.seq_len(b) for b in range(3)]
        assert now == [n + step for n in lens]
        pages = [-(-n // 16) for n in now]
        pool, table, at = torch.zeros((sum(pages), 2, hkv, 16, hd), dtype=dtype), torch.zeros((3, max(pages)), dtype=torch.int32), 0
        for b, n in enumerate(now):
            k, v = ctx.kv_read(b, layer, 0, n)
            for p in range(n):
                pool[at + p // 16, 0, :, p % 16], pool[at + p // 16, 1, :, p % 16] = k[p].cpu().to(dtype), v[p].cpu().to(dtype)
            table[b, :pages[b]] = torch.arange(at, at + pages[b])
            at += pages[b]
        _tree_compare({**t, "pool": pool, "table": table, "lens": torch.tensor(now)}, out, lse)
        ctx.decode_step(tok, None, tok.clone())
    with pytest.raises(P.FirstError) as e:
        ctx.tree_attn(desc.n_layers, d["q"], d["k"], d["v"], d["offs"], out, 5)
    assert e.value.code == -1
    ctx.close()


# ---- draws ---------------------------------------------------------------------------------------------------------------


def _sample_check(logits, u, least=0.95, **rules):
    """rules: temperature, top_k, top_p, min_p, a number or a list per row."""
    import paper_2410_12513_amd as P
    logits = np.asarray(logits, dtype=np.float32)
    rows = logits.shape[0]
    per = {k: np.broadcast_to(np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32), (rows,)).copy() for k, v in rules.items()}
    u = np.broadcast_to(np.asarray(u, dtype=np.float32), (rows,)).copy()
    tok, lp, kept = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    P.sample(torch.from_numpy(logits).cuda(), torch.from_numpy(u).cuda(), tok, logprob=lp, kept=kept, **{k: torch.from_numpy(v).cuda() for k, v in per.items()})
    tok, lp, kept, sure = tok.cpu(), lp.cpu(), kept.cpu(), 0
    for b in range(rows):
        want, wlp, n, margin = F.sample(logits[b], float(u[b]), **{k: (int if k == "top_k" else float)(v[b]) for k, v in per.items()})
        if margin <= 1e-9:
            continue
        sure += 1
        assert (int(tok[b]), int(kept[b])) == (want, n), (b, {k: v[b] for k, v in per.items()})
        assert float(lp[b]) == wlp if math.isinf(wlp) else abs(float(lp[b]) - wlp) <= 1e-6 * max(1.0, abs(wlp))
    assert sure >= least * rows
    return tok, lp, kept


def _logits(rows, vocab, seed=0, std=2.0):
    rng = np.random.default_rng(seed)
    l = rng.normal(size=(rows, vocab)).astype(np.float32) * np.float32(std)
    l[np.arange(rows), rng.integers(0, vocab, rows)] += 8.0
    return l


@pytest.mark.parametrize("vocab", [1, 2, 37, 1000, 1024, 4099, 32000, 128256])
@pytest.mark.parametrize("rules", [{}, {"temperature": 0.7}, {"top_k": 10}, {"top_p": 0.9}, {"min_p": 0.05}, {"temperature": 1.3, "top_k": 40, "top_p": 0.95, "min_p": 0.02},
                                   {"temperature": 5.0, "top_p": 0.99}])
def test_sample(vocab, rules):
    rng = np.random.default_rng(vocab)
    _sample_check(_logits(9, vocab, vocab), rng.random(9), **rules)


@pytest.mark.parametrize("vocab", [600, 5000, 32000, 128256])
@pytest.mark.parametrize("rules", [{"top_p": 0.95, "min_p": 0.01}, {"top_p": 0.3, "min_p": 1e-4}, {"top_k": 2000}, {"top_k": 500, "top_p": 0.9}, {"top_k": 100, "min_p": 1e-3},
                                   {"top_p": 0.999999}, {"min_p": 1e-20}, {"temperature": 0.05}, {"temperature": 0.05, "top_p": 0.99}, {"temperature": 1e4, "top_p": 0.5},
                                   {"min_p": 1.0}, {"min_p": 0.999}])
def test_sample_cuts(vocab, rules):
    rng = np.random.default_rng(vocab + 1)
    _sample_check(_logits(5, vocab, vocab + 1, 1.0), rng.random(5), least=0.6, **rules)


@pytest.mark.parametrize("rules", [{}, {"top_p": 0.6}, {"min_p": 0.5}, {"top_k": 700, "top_p": 0.8}])
def test_sample_crowded_logits(rules):
    """Logits so near each other that parts of the range hold thousands, and one far away that stretches it."""
    rng = np.random.default_rng(21)
    l = (rng.normal(size=(6, 60000)) * 1e-3).astype(np.float32)
    l[1, 7], l[2, 59999] = 30.0, 5.0
    l[3] *= 50
    l[4, ::2] = -1e30
    l[5] = l[5].astype(np.float16).astype(np.float32)
    _sample_check(l, rng.random(6), least=0.6, **rules)


def test_sample_many_rows_and_a_large_vocabulary():
    rng = np.random.default_rng(22)
    _sample_check(_logits(300, 700, 23), rng.random(300), temperature=0.9, top_p=0.9)
    _sample_check(_logits(2, 1000003, 24), rng.random(2), temperature=0.9, top_p=0.9)
    _sample_check(_logits(2, 1000003, 25), rng.random(2), top_k=50)


def test_sample_rules_of_rows():
    rng = np.random.default_rng(2)
    n = 64
    _sample_check(_logits(n, 5000, 4, 1.0), rng.random(n), temperature=rng.uniform(0.1, 2, n), top_k=rng.integers(-3, 6000, n), top_p=rng.uniform(-0.1, 1.1, n),
                  min_p=rng.uniform(-0.1, 0.3, n))


@pytest.mark.parametrize("vocab", [50, 5000, 70000])
def test_sample_equal_logits_go_by_index(vocab):
    rng = np.random.default_rng(vocab)
    flat = np.zeros((8, vocab), np.float32)
    flat[1], flat[2, ::3], flat[3] = -1e30, 1.0, np.round(rng.normal(size=vocab))
    flat[4, ::2] = -0.0
    _sample_check(flat, rng.random(8), 0.6)
    _sample_check(flat, rng.random(8), 0.6, top_k=vocab // 3)
    _sample_check(flat, rng.random(8), 0.6, top_p=0.37)
    _sample_check(flat, rng.random(8), 0.6, top_k=[1, 2, 3, 7, vocab - 1, vocab, vocab + 1, 5], min_p=0.4, temperature=0.5)


def test_sample_masked_logits():
    inf, nan = math.inf, math.nan
    rng = np.random.default_rng(8)
    l = _logits(10, 3001, 5)
    l[0], l[1] = -inf, nan
    l[2, :], l[2, 77] = -inf, -3.0
    l[3, ::2] = nan
    l[4, 1::2] = -inf
    l[5, [9, 700, 3000]] = inf
    l[6] = np.float32(-3.4028235e38)
    l[7, 100:] = np.float32(-3.4028235e38)
    l[8, ::5] = np.float32(3.4028235e38)
    l[9, :2999] = -1e30
    for rules in ({}, {"top_k": 4}, {"top_p": 0.8}, {"min_p": 0.5}, {"temperature": 0.0}, {"temperature": nan}, {"temperature": 1e-30, "top_p": 0.9},
                  {"temperature": 1e30, "top_p": 0.5}, {"top_p": 0.0}, {"top_p": nan, "min_p": nan, "top_k": 0}, {"min_p": 2.0}, {"top_k": 2 ** 31 - 1}, {"top_k": -2 ** 31}):
        _sample_check(l, rng.random(10), 0.5, **rules)


@pytest.mark.parametrize("vocab", [5000, 40001])
@pytest.mark.parametrize("fourths", [[0], [1], [2, 3], [0, 1, 2]])
def test_sample_rows_whose_fourths_differ(vocab, fourths):
    """Grammars that mask by index: every fourth token at the top, masked, far below, or no number."""
    rng = np.random.default_rng(vocab + fourths[0])
    l = _logits(6, vocab, 21)
    for f in fourths:
        for b, v in enumerate((l[0].max(), -math.inf, math.nan, -3.4028235e38, -1e4)):
            l[b, f::4] = np.float32(v)
    for rules in ({}, {"top_k": 7}, {"top_p": 0.7}, {"min_p": 0.02, "top_p": 0.97}, {"temperature": 40.0, "top_p": 0.9}, {"temperature": 1e20, "min_p": 0.1}, {"temperature": 0.01}):
        _sample_check(l, rng.random(6), 0.5, **rules)


def test_sample_uniforms_at_the_ends():
    l = _logits(6, 900, 11)
    edge = [0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, 1e-30]
    _sample_check(l, edge, 0.6, top_p=0.9)
    import paper_2410_12513_amd as P
    tok = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    P.sample(torch.from_numpy(l[:1]).cuda(), torch.tensor([math.nan], device="cuda"), tok)
    assert 0 <= int(tok[0]) < 900


def test_sample_of_strided_rows_leaves_the_rest():
    import paper_2410_12513_amd as P
    l = _logits(7, 1200, 12)
    for first in (0, 1, 3):
        view = torch.from_numpy(l).cuda()[:, first:1100]
        tok = torch.empty(7, dtype=torch.int32, device="cuda")
        u = torch.linspace(0.05, 0.93, 7)
        P.sample(view, u.cuda(), tok, top_k=torch.full((7,), 20, dtype=torch.int32, device="cuda"))
        for b in range(7):
            want, _, _, margin = F.sample(l[b, first:1100], float(u[b]), top_k=20)
            assert margin <= 1e-9 or int(tok[b]) == want


def test_sample_agrees_with_the_top_k_draw():
    """top_k and one temperature alone: the rule of first_sample_top_k_static, which sums in fp32."""
    import paper_2410_12513_amd as P
    l = _logits(16, 32000, 13)
    u = torch.rand(16, generator=torch.Generator().manual_seed(3))
    a, b = (torch.empty(16, dtype=torch.int32, device="cuda") for _ in range(2))
    P.sample_top_k_static(torch.from_numpy(l).cuda(), u.cuda(), 0.8, 10, a)
    P.sample(torch.from_numpy(l).cuda(), u.cuda(), b, temperature=torch.full((16,), 0.8, device="cuda"), top_k=torch.full((16,), 10, dtype=torch.int32, device="cuda"))
    for i in range(16):
        if F.sample(l[i], float(u[i]), temperature=float(np.float32(0.8)), top_k=10)[3] > 1e-5:
            assert int(a[i]) == int(b[i])


# ---- together, captured, on other streams --------------------------------------------------------------------------------


def _step(seed, lens, nodes, ads=3):
    """The calls of one layer's attention block and the draw, over drafted tokens of requests with adapters of their own: outputs and a replayable call."""
    import paper_2410_12513_amd as P
    hq, hkv, hd, D, V, r = 8, 2, 64, 256, 1500, 8
    g = torch.Generator().manual_seed(seed)
    t = _tree_inputs(BF, lens, nodes, hq, hkv, hd, seed=seed)
    N, heads = sum(nodes), hq + 2 * hkv
    x = _randn(g, (N, D), BF)
    w = {"qkv": _randn(g, (heads * hd, D), BF, D ** -0.5), "o": _randn(g, (D, hq * hd), BF, (hq * hd) ** -0.5), "head": _randn(g, (V, D), BF, 0.2)}
    la = {"qkv": (_randn(g, (ads, r, D), BF, D ** -0.5), _randn(g, (ads, heads * hd, r), BF, 0.3)), "o": (_randn(g, (ads, r, hq * hd), BF, 0.05), _randn(g, (ads, D, r), BF, 0.3))}
    owner = torch.repeat_interleave(torch.arange(len(nodes)), torch.tensor(nodes))
    adapter = (owner % (ads + 1) - 1).int()
    depth = torch.tensor([bin(int(m[0]) & (1 << 64) - 1).count("1") - 1 for m in t["mask"]])
    pos = (t["lens"].long()[owner] + depth).int()
    scale = torch.rand(ads, generator=g) + 0.5
    u, p = torch.rand(N, generator=g), torch.full((N,), 0.9)
    dev = {k: v.cuda() for k, v in dict(x=x, adapter=adapter, pos=pos, scale=scale, u=u, p=p, **{f"w_{k}": v for k, v in w.items()},
                                        **{f"a_{k}": v[0] for k, v in la.items()}, **{f"b_{k}": v[1] for k, v in la.items()}).items()}
    td = {k: v.cuda() for k, v in t.items()}
    o = dict(qkv=torch.zeros((N, heads * hd), device="cuda"), h=torch.zeros((N, heads, hd), dtype=BF, device="cuda"), att=torch.zeros((N, hq, hd), dtype=BF, device="cuda"),
             y=torch.zeros((N, D), device="cuda"), yb=torch.zeros((N, D), dtype=BF, device="cuda"), logits=torch.zeros((N, V), device="cuda"),
             token=torch.zeros(N, dtype=torch.int32, device="cuda"), lp=torch.zeros(N, device="cuda"))
    q, k, v = (torch.zeros((N, c, hd), dtype=BF, device="cuda") for c in (hq, hkv, hkv))
    ws = {n: torch.empty(max(1, s), dtype=torch.uint8, device="cuda") for n, s in (
        ("l", P.op_gemm_nt_lora_workspace(dev["x"], dev["w_qkv"], dev["a_qkv"])), ("o", P.op_gemm_nt_lora_workspace(o["att"].view(N, -1), dev["w_o"], dev["a_o"])),
        ("t", P.op_tree_attn_workspace(td["q"], td["k"], max(nodes), max(lens), len(lens))), ("s", P.sample_workspace(o["logits"])))}
    o["y0"] = torch.randn((N, D), generator=g).cuda()

    def call():
        P.op_gemm_nt_lora(dev["x"], dev["w_qkv"], dev["a_qkv"], dev["b_qkv"], dev["adapter"], dev["scale"], o["qkv"], workspace=ws["l"])
        o["h"].copy_(o["qkv"].view(N, heads, hd))
        P.op_rope(o["h"][:, :hq + hkv], dev["pos"], o["h"][:, :hq + hkv], base=500000.0, scaling="bands", factor=8.0)
        q.copy_(o["h"][:, :hq]); k.copy_(o["h"][:, hq:hq + hkv]); v.copy_(o["h"][:, hq + hkv:])
        P.op_tree_attn(q, k, v, td["pool"], td["table"], td["lens"], td["offs"], o["att"], max(nodes), max(lens), mask=td["mask"], workspace=ws["t"])
        o["y"].copy_(o["y0"])
        P.op_gemm_nt_lora(o["att"].view(N, -1), dev["w_o"], dev["a_o"], dev["b_o"], dev["adapter"], dev["scale"], o["y"], accumulate=True, workspace=ws["o"])
        o["yb"].copy_(o["y"])
        P.op_gemm_nt(o["yb"], dev["w_head"], o["logits"], stream=torch.cuda.current_stream())
        P.sample(o["logits"], dev["u"], o["token"], top_p=dev["p"], logprob=o["lp"], workspace=ws["s"])
    return call, o, dict(x=x, w=w, la=la, adapter=adapter, pos=pos, scale=scale, u=u, t=t, hq=hq, hkv=hkv, hd=hd, q=q, k=k, v=v)


def test_a_step_of_them_together():
    call, o, s = _step(1, [70, 0, 33], [7, 3, 12])
    call()
    torch.cuda.synchronize()
    hq, hkv, hd = s["hq"], s["hkv"], s["hd"]
    qkv, size = F.lora(s["x"], s["w"]["qkv"], *s["la"]["qkv"], s["adapter"], s["scale"])
    assert bool(((o["qkv"].cpu().double() - qkv).abs() <= 2e-6 * size).all())
    h = o["qkv"].cpu().to(BF).view(-1, hq + 2 * hkv, hd)
    turned = F.rope(h[:, :hq + hkv], s["pos"], hd, "half", F.rope_frequencies(hd, 500000.0, "bands", 8.0))
    assert bool(((o["h"].cpu()[:, :hq + hkv].double() - turned).abs() <= HALF[BF] * turned.abs() + 16 * U32 * h.double().abs().max()).all())
    t = {**s["t"], "q": s["q"].cpu(), "k": s["k"].cpu(), "v": s["v"].cpu()}
    lse = torch.full(t["q"].shape[:2], 0.0)
    ref, rlse, mag, size = F.tree_attention(t["q"], t["k"], t["v"], t["pool"], t["table"], t["lens"], t["offs"], t["mask"], hd ** -0.5)
    assert bool(((o["att"].cpu().double() - ref).abs() <= HALF[BF] * ref.abs() + (1e-4 + 2e-5 * size[..., None]) * mag).all())
    y, size = F.lora(o["att"].cpu().view(-1, hq * hd), s["w"]["o"], *s["la"]["o"], s["adapter"], s["scale"])
    assert bool(((o["y"].cpu().double() - y - o["y0"].cpu().double()).abs() <= 2e-6 * (size + 4)).all())
    for i in range(o["token"].shape[0]):
        want, _, _, margin = F.sample(o["logits"][i].cpu().numpy(), float(s["u"][i]), top_p=float(np.float32(0.9)))
        assert margin <= 1e-9 or int(o["token"][i]) == want


def test_captured_steps_side_by_side():
    """Two captured steps with workspaces of their own, replayed on two streams again and again, between eager calls: every replay is the eager result."""
    steps = [_step(2, [70, 0, 33], [7, 3, 12]), _step(3, [300, 5], [1, 30])]
    want, graphs, streams = [], [], [torch.cuda.Stream() for _ in steps]
    for call, o, _ in steps:
        call()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in o.items()})
    for (call, o, _), st in zip(steps, streams):
        st.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            call()
        graphs.append(g)
    for _ in range(4):
        for (_, o, _), w in zip(steps, want):
            for key in ("qkv", "h", "att", "y", "logits", "token", "lp"):
                o[key].zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for (call, o, _), w in zip(steps, want):
            for key in w:
                assert torch.equal(o[key], w[key]), key
        steps[0][0]()                                       # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(steps[0][1][k], want[0][k]) for k in want[0])


def test_calls_follow_the_current_stream():
    call, o, _ = _step(4, [40], [9])
    call()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in o.items()}
    for key in ("qkv", "att", "token"):
        o[key].zero_()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    assert all(torch.equal(o[k], want[k]) for k in want)


def test_results_are_the_same_bits_every_time():
    for _ in range(2):
        a, b = _step(5, [500, 20], [16, 40]), _step(5, [500, 20], [16, 40])
        a[0](); b[0]()
        torch.cuda.synchronize()
        assert all(torch.equal(a[1][k], b[1][k]) for k in a[1])


def test_workspaces_of_another_stream():
    """Memory that the current stream has given back and still writes is no workspace for a call on another one."""
    import paper_2410_12513_amd as P
    args = [t.cuda() for t in _lora_inputs(BF, 8, 600, 512, 8, 3, seed=9)]
    plain, C, side = torch.empty((8, 600), device="cuda"), torch.empty((8, 600), device="cuda"), torch.cuda.Stream()
    need = P.op_gemm_nt_lora_workspace(args[0], args[1], args[2])
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    P.op_gemm_nt_lora(*args, plain, workspace=ws)
    torch.cuda.synchronize()
    for _ in range(300):
        ws.fill_(255)
    at = ws.data_ptr()
    del ws
    from paper_2410_12513_amd import binding
    assert binding._scratch(need, 0, side).data_ptr() != at
    P.op_gemm_nt_lora(*args, C, stream=side)
    side.synchronize()
    assert torch.equal(C, plain)
