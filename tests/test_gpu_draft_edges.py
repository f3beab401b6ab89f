"""The drafted-token calls at their edges: values that are not finite and pages that are not there in every form of the tree
attention's work, sizes beyond one launch, arrays and streams other than the usual ones."""
import numpy as np
import pytest
import torch

import draft_util as D
from paper_2507_21276_amd import binding as Bd
from test_gpu_attn_tree import DT, Case, f64, i32

pytestmark = pytest.mark.gpu

# (nodes, heads, key heads): 8 and 24 rows of a key head are a wavefront's own, 50 are shared by two, 160 by four
ROWS = [(8, 1, 1), (24, 1, 1), (25, 2, 1), (40, 4, 1)]


@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("nodes,h,hk", ROWS)
@pytest.mark.parametrize("dtype,dh", [("f16", 64), ("bf16", 64), ("f16", 128), ("bf16", 128), ("bf16", 32), ("f32", 64), ("f16", 80)])
def test_an_infinite_value_of_the_context_reaches_every_row(dtype, dh, nodes, h, hk, value):
    """Cached tokens are seen by all rows: an infinity in one of their values is the result there, whatever its weight
    (e^-30: less than 16 bits hold beside 1), and the other dimensions do not notice."""
    for key, weight, scratch in ((0, 0.0, None), (333, -30.0, None), (640, 0.0, torch.empty(0, device="cuda"))):
        c = Case(21, [700], [nodes], h, hk, dh, 16, dtype)
        c.q.view(-1, dh)[:, 0] = 8.0
        page = c.bt[0]
        for j in range(700 + nodes):
            c.kp[page[j // 16], :, j % 16, 0] = weight * dh ** 0.5 / 8 if j == key else 0.0
        at = page[key // 16], slice(None), key % 16, dh - 3
        c.vp[at] = value
        o = c.run(scratch=scratch).view(nodes, h, dh)
        assert (o[..., dh - 3].float() == value).all()
        c.vp[at] = 0.0
        zero = c.run(scratch=scratch).view(nodes, h, dh)
        o[..., dh - 3] = zero[..., dh - 3]
        c.check(o.view(nodes, h * dh), set(range(0, nodes, 7)))


@pytest.mark.parametrize("nodes,h,hk", ROWS)
def test_infinities_of_both_signs_are_no_number(nodes, h, hk):
    for dtype in ("f16", "bf16", "f32"):
        c = Case(22, [300], [nodes], h, hk, 64, 16, dtype)
        c.vp[c.bt[0, 1], :, 3, 5], c.vp[c.bt[0, 9], :, 8, 5] = float("inf"), -float("inf")
        o = c.run().view(-1, 64).float()
        assert torch.isnan(o[:, 5]).all() and torch.isfinite(o[:, :5]).all() and torch.isfinite(o[:, 6:]).all()


@pytest.mark.parametrize("T,h,hk,dh", [((1 << 25) + 3, 1, 1, 2), ((1 << 28) + 5, 1, 1, 8)])
def test_rows_of_more_workgroups_than_one_grid_dimension_counts(T, h, hk, dh):
    """More than 2^32 work-items, in the kernel for any size and in the vectorised one: every row is written."""
    x = torch.empty(T, (h + 2 * hk) * dh, dtype=torch.float16, device="cuda").random_(-2048, 2049)
    y = torch.full_like(x, 7.0)
    Bd.lsk_qk_norm_rope(x, y, h, hk, dh, norm=False)
    assert torch.equal(x, y)
    # in place, with a norm: the rows at both ends, around the border of the first grid row, and none left as it was
    ends = torch.cat([torch.arange(9), torch.tensor([(1 << 24) - 1, 1 << 24, T // 2]), torch.arange(T - 9, T)]).cuda()
    want = torch.empty_like(x[ends])
    Bd.lsk_qk_norm_rope(x[ends].contiguous(), want, h, hk, dh)
    Bd.lsk_qk_norm_rope(x, x, h, hk, dh)
    assert torch.equal(x[ends], want)
    assert float(x[:, :2 * dh].max()) <= dh ** 0.5 * (1 + D.HALF["f16"])


def test_contexts_stay_whole_where_the_join_would_be_too_large_a_launch():
    """16384 requests of up to 256 nodes by 32 heads: a workgroup for each four (node, head) pairs of each is more than a launch
    counts."""
    B = 16384
    past, counts = [0] * (B - 1) + [6500], [1] * (B - 2) + [256, 3]
    c = Case(23, past, counts, 32, 1, 64, 16, "f16")
    assert Bd.lib().lsk_attn_tree_scratch_floats(c.T, B, 32, 1, 64, 256, 6500) > 0
    c.check(c.run(), {0, 5000, B - 3, B - 2, B + 100, c.T - 3, c.T - 1})


def test_scratch_of_another_stream_is_no_block_of_the_current_one():
    """A block that the current stream's work may still be using is not given to a call on another stream, and the call's own goes
    back to its stream."""
    n, t, side = 3 << 20, torch.empty(1, device="cuda"), torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        block = torch.empty(n, device="cuda")
        at = block.data_ptr()
        del block                                    # free for the current stream, on which work with it may be pending
        s = Bd._scratch(n, t, stream)
        assert s.data_ptr() != at and s.numel() == n and s.dtype is torch.float32
        mine = s.data_ptr()
        del s
        later = [torch.empty(n, device="cuda") for _ in range(3)]
        assert mine not in [x.data_ptr() for x in later]
        assert Bd._scratch(n, t, stream).data_ptr() == mine
        del later
    # the current stream's own: its blocks in turn
    s = Bd._scratch(n, t, None)
    at = s.data_ptr()
    del s
    assert Bd._scratch(n, t, torch.cuda.current_stream()).data_ptr() == at


def test_a_refused_call_is_not_recorded_by_the_launch_timing():
    c = Case(24, [9], [3], 1, 1, 64, 16, "f16")
    q = c.q.cuda()
    Bd.lsk_timing_begin()
    with pytest.raises(Bd.LsError, match="evenly"):
        Bd._check(Bd.lib().lsk_attn_tree(q.data_ptr(), 192, Bd.LS_F16, 3, 1, 3, 3, 2, 64, *[q.data_ptr()] * 6, 1, 16, 1, 9, q.data_ptr(), 192,
                                         None, 0, None))
    assert Bd.lsk_timing_end()["decode_attn"][1] == 0
    Bd.lsk_timing_begin()
    c.run(q=q)
    Bd.lsk_attn_tree(q, torch.empty_like(q), 1, 1, 64, i32(c.start), i32(c.past), c.mask(), 3, c.kp.cuda()[..., :12, :].contiguous(),
                     c.vp.cuda()[..., :12, :].contiguous(), i32(c.bt), 12, 9)      # pages that are no power of two: the other kernel
    assert Bd.lsk_timing_end()["decode_attn"][1] == 2


def kept_keys(c, b, t, gone):
    """Keys that row t of request b sees: cached tokens and its mask's nodes, none of them on the table's entries `gone`."""
    p = c.past[b]
    return np.array([j for j in list(range(p)) + [p + i for i in c.seen[t]] if j // c.page not in gone], np.int64)


def check_rows(c, o, rows, gone=()):
    """The given rows of request 0 against 64 bits, over the keys that are there."""
    q, kp, vp, got = f64(c.q), f64(c.kp), f64(c.vp), f64(o)
    half = D.HALF[c.dtype] if c.dtype != "f32" else 2 * D.F32
    for t in rows:
        j = kept_keys(c, 0, t, gone)
        for head in range(c.h):
            at = c.bt[0, j // c.page], head // (c.h // c.hk), j % c.page
            cols = slice(head * c.dh, (head + 1) * c.dh)
            ref, tol = D.attend(q[t, cols], kp[at], vp[at], np.arange(len(j)), c.dtype, half)
            assert (np.abs(got[t, cols] - ref) <= tol).all(), (t, head)


# nodes, heads and key heads as in ROWS; a tile of 64 keys holds nodes in both halves: the context ends at 52 of 64
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("nodes,h,hk", ROWS)
@pytest.mark.parametrize("dtype,dh", [("f16", 64), ("bf16", 128), ("bf16", 32), ("f32", 64), ("f16", 80)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, dh, nodes, h, hk, value):
    past = 692
    bad = [2, nodes - 2]                             # slots 694 and, from 24 nodes on, one of the next tile
    rng = np.random.default_rng(31)
    seen = [sorted({i} | set(np.flatnonzero(rng.random(nodes) < 0.4).tolist())) for i in range(nodes)]
    sees = [t for t in range(nodes) if set(bad) & set(seen[t])]
    blind = [t for t in range(nodes) if t not in sees]
    assert len(blind) >= 2 and len(sees) >= 2
    some = blind[::max(1, len(blind) // 4)]
    for scratch in (None, torch.empty(0, device="cuda")):      # the context in parts, and whole
        c = Case(31, [past], [nodes], h, hk, dh, 16, dtype, seen=seen)
        for i in bad:
            c.vp[c.bt[0, (past + i) // 16], :, (past + i) % 16] = value
        o = c.run(scratch=scratch)
        check_rows(c, o, some)
        hit = o[sees].float()
        assert torch.isnan(hit).all() if np.isnan(value) else (hit == value).all()
        for i in bad:
            c.kp[c.bt[0, (past + i) // 16], :, (past + i) % 16] = value
        o = c.run(scratch=scratch)
        check_rows(c, o, some)
        assert not torch.isfinite(o[sees].float()).any()


@pytest.mark.parametrize("nodes,h,hk", ROWS)
@pytest.mark.parametrize("dtype,dh", [("f16", 64), ("bf16", 128), ("bf16", 32), ("f32", 64), ("f16", 80)])
def test_missing_pages_of_the_context_and_of_the_nodes(dtype, dh, nodes, h, hk):
    past = 692                                       # pages 0 .. 42, four tokens of page 43 and the nodes behind them
    for gone in ((5,), (0, 1, 2, 3), (20, 43), (42, 44)):
        c = Case(32, [past], [nodes], h, hk, dh, 16, dtype)
        bt = c.bt.copy()
        for i, p in enumerate(g for g in gone if g < bt.shape[1]):
            bt[0, p] = -1 if i % 2 else c.n_pages
        for scratch in (None, torch.empty(0, device="cuda")):
            o = c.run(bt=i32(bt), scratch=scratch)
            check_rows(c, o, range(0, nodes, max(1, nodes // 5)), gone)
            assert torch.isfinite(o.float()).all()


@pytest.mark.parametrize("nodes", [8, 24])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_weights_of_few_rows_come_in_two_parts(dh, dtype, nodes):
    """Up to 32 rows the softmax weights enter the product rounded and as a remainder, each of 16 bits.  Outputs are made nearly
    zero by cancellation, so that their own rounding hides nothing: weights rounded once would be outside the bound."""
    past = 40
    c = Case(33, [past], [nodes], 1, 1, dh, 16, dtype, seen=[[i] for i in range(nodes)])
    c.q[:, 2:] = 0                                   # scores of two products each
    q, kp, vp = f64(c.q), f64(c.kp), f64(c.vp)
    slot = lambda j: (c.bt[0, j // 16], 0, j % 16)   # noqa: E731
    seen = [np.array(list(range(past)) + [past + t]) for t in range(nodes)]
    scores = [kp[slot(seen[t])] @ q[t] / np.sqrt(dh) for t in range(nodes)]
    weights = [np.exp(s - s.max()) / np.exp(s - s.max()).sum() for s in scores]
    # dimension d is balanced for row d % nodes by the value of that row's own key
    for d in range(dh):
        t = d % nodes
        v = vp[slot(seen[t])][:, d]
        c.vp[slot(past + t) + (d,)] = float(np.clip(-(weights[t][:-1] @ v[:-1]) / weights[t][-1], -1e3, 1e3))
    vp, got = f64(c.vp), f64(c.run())
    once = 0
    for t in range(nodes):
        v, w, s = vp[slot(seen[t])], weights[t], scores[t]
        ref, mag = w @ v, w @ np.abs(v)
        # a remainder is at most HALF of its weight and is rounded by HALF of itself; the score is two exact products, their sum,
        # the scaling and the exponential's argument; sums over the keys in fp32
        rel = D.HALF[dtype] ** 2 + 2 * 8 * D.F32 * max(1.0, np.abs(s).max()) + (len(w) / 4 + 80) * D.F32
        tol = 1.01 * rel * mag + 1.01 * D.HALF[dtype] * np.abs(ref) + 2.0 ** -24 * (dtype == "f16")
        if dtype == "f16":                           # parts below 2^-20 of the largest weight are subnormal, and lost
            tol = tol + 2.0 ** -20 * w.max() * np.abs(v).sum(0)
        assert (np.abs(got[t] - ref) <= tol).all(), (t, float((np.abs(got[t] - ref) / tol).max()))
        p = torch.from_numpy(np.exp(s - s.max()).astype(np.float32))
        single = (f64(p.to(DT[dtype])) @ v) / f64(p).sum()
        once += int((np.abs(single - ref) > tol).sum())
    assert once > dh // 8


@pytest.mark.parametrize("T", [1, 2])
def test_q_in_place_of_its_columns_of_the_projection(T):
    """q_out is the q columns of qkv, for one row as for several; so are q and o of the attention a part of wider rows."""
    h, hk, dh, page = 4, 2, 64, 16
    g = torch.Generator()
    g.manual_seed(41)
    x = torch.randn(T, (h + 2 * hk) * dh, generator=g).half().cuda()
    kp, vp = (torch.zeros(1, hk, page, dh, dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.from_numpy(D.table(16, dh)).cuda()
    args = (h, hk, dh, i32(range(T)), i32([0] * T), kp, vp, i32([[0]]), page)
    want = torch.empty(T, h * dh, dtype=torch.float16, device="cuda")
    Bd.lsk_qk_norm_rope_kv_write(x, want, *args, table=table)
    k = kp.clone()
    y = x.clone()
    Bd.lsk_qk_norm_rope_kv_write(y, y[:, :h * dh], *args, table=table)
    assert torch.equal(y[:, :h * dh], want) and torch.equal(y[:, h * dh:], x[:, h * dh:]) and torch.equal(kp, k)
    mask = torch.tensor([[(2 << t) - 1] for t in range(T)], device="cuda")
    tree = (h, hk, dh, i32([0, T]), i32([0]), mask, T, kp, vp, i32([[0]]), page, 0)
    o, wide = torch.empty_like(want), torch.full((T, h * dh + 3), 7.0, dtype=torch.float16, device="cuda")
    Bd.lsk_attn_tree(want, o, *tree)
    Bd.lsk_attn_tree(y[:, :h * dh], wide[:, :h * dh], *tree)
    assert torch.allclose(wide[:, :h * dh].float(), o.float(), rtol=2 ** -9, atol=2 ** -12) and (wide[:, h * dh:] == 7).all()


def test_scratch_of_the_default_stream_from_within_another():
    n, t, side = 3 << 20, torch.empty(1, device="cuda"), torch.cuda.Stream()
    for stream in (0, torch.cuda.default_stream()):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        with torch.cuda.stream(side):
            s = Bd._scratch(n, t, stream)
            at = s.data_ptr()
            del s
            assert torch.empty(n, device="cuda").data_ptr() != at
        assert torch.empty(n, device="cuda").data_ptr() == at      # the default stream's block again


def test_a_captured_call_with_scratch_of_its_own():
    """The wrapper's scratch belongs to the graph: replays with eager calls and allocations of that size between them."""
    c = Case(42, [3000, 1200], [9, 4], 4, 2, 128, 16, "bf16")
    args = dict(kp=c.kp.cuda(), vp=c.vp.cuda(), bt=i32(c.bt), mask=c.mask(), start=i32(c.start), ctx=i32(c.past))
    n = Bd.lib().lsk_attn_tree_scratch_floats(c.T, 2, 4, 2, 128, c.max_nodes, 3000)
    assert n > 0
    q, o = c.q.cuda(), torch.empty(c.T, 512, dtype=torch.bfloat16, device="cuda")
    c.run(q=q, o=o, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(q=q, o=o, **args)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for _ in range(3):
        q.normal_(generator=g)
        others = [torch.full((n,), float("nan"), device="cuda") for _ in range(3)]
        graph.replay()
        want = c.run(q=q.clone(), **args)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        del others
