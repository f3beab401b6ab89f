"""Attention of drafted trees over the paged cache, and the index arrays made from the parents, against 64-bit definitions."""
import numpy as np
import pytest
import torch

import draft_util as D
from paper_2507_21276_amd import binding as Bd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def f64(t):
    return t.detach().cpu().double().numpy()


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32)).cuda()


class Case:
    """Ragged requests over a shuffled pool; everything that no row sees is NaN."""

    def __init__(self, seed, past, counts, h, hk, dh, page, dtype, seen=None, max_nodes=None, pad_rows=0, std=1.0):
        rng = np.random.default_rng(seed)
        self.past, self.counts, self.h, self.hk, self.dh, self.page, self.dtype = past, counts, h, hk, dh, page, dtype
        self.T = sum(counts)
        self.max_nodes = max(max(counts), 1) if max_nodes is None else max_nodes
        self.words = (self.max_nodes + 63) // 64
        self.start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.parents = D.trees(rng, counts)
        self.seen = seen if seen is not None else [a for p in self.parents for a in D.ancestors(p)]
        self.bt, self.n_pages = D.page_table(rng, [p + n for p, n in zip(past, counts)], page)
        q = rng.standard_normal((self.T + pad_rows, h * dh)) * std
        self.q = torch.from_numpy(q.astype(np.float32)).to(DT[dtype])
        kp = np.full((self.n_pages, hk, page, dh), np.nan, np.float32)
        vp = kp.copy()
        for b, (p, n) in enumerate(zip(past, counts)):
            for j in range(p + n):
                kp[self.bt[b, j // page], :, j % page] = rng.standard_normal((hk, dh)) * std
                vp[self.bt[b, j // page], :, j % page] = rng.standard_normal((hk, dh))
        self.kp, self.vp = torch.from_numpy(kp).to(DT[dtype]), torch.from_numpy(vp).to(DT[dtype])

    def mask(self):
        rows = self.q.shape[0]
        m = np.zeros((rows, self.words), np.int64)
        m[:self.T] = D.mask_words(self.seen, self.words)
        return torch.from_numpy(m).cuda()

    def run(self, scratch=None, max_ctx=None, q=None, o=None, **over):
        q = self.q.cuda() if q is None else q
        o = torch.full((q.shape[0], self.h * self.dh), 7.0, dtype=DT[self.dtype], device="cuda") if o is None else o
        made = dict(kp=self.kp.cuda, vp=self.vp.cuda, bt=lambda: i32(self.bt), mask=self.mask, start=lambda: i32(self.start),
                    ctx=lambda: i32(self.past))
        a = {k: over[k] if k in over else f() for k, f in made.items()}
        Bd.lsk_attn_tree(q, o, self.h, self.hk, self.dh, a["start"], a["ctx"], a["mask"], self.max_nodes, a["kp"], a["vp"], a["bt"],
                         self.page, max(self.past) if max_ctx is None else max_ctx, scratch=scratch)
        return o

    def check(self, o, rows=None):
        """Every row and head (or the given rows) within the bound of the kernel's roundings."""
        got, q, kp, vp = f64(o), f64(self.q), f64(self.kp), f64(self.vp)
        half = D.HALF[self.dtype] if self.dtype != "f32" else 2 * D.F32
        g = self.h // self.hk
        for b, (p, n) in enumerate(zip(self.past, self.counts)):
            j = np.arange(p + n)
            keys, values = kp[self.bt[b, j // self.page], :, j % self.page], vp[self.bt[b, j // self.page], :, j % self.page]
            for i in range(n):
                t = int(self.start[b]) + i
                if rows is not None and t not in rows:
                    continue
                seen = np.concatenate([np.arange(p), p + np.asarray(self.seen[t], np.int64)]).astype(np.int64)
                for head in range(self.h):
                    ref, tol = D.attend(q[t, head * self.dh:(head + 1) * self.dh], keys[:, head // g], values[:, head // g], seen,
                                        self.dtype, half)
                    err = np.abs(got[t, head * self.dh:(head + 1) * self.dh] - ref)
                    assert (err <= tol).all(), (t, head, float((err - tol).max()), float(err.max()))


# requests' contexts and tree sizes: no context, no tree, one token, tiles and pages that end anywhere
RAGGED = [([0], [1]), ([1], [1]), ([77], [5]), ([0, 40, 3], [4, 0, 9]), ([31, 32, 33, 64], [1, 16, 17, 3]), ([200, 0, 15], [33, 64, 2]),
          ([129, 500], [65, 12])]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("h,hk,dh,page", [(2, 2, 64, 16), (4, 1, 128, 16), (6, 2, 32, 8), (5, 5, 128, 64), (3, 1, 64, 32)])
@pytest.mark.parametrize("past,counts", RAGGED)
def test_ragged_trees(past, counts, h, hk, dh, page, dtype):
    c = Case(1, past, counts, h, hk, dh, page, dtype)
    c.check(c.run())


@pytest.mark.parametrize("dtype,h,hk,dh,page", [("f16", 2, 1, 80, 16), ("bf16", 3, 3, 256, 16), ("f32", 2, 2, 7, 5), ("f16", 2, 2, 64, 12)])
def test_sizes_that_the_matrix_core_kernel_does_not_take(dtype, h, hk, dh, page):
    c = Case(2, [37, 0, 70], [5, 3, 1], h, hk, dh, page, dtype)
    c.check(c.run())


@pytest.mark.parametrize("dtype,h,hk,dh", [("f16", 2, 2, 128), ("bf16", 8, 1, 64), ("f32", 1, 1, 32), ("bf16", 5, 1, 128)])
def test_long_contexts_are_split_and_joined(dtype, h, hk, dh):
    c = Case(3, [2500, 700, 0], [7, 33, 1], h, hk, dh, 16, dtype)
    whole = c.run()
    rows = set(range(0, c.T, 5)) | {c.T - 1}
    c.check(whole, rows)
    # less scratch, fewer parts; none at all: one
    n = Bd.lib().lsk_attn_tree_scratch_floats(c.T, 3, h, hk, dh, c.max_nodes, max(c.past))
    if n:
        c.check(c.run(scratch=torch.empty(n // 2, dtype=torch.float32, device="cuda")), rows)
    c.check(c.run(scratch=torch.empty(0, dtype=torch.float32, device="cuda")), rows)
    # a wrong bound on the contexts changes the launch and not the result
    c.check(c.run(max_ctx=64), rows)
    c.check(c.run(max_ctx=100000), rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_largest_trees_and_shared_heads(dtype):
    c = Case(4, [50, 3], [256, 130], 4, 1, 64, 16, dtype)
    c.check(c.run(), set(range(0, c.T, 23)) | {255, 256, c.T - 1})


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_any_mask_and_rows_that_see_nothing(dtype):
    rng = np.random.default_rng(5)
    past, counts = [0, 20, 0], [40, 6, 3]
    seen = [list(np.flatnonzero(rng.random(n) < 0.3)) for n in counts for _ in range(n)]
    seen[0] = seen[7] = []            # request 0 has no context: these rows see nothing
    seen[-1] = [2]
    c = Case(5, past, counts, 2, 1, 64, 16, dtype, seen=seen)
    o = c.run()
    c.check(o)
    assert (o[0] == 0).all() and (o[7] == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_what_a_node_does_not_see_does_not_reach_it(dtype, value):
    """Keys and values of one node are not finite: the rows that do not see it are as if it were not there."""
    past, counts = [45], [20]
    c = Case(6, past, counts, 4, 2, 128, 16, dtype)
    bad = 3
    at = c.bt[0, (45 + bad) // 16], slice(None), (45 + bad) % 16
    clean = c.run()
    c.kp[at], c.vp[at] = value, value
    o = c.run()
    blind = [i for i in range(20) if bad not in c.seen[i]]
    assert blind and len(blind) < 20
    assert torch.equal(o[blind], clean[blind])
    assert not torch.isfinite(o[[i for i in range(20) if bad in c.seen[i]]].float()).any()
    # only the values: an infinity of either sign reaches the rows that see it with its sign
    c = Case(6, past, counts, 4, 2, 128, 16, dtype)
    c.vp[at] = value
    o = c.run()
    sees = o[[i for i in range(20) if bad in c.seen[i]]].float()
    assert torch.equal(o[blind], clean[blind])
    assert torch.isnan(sees).all() if np.isnan(value) else (sees == value).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_large_scores(dtype):
    """Scores of several hundred: one key takes nearly all the weight."""
    c = Case(7, [70, 300], [9, 4], 2, 1, 64, 16, dtype, std=8.0)
    c.check(c.run())


def test_scores_that_overflow():
    """bf16 products beyond fp32: a key at -inf has no weight beside finite ones."""
    c = Case(8, [40], [3], 1, 1, 64, 16, "bf16")
    clean = c.run()
    page = c.bt[0]
    c.q[:, 0] = 1e20
    c.kp[page[0], :, 5, :] = 0
    c.kp[:, :, :, 0] = torch.where(torch.isnan(c.kp[:, :, :, 0]), c.kp[:, :, :, 0], torch.zeros_like(c.kp[:, :, :, 0]))
    c.kp[page[0], :, 5, 0] = -1e20          # score -inf
    o = c.run()
    assert torch.isfinite(o.float()).all()
    seen = c.seen
    vp, kp = f64(c.vp), f64(c.kp)
    j = np.array([i for i in range(43) if i != 5])
    keys, values = kp[page[j // 16], 0, j % 16], vp[page[j // 16], 0, j % 16]
    for t in range(3):
        idx = np.array([k for k, jj in enumerate(j) if jj < 40 or jj - 40 in seen[t]])
        ref, tol = D.attend(f64(c.q)[t], keys, values, idx, "bf16", D.HALF["bf16"])
        assert (np.abs(f64(o)[t] - ref) <= tol).all()
    assert clean.shape == o.shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_the_last_tree_and_strided_rows(dtype):
    c = Case(9, [33, 5], [4, 7], 4, 2, 64, 16, dtype, pad_rows=3)
    wide_q = torch.full((c.T + 3, 4 * 64 + 24), 2.0, dtype=DT[dtype], device="cuda")
    wide_o = torch.full((c.T + 3, 4 * 64 + 40), 7.0, dtype=DT[dtype], device="cuda")
    wide_q[:, 8:8 + 256] = c.q.cuda()
    c.run(q=wide_q[:, 8:8 + 256], o=wide_o[:, 16:16 + 256])
    c.check(wide_o[:, 16:16 + 256])
    assert (wide_o[c.T:] == 7).all() and (wide_o[:, :16] == 7).all() and (wide_o[:, 272:] == 7).all()
    # rows and pools that are not aligned to 16 bytes
    odd_q = torch.full((c.T + 3, 4 * 64 + 3), 2.0, dtype=DT[dtype], device="cuda")
    odd_q[:, 1:257] = c.q.cuda()
    flat = lambda x: torch.cat([x.flatten()[:1], x.flatten()]).cuda()[1:].view(x.shape)  # noqa: E731
    odd_o = torch.full((c.T + 3, 4 * 64 + 5), 7.0, dtype=DT[dtype], device="cuda")
    c.run(q=odd_q[:, 1:257], o=odd_o[:, 3:259], kp=flat(c.kp), vp=flat(c.vp))
    c.check(odd_o[:, 3:259])
    assert (odd_o[c.T:] == 7).all() and (odd_o[:, :3] == 7).all() and (odd_o[:, 259:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_pages_that_do_not_exist_are_not_seen(dtype):
    """Table entries outside the pool, and a context longer than the table row: those keys do not count."""
    c = Case(10, [60], [4], 2, 1, 64, 16, dtype)
    bt = c.bt.copy()
    bt[0, 1] = -1
    kept = [j for j in range(64) if j // 16 != 1]
    o = c.run(bt=i32(bt))
    q, kp, vp = f64(c.q), f64(c.kp), f64(c.vp)
    j = np.array(kept)
    keys, values = kp[c.bt[0, j // 16], 0, j % 16], vp[c.bt[0, j // 16], 0, j % 16]
    for t in range(4):
        idx = np.array([k for k, jj in enumerate(kept) if jj < 60 or jj - 60 in c.seen[t]])
        for head in range(2):
            ref, tol = D.attend(q[t, head * 64:head * 64 + 64], keys, values, idx, dtype, 2 * D.HALF[dtype])
            assert (np.abs(f64(o)[t, head * 64:head * 64 + 64] - ref) <= tol).all()
    # 60 cached tokens of which the two-page row holds 32: the nodes' own keys are out of reach
    o = c.run(bt=i32(c.bt[:, :2]))
    keys, values = keys[:0], values[:0]
    j = np.arange(32)
    keys, values = kp[c.bt[0, j // 16], 0, j % 16], vp[c.bt[0, j // 16], 0, j % 16]
    for t in range(4):
        ref, tol = D.attend(q[t, :64], keys, values, j, dtype, 2 * D.HALF[dtype])
        assert (np.abs(f64(o)[t, :64] - ref) <= tol).all()


def test_nodes_beyond_the_stated_most_are_left_alone():
    c = Case(11, [10, 4], [6, 3], 2, 2, 64, 16, "f16", max_nodes=4, seen=[[0]] * 9)
    o = c.run()
    assert (o[4:6] == 7).all()
    c.check(o, {0, 1, 2, 3, 6, 7, 8})


@pytest.mark.parametrize("counts,max_nodes,extra", [([1], 1, 0), ([5, 0, 64], 64, 3), ([65, 7], 130, 5), ([256, 1, 2], 256, 300), ([9, 3], 4, 0)])
def test_index_arrays(counts, max_nodes, extra):
    rng = np.random.default_rng(12)
    parents = D.trees(rng, counts)
    T, past = sum(counts) + extra, [int(v) for v in rng.integers(0, 500, len(counts))]
    start = np.concatenate([[0], np.cumsum(counts)])
    flat = np.array([p for t in parents for p in t] + [55] * extra, np.int32)
    words = (max_nodes + 63) // 64
    pos, slot, req = (torch.full((T,), 99, dtype=torch.int32, device="cuda") for _ in range(3))
    mask = torch.full((T, words), -1, dtype=torch.int64, device="cuda")
    Bd.lsk_tree_index(i32(flat), i32(start), i32(past), max_nodes, pos, slot, req, mask)
    wp, ws, wr = np.zeros(T), np.zeros(T), np.full(T, -1)
    wm = np.zeros((T, words), np.int64)
    for b, (n, par) in enumerate(zip(counts, parents)):
        seen = D.ancestors(par)
        for i in range(min(n, max_nodes)):
            t = start[b] + i
            wp[t], ws[t], wr[t] = past[b] + len(seen[i]) - 1, past[b] + i, b
            wm[t] = D.mask_words([seen[i]], words)[0]
    for got, want in ((pos, wp), (slot, ws), (req, wr), (mask, wm)):
        assert (got.cpu().numpy() == want).all()


def test_parents_that_are_not_earlier_nodes_count_as_the_context():
    parent = i32([0, 5, -9, 1, 3])
    pos, slot, req = (torch.empty(5, dtype=torch.int32, device="cuda") for _ in range(3))
    mask = torch.empty(5, 1, dtype=torch.int64, device="cuda")
    Bd.lsk_tree_index(parent, i32([0, 5]), i32([10]), 8, pos, slot, req, mask)
    assert mask.flatten().tolist() == [1, 2, 4, 0b1010, 0b11010] and pos.tolist() == [10, 10, 10, 11, 12]


@pytest.mark.parametrize("dtype,h,hk,dh", [("f16", 4, 4, 128), ("bf16", 4, 1, 64), ("f32", 2, 2, 32)])
def test_one_node_is_a_decode_step(dtype, h, hk, dh):
    """A tree of one node per request gives what lsk_attn_paged gives for the same row."""
    c = Case(13, [0, 17, 300, 64], [1, 1, 1, 1], h, hk, dh, 16, dtype)
    o = c.run()
    c.check(o)
    if h != hk:
        return
    kp, vp, bt = c.kp.cuda(), c.vp.cuda(), i32(np.where(c.bt < c.n_pages, c.bt, 0))
    qkv = torch.cat([c.q.cuda(), torch.zeros(4, 2 * h * dh, dtype=c.q.dtype, device="cuda")], 1).contiguous()
    o2 = torch.empty_like(o)
    Bd.lsk_attn_paged(0 if dtype == "f32" else 1, qkv, h, dh, i32(c.past), i32([0, 1, 2, 3]), kp, vp, bt, 16, 301, o2)
    c.check(o2)


def test_captured_calls_on_other_streams():
    """Index, page write and attention in a graph: replayed with eager work of the same kind between the replays, and two
    calls on two streams at once with a scratch each."""
    c = Case(14, [1500, 90], [12, 5], 4, 2, 128, 16, "f16")
    args = dict(kp=c.kp.cuda(), vp=c.vp.cuda(), bt=i32(c.bt), mask=c.mask(), start=i32(c.start), ctx=i32(c.past))
    n = max(1, Bd.lib().lsk_attn_tree_scratch_floats(c.T, 2, 4, 2, 128, c.max_nodes, 1500))
    q, o = c.q.cuda(), torch.empty(c.T, 512, dtype=torch.float16, device="cuda")
    scratch = torch.empty(n, dtype=torch.float32, device="cuda")
    c.run(q=q, o=o, scratch=scratch, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(q=q, o=o, scratch=scratch, **args)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for _ in range(3):
        q.normal_(generator=g)
        graph.replay()
        want = c.run(q=q.clone(), **args)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    qs = [torch.empty_like(q).normal_(generator=g) for _ in streams]
    wants = [c.run(q=x, **args) for x in qs]
    outs = [torch.empty_like(o) for _ in streams]
    scr = [torch.empty(n, dtype=torch.float32, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for s, x, y, z in zip(streams, qs, outs, scr):
        with torch.cuda.stream(s):
            c.run(q=x, o=y, scratch=z, **args)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))


def test_scratch_of_a_call_on_a_stream_that_is_not_the_current_one():
    """The wrapper's own scratch is not handed to the current stream's work while the call has yet to run on its own."""
    c = Case(15, [1500, 90], [12, 5], 4, 2, 128, 16, "f16")
    args = [i32(c.start), i32(c.past), c.mask(), c.max_nodes, c.kp.cuda(), c.vp.cuda(), i32(c.bt), 16, 1500]
    q, o = c.q.cuda(), torch.empty(c.T, 512, dtype=torch.float16, device="cuda")
    n = Bd.lib().lsk_attn_tree_scratch_floats(c.T, 2, 4, 2, 128, c.max_nodes, 1500)
    assert n > 0
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        o.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2000000)
        Bd.lsk_attn_tree(q, o, 4, 2, 128, *args, stream=stream)
        others = [torch.full((n,), float("nan"), device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        c.check(o)
        del others


# more workgroups than the chip holds at once, whose requests go by length: equal and empty contexts, more than 64 requests, a
# last group of a few, shared key heads and parts
@pytest.mark.parametrize("dtype,B,lo,hi,n,h,hk,dh", [("f16", 131, 0, 40, 2, 4, 4, 64), ("bf16", 65, 0, 3, 40, 10, 10, 32), ("f16", 66, 0, 90, 70, 8, 8, 128),
                                                     ("f32", 129, 5, 9, 3, 5, 5, 32), ("bf16", 17, 100, 1500, 30, 16, 8, 64),
                                                     ("f32", 3, 0, 3000, 9, 64, 64, 32), ("f16", 600, 0, 4, 1, 1, 1, 128)])
def test_many_requests_of_different_lengths(dtype, B, lo, hi, n, h, hk, dh):
    rng = np.random.default_rng(16)
    past, counts = [int(v) for v in rng.integers(lo, hi + 1, B)], [int(v) for v in rng.integers(0, n + 1, B)]
    counts[B // 2] = n
    c = Case(17, past, counts, h, hk, dh, 16, dtype)
    scratch = torch.empty(max(1, Bd.lib().lsk_attn_tree_scratch_floats(c.T, B, h, hk, dh, c.max_nodes, max(past))), device="cuda")
    o = c.run(scratch=scratch)
    c.check(o, rows=None if c.T * h < 4000 else set(rng.choice(c.T, 4000 // h, replace=False).tolist()))
    assert not torch.isnan(o).any() and not (o == 7.0).all(1).any()      # every row was written
