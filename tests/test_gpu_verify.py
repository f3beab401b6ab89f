"""stage_verify and the calls around it: drafted trees through a whole stage, acceptance, forks and compaction, against the
oracle's causal forward along every path of the tree."""
import copy

import numpy as np
import pytest
import torch

import draft_util as D
from oracle import stage_oracle as O
from paper_2507_21276_amd import binding as Bd
from paper_2507_21276_amd import sched
from paper_2507_21276_amd import synth_inputs as S
from parity_util import TOL, assert_close, dev, host

pytestmark = pytest.mark.gpu

LLAMA = S.scaled(S.CONFIGS["llama7b_bf16"], n_layers=2, d_model=256, n_heads=2, d_ff=704, max_pos=512)
GPT = S.scaled(S.CONFIGS["gpt2s_bf16"], n_layers=2, d_model=192, n_heads=3, d_ff=768)
SMALL = S.scaled(S.CONFIGS["tiny_gpt_f32"], n_layers=2)
CASES = [("llama", LLAMA, "f16"), ("llama", LLAMA, "bf16"), ("gpt", GPT, "f16"), ("f32", SMALL, "f32")]


def make(cfg, mma):
    st = Bd.Stage(cfg, io_dtype="f32", mma_dtype=mma)
    flat = S.make_params(cfg, perturb_norm=0.1)
    st.ls_bind_params(dev(flat, st.param_torch))
    return st, flat.astype(np.float64)


def tree_forward(cfg, f64, X, parents, cache, b):
    """Y of every node of request b's tree: the causal forward along the path that ends at it, and each node's K and V rows."""
    out = np.empty_like(X)
    rows = [None] * len(parents)
    for path in D.ancestors(parents):
        c = [[copy.copy(l[b])] for l in cache]
        y = O.stage_prefill(cfg, f64, [X[path]], c)[0]
        out[path[-1]] = y[-1]
        rows[path[-1]] = [(l[0][0][-1], l[0][1][-1]) for l in c]
    return out, rows


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32)).cuda()


@pytest.mark.parametrize("name,cfg,mma", CASES)
@pytest.mark.parametrize("past,counts", [([0], [1]), ([21, 0, 40], [7, 12, 1]), ([33, 5], [60, 90])])
def test_verify_and_accept(name, cfg, mma, past, counts):
    rng = np.random.default_rng(1)
    d, page, B = cfg["d_model"], cfg["page_size"], len(past)
    st, f64 = make(cfg, mma)
    bt, n_pages = D.page_table(rng, [p + n + 1 for p, n in zip(past, counts)], page)
    bt = np.where(bt < n_pages, bt, 0).astype(np.int32)
    kv = Bd.KV(st, n_pages, bt, [0] * B)
    kv.k_pool.fill_(float("nan"))
    kv.v_pool.fill_(float("nan"))
    cache = O.new_cache(cfg, B)
    T = sum(counts)
    ws = st.new_workspace(max(sum(past), T, 1))
    live = [b for b in range(B) if past[b]]
    if live:
        P = [S.make_activations(cfg, "P%d" % b, (past[b], d)) for b in live]
        sub = Bd.KV.of(kv.k_pool, kv.v_pool, i32(bt[live]), [0] * len(live))
        Y = torch.empty(sum(past), d, device="cuda")
        st.stage_prefill(dev(np.concatenate(P), torch.float32), [past[b] for b in live], sub, Y, ws)
        part = [[l[b] for b in live] for l in cache]
        O.stage_prefill(cfg, f64, [p.astype(np.float64) for p in P], part)
        for l in range(cfg["n_layers"]):
            for i, b in enumerate(live):
                cache[l][b] = part[l][i]
    kv.set_ctx(past)
    parents = D.trees(rng, counts)
    start = np.concatenate([[0], np.cumsum(counts)])
    X = S.make_activations(cfg, "X", (T, d))
    Y = torch.full((T, d), 7.0, device="cuda")
    st.stage_verify(dev(X, torch.float32), i32(sum(parents, [])), i32(start), counts, kv, Y, ws)
    refs, rows = zip(*[tree_forward(cfg, f64, X[start[b]:start[b + 1]].astype(np.float64), parents[b], cache, b) for b in range(B)])
    ref = np.concatenate(refs)
    tol = TOL["f32" if mma == "f32" else "bf16"]   # the stage tests' bar for Y
    assert_close(host(Y), ref, tol, "Y")
    # the last node's path is accepted; one more token behind it
    paths = [D.ancestors(p)[-1] for p in parents]
    most = max(len(p) for p in paths)
    Bd.lsk_kv_move_rows(st.c, kv, i32([p + [0] * (most - len(p)) for p in paths]), i32([len(p) for p in paths]))
    kv.set_ctx([a + len(p) for a, p in zip(past, paths)])
    for l in range(cfg["n_layers"]):
        for b, path in enumerate(paths):
            K, V = cache[l][b]
            K = np.concatenate([K] + [rows[b][i][l][0][None] for i in path]) if K.size else np.stack([rows[b][i][l][0] for i in path])
            V = np.concatenate([V] + [rows[b][i][l][1][None] for i in path]) if V.size else np.stack([rows[b][i][l][1] for i in path])
            cache[l][b] = [K, V]
    xt = S.make_activations(cfg, "xt", (B, d))
    yt = torch.empty(B, d, device="cuda")
    st.stage_decode(dev(xt, torch.float32), B, kv, yt, ws)
    assert_close(host(yt), O.stage_decode(cfg, f64, xt.astype(np.float64), cache), tol, "the step after")
    st.close()


@pytest.mark.parametrize("name,cfg,mma", CASES)
def test_a_chain_is_a_prompt_chunk_and_one_node_a_decode_step(name, cfg, mma):
    rng = np.random.default_rng(2)
    st, _ = make(cfg, mma)
    d, past, n = cfg["d_model"], [19, 50], [6, 6]
    bt, n_pages = D.page_table(rng, [60, 60], cfg["page_size"])
    kvs = [Bd.KV(st, n_pages, bt, past) for _ in range(2)]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    kvs[0].k_pool.normal_(generator=g)
    kvs[0].v_pool.normal_(generator=g)
    kvs[1].k_pool.copy_(kvs[0].k_pool)
    kvs[1].v_pool.copy_(kvs[0].v_pool)
    X = dev(S.make_activations(cfg, "X", (12, d)), torch.float32)
    ws, Ya, Yb = st.new_workspace(12), torch.empty(12, d, device="cuda"), torch.empty(12, d, device="cuda")
    st.stage_verify(X, i32([-1, 0, 1, 2, 3, 4] * 2), i32([0, 6, 12]), n, kvs[0], Ya, ws)
    st.stage_prefill(X, n, kvs[1], Yb, ws)
    tol = 2 * TOL["f32" if mma == "f32" else "bf16"]   # each of the two within the bar
    assert_close(host(Ya), host(Yb), tol, "chain")
    # without the lengths on the host the same launch is sized by the table
    st.stage_verify(X, i32([-1, 0, 1, 2, 3, 4] * 2), i32([0, 6, 12]), n, kvs[0], Yb, ws, with_host=False)
    assert_close(host(Yb), host(Ya), tol, "without host lengths")
    st.stage_verify(X, i32([-1, -1]), i32([0, 1, 2]), [1, 1], kvs[0], Ya, ws)
    st.stage_decode(X, 2, kvs[1], Yb, ws)
    assert_close(host(Ya)[:2], host(Yb)[:2], tol, "single nodes")
    st.close()


def test_forks_and_compaction_leave_every_continuation_as_it_was():
    """One prompt, forked twice; the forks continue on their own, the first is dropped and the pool packed."""
    cfg, mma = LLAMA, "f16"
    st, f64 = make(cfg, mma)
    d, page = cfg["d_model"], cfg["page_size"]
    books = sched.Pages(14, page, 3, 6)
    kv = Bd.KV(st, 14, books.table(), [0, 0, 0])
    ws = st.new_workspace(64)
    cache = O.new_cache(cfg, 3)

    def sync(pairs):
        Bd.lsk_kv_copy_pages(st.c, kv, *pairs)
        kv.block_table = i32(books.table())

    sync(books.grow(0, 0, 39))
    P = S.make_activations(cfg, "P", (39, d))
    Y = torch.empty(39, d, device="cuda")
    st.stage_prefill(dev(P, torch.float32), [39], Bd.KV.of(kv.k_pool, kv.v_pool, kv.block_table[:1], [0]), Y, ws)
    part = [[c[0]] for c in cache]
    O.stage_prefill(cfg, f64, [P.astype(np.float64)], part)
    for l in range(cfg["n_layers"]):
        cache[l] = [[a.copy() for a in part[l][0]] for _ in range(3)]
    for r in (1, 2):
        books.fork(0, r, 39)
    ctx = [39, 39, 39]

    def steps(rows, n, tag):
        for i in range(n):
            for r in rows:
                sync(books.grow(r, ctx[r], ctx[r] + 1))
            x = S.make_activations(cfg, "%s%d" % (tag, i), (len(rows), d))
            y = torch.empty(len(rows), d, device="cuda")
            st.stage_decode(dev(x, torch.float32), len(rows), Bd.KV.of(kv.k_pool, kv.v_pool, kv.block_table[rows].contiguous(),
                                                                      [ctx[r] for r in rows]), y, ws)
            part = [[l[r] for r in rows] for l in cache]
            ref = O.stage_decode(cfg, f64, x.astype(np.float64), part)
            for l in range(cfg["n_layers"]):
                for j, r in enumerate(rows):
                    cache[l][r] = part[l][j]
            for r in rows:
                ctx[r] += 1
            assert_close(host(y), ref, TOL["bf16"], tag)

    steps([0, 1, 2], 12, "apart")               # the shared last page is copied for two of the three
    books.truncate(0, 0)
    sync(books.compact())
    assert max(max(books.row(1)), max(books.row(2))) == 14 - books.available() - 1
    steps([1, 2], 6, "packed")
    st.close()


def test_verify_refuses_bad_arguments():
    st, _ = make(SMALL, "f32")
    kv = Bd.KV(st, 8, np.arange(8).reshape(2, 4), [10, 60])
    d = SMALL["d_model"]
    X, Y, ws = torch.zeros(300, d, device="cuda"), torch.empty(300, d, device="cuda"), st.new_workspace(300)
    parent, start = i32([-1] * 300), i32([0, 1, 2])
    for n, frag in (([1, 5], "block table"), ([0, 1], "nodes"), ([257, 1], "nodes"), ([-1, 1], "nodes"), ([], "B must be")):
        with pytest.raises(Bd.LsError, match=frag):
            st.stage_verify(X, parent, start, n, kv, Y, ws)
    with pytest.raises(Bd.LsError, match="null"):
        st.stage_verify(X, None, start, [1, 1], kv, Y, ws)
    st.stage_verify(X, parent, start, [1, 4], kv, Y, ws)
    torch.cuda.synchronize()
    st.close()


def test_a_captured_verification_replays():
    rng = np.random.default_rng(4)
    cfg, counts, past = LLAMA, [9, 4], [30, 111]
    st, _ = make(cfg, "f16")
    bt, n_pages = D.page_table(rng, [p + n for p, n in zip(past, counts)], cfg["page_size"])
    kv = Bd.KV(st, n_pages, np.where(bt < n_pages, bt, 0), past)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    kv.k_pool.normal_(generator=g)
    kv.v_pool.normal_(generator=g)
    parent, start = i32(sum(D.trees(rng, counts), [])), i32([0, 9, 13])
    X, Y, ws = torch.zeros(13, cfg["d_model"], device="cuda"), torch.empty(13, cfg["d_model"], device="cuda"), st.new_workspace(13)
    st.stage_verify(X, parent, start, counts, kv, Y, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.stage_verify(X, parent, start, counts, kv, Y, ws)
    ws2, Y2 = st.new_workspace(13), torch.empty_like(Y)
    for _ in range(3):
        X.normal_(generator=g)
        graph.replay()
        st.stage_verify(X, parent, start, counts, kv, Y2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(Y, Y2)
    st.close()
