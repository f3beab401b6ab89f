"""Moving cached pages and rows: bit for bit what the same moves give on the host."""
import numpy as np
import pytest
import torch

import draft_util as D
from paper_2507_21276_amd import binding as Bd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def config(layers, h, dh, page, dtype):
    return Bd.make_config(dict(block="gpt", dtype="f32" if dtype == "f32" else "bf16", n_layers=layers, d_model=h * dh, n_heads=h,
                               head_dim=dh, d_ff=64, act="gelu_tanh", norm_eps=1e-5, rope_theta=1e4, page_size=page, max_pos=0),
                          mma_dtype=dtype)


def pools(seed, layers, n_pages, h, page, dh, dtype):
    """Any bit pattern, not numbers only."""
    g = torch.Generator()
    g.manual_seed(seed)
    out = []
    for _ in range(2):
        size = layers * n_pages * h * page * dh * (4 if dtype == "f32" else 2)
        out.append(torch.randint(0, 256, (size,), generator=g, dtype=torch.uint8).view(DT[dtype]).view(layers, n_pages, h, page, dh))
    return out


def bits(t):
    return t.contiguous().view(torch.uint8).cpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layers,n_pages,h,page,dh,n", [(1, 2, 1, 8, 32, 1), (2, 30, 3, 16, 64, 11), (3, 9, 5, 64, 128, 4), (1, 700, 1, 16, 64, 333),
                                                      (2, 40, 2, 12, 24, 13)])
def test_pages_are_copied(layers, n_pages, h, page, dh, n, dtype):
    k, v = pools(1, layers, n_pages, h, page, dh, dtype)
    ids = np.random.default_rng(1).permutation(n_pages)
    src, dst = [int(i) for i in ids[:n]], [int(i) for i in ids[n:2 * n]]
    if n > 2:
        src[1] = src[0]            # one page may be copied to several
    kv = Bd.KV.of(k.cuda(), v.cuda())
    Bd.lsk_kv_copy_pages(config(layers, h, dh, page, dtype), kv, src, dst)
    for ref, got in ((k, kv.k_pool), (v, kv.v_pool)):
        ref = ref.clone()
        ref.view(torch.uint8)[:, dst] = ref.view(torch.uint8)[:, src].clone()
        assert torch.equal(bits(got), bits(ref))


def moved(pool, bt, past, paths, page):
    pool = pool.clone()
    flat = pool.view(torch.uint8)
    for b, (p, path) in enumerate(zip(past, paths)):
        for i, node in enumerate(path):
            s, d = p + node, p + i
            if s // page >= bt.shape[1]:
                break
            if not (0 <= bt[b, s // page] < pool.shape[1] and 0 <= bt[b, d // page] < pool.shape[1]):
                continue
            flat[:, bt[b, d // page], :, d % page] = flat[:, bt[b, s // page], :, s % page].clone()
    return pool


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layers,h,page,dh", [(1, 1, 8, 32), (3, 5, 16, 64), (2, 40, 16, 128), (1, 3, 64, 8)])
def test_accepted_rows_move_to_the_end_of_the_context(layers, h, page, dh, dtype):
    rng = np.random.default_rng(2)
    past = [0, 7, page - 1, 3 * page, 100, 5]
    paths = [[0], [], [0, 1, 2], [1, 3, 4, 9, 17, 18, 30], [5], [int(i) for i in np.flatnonzero(rng.random(60) < 0.5)]]
    bt, n_pages = D.page_table(rng, [p + 60 for p in past], page)
    k, v = pools(3, layers, n_pages, h, page, dh, dtype)
    most = max(len(p) for p in paths)
    path = torch.tensor([p + [-5] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    n_path = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    kv = Bd.KV.of(k.cuda(), v.cuda(), torch.from_numpy(bt).cuda(), past)
    Bd.lsk_kv_move_rows(config(layers, h, dh, page, dtype), kv, path, n_path)
    assert torch.equal(bits(kv.k_pool), bits(moved(k, bt, past, paths, page)))
    assert torch.equal(bits(kv.v_pool), bits(moved(v, bt, past, paths, page)))


def test_paths_that_are_none_are_cut():
    """A node twice or out of order, a length beyond the array, a slot beyond the table row, a page outside the pool."""
    page, dh, h = 16, 64, 2
    bt = np.array([[0, 1], [2, 3], [4, 5], [6, 99], [8, 9]], np.int32)
    past = [4, 4, 4, 4, -3]
    k, v = pools(4, 1, 10, h, page, dh, "f16")
    path = torch.tensor([[2, 2, 5, 6], [3, 1, 5, 6], [1, 2, 28, 30], [1, 15, 16, 17], [1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    n_path = torch.tensor([4, 4, 9, 4, 4], dtype=torch.int32, device="cuda")
    kv = Bd.KV.of(k.cuda(), v.cuda(), torch.from_numpy(bt).cuda(), past)
    Bd.lsk_kv_move_rows(config(1, h, dh, page, "f16"), kv, path, n_path)
    # cut after the first node; after the first; before slot 32 (of two pages); rows of page 99 skipped
    want = moved(k, bt[:4], past[:4], [[2], [3], [1, 2], [1, 15, 16, 17]], page)
    assert torch.equal(bits(kv.k_pool), bits(want))


def test_a_captured_move_replays():
    layers, h, page, dh = 2, 4, 16, 64
    rng = np.random.default_rng(5)
    bt, n_pages = D.page_table(rng, [60, 90], page)
    past, paths = [20, 40], [[1, 2, 5], [0, 7]]
    k, v = pools(6, layers, n_pages, h, page, dh, "bf16")
    cfg, kv = config(layers, h, dh, page, "bf16"), Bd.KV.of(k.cuda(), v.cuda(), torch.from_numpy(bt).cuda(), past)
    path, n_path = torch.tensor([[1, 2, 5], [0, 7, 0]], dtype=torch.int32, device="cuda"), torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    used = set(int(i) for b in range(2) for i in bt[b] if i < n_pages)
    spare = [i for i in range(n_pages) if i not in used]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        Bd.lsk_kv_move_rows(cfg, kv, path, n_path)
        Bd.lsk_kv_copy_pages(cfg, kv, [int(bt[0, 1])], [spare[0]])
    for i in range(3):
        k, v = pools(7 + i, layers, n_pages, h, page, dh, "bf16")
        kv.k_pool.copy_(k)
        kv.v_pool.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for ref, got in ((k, kv.k_pool), (v, kv.v_pool)):
            ref = moved(ref, bt, past, paths, page)
            ref.view(torch.uint8)[:, spare[0]] = ref.view(torch.uint8)[:, int(bt[0, 1])].clone()
            assert torch.equal(bits(got), bits(ref))


def test_pools_beyond_32_bits_of_elements():
    """Pages at both ends of pools of more than 2^31 elements: written, attended to, copied and moved."""
    h, page, dh, n_pages = 8, 16, 128, 140000
    assert n_pages * h * page * dh > 2 ** 31
    k = torch.empty(1, n_pages, h, page, dh, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    rng = np.random.default_rng(8)
    bt = np.array([[n_pages - 1, 0, n_pages - 2], [1, n_pages - 3, 2]], np.int32)
    past, counts, T = [30, 17], [3, 4], 7
    qkv = torch.from_numpy(rng.standard_normal((T + 47, 3 * h * dh)).astype(np.float32)).half().cuda()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q, table = torch.empty(T + 47, h * dh, dtype=torch.float16, device="cuda"), i32(bt)
    # the contexts' rows, then the nodes'
    req = [0] * 30 + [1] * 17 + [0] * 3 + [1] * 4
    slot = list(range(30)) + list(range(17)) + [30, 31, 32] + [17, 18, 19, 20]
    Bd.lsk_qk_norm_rope_kv_write(qkv, q, h, h, dh, None, i32(req), k[0], v[0], table, page, slot=i32(slot), norm=False)
    keys, values = qkv[:, h * dh:2 * h * dh].reshape(-1, h, dh), qkv[:, 2 * h * dh:].reshape(-1, h, dh)
    for t in (0, 29, 30, 46, 47, 53):
        at = 0, int(bt[req[t], slot[t] // page]), slice(None), slot[t] % page
        assert torch.equal(k[at], keys[t]) and torch.equal(v[at], values[t])
    o = torch.empty(T, h * dh, dtype=torch.float16, device="cuda")
    chains = [[0], [0, 1], [0, 1, 2], [0], [0, 1], [0, 1, 2], [0, 1, 2, 3]]
    Bd.lsk_attn_tree(q[47:], o, h, h, dh, i32([0, 3, 7]), i32(past), torch.from_numpy(D.mask_words(chains, 1)).cuda(), 4, k[0], v[0],
                     table, page, 30)
    f64 = lambda x: x.cpu().double().numpy()  # noqa: E731
    K, V, Q, O = f64(keys), f64(values), f64(q), f64(o)
    for t in range(T):
        b = 0 if t < 3 else 1
        rows = [r for r in range(47) if req[r] == b] + [47 + (0 if b == 0 else 3) + j for j in chains[t]]
        for head in (0, 7):
            ref, tol = D.attend(Q[47 + t, head * dh:(head + 1) * dh], K[rows, head], V[rows, head], np.arange(len(rows)), "f16", D.HALF["f16"])
            assert (np.abs(O[t, head * dh:(head + 1) * dh] - ref) <= tol).all()
    kv, cfg = Bd.KV.of(k, v, table, past), config(1, h, dh, page, "f16")
    Bd.lsk_kv_copy_pages(cfg, kv, [n_pages - 2, 1], [n_pages - 4, n_pages - 5])
    assert torch.equal(bits(k[0, n_pages - 4]), bits(k[0, n_pages - 2])) and torch.equal(bits(v[0, n_pages - 5]), bits(v[0, 1]))
    Bd.lsk_kv_move_rows(cfg, kv, i32([[2], [3]]), i32([1, 1]))      # slot 32 -> 30, slot 20 -> 17
    assert torch.equal(k[0, 0, :, 14], keys[49]) and torch.equal(v[0, n_pages - 3, :, 1], values[53])
