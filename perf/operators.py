"""The cache path of drafted tokens, operator by operator: rotary tables, per-head norms of queries and keys with the
rotation (training and page-writing forms), attention of drafted trees over the paged cache, and the moving of cached pages
and rows.

A case's `kind`:

  table  lsk_rope_table: cos / sin of every position and frequency, plain or scaled
  train  lsk_qk_norm_rope and lsk_qk_norm_rope_bwd over packed q | k | v rows; outputs out, din and the gains' gradients
  serve  lsk_qk_norm_rope_kv_write: the rows of a serving batch, K and V to their page slots; outputs q and the pools
  tree   lsk_attn_tree: every request's drafted nodes over its pages; output o
  copy   lsk_kv_copy_pages: whole pages of all layers to other pages; outputs the pools
  step   lsk_tree_index, then for each layer lsk_qk_norm_rope_kv_write and lsk_attn_tree, then lsk_kv_move_rows: a
         verification step and the acceptance of a path of each tree; outputs o of each layer and the pools

Inputs are Gaussian as the stage's workloads have them; gains lie around 1; pages are shuffled.  With `own` false the plain
forms run, otherwise the calls of `binding`.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PAGE = 16


def listed():
    return [
        # the table that a stage of 4352 positions makes once: launch latency
        dict(name="table_4k_plain", kind="table", n_pos=4352, rot=128, theta=10000.0, scaling="plain", factor=1.0),
        # the table of a context stretched eight times
        dict(name="table_128k_parts", kind="table", n_pos=131072, rot=128, theta=10000.0, scaling="parts", factor=8.0),
        # the fp32 stage's micro-batch: the smallest training call
        dict(name="train_tiny_f32", kind="train", dtype="f32", tokens=128, heads=4, kv_heads=4, dim=32, rot=32, layout=0),
        # a wide stage's micro-batch, forward and backward
        dict(name="train_wide_4096", kind="train", dtype="f16", tokens=4096, heads=32, kv_heads=32, dim=128, rot=128, layout=0),
        # one request decoding alone on a small stage
        dict(name="serve_1", kind="serve", dtype="f16", rows="1", past="77", heads=12, kv_heads=12, dim=64, rot=64, layout=0),
        # prompt chunks as the server cuts them, shared key heads, half of each head rotated in neighbouring pairs
        dict(name="serve_chunks_890", kind="serve", dtype="bf16", rows="512,301,77", past="0,512,1030", heads=32, kv_heads=8,
             dim=128, rot=64, layout=1),
        # five drafted tokens of one request on a small stage: per-step latency
        dict(name="tree_1x5", kind="tree", dtype="f16", batch=1, nodes_lo=5, nodes_hi=5, ctx_lo=77, ctx_hi=77, lengths=0,
             heads=12, kv_heads=12, dim=64),
        # the serving batch of uneven contexts with a small draft each
        dict(name="tree_64x8", kind="tree", dtype="f16", batch=64, nodes_lo=4, nodes_hi=12, ctx_lo=128, ctx_hi=2048, lengths=0,
             heads=32, kv_heads=32, dim=128),
        # few requests with long contexts, wide drafts and shared key heads
        dict(name="tree_12x61_long", kind="tree", dtype="bf16", batch=12, nodes_lo=40, nodes_hi=61, ctx_lo=3000, ctx_hi=16001,
             lengths=1, heads=40, kv_heads=8, dim=128),
        # a fork on a small stage: its last page and the next one get copies
        dict(name="copy_2_pages", kind="copy", dtype="bf16", pages=2, layers=6, heads=12, dim=64),
        # half a cache moved to other pages
        dict(name="copy_256_pages", kind="copy", dtype="bf16", pages=256, layers=8, heads=32, dim=128),
        # a whole verification step of two blocks with the acceptance of one branch of each tree
        dict(name="step_32x13", kind="step", dtype="bf16", batch=32, branches=3, depth=4, ctx_lo=64, ctx_hi=1024, lengths=2,
             layers=2, heads=32, kv_heads=32, dim=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges; none needs more than the largest listed one of its kind."""
    kind = rng.choice(["table", "train", "train", "serve", "serve", "tree", "tree", "tree", "copy", "step"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    dim = 32 if dtype == "f32" else rng.choice([64, 128])
    kv_heads = rng.randint(1, 8) if dtype == "f32" else rng.randint(1, 2048 // dim)
    heads = kv_heads * rng.choice([1, 1, 2, 4] if dtype == "f32" else [g for g in (1, 1, 2, 4, 5) if g * kv_heads <= 40])
    if kind == "table":
        scaling = rng.choice(["plain", "linear", "base", "parts"])
        return dict(kind=kind, n_pos=_log_int(rng, 64, 131072), rot=rng.choice([32, 48, 64, 96, 128]),
                    theta=rng.choice([10000.0, 500000.0]), scaling=scaling,
                    factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0]))
    if kind == "train":
        return dict(kind=kind, dtype=dtype, tokens=_log_int(rng, 16, 4096), heads=heads, kv_heads=kv_heads, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim // 4]), layout=rng.randint(0, 1))
    if kind == "serve":
        n = rng.randint(1, 32)
        most = 1 if rng.random() < 0.5 else max(1, 890 // n)
        return dict(kind=kind, dtype=dtype, rows=",".join(str(_log_int(rng, 1, most)) for _ in range(n)),
                    past=",".join(str(rng.choice([0, rng.randint(1, 2048)])) for _ in range(n)), heads=heads,
                    kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim, dim // 2]), layout=rng.randint(0, 1))
    if kind == "tree":
        hi = _log_int(rng, 1, 64)
        ctx = _log_int(rng, 64, 256 if dtype == "f32" else 8192)
        batch = max(1, min(_log_int(rng, 1, 64), (1 << 17) // ctx))
        return dict(kind=kind, dtype=dtype, batch=batch, nodes_lo=rng.randint(1, hi), nodes_hi=hi, ctx_lo=rng.randint(0, ctx),
                    ctx_hi=ctx, lengths=rng.randint(3, 1 << 20), heads=heads, kv_heads=kv_heads, dim=dim)
    if kind == "copy":
        return dict(kind=kind, dtype=dtype, pages=_log_int(rng, 1, 256), layers=rng.randint(1, 8), heads=kv_heads, dim=dim)
    return dict(kind=kind, dtype=dtype, batch=_log_int(rng, 1, 32), branches=rng.randint(1, 4), depth=rng.randint(1, 5),
                ctx_lo=rng.randint(0, 64), ctx_hi=_log_int(rng, 64, 256 if dtype == "f32" else 1024),
                lengths=rng.randint(3, 1 << 20), layers=rng.randint(1, 2), heads=kv_heads, kv_heads=kv_heads, dim=dim)


# ---- what a case fixes beside its inputs --------------------------------------------------------

def _numbers(text):
    return [int(v) for v in text.split(",")]


def _requests(case):
    """(cached tokens, new rows) of every request."""
    if case["kind"] == "serve":
        return _numbers(case["past"]), _numbers(case["rows"])
    rng = random.Random(case["lengths"])
    n = case["batch"]
    past = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(n)]
    if case["kind"] == "step":
        return past, [1 + case["branches"] * case["depth"]] * n
    return past, [rng.randint(case["nodes_lo"], case["nodes_hi"]) for _ in range(n)]


def _parents(case):
    """The drafted trees: parent node of every node (-1: the context's last token), one list a request."""
    new = _requests(case)[1]
    if case["kind"] == "step":   # a root with branches of equal depth, one branch after the other
        d = case["depth"]
        return [[-1] + [0 if i % d == 0 else i for i in range(n - 1)] for n in new]
    rng = random.Random(case["lengths"] + 1)
    # chains with side branches: a node mostly continues the one before it
    return [[i - 1 if rng.random() < 0.6 else rng.randint(-1, i - 1) for i in range(n)] for n in new]


def _ancestors(parents):
    """Nodes that each node sees: itself and its ancestors."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [i])
    return out


def _accepted(case):
    """The accepted path of each tree of a step: the root and the first nodes of the last branch."""
    rng = random.Random(case["lengths"] + 2)
    b, d = case["branches"], case["depth"]
    return [[0] + [1 + (b - 1) * d + k for k in range(rng.randint(0, d))] for _ in range(case["batch"])]


def _frequencies(case):
    rot = case["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    theta = case.get("theta", 10000.0)
    kind, factor = case.get("scaling", "plain"), case.get("factor", 1.0)
    if kind == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * i / rot)
    if kind == "linear":
        f = f / factor
    if kind == "parts":
        turns = 4096 * f / (2 * math.pi)
        g = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = f * (g + (1 - g) / factor)
    return f


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case.get("scaling") == "parts" else 1.0


# ---- inputs -------------------------------------------------------------------------------------

def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 16 + n)
    return g


def _normal(seed, n, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=_gen(seed, n)).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(case, seed):
    """Block table [requests, most pages] of shuffled page ids, and the number of pages with a few spare ones."""
    past, new = _requests(case)
    need = [(p + n + PAGE - 1) // PAGE for p, n in zip(past, new)]
    total = sum(need) + 3
    ids = list(range(total))
    random.Random(seed).shuffle(ids)
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [0] * (max(need) - n))
        at += n
    return table, total


def _pool(seed, n, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=_gen(seed, n))


def _rope_table(case, n_pos):
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * _frequencies(case)[None]
    return torch.stack([ang.cos(), ang.sin()], -1).float().cuda()


def _masks(case, words):
    rows = []
    for parents in _parents(case):
        for seen in _ancestors(parents):
            bits = sum(1 << j for j in seen)
            word = [(bits >> (64 * w)) & ((1 << 64) - 1) for w in range(words)]
            rows.append([w - (1 << 64) if w >> 63 else w for w in word])
    return torch.tensor(rows, dtype=torch.int64, device="cuda")


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    kind = case["kind"]
    st = dict(case=case, kind=kind)
    if kind == "table":
        # the smallest position of a user's table is 0: the seed moves the base a little
        st["theta"] = case["theta"] + float(seed % 64)
        st["table"] = torch.empty(case["n_pos"], case["rot"] // 2, 2, dtype=torch.float32, device="cuda")
        return st
    dt, dh = TORCH[case["dtype"]], case["dim"]
    if kind == "copy":
        n, shape = case["pages"], (case["layers"], 2 * case["pages"] + 1, case["heads"], PAGE, dh)
        ids = list(range(2 * n + 1))
        random.Random(seed).shuffle(ids)
        st.update(k_pool=_pool(seed, 0, shape, dt), v_pool=_pool(seed, 1, shape, dt), src=ids[:n], dst=ids[n:2 * n])
        if own:
            _stage(st, case)
        return st
    h, hk = case["heads"], case["kv_heads"]
    width = (h + 2 * hk) * dh
    if kind != "tree":
        st.update(gain_q=_normal(seed, 2, (dh,), torch.float32 if dt == torch.float32 else torch.bfloat16, 0.1, 1.0),
                  gain_k=_normal(seed, 3, (dh,), torch.float32 if dt == torch.float32 else torch.bfloat16, 0.1, 1.0))
    if kind == "train":
        n = case["tokens"]
        length = max(1, n // 2)   # two sequences
        st.update(qkv=_normal(seed, 0, (n, width), dt), dout=_normal(seed, 1, (n, width), dt, 1e-2),
                  out=torch.empty(n, width, dtype=dt, device="cuda"), din=torch.empty(n, width, dtype=dt, device="cuda"),
                  dgain_q=torch.empty(dh, dtype=torch.float32, device="cuda"),
                  dgain_k=torch.empty(dh, dtype=torch.float32, device="cuda"),
                  pos=_ints([t % length for t in range(n)]), table=_rope_table(case, length))
        return st
    past, new = _requests(case)
    table, n_pages = _pages(case, seed)
    rows = sum(new)
    st.update(ctx=_ints(past), max_ctx=max(past), block_table=_ints(table))
    if kind == "serve":
        st.update(qkv=_normal(seed, 0, (rows, width), dt), q=torch.empty(rows, h * dh, dtype=dt, device="cuda"),
                  pos=_ints([p + i for p, n in zip(past, new) for i in range(n)]),
                  req=_ints([b for b, n in enumerate(new) for _ in range(n)]),
                  table=_rope_table(dict(rot=case["rot"]), max(p + n for p, n in zip(past, new))),
                  k_pool=_pool(seed, 4, (n_pages, hk, PAGE, dh), dt), v_pool=_pool(seed, 5, (n_pages, hk, PAGE, dh), dt))
        return st
    st.update(start=_ints(_starts(new)), new=new, past=past, max_nodes=max(new))
    if kind == "tree":
        st.update(q=_normal(seed, 0, (rows, h * dh), dt), o=torch.empty(rows, h * dh, dtype=dt, device="cuda"),
                  mask=_masks(case, (max(new) + 63) // 64),
                  k_pool=_pool(seed, 4, (n_pages, hk, PAGE, dh), dt), v_pool=_pool(seed, 5, (n_pages, hk, PAGE, dh), dt))
        return st
    layers, paths = case["layers"], _accepted(case)
    most = max(len(p) for p in paths)
    st.update(parent=_ints([p for tree in _parents(case) for p in tree]),
              qkv=_normal(seed, 0, (layers, rows, width), dt), q=torch.empty(rows, h * dh, dtype=dt, device="cuda"),
              o=torch.empty(layers, rows, h * dh, dtype=dt, device="cuda"),
              pos=torch.empty(rows, dtype=torch.int32, device="cuda"), slot=torch.empty(rows, dtype=torch.int32, device="cuda"),
              req=torch.empty(rows, dtype=torch.int32, device="cuda"),
              mask=torch.empty(rows, (max(new) + 63) // 64, dtype=torch.int64, device="cuda"),
              table=_rope_table(dict(rot=dh), max(past) + max(new)),
              path=_ints([p + [0] * (most - len(p)) for p in paths]), n_path=_ints([len(p) for p in paths]), paths=paths,
              k_pool=_pool(seed, 4, (layers, n_pages, hk, PAGE, dh), dt),
              v_pool=_pool(seed, 5, (layers, n_pages, hk, PAGE, dh), dt))
    if own:
        _stage(st, case)
    return st


def _stage(st, case):
    """The descriptors that a program serving from these pools keeps: the stage's configuration and its cache."""
    from paper_2507_21276_amd import binding as B
    f32 = case["dtype"] == "f32"
    cfg = dict(block="gpt", dtype="f32" if f32 else "bf16", n_layers=case["layers"], d_model=case["heads"] * case["dim"],
               n_heads=case["heads"], head_dim=case["dim"], d_ff=64, act="gelu_tanh", norm_eps=1e-5, rope_theta=1e4,
               page_size=PAGE, max_pos=0)
    st["config"] = B.make_config(cfg, mma_dtype=case["dtype"])
    st["kv"] = B.KV.of(st["k_pool"], st["v_pool"], st.get("block_table"), st.get("past"))


# ---- plain forms --------------------------------------------------------------------------------

def _pairs(x, rot, layout):
    """The two elements of every rotated pair, and the rest."""
    r = x[..., :rot]
    if layout == 0:
        return r[..., :rot // 2], r[..., rot // 2:], x[..., rot:]
    return r[..., 0::2], r[..., 1::2], x[..., rot:]


def _join(a, b, rest, layout):
    r = torch.cat([a, b], -1) if layout == 0 else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _plain_norm_rope(x, gain, cs, rot, layout, eps=1e-5):
    """x [T, heads, dh] fp32 -> normalised, scaled, rotated."""
    u = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain
    a, b, rest = _pairs(u, rot, layout)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    return _join(a * c - b * s, a * s + b * c, rest, layout)


def _plain_norm_rope_bwd(dy, x, gain, cs, rot, layout, eps=1e-5):
    a, b, rest = _pairs(dy, rot, layout)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    du = _join(a * c + b * s, b * c - a * s, rest, layout)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    dn = du * gain
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (du * n).sum((0, 1))


def _split(x, h, hk, dh):
    x = x.float()
    return (x[:, :h * dh].reshape(-1, h, dh), x[:, h * dh:(h + hk) * dh].reshape(-1, hk, dh),
            x[:, (h + hk) * dh:].reshape(-1, hk, dh))


def _plain_train(st):
    case = st["case"]
    h, hk, dh, rot, layout = case["heads"], case["kv_heads"], case["dim"], case["rot"], case["layout"]
    gq, gk = st["gain_q"].float(), st["gain_k"].float()
    cs = st["table"][st["pos"].long()]
    q, k, v = _split(st["qkv"], h, hk, dh)
    dq, dk, dv = _split(st["dout"], h, hk, dh)
    dt, flat = st["qkv"].dtype, lambda *p: torch.cat([t.flatten(1) for t in p], 1)
    out = flat(_plain_norm_rope(q, gq, cs, rot, layout), _plain_norm_rope(k, gk, cs, rot, layout), v).to(dt)
    dq, dgq = _plain_norm_rope_bwd(dq, q, gq, cs, rot, layout)
    dk, dgk = _plain_norm_rope_bwd(dk, k, gk, cs, rot, layout)
    return dict(out=out, din=flat(dq, dk, dv).to(dt), dgain_q=dgq, dgain_k=dgk)


def _plain_write(qkv, case, st, rot, layout, pos, slot, req, k_pool, v_pool):
    h, hk, dh = case["heads"], case["kv_heads"], case["dim"]
    cs = st["table"][pos.long()]
    q, k, v = _split(qkv, h, hk, dh)
    page = st["block_table"][req.long(), slot.long() // PAGE].long()
    k_pool[page, :, slot.long() % PAGE] = _plain_norm_rope(k, st["gain_k"].float(), cs, rot, layout).to(k_pool.dtype)
    v_pool[page, :, slot.long() % PAGE] = v.to(v_pool.dtype)
    return _plain_norm_rope(q, st["gain_q"].float(), cs, rot, layout).flatten(1)


def _plain_tree(q, case, st, sees, k_pool, v_pool):
    """q [T, h dh]; sees: [n, n] truth values of each request's nodes."""
    h, hk, dh = case["heads"], case["kv_heads"], case["dim"]
    g, at, out = h // hk, 0, []
    for b, (past, n) in enumerate(zip(st["past"], st["new"])):
        pages = st["block_table"][b, :(past + n + PAGE - 1) // PAGE].long()
        keys = k_pool[pages].float().transpose(0, 1).reshape(hk, -1, dh)[:, :past + n]
        values = v_pool[pages].float().transpose(0, 1).reshape(hk, -1, dh)[:, :past + n]
        rows = q[at:at + n].float().reshape(n, hk, g, dh).permute(1, 0, 2, 3).reshape(hk, n * g, dh)
        s = torch.matmul(rows, keys.transpose(1, 2).contiguous()) / math.sqrt(dh)
        seen = torch.cat([torch.ones(n, past, dtype=torch.bool, device=q.device), sees[b]], 1).repeat_interleave(g, 0)
        s = s.masked_fill(~seen, -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(p / p.sum(-1, keepdim=True), values)
        out.append(o.reshape(hk, n, g, dh).permute(1, 0, 2, 3).reshape(n, h * dh))
        at += n
    return torch.cat(out)


def _plain_step(st):
    case, new = st["case"], st["new"]
    # ancestors: powers of the parent relation, doubled until every depth is covered
    sees, pos, at = [], [], 0
    for b, n in enumerate(new):
        i = torch.arange(n, device="cuda")
        p = st["parent"][at:at + n].long()
        reach = ((p[:, None] == i[None]) | (i[:, None] == i[None])).float()
        for _ in range(max(1, (n - 1).bit_length())):
            reach = (torch.matmul(reach, reach) > 0).float()
        sees.append(reach > 0)
        pos.append(st["ctx"][b] + reach.sum(1).int() - 1)
        at += n
    pos = torch.cat(pos)
    slot = torch.cat([st["ctx"][b] + torch.arange(n, device="cuda", dtype=torch.int32) for b, n in enumerate(new)])
    req = torch.cat([torch.full((n,), b, device="cuda", dtype=torch.int32) for b, n in enumerate(new)])
    out = []
    for l in range(case["layers"]):
        q = _plain_write(st["qkv"][l], case, st, case["dim"], 0, pos, slot, req, st["k_pool"][l], st["v_pool"][l])
        out.append(_plain_tree(q, case, st, sees, st["k_pool"][l], st["v_pool"][l]))
    m = st["path"].shape[1]
    i = torch.arange(m, device="cuda")[None]
    keep = i < st["n_path"][:, None]
    src, dst = (st["ctx"][:, None] + st["path"]).long(), (st["ctx"][:, None] + i).long()
    src, dst = src.where(keep, dst), dst
    b = torch.arange(len(new), device="cuda")[:, None]
    clamp = st["block_table"].shape[1] - 1
    ps, pd = st["block_table"][b, (src // PAGE).clamp(max=clamp)].long(), st["block_table"][b, (dst // PAGE).clamp(max=clamp)].long()
    for pool in (st["k_pool"], st["v_pool"]):
        rows = pool[:, ps[keep], :, (src % PAGE)[keep]]
        pool[:, pd[keep], :, (dst % PAGE)[keep]] = rows
    return dict(o=torch.stack(out).to(st["qkv"].dtype), k_pool=st["k_pool"], v_pool=st["v_pool"])


def _plain(st):
    case, kind = st["case"], st["kind"]
    if kind == "table":
        # the angles of far positions are taken in 64 bits
        f = _frequencies(dict(case, theta=st["theta"])).to("cuda")
        ang = torch.arange(case["n_pos"], dtype=torch.float64, device="cuda")[:, None] * f[None]
        return torch.stack([ang.cos(), ang.sin()], -1).mul(_magnitude(case)).float()
    if kind == "train":
        return _plain_train(st)
    if kind == "serve":
        q = _plain_write(st["qkv"], case, st, case["rot"], case["layout"], st["pos"], st["pos"], st["req"], st["k_pool"],
                         st["v_pool"])
        return dict(q=q.to(st["qkv"].dtype), k_pool=st["k_pool"], v_pool=st["v_pool"])
    if kind == "tree":
        sees, at = [], 0
        for n in st["new"]:
            j = torch.arange(n, device="cuda")
            sees.append(((st["mask"][at:at + n][:, j // 64] >> (j % 64)) & 1) > 0)
            at += n
        return _plain_tree(st["q"], case, st, sees, st["k_pool"], st["v_pool"]).to(st["q"].dtype)
    if kind == "copy":
        src, dst = torch.tensor(st["src"], device="cuda"), torch.tensor(st["dst"], device="cuda")
        for pool in (st["k_pool"], st["v_pool"]):
            pool[:, dst] = pool[:, src]
        return dict(k_pool=st["k_pool"], v_pool=st["v_pool"])
    return _plain_step(st)


# ---- the framework's calls ----------------------------------------------------------------------

def _own(st):
    from paper_2507_21276_amd import binding as B
    case, kind = st["case"], st["kind"]
    if kind == "table":
        code = {"plain": B.LSK_ROPE_PLAIN, "linear": B.LSK_ROPE_LINEAR, "base": B.LSK_ROPE_BASE, "parts": B.LSK_ROPE_PARTS}
        B.lsk_rope_table(st["table"], st["theta"],
                         B.lsk_rope_scaling(code[case["scaling"]], case["factor"], 4096, 32.0, 1.0, _magnitude(case)))
        return st["table"]
    if kind == "copy":
        B.lsk_kv_copy_pages(st["config"], st["kv"], st["src"], st["dst"])
        return dict(k_pool=st["k_pool"], v_pool=st["v_pool"])
    h, hk, dh = case["heads"], case["kv_heads"], case["dim"]
    if kind == "tree":
        B.lsk_attn_tree(st["q"], st["o"], h, hk, dh, st["start"], st["ctx"], st["mask"], st["max_nodes"], st["k_pool"],
                        st["v_pool"], st["block_table"], PAGE, st["max_ctx"])
        return st["o"]
    norm = dict(gain_q=st["gain_q"], gain_k=st["gain_k"], eps=1e-5, table=st["table"])
    if kind == "train":
        B.lsk_qk_norm_rope(st["qkv"], st["out"], h, hk, dh, pos=st["pos"], layout=case["layout"], **norm)
        B.lsk_qk_norm_rope_bwd(st["dout"], st["qkv"], st["din"], h, hk, dh, pos=st["pos"], layout=case["layout"],
                               dgain_q=st["dgain_q"], dgain_k=st["dgain_k"], **norm)
        return dict(out=st["out"], din=st["din"], dgain_q=st["dgain_q"], dgain_k=st["dgain_k"])
    if kind == "serve":
        B.lsk_qk_norm_rope_kv_write(st["qkv"], st["q"], h, hk, dh, st["pos"], st["req"], st["k_pool"], st["v_pool"],
                                    st["block_table"], PAGE, layout=case["layout"], **norm)
        return dict(q=st["q"], k_pool=st["k_pool"], v_pool=st["v_pool"])
    B.lsk_tree_index(st["parent"], st["start"], st["ctx"], st["max_nodes"], st["pos"], st["slot"], st["req"], st["mask"])
    for l in range(case["layers"]):
        B.lsk_qk_norm_rope_kv_write(st["qkv"][l], st["q"], h, hk, dh, st["pos"], st["req"], st["k_pool"][l], st["v_pool"][l],
                                    st["block_table"], PAGE, slot=st["slot"], **norm)
        B.lsk_attn_tree(st["q"], st["o"][l], h, hk, dh, st["start"], st["ctx"], st["mask"], st["max_nodes"], st["k_pool"][l],
                        st["v_pool"][l], st["block_table"], PAGE, st["max_ctx"])
    B.lsk_kv_move_rows(st["config"], st["kv"], st["path"], st["n_path"])
    return dict(o=st["o"], k_pool=st["k_pool"], v_pool=st["v_pool"])


def run(st):
    return _own(st) if own else _plain(st)


# ---- the definition in 64 bits ------------------------------------------------------------------

def _exact_turn(u, cs, rot, layout):
    """u [T, heads, dh] turned by the angles of its rows, element by element of the pairs."""
    y = u.clone()
    half = rot // 2
    first = torch.arange(half, device=u.device) * (2 if layout else 1)
    second = first + (1 if layout else half)
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    y[..., first] = u[..., first] * c - u[..., second] * s
    y[..., second] = u[..., first] * s + u[..., second] * c
    return y


def _exact_unit(x, eps=1e-5):
    return x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + eps).sqrt()


def _exact_heads(x, h, hk, dh):
    return [p.double().reshape(x.shape[0], -1, dh) for p in x.split([h * dh, hk * dh, hk * dh], 1)]


def _exact_tree(q, keys, values, parents, past):
    """One request: q [n, h, dh], keys / values [past + n, hk, dh]; one node after the other."""
    n, h, dh = q.shape
    g = h // keys.shape[1]
    out = torch.empty_like(q)
    for i, seen in enumerate(_ancestors(parents)):
        idx = torch.cat([torch.arange(past), past + torch.tensor(seen)]).to(q.device)
        k, v = keys[idx], values[idx]
        for first in range(0, h, g):
            s = (k[:, first // g] @ q[i, first:first + g].T) * dh ** -0.5
            out[i, first:first + g] = torch.softmax(s, 0).T @ v[:, first // g]
    return out


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    if kind == "table":
        f = _frequencies(dict(case, theta=st["theta"])).tolist()
        cols = []
        p = torch.arange(case["n_pos"], dtype=torch.float64)
        for fi in f:
            cols.append(torch.stack([torch.cos(p * fi), torch.sin(p * fi)], -1))
        return torch.stack(cols, 1) * _magnitude(case)
    if kind == "copy":
        k, v = st["k_pool"], st["v_pool"]
        where = torch.arange(k.shape[1])
        for s, d in zip(st["src"], st["dst"]):
            where[d] = s
        where = where.to(k.device)
        return dict(k_pool=k.double().index_select(1, where), v_pool=v.double().index_select(1, where))
    h, hk, dh = case["heads"], case["kv_heads"], case["dim"]
    if kind == "tree":
        past, new = _requests(case)
        if sum(new) * hk > 100000:   # one node and key head after the other: too long
            return None
        out, at = [], 0
        for b, (p, n, parents) in enumerate(zip(past, new, _parents(case))):
            j = torch.arange(p + n, device="cuda")
            page = st["block_table"][b].long()[j // PAGE]
            keys, values = st["k_pool"][page, :, j % PAGE].double(), st["v_pool"][page, :, j % PAGE].double()
            out.append(_exact_tree(st["q"][at:at + n].double().reshape(n, h, dh), keys, values, parents, p).reshape(n, h * dh))
            at += n
        return torch.cat(out)
    gq, gk = st["gain_q"].double(), st["gain_k"].double()
    if kind == "train":
        rot, layout = case["rot"], case["layout"]
        cs = st["table"][st["pos"].long()]
        back = cs * torch.tensor([1.0, -1.0], device="cuda")
        q, k, v = _exact_heads(st["qkv"], h, hk, dh)
        dq, dk, dv = _exact_heads(st["dout"], h, hk, dh)
        outs, dins, dgains = [], [], []
        for x, dy, g in ((q, dq, gq), (k, dk, gk)):
            n = _exact_unit(x)
            outs.append(_exact_turn(n * g, cs, rot, layout))
            du = _exact_turn(dy, back, rot, layout)
            dgains.append((du * n).flatten(0, 1).sum(0))
            # d(unit)/dx = (I - n n^T / dh) / rms
            rms = (x.square().mean(-1, keepdim=True) + 1e-5).sqrt()
            w = du * g
            dins.append((w - n * (n * w).sum(-1, keepdim=True) / dh) / rms)
        t = q.shape[0]
        return dict(out=torch.cat([outs[0].reshape(t, -1), outs[1].reshape(t, -1), v.reshape(t, -1)], 1),
                    din=torch.cat([dins[0].reshape(t, -1), dins[1].reshape(t, -1), dv.reshape(t, -1)], 1),
                    dgain_q=dgains[0], dgain_k=dgains[1])
    past, new = _requests(case)
    bt = st["block_table"].long()
    if kind == "serve":
        q, k, v = _exact_heads(st["qkv"], h, hk, dh)
        cs = st["table"][st["pos"].long()]
        kp, vp = st["k_pool"].double(), st["v_pool"].double()
        page, at = bt[st["req"].long(), st["pos"].long() // PAGE], st["pos"].long() % PAGE
        kp[page, :, at] = _exact_turn(_exact_unit(k) * gk, cs, case["rot"], case["layout"])
        vp[page, :, at] = v
        return dict(q=_exact_turn(_exact_unit(q) * gq, cs, case["rot"], case["layout"]).flatten(1), k_pool=kp, v_pool=vp)
    if sum(new) * hk * case["layers"] > 100000:
        return None
    kp, vp = st["k_pool"].double(), st["v_pool"].double()
    os = []
    trees = _parents(case)
    pos = [p + len(a) - 1 for p, t in zip(past, trees) for a in _ancestors(t)]
    cs = st["table"][torch.tensor(pos, device="cuda")]
    for l in range(case["layers"]):
        q, k, v = _exact_heads(st["qkv"][l], h, hk, dh)
        q, k = _exact_turn(_exact_unit(q) * gq, cs, dh, 0), _exact_turn(_exact_unit(k) * gk, cs, dh, 0)
        rows, at = [], 0
        for b, (p, n) in enumerate(zip(past, new)):
            j = torch.arange(p + n, device="cuda")
            page = bt[b][j // PAGE]
            kp[l, page[p:], :, j[p:] % PAGE], vp[l, page[p:], :, j[p:] % PAGE] = k[at:at + n], v[at:at + n]
            rows.append(_exact_tree(q[at:at + n], kp[l, page, :, j % PAGE], vp[l, page, :, j % PAGE], trees[b], p).reshape(n, -1))
            at += n
        os.append(torch.cat(rows))
    for b, (p, path) in enumerate(zip(past, st["paths"])):
        for i, node in enumerate(path):
            if i != node:
                s, d = p + node, p + i
                kp[:, bt[b, d // PAGE], :, d % PAGE] = kp[:, bt[b, s // PAGE], :, s % PAGE]
                vp[:, bt[b, d // PAGE], :, d % PAGE] = vp[:, bt[b, s // PAGE], :, s % PAGE]
    return dict(o=torch.stack(os), k_pool=kp, v_pool=vp)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "table":
        n = case["n_pos"] * case["rot"] // 2
        return dict(bytes=8 * n, flops=6 * n)
    e, dh = (4 if case["dtype"] == "f32" else 2), case["dim"]
    if kind == "copy":
        return dict(bytes=2 * 2 * case["pages"] * case["layers"] * case["heads"] * PAGE * dh * e, flops=0)
    h, hk = case["heads"], case["kv_heads"]
    turned, whole = (h + hk) * dh, (h + 2 * hk) * dh
    if kind == "train":
        n = case["tokens"]
        table = (n // 2 + n % 2) * case["rot"] * 4
        return dict(bytes=n * e * (2 * whole + turned + 2 * whole) + 2 * table, flops=n * turned * 24)
    past, new = _requests(case)
    rows = sum(new)
    if kind == "serve":
        return dict(bytes=rows * (2 * whole * e + case["rot"] * 4), flops=rows * turned * 10)
    pairs = sum(p * n + sum(len(a) for a in _ancestors(t)) for p, n, t in zip(past, new, _parents(case)))
    cached = sum(p + n for p, n in zip(past, new)) * 2 * hk * dh * e
    attention = dict(bytes=cached + rows * 2 * h * dh * e, flops=4.0 * pairs * h * dh)
    if kind == "tree":
        return attention
    moved = sum(len([1 for i, n in enumerate(p) if i != n]) for p in _accepted(case)) * 2 * 2 * hk * dh * e
    return dict(bytes=case["layers"] * (attention["bytes"] - rows * h * dh * e + rows * whole * 2 * e + moved),
                flops=case["layers"] * (attention["flops"] + rows * turned * 10.0))
