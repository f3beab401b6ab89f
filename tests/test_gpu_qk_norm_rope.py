"""Per-head norms of queries and keys with the rotation: forward, backward, the page-writing form and the tables of angles,
each against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import draft_util as D
from paper_2507_21276_amd import binding as Bd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rand(seed, shape, dtype, std=1.0, mean=0.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(DT[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def heads_of(x, h, hk, dh):
    x = f64(x)
    return (x[:, :h * dh].reshape(-1, h, dh), x[:, h * dh:(h + hk) * dh].reshape(-1, hk, dh), x[:, (h + hk) * dh:])


def rounded_bound(dtype, ref, big):
    """One rounding of the result to its type, and fp32 sums and products whose terms do not exceed `big`."""
    return 1.01 * D.HALF[dtype] * np.abs(ref) + 48 * D.F32 * big + (2.0 ** -25 if dtype == "f16" else 0)


# (T, heads, key heads, head_dim, rotated, layout): single rows, odd sizes, shared key heads, part of the head, sizes that
# the vectorised kernels do not take (head_dim or rot not a multiple of 8), lanes left over in a head
SHAPES = [(1, 1, 1, 2, 2, 0), (1, 12, 12, 64, 64, 0), (5, 3, 3, 32, 32, 1), (7, 8, 2, 128, 128, 0), (7, 8, 2, 128, 64, 1),
          (3, 4, 4, 80, 32, 0), (9, 6, 3, 96, 96, 1), (33, 5, 1, 64, 16, 0), (4, 2, 1, 36, 20, 0), (4, 2, 1, 36, 20, 1),
          (2, 2, 2, 256, 256, 0), (2, 2, 1, 512, 128, 1), (3, 2, 2, 130, 130, 0), (65, 4, 2, 128, 0, 0), (333, 12, 12, 64, 64, 0)]


def case(seed, T, h, hk, dh, rot, layout, dtype, pdtype, norm=True):
    width = (h + 2 * hk) * dh
    n_pos = max(T, 9)
    c = dict(qkv=rand(seed, (T, width), dtype), gq=rand(seed + 1, (dh,), pdtype, 0.2, 1.0), gk=rand(seed + 2, (dh,), pdtype, 0.2, 1.0),
             table=D.table(n_pos, rot) if rot else None, pos=np.random.default_rng(seed).integers(0, n_pos, T).astype(np.int32))
    c["cs"] = c["table"].astype(np.float64)[c["pos"]] if rot else None
    c["kw"] = dict(layout=layout, norm=norm)
    if norm:
        c["kw"].update(gain_q=c["gq"].cuda(), gain_k=c["gk"].cuda())
    if rot:
        c["kw"].update(pos=torch.from_numpy(c["pos"]).cuda(), table=torch.from_numpy(c["table"]).cuda())
    return c


def check_forward(out, c, h, hk, dh, rot, layout, dtype, norm=True):
    q, k, v = heads_of(c["qkv"], h, hk, dh)
    got = heads_of(out, h, hk, dh)
    for g, x, gain in ((got[0], q, c["gq"]), (got[1], k, c["gk"])):
        ref, big = D.norm_rope(x, f64(gain) if norm else None, c["cs"], rot, layout, norm)
        assert (np.abs(g - ref) <= rounded_bound(dtype, ref, big)).all()
    assert (got[2] == v).all()


@pytest.mark.parametrize("dtype,pdtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("T,h,hk,dh,rot,layout", SHAPES)
def test_forward(T, h, hk, dh, rot, layout, dtype, pdtype):
    c = case(11, T, h, hk, dh, rot, layout, dtype, pdtype)
    x = c["qkv"].cuda()
    out = torch.empty_like(x)
    Bd.lsk_qk_norm_rope(x, out, h, hk, dh, **c["kw"])
    check_forward(out, c, h, hk, dh, rot, layout, dtype)
    assert torch.equal(x.cpu(), c["qkv"])
    Bd.lsk_qk_norm_rope(x, x, h, hk, dh, **c["kw"])      # in place: the same values
    assert torch.equal(x, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("off,pad", [(0, 8), (1, 3), (4, 4), (2, 5)])
def test_strided_rows_of_any_alignment(dtype, off, pad):
    T, h, hk, dh, rot = 6, 4, 2, 64, 32
    c = case(12, T, h, hk, dh, rot, 0, dtype, "f32")
    width = (h + 2 * hk) * dh
    big_in = torch.full((T, width + pad), 3.0, dtype=DT[dtype], device="cuda").flatten()
    big_out = torch.full_like(big_in, 7.0)
    big_in, big_out = torch.cat([big_in, big_in[:8]]), torch.cat([big_out, big_out[:8]])
    x = big_in[off:].as_strided((T, width), (width + pad, 1))
    out = big_out[off:].as_strided((T, width), (width + pad, 1))
    x.copy_(c["qkv"])
    Bd.lsk_qk_norm_rope(x, out, h, hk, dh, **c["kw"])
    check_forward(out, c, h, hk, dh, rot, 0, dtype)
    gap = big_out[off:].as_strided((T, pad), (width + pad, 1), off + width)
    assert (gap == 7).all() and (big_out[:off] == 7).all()
    dout, din = big_in, torch.full_like(big_in, 7.0)
    dx = din[off:].as_strided((T, width), (width + pad, 1))
    Bd.lsk_qk_norm_rope_bwd(x, x, dx, h, hk, dh, **c["kw"])
    for g, xx, gain in zip(heads_of(dx, h, hk, dh), heads_of(c["qkv"], h, hk, dh)[:2], (c["gq"], c["gk"])):
        ref, mag, _, _ = D.norm_rope_bwd(xx, xx, f64(gain), c["cs"], rot, 0)
        assert (np.abs(g - ref) <= rounded_bound(dtype, ref, mag)).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("norm,rot", [(False, 64), (True, 0), (False, 0)])
def test_without_norm_gains_or_rotation(layout, norm, rot):
    T, h, hk, dh = 17, 4, 2, 64
    for dtype in ("f32", "bf16"):
        c = case(13, T, h, hk, dh, rot, layout, dtype, "f32", norm)
        x = c["qkv"].cuda()
        out = torch.empty_like(x)
        Bd.lsk_qk_norm_rope(x, out, h, hk, dh, **c["kw"])
        check_forward(out, c, h, hk, dh, rot, layout, dtype, norm)
        if norm:   # gains left out are gains of one
            kw = dict(c["kw"], gain_q=None, gain_k=None)
            one = dict(c["kw"], gain_q=torch.ones(dh, device="cuda"), gain_k=torch.ones(dh, device="cuda"))
            a, b = torch.empty_like(x), torch.empty_like(x)
            Bd.lsk_qk_norm_rope(x, a, h, hk, dh, **kw)
            Bd.lsk_qk_norm_rope(x, b, h, hk, dh, **one)
            assert torch.equal(a, b)
            Bd.lsk_qk_norm_rope(x, a, h, hk, dh, **dict(c["kw"], gain_k=None))
            assert torch.equal(a[:, :h * dh], out[:, :h * dh]) and torch.equal(a[:, h * dh:], b[:, h * dh:])
        else:      # the backward needs no input
            dy = rand(14, x.shape, dtype).cuda()
            dx = torch.empty_like(dy)
            Bd.lsk_qk_norm_rope_bwd(dy, None, dx, h, hk, dh, **c["kw"])
            for g, d in zip(heads_of(dx, h, hk, dh)[:2], heads_of(dy, h, hk, dh)[:2]):
                ref, mag, _, _ = D.norm_rope_bwd(d, None, None, c["cs"], rot, layout, False)
                assert (np.abs(g - ref) <= rounded_bound(dtype, ref, mag)).all()


def test_rotation_alone_is_the_rotary_kernels():
    """Half layout, whole head, no norm: bit for bit what lsk_rope gives."""
    T, h, dh = 37, 6, 128
    x = rand(15, (T, 3 * h * dh), "bf16").cuda()
    pos, table = torch.arange(T, dtype=torch.int32, device="cuda"), torch.from_numpy(D.table(T, dh)).cuda()
    a, b = x.clone(), torch.empty_like(x)
    Bd.lsk_rope(a, h, dh, pos, table, 1.0)
    Bd.lsk_qk_norm_rope(x, b, h, h, dh, norm=False, pos=pos, table=table)
    assert (a.float() - b.float()).abs().max() <= 2 * D.HALF["bf16"] * a.float().abs().max()
    assert (a != b).float().mean() < 1e-3    # a contracted multiply-add may round another way


@pytest.mark.parametrize("dtype,pdtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("T,h,hk,dh,rot,layout", SHAPES + [(2100, 8, 2, 64, 64, 0)])
def test_backward(T, h, hk, dh, rot, layout, dtype, pdtype):
    c = case(16, T, h, hk, dh, rot, layout, dtype, pdtype)
    x, dy = c["qkv"].cuda(), rand(17, c["qkv"].shape, dtype).cuda()
    dx = torch.empty_like(x)
    dgq = torch.full((dh,), 5.0, device="cuda")
    dgk = torch.full((dh,), -3.0, device="cuda")
    alpha = torch.tensor([0.25], device="cuda")
    Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=dgq, dgain_k=dgk, **c["kw"])
    xs, dys, got = heads_of(x, h, hk, dh), heads_of(dy, h, hk, dh), heads_of(dx, h, hk, dh)
    refs = []
    for i, (gain, dg) in enumerate(((c["gq"], dgq), (c["gk"], dgk))):
        ref, mag, rg, mg = D.norm_rope_bwd(dys[i], xs[i], f64(gain), c["cs"], rot, layout)
        assert (np.abs(got[i] - ref) <= rounded_bound(dtype, ref, mag)).all()
        # fp32 sums over rows and heads, in parts of at most a few hundred terms one after the other
        assert (np.abs(f64(dg) - rg) <= (T * h / 1024 + 100) * D.F32 * mg).all()
        refs.append((rg, mg))
    assert (got[2] == dys[2]).all()
    # added to what is there, scaled
    Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=dgq, dgain_k=dgk, accumulate=True, alpha=alpha, **c["kw"])
    for dg, (rg, mg) in zip((dgq, dgk), refs):
        assert (np.abs(f64(dg) - 1.25 * rg) <= 2 * (T * h / 1024 + 100) * D.F32 * mg).all()
    # in place, and without the gains' gradients: the same values
    Bd.lsk_qk_norm_rope_bwd(dy, x, dy, h, hk, dh, **c["kw"])
    assert torch.equal(dy, dx)


def test_backward_agrees_with_differences():
    """Central differences of the forward in fp32: sum(out * dy) along a random direction of the input and of the gains."""
    T, h, hk, dh, rot = 5, 4, 2, 64, 32
    c = case(18, T, h, hk, dh, rot, 1, "f32", "f32")
    x, dy = c["qkv"].cuda(), rand(19, c["qkv"].shape, "f32").cuda()
    dx, dgq, dgk = torch.empty_like(x), torch.empty(dh, device="cuda"), torch.empty(dh, device="cuda")
    Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=dgq, dgain_k=dgk, **c["kw"])
    v, vq, vk = rand(20, x.shape, "f32").cuda(), rand(21, (dh,), "f32").cuda(), rand(22, (dh,), "f32").cuda()

    def value(step):
        out = torch.empty_like(x)
        kw = dict(c["kw"], gain_q=c["kw"]["gain_q"] + step * vq, gain_k=c["kw"]["gain_k"] + step * vk)
        Bd.lsk_qk_norm_rope(x + step * v, out, h, hk, dh, **kw)
        return float((out.double() * dy.double()).sum())

    e = 1e-2
    slope = (8 * (value(e / 2) - value(-e / 2)) - (value(e) - value(-e))) / (6 * e)
    want = float((dx.double() * v.double()).sum() + (dgq.double() * vq.double()).sum() + (dgk.double() * vk.double()).sum())
    # each value carries about sqrt(n) roundings of 2^-24; the differences' own error is of fourth order
    assert abs(slope - want) <= 2e-3 * (1 + abs(want))


def test_positions_outside_the_table_take_its_nearest_row():
    T, h, dh = 4, 2, 64
    x = rand(23, (T, 3 * h * dh), "f32").cuda()
    table = torch.from_numpy(D.table(5, dh)).cuda()
    a, b = torch.empty_like(x), torch.empty_like(x)
    Bd.lsk_qk_norm_rope(x, a, h, h, dh, norm=False, pos=torch.tensor([-7, 0, 5, 1 << 30], dtype=torch.int32, device="cuda"), table=table)
    Bd.lsk_qk_norm_rope(x, b, h, h, dh, norm=False, pos=torch.tensor([0, 0, 4, 4], dtype=torch.int32, device="cuda"), table=table)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("h,hk,dh,rot,layout,page", [(12, 12, 64, 64, 0, 16), (8, 2, 128, 64, 1, 8), (4, 2, 36, 20, 0, 16), (5, 1, 32, 32, 1, 64)])
def test_rows_go_to_their_slots(h, hk, dh, rot, layout, page, dtype):
    rng = np.random.default_rng(24)
    past, new = [0, 30, page - 1, 5], [3, 1, 2, 4]
    T = sum(new) + 2                                 # two padded rows at the end
    bt, n_pages = D.page_table(rng, [p + n for p, n in zip(past, new)], page)
    req = np.array([b for b, n in enumerate(new) for _ in range(n)] + [-1, -1], np.int32)
    slot = np.array([p + i for p, n in zip(past, new) for i in range(n)] + [0, 0], np.int32)
    c = case(25, T, h, hk, dh, rot, layout, dtype, "f32")
    c["kw"].pop("norm")
    pool = lambda: torch.full((n_pages, hk, page, dh), 9.0, dtype=DT[dtype], device="cuda")  # noqa: E731
    kp, vp, q = pool(), pool(), torch.full((T, h * dh), 5.0, dtype=DT[dtype], device="cuda")
    x = c["qkv"].cuda()
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    kw = c["kw"]
    Bd.lsk_qk_norm_rope_kv_write(x, q, h, hk, dh, kw.pop("pos"), dev(req), kp, vp, dev(bt), page, slot=dev(slot), **kw)
    full = torch.cat([q, torch.zeros(T, 2 * hk * dh, dtype=q.dtype, device="cuda")], 1)
    wk, wv = np.full((n_pages, hk, page, dh), 9.0), np.full((n_pages, hk, page, dh), 9.0)
    xq, xk, xv = heads_of(c["qkv"], h, hk, dh)
    live = T - 2
    ref, big = D.norm_rope(xq, f64(c["gq"]), c["cs"], rot, layout)
    assert (np.abs(heads_of(full, h, hk, dh)[0] - ref) <= rounded_bound(dtype, ref, big))[:live].all()
    assert (q[live:] == 5).all()
    ref, big = D.norm_rope(xk, f64(c["gk"]), c["cs"], rot, layout)
    tol = np.zeros_like(wk)
    for t in range(live):
        at = bt[req[t], slot[t] // page], slice(None), slot[t] % page
        wk[at], wv[at], tol[at] = ref[t], xv[t].reshape(hk, dh), rounded_bound(dtype, ref[t], big[t])
    assert (np.abs(f64(kp) - wk) <= tol).all() and (f64(vp) == wv).all()
    assert torch.equal(x.cpu(), c["qkv"])
    # q in place of the projection's rows
    Bd.lsk_qk_norm_rope_kv_write(x, x, h, hk, dh, dev(c["pos"]), dev(req), kp, vp, dev(bt), page, slot=dev(slot), **kw)
    assert torch.equal(x[:live, :h * dh], q[:live]) and torch.equal(x[:, h * dh:].cpu(), c["qkv"][:, h * dh:])
    assert (np.abs(f64(kp) - wk) <= tol).all()


def test_slots_and_pages_that_do_not_exist_are_not_written():
    h, dh, page, T = 2, 64, 16, 5
    x = rand(26, (T, 3 * h * dh), "f16").cuda()
    kp = torch.full((3, h, page, dh), 9.0, dtype=torch.float16, device="cuda")
    vp, q = kp.clone(), torch.empty(T, h * dh, dtype=torch.float16, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    bt = i32(1, -1, 2, 3).reshape(2, 2)     # request 0: page 1, none; request 1: page 2, one beyond the pool
    Bd.lsk_qk_norm_rope_kv_write(x, q, h, h, dh, i32(0, 17, 32, -1, 16), i32(0, 0, 0, 1, 1), kp, vp, bt, page)
    assert (kp[[0, 2]] == 9).all() and (kp[1, :, 1:] == 9).all() and (kp[1, :, 0] != 9).any()
    assert torch.equal(vp[1, :, 0].flatten(), x[0, 2 * h * dh:]) and (vp[1, :, 1:] == 9).all()
    assert torch.isfinite(q.float()).all()


@pytest.mark.parametrize("n_pos,rot", [(1, 2), (5, 64), (17, 48), (4352, 128), (70001, 96)])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "parts"])
def test_tables(n_pos, rot, scaling):
    if scaling == "base" and rot == 2:
        pytest.skip("refused: the base of a single pair")
    theta, factor, mag = 10000.0, 4.0, 1.0
    i = np.arange(rot // 2)
    f = theta ** (-2.0 * i / rot)
    sc = None
    if scaling == "linear":
        f, sc = f / factor, Bd.lsk_rope_scaling(Bd.LSK_ROPE_LINEAR, factor, 0, 0, 0, 1.0)
    elif scaling == "base":
        f, sc = (theta * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot), Bd.lsk_rope_scaling(Bd.LSK_ROPE_BASE, factor, 0, 0, 0, 1.0)
    elif scaling == "parts":
        mag = 1.125
        g = np.clip((2048 * f / (2 * np.pi) - 1) / 31, 0, 1)
        f, sc = f * (g + (1 - g) / factor), Bd.lsk_rope_scaling(Bd.LSK_ROPE_PARTS, factor, 2048, 32.0, 1.0, mag)
    t = torch.empty(n_pos, rot // 2, 2, device="cuda")
    Bd.lsk_rope_table(t, theta, sc)
    a = np.arange(n_pos)[:, None] * f[None]
    ref = mag * np.stack([np.cos(a), np.sin(a)], -1)
    # half a step of fp32, and the 64-bit angle's own rounding: 2^-52 of the angle
    assert (np.abs(f64(t) - ref) <= 1.001 * 2.0 ** -24 * np.abs(ref) + n_pos * 2.0 ** -50).all()


def test_a_captured_training_pass_replays():
    """Forward and backward in a graph, replayed over new inputs with eager work between the replays."""
    T, h, hk, dh = 200, 8, 2, 128
    c = case(27, T, h, hk, dh, dh, 0, "bf16", "f32")
    x, dy = torch.empty_like(c["qkv"]).cuda(), torch.empty_like(c["qkv"]).cuda()
    out, dx = torch.empty_like(x), torch.empty_like(x)
    dgq, dgk = torch.empty(dh, device="cuda"), torch.empty(dh, device="cuda")

    def step(out, dx, dgq, dgk):
        Bd.lsk_qk_norm_rope(x, out, h, hk, dh, **c["kw"])
        Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=dgq, dgain_k=dgk, **c["kw"])

    x.copy_(c["qkv"])
    dy.copy_(rand(28, x.shape, "bf16"))
    step(out, dx, dgq, dgk)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, dx, dgq, dgk)
    for i in range(3):
        x.copy_(rand(30 + i, x.shape, "bf16"))
        dy.copy_(rand(40 + i, x.shape, "bf16"))
        graph.replay()
        e = [torch.empty_like(t) for t in (out, dx, dgq, dgk)]
        step(*e)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(e, (out, dx, dgq, dgk)))


def test_partial_sums_of_a_backward_on_a_stream_that_is_not_the_current_one():
    T, h, hk, dh = 300, 4, 2, 128
    c = case(29, T, h, hk, dh, dh, 0, "bf16", "f32")
    x, dy = c["qkv"].cuda(), rand(50, c["qkv"].shape, "bf16").cuda()
    n = Bd.lib().lsk_qk_norm_rope_bwd_partial_floats(T, h, hk, dh)
    assert n > 0
    want, got, dx = [torch.empty(dh, device="cuda") for _ in range(2)], [torch.empty(dh, device="cuda") for _ in range(2)], torch.empty_like(x)
    Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=want[0], dgain_k=want[1], **c["kw"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2000000)
    Bd.lsk_qk_norm_rope_bwd(dy, x, dx, h, hk, dh, dgain_q=got[0], dgain_k=got[1], stream=side, **c["kw"])
    others = [torch.full((n,), float("nan"), device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    del others
