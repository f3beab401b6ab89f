"""CPU checks of the drafted-token cache path's entry points: every refusal happens on the host, before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2507_21276_amd import binding as Bd

P = 0x10000   # never dereferenced: every case below fails validation on the host
F16, F32 = Bd.LS_F16, Bd.LS_F32


def err():
    return Bd.lib().ls_last_error().decode()


def norm_args(**over):
    a = dict(in_=P, ld_in=384, out=2 * P, ld_out=384, dtype=F16, T=4, h=4, hk=1, dh=64, kind=1, gq=P, gk=P, pdt=F16, eps=1e-5,
             rot=64, layout=0, pos=P, table=P, max_pos=16)
    a.update(over)
    return a


NORM_REFUSALS = [(dict(dtype=7), "dtype"), (dict(T=0), "non-positive"), (dict(h=0), "non-positive"), (dict(hk=-1), "non-positive"),
                 (dict(hk=3), "evenly"), (dict(dh=63), "head_dim"), (dict(dh=514), "head_dim"), (dict(kind=0), "kind"),
                 (dict(kind=-1), "gains without"), (dict(eps=0.0), "eps"), (dict(pdt=9), "gains"), (dict(rot=63), "rotated"),
                 (dict(rot=66), "rotated"), (dict(rot=-2), "rotated"), (dict(pos=None), "rotation without"),
                 (dict(table=None), "rotation without"), (dict(max_pos=0), "rotation without"), (dict(layout=2), "layout"),
                 (dict(in_=None), "null"), (dict(out=None), "null"), (dict(ld_in=383), "apart"), (dict(ld_out=0), "apart"),
                 (dict(out=P, ld_out=392), "in place")]


@pytest.mark.parametrize("over,frag", NORM_REFUSALS)
def test_qk_norm_rope_refuses_bad_arguments(over, frag):
    a = norm_args(**over)
    assert Bd.lib().lsk_qk_norm_rope(*a.values(), None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("over,frag", [(dict(dout=None), "null"), (dict(in_=None), "null"), (dict(din=None), "null"),
                                       (dict(ld_dout=383), "apart"), (dict(ld_din=100), "apart"), (dict(din=3 * P, ld_din=392), "in place"),
                                       (dict(din=P), "forward's input"), (dict(dgk=None), "one of"), (dict(partial=None), "partial"),
                                       (dict(gq=None), "not there"), (dict(T=0), "non-positive"), (dict(rot=3), "rotated")])
def test_qk_norm_rope_bwd_refuses_bad_arguments(over, frag):
    a = dict(dout=3 * P, ld_dout=384, in_=P, ld_in=384, din=2 * P, ld_din=384, dtype=F16, T=4, h=4, hk=1, dh=64, kind=1, gq=P,
             gk=P, pdt=F16, eps=1e-5, rot=64, layout=0, pos=P, table=P, max_pos=16, dgq=P, dgk=P, acc=0, alpha=None, partial=P)
    a.update(over)
    assert Bd.lib().lsk_qk_norm_rope_bwd(*a.values(), None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("over,frag", [(dict(qkv=None), "null"), (dict(q=None), "null"), (dict(req=None), "null"),
                                       (dict(kp=None), "null"), (dict(bt=None), "null"), (dict(pos=None, rot=0), "slots"),
                                       (dict(pages=0), "page counts"), (dict(n_pages=0), "page counts"), (dict(page=0), "page counts"),
                                       (dict(ldq=255), "overlap"), (dict(ld=300), "overlap"), (dict(q=P, ldq=256), "in place")])
def test_qk_norm_rope_kv_write_refuses_bad_arguments(over, frag):
    a = dict(qkv=P, ld=384, q=2 * P, ldq=256, dtype=F16, T=4, h=4, hk=1, dh=64, kind=1, gq=P, gk=P, pdt=F16, eps=1e-5, rot=64,
             layout=0, pos=P, table=P, max_pos=16, req=P, slot=None, kp=P, vp=P, bt=P, pages=2, page=16, n_pages=8)
    a.update(over)
    assert Bd.lib().lsk_qk_norm_rope_kv_write(*a.values(), None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("over,frag", [(dict(table=None), "null"), (dict(n=0), "positions"), (dict(rot=3), "rot_dim"),
                                       (dict(rot=514), "rot_dim"), (dict(rot=0), "rot_dim"), (dict(theta=0.0), "theta"),
                                       (dict(theta=float("inf")), "theta")])
def test_rope_table_refuses_bad_arguments(over, frag):
    a = dict(table=P, n=4, rot=64, theta=1e4)
    a.update(over)
    assert Bd.lib().lsk_rope_table(*a.values(), None, None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("sc,rot,frag", [((9, 2., 0, 0., 0., 1.), 64, "scaling"), ((1, 0.5, 0, 0., 0., 1.), 64, "factor"),
                                         ((2, 2., 0, 0., 0., 1.), 2, "single pair"), ((3, 2., 0, 32., 1., 1.), 64, "parts"),
                                         ((3, 2., 64, 1., 1., 1.), 64, "parts"), ((3, 2., 64, 4., -1., 1.), 64, "parts"),
                                         ((0, 1., 0, 0., 0., 0.), 64, "magnitude")])
def test_rope_table_refuses_bad_scalings(sc, rot, frag):
    s = Bd.lsk_rope_scaling(*sc)
    assert Bd.lib().lsk_rope_table(P, 4, rot, 1e4, C.byref(s), None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("over,frag", [(dict(parent=None), "null"), (dict(mask=None), "null"), (dict(B=0), "non-positive"),
                                       (dict(T=0), "non-positive"), (dict(nodes=0), "max_nodes"), (dict(nodes=257), "max_nodes")])
def test_tree_index_refuses_bad_arguments(over, frag):
    a = dict(parent=P, start=P, ctx=P, B=2, T=8, nodes=8, pos=P, slot=P, req=P, mask=P)
    a.update(over)
    assert Bd.lib().lsk_tree_index(*a.values(), None) == Bd.LS_EINVAL and frag in err()


@pytest.mark.parametrize("over,frag", [(dict(q=None), "null"), (dict(o=None), "null"), (dict(mask=None), "null"),
                                       (dict(dtype=3), "dtype"), (dict(T=0), "non-positive"), (dict(B=-1), "non-positive"),
                                       (dict(pages=0), "non-positive"), (dict(n_pages=0), "non-positive"), (dict(max_ctx=-1), "non-positive"),
                                       (dict(hk=3), "evenly"), (dict(dh=257), "head_dim"), (dict(nodes=300), "max_nodes"),
                                       (dict(ldq=255), "overlap"), (dict(ldo=0), "overlap")])
def test_attn_tree_refuses_bad_arguments(over, frag):
    a = dict(q=P, ldq=256, dtype=F16, T=8, B=2, nodes=8, h=4, hk=1, dh=64, start=P, ctx=P, mask=P, kp=P, vp=P, bt=P, pages=4,
             page=16, n_pages=16, max_ctx=50, o=P, ldo=256, scratch=None, floats=0)
    a.update(over)
    assert Bd.lib().lsk_attn_tree(*a.values(), None) == Bd.LS_EINVAL and frag in err()


def pool_config(**over):
    cfg = dict(block="gpt", dtype="bf16", n_layers=2, d_model=128, n_heads=2, head_dim=64, d_ff=64, act="gelu_tanh", norm_eps=1e-5,
               rope_theta=1e4, page_size=16, max_pos=0)
    cfg.update(over)
    return Bd.make_config(cfg)


def ints(v):
    return (C.c_int32 * max(1, len(v)))(*v)


@pytest.mark.parametrize("src,dst,frag", [([0], [8], "outside"), ([-1], [2], "outside"), ([8], [2], "outside"), ([0, 1], [2, 2], "twice"),
                                          ([0, 2], [2, 3], "read and written"), ([1], [1], "read and written")])
def test_copy_pages_refuses_bad_pairs(src, dst, frag):
    c, kv = pool_config(), Bd.ls_kv(P, P, None, None, None, 8, 0)
    assert Bd.lib().lsk_kv_copy_pages(C.byref(c), C.byref(kv), ints(src), ints(dst), len(src), None) == Bd.LS_EINVAL and frag in err()


def test_page_moves_refuse_bad_pools():
    lib, kv = Bd.lib(), Bd.ls_kv(P, P, P, P, None, 8, 4)
    one = ints([0])
    assert lib.lsk_kv_copy_pages(None, C.byref(kv), one, ints([1]), 1, None) == Bd.LS_EINVAL and "null" in err()
    c = pool_config()
    assert lib.lsk_kv_copy_pages(C.byref(c), C.byref(Bd.ls_kv(P, None, None, None, None, 8, 4)), one, ints([1]), 1, None) == Bd.LS_EINVAL
    assert lib.lsk_kv_copy_pages(C.byref(c), C.byref(kv), one, ints([1]), -1, None) == Bd.LS_EINVAL and "negative" in err()
    assert lib.lsk_kv_copy_pages(C.byref(c), C.byref(kv), None, None, 0, None) == Bd.LS_OK      # nothing to copy
    assert lib.lsk_kv_copy_pages(C.byref(c), C.byref(Bd.ls_kv(P + 8, P, None, None, None, 8, 4)), one, ints([1]), 1, None) == Bd.LS_EINVAL
    assert "16 bytes" in err()
    odd = pool_config(head_dim=4, d_model=8)
    assert lib.lsk_kv_copy_pages(C.byref(odd), C.byref(kv), one, ints([1]), 1, None) == Bd.LS_EINVAL and "16 bytes" in err()
    assert lib.lsk_kv_move_rows(C.byref(c), C.byref(kv), 0, P, 4, P, None) == Bd.LS_EINVAL and "requests" in err()
    assert lib.lsk_kv_move_rows(C.byref(c), C.byref(kv), 2, None, 4, P, None) == Bd.LS_EINVAL and "null" in err()
    assert lib.lsk_kv_move_rows(C.byref(c), C.byref(kv), 2, P, 0, P, None) == Bd.LS_EINVAL and "non-positive" in err()
    assert lib.lsk_kv_move_rows(C.byref(c), C.byref(Bd.ls_kv(P, P, None, P, None, 8, 4)), 2, P, 4, P, None) == Bd.LS_EINVAL
    c.n_layers = 0
    assert lib.lsk_kv_move_rows(C.byref(c), C.byref(kv), 2, P, 4, P, None) == Bd.LS_EINVAL and "non-positive" in err()


def test_scratch_sizes_of_empty_calls_are_zero():
    lib = Bd.lib()
    assert lib.lsk_qk_norm_rope_bwd_partial_floats(0, 4, 4, 64) == 0
    assert lib.lsk_qk_norm_rope_bwd_partial_floats(5, 4, 4, 64) > 0
    assert lib.lsk_attn_tree_scratch_floats(0, 0, 4, 4, 64, 8, 100) == 0


def test_stage_verify_validates_its_arguments_before_any_launch():
    """An fp32 stage without a rotary table allocates nothing on the device."""
    from paper_2507_21276_amd import synth_inputs as S
    lib = Bd.lib()
    c, h = Bd.make_config(S.CONFIGS["tiny_gpt_f32"]), C.c_void_p()
    assert lib.ls_create(C.byref(c), C.byref(h)) == Bd.LS_OK
    ctx = (C.c_int32 * 2)(10, 30)
    kv = Bd.ls_kv(P, P, P, P, C.cast(ctx, C.c_void_p), 8, 3)   # rows of three pages of 16

    def call(n=(1, 2), X=P, parent=P, start=P, kv=kv, Y=P, ws=P, B=None):
        return lib.stage_verify(h, X, parent, start, ints(n), len(n) if B is None else B, C.byref(kv), Y, ws, None)

    assert lib.stage_verify(None, P, P, P, ints([1]), 1, C.byref(kv), P, P, None) == Bd.LS_EINVAL
    assert call() == Bd.LS_ESTATE                      # no parameters bound yet
    assert lib.ls_bind_params(h, P, None) == Bd.LS_OK
    for over in (dict(X=None), dict(parent=None), dict(start=None), dict(Y=None), dict(ws=None)):
        assert call(**over) == Bd.LS_EINVAL and "null" in err()
    assert lib.stage_verify(h, P, P, P, None, 2, C.byref(kv), P, P, None) == Bd.LS_EINVAL and "null" in err()
    for B in (0, -1, 65536):
        assert call(B=B) == Bd.LS_EINVAL and "B must be" in err()
    assert call(n=(0, 1)) == Bd.LS_EINVAL and "nodes" in err()
    assert call(n=(1, 257)) == Bd.LS_EINVAL and "nodes" in err()
    assert call(n=(1, 19)) == Bd.LS_EINVAL and "block table" in err()          # 30 + 19 tokens on three pages
    ctx[0] = -1
    assert call() == Bd.LS_EINVAL and "negative" in err()
    assert call(kv=Bd.ls_kv(P, P, None, P, None, 8, 3)) == Bd.LS_EINVAL and "null field" in err()
    lib.ls_destroy(h)


def test_wrappers_refuse_tables_and_pools_that_are_too_small():
    """Tensors on the CPU: each call is refused before anything looks at the device."""
    z = lambda *n, t=torch.int32: torch.zeros(*n, dtype=t)  # noqa: E731
    q, pool, mask = z(4, 128, t=torch.float16), z(8, 2, 16, 64, t=torch.float16), z(4, 1, t=torch.int64)
    with pytest.raises(AssertionError, match="page ids"):
        Bd.lsk_attn_tree(q, q.clone(), 2, 2, 64, z(4), z(3), mask, 4, pool, pool, z(2, 4), 16, 30)
    pools, c = z(2, 8, 2, 16, 64, t=torch.bfloat16), pool_config(mma_dtype="bf16")
    path, n_path = z(3, 4), z(3)
    with pytest.raises(AssertionError, match="page ids"):
        Bd.lsk_kv_move_rows(c, Bd.KV.of(pools, pools, z(2, 4), [0, 0, 0]), path, n_path)
    with pytest.raises(AssertionError, match="without"):
        Bd.lsk_kv_move_rows(c, Bd.KV.of(pools, pools, z(3, 4)), path, n_path)
    with pytest.raises(AssertionError, match="length"):
        Bd.lsk_kv_move_rows(c, Bd.KV.of(pools, pools, z(3, 4), [0, 0]), path, n_path)
    kv = Bd.KV.of(pools, pools, z(3, 4), [0, 0, 0])
    for other in (dict(n_layers=3), dict(page_size=32), dict(n_heads=4, d_model=256), dict(mma_dtype="f16")):
        with pytest.raises(AssertionError, match="another configuration"):
            Bd.lsk_kv_move_rows(pool_config(**{"mma_dtype": "bf16", **other}), kv, path, n_path)
        with pytest.raises(AssertionError, match="another configuration"):
            Bd.lsk_kv_copy_pages(pool_config(**{"mma_dtype": "bf16", **other}), kv, [0], [1])
    with pytest.raises(AssertionError):
        Bd.KV.of(pools, pools, z(3, 4, t=torch.int64))
