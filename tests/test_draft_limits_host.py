"""Bounds and refusals of the drafted-token calls that need no GPU: sizes beyond a launch, scratch, arrays that do not fit."""
import pytest
import torch

from paper_2507_21276_amd import binding as Bd

P = 1 << 20   # an address that no call here may reach: every one of them is refused before its launch


def tree(T, B, max_nodes, h, hk, dh, page=16, ptr=P):
    Bd._check(Bd.lib().lsk_attn_tree(ptr, h * dh, Bd.LS_F16, T, B, max_nodes, h, hk, dh, P, P, P, P, P, P, 4, page, 100, 50, ptr, h * dh,
                                     None, 0, None))


def test_more_workgroups_than_a_launch_counts_are_refused():
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 1 << 22, 256, 4, 4, 64)              # 2^22 requests x 4 key heads x 2 blocks of 128 rows
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 1 << 20, 4, 64, 16, 128)             # 2^24 pairs of one block
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 3, 4, 2, 2, 80)                      # the kernel for any size: a workgroup a row and head
    with pytest.raises(Bd.LsError, match="too many"):
        Bd._check(Bd.lib().lsk_tree_index(P, P, P, (1 << 24) - 1, 1 << 24, 4, P, P, P, P, None))


def test_scratch_of_the_tree_attention_is_bounded():
    need = Bd.lib().lsk_attn_tree_scratch_floats
    row = 32 * (128 + 4)
    for args in ((16384, 64, 32, 32, 128, 256, 131072), (4096, 64, 32, 32, 128, 64, 32768), (65536, 256, 32, 32, 128, 256, 131072),
                 (1, 1, 32, 32, 128, 1, 1 << 20)):
        n = need(*args)
        assert n <= 1 << 28 and n % (args[0] * row) == 0 and n != args[0] * row
    assert need(16384, 64, 32, 32, 128, 256, 131072) == 3 * 16384 * row           # as many parts as fit
    assert need(65536, 256, 32, 32, 128, 256, 131072) == 0                        # one part: no partial results
    assert need(4096, 64, 32, 32, 128, 64, 32768) == 8 * 4096 * row               # within the bound: all of them
    # sizes whose kernel does not split a context
    assert need(8, 1, 8, 8, 256, 8, 4096) == need(8, 1, 8, 8, 80, 8, 4096) == 0 < need(8, 1, 8, 8, 128, 8, 4096)


def test_a_short_call_of_the_tree_attention_needs_no_scratch():
    """What the wrapper takes for granted: contexts of up to 512 keys stay whole."""
    need = Bd.lib().lsk_attn_tree_scratch_floats
    for B, hk, g, dh, nodes in ((1, 1, 1, 128, 1), (1, 8, 5, 64, 64), (3, 1, 1, 32, 256), (64, 32, 1, 128, 12)):
        assert need(B * nodes, B, hk * g, hk, dh, nodes, 512 - nodes) == 0
    assert need(1, 1, 1, 1, 128, 1, 512) > 0


# ---- tensors on different devices: every array of a call is looked at before the library sees its address ----------------

class Elsewhere(torch.Tensor):
    """A tensor that says that it lies on another device."""

    def get_device(self):
        return 3


def z(*n, t=torch.int32):
    return torch.zeros(*n, dtype=t)


H, HK, DH, T, B = 4, 2, 64, 5, 2
GAIN, F16, F32 = dict(t=torch.bfloat16), dict(t=torch.float16), dict(t=torch.float32)


def norm():
    return dict(gain_q=z(DH, **GAIN), gain_k=z(DH, **GAIN), pos=z(T), table=z(9, DH // 2, 2, **F32))


def pools():
    return dict(k_pool=z(8, HK, 16, DH, **F16), v_pool=z(8, HK, 16, DH, **F16), block_table=z(B, 4))


CALLS = {
    "lsk_qk_norm_rope": (lambda: dict(qkv=z(T, 8 * DH, **F16), out=z(T, 8 * DH, **F16), **norm()), (H, HK, DH), 2),
    "lsk_qk_norm_rope_bwd": (lambda: dict(dout=z(T, 8 * DH, **F16), qkv=z(T, 8 * DH, **F16), din=z(T, 8 * DH, **F16), **norm(),
                                          dgain_q=z(DH, **F32), dgain_k=z(DH, **F32), alpha=z(1, **F32)), (H, HK, DH), 3),
    "lsk_qk_norm_rope_kv_write": (lambda: dict(qkv=z(T, 8 * DH, **F16), q_out=z(T, H * DH, **F16), req=z(T), slot=z(T), **pools(), **norm()),
                                  dict(n_heads=H, n_kv_heads=HK, head_dim=DH, page_size=16), None),
    "lsk_tree_index": (lambda: dict(parent=z(T), start=z(B + 1), ctx_len=z(B), pos=z(T), slot=z(T), req=z(T), mask=z(T, 1, t=torch.int64)),
                       dict(max_nodes=4), None),
    "lsk_attn_tree": (lambda: dict(q=z(T, H * DH, **F16), o=z(T, H * DH, **F16), start=z(B + 1), ctx_len=z(B), mask=z(T, 1, t=torch.int64),
                                   scratch=z(64, **F32), **pools()),
                      dict(n_heads=H, n_kv_heads=HK, head_dim=DH, max_nodes=4, page_size=16, max_ctx=50), None),
}


@pytest.fixture
def host_calls(monkeypatch):
    """CPU tensors count as the current device's, and the entry points only note that they were reached."""
    reached, real = [], Bd.lib()

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_floats") else lambda *a: reached.append(name) or Bd.LS_OK

    monkeypatch.setattr(Bd, "lib", Lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    return reached


def arguments(name, tensors):
    _, sizes, lead = CALLS[name]
    if lead is None:
        return (), dict(tensors, **sizes)
    names = list(tensors)
    return tuple(tensors[n] for n in names[:lead]) + sizes, {n: tensors[n] for n in names[lead:]}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_one_call_lie_on_one_device(name, host_calls):
    made = CALLS[name][0]()
    args, kw = arguments(name, made)
    getattr(Bd, name)(*args, **kw)
    assert host_calls == [name]
    for which in made:
        args, kw = arguments(name, dict(made, **{which: made[which].as_subclass(Elsewhere)}))
        with pytest.raises(AssertionError, match="device"):
            getattr(Bd, name)(*args, **kw)
        assert host_calls == [name], which


def test_pools_tables_and_paths_lie_on_one_device(host_calls):
    cfg = Bd.make_config(dict(block="gpt", dtype="bf16", n_layers=2, d_model=128, n_heads=2, head_dim=64, d_ff=64, act="gelu_tanh",
                              norm_eps=1e-5, rope_theta=1e4, page_size=16, max_pos=0), mma_dtype="bf16")
    k, path, n_path = z(2, 8, 2, 16, 64, t=torch.bfloat16), z(B, 3), z(B)
    with pytest.raises(AssertionError, match="device"):
        Bd.KV.of(k, k.to("meta"), z(B, 4), [0] * B)
    with pytest.raises(AssertionError, match="device"):
        Bd.KV.of(k, k, z(B, 4).to("meta"), [0] * B)
    kv = Bd.KV.of(k, k.clone(), z(B, 4), [0] * B)
    Bd.lsk_kv_move_rows(cfg, kv, path, n_path)
    Bd.lsk_kv_copy_pages(cfg, kv, [0], [1])
    assert host_calls == ["lsk_kv_move_rows", "lsk_kv_copy_pages"]
    with pytest.raises(AssertionError, match="device"):
        Bd.lsk_kv_move_rows(cfg, kv, path, n_path.as_subclass(Elsewhere))
    for field in ("v_pool", "block_table", "ctx_len"):
        old = getattr(kv, field)
        setattr(kv, field, old.as_subclass(Elsewhere))
        with pytest.raises(AssertionError, match="device"):
            Bd.lsk_kv_move_rows(cfg, kv, path, n_path)
        setattr(kv, field, old)
    kv.v_pool = kv.v_pool.as_subclass(Elsewhere)
    with pytest.raises(AssertionError, match="device"):
        Bd.lsk_kv_copy_pages(cfg, kv, [0], [1])
    assert len(host_calls) == 2


def test_stage_verify_looks_at_its_arrays(host_calls):
    """Parents of another type, arrays shorter than the trees and a table of fewer rows: refused before the library reads them."""
    class Small:
        h, io_torch = None, torch.float32

        class c:
            d_model = 16

    pool = z(1, 8, 1, 16, 16, t=torch.bfloat16)

    def call(X=z(5, 16, **F32), parent=z(5), start=z(3), n=(2, 3), table=z(2, 4), ctx=(0, 0), Y=z(5, 16, **F32)):
        Bd.Stage.stage_verify(Small(), X, parent, start, n, Bd.KV.of(pool, pool, table, ctx), Y, z(64), stream=0)

    call()
    assert host_calls == ["stage_verify"]
    for over, text in ((dict(parent=z(5, t=torch.int64)), "32-bit"), (dict(parent=z(4)), "32-bit"), (dict(start=z(3, t=torch.int64)), "32-bit"),
                       (dict(start=z(2)), "32-bit"), (dict(X=z(4, 16, **F32)), "io type"), (dict(Y=z(5, 15, **F32)), "io type"),
                       (dict(X=z(5, 16, t=torch.bfloat16)), "io type"), (dict(table=z(1, 4)), "page ids"), (dict(ctx=(0,)), "length")):
        with pytest.raises(AssertionError, match=text):
            call(**over)
    for name in ("X", "Y", "parent", "start"):
        there = dict(X=z(5, 16, **F32), Y=z(5, 16, **F32), parent=z(5), start=z(3))[name].as_subclass(Elsewhere)
        with pytest.raises(AssertionError, match="device"):
            call(**{name: there})
    assert len(host_calls) == 1


def test_the_gradients_of_both_gains_need_a_place_each():
    def call(dgq, dgk):
        return Bd.lib().lsk_qk_norm_rope_bwd(P, 384, 2 * P, 384, 3 * P, 384, Bd.LS_F16, 4, 4, 1, 64, 1, P, P, Bd.LS_F16, 1e-5, 64, 0, P, P, 16,
                                             dgq, dgk, 0, None, P, None)

    assert call(4 * P, 4 * P) == Bd.LS_EINVAL and "one place" in Bd.lib().ls_last_error().decode()
