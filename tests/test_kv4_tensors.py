"""Which tensors the calls around the paged 4-bit cache take, without a GPU: every word that a call reads or writes is inside the tensors it is
given, and nothing is refused that could be passed on.  Host tensors that call themselves CUDA tensors go through the binding; a host-only
context refuses to launch what gets as far as the library."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry

entry.build()

from paper_2609_23900_b200 import binding as B               # noqa: E402


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def gpu(t):
    return t.as_subclass(OnGpu)


def bf16(*shape):
    return gpu(torch.zeros(*shape, dtype=torch.bfloat16))


def i32(*shape):
    return gpu(torch.zeros(*shape, dtype=torch.int32))


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda stream: None)   # (the current stream is a question to the driver)
    return B.Context(-1)


def reaches_launch(call):
    with pytest.raises(B.LumoError, match="host-only"):
        call()


def refused(call, what):
    with pytest.raises(ValueError, match=what):
        call()


def cache(H=2, page=16):
    return dict(Hq=H, Hkv=H, pages=gpu(torch.zeros(4, H, 2, page * 72, dtype=torch.uint8)), table=i32(2, 3), page_size=page)


# ---- tokens that are one and the same row ----
@pytest.mark.parametrize("shape,expanded", [((1, 2, 128), (5, 2, 128)), ((1, 1, 2, 128), (3, 4, 2, 128)), ((1, 4, 2, 128), (3, 4, 2, 128)),
                                            ((3, 1, 2, 128), (3, 4, 2, 128))])
def test_an_expanded_tensor_is_refused(shape, expanded):
    """Its tokens are not heads * dh elements apart (the library takes a stride of 0 for that), so T rows would be read where there is one."""
    x, one = bf16(*expanded), bf16(*shape).expand(*expanded)
    assert isinstance(one, OnGpu) and 0 in one.stride()
    for kw in (dict(q=one, q_out=x), dict(q=x, q_out=one), dict(q=x, q_out=x, k=one, k_out=x), dict(q=x, q_out=x, k=x, k_out=one)):
        refused(lambda: B.QkNormRope(**kw), "tokens")
    for kw in (dict(q=one), dict(k_new=one, v_new=one), dict(k_new=one, v_new=x), dict(k_new=x, v_new=one)):
        refused(lambda: B.Kv4Layer(**cache(), **kw), "tokens")


def test_overlapping_tokens_are_refused():
    part = gpu(torch.zeros(4096, dtype=torch.bfloat16)).as_strided((5, 2, 128), (128, 128, 1))
    refused(lambda: B.QkNormRope(q=part, q_out=bf16(5, 2, 128)), "tokens")
    refused(lambda: B.Kv4Layer(**cache(), k_new=part, v_new=part), "tokens")
    assert B._rows_ptr(bf16(1, 2, 128).expand(1, 2, 128), 2, 128, "q")[1] == 0          # one token: nothing to be apart


# ---- axes of one entry ----
def test_an_axis_of_one_entry_has_no_say_in_the_spacing():
    """Parts of a packed projection of one token a sequence: the stride of the axis of size one says nothing."""
    packed = bf16(3, 6144)                                   # 32 + 8 + 8 heads
    q, k, v = packed[:, :4096].view(3, 1, 32, 128), packed[:, 4096:5120].view(3, 1, 8, 128), packed[:, 5120:].view(3, 1, 8, 128)
    one = packed[:, None].unflatten(-1, (48, 128))[:, :, :32]
    for t, heads in ((q, 32), (k, 8), (v, 8), (one, 32), (packed[:, :4096].view(3, 1, 1, 32, 128), 32), (packed[:, :4096].view(1, 3, 1, 32, 128), 32)):
        assert B._rows_ptr(t, heads, 128, "t") == (t.data_ptr(), 6144)
    assert B._rows_ptr(packed[:1, :4096].view(1, 1, 32, 128), 32, 128, "t")[1] == 0           # one token
    a = B.Kv4Layer(**cache(8), q=None, k_new=k, v_new=v).args
    assert a.kv_stride == 6144
    a = B.QkNormRope(q=q, k=k, q_out=q, k_out=bf16(3, 1, 8, 128)).args
    assert (a.T, a.q_stride, a.k_stride, a.q_out_stride, a.k_out_stride) == (3, 6144, 6144, 6144, 0)
    deep = bf16(2, 5, 6144)[..., :4096].unflatten(-1, (32, 128))
    assert B._rows_ptr(deep, 32, 128, "t")[1] == 6144 and B._rows_ptr(deep[:, None], 32, 128, "t")[1] == 6144


def test_unevenly_spaced_tokens_are_refused():
    x = bf16(2, 5, 6144)[..., :4096].unflatten(-1, (32, 128))
    for t in (x[:, :4], x[:, ::2], x.transpose(0, 1)):
        refused(lambda: B._rows_ptr(t, 32, 128, "t"), "evenly spaced")
    assert B._rows_ptr(x[:, 1:2], 32, 128, "t")[1] == 5 * 6144
    assert B._rows_ptr(x[1:], 32, 128, "t")[1] == 6144


# ---- how many tokens the keys and values hold ----
def test_a_list_is_no_longer_than_the_keys(ctx):
    """Also for layers packed beforehand, and by the layer that has the fewest."""
    seven, five = B.Kv4Layer(**cache(), k_new=bf16(7, 2, 128), v_new=bf16(7, 2, 128)), B.Kv4Layer(**cache(), k_new=bf16(5, 2, 128), v_new=bf16(5, 2, 128))
    uneven = B.Kv4Layer(**cache(), k_new=bf16(9, 2, 128), v_new=bf16(6, 2, 128))
    tree = B.Kv4Layer(**cache(), k_new=bf16(2, 3, 2, 128), v_new=bf16(2, 3, 2, 128))
    for layer, n in ((seven, 7), (five, 5), (uneven, 6), (tree, 6)):
        for layers in ([layer], ctx.pack_kv4([layer])):
            reaches_launch(lambda: ctx.kv4_append(layers, i32(n), i32(n)))
            reaches_launch(lambda: ctx.kv4_append(layers, i32(1), i32(1)))
            refused(lambda: ctx.kv4_append(layers, i32(n + 1), i32(n + 1)), "k_new and v_new")
    shared = [B.Kv4Layer(**{**cache(), "table": seven.tensors["table"]}, k_new=bf16(n, 2, 128), v_new=bf16(n, 2, 128)) for n in (8, 5, 7)]
    for layers in (shared, ctx.pack_kv4(shared)):
        reaches_launch(lambda: ctx.kv4_append(layers, i32(5), i32(5)))
        refused(lambda: ctx.kv4_append(layers, i32(6), i32(6)), "k_new and v_new")
    with pytest.raises(B.LumoError, match="k_new"):
        ctx.kv4_append([B.Kv4Layer(**cache())], i32(1), i32(1))


def test_packed_layers_keep_their_tensors(ctx):
    import weakref
    keys = bf16(3, 2, 128)
    gone = weakref.ref(keys)
    packed = ctx.pack_kv4([B.Kv4Layer(**cache(), k_new=keys, v_new=bf16(3, 2, 128))])
    del keys
    assert gone() is not None and len(packed) == 1
    with pytest.raises(ValueError, match="pack_kv4"):                     # an array of another making says nothing of its tensors
        ctx.kv4_append((B._Kv4Args * 1)(packed[0]), i32(1), i32(1))


# ---- what a call on trees reads and writes ----
def on_trees(**kw):
    """A layer for two trees of three nodes, four query and two KV heads."""
    t = dict(ctx_len=i32(2), cache_row=i32(2), status=i32(2), q=bf16(2, 3, 4, 128), k_new=bf16(2, 3, 2, 128), v_new=bf16(2, 3, 2, 128), out=bf16(2, 3, 4, 128),
             lse=gpu(torch.zeros(2, 3, 4)), work=gpu(torch.zeros(64, dtype=torch.uint8)))
    t.update(kw)
    return B.Kv4Layer(**{**cache(), "Hq": 4}, **t)


def test_the_layers_tensors_hold_what_the_trees_need(ctx):
    desc = ctx.tree_desc(np.array([[-1, 0, 0]] * 2, dtype=np.int32))
    acc, n = i32(2, 2), i32(2)
    write, attend, publish = (lambda l: ctx.kv4_write_tree(desc, l), lambda l: ctx.kv4_attention(desc, l), lambda l: ctx.kv4_publish(desc, l, acc, n))
    kept = gpu(torch.zeros(1 << 20, dtype=torch.uint8))
    for good in (on_trees(work=kept), on_trees(work=kept, status=None, lse=None), on_trees(work=kept, ctx_len=i32(9), out=bf16(7, 4, 128))):
        for call in (write, attend, publish):
            for layers in ([good], ctx.pack_kv4([good])):
                reaches_launch(lambda: call(layers))
    small = {"ctx_len": (i32(1), "seq"), "cache_row": (i32(1), "seq"), "status": (i32(1), "seq"), "q": (bf16(5, 4, 128), "attn"), "out": (bf16(5, 4, 128), "attn"),
             "lse": (gpu(torch.zeros(2, 3, 3)), "attn"), "k_new": (bf16(2, 2, 2, 128), "new"), "v_new": (bf16(5, 2, 128), "new")}
    for name, (t, kind) in small.items():
        layer = on_trees(**{name: t, "work": kept})
        for layers in ([layer], ctx.pack_kv4([layer])):
            for call, own in ((write, "new"), (attend, "attn"), (publish, "publish")):
                if kind in ("seq", own):
                    refused(lambda: call(layers), "too small")
                else:
                    reaches_launch(lambda: call(layers))
    shared = {k: on_trees().tensors[k] for k in ("table", "ctx_len", "cache_row")}
    two = [B.Kv4Layer(Hq=4, Hkv=2, page_size=16, **{**on_trees(work=kept).tensors, **shared, "out": o}) for o in (bf16(2, 3, 4, 128), bf16(2, 2, 4, 128))]
    refused(lambda: attend(two), "too small")


def test_publication_takes_int32_paths_of_every_tree(ctx):
    desc = ctx.tree_desc(np.array([[-1, 0, 0]] * 2, dtype=np.int32))
    layers = ctx.pack_kv4([on_trees()])
    publish = lambda acc, n, out=None: lambda: ctx.kv4_publish(desc, layers, acc, n, out)     # noqa: E731
    reaches_launch(publish(i32(2, 2), i32(2)))
    reaches_launch(publish(i32(5, 3), i32(4), i32(2)))
    for acc, n, out in ((i32(2, 2).long(), i32(2), None), (gpu(torch.zeros(2, 2)), i32(2), None), (i32(2, 2), i32(2).long(), None), (i32(2, 2), i32(2), i32(2).long()),
                        (i32(1, 2), i32(2), None), (i32(4), i32(2), None), (i32(2, 2, 1), i32(2), None), (i32(2, 2), i32(1), None), (i32(2, 2), i32(2), i32(1))):
        refused(publish(acc, n, out), "accepted")


def test_the_rotation_has_a_context_length_for_every_tree(ctx):
    desc = ctx.tree_desc(np.array([[-1, 0, 0]] * 2, dtype=np.int32))
    x, freq = bf16(2, 3, 4, 128), gpu(torch.zeros(64))
    rope = lambda d=desc, **kw: lambda: ctx.qk_norm_rope(B.QkNormRope(q=x, q_out=x, **kw), d)                 # noqa: E731
    reaches_launch(rope(inv_freq=freq, ctx_len=i32(2)))
    reaches_launch(rope(inv_freq=freq, ctx_len=i32(5)))
    reaches_launch(rope(inv_freq=freq, pos=i32(6), ctx_len=i32(1)))       # positions given: lengths are not read
    reaches_launch(rope(inv_freq=freq, pos=i32(6), ctx_len=i32(1), d=None))
    reaches_launch(rope(ctx_len=i32(1)))                                  # the norm alone
    refused(rope(inv_freq=freq, ctx_len=i32(1)), "ctx_len")
    with pytest.raises(B.LumoError, match="ctx_len"):
        rope(inv_freq=freq)()
