"""Argument checks of the calls around the paged 4-bit cache, on a host-only context: everything that is wrong with the arguments is refused
before anything else, and arguments that are right get as far as the refusal to launch."""
import ctypes

import numpy as np
import pytest
import torch

import __graft_entry__ as entry

entry.build()

from paper_2609_23900_b200 import binding as B               # noqa: E402

ARG, UNSUPPORTED = 1, 4
PTR = 4096                # any 16-byte aligned address: nothing is launched


@pytest.fixture(scope="module")
def ctx():
    return B.Context(-1)


def code(ctx, call):
    with pytest.raises(B.LumoError) as e:
        ctx._check(call())
    return e.value.code, str(e.value)


def reaches_launch(ctx, call):
    c, msg = code(ctx, call)
    assert c == UNSUPPORTED and "host-only" in msg, msg


def refused(ctx, call, what, want=ARG):
    c, msg = code(ctx, call)
    assert c == want and what in msg, msg


# ---- norm and rotation ----
def qk(**kw):
    a = B._QkArgs()
    v = dict(T=6, Hq=4, Hkv=2, dh=128, dtype=1, rot=64, style=0, axes=1, turns=0, normalise=1, eps=1e-6, weight_offset=0.0, mscale=1.0, q=PTR, k=PTR,
             q_out=PTR, k_out=PTR, inv_freq=PTR, pos=PTR)
    v.update(kw)
    sections = v.pop("section", None)
    for n, x in v.items():
        setattr(a, n, x)
    if sections:
        a.section[:] = sections
    return a


def test_norm_rope_refusals(ctx):
    desc = ctx.tree_desc(np.array([[-1, 0, 0]] * 2, dtype=np.int32))
    call = lambda d=None, **kw: (lambda: B._lib.lumo_qk_norm_rope(ctx._h, d._h if d else None, qk(**kw), None))       # noqa: E731
    reaches_launch(ctx, call())
    reaches_launch(ctx, call(desc, pos=None, ctx_len=PTR))
    reaches_launch(ctx, call(rot=0, inv_freq=None, pos=None))
    reaches_launch(ctx, call(Hkv=0, k=None, k_out=None))
    reaches_launch(ctx, call(axes=3, section=[16, 8, 8]))
    reaches_launch(ctx, call(axes=3, turns=1, section=[12, 10, 10]))
    for kw, what, want in [
            (dict(dh=96), "dh", UNSUPPORTED), (dict(dtype=2), "dtype", UNSUPPORTED), (dict(T=0), "T >= 1", ARG), (dict(Hq=0), "Hq", ARG),
            (dict(Hkv=-1), "Hkv", ARG), (dict(rot=8), "rot", UNSUPPORTED), (dict(rot=144), "rot", UNSUPPORTED), (dict(style=2), "style", ARG),
            (dict(axes=2), "axes", ARG), (dict(eps=-1.0), "eps", ARG), (dict(eps=float("nan")), "eps", ARG), (dict(q=None), "required", ARG),
            (dict(k_out=None), "required", ARG), (dict(inv_freq=None), "inv_freq", ARG), (dict(axes=3, section=[16, 8, 9]), "add up", ARG),
            (dict(axes=3, section=[40, -8, 0]), "sections", ARG), (dict(axes=3, turns=1, section=[0, 16, 16]), "turns", ARG),
            (dict(axes=3, section=[16, 8, 8], pos=None), "pos", ARG), (dict(pos=None), "desc", ARG), (dict(q=PTR + 8), "aligned", ARG),
            (dict(q_stride=500), "strides", ARG), (dict(k_stride=260), "strides", ARG), (dict(q_out_stride=1024), "same stride", ARG)]:
        refused(ctx, call(**kw), what, want)
    refused(ctx, call(desc, pos=None, ctx_len=PTR, T=5), "batch * nodes")
    other = B.Context(-1)
    refused(ctx, call(other.tree_desc(np.array([[-1]], dtype=np.int32))), "another context")


# ---- the 4-bit cache ----
def kv(**kw):
    a = B._Kv4Args()
    v = dict(Hq=8, Hkv=2, dh=128, scale=0.1, n_rows=3, max_pages=10, n_pages=40, page_size=16, k_exp=0, v_exp=0, pages=PTR, table=PTR, ctx_len=PTR,
             cache_row=PTR, q=PTR, k_new=PTR, v_new=PTR, out=PTR, out_dtype=1, n_splits=0, work=PTR, work_bytes=1 << 30)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return a


COMMON = [(dict(dh=64), "dh", UNSUPPORTED), (dict(Hq=7), "multiple", UNSUPPORTED), (dict(Hkv=0), "multiple", UNSUPPORTED),
          (dict(page_size=48), "page_size", UNSUPPORTED), (dict(page_size=256), "page_size", UNSUPPORTED), (dict(page_size=8), "page_size", UNSUPPORTED),
          (dict(n_rows=0), "n_rows", ARG), (dict(max_pages=1 << 27), "positions", ARG), (dict(k_exp=25), "k_exp", ARG), (dict(v_exp=-25), "v_exp", ARG),
          (dict(table=None), "table", ARG), (dict(pages=None), "pages", ARG), (dict(pages=PTR + 8), "aligned", ARG), (dict(kv_stride=255), "strides", ARG),
          (dict(kv_stride=248), "strides", ARG), (dict(q_stride=1028), "strides", ARG)]


def test_kv4_refusals(ctx):
    desc = ctx.tree_desc(np.array([[-1, 0, 0]] * 2, dtype=np.int32), n_slots=5)
    wide = ctx.tree_desc(np.array([[-1, 0, 0]], dtype=np.int32), n_slots=300)
    lib = B._lib

    def layers(*ls):
        return (B._Kv4Args * len(ls))(*ls)

    calls = {
        "write": lambda *ls, d=desc, n=None: (lambda: lib.lumo_kv4_write_tree(ctx._h, d._h, layers(*ls), len(ls) if n is None else n, None)),
        "attention": lambda *ls, d=desc, n=None: (lambda: lib.lumo_kv4_attention(ctx._h, d._h, layers(*ls), len(ls) if n is None else n, None)),
        "publish": lambda *ls, d=desc, n=None, lmax=4: (lambda: lib.lumo_kv4_publish(ctx._h, d._h, layers(*ls), len(ls) if n is None else n, PTR, PTR,
                                                                                      lmax, None, None)),
        "append": lambda *ls, n=None, T=9: (lambda: lib.lumo_kv4_append(ctx._h, layers(*ls), len(ls) if n is None else n, T, PTR, PTR, None, None)),
        "read": lambda *ls, T=9: (lambda: lib.lumo_kv4_read(ctx._h, layers(*ls), T, PTR, PTR, PTR, PTR, None, None)),
    }
    for name, call in calls.items():
        reaches_launch(ctx, call(kv()))
        for kw, what, want in COMMON:
            refused(ctx, call(kv(**kw)), what, want)
        if name != "read":
            reaches_launch(ctx, call(kv(), kv()))
            refused(ctx, call(kv(), kv(n_pages=41)), "share")
            refused(ctx, call(kv(), n=0), "n_layers")
            refused(ctx, call(kv(), n=33), "n_layers")
        if name in ("write", "attention", "publish"):
            refused(ctx, call(kv(ctx_len=None)), "ctx_len")
            refused(ctx, call(kv(max_pages=1, page_size=16), d=ctx.tree_desc(np.array([[-1]], dtype=np.int32), n_slots=17)), "n_slots")
            refused(ctx, call(kv(), d=wide), "256", UNSUPPORTED)
        if name in ("write", "append"):
            refused(ctx, call(kv(k_new=None)), "k_new")
        if name in ("append", "read"):
            refused(ctx, call(kv(), T=0), "T must")
            refused(ctx, call(kv(), T=1 << 29), "T must")
    for kw, what in [(dict(scale=0.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(n_splits=33), "n_splits"), (dict(n_splits=-1), "n_splits"), (dict(q=None), "q and out"),
                     (dict(out=None), "q and out"), (dict(work=None), "work"), (dict(work_bytes=16), "lumo_kv4_work_bytes")]:
        refused(ctx, calls["attention"](kv(**kw)), what)
    refused(ctx, calls["attention"](kv(out_dtype=2)), "out_dtype", UNSUPPORTED)
    for lmax in (0, 257):
        refused(ctx, calls["publish"](kv(), lmax=lmax), "lmax")
    assert ctx.kv4_work_bytes(desc, 8, 3) == 0 and ctx.kv4_work_bytes(desc, 8, 2, 33) == 0


def test_lists_have_one_length(ctx, monkeypatch):
    """Every word a call on a list writes or reads is inside the tensors given: refused before the library is asked."""
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())      # host tensors will do
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)    # noqa: E731
    pages, t = torch.zeros(4, 2, 2, 16 * 72, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.int32)
    layer = B.Kv4Layer(Hq=2, Hkv=2, pages=pages, table=t, page_size=16, status=i32(1))
    out = torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    for kw in (dict(pos=i32(4)), dict(status=i32(4)), dict(status=torch.zeros(5)), dict(pos=i32(5).long())):
        pos, st = kw.get("pos", i32(5)), kw.get("status")
        with pytest.raises(ValueError):
            ctx.kv4_append([layer], i32(5), pos, status=st)
        with pytest.raises(ValueError):
            ctx.kv4_read(layer, i32(5), pos, out, out, status=st)
    for bad in (out[:4], out.float(), out.transpose(0, 1)):
        with pytest.raises(ValueError):
            ctx.kv4_read(layer, i32(5), i32(5), out, bad)
    with pytest.raises(ValueError):
        B.Kv4Layer(Hq=2, Hkv=2, pages=pages, table=t, page_size=16, refs=i32(3))
    tab = B.PageTable(page_size=16, table=t, row_pages=i32(2), refs=i32(4), free_list=i32(4), free_count=i32(1), work=i32(B.pages_work_ints(2, 4)))
    blocks = B.RowBlocks([torch.zeros(4, 8)])
    for call in (lambda st: ctx.pages_fork(tab, i32(2), i32(2), status=st), lambda st: ctx.pages_free(tab, i32(2), status=st),
                 lambda st: ctx.pages_reserve(tab, i32(2), i32(2), add=1, status=st), lambda st: ctx.rows_copy(blocks, i32(2), i32(2), status=st),
                 lambda st: ctx.pages_fork(tab, i32(2), i32(1)), lambda st: ctx.rows_copy(blocks, i32(2), i32(3)),
                 lambda st: ctx.pages_reserve(tab, i32(2), i32(2), end=i32(1)), lambda st: ctx.pages_free(tab, i32(2), keep=i32(1))):
        with pytest.raises(ValueError):
            call(i32(1))


# ---- pages ----
def table(**kw):
    a = B._PageTableArgs()
    ptrs = (ctypes.c_void_p * 2)(PTR, PTR)
    v = dict(n_rows=4, max_pages=8, n_pages=20, page_size=16, table=PTR, row_pages=PTR, refs=PTR, free_list=PTR, free_count=PTR, work=PTR, n_pools=2,
             pools=ctypes.addressof(ptrs), page_bytes=64)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    a._keep = ptrs
    return a


def test_page_refusals(ctx):
    lib = B._lib
    calls = {
        "init": lambda t, n=1: (lambda: lib.lumo_pages_init(ctx._h, t, None)),
        "compact": lambda t, n=1: (lambda: lib.lumo_pages_compact(ctx._h, t, None)),
        "fork": lambda t, n=1: (lambda: lib.lumo_pages_fork(ctx._h, t, PTR, PTR, n, None, None)),
        "free": lambda t, n=1: (lambda: lib.lumo_pages_free(ctx._h, t, PTR, None, n, None, None)),
        "reserve": lambda t, n=1, add=1: (lambda: lib.lumo_pages_reserve(ctx._h, t, PTR, PTR, None, add, n, None, None)),
    }
    for name, call in calls.items():
        reaches_launch(ctx, call(table()))
        reaches_launch(ctx, call(table(n_pools=0, pools=None)))
        for kw in (dict(n_rows=0), dict(max_pages=0), dict(n_pages=0), dict(n_pages=262145), dict(max_pages=262145), dict(page_size=0), dict(page_size=4097)):
            refused(ctx, call(table(**kw)), "need")
        for field in ("table", "row_pages", "refs", "free_list", "free_count", "work"):
            refused(ctx, call(table(**{field: None})), "required")
        refused(ctx, call(table(n_pools=65)), "n_pools")
        refused(ctx, call(table(pools=None)), "n_pools")
        refused(ctx, call(table(page_bytes=24)), "page_bytes")
        if name in ("fork", "free", "reserve"):
            for n in (0, 1025):
                refused(ctx, call(table(), n=n), "1 to 1024")
    refused(ctx, calls["reserve"](table(), add=-1), "add")
    blocks, size = (ctypes.c_void_p * 1)(PTR), (ctypes.c_int64 * 1)(64)
    copy = lambda n=1, rows=4, nb=1, sz=size: (lambda: lib.lumo_rows_copy(ctx._h, blocks, sz, nb, rows, PTR, PTR, n, None, None))    # noqa: E731
    reaches_launch(ctx, copy())
    refused(ctx, copy(n=1025), "1 to 1024")
    refused(ctx, copy(rows=0), "n_rows")
    refused(ctx, copy(nb=65), "n_blocks")
    refused(ctx, copy(sz=(ctypes.c_int64 * 1)(40)), "row_bytes")
    assert B.pages_work_ints(0, 5) == 0 and B.pages_work_ints(3, 5) >= 23


def test_the_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.QkNormRope(q=x, q_out=x, pos=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.QkNormRope(q=x, q_out=x)                                             # not on a GPU
    with pytest.raises(ValueError):
        B.Kv4Layer(Hq=2, Hkv=2, pages=torch.zeros(3, 2, 2, 16 * 64, dtype=torch.uint8), table=torch.zeros(1, 2, dtype=torch.int32), page_size=16)
    with pytest.raises(ValueError):
        B.PageTable(page_size=16, table=torch.zeros(1, 2, dtype=torch.int32), row_pages=torch.zeros(2, dtype=torch.int32), refs=torch.zeros(4, dtype=torch.int32),
                    free_list=torch.zeros(4, dtype=torch.int32), free_count=torch.zeros(1, dtype=torch.int32), work=torch.zeros(99, dtype=torch.int32))
