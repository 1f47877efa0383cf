"""The largest calls of the attention over the 4-bit cache: its kernels number the key tiles of all units, and the idle positions in front of each, in
32 bits, so the host refuses a call whose line would not fit (on a host-only context; nothing is launched)."""
import numpy as np
import pytest

import __graft_entry__ as entry

entry.build()

from paper_2609_23900_b200 import binding as B               # noqa: E402

PTR = 4096


def answer(ctx, desc, **kw):
    a = B._Kv4Args()
    v = dict(Hq=900, Hkv=900, dh=128, scale=0.1, n_rows=1, max_pages=193, n_pages=9, page_size=16, pages=PTR, table=PTR, ctx_len=PTR, cache_row=PTR, q=PTR, out=PTR,
             out_dtype=1, work=PTR, work_bytes=1 << 60)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    with pytest.raises(B.LumoError) as e:
        ctx._check(B._lib.lumo_kv4_attention(ctx._h, desc._h, a, 1, None))
    return "large" if "too large" in str(e.value) else "launch" if "host-only" in str(e.value) else str(e.value)


def test_the_line_of_tiles_fits_32_bits():
    ctx = B.Context(-1)
    one = ctx.tree_desc(np.full((65535, 1), -1, dtype=np.int32))
    # 65535 x 900 units of up to 25 tiles, each charged 12 more: 2.18e9 positions
    assert answer(ctx, one) == "large"
    assert answer(ctx, one, Hq=800, Hkv=800) == "launch"                  # 1.94e9
    assert answer(ctx, one, max_pages=160) == "launch"                    # 20 tiles: 1.89e9
    assert answer(ctx, one, Hq=2000, Hkv=2000, max_pages=1) == "large"    # more slots than 32 bits number at the largest split
    few = ctx.tree_desc(np.full((4, 1), -1, dtype=np.int32))
    assert answer(ctx, few, Hq=64, Hkv=64, max_pages=1 << 23, page_size=128) == "large"       # 256 units of 2^23 tiles
    assert answer(ctx, few, Hq=32, Hkv=32, max_pages=1 << 23, page_size=128) == "launch"      # 2^30 and a little
