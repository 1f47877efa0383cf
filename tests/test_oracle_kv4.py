"""Pins of the 4-bit cache's oracle: number formats against closed forms and torch's e4m3, quantisation against an exhaustive search and error
bounds, the rotation against complex numbers and its invariants, page tables against hand-worked cases and invariants."""
import random

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O


def test_e4m3_values_are_torchs():
    bits = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    ref = bits.view(torch.float8_e4m3fn).double().numpy()
    got = np.array([O.e4m3_value(b) for b in range(256)])
    assert np.array_equal(np.isnan(ref), np.isnan(got)) and np.array_equal(ref[~np.isnan(ref)], got[~np.isnan(ref)])
    assert O.E4M3[-1] == 448.0 and (np.diff(O.E4M3) > 0).all()


def test_rounding_ties_go_to_the_even_code_and_the_largest_is_the_end():
    assert [O.nearest(x, O.E2M1) for x in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 9.0)] == [0, 2, 2, 4, 4, 6, 6, 7]
    assert O.nearest(2.0 ** -10, O.E4M3) == 0 and O.nearest(1.5 * 2.0 ** -9, O.E4M3) == 2 and O.nearest(1e9, O.E4M3) == 126
    x = torch.rand(2000, generator=torch.Generator().manual_seed(3)) * 500
    ref = x.clamp(max=448).to(torch.float8_e4m3fn).view(torch.uint8)
    assert [O.nearest(float(v), O.E4M3) for v in x] == ref.tolist()


@pytest.mark.parametrize("e", [0, 4, -6])
def test_a_block_is_reproduced_within_its_format(e):
    rs = np.random.default_rng(5)
    for _ in range(50):
        x = rs.standard_normal(16) * 2.0 ** rs.integers(-6, 6)
        codes, sb = O.quantise_block(x, e)
        s, top = O.E4M3[sb] * 2.0 ** e, np.abs(x).max()
        # the scale is top / 6 to half a step of e4m3 (448 beyond its end); a code is off by at most half the widest gap (6 - 4), or by the
        # largest's cut
        assert s == 448.0 * 2.0 ** e < top / 6 or abs(s - top / 6) <= max(2.0 ** -4 * s, 2.0 ** (e - 10))
        assert (np.abs(O.block_values(codes, sb, e) - x) <= s * 1.0 + 6 * max(0.0, top / 6 - s) + 1e-12).all()
        if sb < 8:             # below e4m3's normal numbers a step is more than a sixteenth
            continue
        # the largest is 6 scales (top over scale is above 5, where 6 begins), so a second pass over the values changes nothing
        assert (codes & 7).max() == 7
        c2, sb2 = O.quantise_block(O.block_values(codes, sb, e), e)
        assert np.array_equal(O.block_values(c2, sb2, e), O.block_values(codes, sb, e))
    assert (O.quantise(np.zeros(128)) == 0).all()
    bad = np.full(128, 6.0)                                   # scale 1, codes of 6
    bad[17] = np.nan
    assert np.isnan(O.quantise(bad)[16:32]).all() and (O.quantise(bad)[:16] == 6.0).all()
    big = np.ones(128)
    big[3] = np.inf
    assert O.quantise(big)[3] == 2688.0 and (O.quantise(big)[[0, 1, 2]] == 0).all()


def test_values_have_six_significant_bits():
    """What the kernels rest on: a code times a scale is exact in f16 and in bf16."""
    prod = np.unique(np.outer(O.E2M1, O.E4M3).ravel())
    assert np.array_equal(torch.from_numpy(prod).to(torch.float16).double().numpy(), prod)
    assert np.array_equal(torch.from_numpy(prod).to(torch.bfloat16).double().numpy(), prod)


def test_entry_and_cache_values_agree_on_a_hand_made_page():
    P, H = 16, 2
    rs = np.random.default_rng(9)
    pages = rs.integers(0, 120, (5, H, 2, P * 72), dtype=np.uint8)
    table = np.array([[3, 0, -1], [4, 1, 2]])
    k, v = O.cache_values(pages, table, 1, 40, P, k_exp=2, v_exp=-1)
    for p in (0, 15, 16, 39):
        for h in range(H):
            assert np.array_equal(k[p, h], O.entry(pages, table, 1, p, h, 0, P, 2)) and np.array_equal(v[p, h], O.entry(pages, table, 1, p, h, 1, P, -1))
    raw = np.zeros((1, 1, 2, P * 72), np.uint8)
    raw[0, 0, 0, 5 * 64 + 8] = 0x2 | 0xD << 4                 # position 5, elements 16 and 17: 1.0 and -3.0
    raw[0, 0, 0, P * 64 + 5 * 8 + 1] = 0x40                   # its second block's scale: 2.0
    got = O.entry(raw, np.array([[0]]), 0, 5, 0, 0, P)
    assert got[16] == 2.0 and got[17] == -6.0 and np.abs(got).sum() == 8.0


@pytest.mark.parametrize("style", ["half", "pairs"])
def test_rotation_is_a_rotation(style):
    rs = np.random.default_rng(2)
    x, freq = rs.standard_normal((3, 2, 64)), 10.0 ** -np.arange(16.0) / 3
    pos = np.array([[0, 7, 100000]])
    y = O.norm_rope(x, pos, freq, normalise=False, style=style)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
    # products of queries and keys depend on the distance of their positions alone
    q = O.norm_rope(np.repeat(x[:1], 3, 0), np.array([[5, 105, 1005]]), freq, normalise=False, style=style)
    k = O.norm_rope(np.repeat(x[1:2], 3, 0), np.array([[0, 100, 1000]]), freq, normalise=False, style=style)
    dots = (q * k).sum(-1)
    assert np.allclose(dots, dots[0], rtol=1e-9)


def test_norm_and_axes():
    rs = np.random.default_rng(4)
    x, w = rs.standard_normal((2, 3, 64)) * 9, rs.standard_normal(64)
    y = O.norm_rope(x, [[0, 0]], [], weight=w, offset=1.0, eps=0.0)
    assert np.allclose(y / (w + 1.0), x / np.sqrt((x ** 2).mean(-1, keepdims=True)))
    assert O.axis_of(8, [4, 2, 2]) == [0, 0, 0, 0, 1, 1, 2, 2]
    assert O.axis_of(8, [4, 2, 2], turns=True) == [0, 1, 2, 0, 1, 2, 0, 0]
    # three equal axes are one
    freq = np.array([1.0, 0.3, 0.1, 0.03])
    p = [[3, 900]]
    assert np.array_equal(O.norm_rope(x, p * 3, freq, sections=[2, 1, 1], turns=True), O.norm_rope(x, p, freq))


def test_pages_by_hand():
    pool = np.arange(8)
    t = O.Pages(4, 6, 8, 4, [pool])
    assert t.reserve([0], [0], [10]) == [O.SEQ_OK] and t.rows[0] == [0, 1, 2] and t.free[-1] == 3
    assert t.fork([0, 0], [1, 2]) == [O.SEQ_OK, O.SEQ_OK] and t.refs()[:3] == [3, 3, 3]
    # both continuations write position 10: page 2 is copied for each, row 0 keeps it; then page 3 of each
    assert t.reserve([1, 2], [10, 10], [13, 12]) == [0, 0]
    assert t.rows == [[0, 1, 2], [0, 1, 3, 4], [0, 1, 5], []] and t.pools[0].tolist()[3] == 2 and t.pools[0].tolist()[5] == 2
    assert t.refs()[:6] == [3, 3, 1, 1, 1, 1]
    # all three sharers of page 1 listed: the last keeps it
    assert t.reserve([2, 0, 1], [4, 4, 4], [8, 8, 8]) == [0, 0, 0] and t.rows == [[0, 7, 2], [0, 1, 3, 4], [0, 6, 5], []]
    assert t.reserve([3], [0], [4]) == [O.SEQ_NO_PAGES] and t.rows[3] == []
    assert t.release([1, 0], [5, 0]) == [0, 0] and t.rows == [[], [0, 1], [0, 6, 5], []] and t.free == [2, 7, 4, 3]
    assert t.compact() == {5: 2, 6: 3} and t.rows[2] == [0, 3, 2] and t.free == [7, 6, 5, 4]
    assert t.pools[0].tolist()[2] == 2 and t.pools[0].tolist()[3] == 1


@pytest.mark.parametrize("seed", range(4))
def test_pages_never_lose_nor_double_a_page(seed):
    rng = random.Random(seed)
    t = O.Pages(6, 10, 20, 4)
    for _ in range(200):
        what, row = rng.randrange(4), rng.randrange(6)
        if what == 0:
            a = rng.randrange(0, 30)
            t.reserve([row], [a], [a + rng.randrange(10)])
        elif what == 1:
            t.release([row], [rng.randrange(40)])
        elif what == 2:
            t.fork([row], [rng.randrange(6)])
        else:
            t.compact()
        refs = t.refs()
        assert sorted(t.free) == [p for p in range(20) if refs[p] == 0]
        assert all(len(r) == len(set(r)) for r in t.rows)
