"""Parity of the paged 4-bit cache (append, tree write, read, attention, publication) with the fp64 oracle, through the C ABI.  The number
formats are compared bit for bit; the tolerance of the attention outputs is derived in tests/kv4_case.py."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from synthetic import workload as W
from tests.harness import ctx
from tests.kv4_case import Kv4Case, bf16

pytestmark = pytest.mark.gpu


def trees(kind, B, N, seed):
    if kind == "paper":
        return [W.tree_paper_geometry() for _ in range(B)]
    if kind == "chain":
        return [W.tree_chain(N) for _ in range(B)]
    if kind == "star":
        return [W.tree_star(N) for _ in range(B)]
    return [W.tree_random(W.IntStream(W.stream_key(seed, b)), N, 8) for b in range(B)]


def special_blocks():
    """Rows of 128 numbers that go wrong easily: ties of codes and scales, tiny and huge blocks, zeros of both signs, infinities, NaN."""
    rows = [np.zeros(128), -np.zeros(128), np.full(128, 2.0 ** -10), np.full(128, 6 * 2.0 ** -10), np.full(128, 9 * 2.0 ** -10), np.full(128, 1e30), np.full(128, -3e38),
            np.full(128, 2688.0), np.full(128, 1e-38)]
    ties = np.tile(np.array([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0]), 8)
    rows += [ties, ties * 1.125, ties * 2.0 ** 6 * 1.75, ties * 2.0 ** -7]
    scale_ties = np.zeros(128)
    scale_ties[::16] = 6 * (1 + (2 * np.arange(8) + 1) / 16.0)            # top / 6 half way between two scales
    rows += [scale_ties, -scale_ties]
    for bad in (np.inf, -np.inf, np.nan):
        r = np.random.default_rng(7).standard_normal(128)
        r[5] = bad
        rows.append(r)
    r = np.random.default_rng(8).standard_normal(128)
    r[16], r[20], r[127] = np.nan, np.inf, 3e38
    rows.append(r)
    return np.array(rows)


@pytest.mark.parametrize("e", [(0, 0), (3, -5), (-24, 24)])
@pytest.mark.parametrize("page", [16, 128])
def test_append_and_read_are_the_oracles_bit_for_bit(page, e):
    """Listed tokens in any order, rows passed over, bad ones refused; keys and values as parts of longer rows; nothing else changes."""
    rs = np.random.default_rng(11)
    H, T, n_pages = 3, 40, 12
    sp = special_blocks()
    x = rs.standard_normal((T, 2 * H, 128)) * 2.0 ** rs.integers(-12, 12, (T, 2 * H, 1))
    x.reshape(-1, 128)[:len(sp)] = sp
    packed = bf16(x.reshape(T, -1))
    k, v = packed[:, :H * 128].unflatten(1, (H, 128)), packed[:, H * 128:].unflatten(1, (H, 128))
    per = 4
    table = torch.from_numpy(rs.permutation(n_pages)[:2 * per].reshape(2, per).astype(np.int32)).cuda()
    table[1, 3] = n_pages                                                 # no such page
    table[0, 3] = -1
    pages = torch.from_numpy(rs.integers(0, 256, (n_pages, H, 2, page * 72), dtype=np.uint8)).cuda()
    before = pages.clone()
    place = rs.permutation(2 * 3 * page)[:T]
    row, pos = (place // (3 * page)).astype(np.int32), (place % (3 * page)).astype(np.int32)
    want = np.zeros(T, np.int32)
    for t, (r, p, st) in {5: (-1, 0, 0), 9: (2, 0, O.SEQ_BAD_ROW), 13: (-2, 4, O.SEQ_BAD_ROW), 17: (0, -1, O.SEQ_BAD_CTX), 21: (1, 4 * page, O.SEQ_BAD_CTX),
                          25: (0, 3 * page, O.SEQ_BAD_PAGE), 29: (1, 3 * page + 5, O.SEQ_BAD_PAGE)}.items():
        row[t], pos[t], want[t] = r, p, st
    row_d, pos_d = torch.from_numpy(row).cuda(), torch.from_numpy(pos).cuda()
    status = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    own = torch.full((T,), -7, dtype=torch.int32, device="cuda")            # a layer's own words are for the calls on trees
    layer = binding.Kv4Layer(Hq=H, Hkv=H, pages=pages, table=table, page_size=page, k_new=k, v_new=v, k_exp=e[0], v_exp=e[1], status=own)
    ctx().kv4_append([layer], row_d, pos_d, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == want.tolist()
    got, expect, tab = pages.cpu().numpy(), before.cpu().numpy(), table.cpu().numpy()
    xq = packed.double().cpu().numpy().reshape(T, 2 * H, 128)
    for t in range(T):
        if row[t] < 0 or want[t]:
            continue
        for h in range(H):
            for w in range(2):
                raw = expect[tab[row[t], pos[t] // page], h, w]
                at = pos[t] % page
                for j in range(8):
                    c, sb = O.quantise_block(xq[t, w * H + h, 16 * j:16 * j + 16], e[w])
                    neg = np.signbit(xq[t, w * H + h, 16 * j:16 * j + 16]) & (sb != 0x7F)
                    c = (c & 7) | (neg.astype(np.uint8) << 3)             # a zero keeps its sign
                    raw[at * 64 + 8 * j:at * 64 + 8 * j + 8] = c[0::2] | (c[1::2] << 4)
                    raw[page * 64 + at * 8 + j] = sb
    assert np.array_equal(got, expect)
    kb, vb = torch.full((T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    status.fill_(-1)
    ctx().kv4_read(layer, row_d, pos_d, kb, vb, status=status)
    torch.cuda.synchronize()
    assert status.tolist() == want.tolist() and set(own.tolist()) == {-7}
    for t in range(T):
        for h in range(H):
            for w, back in enumerate((kb, vb)):
                ref = O.entry(expect, tab, row[t], pos[t], h, w, page, e[w]) if row[t] >= 0 and not want[t] else np.zeros(128)
                assert np.array_equal(back[t, h].double().cpu().numpy(), ref, equal_nan=True), (t, h, w)


@pytest.mark.parametrize("H", [1, 2, 5, 8, 10, 33])
def test_long_lists_of_any_number_of_heads(H):
    """Several tokens a CTA, heads that do not fill its groups of lanes or take several passes: what is read back is what was quantised."""
    rs = np.random.default_rng(H)
    T, page = 1501, 32
    per = -(-T // page)
    table = torch.from_numpy(rs.permutation(per + 3)[None, :per].astype(np.int32)).cuda()
    pages = torch.from_numpy(rs.integers(0, 256, (per + 3, H, 2, page * 72), dtype=np.uint8)).cuda()
    before = pages.clone()
    k, v = (bf16(rs.standard_normal((T, H, 128))) for _ in range(2))
    layer = binding.Kv4Layer(Hq=H, Hkv=H, pages=pages, table=table, page_size=page, k_new=k, v_new=v)
    pos = torch.from_numpy(rs.permutation(T).astype(np.int32)).cuda()
    row = torch.zeros_like(pos)
    row[7] = -1                                                            # passed over
    status = torch.full((T + 5,), -1, dtype=torch.int32, device="cuda")
    ctx().kv4_append([layer], row, pos, status=status)
    kb, vb = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    ctx().kv4_read(layer, row, pos, kb, vb)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * T + [-1] * 5
    for x, back in ((k, kb), (v, vb)):
        pick = np.unique(np.concatenate([[0, 7, T - 1], rs.choice(T, max(8, 300 // H), replace=False)]))
        want = torch.from_numpy(O.quantise(x[pick].double().cpu().numpy()))
        want[list(pick).index(7)] = 0
        assert torch.equal(back[pick].double().cpu(), want)
        assert bool((back[7] == 0).all()) and not bool((back == 7.0).all(-1).any())
    hole = int(pos[7])                                                     # its entry, the last page's rest and the spare pages are as they were
    pg, at = int(table[0, hole // page]), hole % page
    assert torch.equal(pages[pg, :, :, at * 64:at * 64 + 64], before[pg, :, :, at * 64:at * 64 + 64])
    spare = sorted(set(range(per + 3)) - set(table[0].tolist()))
    assert torch.equal(pages[spare], before[spare])
    last, used = int(table[0, -1]), T % page
    assert torch.equal(pages[last, :, :, used * 64:page * 64], before[last, :, :, used * 64:page * 64])
    assert torch.equal(pages[last, :, :, page * 64 + used * 8:], before[last, :, :, page * 64 + used * 8:])


def test_every_quotient_lands_on_the_right_side():
    """All bf16 numbers of four binades against a block maximum that runs through all scales of a binade: codes as by exhaustive search."""
    bits = torch.arange(0x3E00, 0x4000, dtype=torch.int32)               # 0.125 to 2, 512 numbers
    vals = (bits << 16).view(torch.float32).numpy()
    H, T = 1, 16 * len(vals) // 8 // 8
    rows = []
    for i, top in enumerate(np.linspace(6.0, 11.8, 30)):                  # scales 1 to 1.875 and what rounds to them
        top = float(torch.tensor(top).bfloat16())
        for j in range(0, len(vals), 15):
            chunk = vals[j:j + 15] * 4.0
            rows.append(np.concatenate([[top], chunk, np.zeros(15 - len(chunk))]))
    rows = np.array(rows)
    rows = rows[:len(rows) // 8 * 8].reshape(-1, 1, 128)
    T = rows.shape[0]
    pages = torch.zeros(-(-T // 128), 1, 2, 128 * 72, dtype=torch.uint8, device="cuda")
    table = torch.arange(pages.shape[0], dtype=torch.int32, device="cuda")[None]
    x = bf16(rows)
    layer = binding.Kv4Layer(Hq=1, Hkv=1, pages=pages, table=table, page_size=128, k_new=x, v_new=x)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    ctx().kv4_append([layer], torch.zeros_like(pos), pos)
    kb, vb = torch.empty_like(x), torch.empty_like(x)
    ctx().kv4_read(layer, torch.zeros_like(pos), pos, kb, vb)
    torch.cuda.synchronize()
    b = x.double().cpu().numpy().reshape(-1, 16)
    s = O.E4M3[np.array([O.nearest(t, O.E4M3) for t in np.abs(b).max(1) / 6])][:, None]
    d = np.abs(np.abs(b / s)[:, :, None] - O.E2M1)
    place = d.argmin(2)
    tie = (d[..., 1:] == d[..., :-1]) & (d[..., 1:] == d.min(2)[..., None])            # equally near to i and i + 1: the even one
    i = tie.argmax(2)
    place = np.where(tie.any(2), i + i % 2, place)
    ref = (np.sign(b) * O.E2M1[place] * s).reshape(T, 1, 128)
    assert np.array_equal(kb.double().cpu().numpy(), ref) and np.array_equal(vb.double().cpu().numpy(), ref)


CASES = [
    # name, tree kind, B, N, Ns, Hq, Hkv, ctx lengths, page, n_splits
    ("one_token_no_context", "chain", 1, 1, 1, 2, 1, [0], 16, 0),
    ("one_token", "chain", 3, 1, 1, 8, 2, [1, 127, 300], 32, 0),
    ("one_token_padded", "chain", 2, 1, 32, 4, 1, [128, 95], 64, 0),
    ("eight_rows", "random", 2, 2, 2, 8, 2, [255, 256], 128, 0),
    ("nine_rows", "random", 2, 3, 5, 3, 1, [129, 64], 16, 0),
    ("sixteen_rows", "random", 2, 4, 4, 8, 2, [513, 31], 64, 2),
    ("seventeen_rows", "random", 2, 17, 17, 2, 2, [200, 1], 32, 0),
    ("tiny_ctx0", "random", 2, 7, 7, 2, 1, [0, 3], 16, 1),
    ("paper_b1_split4", "paper", 1, 28, 32, 8, 2, [1000], 64, 4),
    ("paper_b3_auto", "paper", 3, 28, 32, 8, 2, [517, 64, 1999], 64, 0),
    ("ragged_tiles", "random", 4, 16, 24, 4, 4, [63, 64, 65, 127], 16, 3),
    ("full_tile_of_rows", "random", 1, 32, 32, 4, 1, [300], 128, 0),
    ("two_row_tiles", "random", 2, 40, 48, 8, 1, [200, 333], 32, 2),
    ("wide_suffix", "star", 1, 200, 256, 2, 2, [130], 64, 2),
    ("deep_chain", "chain", 2, 64, 64, 4, 2, [0, 1], 128, 1),
    ("more_splits_than_tiles", "random", 2, 8, 8, 4, 2, [10, 100], 16, 8),
    ("long_one_token", "chain", 1, 1, 1, 4, 1, [9000], 64, 0),
    ("long_b1_auto", "paper", 1, 28, 32, 4, 1, [9001], 16, 0),
    ("split32", "paper", 1, 28, 32, 4, 1, [5000], 128, 32),
]


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name,kind,B,N,Ns,Hq,Hkv,ctxs,page,splits", CASES, ids=[c[0] for c in CASES])
def test_write_attend_publish_match_the_oracle(name, kind, B, N, Ns, Hq, Hkv, ctxs, page, splits, out):
    c = Kv4Case(trees(kind, B, N, 900), ctxs, Hq=Hq, Hkv=Hkv, page=page, Ns=Ns, n_splits=splits, out=out, seed=len(name))
    before = c.get("pages").copy()
    c.write()
    torch.cuda.synchronize()
    after = c.get("pages")
    for b in range(B):                                                    # the entries, bit for bit in values
        k, v = O.cache_values(after, c.table, c.row[b], c.ctx_len[b] + Ns, page)
        kn, vn = O.quantise(c.d["k_new"][b].double().cpu().numpy()), O.quantise(c.d["v_new"][b].double().cpu().numpy())
        at = c.ctx_len[b] + c.slot[b]
        assert np.array_equal(k[at], kn) and np.array_equal(v[at], vn), "tree write"
    touched = np.zeros((c.n_pages, page), bool)
    for b in range(B):
        for p in c.ctx_len[b] + c.slot[b]:
            touched[c.table[c.row[b], p // page], p % page] = True
    keep = ~touched[:, None, None, :]
    for lo, n in ((0, 64), (page * 64, 8)):
        part = lambda a: a[..., lo:lo + page * n].reshape(c.n_pages, Hkv, 2, page, n)        # noqa: E731
        assert ((part(before) == part(after)).all(-1) | ~keep).all(), "a write outside the tree's entries"
    c.attend()
    torch.cuda.synchronize()
    c.check(name)
    first = c.d["out"].clone()
    c.attend()
    torch.cuda.synchronize()
    assert torch.equal(first, c.d["out"])                                 # bitwise reproducible
    # publication of a path
    rs = np.random.default_rng(3)
    depth = max(len(A.ancestry(c.parent[b], i)) for b in range(B) for i in range(N))
    acc, ln = np.full((B, depth + 2), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        path = A.ancestry(c.parent[b], int(rs.integers(N)))
        acc[b, :len(path)], ln[b] = path, len(path)
    k1, v1 = c.caches()
    k2, v2, ctx2, st = A.kv_publish(c.parent, c.slot, k1, v1, c.ctx_len, c.row, acc, ln)
    ctx_out = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ctx().kv4_publish(c.desc, [c.layer], torch.from_numpy(acc).cuda(), torch.from_numpy(ln).cuda(), ctx_out)
    torch.cuda.synchronize()
    k3, v3 = c.caches()
    assert np.array_equal(k2, k3, equal_nan=True) and np.array_equal(v2, v3, equal_nan=True) and ctx_out.tolist() == ctx2.tolist()
    assert c.get("status").tolist() == [0] * B


@pytest.mark.parametrize("N,G", [(1, 4), (3, 4), (20, 4)], ids=["few_rows", "sixteen_rows", "many_rows"])
def test_bytes_that_nobody_sees_never_reach_an_output(N, G):
    """Other random bytes (NaN scales among them) in padding slots, beyond the suffix, in other rows and spare pages, and in every other branch of one
    node: bitwise the same outputs."""
    c = Kv4Case(trees("random", 2, N, 31), [150, 70], Hq=G * 2, Hkv=2, page=32, Ns=N + 20, seed=5, extra=2)
    c.write()
    c.attend()
    torch.cuda.synchronize()
    out, lse = c.d["out"].clone(), c.d["lse"].clone()
    P, pages = c.page, c.get("pages").copy()
    seen = np.zeros((c.n_pages, P), bool)

    def mark(b, positions):
        for p in positions:
            seen[c.table[c.row[b], p // P], p % P] = True

    def scramble():
        new = np.random.default_rng(77).integers(0, 256, pages.shape, dtype=np.uint8)
        new[..., P * 64:] = 0x7F                                          # every scale a NaN
        codes, scales = np.repeat(seen, 64, axis=1), np.repeat(seen, 8, axis=1)
        m = np.concatenate([codes, scales], axis=1)[:, None, None, :]
        c.d["pages"].copy_(torch.from_numpy(np.where(m, pages, new)))

    for b in range(2):
        mark(b, list(range(c.ctx_len[b])) + [c.ctx_len[b] + s for s in c.slot[b]])
    scramble()
    c.attend()
    torch.cuda.synchronize()
    assert torch.equal(c.d["out"], out) and torch.equal(c.d["lse"], lse)
    seen[:] = False
    i = N - 1
    for b in range(2):
        mark(b, list(range(c.ctx_len[b])) + [c.ctx_len[b] + c.slot[b][a] for a in A.ancestry(c.parent[b], i)])
    scramble()                                                            # now the other branches hold NaN too
    c.attend()
    torch.cuda.synchronize()
    assert torch.equal(c.d["out"][:, i], out[:, i]) and torch.equal(c.d["lse"][:, i], lse[:, i])


@pytest.mark.parametrize("N,G", [(2, 4), (4, 4), (24, 2)], ids=["few_rows", "sixteen_rows", "many_rows"])
def test_a_nan_reaches_those_who_see_it(N, G):
    """NaN keys make whole outputs NaN, a NaN block of values sixteen numbers of them, for the nodes that see the position and no others."""
    c = Kv4Case([W.tree_star(N) if N > 2 else [-1, -1] for _ in range(3)], [140, 40, 257], Hq=G, Hkv=1, page=16, Ns=N + 3, seed=6)
    c.write()
    ent = {0: 1, 1: 0}
    v = c.d["v_new"]
    v[0, 1, 0, 40] = float("nan")                                         # sequence 0: values of node 1, block 2
    c.d["k_new"][1, N - 1, 0, 3] = float("nan")                           # sequence 1: keys of the last node
    c.write()
    P, tab = c.page, c.table
    pos = 5                                                               # sequence 2: context values, block 7, and that is seen by all
    c.d["pages"][int(tab[c.row[2], pos // P]), 0, 1, P * 64 + (pos % P) * 8 + 7] = 0xFF
    c.attend()
    torch.cuda.synchronize()
    out, lse = c.get("out"), c.get("lse")
    want, want_lse = np.zeros(out.shape, bool), np.zeros(lse.shape, bool)
    for i in range(N):
        if 1 in A.ancestry(c.parent[0], i):
            want[0, i, :, 32:48] = True
        if N - 1 in A.ancestry(c.parent[1], i):
            want[1, i], want_lse[1, i] = True, True
    want[2, :, :, 112:128] = True
    assert np.array_equal(np.isnan(out), want) and np.array_equal(np.isnan(lse), want_lse)
    ref, rl, bound = c.reference()
    good = ~want & ~np.isnan(ref)
    good[2, :, :, :112] = True
    good[1] &= ~want[1]
    err = np.abs(out - ref)[good & ~np.isnan(ref)]
    assert (err <= (2.0 ** -11 * bound + 2e-5 * (1 + np.abs(ref)))[good & ~np.isnan(ref)]).all()
    assert c.get("status").tolist() == [0, 0, 0]


def test_bad_sequences_are_left_alone_and_the_others_served():
    c = Kv4Case(trees("random", 6, 6, 8), [100, 40, 70, 90, 33, 20], Hq=8, Hkv=2, page=16, Ns=8, seed=9, n_splits=0)
    row, ctx_len = c.d["row"], c.d["ctx_len"]
    row[1], ctx_len[2] = 7, -1
    ctx_len[3] = c.table.shape[1] * 16 - 7
    c.d["table"][int(c.row[4]), 2] = -1                                   # context page, and the first of the suffix
    c.d["table"][int(c.row[0]), 100 // 16] = c.n_pages
    before = c.d["pages"].clone()
    want = [O.SEQ_BAD_PAGE, O.SEQ_BAD_ROW, O.SEQ_BAD_CTX, O.SEQ_BAD_CTX, O.SEQ_BAD_PAGE, 0]
    c.write()
    torch.cuda.synchronize()
    assert c.get("status").tolist() == want
    changed = (before != c.d["pages"]).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= set(c.table[c.row[5]].tolist())
    c.d["status"].fill_(-1)
    c.attend()
    torch.cuda.synchronize()
    assert c.get("status").tolist() == want
    out, lse = c.get("out"), c.get("lse")
    assert (out[:5] == 0).all() and (lse[:5] == 0).all()
    k, v = O.cache_values(c.get("pages"), c.table, c.row[5], 28, 16)
    kk, vv = np.zeros((1, 28, 2, 128)), np.zeros((1, 28, 2, 128))
    kk[0], vv[0] = k, v
    ref, rl = A.tree_attention(c.parent[5:], c.slot[5:], c.get("q")[5:], kk, vv, [20], [0], c.scale)
    assert np.abs(out[5] - ref[0]).max() < 2e-3 and np.abs(lse[5] - rl[0]).max() < 1e-4
    c.d["status"].fill_(-1)
    acc = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    before, n = c.d["pages"].clone(), torch.ones(6, dtype=torch.int32, device="cuda")
    ctx_out = torch.full((6,), -5, dtype=torch.int32, device="cuda")
    ctx().kv4_publish(c.desc, [c.layer], acc, n, ctx_out)
    torch.cuda.synchronize()
    assert c.get("status").tolist() == want and ctx_out.tolist() == ctx_len.tolist()[:5] + [21]
    changed = (before != c.d["pages"]).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= set(c.table[c.row[5]].tolist())


@pytest.mark.parametrize("N", [1, 4, 12])
@pytest.mark.parametrize("ctx_len", [100, 200, 330, 700, 1500])
def test_a_page_missing_at_the_very_end(N, ctx_len):
    """The last tile's page is the one that is missing, every call in a row: no output and no status goes by what was known before it."""
    c = Kv4Case(trees("random", 2, N, 3), [ctx_len, ctx_len // 2], Hq=8, Hkv=2, page=16, seed=31, n_splits=1)
    c.write()
    last = (ctx_len + c.Ns - 1) // 16
    keep = int(c.table[c.row[0], last])
    table, want = c.d["table"], None
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    c.attend()
    torch.cuda.synchronize()
    c.check("whole")
    want = c.d["out"].clone()
    for _ in range(30):
        table[int(c.row[0]), last] = -1
        c.attend()
        wrong += (c.d["out"][0] != 0).sum() + (c.d["lse"][0] != 0).sum() + (c.d["out"][1] != want[1]).sum()
        wrong += (c.d["status"] != torch.tensor([O.SEQ_BAD_PAGE, 0], dtype=torch.int32, device="cuda")).sum()
        table[int(c.row[0]), last] = keep
        c.attend()
        wrong += (c.d["out"] != want).sum() + (c.d["status"] != 0).sum()
    torch.cuda.synchronize()
    assert int(wrong) == 0


def test_publication_refuses_what_is_no_path():
    c = Kv4Case([[-1, 0, 1, 0]] * 5, [20] * 5, Hq=2, Hkv=1, page=16, seed=4)
    c.write()
    torch.cuda.synchronize()
    before = c.d["pages"].clone()
    acc = torch.tensor([[0, 1, 2], [1, 2, 0], [0, 2, 1], [0, 9, 0], [0, 1, 2]], dtype=torch.int32, device="cuda")
    n = torch.tensor([4, 2, 3, 2, -1], dtype=torch.int32, device="cuda")
    ctx().kv4_publish(c.desc, [c.layer], acc, n)
    torch.cuda.synchronize()
    assert c.get("status").tolist() == [1, 3, 4, 2, 1] and torch.equal(before, c.d["pages"])


def test_writes_keep_off_shared_pages():
    c = Kv4Case(trees("random", 2, 4, 3), [20, 50], Hq=2, Hkv=1, page=16, seed=12)
    refs = torch.ones(c.n_pages, dtype=torch.int32, device="cuda")
    refs[int(c.table[c.row[0], 1])] = 2
    c.layer.args.refs = refs.data_ptr()
    before = c.d["pages"].clone()
    c.write()
    torch.cuda.synchronize()
    assert c.get("status").tolist() == [O.SEQ_BAD_PAGE, 0]
    changed = (before != c.d["pages"]).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= set(c.table[c.row[1]].tolist()) and changed
    c.attend()                                                            # reading shared pages is what they are for
    torch.cuda.synchronize()
    assert c.get("status").tolist() == [0, 0]


@pytest.mark.parametrize("gain", [0.0, 2.0 ** -40, 2.0 ** -12, 2.0 ** 6])
def test_queries_of_any_size(gain):
    c = Kv4Case(trees("random", 2, 5, 21), [130, 77], Hq=4, Hkv=2, page=32, seed=13, q_gain=gain)
    c.write()
    c.attend()
    torch.cuda.synchronize()
    c.check(str(gain))


def test_queries_as_parts_of_longer_rows_and_scaled_caches():
    c = Kv4Case(trees("random", 2, 9, 22), [130, 77], Hq=8, Hkv=2, page=32, seed=14, k_exp=-4, v_exp=5)
    packed = torch.zeros(2, 9, 12 * 128, dtype=torch.bfloat16, device="cuda")
    packed[..., :1024] = c.d["q"].flatten(2)
    packed[..., 1024:1280] = c.d["k_new"].flatten(2)
    packed[..., 1280:] = c.d["v_new"].flatten(2)
    part = lambda lo, h: packed[..., lo:lo + h * 128].unflatten(-1, (h, 128))                # noqa: E731
    d = c.d
    c.layer = binding.Kv4Layer(Hq=8, Hkv=2, pages=d["pages"], table=d["table"], page_size=32, scale=c.scale, ctx_len=d["ctx_len"], cache_row=d["row"],
                               q=part(0, 8), k_new=part(1024, 2), v_new=part(1280, 2), out=d["out"], lse=d["lse"], k_exp=-4, v_exp=5, status=d["status"],
                               work=d["work"])
    c.write()
    c.attend()
    torch.cuda.synchronize()
    c.check("parts")


def test_many_sequences_and_layers():
    """More sequences than the kernels keep in shared memory, and two layers that share the workspace."""
    c = Kv4Case([[-1, 0]] * 70, [int(x) for x in np.random.default_rng(1).integers(0, 60, 70)], Hq=2, Hkv=1, page=16, seed=15)
    d = c.d
    pages2, out2 = d["pages"].clone(), torch.empty_like(d["out"])
    other = binding.Kv4Layer(Hq=2, Hkv=1, pages=pages2, table=d["table"], page_size=16, scale=c.scale, ctx_len=d["ctx_len"], cache_row=d["row"], q=d["q"],
                             k_new=d["v_new"], v_new=d["k_new"], out=out2, work=d["work"])
    ctx().kv4_write_tree(c.desc, [c.layer, other])
    ctx().kv4_attention(c.desc, [c.layer, other])
    torch.cuda.synchronize()
    c.check("layer 0")
    k, v = c.caches()
    swap = Kv4Case.__new__(Kv4Case)
    swap.__dict__.update(c.__dict__)
    swap.d = dict(d, pages=pages2, out=out2, lse=d["lse"])
    ref, _, bound = swap.reference()
    assert (np.abs(swap.get("out") - ref) <= 2.0 ** -11 * bound + 2e-5 * (1 + np.abs(ref))).all()


@pytest.mark.parametrize("N", [1, 12])
def test_captured_replayed_and_on_another_stream(N):
    c = Kv4Case(trees("random", 2, N, 41), [700, 90], Hq=8, Hkv=2, page=64, seed=16, out=torch.bfloat16)
    c.write()
    c.attend()
    torch.cuda.synchronize()
    want = c.d["out"].clone()
    side = torch.cuda.Stream()
    c.d["out"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.attend()
    side.synchronize()
    assert torch.equal(c.d["out"], want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.write()
        c.attend()
    for _ in range(3):
        c.d["out"].zero_()
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.d["out"], want)
    c.d["ctx_len"][0] = 301                                               # a replay goes by what the arrays hold then
    c.ctx_len = c.get("ctx_len")
    g.replay()
    torch.cuda.synchronize()
    c.check("replay")
    del g


@pytest.mark.parametrize("N", [1, 4, 12, 40])
def test_two_calls_at_once_and_many_times_over(N):
    """Two batches on two streams, each with its own workspace, forty times: the same bits as each alone."""
    cases = [Kv4Case(trees("random", 3, N, 5 + i), ctxs, Hq=8, Hkv=2, page=page, seed=21 + i, out=out)
             for i, (ctxs, page, out) in enumerate([([5000, 130, 2300], 64, torch.bfloat16), ([0, 3100, 77], 16, torch.float32)])]
    want, sides, wrong = [], [torch.cuda.Stream(), torch.cuda.Stream()], []
    for c in cases:
        c.write()
        c.attend()
        torch.cuda.synchronize()
        c.check("alone")
        want.append((c.d["out"].clone(), c.d["lse"].clone()))
        wrong.append(torch.zeros((), dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(40):
        for c, s, w, n in zip(cases, sides, want, wrong):
            with torch.cuda.stream(s):
                c.d["out"].zero_()
                c.d["lse"].zero_()
                c.attend()
                n += (c.d["out"] != w[0]).sum() + (c.d["lse"] != w[1]).sum()
    torch.cuda.synchronize()
    assert [int(n) for n in wrong] == [0, 0]
    for c in cases:
        c.check("afterwards")


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB: a page at its end holds what was written there."""
    P, H = 128, 8
    page_bytes = H * 2 * P * 72
    n_pages = (1 << 32) // page_bytes + 5
    if torch.cuda.mem_get_info()[0] < 2 * n_pages * page_bytes:
        pytest.skip("not enough free memory")
    pages = torch.empty(n_pages, H, 2, P * 72, dtype=torch.uint8, device="cuda")
    rs = np.random.default_rng(2)
    k, v = bf16(rs.standard_normal((1, 1, H, 128))), bf16(rs.standard_normal((1, 1, H, 128)))
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    desc = ctx().tree_desc(np.array([[-1]], dtype=np.int32))
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")                      # noqa: E731
    out = torch.empty(1, 1, H, 128, device="cuda")
    work = torch.empty(ctx().kv4_work_bytes(desc, H, H), dtype=torch.uint8, device="cuda")
    layer = binding.Kv4Layer(Hq=H, Hkv=H, pages=pages, table=table, page_size=P, ctx_len=i32(0), cache_row=i32(0), q=k, k_new=k, v_new=v, out=out, work=work)
    ctx().kv4_write_tree(desc, [layer])
    ctx().kv4_attention(desc, [layer])
    torch.cuda.synchronize()
    ref = O.quantise(v.double().cpu().numpy())
    assert np.allclose(out.double().cpu().numpy(), ref, rtol=2.0 ** -11, atol=0)            # one key: its values, probability one
