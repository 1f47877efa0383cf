"""Calls of several layers, as a model makes them: every layer has its own pool, keys, values, outputs and status words, and gets what a call of its
own would give it, bit for bit; words that a call has once come from its first layer."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from synthetic import workload as W
from tests.harness import ctx
from tests.kv4_case import bf16

pytestmark = pytest.mark.gpu

HQ, HKV, P, B = 4, 2, 16, 3


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()


def filled(value, *shape, dtype=torch.int32):
    return torch.full(shape, value, dtype=dtype, device="cuda")


@pytest.mark.parametrize("N", [2, 6])
@pytest.mark.parametrize("L", [1, 2, 4, 5, 32])
def test_layers_together_and_one_by_one(L, N):
    rs = np.random.default_rng(100 * L + N)
    Ns, ctx_lens = N + 2, [37, 0, 90]
    per = -(-(max(ctx_lens) + Ns) // P)
    n_pages = B * per + 2
    table, rows = i32(rs.permutation(n_pages)[:B * per].reshape(B, per)), i32(rs.permutation(B))
    parent = np.array([W.tree_random(W.IntStream(W.stream_key(5, b)), N, 4) for b in range(B)], dtype=np.int32)
    desc = ctx().tree_desc(parent, slot=np.array([rs.permutation(Ns)[:N] for _ in range(B)]), n_slots=Ns)
    ctx_len = i32(ctx_lens)
    tok = [(int(rows[b]), p) for b in range(B) for p in range(ctx_lens[b])] + [(-1, 0), (B, 0), (0, per * P)]
    want = [0] * (len(tok) - 2) + [O.SEQ_BAD_ROW, O.SEQ_BAD_CTX]
    tok_row, tok_pos = i32([r for r, _ in tok]), i32([p for _, p in tok])
    T = len(tok)
    work = torch.empty(ctx().kv4_work_bytes(desc, HQ, HKV), dtype=torch.uint8, device="cuda")
    pools = [torch.from_numpy(rs.integers(0, 256, (n_pages, HKV, 2, P * 72), dtype=np.uint8)).cuda() for _ in range(L)]
    prompt = [[bf16(rs.standard_normal((T, HKV, 128))) for _ in range(2)] for _ in range(L)]
    new = [[bf16(rs.standard_normal((B, N, h, 128))) for h in (HQ, HKV, HKV)] for _ in range(L)]
    shared = dict(Hq=HQ, Hkv=HKV, table=table, page_size=P, scale=128 ** -0.5, ctx_len=ctx_len, cache_row=rows)
    node = i32(rs.integers(0, N, B))
    acc, ln = filled(-1, B, 6), filled(0, B)
    ctx().path_from_node(desc, node, 6, acc, ln)
    bad = int(rows[0])                                                    # the first sequence goes bad before the publication

    def cycle(split):
        """Append, tree write, attention, publication: all layers in one call each, or (split) a call per layer."""
        mine = [p.clone() for p in pools]
        out, lse = [filled(float("nan"), B, N, HQ, 128, dtype=torch.float32) for _ in range(L)], [filled(float("nan"), B, N, HQ, dtype=torch.float32) for _ in range(L)]
        st, tok_st = [filled(-1, B) for _ in range(L)], [filled(-1, T) for _ in range(L)]
        ctx_out, seen = [filled(-1, B) for _ in range(L)], []
        app = [binding.Kv4Layer(**shared, pages=mine[l], k_new=prompt[l][0], v_new=prompt[l][1], status=st[l]) for l in range(L)]
        tree = [binding.Kv4Layer(**shared, pages=mine[l], q=new[l][0], k_new=new[l][1], v_new=new[l][2], out=out[l], lse=lse[l], status=st[l], work=work)
                for l in range(L)]

        def look():
            torch.cuda.synchronize()
            seen.append([s.tolist() for s in st])
            for s in st:
                s.fill_(-1)

        groups = [[l] for l in range(L)] if split else [list(range(L))]
        for g in groups:
            ctx().kv4_append([app[l] for l in g], tok_row, tok_pos, status=tok_st[g[0]])
        look()
        for call in (ctx().kv4_write_tree, ctx().kv4_attention):
            for g in groups:
                call(desc, [tree[l] for l in g])
            look()
        keep = table[bad, 2].clone()
        table[bad, 2] = -1
        for g in groups:
            ctx().kv4_publish(desc, [tree[l] for l in g], acc, ln, ctx_out[g[0]])
        look()
        table[bad, 2] = keep
        torch.cuda.synchronize()
        return mine, out, lse, seen, tok_st, ctx_out

    one, many = cycle(True), cycle(False)
    for name, a, b in zip(("pools", "outputs", "lse"), one[:3], many[:3]):
        for l in range(L):
            assert torch.equal(a[l], b[l]), f"{name} of layer {l}"
    for a, b, p in zip(many[0], many[0][1:], pools[1:]):
        assert not torch.equal(a, b)                                      # (the layers hold different things)
    assert one[3] == many[3]
    after = [O.SEQ_BAD_PAGE, 0, 0]
    assert many[3] == [[[-1] * B] * L, [[0] * B] * L, [[0] * B] * L, [after] * L]          # the listing call leaves the layers' words alone
    ends = [ctx_lens[0]] + [c + int(n) for c, n in zip(ctx_lens[1:], ln[1:].tolist())]
    for l in range(L):
        assert one[4][l].tolist() == want and one[5][l].tolist() == ends
        assert many[4][l].tolist() == (want if l == 0 else [-1] * T) and many[5][l].tolist() == (ends if l == 0 else [-1] * B)
    # and what the last layer holds is what it was given
    l = L - 1
    kb, vb = (torch.empty(T, HKV, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx().kv4_read(binding.Kv4Layer(**shared, pages=many[0][l]), tok_row, tok_pos, kb, vb)
    torch.cuda.synchronize()
    for got, x in ((kb, prompt[l][0]), (vb, prompt[l][1])):
        ref = O.quantise(x.double().cpu().numpy())
        ref[T - 3:] = 0
        assert np.array_equal(got.double().cpu().numpy(), ref)


def test_plain_stream_order_gives_the_same_bits():
    """A cycle of every call, with the library's overlap of kernels and without it, many times over: each call waits for what it reads."""
    cx = ctx()
    N, Ns = 12, 16
    parent = np.array([W.tree_random(W.IntStream(W.stream_key(9, b)), N, 5) for b in range(B)], dtype=np.int32)
    desc = cx.tree_desc(parent, slot=np.array([np.random.default_rng(b).permutation(Ns)[:N] for b in range(B)]), n_slots=Ns)
    freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    res = {}
    try:
        for on in (False, True):
            cx.set_overlap(on)
            rs = np.random.default_rng(8)
            t = dict(table=filled(0, B + 1, 40), row_pages=filled(0, B + 1), refs=filled(0, 130), free_list=filled(0, 130), free_count=filled(0, 1),
                     work=filled(0, binding.pages_work_ints(B + 1, 130)))
            pool = torch.zeros(130, HKV, 2, P * 72, dtype=torch.uint8, device="cuda")
            pt = binding.PageTable(page_size=P, pools=[pool], **t)
            cx.pages_init(pt)
            rows, ctx_len, ctx_next = i32([2, 0, 3]), i32([0, 0, 0]), i32([0, 0, 0])
            qo, ko = (torch.empty(B, N, h, 128, dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV))
            out, work = torch.empty(B, N, HQ, 128, device="cuda"), torch.empty(cx.kv4_work_bytes(desc, HQ, HKV), dtype=torch.uint8, device="cuda")
            st, acc, ln, node = filled(-1, B), filled(-1, B, 6), filled(0, B), i32(rs.integers(0, N, B))
            state = torch.zeros(B + 1, 64, device="cuda")
            state.copy_(torch.arange(B + 1, device="cuda")[:, None])
            q, k, v = (bf16(rs.standard_normal((B, N, h, 128))) for h in (HQ, HKV, HKV))
            layer = binding.Kv4Layer(Hq=HQ, Hkv=HKV, pages=pool, table=t["table"], page_size=P, refs=t["refs"], scale=128 ** -0.5, ctx_len=ctx_len, cache_row=rows,
                                     q=qo, k_new=ko, v_new=v, out=out, status=st, work=work)
            rope = binding.QkNormRope(q=q, k=k, q_out=qo, k_out=ko, inv_freq=freq, ctx_len=ctx_len)
            blocks, packed, sums = binding.RowBlocks([state]), cx.pack_kv4([layer]), []
            kb, vb = (torch.empty(B, HKV, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            for cycle in range(30):
                cx.pages_reserve(pt, rows, ctx_len, add=Ns)
                cx.qk_norm_rope(rope, desc)
                cx.kv4_write_tree(desc, packed)
                cx.kv4_attention(desc, packed)
                cx.path_from_node(desc, node, 6, acc, ln)
                cx.kv4_publish(desc, packed, acc, ln, ctx_next)
                cx.pages_free(pt, rows, ctx_next)
                cx.kv4_read(layer, rows, ctx_len, kb, vb)
                cx.rows_copy(blocks, rows[:1], i32([1]))
                if cycle % 5 == 4:
                    cx.pages_compact(pt)
                ctx_len.copy_(ctx_next)
                sums.append((out.clone(), kb.clone(), vb.clone(), st.clone(), ctx_len.clone(), t["table"].clone(), state.clone()))
            torch.cuda.synchronize()
            res[on] = sums
    finally:
        cx.set_overlap(True)
    assert all((s[3] == 0).all() for s in res[False]) and int(res[False][-1][4].sum()) > 30
    for cycle, (a, b) in enumerate(zip(res[False], res[True])):
        for x, y in zip(a, b):
            assert torch.equal(x, y), cycle
