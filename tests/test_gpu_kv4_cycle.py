"""The operators as a server uses them: requests over a paged 4-bit cache through several cycles (pages reserved, queries and keys normed and
rotated, entries written, trees attended, a path accepted and published), a prompt forked into continuations together with its recurrent
state, requests retired and the pool compacted."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from synthetic import workload as W
from tests.harness import ctx
from tests.kv4_case import bf16

pytestmark = pytest.mark.gpu

HQ, HKV, P = 8, 2, 16


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def pool_and_table(n_rows, max_pages, n_pages, layers=1):
    z = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")                          # noqa: E731
    t = dict(table=z(n_rows, max_pages), row_pages=z(n_rows), refs=z(n_pages), free_list=z(n_pages), free_count=z(1),
             work=z(binding.pages_work_ints(n_rows, n_pages)))
    pools = [torch.randint(0, 256, (n_pages, HKV, 2, P * 72), dtype=torch.uint8, device="cuda") for _ in range(layers)]
    pt = binding.PageTable(page_size=P, pools=pools, **t)
    ctx().pages_init(pt)
    return pt, t, pools


def test_cycles_of_a_batch_with_forks_and_compaction():
    rs = np.random.default_rng(21)
    B, N, Ns, n_rows = 3, 7, 8, 6
    pt, t, (pool,) = pool_and_table(n_rows, 12, 60)
    freq = (1e4 ** (-torch.arange(32, dtype=torch.float64) / 32)).float().cuda()
    rows, ctx_len = i32([4, 0, 2]), i32([37, 16, 5])
    st = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ctx().pages_reserve(pt, rows, i32([0, 0, 0]), end=ctx_len, status=st)
    # the prompts: normed and rotated keys appended
    lens, names = ctx_len.tolist(), rows.tolist()
    tok = [(r, p) for r, n in zip(names, lens) for p in range(n)]
    T = len(tok)
    qkv = bf16(rs.standard_normal((T, (HQ + 2 * HKV) * 128)) * 2)
    q, k = qkv[:, :HQ * 128].unflatten(1, (HQ, 128)), qkv[:, HQ * 128:(HQ + HKV) * 128].unflatten(1, (HKV, 128))
    v = qkv[:, (HQ + HKV) * 128:].unflatten(1, (HKV, 128))
    qo, ko = torch.empty(T, HQ, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(T, HKV, 128, dtype=torch.bfloat16, device="cuda")
    tok_row, tok_pos = i32([x[0] for x in tok]), i32([x[1] for x in tok])
    ctx().qk_norm_rope(binding.QkNormRope(q=q, k=k, q_out=qo, k_out=ko, inv_freq=freq, pos=tok_pos))
    ctx().kv4_append([binding.Kv4Layer(Hq=HQ, Hkv=HKV, pages=pool, table=t["table"], page_size=P, refs=t["refs"], k_new=ko, v_new=v.contiguous())], tok_row, tok_pos)
    held = {r: (list(), list()) for r in names}                            # what every row should hold, position by position
    kq, vq = O.quantise(ko.double().cpu().numpy()), O.quantise(v.double().cpu().numpy())
    for i, (r, _) in enumerate(tok):
        held[r][0].append(kq[i])
        held[r][1].append(vq[i])
    for cycle in range(4):
        parent = np.array([W.tree_random(W.IntStream(W.stream_key(cycle, b)), N, 4) for b in range(B)], dtype=np.int32)
        slot = np.array([rs.permutation(Ns)[:N] for _ in range(B)], dtype=np.int32)
        desc = ctx().tree_desc(parent, slot=slot, n_slots=Ns)
        q, k, v = (bf16(rs.standard_normal((B, N, h, 128))) for h in (HQ, HKV, HKV))
        qo, ko, out = torch.empty_like(q), torch.empty_like(k), torch.empty(B, N, HQ, 128, device="cuda")
        work = torch.empty(ctx().kv4_work_bytes(desc, HQ, HKV), dtype=torch.uint8, device="cuda")
        layer = binding.Kv4Layer(Hq=HQ, Hkv=HKV, pages=pool, table=t["table"], page_size=P, refs=t["refs"], scale=128 ** -0.5, ctx_len=ctx_len, cache_row=rows,
                                 q=qo, k_new=ko, v_new=v, out=out, status=st, work=work)
        nxt, acc, ln, fin = i32([0] * B), i32([[-1] * 5] * B), i32([0] * B), i32([0] * B)
        node = i32([int(x) for x in rs.integers(0, N, B)])
        ctx_next = torch.empty_like(ctx_len)
        ctx().pages_reserve(pt, rows, ctx_len, add=Ns)
        ctx().qk_norm_rope(binding.QkNormRope(q=q, k=k, q_out=qo, k_out=ko, inv_freq=freq, ctx_len=ctx_len), desc)
        ctx().kv4_write_tree(desc, [layer])
        ctx().kv4_attention(desc, [layer])
        ctx().path_from_node(desc, node, 5, acc, ln)
        ctx().kv4_publish(desc, [layer], acc, ln, ctx_next)
        ctx().pages_free(pt, rows, ctx_next)
        torch.cuda.synchronize()
        assert st.tolist() == [0] * B
        # attention: the oracle over what the rows should hold and the tree's quantised entries
        kq, vq = O.quantise(ko.double().cpu().numpy()), O.quantise(v.double().cpu().numpy())
        S = max(ctx_len.tolist()) + Ns
        kc, vc = np.zeros((n_rows, S, HKV, 128)), np.zeros((n_rows, S, HKV, 128))
        for b, r in enumerate(names):
            n = len(held[r][0])
            assert n == int(ctx_len[b])
            kc[r, :n], vc[r, :n] = held[r][0], held[r][1]
            kc[r, n + slot[b]], vc[r, n + slot[b]] = kq[b], vq[b]
        args = (parent, slot, qo.double().cpu().numpy(), kc)
        ref, _ = A.tree_attention(*args, vc, ctx_len.tolist(), names, 128 ** -0.5)
        bound, _ = A.tree_attention(*args, np.abs(vc), ctx_len.tolist(), names, 128 ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -11 * bound + 2e-5 * (1 + np.abs(ref))).all()
        for b, r in enumerate(names):
            for i in A.ancestry(parent[b], int(node[b])):
                held[r][0].append(kq[b, i])
                held[r][1].append(vq[b, i])
        ctx_len.copy_(ctx_next)
        if cycle == 0:                                                     # the second request continues a copy of the first
            ctx().pages_free(pt, rows[1:2])
            ctx().pages_fork(pt, rows[:1], i32([5]), st[:1])
            rows[1], ctx_len[1] = 5, ctx_len[0]
            held[5] = (list(held[4][0]), list(held[4][1]))
            names = rows.tolist()
        if cycle == 1:
            ctx().pages_compact(pt)
        torch.cuda.synchronize()
        used = (t["refs"] > 0).sum().item()
        assert used + t["free_count"].item() == 60
        if cycle == 1:
            assert (t["refs"][:used] > 0).all()
    pages, table = pool.cpu().numpy(), t["table"].cpu().numpy()
    for b, r in enumerate(names):
        kk, vv = O.cache_values(pages, table, r, len(held[r][0]), P)
        assert np.array_equal(kk, np.array(held[r][0])) and np.array_equal(vv, np.array(held[r][1]))


@pytest.mark.parametrize("N,ctx_lens", [(1, [300, 129]), (20, [300, 77])])
def test_agrees_with_the_bf16_attention_over_the_entries_read_back(N, ctx_lens):
    """kv4_read gives bf16 entries exactly, so both attentions see the same numbers: they differ by the roundings of probabilities, 2^-8 (bf16)
    and 2^-11 (f16) of sum p |v|."""
    rs = np.random.default_rng(2)
    B, S = 2, max(ctx_lens) + N
    pt, t, (pool,) = pool_and_table(B, -(-S // P), 80)
    rows, ctx_len = i32([0, 1]), i32(ctx_lens)
    ctx().pages_reserve(pt, rows, i32([0, 0]), end=i32([c + N for c in ctx_lens]))
    tok_row, tok_pos = i32([b for b in range(B) for _ in range(ctx_lens[b])]), i32([p for b in range(B) for p in range(ctx_lens[b])])
    T = tok_row.numel()
    desc = ctx().tree_desc(np.array([[-1] + list(range(N - 1))] * B, dtype=np.int32))
    q, kn, vn = (bf16(rs.standard_normal((B, N, h, 128))) for h in (HQ, HKV, HKV))
    out = torch.empty(B, N, HQ, 128, device="cuda")
    work = torch.empty(ctx().kv4_work_bytes(desc, HQ, HKV), dtype=torch.uint8, device="cuda")
    kw = dict(Hq=HQ, Hkv=HKV, pages=pool, table=t["table"], page_size=P, scale=128 ** -0.5, ctx_len=ctx_len, cache_row=rows)
    ctx().kv4_append([binding.Kv4Layer(**kw, k_new=bf16(rs.standard_normal((T, HKV, 128))), v_new=bf16(rs.standard_normal((T, HKV, 128))))], tok_row, tok_pos)
    layer = binding.Kv4Layer(**kw, q=q, k_new=kn, v_new=vn, out=out, work=work)
    ctx().kv4_write_tree(desc, [layer])
    ctx().kv4_attention(desc, [layer])
    all_row, all_pos = i32([b for b in range(B) for _ in range(ctx_lens[b] + N)]), i32([p for b in range(B) for p in range(ctx_lens[b] + N)])
    kb, vb = (torch.empty(all_row.numel(), HKV, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx().kv4_read(layer, all_row, all_pos, kb, vb)
    kc, vc = (torch.zeros(B, S, HKV, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc[all_row.long(), all_pos.long()], vc[all_row.long(), all_pos.long()] = kb, vb
    outs = []
    for v in (vc, vc.abs()):
        o = torch.empty_like(out)
        ctx().tree_attention(desc, [binding.AttnLayer(Hq=HQ, Hkv=HKV, k_cache=kc, v_cache=v, ctx_len=ctx_len, cache_row=rows, scale=128 ** -0.5, q=q, out=o)])
        outs.append(o)
    torch.cuda.synchronize()
    err = (out - outs[0]).abs()
    assert (err <= (2.0 ** -8 + 2.0 ** -11) * 1.02 * outs[1] + 4e-5 * (1 + outs[0].abs())).all()


def test_a_hybrid_request_forked_with_its_recurrent_state():
    """rows_copy takes the recurrent state and the convolution history along: both continuations then commit alike, bit for bit."""
    from synthetic.device_case import DeviceCase
    case = W.config1()
    dc = DeviceCase(ctx(), case)
    state, hist = dc.t("state"), dc.t("conv_hist")
    row = int(case.state_row[0])
    other = (row + 1) % state.shape[0]
    assert other != row
    blocks = binding.RowBlocks([state, hist])
    ctx().rows_copy(blocks, i32([row]), i32([other]))
    dc.verify()
    dc.commit()
    dc.t("state_row")[0] = other
    dc.verify()                                                            # the copy had the state before the commit
    dc.commit()
    torch.cuda.synchronize()
    assert torch.equal(state[row], state[other]) and torch.equal(hist[row], hist[other])
