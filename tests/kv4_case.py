"""A batch of trees over a paged 4-bit cache, for the GPU tests: host arrays, device tensors and the oracle's answer."""
import numpy as np
import torch

from oracle import attn_oracle as A
from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from tests.harness import ctx


def bf16(a, dev="cuda"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16).to(dev)


class Kv4Case:
    """parents [B, N]; the pool starts as random bytes (NaN scales among them) and only the committed contexts are written, so that whatever
    a kernel reads beyond them shows.  The last row and the spare pages belong to nobody."""

    def __init__(self, parents, ctxs, *, Hq, Hkv, page, Ns=None, seed=0, slots=None, k_exp=0, v_exp=0, n_splits=0, out=torch.float32, q_gain=1.0,
                 extra=0):
        self.rs = rs = np.random.default_rng(seed)
        self.parent = np.asarray(parents, np.int32)
        self.B, self.N = self.parent.shape
        self.Ns = Ns or self.N
        self.Hq, self.Hkv, self.page, self.k_exp, self.v_exp = Hq, Hkv, page, k_exp, v_exp
        self.slot = np.asarray(slots if slots is not None else [rs.permutation(self.Ns)[:self.N] for _ in range(self.B)], np.int32)
        self.ctx_len = np.asarray(ctxs, np.int32)
        per = -(-(max(ctxs) + self.Ns) // page) + extra
        self.n_pages = (self.B + 1) * per + 3
        self.table = rs.permutation(self.n_pages)[:(self.B + 1) * per].reshape(self.B + 1, per).astype(np.int32)
        self.row = rs.permutation(self.B + 1)[:self.B].astype(np.int32)
        self.scale = 128 ** -0.5
        d = self.d = {}
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()        # noqa: E731
        d["pages"] = torch.from_numpy(rs.integers(0, 256, (self.n_pages, Hkv, 2, page * 72), dtype=np.uint8)).cuda()
        d["table"], d["ctx_len"], d["row"] = i32(self.table), i32(self.ctx_len), i32(self.row)
        d["q"] = bf16(rs.standard_normal((self.B, self.N, Hq, 128)) * q_gain)
        d["k_new"], d["v_new"] = bf16(rs.standard_normal((self.B, self.N, Hkv, 128))), bf16(rs.standard_normal((self.B, self.N, Hkv, 128)))
        d["out"] = torch.full((self.B, self.N, Hq, 128), float("nan"), dtype=out, device="cuda")
        d["lse"] = torch.full((self.B, self.N, Hq), float("nan"), device="cuda")
        d["status"] = torch.full((self.B,), -1, dtype=torch.int32, device="cuda")
        self.desc = ctx().tree_desc(self.parent, slot=self.slot, n_slots=self.Ns)
        d["work"] = torch.empty(max(16, ctx().kv4_work_bytes(self.desc, Hq, Hkv, n_splits)), dtype=torch.uint8, device="cuda")
        self.layer = binding.Kv4Layer(Hq=Hq, Hkv=Hkv, pages=d["pages"], table=d["table"], page_size=page, scale=self.scale, ctx_len=d["ctx_len"],
                                      cache_row=d["row"], q=d["q"], k_new=d["k_new"], v_new=d["v_new"], out=d["out"], lse=d["lse"],
                                      k_exp=k_exp, v_exp=v_exp, n_splits=n_splits, status=d["status"], work=d["work"])
        tok = [(int(self.row[b]), p) for b in range(self.B) for p in range(self.ctx_len[b])]
        if tok:
            rows, pos = (i32(np.array(x)) for x in zip(*tok))
            kc, vc = (bf16(rs.standard_normal((len(tok), Hkv, 128))) for _ in range(2))
            fill = binding.Kv4Layer(Hq=Hq, Hkv=Hkv, pages=d["pages"], table=d["table"], page_size=page, k_new=kc, v_new=vc, k_exp=k_exp, v_exp=v_exp)
            ctx().kv4_append([fill], rows, pos)
            torch.cuda.synchronize()

    def write(self):
        ctx().kv4_write_tree(self.desc, [self.layer])

    def attend(self, stream=None):
        ctx().kv4_attention(self.desc, [self.layer], stream)

    def get(self, name):
        t = self.d[name]
        return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()

    def caches(self):
        """Keys and values [rows, positions, Hkv, 128] that the pool holds for the sequences' rows (zeros elsewhere)."""
        pages, S = self.get("pages"), self.table.shape[1] * self.page
        k, v = np.zeros((self.B + 1, S, self.Hkv, 128)), np.zeros((self.B + 1, S, self.Hkv, 128))
        for b in range(self.B):
            k[self.row[b]], v[self.row[b]] = O.cache_values(pages, self.table, self.row[b], S, self.page, self.k_exp, self.v_exp)
        return k, v

    def reference(self):
        """(out, lse, sum of p |v|) of the oracle over what the pool holds."""
        k, v = self.caches()
        q = self.get("q")
        out, lse = A.tree_attention(self.parent, self.slot, q, k, v, self.ctx_len, self.row, self.scale)
        bound, _ = A.tree_attention(self.parent, self.slot, q, k, np.abs(v), self.ctx_len, self.row, self.scale)
        return out, lse, bound

    def check(self, what=""):
        """Probabilities are rounded to f16 (half a step: 2^-11 relative each), so an output is off by at most 2^-11 sum p |v|, plus the fp32 sums
        and exp2 (2e-5 (1 + |ref|), as for the bf16 attention) and, in bf16, the last rounding (2^-8 |out|).  What f16's smallest numbers
        lose is below 2^-30 of the largest probability a key."""
        ref, lse, bound = self.reference()
        got, got_lse = self.get("out"), self.get("lse")
        assert np.isfinite(got).all() and np.isfinite(got_lse).all(), f"{what}: non-finite values"
        tol = 2.0 ** -11 * bound + 2e-5 * (1 + np.abs(ref))
        if self.d["out"].dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
        err = np.abs(got - ref)
        assert (err <= tol).all(), f"{what}: {(err > tol).sum()} outputs outside tolerance, worst ratio {(err / tol).max():.2f}"
        el = np.abs(got_lse - lse)
        assert (el <= 2e-5 * (1 + np.abs(lse))).all(), f"{what}: lse worst {el.max():.3e}"
        assert self.get("status").tolist() == [0] * self.B
