"""One token a sequence out of a packed projection: the same bits as from tensors of their own."""
import pytest
import torch

from paper_2609_23900_b200 import binding
from tests.harness import ctx
from tests.kv4_case import Kv4Case

pytestmark = pytest.mark.gpu


def test_single_tokens_as_parts_of_longer_rows():
    B, Hq, Hkv = 3, 8, 2
    c = Kv4Case([[-1]] * B, [130, 0, 77], Hq=Hq, Hkv=Hkv, page=32, seed=18)
    d = c.d
    packed = torch.zeros(B, (Hq + 2 * Hkv) * 128, dtype=torch.bfloat16, device="cuda")
    for lo, t in ((0, d["q"]), (Hq * 128, d["k_new"]), ((Hq + Hkv) * 128, d["v_new"])):
        packed[:, lo:lo + t.flatten(1).shape[1]] = t.flatten(1)
    part = lambda lo, h: packed[:, lo * 128:(lo + h) * 128].view(B, 1, h, 128)               # noqa: E731
    q, k, v = part(0, Hq), part(Hq, Hkv), part(Hq + Hkv, Hkv)
    c.write()
    c.attend()
    torch.cuda.synchronize()
    c.check("tensors of their own")
    want, pages = d["out"].clone(), d["pages"].clone()
    d["out"].fill_(float("nan"))
    c.layer = binding.Kv4Layer(Hq=Hq, Hkv=Hkv, pages=d["pages"], table=d["table"], page_size=32, scale=c.scale, ctx_len=d["ctx_len"], cache_row=d["row"],
                               q=q, k_new=k, v_new=v, out=d["out"], lse=d["lse"], status=d["status"], work=d["work"])
    c.write()
    c.attend()
    torch.cuda.synchronize()
    assert torch.equal(d["out"], want) and torch.equal(d["pages"], pages)
    freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    outs = []
    for x, y in ((d["q"], d["k_new"]), (q, k)):
        xo, yo = torch.empty_like(d["q"]), torch.empty_like(d["k_new"])
        ctx().qk_norm_rope(binding.QkNormRope(q=x, k=y, q_out=xo, k_out=yo, inv_freq=freq, ctx_len=d["ctx_len"]), c.desc)
        outs.append((xo, yo))
    ctx().qk_norm_rope(binding.QkNormRope(q=q, k=k, q_out=q, k_out=k, inv_freq=freq, ctx_len=d["ctx_len"]), c.desc)          # in place
    torch.cuda.synchronize()
    for x, y, z in zip(outs[0], outs[1], (q, k)):
        assert torch.equal(x, y) and torch.equal(x, z)
    assert torch.equal(v, d["v_new"])
