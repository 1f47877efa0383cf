"""The failure path of the attention over the 4-bit cache: with the drill on it issues no copies and no products, so that every bounded wait runs
out.  Every sequence hears of it, and the next ordinary call has the bits it had before."""
import pytest
import torch

from paper_2609_23900_b200 import binding
from synthetic import workload as W
from tests.harness import ctx
from tests.kv4_case import Kv4Case

pytestmark = pytest.mark.gpu


@pytest.fixture
def drill():
    """Switches the drill of the shared context, which is left as it was found."""
    c = ctx()
    yield c.set_timeout_drill
    c.set_timeout_drill(False)


def _trees(B, N):
    return [W.tree_random(W.IntStream(W.stream_key(17, b)), N, 8) if N > 1 else [-1] for b in range(B)]


@pytest.mark.parametrize("N,Hq,ctxs,splits", [
    (1, 4, [3], 0), (1, 8, [5000, 130, 2300], 0), (2, 8, [700] * 40, 0), (1, 8, [4000, 1], 5),                # up to eight rows a KV head
    (4, 8, [100], 0), (3, 8, [9000, 40, 800], 0), (4, 8, [2000, 10], 3),                                      # up to sixteen
    (20, 4, [60], 0), (12, 8, [9000, 77, 3000], 0), (40, 16, [3000, 500], 0), (28, 8, [1500, 8], 4),          # more: tensor memory
])
def test_every_sequence_reports_the_timeout(N, Hq, ctxs, splits, drill):
    B = len(ctxs)
    c = Kv4Case(_trees(B, N), ctxs, Hq=Hq, Hkv=2, page=32, seed=N, n_splits=splits)
    c.write()
    c.attend()
    torch.cuda.synchronize()
    assert c.get("status").tolist() == [binding.SEQ_OK] * B
    want, lse = c.d["out"].clone(), c.d["lse"].clone()
    row = int(c.row[0])
    for bad in ((False, True) if B > 1 else (False,)):
        c.d["row"][0] = 99 if bad else row                                # a sequence that fails its check says so as ever
        drill(True)
        for _ in range(2):
            c.d["status"].fill_(-1)
            c.attend()
            torch.cuda.synchronize()
            assert c.get("status").tolist() == [binding.SEQ_BAD_ROW if bad else binding.SEQ_TIMEOUT] + [binding.SEQ_TIMEOUT] * (B - 1)
        drill(False)
        c.d["row"][0] = row
        c.d["out"].fill_(float("nan"))
        c.d["lse"].fill_(float("nan"))
        c.d["status"].fill_(-1)
        c.attend()
        torch.cuda.synchronize()
        assert c.get("status").tolist() == [binding.SEQ_OK] * B
        assert torch.equal(c.d["out"], want) and torch.equal(c.d["lse"], lse)


@pytest.mark.parametrize("N", [1, 12])
def test_nothing_to_do_takes_no_wait(N, drill):
    """All sequences fail their check: no tile, no copy, no product, and nothing runs out."""
    c = Kv4Case(_trees(2, N), [300, 40], Hq=8, Hkv=2, page=16, seed=3)
    c.d["ctx_len"].fill_(-1)
    drill(True)
    c.attend()
    torch.cuda.synchronize()
    assert c.get("status").tolist() == [binding.SEQ_BAD_CTX] * 2 and bool((c.d["out"] == 0).all())
