"""Lists of pairs (pages forked, rows copied) by their contract: a destination that an earlier pair names, or that is a source of the call, is
refused; everything else goes through, and a pair with -1 on either side is as if it were not there.  Both calls judge one list alike."""
import random

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from tests.harness import ctx

pytestmark = pytest.mark.gpu

N_ROWS, MAX_PAGES, P = 10, 3, 4


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def verdict(src, dst):
    """Status words of a list, from the contract; every destination in range is empty."""
    pairs = [(i, s, d) for i, (s, d) in enumerate(zip(src, dst)) if s != -1 and d != -1]
    st = [O.SEQ_OK] * len(src)
    for i, s, d in pairs:
        outside = not (0 <= s < N_ROWS and 0 <= d < N_ROWS)
        named = any(e == d for j, _, e in pairs if j < i)
        if outside or named or any(t == d for _, t, _ in pairs):
            st[i] = O.SEQ_BAD_ROW
    return st


LISTS = {
    "chain": ([0, 1], [1, 5]),                              # 1 is a source: refused as a destination, and forked as it was
    "long_chain": ([0, 1, 2, 5], [1, 2, 5, 6]),
    "source_of_several": ([0, 0, 1, 2], [5, 6, 7, 0]),
    "padding_names_no_destination": ([-1, 0], [5, 5]),
    "padding_names_no_source": ([5, 0], [-1, 5]),
    "padding_on_both_sides": ([-1, -1, 0, 1, -1], [-1, 5, 5, 6, 6]),
    "all_padding": ([-1, 3, -1], [2, -1, -1]),
    "named_twice": ([0, 1, 2], [5, 5, 6]),
    "named_first_by_a_refused_pair": ([99, 0], [5, 5]),
    "onto_itself": ([0, 1], [0, 5]),
    "outside": ([0, 10, 1, -2], [10, 5, 6, 7]),
}


@pytest.mark.parametrize("name", list(LISTS) + [f"random{i}" for i in range(12)])
def test_both_calls_go_by_the_contract(name):
    if name in LISTS:
        src, dst = LISTS[name]
    else:
        rng = random.Random(name)
        n = rng.randint(1, 9)
        src, dst = [rng.choice([-1, 0, 0, 1, 2, 3, 4, 7, 12]) for _ in range(n)], [rng.choice([-1, -1, 5, 6, 7, 8, 9, 3]) for _ in range(n)]
    want = verdict(src, dst)
    t = {k: i32(v) for k, v in dict(table=[[-7] * MAX_PAGES] * N_ROWS, row_pages=[0] * N_ROWS, refs=[0] * 20, free_list=[0] * 20, free_count=[0],
                                    work=[0] * binding.pages_work_ints(N_ROWS, 20)).items()}
    pt = binding.PageTable(page_size=P, **t)
    ctx().pages_init(pt)
    held = {r: n for r, n in zip((0, 1, 2), (3, 1, 2))}
    ctx().pages_reserve(pt, i32(list(held)), i32([0] * 3), end=i32([n * P for n in held.values()]))
    torch.cuda.synchronize()
    before, rows = t["table"].tolist(), t["row_pages"].tolist()
    empty = [d for d in range(N_ROWS) if rows[d] == 0]
    st = torch.full((len(src),), -1, dtype=torch.int32, device="cuda")
    ctx().pages_fork(pt, i32(src), i32(dst), st)
    torch.cuda.synchronize()
    fork = [O.SEQ_BAD_ROW if s != -1 and 0 <= d < N_ROWS and d not in empty else w for s, d, w in zip(src, dst, want)]
    assert st.tolist() == fork
    after = [list(r) for r in before]
    for s, d, w in zip(src, dst, fork):
        if s != -1 and d != -1 and not w:
            after[d] = list(before[s])
    assert t["table"].tolist() == after
    assert t["row_pages"].tolist() == [sum(p >= 0 for p in r) for r in after]
    count = [0] * 20
    for r in after:
        for p in r:
            if p >= 0:
                count[p] += 1
    assert t["refs"].tolist() == count

    block = torch.from_numpy(np.random.default_rng(3).integers(0, 99, (N_ROWS, 4)).astype(np.int32)).cuda()
    old = block.tolist()
    st.fill_(-1)
    ctx().rows_copy(binding.RowBlocks([block]), i32(src), i32(dst), st)
    torch.cuda.synchronize()
    assert st.tolist() == want
    new = list(old)
    for s, d, w in zip(src, dst, want):
        if s != -1 and d != -1 and not w:
            new[d] = old[s]
    assert block.tolist() == new
