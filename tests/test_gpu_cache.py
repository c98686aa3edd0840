"""Page tables and slot maps on the GPU against the obvious loops."""
import random

import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def laga():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_17644_b200 import laga as _laga
    _laga.lib()
    return _laga


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def state(n, page, longest, new_most, seed, spare=3):
    r = random.Random(seed)
    lens = [r.randint(0, longest) for _ in range(n)]
    new = [r.randint(0, new_most) for _ in range(n)]
    columns = -(-(longest + new_most) // page)
    pages = list(range(sum(-(-s // page) for s in lens) + sum(-(-(s + a) // page) - -(-s // page) for s, a in zip(lens, new)) + spare))
    r.shuffle(pages)
    table = []
    for s in lens:
        held = -(-s // page)
        table.append([pages.pop() for _ in range(held)] + [-7] * (columns - held))
    return lens, new, table, pages


def run(laga, lens, new, table, free, page, max_tokens, n_free=None):
    t = i32(table)
    p = laga.cache_plan(i32(lens), i32(new), t, i32(free if free else [0]), i32([len(free) if n_free is None else n_free]), page, max_tokens)
    return p, t


@pytest.mark.parametrize("n,page,longest,new_most", [(1, 16, 0, 1), (1, 64, 100, 70), (48, 64, 900, 1), (300, 16, 90, 40), (1000, 32, 50, 3),
                                                     (8192, 16, 40, 2), (513, 1024, 5000, 9), (5, 128, 0, 3000)])
def test_against_loops(laga, n, page, longest, new_most):
    lens, new, table, free = state(n, page, longest, new_most, n + page)
    rows = max(1, n * new_most)
    want = ref.plan(lens, new, table, free, len(free), page, rows)
    p, t = run(laga, lens, new, table, free, page, rows)
    laga.check_status(p.status)
    assert p.slots.tolist() == want["slots"] and p.positions.tolist() == want["positions"]
    assert p.cu_new_lens.tolist() == want["cu"] and p.seq_lens.tolist() == want["lens"] and p.n_free.tolist() == [want["n_free"]]
    assert t.tolist() == want["table"]
    q, _ = run(laga, lens, new, table, free, page, max(1, want["cu"][-1]))       # exactly as many rows as there are tokens
    assert q.status.item() == 0 and q.slots.tolist()[: want["cu"][-1]] == want["slots"][: want["cu"][-1]]


def test_refusals_take_nothing(laga):
    lens, new, table, free = [5, 0, 40], [60, 20, 0], [[3, -1, -1, -1, -1], [-1] * 5, [4, 5, 6, -1, -1]], [9, 8, 7, 2, 1, 0]

    def check(why, lens=lens, new=new, free=free, rows=100, n_free=None):
        p, t = run(laga, lens, new, table, free, 16, rows, n_free)
        code, detail = laga.query_status(p.status)
        assert code == laga.ERR_CACHE_PLAN and detail == 0x50000000 + why and laga.status_string(code) == "LAGA_ERR_CACHE_PLAN"
        assert t.tolist() == table and p.seq_lens.tolist() == lens and p.slots.tolist() == [-1] * rows and p.cu_new_lens.tolist() == [0] * 4
        assert p.n_free.tolist() == [len(free) if n_free is None else n_free] and p.positions.tolist() == [0] * rows

    p, _ = run(laga, lens, new, table, free, 16, 100)
    assert p.status.item() == 0 and p.n_free.item() == 0                             # 4 + 2 pages: all of them
    check(1, new=[60, -1, 0])
    check(1, lens=[5, 0, -40])
    check(1, n_free=7)                                                               # above the stack's capacity
    check(1, n_free=-1)
    check(2, free=free[:5])
    check(3, new=[76, 0, 0])                                                         # 81 tokens in five columns of 16
    check(3, new=[2147483647, 0, 0])
    check(4, rows=79)


def test_binding_refuses_and_reuses(laga):
    lens, new, table, free = state(4, 16, 50, 20, 1)
    p, t = run(laga, lens, new, table, free, 16, 80)
    q = laga.cache_plan(i32(lens), i32(new), i32(table), i32(free), i32([len(free)]), 16, 80, out=p)
    assert q is p
    with pytest.raises(ValueError):
        laga.cache_plan(i32(lens), i32(new), i32(table), i32(free), i32([len(free)]), 16, 81, out=p)
    with pytest.raises(laga.LagaError):
        laga.cache_plan(p.seq_lens, i32(new), i32(table), i32(free), i32([len(free)]), 16, 80, out=p)     # output over its input
    with pytest.raises(laga.LagaError):
        laga.cache_plan(i32(lens), i32(new), i32(table), i32(free), i32([len(free)]), 24, 80)
