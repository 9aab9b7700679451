"""A serving step's tables on the GPU against a plain loop over the requests.  Whole numbers: equal.  Needs an MI355X: ``-m gpu``."""
import os
import random

import numpy as np
import pytest
import torch

from paper_2604_24013_amd import binding as cf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOP = 2 ** 31 - 1


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    yield
    torch.cuda.synchronize()


def _plain(c):
    """The definition, on Python's numbers."""
    page, width, pool, rows = c["page"], c["width"], c["pool"], c["rows"]
    table, free = [list(r) for r in c["table"]], list(c["free"])
    count = min(max(c["count"], 0), pool)
    if c["back"] is not None:
        for s, (a, b) in enumerate(c["back"]):
            for i in range(max(a, 0), max(min(b, width), 0)):
                x = table[s][i]
                if 0 <= x < pool:
                    if count < pool:
                        free[count] = x
                        count += 1
                    if c.get("clear"):
                        table[s][i] = -1
    starts, lens, slots, positions, taken = [0], [], [-1] * rows, [0] * rows, 0
    owed = []
    for s, (held, new) in enumerate(zip(c["held"], c["new"])):
        held, new = max(held, 0), max(new, 0)
        m = min(new, rows - starts[-1])
        for i in range(min(-(-held // page), width), min(-(-(held + m) // page), width)):
            table[s][i] = free[count - 1 - taken] if taken < count else -1
            taken += 1
        owed.append((s, held, m, starts[-1]))
        starts.append(starts[-1] + m)
        lens.append(min(held + m, TOP))
    for s, held, m, at in owed:
        for i in range(m):
            p = held + i
            number = table[s][p // page] if p // page < width else -1
            positions[at + i] = min(p, TOP)
            slots[at + i] = number * page + p % page if 0 <= number < pool else -1
    return dict(table=table, free=free, left=[count - taken], q_start=starts, kv_len=lens, slots=slots, positions=positions)


class _Call:
    """Device tensors of a case, filled from it; ``run`` enqueues the call, ``got`` reads back."""

    def __init__(self, c, in_place=False):
        n, i32 = len(c["held"]), torch.int32
        self.desc = cf.tables_desc(n, c["page"], c["pool"], c["width"], c["rows"], c.get("clear", False))
        t = lambda v, *shape: torch.tensor(np.array(v, dtype=np.int32).reshape(shape or -1), device=DEV)
        back = c["back"]
        self.t = dict(held=t(c["held"]), new_tokens=t(c["new"]), page_table=t(c["table"], n, c["width"]), free_pages=t(c["free"]), free_count=t([c["count"]]),
                      q_start=torch.full((n + 2,), -7, dtype=i32, device=DEV), kv_len=torch.full((n + 1,), -7, dtype=i32, device=DEV),
                      slots=torch.full((c["rows"] + 1,), -7, dtype=torch.int64, device=DEV), positions=torch.full((c["rows"] + 1,), -7, dtype=i32, device=DEV),
                      back_from=None if back is None else t([a for a, _ in back]), back_to=None if back is None else t([b for _, b in back]))
        self.t["free_left"] = self.t["free_count"] if in_place else torch.full((1,), -7, dtype=i32, device=DEV)
        self.tables = cf.make_tables(**self.t)

    def fill(self, c):
        fresh = _Call(c)
        for name, x in self.t.items():
            if x is not None and name != "free_left":
                x.copy_(fresh.t[name])

    def run(self, stream=None):
        cf.step_tables(self.desc, self.tables, stream)

    def got(self):
        torch.cuda.synchronize()
        x = self.t
        for name in ("q_start", "kv_len", "slots", "positions"):
            assert int(x[name][-1]) == -7                            # nothing behind the end
        return dict(table=x["page_table"].tolist(), free=x["free_pages"].tolist(), left=x["free_left"].tolist(), q_start=x["q_start"][:-1].tolist(),
                    kv_len=x["kv_len"][:-1].tolist(), slots=x["slots"][:-1].tolist(), positions=x["positions"][:-1].tolist())


def _case(seed, n, page, width, rows, most, longest, short=0, odd=False, back=True):
    """Requests with pages of their own out of a pool; ``short``: free pages that are missing; ``odd``: tables with nonsense among the entries."""
    rng = random.Random(seed)
    held = [rng.choice([0, rng.randint(0, most), page * rng.randint(0, most // page + 1)]) for _ in range(n)]
    new = [rng.choice([0, 1, 1, rng.randint(1, longest)]) for _ in range(n)]
    owned = [min(-(-h // page), width) for h in held]
    need = sum(min(-(-(h + m) // page), width) - o for h, m, o in zip(held, new, owned))
    pool = max(1, sum(owned) + need + 3)
    order = rng.sample(range(pool), pool)
    table, at = [], 0
    for o in owned:
        table.append(order[at:at + o] + [rng.randint(-5, pool + 5) for _ in range(width - o)])
        at += o
    if odd:
        for row in table:
            for i in range(width):
                if rng.random() < 0.1:
                    row[i] = rng.choice([-1, pool, TOP, -TOP - 1])
    count = max(0, pool - at - short)
    free = order[at:at + count]
    backs = None
    if back:
        backs = [(0, 0)] * n
        for s in rng.sample(range(n), n // 5):                       # finished: idle from now on
            backs[s] = (0, owned[s])
            held[s] = new[s] = 0
        if odd and n > 3:
            backs[1], backs[2], backs[3] = (-4, 2), (1, width + 9), (5, 2)
    return dict(page=page, width=width, pool=pool, rows=rows, held=held, new=new, table=table, free=free + [-9] * (pool - count), count=count, back=backs)


CASES = [
    _case(1, 1, 16, 4, 1, 40, 1, back=False), _case(2, 1, 16, 70, 1000, 40, 900), _case(3, 64, 16, 260, 64, 4096, 1), _case(4, 64, 64, 70, 128, 4096, 1, odd=True),
    _case(5, 200, 32, 40, 3000, 600, 300, short=50), _case(6, 200, 16, 40, 3000, 600, 300, odd=True, short=5000), _case(7, 37, 1024, 3, 20000, 2500, 900),
    _case(8, 1500, 16, 20, 8192, 300, 20), _case(9, 1025, 128, 5, 8193, 500, 40, odd=True), _case(10, 4096, 16, 9, 5000, 100, 3), _case(11, 3, 16, 600, 16000, 10, 9000),
    _case(12, 20, 16, 0, 50, 100, 4), _case(13, 50, 16, 30, 0, 100, 4)]


@pytest.mark.parametrize("clear", [False, True])
@pytest.mark.parametrize("c", CASES, ids=range(1, len(CASES) + 1))
def test_tables(c, clear):
    c = dict(c, clear=clear)
    call = _Call(c)
    call.run()
    got, want = call.got(), _plain(c)
    for name in want:
        assert got[name] == want[name], name


@pytest.mark.parametrize("seed", range(30))
def test_tables_drawn(seed):
    rng = random.Random(100 + seed)
    n = rng.choice([1, 2, 7, 63, 64, 65, 129, 700, 1024, 2000])
    c = _case(seed, n, rng.choice([16, 32, 256]), rng.randint(1, 60), rng.choice([1, 50, 3000, 9000]), rng.randint(16, 2000), rng.randint(1, 2000 // n + 2),
              short=rng.choice([0, 0, 3, 100]), odd=rng.random() < 0.5, back=rng.random() < 0.7)
    c["clear"] = seed % 2 == 0
    call = _Call(c)
    call.run()
    got, want = call.got(), _plain(c)
    for name in want:
        assert got[name] == want[name], name


def test_no_requests():
    c = dict(page=16, width=3, pool=4, rows=5, held=[], new=[], table=[], free=[1, 2, 0, 3], count=3, back=None)
    call = _Call(c)
    call.run()
    got = call.got()
    assert got["q_start"] == [0] and got["left"] == [3] and got["slots"] == [-1] * 5 and got["positions"] == [0] * 5 and got["free"] == [1, 2, 0, 3]


def test_lengths_out_of_range():
    """Lengths at the end of 31 bits, sums beyond it, and values below zero."""
    c = dict(page=16, width=4, pool=8, rows=40, held=[TOP, TOP - 3, -5, 60, 0, 3], new=[TOP, 5, 7, -TOP - 1, TOP, TOP], table=[[0, 1, 2, 3]] * 6,
             free=[4, 5, 6, 7, -9, -9, -9, -9], count=4, back=None)
    call = _Call(c)
    call.run()
    assert call.got() == _plain(c)
    c = dict(c, new=[3, 9, 4, 2, 1, 6], count=-3)
    call = _Call(c)
    call.run()
    assert call.got() == _plain(c)
    c = dict(c, count=99, back=[(0, 4)] * 6)                         # a full stack takes no more
    call = _Call(c)
    call.run()
    assert call.got() == _plain(c)


def test_steps_in_place_and_replayed():
    """The count in place over several steps, as a serving loop runs them, captured once and replayed: lengths grow by what each step brought."""
    rng = random.Random(5)
    c = _case(21, 40, 16, 50, 96, 200, 1)
    call = _Call(c, in_place=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call.run(torch.cuda.current_stream())
    for step in range(6):
        call.fill(c)
        graph.replay()
        got, want = call.got(), _plain(c)
        for name in want:
            assert got[name] == want[name], (step, name)
        c = dict(c, table=want["table"], free=want["free"], count=want["left"][0], held=want["kv_len"], back=[(0, 0)] * 40,
                 new=[rng.choice([0, 1, 1, 1, 3]) for _ in range(40)])
        if step % 2:
            s = rng.randrange(40)
            c["back"][s] = (0, -(-c["held"][s] // 16))
            c["held"][s] = c["new"][s] = 0


def test_pages_that_go_back_twice_are_cleared():
    """With clear_back the same range in every step gives each page back once."""
    c = dict(page=16, width=6, pool=10, rows=4, held=[90, 33], new=[1, 1], table=[[3, 1, 4, 5, 9, 2], [6, 8, 7, -1, -1, -1]], free=[0] + [-9] * 9, count=1,
             back=[(1, 4), (0, 0)], clear=True)
    call = _Call(c, in_place=True)
    for left in (4, 4, 4):
        call.run()
        got = call.got()
        assert got["left"] == [left] and got["table"] == [[3, -1, -1, -1, 9, 2], [6, 8, 7, -1, -1, -1]] and got["free"][:4] == [0, 1, 4, 5]
