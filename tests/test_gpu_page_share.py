"""Forks, compaction and page copies against plain lists: whole numbers and moved bits, so everything has to be equal."""
import numpy as np
import pytest
import torch

import sampling_reference as ref
from paper_2502_17421_amd import binding as ls

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def canary(*shape):
    return torch.full(shape, -77, dtype=torch.int32, device="cuda")


class Tables:
    """Requests over a pool whose pages were handed out in random order; groups of `share` requests share the full pages of some prefix."""

    def __init__(self, seed, batch, page_size, max_rows, share=1, spare=50, stride_extra=3):
        rng = np.random.default_rng(seed)
        self.rng, self.batch, self.page_size = rng, batch, page_size
        self.kv = rng.integers(0, max_rows + 1, batch)
        self.stride = -(-max_rows // page_size) + stride_extra
        self.held = [min(self.stride, -(-int(n) // page_size) + int(rng.integers(0, 2))) for n in self.kv]
        shared = [0] * batch
        for b in range(batch):
            g = b // share * share
            if b > g:
                shared[b] = min(int(self.kv[b]) // page_size, int(self.kv[g]) // page_size, int(rng.integers(0, 1000)))
        need = sum(h - s for h, s in zip(self.held, shared))
        self.n_pages = need + spare
        order = rng.permutation(self.n_pages).tolist()
        self.table = []
        for b in range(batch):
            row = self.table[b // share * share][:shared[b]] if b % share else []
            own = self.held[b] - len(row)
            self.table.append(row + [order.pop() for _ in range(own)])
        self.free_count = len(order)
        self.free = order + [-5] * (self.n_pages - len(order))
        self.table = [row + [-9] * (self.stride - len(row)) for row in self.table]

    def fork(self, sources, keep=None, stream=None):
        t = self
        desc = ls.ls_page_desc(t.batch, 0, t.page_size, t.n_pages, t.stride)
        self.free_dev = ints(t.free)
        out = {"table": canary(t.batch, t.stride), "kv": canary(t.batch), "held": canary(t.batch), "count": canary(1),
               "copies": canary(t.batch, 4), "n": canary(1), "err": canary(t.batch)}
        ws = torch.full((ls.ls_page_fork_workspace_bytes(desc),), 0x5a, dtype=torch.uint8, device="cuda")
        self.args = [desc, ints(sources), None if keep is None else ints(keep), ints(t.kv), ints(t.held), ints(t.table), self.free_dev,
                     ints([t.free_count]), out["table"], out["kv"], out["held"], out["count"], out["copies"], out["n"], out["err"], ws]
        ls.ls_page_fork(*self.args, stream=stream)
        self.out = out
        return out

    def check_fork(self, sources, keep=None):
        rows, lens, held, free, count, copies, err = ref.fork(list(map(int, sources)), None if keep is None else list(map(int, keep)),
                                                              list(map(int, self.kv)), list(map(int, self.held)), self.table, self.free,
                                                              self.free_count, self.page_size, self.n_pages)
        got = {k: v.cpu().numpy() for k, v in self.out.items()}
        assert got["err"].tolist() == err
        assert got["kv"].tolist() == lens and got["held"].tolist() == held
        want = np.full((self.batch, self.stride), -77)
        for b, row in enumerate(rows):
            want[b, :len(row)] = row
        assert np.array_equal(got["table"], want)
        assert got["n"].tolist() == [len(copies)] and got["count"].tolist() == [count]
        assert got["copies"][:len(copies)].tolist() == [list(c) for c in copies] and (got["copies"][len(copies):] == -77).all()
        assert self.free_dev.cpu().tolist() == free
        return rows, lens, copies, err


@pytest.mark.parametrize("batch,page_size,max_rows,share", [(1, 16, 100, 1), (2, 1, 9, 1), (7, 16, 200, 3), (64, 16, 900, 8), (65, 64, 5000, 1),
                                                           (257, 32, 700, 4), (1000, 16, 300, 2), (4096, 16, 100, 5), (6, 16, 70000, 2)])
@pytest.mark.parametrize("keep", [False, True])
def test_forks(batch, page_size, max_rows, share, keep):
    """Any request from any other, some from none, and from fewer rows than it has."""
    t = Tables(batch + page_size, batch, page_size, max_rows, share, spare=batch)
    sources = t.rng.integers(-1, batch, batch)
    same = t.rng.random(batch) < 0.4
    sources[same] = np.arange(batch)[same]
    keeps = [int(t.rng.integers(0, t.kv[s] + 1)) if s >= 0 else int(t.rng.integers(-3, 9)) for s in sources] if keep else None
    t.fork(sources, keeps)
    t.check_fork(sources, keeps)


def test_every_request_goes_on_alone():
    """Nothing moves but the pages reserved beyond the rows."""
    t = Tables(3, 50, 16, 500)
    t.fork(np.arange(50))
    rows, lens, copies, err = t.check_fork(np.arange(50))
    assert not copies and lens == t.kv.tolist() and all(len(r) == -(-n // 16) for r, n in zip(rows, lens))


def test_one_prompt_for_all_and_the_end_of_all():
    t = Tables(4, 300, 16, 300, spare=1000)
    t.kv[0] = 16 * 15 + 3 if t.held[0] >= 16 else t.kv[0]
    for sources in ([0] * 300, [-1] * 300, [299] * 150 + [-1] * 150):
        t.fork(sources)
        t.check_fork(sources)


@pytest.mark.parametrize("spare", [0, 1, 20])
def test_pools_that_run_out(spare):
    """Requests are left with their full pages; those before them, and those that need no page, are served."""
    t = Tables(5 + spare, 60, 16, 300, spare=spare)
    sources = [b // 12 * 12 for b in range(60)]
    t.fork(sources)
    _, _, _, err = t.check_fork(sources)
    held_back = Tables(6, 60, 16, 300, spare=spare)
    held_back.fork([0] * 60)
    held_back.check_fork([0] * 60)
    assert 0 in err


def test_requests_that_are_none():
    """Sources and lengths out of range, page ids outside the pool, a stack count that is none: flagged, or taken over as they are."""
    t = Tables(7, 40, 16, 400, share=2)
    sources = [int(s) for s in t.rng.integers(-1, 40, 40)]
    keeps = [0 if s < 0 else int(t.kv[s]) for s in sources]
    sources[3], sources[4], keeps[5] = 40, -2, -1
    keeps[6], sources[6] = int(t.kv[8]) + 1, 8
    t.kv[10], t.kv[11], t.held[12], t.held[13] = -1, t.held[11] * 16 + 1, -3, t.stride + 1
    sources[14:18] = [10, 11, 12, 13]
    keeps[14:18] = [0, 0, 0, 0]
    t.table[20][0], t.table[21][0], t.table[22][0] = -1, t.n_pages, 2 ** 31 - 1
    sources[23:26] = [20, 21, 22]
    keeps[23:26] = [int(min(t.kv[20], 7)), int(min(t.kv[21], 16)), int(min(t.kv[22], 17))]
    t.fork(sources, keeps)
    t.check_fork(sources, keeps)
    for count in (-4, t.n_pages + 5, 0):
        t.free_count, t.free = count, t.rng.permutation(t.n_pages).tolist()
        t.fork(sources, keeps)
        t.check_fork(sources, keeps)


def test_forks_repeated_recorded_and_on_another_stream():
    t = Tables(8, 90, 16, 600, share=3)
    sources = t.rng.integers(-1, 90, 90)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        t.fork(sources, stream=s)
        for _ in range(3):
            ls.ls_page_fork(*t.args, stream=s)
    s.synchronize()
    t.check_fork(sources)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ls.ls_page_fork(*t.args)
    for _ in range(3):
        sources = t.rng.integers(-1, 90, 90)
        t.args[1].copy_(ints(sources))
        t.free_dev.copy_(ints(t.free))
        for v in t.out.values():
            v.fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        t.check_fork(sources)


def check_compact(t, repeats=1, stream=None):
    desc = ls.ls_page_desc(t.batch, 0, t.page_size, t.n_pages, t.stride)
    table, free, count, n = canary(t.batch, t.stride), canary(t.n_pages), canary(1), canary(1)
    copies = canary(t.n_pages // 2 + 1, 4)
    ws = torch.full((ls.ls_page_compact_workspace_bytes(desc),), 0x5a, dtype=torch.uint8, device="cuda")
    args = [desc, ints(t.held), ints(t.table), table, free, count, copies, n, ws]
    for _ in range(repeats):
        ls.ls_page_compact(*args, stream=stream)
    rows, stack, moves = ref.compact(list(map(int, t.held)), t.table, t.page_size, t.n_pages)
    want = np.full((t.batch, t.stride), -77)
    for b, row in enumerate(rows):
        want[b, :len(row)] = row
    assert np.array_equal(table.cpu().numpy(), want)
    assert free.cpu().tolist() == stack + [-77] * (t.n_pages - len(stack)) and count.item() == len(stack)
    assert n.item() == len(moves)
    assert copies[:len(moves)].cpu().tolist() == [list(m) for m in moves] and (copies[len(moves):] == -77).all()
    return args


@pytest.mark.parametrize("batch,page_size,max_rows,share,spare", [(1, 16, 100, 1, 0), (1, 16, 0, 1, 1), (3, 1, 40, 1, 25), (5, 16, 1500, 1, 64),
                                                                 (40, 16, 900, 4, 3000), (64, 64, 5000, 1, 5000), (300, 16, 3000, 3, 70000),
                                                                 (4096, 16, 90, 2, 9), (2, 16, 70000, 1, 200000)])
def test_compaction(batch, page_size, max_rows, share, spare):
    check_compact(Tables(batch + spare, batch, page_size, max_rows, share, spare), repeats=2)


def test_compaction_of_what_is_compact_and_of_nothing():
    t = Tables(9, 20, 16, 500, spare=300)
    order = iter(range(t.n_pages))
    t.table = [[next(order) if i < h else -9 for i in range(t.stride)] for h in t.held]
    check_compact(t)
    t.held = [0] * 20
    check_compact(t)


def test_compaction_with_ids_outside_the_pool_and_lengths_out_of_range():
    t = Tables(10, 30, 16, 600, spare=400)
    t.table[2][0], t.table[3][0], t.table[4][0] = -1, t.n_pages, 2 ** 31 - 1
    t.held[5], t.held[6] = -2, t.stride + 9
    t.table[6] = [7] * t.stride
    check_compact(t)


def test_a_large_pool():
    """Page ids and counts beyond 16 bits, the last word of bits not full."""
    t = Tables(11, 9, 16, 40000, spare=(1 << 22) + 37)
    desc = ls.ls_page_desc(t.batch, 0, t.page_size, t.n_pages, t.stride)
    table, free, count, n = canary(t.batch, t.stride), canary(t.n_pages), canary(1), canary(1)
    copies = canary(t.n_pages // 2 + 1, 4)
    ws = torch.empty(ls.ls_page_compact_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    ls.ls_page_compact(desc, ints(t.held), ints(t.table), table, free, count, copies, n, ws)
    rows, stack, moves = ref.compact(list(map(int, t.held)), t.table, t.page_size, t.n_pages)
    assert [table[b, :len(r)].tolist() for b, r in enumerate(rows)] == rows
    assert torch.equal(free[:len(stack)].cpu(), torch.tensor(stack, dtype=torch.int32)) and (free[len(stack):] == -77).all()
    assert n.item() == len(moves) and copies[:len(moves)].cpu().tolist() == [list(m) for m in moves]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("layers,heads,page_size,d,layout", [(1, 1, 1, 8, "head"), (2, 8, 16, 128, "head"), (3, 4, 32, 64, "token"), (1, 32, 16, 128, "token"),
                                                            (2, 3, 24, 40, "head"), (4, 5, 16, 72, "gaps"), (1, 2, 256, 512, "head"),
                                                            # pages that several workgroups take shares of
                                                            (2, 7, 72, 136, "head"), (2, 7, 72, 136, "token"), (1, 7, 72, 136, "gaps"), (2, 7, 72, 136, "wide"),
                                                            (3, 8, 128, 128, "head"), (1, 3, 16, 64, "wide")])
@pytest.mark.parametrize("n", [0, 1, 9, 60])
def test_copies(dtype, layers, heads, page_size, d, layout, n):
    rng = np.random.default_rng(n + page_size)
    pages = 2 * n + 5
    make = lambda: torch.randint(-30000, 30000, (layers, pages, heads, page_size, d * dtype.itemsize // 2), dtype=torch.int16,  # noqa: E731
                                 device="cuda").view(dtype)
    if layout == "token":
        make_ = make
        make = lambda: make_().transpose(2, 3).contiguous().transpose(2, 3)  # noqa: E731
    elif layout == "wide":  # rows token after token, of more heads than these
        make = lambda: torch.randint(-30000, 30000, (layers, pages, page_size, heads + 1, d * dtype.itemsize // 2), dtype=torch.int16,  # noqa: E731
                                     device="cuda").view(dtype)[:, :, :, :heads].transpose(2, 3)
    elif layout == "gaps":  # rows further apart than they are long
        make = lambda: torch.randint(-30000, 30000, (layers, pages, heads, page_size + 1, (d + 8) * dtype.itemsize // 2), dtype=torch.int16,  # noqa: E731
                                     device="cuda").view(dtype)[:, :, :, :page_size, :d]
    k, v = make(), make()
    order = rng.permutation(pages)
    entries = np.stack([order[:n], order[n:2 * n], rng.integers(1, page_size + 1, n), np.zeros(n, int)], 1).astype(np.int64).reshape(-1, 4)
    bad = [[pages, order[-1], 3, 0], [order[-1], -1, 3, 0], [order[-1], order[-1], 3, 0], [order[-1], order[-2], 0, 0], [order[-1], order[-2], -5, 0],
           [order[-1], order[-3], page_size + 9, 0]]  # the last one is clamped
    if n:
        entries = np.concatenate([entries, bad])
    want = [x.clone() for x in (k, v)]
    for a, b, r, _ in entries:
        if 0 <= a < pages and 0 <= b < pages and a != b:
            r = max(0, min(page_size, r))
            for w in want:
                w[:, b, :, :r] = w[:, a, :, :r]
    whole = lambda x: x.contiguous().view(torch.uint8).cpu()  # noqa: E731
    table = torch.full((len(entries) + 4, 4), 1, dtype=torch.int32, device="cuda")  # what is behind n_copies does not count
    table[:, 1] = 2
    table[:len(entries)] = ints(entries)
    ls.ls_page_copy(ls.make_copy_desc(k, v, len(entries) + 4), table, ints([len(entries)]), k, v)
    assert torch.equal(whole(k), whole(want[0])) and torch.equal(whole(v), whole(want[1]))


def test_copies_of_one_pool_and_counts_out_of_range():
    k = torch.randn((2, 40, 4, 16, 64), dtype=torch.bfloat16, device="cuda")
    table = ints([[i, i + 20, 16, 0] for i in range(6)])
    first = k.clone()
    ls.ls_page_copy(ls.make_copy_desc(k, None, 6), table, ints([-3]), k, None)
    assert torch.equal(k, first)
    ls.ls_page_copy(ls.make_copy_desc(k, None, 4), table, ints([1000]), k, None)  # max_copies are looked at
    first[:, 20:24] = first[:, 0:4]
    assert torch.equal(k, first)


def test_copies_beyond_32_bits():
    """A pool of 6 GiB, pages at both ends, and a layer stride beyond 2^31 elements."""
    k = torch.zeros((2, 200000, 1, 16, 512), dtype=torch.bfloat16, device="cuda")
    k[:, 199999] = torch.randn((2, 1, 16, 512), device="cuda").to(torch.bfloat16)
    k[:, 3] = 1
    ls.ls_page_copy(ls.make_copy_desc(k, None, 2), ints([[199999, 0, 16, 0], [3, 199998, 5, 0]]), ints([2]), k, None)
    assert torch.equal(k[:, 0], k[:, 199999]) and (k[:, 199998, :, :5] == 1).all() and not k[:, 199998, :, 5:].any()
    assert not k[:, 1].any() and not k[:, 199997].any()


def test_copies_on_another_stream_and_recorded():
    k, v = (torch.randn((3, 64, 8, 16, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    table, n = ints([[i, i + 32, 16 - i, 0] for i in range(12)]), ints([12])
    desc = ls.make_copy_desc(k, v, 12)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ls.ls_page_copy(desc, table, n, k, v, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ls.ls_page_copy(desc, table, n, k, v)
    for count in (12, 5, 0):
        k.normal_()
        want = k.clone()
        n.fill_(count)
        graph.replay()
        torch.cuda.synchronize()
        for i in range(count):
            want[:, i + 32, :, :16 - i] = want[:, i, :, :16 - i]
        assert torch.equal(k, want)
