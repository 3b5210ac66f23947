"""Sampled decoding of several continuations, the operators together as a serving program calls them: prompts, forks, trees verified at
a temperature and committed, beams dealt anew, requests that end, compaction.  After every step each request's cached rows are compared, bit for
bit, with a list of rows that is kept on the host."""
import subprocess
import sys

import numpy as np
import pytest
import torch

import sampling_reference as ref
from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd.paged_step import PagedCache

pytestmark = pytest.mark.gpu
LAYERS, HKV, D = 2, 2, 64


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, seed, batch, n_pages, page_size, max_rows, dtype=torch.bfloat16):
        self.rng = np.random.default_rng(seed)
        self.cache = PagedCache(batch, LAYERS, HKV, D, n_pages, page_size, max_rows, dtype)
        self.batch, self.dtype = batch, dtype
        self.rows = [[] for _ in range(batch)]  # per request: k of layer 0 and v of the last layer, of each row
        self.cos_sin = torch.cat([torch.ones(max_rows, D // 2), torch.zeros(max_rows, D // 2)], 1).cuda()  # no rotation

    def values(self, *shape):
        return torch.randn(shape, device="cuda").to(self.dtype)

    def new_tokens(self, news):
        t = sum(news)
        self.cache.plan(ints(news), t)
        kept = []
        for layer in range(LAYERS):
            q, k, v = self.values(t, 4, D), self.values(t, HKV, D), self.values(t, HKV, D)
            self.cache.write(layer, q, k, v, self.cos_sin, q)
            kept.append((k, v))
        self.cache.keep_new()
        at = 0
        for b, n in enumerate(news):
            if self.cache.err[b].item() == 0:
                self.rows[b] = self.rows[b] + [(kept[0][0][at + i].clone(), kept[-1][1][at + i].clone()) for i in range(n)]
            at += n

    def fork(self, sources, keep=None):
        before = [list(r) for r in self.rows]
        self.cache.fork(ints(sources), None if keep is None else ints(keep))
        lens = self.cache.kv_lens.tolist()
        for b, s in enumerate(sources):
            self.rows[b] = [] if s < 0 else before[s][:lens[b]]
            if self.cache.err[b].item() == 0 and s >= 0:
                assert lens[b] == (len(before[s]) if keep is None else keep[b])

    def round(self, vocab=501):
        """A tree of seven nodes for every request with rows, verified at a temperature and committed."""
        b, parents = self.batch, [-1, 0, 0, 1, 1, 2, 3]
        self.cache.plan(ints([4 if r else 0 for r in self.rows]))
        target = self.values(b, 7, vocab) * 2
        draft = target + self.values(b, 7, vocab) * 0.5
        tokens = torch.zeros((b, 7), dtype=torch.int64)
        for above, kids in ((0, [1, 2]), (1, [3, 4]), (2, [5]), (3, [6])):
            p = torch.softmax(draft[:, above].float().cpu(), -1)
            tokens[:, kids] = torch.multinomial(p, len(kids), generator=torch.Generator().manual_seed(int(self.rng.integers(1 << 30))))
        u, u_next = torch.rand((b, 7)), torch.rand(b)
        path, logprobs = torch.empty((b, 7), dtype=torch.int32, device="cuda"), torch.empty((b, 7), device="cuda")
        n, nxt, err = (torch.empty(b, dtype=torch.int32, device="cuda") for _ in range(3))
        heat = torch.full((b,), 0.9)
        self.cache.accept(ints([parents] * b), tokens.to(torch.int32).cuda(), target, draft, heat.cuda(), u.cuda(), u_next.cuda(), path, n, nxt,
                          logprobs, err)
        n = torch.where(torch.tensor([bool(r) for r in self.rows], device="cuda"), n, 0)
        trees = [(self.values(b, HKV, 7, D), self.values(b, HKV, 7, D)) for _ in range(LAYERS)]
        self.cache.commit([k for k, _ in trees], [v for _, v in trees], path, n)
        for i in range(b):
            want, token, _, _ = ref.accept_sampled(parents, tokens[i].tolist(), target[i].float().cpu().numpy(), draft[i].float().cpu().numpy(),
                                                   float(heat[i]), None, u[i].tolist(), float(u_next[i]), False)
            assert path[i, :len(want)].tolist() == want and nxt[i].item() == token
            if self.rows[i] and self.cache.err[i].item() == 0:
                self.rows[i] = self.rows[i] + [(trees[0][0][i, :, x].clone(), trees[-1][1][i, :, x].clone()) for x in want]

    def check(self):
        c = self.cache
        assert c.kv_lens.tolist() == [len(r) for r in self.rows]
        held, table = c.pages_held.tolist(), c.block_table.cpu()
        for b, rows in enumerate(self.rows):
            if not rows:
                continue
            at = torch.arange(len(rows))
            page, inside = table[b].long()[at // c.page_size].cuda(), (at % c.page_size).cuda()
            assert torch.equal(c.k_pages[0][page, :, inside], torch.stack([k for k, _ in rows])), b
            assert torch.equal(c.v_pages[-1][page, :, inside], torch.stack([v for _, v in rows])), b
        used = [p for b in range(self.batch) for p in table[b, :held[b]].tolist()]
        free = c.free_pages[:c.free_count.item()].tolist()
        assert len(set(free)) == len(free) and not set(free) & set(used) and sorted(set(used) | set(free)) == list(range(c.n_pages))
        # a page that a request goes on writing in is its own
        for b, rows in enumerate(self.rows):
            for p in table[b, len(rows) // c.page_size:held[b]].tolist():
                assert used.count(p) == 1
        return len(set(used))


@pytest.mark.parametrize("page_size", [16, 64])
def test_samples_of_prompts(page_size):
    s = Server(1, 8, 700, page_size, 1024)
    s.new_tokens([300, 0, 0, 0, 97, 0, 0, 0])
    s.check()
    s.fork([0, 0, 0, 0, 4, 4, 4, 4])
    s.check()
    for _ in range(3):
        s.round()
        s.check()
    s.new_tokens([1, 1, 0, 5, 1, 1, 40, 1])
    s.check()
    s.cache.release(5)  # its prompt's pages are the others' too
    s.rows[5] = []
    s.check()
    s.cache.compact()
    n = s.check()
    assert max(p for b in range(8) for p in s.cache.block_table[b, :s.cache.pages_held[b]].tolist()) == n - 1
    s.round()
    s.new_tokens([1, 2, 3, 4, 5, 300, 7, 8])
    s.check()


def test_beams_that_are_dealt_anew_and_go_back():
    s = Server(2, 12, 400, 16, 512)
    s.new_tokens([int(x) for x in s.rng.integers(1, 90, 12)])
    for step in range(6):
        groups = [3 * (b // 3) for b in range(12)]
        sources = [g + int(s.rng.integers(0, 3)) for g in groups]
        if step == 3:
            sources[6:9] = [-1, -1, -1]
        keep = [int(s.rng.integers(len(s.rows[x]) // 2, len(s.rows[x]) + 1)) if x >= 0 else 0 for x in sources] if step % 2 else None
        s.fork(sources, keep)
        s.check()
        s.round()
        s.check()
        s.new_tokens([1 if r else 0 for r in s.rows])
        s.check()
        if step in (2, 4):
            s.cache.compact()
            s.check()


def test_a_pool_that_runs_out():
    """Requests that get no page for their copy end with their full pages, and go on from there when pages are free again."""
    s = Server(3, 6, 24, 16, 256)
    s.new_tokens([200, 0, 0, 100, 0, 0])  # 13 and 7 pages of 24
    s.fork([0, 0, 0, 3, 3, 3])
    s.check()
    assert s.cache.err.tolist() == [0] * 6
    s.fork([0, 0, 0, 0, 0, 0])
    s.check()
    s.new_tokens([30, 30, 30, 30, 30, 30])
    s.check()
    s.fork([0, -1, -1, 3, 3, -1])
    s.check()
    s.new_tokens([3, 0, 0, 2, 1, 30])
    s.check()


def test_shared_pages_are_read_by_the_tree_attention():
    """Every sample's tree attends to the prompt through the same pages: bit for bit what it gets from pages of its own."""
    s = Server(4, 4, 300, 16, 1024)
    s.new_tokens([333, 0, 0, 0])
    alone = PagedCache(4, LAYERS, HKV, D, 300, 16, 1024)
    alone.plan(ints([333] * 4))
    alone.keep_new()
    for b in range(4):
        at = torch.arange(333, device="cuda")
        for x, y in ((alone.k_pages, s.cache.k_pages), (alone.v_pages, s.cache.v_pages)):
            x[:, alone.block_table[b].long()[at // 16], :, at % 16] = y[:, s.cache.block_table[0].long()[at // 16], :, at % 16]
    s.fork([0, 0, 0, 0])
    parents = ints([[-1, 0, 0, 1, 1]] * 4)
    q, k, v = s.values(4, 8, 5, D), s.values(4, HKV, 5, D), s.values(4, HKV, 5, D)
    outs = []
    for cache in (s.cache, alone):
        out, lse = torch.empty_like(q), torch.empty((4, 8, 5), device="cuda")
        cache.verify(1, q, k, v, parents, out, lse, 400)
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_recorded_forks_and_compactions():
    """A step of beam search recorded into a graph: fork, new rows, and compaction, replayed with other sources, other work in between."""
    s = Server(5, 6, 200, 16, 512)
    s.new_tokens([40, 41, 42, 43, 44, 45])
    c, sources = s.cache, ints([0, 0, 1, 3, 3, 4])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    state = [x.clone() for x in (c.block_table, c.kv_lens, c.pages_held, c.free_pages, c.free_count, c.k_pages, c.v_pages)]
    with torch.cuda.stream(side):  # buffers are made before the recording
        c.fork(sources)
        c.compact()
    side.synchronize()
    for kept, was in zip((c.block_table, c.kv_lens, c.pages_held, c.free_pages, c.free_count, c.k_pages, c.v_pages), state):
        kept.copy_(was)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fork(sources)
        c.compact()
    for dealt in ([0, 0, 1, 3, 3, 4], [5, 5, 5, 0, 1, 2], [0, 1, 2, 3, 4, 5], [2, 2, 2, 2, -1, 2]):
        sources.copy_(ints(dealt))
        graph.replay()
        torch.cuda.synchronize()
        s.rows = [s.rows[x] if x >= 0 else [] for x in dealt]
        s.check()
        s.new_tokens([3 if r else 0 for r in s.rows])
        s.check()


def test_the_example_runs():
    out = subprocess.run([sys.executable, "-m", "paper_2502_17421_amd.paged_step"], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0, out.stderr[-2000:]
    assert "accepted at a temperature" in out.stdout and "compacted" in out.stdout


FIRST_CALLS = """
import torch
from paper_2502_17421_amd import binding as ls
ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
b, n, vocab = 2, 3, 40000
target = torch.randn((b, n, vocab), device="cuda")
parents, tokens = ints([[-1, 0, 1]] * b), ints([[0, 5, 6]] * b)
ones, half = torch.ones(b, device="cuda"), torch.full((b, n), 0.5, device="cuda")
out = [torch.full((b, n), 77, dtype=torch.int32, device="cuda"), ints([77] * b), ints([77] * b)]
desc = ls.make_sample_desc(target)
ws = torch.empty(ls.ls_sample_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
table, free, held = ints([[3, 5], [0, 0]]), ints([0, 1, 2, 4, 6, 7, 0, 0]), ints([2, 0])
pages = ls.make_page_desc(table, 0, 16, 8)
made, moves, count = torch.zeros_like(table), torch.zeros((5, 4), dtype=torch.int32, device="cuda"), ints([0])
lens, new_lens, new_held, new_free = ints([20, 0]), ints([0, 0]), ints([0, 0]), ints([0])
ws_fork = torch.empty(ls.ls_page_fork_workspace_bytes(pages), dtype=torch.uint8, device="cuda")
packed, new_stack, left = torch.zeros_like(table), torch.zeros(8, dtype=torch.int32, device="cuda"), ints([0])
ws_compact = torch.empty(ls.ls_page_compact_workspace_bytes(pages), dtype=torch.uint8, device="cuda")
k = torch.arange(8, device="cuda", dtype=torch.float32)[None, :, None, None, None].expand(1, 8, 2, 16, 8).contiguous()
sources, free_count = ints([0, 0]), ints([6])
more, n_more = torch.zeros((5, 4), dtype=torch.int32, device="cuda"), ints([0])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    ls.ls_tree_accept_sampled(desc, parents, tokens, target, None, ones, None, half, half[:, 0].contiguous(), out[0], out[1], out[2], None, None, ws)
    ls.ls_page_fork(pages, sources, None, lens, held, table, free, free_count, made, new_lens, new_held, new_free, moves, count, None, ws_fork)
    ls.ls_page_copy(ls.make_copy_desc(k, None, 2), moves, count, k, None)
    ls.ls_page_compact(pages, new_held, made, packed, new_stack, left, more, n_more, ws_compact)
graph.replay()
torch.cuda.synchronize()
assert out[1].tolist() == [1, 1] and out[0][:, 0].tolist() == [0, 0] and (out[2] >= 0).all()
assert made.tolist() == [[3, 5], [3, 7]] and moves[0].tolist() == [5, 7, 4, 1] and count.item() == 1 and new_lens.tolist() == [20, 20]
assert (k[0, 7, :, :4] == 5).all() and (k[0, 7, :, 4:] == 7).all()
assert packed.tolist() == [[0, 1], [0, 2]] and left.item() == 5 and n_more.item() == 3
print("all recorded")
"""


def test_the_first_calls_of_a_process_may_be_recorded():
    """Nothing that a first call sets up is in the way of a capture."""
    run = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "all recorded" in run.stdout, run.stderr[-2000:]
