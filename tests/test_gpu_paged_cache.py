"""Requests through a paged cache whose pool is exhausted before a verification round."""
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import paged_step
from test_gpu_paged_step import Run, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 64)), ("f16", (4, 1, 128))])
def test_a_round_that_a_request_was_refused(dtype, heads):
    """Eight pages, of which the prompts take seven: the round finds one for request 1, none for request 3.  What requests 0 to 2
    committed is there, everything else is as it was, and request 3 goes on when others have left."""
    run = Run(dtype, heads, n_pages=8)
    run.step([10, 32, 20, 32])
    c, (hq, hkv, d), had = run.cache, heads, [10, 32, 20, 32]
    parents = [-1, 0, 0, 1, 1, 3]
    c.plan(ints([4] * 4))
    assert c.err.tolist() == [0, 0, 0, 1] and c.pages_held.tolist() == [1, 3, 2, 2] and c.free_count.item() == 0
    trees = [[run.randn(4, 6, hkv, d).cuda().transpose(1, 2) for _ in range(2)] for _ in range(2)]
    path, n, following, err = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4, 6),) + ((4,),) * 3)
    ls.ls_tree_accept_greedy(ints([parents] * 4), ints([[0, 7, 8, 9, 5, 4]] * 4), ints([[7, 9, 0, 4, 0, 2]] * 4), path, n, following, err)
    assert n.tolist() == [4] * 4
    before = [x.clone() for x in (c.k_pages, c.v_pages)]
    c.commit(*trees, path, n)
    lens = [14, 36, 24, 32]
    assert c.kv_lens.tolist() == lens and c.err.tolist() == [0, 0, 0, 1]
    written = torch.zeros((c.n_pages, c.page_size), dtype=torch.bool, device="cuda")
    for b in range(3):
        at = torch.arange(had[b], lens[b], device="cuda")
        written[c.block_table[b][at // c.page_size].long(), at % c.page_size] = True
    for was, now in zip(before, (c.k_pages, c.v_pages)):
        kept = ~written[None, :, None, :, None].expand_as(was)
        assert torch.equal(was[kept].view(torch.int16), now[kept].view(torch.int16))
    for layer in range(2):
        for b in range(4):
            nodes = path[b, :lens[b] - had[b]].cpu().long()
            run.rows[layer][b] = tuple(torch.cat([was, x[layer][b].cpu()[:, nodes]], 1) for was, x in zip(run.rows[layer][b], trees))
            for now, want in zip(run.cached(layer, b, lens[b]), run.rows[layer][b]):
                assert torch.equal(now, want)
    run.pages_add_up(lens)
    run.release(1)
    run.release(2)
    run.step([1, 3, 2, 5])
    assert run.round(parents, [0, 7, 8, 9, 5, 4], [[7, 9, 0, 4, 0, 2], [8, 0, 3, 0, 0, 0], [6, 0, 0, 0, 0, 0], [7, 5, 0, 0, 1, 0]]) == [4, 2, 1, 3]


def test_a_path_longer_than_planned():
    run = Run(n_pages=20)
    run.step([14, 30, 3, 0])
    c = run.cache
    c.plan(ints([1, 1, 1, 1]))
    assert c.pages_held.tolist() == [1, 2, 1, 1]
    path = ints([list(range(6))] * 4)
    trees = [[run.randn(4, 6, 2, 64).cuda().transpose(1, 2) for _ in range(2)] for _ in range(2)]
    free = c.free_pages[:c.free_count.item()].long()
    c.commit(*trees, path, ints([5, 2, 6, 1]))
    lens = [16, 32, 9, 1]
    assert c.kv_lens.tolist() == lens and c.err.tolist() == [1, 0, 0, 0]
    assert (c.k_pages[:, free] == 0).all() and (c.v_pages[:, free] == 0).all()
    for layer in range(2):
        for b, had in enumerate((14, 30, 3, 0)):
            for now, was, tree in zip(run.cached(layer, b, lens[b]), run.rows[layer][b], trees):
                assert torch.equal(now, torch.cat([was, tree[layer][b].cpu()[:, :lens[b] - had]], 1))


def test_steps_of_other_sizes_between_replays():
    """A recorded decoding step next to eager prompts, which need longer slots and a larger workspace, and other tensors that take up
    what memory is free: after each replay state, rows and outputs are those of a side that records nothing, bit for bit."""
    hq, hkv, d, dt = 8, 2, 128, torch.bfloat16
    table = paged_step.rotary_table(8192, d)
    gen = torch.Generator().manual_seed(5)

    class Side:
        def __init__(self):
            self.cache = paged_step.PagedCache(3, 1, hkv, d, 1200, 16, 8192, dt)
            self.sizes = {}

        def step(self, t, max_new, max_kv):
            c, (news, q, k, v, turned, out, lse) = self.cache, self.sizes[t]
            c.plan(news, t)
            c.write(0, q, k, v, table, turned)
            c.attend(0, turned, out, lse, max_new, max_kv)
            c.keep_new()

        def fill(self, t, news, q, k, v):
            if t not in self.sizes:
                new = lambda x: torch.empty_like(x, device="cuda")  # noqa: E731
                self.sizes[t] = (ints(news), new(q), new(k), new(v), new(q), new(q), torch.empty((t, hq), device="cuda"))
            for x, value in zip(self.sizes[t], (torch.tensor(news, dtype=torch.int32), q, k, v)):
                x.copy_(value)

    sides = plain, recorded = Side(), Side()

    def fill(t, news):
        q, k, v = (torch.randn((t, h, d), generator=gen).to(dt) for h in (hq, hkv, hkv))
        for side in sides:
            side.fill(t, news, q, k, v)

    def agree(t, what):
        torch.cuda.synchronize()
        for a, b in ((plain.sizes[t][5], recorded.sizes[t][5]), (plain.cache.k_pages, recorded.cache.k_pages),
                     (plain.cache.v_pages, recorded.cache.v_pages)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), what
        assert torch.equal(plain.sizes[t][6].view(torch.int32), recorded.sizes[t][6].view(torch.int32)), what
        for name in ("kv_lens", "pages_held", "free_count", "block_table", "free_pages", "cu_new", "err"):
            assert torch.equal(getattr(plain.cache, name), getattr(recorded.cache, name)), (what, name)

    for turn in range(2):
        fill(3, [1, 1, 1])
        for side in sides:
            side.step(3, 1, 8192)
        agree(3, turn)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded.step(3, 1, 8192)
    others = []
    for turn, (t, news, max_kv) in enumerate(((90, [60, 0, 30], 100), (2000, [3, 1997, 0], 6000), (40, [1, 38, 1], 7000), (5000, [2, 1998, 3000], 8192))):
        fill(3, [1, 1, 1])
        plain.step(3, 1, 8192)
        graph.replay()
        agree(3, ("replay", turn))
        fill(t, news)
        for side in sides:
            side.step(t, max(news), max_kv)
        agree(t, ("eager", turn))
        others += [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for n in (512, 1024, 8192, 1 << 16, 1 << 20, 1 << 22) for _ in range(4)]
        torch.cuda.synchronize()
    for x in others:
        assert (x == 0x7f).all(), "somebody else's memory"
