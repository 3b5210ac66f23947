"""Requests through a paged cache: prompts, pieces, single tokens and a verification round, each call's result against the plain
forms, the cached rows bit for bit; the same step recorded into a graph."""
import numpy as np
import pytest
import torch

import oracle
from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import paged_step
from step_reference import chunk_attention, rope, rope_bound
from test_gpu_chunk_attn import compare
from util import gates

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Run:
    """A cache and, beside it, every request's rows as they have to be."""

    def __init__(self, dtype="bf16", heads=(8, 2, 64), batch=4, n_pages=120, page_size=16, seed=0):
        self.dtype, self.heads, self.batch = dtype, heads, batch
        self.rng = np.random.default_rng(seed)
        self.cache = paged_step.PagedCache(batch, 2, heads[1], heads[2], n_pages, page_size, 1024, DTYPES[dtype])
        self.table = paged_step.rotary_table(1024, heads[2])
        empty = lambda: torch.zeros((heads[1], 0, heads[2]), dtype=DTYPES[dtype])  # noqa: E731
        self.rows = [[(empty(), empty()) for _ in range(batch)] for _ in range(2)]  # [layer][request]

    def randn(self, *shape):
        return torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32)).to(DTYPES[self.dtype])

    def cached(self, layer, b, n):
        c = self.cache
        pages = c.block_table[b].cpu()[:-(-n // c.page_size)].long()
        take = lambda x: x[layer].cpu()[pages].transpose(0, 1).flatten(1, 2)[:, :n]  # noqa: E731
        return take(c.k_pages), take(c.v_pages)

    def step(self, news):
        c, (hq, hkv, d) = self.cache, self.heads
        t, had = sum(news), c.kv_lens.tolist()
        c.plan(ints(news), t)
        assert c.err.tolist() == [0] * self.batch
        lens = [a + n for a, n in zip(had, news)]
        for layer in range(2):
            q, k, v = self.randn(t, hq, d), self.randn(t, hkv, d), self.randn(t, hkv, d)
            q_out, out, lse = q.cuda(), torch.full((t, hq, d), 7.0, dtype=q.dtype, device="cuda"), torch.full((t, hq), 7.0, device="cuda")
            c.write(layer, q_out, k.cuda(), v.cuda(), self.table, q_out)
            c.attend(layer, q_out, out, lse, max(news), max(lens))
            place = np.concatenate([had[b] + np.arange(n) for b, n in enumerate(news)])[None]
            table = self.table.cpu().numpy()
            turned = {}
            for name, x in (("q", q), ("k", k)):
                turned[name] = rope(x.double().numpy(), place, table, [d // 2], False)
            want, scale = turned["q"]
            assert (np.abs(q_out.cpu().double().numpy() - want) <= rope_bound(want, scale, self.dtype)).all()
            at = 0
            for b, n in enumerate(news):
                k_now, v_now = self.cached(layer, b, lens[b])
                k_was, v_was = self.rows[layer][b]
                assert torch.equal(k_now[:, :had[b]], k_was[:, :had[b]]) and torch.equal(v_now[:, :had[b]], v_was[:, :had[b]]), "rows kept"
                want, scale = (x[at:at + n].transpose(1, 0, 2) for x in turned["k"])
                assert (np.abs(k_now[:, had[b]:].double().numpy() - want) <= rope_bound(want, scale, self.dtype)).all()
                assert torch.equal(v_now[:, had[b]:], v[at:at + n].transpose(0, 1))
                self.rows[layer][b] = (k_now, v_now)
                at += n
            rows = [[r[i].double() for r in self.rows[layer]] for i in (0, 1)]
            want, want_lse, bound, lse_bound = chunk_attention(q_out.cpu().double(), rows[0], rows[1], news, lens, 0, d ** -0.5, self.dtype)
            compare(out.cpu().double(), want, bound, "out")
            compare(lse.cpu().double(), want_lse, lse_bound, "lse")
        c.keep_new()
        assert c.kv_lens.tolist() == lens
        self.pages_add_up(lens)

    def pages_add_up(self, lens):
        c = self.cache
        held = c.pages_held.tolist()
        assert all(h >= -(-n // c.page_size) for h, n in zip(held, lens)) and sum(held) + c.free_count.item() == c.n_pages
        table, free = c.block_table.cpu(), c.free_pages.cpu()
        pages = [int(p) for b, h in enumerate(held) for p in table[b, :h]] + [int(p) for p in free[:c.free_count.item()]]
        assert sorted(pages) == list(range(c.n_pages)), "every page in one place"

    def round(self, parents, draft, target):
        """A verification round; parents: one tree for all requests."""
        c, (hq, hkv, d) = self.cache, self.heads
        nodes, had = len(parents), c.kv_lens.tolist()
        depth = []
        for p in parents:
            depth.append(0 if p < 0 else depth[p] + 1)
        c.plan(ints([max(depth) + 1] * self.batch))
        assert c.err.tolist() == [0] * self.batch
        place = np.add.outer(np.array(had), np.array(depth)).reshape(1, -1)
        all_parents = ints([parents] * self.batch)
        k_trees, v_trees = [], []
        for layer in range(2):
            tree = lambda h: self.randn(self.batch, nodes, h, d).cuda().transpose(1, 2)  # noqa: E731
            q, k, v, out = tree(hq), tree(hkv), tree(hkv), tree(hq)
            lse = torch.empty((self.batch, hq, nodes), device="cuda")
            before = [x.cpu().transpose(1, 2).flatten(0, 1).double().numpy() for x in (q, k)]
            c.rotate_tree(q, k, ints(place), self.table)
            for x, was in zip((q, k), before):
                want, scale = rope(was, place, self.table.cpu().numpy(), [d // 2], False)
                got = x.cpu().transpose(1, 2).flatten(0, 1).double().numpy()
                assert (np.abs(got - want) <= rope_bound(want, scale, self.dtype)).all()
            c.verify(layer, q, k, v, all_parents, out, lse, max(had))
            f32 = lambda x: np.ascontiguousarray(x.float().cpu().numpy())  # noqa: E731
            refs = [oracle.attn_all(f32(q[b]), f32(self.rows[layer][b][0]), f32(self.rows[layer][b][1]), f32(k[b]), f32(v[b]),
                                    np.array(parents, np.int32)) for b in range(self.batch)]
            gates(f32(out), f32(lse), np.stack([r[0] for r in refs]), np.stack([r[1] for r in refs]), self.dtype, "tree", stress=True)
            k_trees.append(k)
            v_trees.append(v)
        path, n, following, err = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((self.batch, nodes),) + ((self.batch,),) * 3)
        ls.ls_tree_accept_greedy(all_parents, ints([draft] * self.batch), ints(target), path, n, following, err)
        c.commit(k_trees, v_trees, path, n)
        lens = [h + a for h, a in zip(had, n.tolist())]
        assert c.kv_lens.tolist() == lens
        for layer in range(2):
            for b in range(self.batch):
                nodes_b = path[b, :n[b]].cpu().long()
                self.rows[layer][b] = tuple(torch.cat([was, x[layer][b].cpu()[:, nodes_b]], 1)
                                            for was, x in zip(self.rows[layer][b], (k_trees, v_trees)))
                for now, want in zip(self.cached(layer, b, lens[b]), self.rows[layer][b]):
                    assert torch.equal(now, want)
        self.pages_add_up(lens)
        return n.tolist()

    def release(self, b):
        self.cache.release(b)
        for layer in self.rows:
            layer[b] = tuple(x[:, :0] for x in layer[b])


@pytest.mark.parametrize("dtype,heads,page_size", [("bf16", (8, 2, 64), 16), ("f16", (4, 1, 128), 16), ("bf16", (3, 3, 128), 32)])
def test_prompts_decoding_verification(dtype, heads, page_size):
    run = Run(dtype, heads, n_pages=100 if page_size == 16 else 60, page_size=page_size)
    run.step([100, 1, 37, 0])
    run.step([200, 1, 1, 333])  # a piece, single tokens, a late prompt
    run.step([1, 1, 1, 1])
    parents = [-1, 0, 0, 1, 1, 3]
    draft = [0, 7, 8, 9, 5, 4]
    target = [[7, 9, 0, 4, 0, 2], [8, 0, 3, 0, 0, 0], [6, 0, 0, 0, 0, 0], [7, 5, 0, 0, 1, 0]]
    assert run.round(parents, draft, target) == [4, 2, 1, 3]
    run.step([1, 1, 1, 1])  # pages of tokens that were not accepted go back here
    run.release(3)
    run.step([1, 1, 64, 17])  # another request takes the place of the one that ended
    assert run.round(parents, draft, target[::-1]) == [3, 1, 2, 4]
    run.step([1, 0, 1, 1])


def test_the_example(capsys):
    paged_step.main()
    lines = capsys.readouterr().out.splitlines()
    assert lines[0] == "new tokens [1000, 37, 300]: rows [1000, 37, 300], pages [63, 3, 19], free 427"
    assert lines[2] == "accepted [4, 2, 1]: rows [1005, 40, 302], pages [63, 3, 20], free 426"
    assert lines[3] == "new tokens [1, 0, 500]: rows [1006, 0, 802], pages [63, 0, 51], free 398"


def test_a_recorded_step():
    """Plan, rope with its write, attention and the new lengths in a graph; after every replay the state and the outputs are those of
    the same step run without it, bit for bit."""
    heads, dt = (8, 2, 128), torch.bfloat16
    hq, hkv, d = heads
    table = paged_step.rotary_table(2048, d)
    gen = torch.Generator().manual_seed(3)

    class Side:
        def __init__(self):
            self.cache = paged_step.PagedCache(3, 1, hkv, d, 80, 16, 1024, dt)
            self.news = ints([200, 5, 90])

        def tokens(self, t, q, k, v):
            self.q, self.k, self.v = q.cuda(), k.cuda(), v.cuda()
            self.out, self.lse = torch.full_like(self.q, 7.0), torch.full((t, hq), 7.0, device="cuda")
            self.turned = torch.empty_like(self.q)

        def step(self, t, max_new):
            self.cache.plan(self.news, t)
            self.cache.write(0, self.q, self.k, self.v, table, self.turned)
            self.cache.attend(0, self.turned, self.out, self.lse, max_new, 400)
            self.cache.keep_new()

    plain, recorded = Side(), Side()
    draw = lambda t, h: torch.randn((t, h, d), generator=gen).to(dt)  # noqa: E731
    for t, max_new, news in ((295, 200, [200, 5, 90]), (40, 38, [1, 38, 1])):
        q, k, v = draw(t, hq), draw(t, hkv), draw(t, hkv)
        for side in (plain, recorded):
            side.news.copy_(ints(news))
            side.tokens(t, q, k, v)
            side.step(t, max_new)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded.step(40, 38)
    for turn, news in enumerate(([1, 1, 38], [1, 1, 1], [20, 20, 0], [0, 0, 1], [2, 1, 37])):
        q, k, v = draw(40, hq), draw(40, hkv), draw(40, hkv)
        for side in (plain, recorded):
            side.news.copy_(ints(news))
            side.q.copy_(q), side.k.copy_(k), side.v.copy_(v)
            side.out.fill_(7.0), side.lse.fill_(7.0)
        plain.step(40, 38)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((plain.out, recorded.out), (plain.cache.k_pages, recorded.cache.k_pages), (plain.cache.v_pages, recorded.cache.v_pages)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), turn
        assert torch.equal(plain.lse.view(torch.int32), recorded.lse.view(torch.int32)), turn
        for name in ("kv_lens", "pages_held", "free_count", "block_table", "free_pages", "cu_new", "slots", "positions"):
            assert torch.equal(getattr(plain.cache, name), getattr(recorded.cache, name)), (turn, name)
        assert (plain.out[sum(news):] == 7).all()
