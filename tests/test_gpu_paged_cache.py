"""Requests through a paged cache whose pool is exhausted before a verification round."""
import pytest
import torch

from paper_2502_17421_amd import binding as ls
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
