"""Acceptance of drafted trees recorded into a graph: what a replay leaves in the workspace, late records of workgroups that have been given up among it,
has no part in the next one, whatever else the program uses the workspace for."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_tree_sample import Case

pytestmark = pytest.mark.gpu
POLLS = [-1, 0, 1, 2, 3, 4, 9, 40]


@pytest.fixture(autouse=True)
def default_polls():
    yield
    ls.ls_set_single_launch_polls(-1)


def records_of(c):
    """The records of all sequences, [batch, 16 words of 64 bits a slice]: they stand behind eight words and one a slice (up to a multiple of eight)."""
    b = c.parents.shape[0]
    whole = c.args[-1].view(torch.int64)
    fit = [s for s in range(2, 65) if (b * (8 + (s + 7) // 8 * 8 + 16 * s) * 8 + 255) // 256 * 256 == c.args[-1].numel()]
    assert len(fit) == 1
    ahead = 8 + (fit[0] + 7) // 8 * 8
    return whole[:b * (ahead + 16 * fit[0])].view(b, -1)[:, ahead:]


def other_numbers(c, rng):
    c.accept_u = torch.from_numpy(rng.random(c.accept_u.shape, dtype=np.float32) * (0.1 if rng.random() < 0.5 else 1))
    c.sample_u = torch.from_numpy(rng.random(c.sample_u.shape, dtype=np.float32))
    c.args[7].copy_(c.accept_u)
    c.args[8].copy_(c.sample_u)
    for v in c.out.values():
        v.fill_(9)


def recorded(c, polls):
    c.run()
    ls.ls_set_single_launch_polls(polls)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ls.ls_tree_accept_sampled(*c.args)
    return graph


@pytest.mark.parametrize("polls", POLLS)
@pytest.mark.parametrize("batch,vocab", [(6, 50021), (40, 20011)])
def test_no_launch_leaves_a_record(batch, vocab, polls):
    """Whether groups get to the end, are given up on the way, or are none from the start: of all workgroups, with other numbers each time."""
    c = Case(101, batch, 6, vocab, on_path=0.9)
    graph, rng = recorded(c, polls), np.random.default_rng(4)
    for i in range(8):
        other_numbers(c, rng)
        if i % 4 == 2:
            ls.ls_tree_accept_sampled(*c.args)
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert not records_of(c).any()
        c.check()


@pytest.mark.parametrize("polls", [-1, 2, 9])
def test_a_program_that_writes_into_the_workspace_between_replays(polls):
    """The same each time, or anything: to its front, all over it, everywhere but in the records."""
    c = Case(105, 5, 9, 40009, "f16", "f32", on_path=0.9)
    graph, rng = recorded(c, polls), np.random.default_rng(5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    whole = c.args[-1].view(torch.int64)
    for i in range(9):
        other_numbers(c, rng)
        if i % 3 == 0:
            whole.view(-1)[:whole.numel() // 5 * 5].view(5, -1)[:, :8] = 7
        elif i % 3 == 1:
            kept = records_of(c).clone()
            whole.fill_(7)
            records_of(c)[:] = kept
        else:
            whole.random_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        c.check()
