"""Acceptance of drafted trees recorded into a graph: what a replay leaves in the workspace, late records of workgroups that have been given up among it,
has no part in the next one."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_tree_sample import Case

pytestmark = pytest.mark.gpu
POLLS = [-1, 0, 1, 2, 4, 9]


@pytest.fixture(autouse=True)
def default_polls():
    yield
    ls.ls_set_single_launch_polls(-1)


def words_of(c):
    """The workspace by sequences, [batch, words of 64 bits]: the state, the count of launches, six more, then 16 a slice."""
    b = c.parents.shape[0]
    whole = c.args[-1].view(torch.int64)
    slices = (whole.numel() // b - 8) // 16  # (three sequences and more: what the size is rounded up by is less than a slice of each)
    assert b >= 3 and slices > 1 and (b * (8 + 16 * slices) * 8 + 255) // 256 * 256 == c.args[-1].numel()
    return whole[:b * (8 + 16 * slices)].view(b, -1)


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
def test_every_launch_leaves_another_count(polls):
    """Of every sequence, whoever wrote its outputs; and a state that is nobody's."""
    c = Case(101, 6, 9, 50021, on_path=0.9)
    graph = recorded(c, polls)
    counts, rng = [words_of(c)[:, 1].clone()], np.random.default_rng(4)
    for i in range(6):
        other_numbers(c, rng)
        if i % 3 == 2:
            ls.ls_tree_accept_sampled(*c.args)
        else:
            graph.replay()
        torch.cuda.synchronize()
        c.check()
        counts.append(words_of(c)[:, 1].clone())
        assert (counts[-1] > counts[-2]).all(), counts[-2:]
        if polls == 0:  # (each workgroup that finds nobody walks)
            assert (words_of(c)[:, 0] == 0).all()


@pytest.mark.parametrize("polls", POLLS)
def test_records_of_earlier_replays_are_not_taken(polls):
    """Before each replay the records are those that the first one, or the one before the last, has left."""
    c = Case(103, 5, 9, 40009, "f16", "f32", on_path=0.9)
    graph, rng, left = recorded(c, polls), np.random.default_rng(5), []
    for i in range(7):
        other_numbers(c, rng)
        if i > 1:
            words_of(c)[:, 8:] = left[0 if i % 2 else -2]
        graph.replay()
        torch.cuda.synchronize()
        c.check()
        left.append(words_of(c)[:, 8:].clone())
    if polls < 0:
        assert not torch.equal(left[-1], left[-2])


@pytest.mark.parametrize("polls", [1, 2, 3, 5])
def test_replays_that_are_given_up_on_the_way(polls):
    """Some groups get to the end, some do not, with other numbers each time."""
    c = Case(105, 40, 6, 20011, on_path=0.9)
    graph, rng = recorded(c, polls), np.random.default_rng(polls)
    for _ in range(6):
        other_numbers(c, rng)
        graph.replay()
        torch.cuda.synchronize()
        c.check()
