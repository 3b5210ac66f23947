"""Acceptance of drafted trees where a slice of the vocabulary, or the draft's distribution, has nothing left, or next to nothing: against the definition
in more than 64 bits, by groups of workgroups and by workgroups alone."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_tree_sample import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["groups", "alone"])
def walks(request):
    ls.ls_set_single_launch_polls(0 if request.param == "alone" else -1)
    yield
    ls.ls_set_single_launch_polls(-1)


def star(seed, batch, n, vocab, dtype="f32"):
    """Sequences of a root with n - 1 chosen children, which are refused unless they have all of the probability."""
    c = Case(seed, batch, n, vocab, dtype, None, kind="star", temperature=[1.0] * batch)
    c.accept_u[:] = 1 - 2.0 ** -24
    c.sample_u[:] = 0.0
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kids", [1, 3, 8])
def test_a_slice_whose_tokens_have_all_been_refused(walks, dtype, kids):
    """The likeliest tokens stand in one slice, and each of them is a refused child: the first of the others, elsewhere, is drawn."""
    c = star(kids, 64, kids + 1, 32000, dtype)
    rng = np.random.default_rng(kids)
    for b in range(64):
        row = torch.full((32000,), -torch.inf)
        first, others = rng.choice(1000, kids, replace=False), 20000 + rng.choice(12000, 5, replace=False)
        row[first] = torch.from_numpy(rng.normal(0, 2, kids).astype(np.float32))
        row[others] = torch.from_numpy(rng.normal(-1, 1, 5).astype(np.float32))
        c.target[b, 0] = row
        c.tokens[b, 1:] = torch.from_numpy(first.astype(np.int32))
    c.run()
    want = c.check()
    assert (want["next"] >= 20000).all() and (want["err"] == 0).all()


@pytest.mark.parametrize("sample_u", [0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24])
@pytest.mark.parametrize("heaviest", [-5, -36])
def test_a_slice_of_which_little_is_left(walks, sample_u, heaviest):
    """What the refused children leave of their slice, down to 2^-100 of it, counts as ever."""
    c = star(7, 40, 4, 50257)
    c.sample_u[:] = sample_u
    rng = np.random.default_rng(7)
    for b in range(40):
        row = torch.full((50257,), -torch.inf)
        first = np.sort(rng.choice(700, 6, replace=False))
        row[first] = torch.tensor([0.0, 0.3, -0.4, *rng.uniform(-70, heaviest, 3)], dtype=torch.float32)
        row[30000 + b] = 0.5
        c.target[b, 0] = row
        c.tokens[b, 1:] = torch.from_numpy(first[:3].astype(np.int32))
    c.run()
    want = c.check()
    assert (want["err"] == 0).all() and (sample_u > 0 or (want["next"] < 1000).all())


def test_a_slice_of_the_least_weights_there_are(walks):
    """Tokens of 2^-1074 of the likeliest ones' weight, 2000 of them in front: whichever is drawn has a weight."""
    c = star(9, 8, 1, 32000)
    c.target[:] = -torch.inf
    c.target[:, 0, :2000] = -744.4
    c.target[:, 0, 31000:31002] = 0.0
    got = {k: v.cpu() for k, v in c.run().items()}
    assert (got["err"] == 0).all() and (got["len"] == 1).all()
    assert ((got["next"] < 2000) & (got["next"] >= 0) | (got["next"] == 31000)).all(), got["next"]


@pytest.mark.parametrize("with_replacement", [False, True])
@pytest.mark.parametrize("vocab", [4, 9001, 50257])
def test_children_behind_a_draft_that_is_used_up(walks, vocab, with_replacement):
    """Drafts of one token, and of two, with three children: those that the draft cannot have drawn have q = 0, and are accepted if they have any
    probability, in whatever order they come."""
    orders = [(0, 1, 2), (1, 0, 2), (1, 2, 0), (0, 2, 1), (3, 0, 1), (0, 3, 1)]
    c = Case(13, 12, 4, vocab, "f32", "f32", kind="star", with_replacement=with_replacement, temperature=[1.0] * 12)
    at = np.array([0, 1, 2, 3]) if vocab == 4 else np.array([17, vocab // 3, vocab // 2, vocab - 5])
    c.target[:] = -torch.inf
    for b in range(12):
        drawn = 1 + b // 6
        c.target[b][:, torch.from_numpy(at[:3])] = torch.tensor([0.0, 0.1, -0.2])  # the last token has none
        c.draft[b] = -torch.inf
        c.draft[b][:, torch.from_numpy(at[:drawn])] = torch.tensor([0.4, 0.0])[:drawn]
        c.tokens[b, 1:] = torch.from_numpy(at[list(orders[b % 6])].astype(np.int32))
    for u in (0.9, 0.5, 1 - 2.0 ** -24):
        c.accept_u[:] = u
        c.run()
        want = c.check()
        assert (want["len"] == 2).any()
