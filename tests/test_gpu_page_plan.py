"""Block tables, slots and positions of a step against the plain form that goes request by request."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from step_reference import page_plan

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class State:
    """A pool whose pages are spread over `held` pages per request and a stack of the rest."""

    def __init__(self, rng, held, width, n_free, page_size):
        n_pages = int(sum(held)) + n_free
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(held), width), -7, np.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.free = np.full(n_pages, -9, np.int32)
        self.free[:n_free] = order[at:]
        self.n_free, self.page_size, self.n_pages = n_free, page_size, n_pages


def check(st, kv, new, held, n_tokens, times=2):
    kv, new, held = (np.asarray(x, np.int32) for x in (kv, new, held))
    want = page_plan(kv, new, held, st.table, st.free, st.n_free, st.page_size, n_tokens)
    b = len(kv)
    table, free = dev(st.table), dev(st.free)
    outs = {"new_held": b, "free_count": 1, "cu": b + 1, "total": b, "slots": n_tokens, "positions": n_tokens, "err": b}
    got = {key: torch.full((n,), -99, dtype=torch.int32, device="cuda") for key, n in outs.items()}
    desc = ls.make_page_desc(table, n_tokens, st.page_size, st.n_pages)
    args = (dev(kv), dev(new), dev(held), table, free, dev([st.n_free]))
    for _ in range(times):  # a call repeated on the same inputs gives the same outputs
        ls.ls_page_plan(desc, *args, got["new_held"], got["free_count"], got["cu"], got["total"],
                        got["slots"] if n_tokens else None, got["positions"] if n_tokens else None, got["err"])
        torch.cuda.synchronize()
        for key in outs:
            np.testing.assert_array_equal(got[key].cpu().numpy(), np.atleast_1d(want[key]), err_msg=key)
        np.testing.assert_array_equal(table.cpu().numpy(), want["table"])
        np.testing.assert_array_equal(free.cpu().numpy(), want["free"])
    return want


@pytest.mark.parametrize("batch,page_size,longest", [(1, 16, 5), (1, 1, 40), (3, 16, 100), (64, 16, 1), (255, 32, 300), (256, 64, 70),
                                                     (257, 16, 9), (1000, 16, 40), (4096, 16, 7)])
def test_random_steps(batch, page_size, longest):
    rng = np.random.default_rng(batch * 131 + page_size)
    for spare in (0, 1, 50):
        kv = rng.integers(0, 200, batch)
        new = rng.integers(0, longest + 1, batch)
        kv[rng.random(batch) < 0.1] = 0
        ended = rng.random(batch) < 0.1
        kv[ended] = new[ended] = 0
        held = -(-kv // page_size) + rng.integers(0, 4, batch)  # some hold more than their rows take
        width = int(max(held.max(), (-(-(kv + new) // page_size)).max())) + 2
        need = int(np.maximum(0, -(-(kv + new) // page_size) - held).sum())
        st = State(rng, held, width, need + 3, page_size)
        check(st, kv, new, held, int(new.sum()) + spare)


def test_too_few_pages():
    """The first request that does not fit and every later one that needs a page are refused; those that need none are not."""
    rng = np.random.default_rng(5)
    kv, new = [10, 16, 0, 5, 40, 31], [3, 1, 100, 2, 20, 1]
    held = [1, 1, 0, 1, 3, 2]
    for n_free in range(0, 11):
        want = check(State(rng, held, 10, n_free, 16), kv, new, held, sum(new))
        assert (want["err"][[0, 3, 5]] == 0).all()
    # exactly enough, thanks to what an ended request gives back
    want = check(State(rng, [4, 0], 5, 1, 16), [0, 0], [0, 75], [4, 0], 75)
    assert (want["err"] == 0).all() and want["free_count"] == 0
    want = check(State(rng, [4, 0], 6, 1, 16), [0, 0], [0, 81], [4, 0], 81)
    assert want["err"].tolist() == [0, 1]


def test_lengths_that_are_refused():
    rng = np.random.default_rng(6)
    kv, new, held = [-1, 20, 5, 16, 90, 3, 0], [4, -3, 1, 1, 7, 1, 5], [1, 2, -1, 0, 6, 9, 0]
    st = State(rng, [max(0, h) for h in held], 6 if max(held) <= 6 else 9, 20, 16)
    st.table = st.table[:, :6].copy()      # held 9 is beyond the table; 97 rows too
    want = check(st, kv, new, held, 24)
    assert want["err"].tolist() == [2, 2, 2, 2, 2, 2, 0]
    # tokens beyond the arrays
    want = check(State(rng, [1, 1, 1], 6, 20, 16), [4, 4, 4], [8, 8, 8], [1, 1, 1], 20)
    assert want["err"].tolist() == [0, 0, 2]


def test_pages_only():
    """The form without tokens, as for reserving the rows of a path that may be accepted."""
    rng = np.random.default_rng(7)
    kv, held = rng.integers(1, 300, 40), None
    held = -(-kv // 16)
    check(State(rng, held, 25, 60, 16), kv, np.full(40, 9), held, 0)


def test_page_ids_outside_the_pool_give_no_slot():
    rng = np.random.default_rng(8)
    st = State(rng, [2, 2], 4, 3, 16)
    st.table[0, 1], st.table[1, 1] = st.n_pages, -1
    check(st, [20, 20], [5, 5], [2, 2], 10)


def test_sizes_and_alignment():
    """Slots and positions that start at odd places of an allocation."""
    rng = np.random.default_rng(9)
    for n_tokens in (1, 2, 3, 5, 1023, 1025, 4097):
        st = State(rng, [1], -(-(n_tokens + 9) // 16) + 1, n_tokens // 16 + 2, 16)
        kv, new, held = (dev([x]) for x in (9, n_tokens, 1))
        want = page_plan(np.array([9]), np.array([n_tokens]), np.array([1]), st.table, st.free, st.n_free, 16, n_tokens)
        table, free = dev(st.table), dev(st.free)
        buf = torch.full((2, n_tokens + 3), -99, dtype=torch.int32, device="cuda")
        slots, positions = buf[0, 1:1 + n_tokens], buf[1, 1:1 + n_tokens]
        small = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (1, 1, 2, 1)]
        ls.ls_page_plan(ls.make_page_desc(table, n_tokens, 16, st.n_pages), kv, new, held, table, free, dev([st.n_free]), *small, slots, positions)
        assert slots.cpu().tolist() == want["slots"].tolist() and positions.cpu().tolist() == want["positions"].tolist()
        assert buf[:, 0].tolist() == [-99, -99] and (buf[:, 1 + n_tokens:] == -99).all()


@pytest.mark.parametrize("n_tokens", [65535, 65536, 65537, 200003])
def test_many_tokens(n_tokens):
    """Around the number of tokens from which a thread takes four."""
    rng = np.random.default_rng(5)
    kv = rng.integers(0, 900, 90)
    new = rng.integers(0, 1500, 90)
    new[[3, 40]] = 0
    kv[3] = 0
    held = -(-kv // 16) + rng.integers(0, 3, 90)
    check(State(rng, held, 400, 9000, 16), kv, new, held, n_tokens)


def test_on_another_stream():
    """The stream given, and torch's current one: the call waits for what that stream holds and for nothing else."""
    rng = np.random.default_rng(6)
    kv, new, held = np.array([20, 0, 7], np.int32), np.array([30, 5, 0], np.int32), np.array([3, 0, 2], np.int32)
    st = State(rng, held, 8, 20, 16)
    want = page_plan(kv, new, held, st.table, st.free, st.n_free, 16, 40)
    for explicit in (False, True):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            late = torch.zeros(3, dtype=torch.int32, device="cuda")
            torch.cuda._sleep(2000000)
            late.copy_(dev(new))  # the lengths arrive on the side stream
            table, free, out = dev(st.table), dev(st.free), [torch.empty(n, dtype=torch.int32, device="cuda") for n in (3, 1, 4, 3, 40, 40, 3)]
            args = (dev(kv), late, dev(held), table, free, dev([st.n_free]), *out)
            desc = ls.make_page_desc(table, 40, 16, st.n_pages)
            if not explicit:
                ls.ls_page_plan(desc, *args)
        if explicit:
            ls.ls_page_plan(desc, *args, stream=side)
        side.synchronize()
        np.testing.assert_array_equal(out[4].cpu().numpy(), want["slots"])
        np.testing.assert_array_equal(table.cpu().numpy(), want["table"])
