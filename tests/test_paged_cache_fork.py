"""Forks, releases and compactions of paged_step.PagedCache on the CPU: plain stand-ins for the device calls, which write what those
write."""
import numpy as np
import pytest
import torch

import sampling_reference as ref
from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import paged_step
from test_paged_cache import filled_cache, ints, plain_calls, request_rows  # noqa: F401  (plain_calls: fixture)


def plain_fork(desc, sources, keep_lens, kv_lens, held, table, free, free_count, new_table, new_lens, new_held, new_free_count, copies, n_copies,
               err, workspace, stream=None, check=True):
    assert new_table is not table and workspace.numel() >= ls.ls_page_fork_workspace_bytes(desc)
    rows, lens, helds, stack, count, moves, errs = ref.fork(sources.tolist(), None if keep_lens is None else keep_lens.tolist(), kv_lens.tolist(),
                                                           held.tolist(), table.tolist(), free.tolist(), int(free_count), desc.page_size, desc.n_pages)
    new_table.fill_(-77)
    for b, row in enumerate(rows):
        new_table[b, :len(row)] = ints(row)
    for x, y in ((new_lens, lens), (new_held, helds), (free, stack), (new_free_count, [count]), (n_copies, [len(moves)]), (err, errs)):
        x.copy_(ints(y))
    copies.fill_(-77)
    copies[:len(moves)] = ints(moves).view(-1, 4)
    return 0


def plain_compact(desc, held, table, new_table, free, new_free_count, copies, n_copies, workspace, stream=None, check=True):
    rows, stack, moves = ref.compact(held.tolist(), table.tolist(), desc.page_size, desc.n_pages)
    new_table.fill_(-77)
    for b, row in enumerate(rows):
        new_table[b, :len(row)] = ints(row)
    free[:len(stack)] = ints(stack)
    new_free_count[0], n_copies[0] = len(stack), len(moves)
    copies[:len(moves)] = ints(moves).view(-1, 4)
    return 0


def plain_copy(desc, copies, n_copies, k_pages, v_pages, stream=None, check=True):
    assert copies.shape[0] == desc.max_copies >= int(n_copies)
    for a, b, rows, _ in copies[:int(n_copies)].tolist():
        for x in (k_pages, v_pages):
            x[:, b, :, :rows] = x[:, a, :, :rows]
    return 0


@pytest.fixture
def plain_forks(plain_calls, monkeypatch):  # noqa: F811
    monkeypatch.setattr(ls, "ls_page_fork", plain_fork)
    monkeypatch.setattr(ls, "ls_page_compact", plain_compact)
    monkeypatch.setattr(ls, "ls_page_copy", plain_copy)


def contents(cache):
    return [request_rows(cache, b, n) for b, n in enumerate(cache.kv_lens.tolist())]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_fork_takes_its_rows_along(plain_forks):
    cache = filled_cache([40, 20, 1], 30)
    before = contents(cache)
    cache.fork(ints([0, 0, 1]))
    assert cache.kv_lens.tolist() == [40, 40, 20] and cache.err.tolist() == [0, 0, 0]
    assert all(same(x, before[s]) for x, s in zip(contents(cache), (0, 0, 1)))
    assert cache.block_table[0, :2].tolist() == cache.block_table[1, :2].tolist() and cache.block_table[0, 2] != cache.block_table[1, 2]
    cache.fork(ints([-1, 1, 2]), ints([0, 33, 16]))
    assert cache.kv_lens.tolist() == [0, 33, 16] and cache.pages_held.tolist() == [0, 3, 1]
    for bad in (torch.zeros(3), ints([0, 1]), torch.zeros(3, dtype=torch.int64)):
        with pytest.raises(ValueError):
            cache.fork(bad)
        with pytest.raises(ValueError):
            cache.fork(ints([0, 1, 2]), bad)


def test_released_requests_keep_what_others_share(plain_forks):
    cache = filled_cache([40, 0, 3], 30)
    before = contents(cache)
    cache.release(2)  # nothing is shared yet: as ever, with the next plan
    assert cache.kv_lens.tolist() == [40, 0, 0] and cache.pages_held.tolist() == [3, 0, 1]
    cache.fork(ints([0, 0, -1]))
    cache.release(0)
    assert cache.kv_lens.tolist() == [0, 40, 0] and cache.pages_held.tolist() == [0, 3, 0] and int(cache.free_count) == 27
    assert same(contents(cache)[1], before[0])
    cache.plan(ints([100, 0, 0]))
    cache.keep_new()
    assert not set(cache.block_table[0, :7].tolist()) & set(cache.block_table[1, :3].tolist())


def test_compaction_keeps_the_rows(plain_forks):
    cache = filled_cache([40, 20, 50], 30)
    cache.fork(ints([-1, 1, 2]))
    before = contents(cache)
    cache.compact()
    assert all(same(x, y) for x, y in zip(contents(cache), before))
    held = [p for b in (1, 2) for p in cache.block_table[b, :cache.pages_held[b]].tolist()]
    assert sorted(held) == list(range(6)) and int(cache.free_count) == 24 and cache.free_pages[:24].tolist() == list(range(29, 5, -1))


def test_acceptance_is_called_with_the_requests_tensors(monkeypatch):
    cache = paged_step.PagedCache(2, 1, 1, 64, 4, 16, 32, torch.float32, device="cpu")
    calls = []
    monkeypatch.setattr(ls, "ls_tree_accept_sampled", lambda desc, *a: calls.append((desc, a)))
    target = torch.zeros((2, 5, 100), dtype=torch.float16)
    t = [torch.zeros(2) for _ in range(10)]
    cache.accept(t[0], t[1], target, None, t[2], t[3], t[4], t[5], t[6], t[7], with_replacement=True)
    desc, a = calls[0]
    assert (desc.batch, desc.n_tree, desc.vocab, desc.with_replacement, desc.target_dtype) == (2, 5, 100, 1, ls.LS_F16)
    assert a[:4] == (t[0], t[1], target, None) and a[5] is None and a[-1].numel() >= ls.ls_sample_workspace_bytes(desc)
    assert np.array_equal([x is y for x, y in zip(a[6:11], t[3:8])], [True] * 5)
