"""Requests of paged_step.PagedCache that end, on the CPU with plain stand-ins for the device calls: recordings that are replayed later."""
import pytest
import torch

from paper_2502_17421_amd import paged_step
from test_paged_cache import filled_cache, ints, plain_calls, request_rows  # noqa: F401  (plain_calls: fixture)
from test_paged_cache_fork import contents, plain_forks, same  # noqa: F401  (plain_forks: fixture)


def tables(cache):
    return [cache.block_table[b, :n].tolist() for b, n in enumerate(cache.pages_held.tolist())]


def check_pages(cache):
    """No page is free and held at once, none is lost, and a page that a request goes on writing in is its own."""
    held, free = [p for row in tables(cache) for p in row], cache.free_pages[:int(cache.free_count)].tolist()
    assert len(set(free)) == len(free) and not set(free) & set(held) and sorted(set(free) | set(held)) == list(range(cache.n_pages))
    for n, row in zip(cache.kv_lens.tolist(), tables(cache)):
        assert n <= len(row) * cache.page_size
        assert all(held.count(p) == 1 for p in row[n // cache.page_size:])


def as_it_is_now(cache):
    """A cache whose device state is this one's and whose host state is a new one's.  What a call does to it is what a
    recording of that call does, made before anything else ran, and replayed now."""
    other = paged_step.PagedCache(cache.batch, 2, 2, 64, cache.n_pages, cache.page_size, 128, torch.float32, device="cpu")
    for name, x in vars(cache).items():
        if isinstance(x, torch.Tensor) and isinstance(getattr(other, name), torch.Tensor):
            getattr(other, name).copy_(x)
    return other


@pytest.fixture
def recording(monkeypatch):
    monkeypatch.setattr(paged_step.PagedCache, "_recording", lambda self: True, raising=False)


def test_a_release_recorded_before_a_fork_and_replayed_after_it(plain_forks, recording):  # noqa: F811
    cache = filled_cache([40, 0, 20], 8)
    cache.fork(ints([0, 0, 2]))
    before = contents(cache)
    cache = as_it_is_now(cache)
    cache.release(0)
    check_pages(cache)
    for news in ([0, 0, 0], [20, 0, 0]):
        cache.plan(ints(news))
        cache.keep_new()
        check_pages(cache)
    assert cache.kv_lens.tolist() == [20, 40, 20] and not set(tables(cache)[0]) & set(tables(cache)[1])
    assert same(contents(cache)[1], before[1]) and same(contents(cache)[2], before[2])
