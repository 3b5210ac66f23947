"""Requests of paged_step.PagedCache that end, on the CPU with plain stand-ins for the device calls: in recordings that are replayed later, and
in a step that has been planned; forks and compactions there."""
import pytest
import torch

from paper_2502_17421_amd import paged_step
from test_paged_cache import filled_cache, ints, plain_calls, trees  # noqa: F401  (plain_calls: fixture)
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


@pytest.mark.parametrize("forked", [False, True])
def test_a_release_in_a_planned_step_leaves_the_others_their_pages(plain_forks, forked):  # noqa: F811
    cache = filled_cache([40, 16, 1], 9)
    if forked:
        cache.fork(ints([0, 1, 2]))
    before = contents(cache)
    cache.plan(ints([20, 3, 0]), 23)
    planned, slots = tables(cache)[0], cache.slots.clone()
    assert len(planned) == 4
    cache.release(1)
    assert tables(cache)[0] == planned and cache.err.tolist() == [0, 1, 0] and torch.equal(cache.slots, slots)
    cache.keep_new()
    assert cache.kv_lens.tolist() == [60, 0, 1]
    check_pages(cache)
    now = contents(cache)
    assert torch.equal(now[0][0][:, :, :40], before[0][0]) and same(now[2], before[2])
    cache.plan(ints([0, 70, 0]))
    cache.keep_new()
    assert cache.err.tolist() == [0, 1, 0] and cache.kv_lens.tolist() == [60, 0, 1]  # (four pages are free, five wanted)
    cache.plan(ints([0, 60, 0]))
    cache.keep_new()
    assert cache.err.tolist() == [0, 0, 0] and cache.kv_lens.tolist() == [60, 60, 1]
    check_pages(cache)


@pytest.mark.parametrize("forked", [False, True])
def test_a_release_between_plan_and_commit(plain_forks, forked):  # noqa: F811
    """One request ends, one was refused: the others' paths are committed whole, the two commit nothing."""
    cache = filled_cache([15, 14, 16, 30], 8)
    if forked:
        cache.fork(ints([0, 1, 2, 3]))
    cache.plan(ints([4, 4, 4, 4]))  # nine pages
    assert cache.err.tolist() == [0, 0, 0, 1]
    cache.release(1)
    path = ints([[0, 1, 2, 3, 4, 5]] * 4)
    k_trees, v_trees = trees(4, 6)
    cache.commit(k_trees, v_trees, path, ints([4, 4, 4, 4]))
    assert cache.kv_lens.tolist() == [19, 0, 20, 30] and cache.err.tolist() == [0, 1, 0, 1]
    check_pages(cache)
    for b in (0, 2):
        for now, tree in zip(contents(cache)[b], (k_trees, v_trees)):
            assert torch.equal(now[:, :, -4:], torch.stack([x[b][:, :4] for x in tree]))


def test_a_fork_ends_a_planned_step(plain_forks):  # noqa: F811
    cache = filled_cache([40, 16, 1], 12)
    cache.plan(ints([20, 3, 0]), 23)
    cache.fork(ints([0, 0, 2]))
    lens, made = cache.kv_lens.tolist(), tables(cache)
    assert lens == [40, 40, 1] and cache.slots is None and cache.positions is None
    k_trees, v_trees = trees(3, 6)
    x = torch.zeros((23, 2, 64))
    for call in (cache.keep_new, lambda: cache.commit(k_trees, v_trees, ints([[0, 1, 2, 3, 4, 5]] * 3), ints([1, 1, 1])),
                 lambda: cache.write(0, x, x, x, None, x, positions=torch.zeros((1, 23), dtype=torch.int32))):
        with pytest.raises((RuntimeError, ValueError)):
            call()
    assert cache.kv_lens.tolist() == lens and tables(cache) == made and cache.err.tolist() == [0, 0, 0]
    check_pages(cache)
    cache.plan(ints([20, 3, 0]), 23)
    cache.keep_new()
    assert cache.kv_lens.tolist() == [60, 43, 1]
    check_pages(cache)


def test_a_fork_ends_a_step_whose_plan_was_recorded(plain_forks, monkeypatch):  # noqa: F811
    """Whether its replay came before the fork or after it nobody can tell on the host: nothing is new until it has."""
    cache = filled_cache([40, 16, 1], 12)
    with monkeypatch.context() as m:
        m.setattr(paged_step.PagedCache, "_recording", lambda self: True, raising=False)
        cache.plan(ints([20, 3, 0]), 23)
    cache.fork(ints([0, 0, 2]))
    cache.keep_new()
    assert cache.kv_lens.tolist() == [40, 40, 1]
    check_pages(cache)


def test_a_compaction_in_a_planned_step(plain_forks):  # noqa: F811
    """Rows that have been written move along and are kept; slots of rows that have not are gone."""
    cache = filled_cache([40, 16, 1], 30)
    cache.release(0)
    cache.plan(ints([0, 0, 20]), 20)
    rows = cache.slots.long()
    for x in (cache.k_pages, cache.v_pages):
        x[:, rows // 16, :, rows % 16] = torch.randn((20, 2, 2, 64))
    want = [[x[:, tables(cache)[b]].transpose(1, 2).flatten(2, 3)[:, :, :n].clone() for x in (cache.k_pages, cache.v_pages)]
            for b, n in ((1, 16), (2, 21))]
    cache.compact()
    assert cache.slots is None and cache.positions is None
    cache.keep_new()
    assert cache.kv_lens.tolist() == [0, 16, 21] and cache.err.tolist() == [0, 0, 0]
    check_pages(cache)
    assert all(same(x, y) for x, y in zip(contents(cache)[1:], want))


def test_forks_and_plans_refuse_columns_and_other_devices(plain_forks):  # noqa: F811
    """A column of a table of beams is not one number after the other, which is what is read."""
    cache = filled_cache([40, 16, 1], 12)
    table = ints([[0, 2], [0, 2], [1, 2]])
    for sources, keep in ((table[:, 0], None), (table[:, 0].contiguous(), table[:, 1]), (table[:, 0].contiguous().to("meta"), None)):
        with pytest.raises(ValueError):
            cache.fork(sources, keep)
        with pytest.raises(ValueError):
            cache.plan(sources if keep is None else keep)
    cache.fork(table[:, 0].contiguous())
    assert cache.kv_lens.tolist() == [40, 40, 16]
