"""The state of paged_step.PagedCache on the CPU: plain stand-ins for the device calls, which write what those write."""
import gc
import weakref

import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import paged_step
from step_reference import page_plan


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def plain_plan(desc, kv_lens, new_lens, pages_held, table, free, free_count, new_held, new_free_count, cu_new, total_lens, slots, positions,
               err, stream=None, check=True):
    want = page_plan(kv_lens.numpy(), new_lens.numpy(), pages_held.numpy(), table.numpy(), free.numpy(), int(free_count[0]), desc.page_size,
                     desc.n_tokens)
    outs = {"table": table, "free": free, "new_held": new_held, "cu": cu_new, "total": total_lens, "err": err}
    if desc.n_tokens:
        outs.update(slots=slots, positions=positions.view(-1))
    for key, x in outs.items():
        x.copy_(torch.from_numpy(want[key]))
    new_free_count[0] = want["free_count"]
    return 0


def plain_commit(desc, k_tree, v_tree, accept_path, accept_len, prefix_lens, k_pages, v_pages, table, page_size, new_prefix_lens,
                 err_flag=None, stream=None, check=True):
    for b in range(k_tree.shape[0]):
        n, had = max(0, int(accept_len[b])), int(prefix_lens[b])
        n = min(n, table.shape[1] * page_size - had)
        for j in range(n):
            page, row, node = int(table[b, (had + j) // page_size]), (had + j) % page_size, int(accept_path[b, j])
            k_pages[page, :, row], v_pages[page, :, row] = k_tree[b, :, node], v_tree[b, :, node]
        new_prefix_lens[b] = had + n
    return 0


@pytest.fixture
def plain_calls(monkeypatch):
    monkeypatch.setattr(ls, "ls_page_plan", plain_plan)
    monkeypatch.setattr(ls, "ls_kv_commit_paged", plain_commit)


def filled_cache(lens, n_pages, page_size=16):
    """Requests of these lengths, every row of the pool with values of its own."""
    cache = paged_step.PagedCache(len(lens), 2, 2, 64, n_pages, page_size, 128, torch.float32, device="cpu")
    for x in (cache.k_pages, cache.v_pages):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(1)))
    cache.plan(ints(lens))
    cache.keep_new()
    assert cache.kv_lens.tolist() == lens
    return cache


def request_rows(cache, b, n):
    pages = cache.block_table[b, :-(-n // cache.page_size)].long()
    return [x[:, pages].transpose(1, 2).flatten(2, 3)[:, :, :n].clone() for x in (cache.k_pages, cache.v_pages)]


def trees(batch, nodes):
    gen = torch.Generator().manual_seed(2)
    return [[torch.randn((batch, 2, nodes, 64), generator=gen) for _ in range(2)] for _ in range(2)]


def test_a_refused_request_commits_nothing(plain_calls):
    """Four pages: request 0 has room in its page, request 1 takes the last free one, none is left for request 2."""
    cache = filled_cache([5, 16, 16], 4)
    cache.plan(ints([4, 4, 4]))
    assert cache.err.tolist() == [0, 0, 1] and cache.pages_held.tolist() == [1, 2, 1]
    before = [request_rows(cache, b, n) for b, n in enumerate([5, 16, 16])]
    path = ints([[0, 2, 3, 5, 0, 0]] * 3)
    k_trees, v_trees = trees(3, 6)
    cache.commit(k_trees, v_trees, path, ints([3, 2, 4]))
    assert cache.kv_lens.tolist() == [8, 18, 16] and cache.err.tolist() == [0, 0, 1]
    for b, (had, n) in enumerate(((5, 3), (16, 2), (16, 0))):
        nodes = path[b, :n].long()
        for was, now, tree in zip(before[b], request_rows(cache, b, had + n), (k_trees, v_trees)):
            want = torch.cat([was, torch.stack([x[b][:, nodes] for x in tree])], 2)
            assert torch.equal(now, want), b
    cache.plan(ints([0, 0, 0]))  # the refused request is as it was: nothing is wrong with it
    assert cache.err.tolist() == [0, 0, 0] and cache.kv_lens.tolist() == [8, 18, 16]


def test_a_path_longer_than_planned_stays_in_its_pages(plain_calls):
    """Rows for which no page was planned are not written; the request is flagged."""
    cache = filled_cache([14, 30], 8)
    cache.plan(ints([1, 1]))
    assert cache.pages_held.tolist() == [1, 2]
    free = cache.free_pages[:cache.free_count.item()].long()
    before = [x[:, free].clone() for x in (cache.k_pages, cache.v_pages)]
    path = ints([[0, 1, 2, 3, 4, 5]] * 2)
    k_trees, v_trees = trees(2, 6)
    cache.commit(k_trees, v_trees, path, ints([5, 2]))
    assert cache.kv_lens.tolist() == [16, 32] and cache.err.tolist() == [1, 0]
    for was, now in zip(before, (cache.k_pages, cache.v_pages)):
        assert torch.equal(was, now[:, free])
    for b in range(2):
        rows = request_rows(cache, b, [16, 32][b])
        for now, tree in zip(rows, (k_trees, v_trees)):
            assert torch.equal(now[:, :, -2:], torch.stack([x[b][:, :2] for x in tree]))


class TestBuffersOfARecordedStep:
    """A recorded step goes on using the addresses it was recorded with: what they point at has to stay the cache's."""

    @pytest.fixture(autouse=True)
    def seen_calls(self, plain_calls, monkeypatch):
        self.used = []  # weak references to the storage of every buffer that a call was given

        def plan(*args, **kwargs):
            self.used += [weakref.ref(x.untyped_storage()) for x in args[11:13] if x is not None]
            return plain_plan(*args, **kwargs)

        def attend(desc, q, k, v, table, cu, lens, out, lse, workspace, stream=None, check=True):
            assert workspace.numel() >= ls.ls_chunk_workspace_bytes(desc)
            self.used.append(weakref.ref(workspace.untyped_storage()))
            return 0

        monkeypatch.setattr(ls, "ls_page_plan", plan)
        monkeypatch.setattr(ls, "ls_chunk_attn_paged", attend)

    def step(self, cache, news, max_kv):
        t = sum(news)
        cache.plan(ints(news), t)
        slots = cache.slots
        assert slots.shape == (t,) and cache.positions.shape == (1, t) and (slots >= 0).all()
        q = torch.zeros((t, 8, 64), dtype=torch.bfloat16)
        cache.attend(0, q, torch.empty_like(q), torch.empty((t, 8)), max(news), max_kv)
        return slots

    def test_they_stay(self):
        cache = paged_step.PagedCache(2, 1, 2, 64, 4000, 16, 30000, torch.bfloat16, device="cpu")
        self.step(cache, [1, 1], 40)
        first = [ref() for ref in self.used]
        assert len(first) == 3 and all(x is not None for x in first)
        addresses = [x.data_ptr() for x in first]
        del first
        for news, max_kv in (([700, 30], 1000), ([3, 1], 30000), ([1, 1], 40), ([2000, 2000], 4000), ([1, 0], 40)):
            self.step(cache, news, max_kv)
            cache.plan(ints([4, 4]))
        gc.collect()
        assert [ref() is not None for ref in self.used] == [True] * len(self.used)
        assert [ref().data_ptr() for ref in self.used[:3]] == addresses

    def test_they_do_not_add_up(self):
        """What is kept is less than four times what the largest step needs, however many sizes there were."""
        cache = paged_step.PagedCache(1, 1, 2, 64, 4000, 16, 30000, torch.bfloat16, device="cpu")
        for n in range(1, 3000, 7):
            cache.plan(ints([n]), n)
        storages = {ref().data_ptr(): ref().nbytes() for ref in self.used}
        assert sum(storages.values()) < 4 * (2 * 4 * 3000)


class TestSizesThatDoNotFit:
    """Tensors that hold fewer tokens than a call would read or write are refused before it is made."""

    @pytest.fixture(autouse=True)
    def calls(self, plain_calls, monkeypatch):
        self.made = []
        for name in ("ls_rope_store_paged", "ls_chunk_attn_paged"):
            monkeypatch.setattr(ls, name, lambda *args, name=name, **kwargs: self.made.append(name))

    def arguments(self, t, **sizes):
        x = lambda name, *rest: torch.zeros((sizes.get(name, t), *rest))  # noqa: E731
        return {"q": x("q", 4, 64), "k": x("k", 2, 64), "v": x("v", 2, 64), "cos_sin": torch.zeros((128, 64)), "q_out": x("q_out", 4, 64)}

    def test_write(self):
        cache = filled_cache([5, 9], 20)
        cache.plan(ints([4, 2]), 8)  # two entries to spare
        cache.write(0, **self.arguments(8))
        cache.write(0, **self.arguments(6))
        cache.write(0, **self.arguments(8), positions=torch.zeros((3, 8), dtype=torch.int32), sections=[8, 12, 12])
        assert self.made == ["ls_rope_store_paged"] * 3
        for sizes in ({"q": 9, "k": 9, "v": 9, "q_out": 9}, {"k": 7}, {"v": 7}, {"q_out": 7}, {"q": 7}):
            with pytest.raises(ValueError):
                cache.write(0, **self.arguments(8, **sizes))
        with pytest.raises(ValueError):
            cache.write(0, **self.arguments(8), positions=torch.zeros((3, 7), dtype=torch.int32), sections=[8, 12, 12])
        for name, bad in (("k", torch.zeros((8, 3, 64))), ("v", torch.zeros((8, 2, 128))), ("q_out", torch.zeros((8, 2, 64))),
                          ("k", torch.zeros((8, 2, 64), dtype=torch.bfloat16)), ("q", torch.zeros((8, 4, 64), dtype=torch.float64))):
            with pytest.raises(ValueError):
                cache.write(0, **{**self.arguments(8), name: bad})
        cache.plan(ints([4, 4]))  # pages only: there are no slots
        with pytest.raises(ValueError):
            cache.write(0, **self.arguments(8))
        assert self.made == ["ls_rope_store_paged"] * 3

    def test_attend(self):
        cache = filled_cache([5, 9], 20)
        cache.plan(ints([4, 2]), 6)
        q, lse = torch.zeros((6, 4, 64), dtype=torch.bfloat16), torch.zeros((6, 4))
        cache.k_pages, cache.v_pages = cache.k_pages.bfloat16(), cache.v_pages.bfloat16()
        cache.attend(0, q, torch.empty_like(q), lse, 4, 20)
        for out, bad_lse in ((torch.empty_like(q)[:5], lse), (torch.empty_like(q), lse[:5]), (torch.empty_like(q), torch.zeros((4, 6)).T),
                             (torch.empty_like(q)[:, :3], lse)):
            with pytest.raises(ValueError):
                cache.attend(0, q, out, bad_lse, 4, 20)
        assert self.made == ["ls_chunk_attn_paged"]

    def test_plan(self):
        cache = filled_cache([5, 9], 20)
        for new_lens in (ints([1]), ints([1, 1]).long(), ints([1, 1, 1])):
            with pytest.raises(ValueError):
                cache.plan(new_lens, 4)
