"""A serving program's state around the entry points of a paged cache: which request holds which pages, and the calls of a
step in their order.  The operators run in the HIP kernels; what is left to torch is the bookkeeping of [batch] integers between them: the
pages held and the free ones taken over after a plan, the lengths after a step, which rows of an accepted path have room.

A step of new tokens (prompts, pieces of prompts, single tokens, any mixture of them):

    cache.plan(new_lens, n_tokens)                                  # ls_page_plan: pages, slots, positions
    for layer in range(n_layers):
        cache.write(layer, q, k, v, cos_sin, q_out)                 # ls_rope_store_paged
        cache.attend(layer, q_out, out, lse, max_new, max_kv)       # ls_chunk_attn_paged
    cache.keep_new()

A verification round over a speculation tree:

    cache.plan(most_accepted)                                       # room for the longest path
    for layer ...: cache.rotate_tree(...); cache.verify(...)        # ls_rope, ls_hybrid_tree_attn_paged
    cache.commit(layers, ...)                                       # ls_kv_commit_paged; surplus pages go back with the next plan

Everything runs on torch's current stream and nothing waits for the GPU: lengths, tables and the number of free pages stay on
the device, so a step can be recorded into a graph and replayed, other steps in between.
`python -m paper_2502_17421_amd.paged_step` runs three requests through both.
"""
from __future__ import annotations

import torch

from . import binding as ls


class PagedCache:
    """max_rows: most rows a request may have (the block table's width in rows)."""

    def __init__(self, batch, n_layers, n_kv_heads, head_dim, n_pages, page_size, max_rows, dtype=torch.bfloat16, device="cuda"):
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.batch, self.n_layers, self.page_size, self.n_pages = batch, n_layers, page_size, n_pages
        self.k_pages = torch.zeros((n_layers, n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device)
        self.v_pages = torch.zeros_like(self.k_pages)
        self.block_table = ints(batch, -(-max_rows // page_size))
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.kv_lens = ints(batch)        # rows cached, before a step's new ones
        self.pages_held, self.free_count = ints(batch), torch.full((1,), n_pages, dtype=torch.int32, device=device)
        self.cu_new, self.total_lens, self.err = ints(batch + 1), ints(batch), ints(batch)
        self._next_held, self._next_free = ints(batch), ints(1)
        self._next_lens = ints(batch)
        self.slots = self.positions = None
        self._buffers = {}

    def _buffer(self, name, size, dtype=torch.uint8):
        """`size` elements or more.  A recorded step goes on using the buffers it was recorded with, so one that a larger step outgrows is
        kept (each is twice the one before, at least: together less than four times what the largest step takes)."""
        kept = self._buffers.setdefault(name, [])
        if not kept or kept[-1].numel() < size:
            kept.append(torch.empty(max([size] + [2 * x.numel() for x in kept]), dtype=dtype, device=self.k_pages.device))
        return kept[-1]

    # ---- the requests' lengths

    def release(self, request):
        """The request has ended: its pages go back with the next plan (its new length must be 0 or a new request's)."""
        self.kv_lens[request] = 0

    def plan(self, new_lens, n_tokens=0):
        """Pages for new_lens (int32 [batch], device) more rows of each request; with n_tokens, the packed tokens' slots and
        positions as well.  err says which requests were refused (they keep what they have)."""
        if new_lens.shape != self.kv_lens.shape or new_lens.dtype != torch.int32:
            raise ValueError(f"new_lens: int32 [{self.batch}]")
        self.slots = self.positions = None
        if n_tokens:
            self.slots = self._buffer("slots", n_tokens, torch.int32)[:n_tokens]
            self.positions = self._buffer("positions", n_tokens, torch.int32)[:n_tokens].view(1, n_tokens)
        ls.ls_page_plan(ls.make_page_desc(self.block_table, n_tokens, self.page_size, self.n_pages), self.kv_lens, new_lens,
                        self.pages_held, self.block_table, self.free_pages, self.free_count, self._next_held, self._next_free,
                        self.cu_new, self.total_lens, self.slots, self.positions, self.err)
        # copied back, not exchanged: a recorded step finds its state in the same place at every replay
        self.pages_held.copy_(self._next_held)
        self.free_count.copy_(self._next_free)

    def keep_new(self):
        """The step's rows have been written: they count as cached (refused requests stay as they were)."""
        self.kv_lens.copy_(torch.where(self.err == 0, self.total_lens, self.kv_lens))

    # ---- new tokens, packed: q [n_tokens, heads, head_dim], k and v [n_tokens, kv heads, head_dim]

    def write(self, layer, q, k, v, cos_sin, q_out, positions=None, sections=None, interleaved=False):
        """positions: [axes, n_tokens] where they are not the rows' own (several axes, say)."""
        positions = self.positions if positions is None else positions
        kp, vp = self.k_pages[layer], self.v_pages[layer]
        n = q.shape[0]
        if self.slots is None or n > self.slots.shape[0] or n > positions.shape[1]:
            raise ValueError("more tokens than were planned")
        if q_out.shape != q.shape or not k.shape == v.shape == (n, kp.shape[1], kp.shape[3]):
            raise ValueError("q_out: the shape of q; k and v: [tokens, kv heads, head_dim] for the same tokens")
        if not q.dtype == k.dtype == v.dtype == q_out.dtype == kp.dtype:
            raise ValueError("q, k, v and q_out: the type of the pages")
        desc = ls.make_rope_desc(q, k, v, q_out, None, kp, vp, positions, cos_sin, sections, interleaved)
        ls.ls_rope_store_paged(desc, q, k, v, positions, cos_sin, self.slots, q_out, kp, vp)

    def attend(self, layer, q, out, lse, max_new, max_kv, window=0):
        """max_new, max_kv: bounds, known to the host, of a request's new tokens and of its rows."""
        if out.shape != q.shape or lse.shape != q.shape[:2] or not lse.is_contiguous():
            raise ValueError("out: the shape of q; lse: [tokens, heads], contiguous")
        kp, vp = self.k_pages[layer], self.v_pages[layer]
        desc = ls.make_chunk_desc(q, kp, vp, self.block_table, out, max_new, max_kv, window)
        ws = self._buffer("chunk", ls.ls_chunk_workspace_bytes(desc))
        ls.ls_chunk_attn_paged(desc, q, kp, vp, self.block_table, self.cu_new, self.total_lens, out, lse, ws)

    # ---- speculation trees: q [batch, heads, nodes, head_dim], k and v [batch, kv heads, nodes, head_dim]

    def rotate_tree(self, q, k, positions, cos_sin, sections=None, interleaved=False):
        """In place; positions: [axes, batch * nodes], a node's row being its request's length plus its depth.  q and k are kept
        token after token (their transposes to [batch, nodes, heads, head_dim] are contiguous)."""
        rows = lambda x: x.transpose(1, 2).flatten(0, 1)  # noqa: E731
        qt, kt = rows(q), rows(k)
        assert qt.data_ptr() == q.data_ptr() and kt.data_ptr() == k.data_ptr(), "trees are kept token after token"
        desc = ls.make_rope_desc(qt, kt, None, qt, kt, None, None, positions, cos_sin, sections, interleaved)
        ls.ls_rope(desc, qt, kt, positions, cos_sin, qt, kt)

    def verify(self, layer, q, k_tree, v_tree, parents, out, lse, max_kv):
        kp, vp = self.k_pages[layer], self.v_pages[layer]
        desc = ls.make_desc(q, kp, vp, k_tree, v_tree, out, max_kv)
        ws = self._buffer("tree", ls.ls_workspace_bytes(desc))
        ls.ls_hybrid_tree_attn_paged(desc, q, kp, vp, self.block_table, self.page_size, self.kv_lens, k_tree, v_tree, parents, out, lse,
                                     ws)

    def commit(self, k_trees, v_trees, accept_path, accept_len):
        """k_trees, v_trees: a tensor per layer.  The accepted rows go into the pages and count as cached, as far as the pages reach that
        the plan before gave the request: a request it refused commits nothing, a path beyond its pages ends with them.  err is then
        1 (or what it was) for requests of which not all rows were committed."""
        room = self.pages_held * self.page_size - self.kv_lens
        fits = torch.where(self.err == 0, torch.minimum(accept_len, room), 0)
        for layer, (k_tree, v_tree) in enumerate(zip(k_trees, v_trees)):
            kp, vp = self.k_pages[layer], self.v_pages[layer]
            desc = ls.make_desc(k_tree, kp, vp, k_tree, v_tree, None, self.block_table.shape[1] * self.page_size)
            ls.ls_kv_commit_paged(desc, k_tree, v_tree, accept_path, fits, self.kv_lens, kp, vp, self.block_table, self.page_size,
                                  self._next_lens)
        self.err.copy_(torch.maximum(self.err, self._next_lens - self.kv_lens < accept_len))
        self.kv_lens.copy_(self._next_lens)


def rotary_table(n_positions, rotary_dim, base=10000.0, device="cuda"):
    """[n_positions, rotary_dim]: the cosines of position / base^(2 i / rotary_dim), then the sines."""
    inv = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def main():
    """Three requests: prompts, a decoding step, a verification round, then one leaves and the others go on."""
    torch.manual_seed(0)
    layers, heads, kv_heads, d, page_size = 2, 32, 8, 128, 16
    cache = PagedCache(3, layers, kv_heads, d, n_pages=512, page_size=page_size, max_rows=4096)
    cos_sin = rotary_table(4096, d)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    randn = lambda *shape: torch.randn(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731

    def step(news, max_kv):
        t = sum(news)
        cache.plan(ints(news), t)
        for layer in range(layers):
            q, out, lse = randn(t, heads, d), randn(t, heads, d), torch.empty((t, heads), device="cuda")
            cache.write(layer, q, randn(t, kv_heads, d), randn(t, kv_heads, d), cos_sin, q)
            cache.attend(layer, q, out, lse, max(news), max_kv)
        cache.keep_new()
        report(f"new tokens {news}")

    def report(what):
        print(f"{what}: rows {cache.kv_lens.tolist()}, pages {cache.pages_held.tolist()}, free {cache.free_count.item()}", flush=True)

    step([1000, 37, 300], 1000)
    step([1, 1, 1], 1001)
    parents, depth = ints([[-1, 0, 0, 1, 1, 3]] * 3), [0, 1, 1, 2, 2, 3]  # a tree of six nodes, four deep
    cache.plan(ints([4, 4, 4]))
    k_trees, v_trees = [], []
    for layer in range(layers):
        tree = lambda h: randn(3, 6, h, d).transpose(1, 2)  # noqa: E731
        q, k, v, out = tree(heads), tree(kv_heads), tree(kv_heads), tree(heads)
        cache.rotate_tree(q, k, (cache.kv_lens[:, None] + ints(depth)).flatten()[None], cos_sin)
        cache.verify(layer, q, k, v, parents, out, torch.empty((3, heads, 6), device="cuda"), 1001)
        k_trees.append(k)
        v_trees.append(v)
    path, accepted, following, err = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((3, 6), (3,), (3,), (3,)))
    ls.ls_tree_accept_greedy(parents, ints([[0, 7, 8, 9, 5, 4]] * 3), ints([[7, 9, 0, 4, 0, 2], [8, 0, 3, 0, 0, 0], [6, 0, 0, 0, 0, 0]]),
                             path, accepted, following, err)
    cache.commit(k_trees, v_trees, path, accepted)
    report(f"accepted {accepted.tolist()}")
    cache.release(1)
    step([1, 0, 500], 1006)


if __name__ == "__main__":
    main()
