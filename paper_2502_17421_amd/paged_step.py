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
    cache.accept(...)                                               # at a temperature: ls_tree_accept_sampled
    cache.commit(layers, ...)                                       # ls_kv_commit_paged; surplus pages go back with the next plan

Several continuations of a prompt, beams, requests that go back to earlier rows:

    cache.fork(sources)                                             # ls_page_fork, ls_page_copy: full pages are shared
    cache.compact()                                                 # ls_page_compact, ls_page_copy: pages in use to the front of the pool

A fork ends a step that has been planned and not kept or committed yet; a release does not, nor does a compaction, but for the slots.

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
        self._next_table = torch.zeros_like(self.block_table)  # of forks and compactions
        self._n_copies = ints(1)
        self._fork_err = ints(batch)
        self._may_share = False  # a fork or compaction has run, or has been recorded
        self._ended = False      # a fork has ended the last plan
        self._recorded = False   # a plan has been recorded: replays are plans that nothing here sees

    def _buffer(self, name, size, dtype=torch.uint8):
        """`size` elements or more.  A recorded step goes on using the buffers it was recorded with, so one that a larger step outgrows is
        kept (each is twice the one before, at least: together less than four times what the largest step takes)."""
        kept = self._buffers.setdefault(name, [])
        if not kept or kept[-1].numel() < size:
            kept.append(torch.empty(max([size] + [2 * x.numel() for x in kept]), dtype=dtype, device=self.k_pages.device))
        return kept[-1]

    def _check_ints(self, names, *given):
        for x in given:
            if x.shape != self.kv_lens.shape or x.dtype != torch.int32 or x.device != self.kv_lens.device or not x.is_contiguous():
                raise ValueError(f"{names}: int32 [{self.batch}], contiguous, on the cache's device")

    # ---- the requests' lengths

    def release(self, request):
        """The request has ended: its pages go back with the next plan (its new length must be 0 or a new request's).  Where requests may
        share pages, by a fork: at once, those that nobody else holds; so too in a recording, which may be replayed after a fork.
        In a step that has been planned it counts as refused from now on (err is 1); the others go on with the pages they were given."""
        for x, value in ((self.kv_lens, 0), (self.total_lens, 0), (self.err, 1)):
            self._set(x, request, value)
        if not self._may_share and not self._recording():
            return
        # (what ls_page_fork does with requests whose source is none: they keep all they hold, and what was reserved for a step)
        sources = torch.full_like(self.kv_lens, -2)
        self._set(sources, request, -1)
        self._next_table.copy_(self.block_table)
        self._fork(sources, None, self._fork_err)

    # ---- requests that share pages

    @staticmethod
    def _set(x, request, value):
        if type(request) is int:
            x[request].fill_(value)  # (an assignment brings the value from the host, which a recording refuses)
        else:
            x[request] = value

    def _recording(self):
        return self.kv_lens.is_cuda and torch.cuda.is_current_stream_capturing()

    def _move_rows(self, copies):
        desc = ls.make_copy_desc(self.k_pages, self.v_pages, copies.shape[0])
        ls.ls_page_copy(desc, copies, self._n_copies, self.k_pages, self.v_pages)

    def _fork(self, sources, keep_lens, err):
        self._may_share = True
        desc = ls.make_page_desc(self.block_table, 0, self.page_size, self.n_pages)
        copies = self._buffer("fork copies", 4 * self.batch, torch.int32)[:4 * self.batch].view(-1, 4)
        ls.ls_page_fork(desc, sources, keep_lens, self.kv_lens, self.pages_held, self.block_table, self.free_pages, self.free_count, self._next_table,
                        self._next_lens, self._next_held, self._next_free, copies, self._n_copies, err,
                        self._buffer("fork", ls.ls_page_fork_workspace_bytes(desc)))
        for kept, made in ((self.block_table, self._next_table), (self.kv_lens, self._next_lens), (self.pages_held, self._next_held),
                           (self.free_count, self._next_free)):
            kept.copy_(made)
        return copies

    def fork(self, sources, keep_lens=None):
        """Request b goes on from the rows (the first keep_lens[b]) of request sources[b], -1: from none, as they are now; int32 [batch], device.
        Full pages are shared, of a page filled in part every request but one gets a copy, and pages that nobody holds any more are free
        at once, those that a plan reserved among them: the step is over, and what comes next has to be planned.
        err: 1 where no page was left for the copy (the request then ends with its full pages), 2 for sources or lengths that are none."""
        self._check_ints("sources, keep_lens", *((sources,) if keep_lens is None else (sources, keep_lens)))
        self._move_rows(self._fork(sources, keep_lens, self.err))
        self.slots = self.positions = None
        self.total_lens.copy_(self.kv_lens)  # (of a recorded plan: nothing is new)
        self._ended = True

    def compact(self):
        """The pages in use to the front of the pool: afterwards they are 0 .. n_pages - free_count - 1.  Rows of a step that are still to be
        written have to be planned again."""
        self._may_share = True
        desc = ls.make_page_desc(self.block_table, 0, self.page_size, self.n_pages)
        n = self.n_pages // 2 + 1
        copies = self._buffer("compact copies", 4 * n, torch.int32)[:4 * n].view(-1, 4)
        ls.ls_page_compact(desc, self.pages_held, self.block_table, self._next_table, self.free_pages, self.free_count, copies, self._n_copies,
                           self._buffer("compact", ls.ls_page_compact_workspace_bytes(desc)))
        self._move_rows(copies)
        self.block_table.copy_(self._next_table)
        self.slots = self.positions = None  # (they say where the pages were)

    def plan(self, new_lens, n_tokens=0):
        """Pages for new_lens (int32 [batch], device) more rows of each request; with n_tokens, the packed tokens' slots and
        positions as well.  err says which requests were refused (they keep what they have)."""
        self._check_ints("new_lens", new_lens)
        self.slots = self.positions = None
        self._ended, self._recorded = False, self._recorded or self._recording()
        if n_tokens:
            self.slots = self._buffer("slots", n_tokens, torch.int32)[:n_tokens]
            self.positions = self._buffer("positions", n_tokens, torch.int32)[:n_tokens].view(1, n_tokens)
        ls.ls_page_plan(ls.make_page_desc(self.block_table, n_tokens, self.page_size, self.n_pages), self.kv_lens, new_lens,
                        self.pages_held, self.block_table, self.free_pages, self.free_count, self._next_held, self._next_free,
                        self.cu_new, self.total_lens, self.slots, self.positions, self.err)
        # copied back, not exchanged: a recorded step finds its state in the same place at every replay
        self.pages_held.copy_(self._next_held)
        self.free_count.copy_(self._next_free)

    def _check_plan(self):
        if self._ended and not self._recorded and not self._recording():
            raise RuntimeError("a fork has ended the step: it has to be planned again")

    def keep_new(self):
        """The step's rows have been written: they count as cached (refused requests stay as they were)."""
        self._check_plan()
        self.kv_lens.copy_(torch.where(self.err == 0, self.total_lens, self.kv_lens))

    # ---- new tokens, packed: q [n_tokens, heads, head_dim], k and v [n_tokens, kv heads, head_dim]

    def write(self, layer, q, k, v, cos_sin, q_out, positions=None, sections=None, interleaved=False):
        """positions: [axes, n_tokens] where they are not the rows' own (several axes, say)."""
        positions = self.positions if positions is None else positions
        kp, vp = self.k_pages[layer], self.v_pages[layer]
        n = q.shape[0]
        if self.slots is None or n > self.slots.shape[0] or n > positions.shape[1]:
            raise ValueError("more tokens than were planned (a fork or a compaction takes the slots away)")
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

    def accept(self, parents, draft_tokens, target_logits, draft_logits, temperature, accept_uniforms, sample_uniforms, accept_path,
               accept_len, next_token, logprobs=None, err=None, draft_temperature=None, with_replacement=False):
        """Acceptance of the drafted trees at a temperature, from given random numbers; draft_logits None: the drafted tokens were chosen."""
        desc = ls.make_sample_desc(target_logits, draft_logits, with_replacement)
        ws = self._buffer("sample", ls.ls_sample_workspace_bytes(desc))
        ls.ls_tree_accept_sampled(desc, parents, draft_tokens, target_logits, draft_logits, temperature, draft_temperature, accept_uniforms,
                                  sample_uniforms, accept_path, accept_len, next_token, logprobs, err, ws)

    def commit(self, k_trees, v_trees, accept_path, accept_len):
        """k_trees, v_trees: a tensor per layer.  The accepted rows go into the pages and count as cached, as far as the pages reach that
        the plan before gave the request: a request it refused commits nothing, a path beyond its pages ends with them.  err is then
        1 (or what it was) for requests of which not all rows were committed."""
        self._check_plan()
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
    # the third request goes on in two ways: its tree is drawn by a draft model and verified at a temperature, in each of them
    cache.fork(ints([0, 2, 2]))
    report("forked")
    cache.plan(ints([4, 4, 4]))
    vocab, uniforms = 32000, torch.rand((3, 6), device="cuda")
    target = 4 * randn(3, 6, vocab)
    draft = target + 0.5 * randn(3, 6, vocab)
    tokens = torch.zeros_like(parents)
    for node, above in ((1, 0), (3, 1), (5, 3), (2, 0), (4, 1)):  # (independent draws)
        tokens[:, node] = torch.multinomial(torch.softmax(draft[:, above].float(), -1), 1)[:, 0].to(torch.int32)
    logprobs = torch.empty((3, 6), device="cuda")
    cache.accept(parents, tokens, target, draft, torch.ones(3, device="cuda"), uniforms, torch.rand(3, device="cuda"), path, accepted, following,
                 logprobs, err, with_replacement=True)
    cache.commit(k_trees, v_trees, path, accepted)
    report(f"accepted at a temperature {accepted.tolist()}")
    cache.compact()
    report("compacted")


if __name__ == "__main__":
    main()
