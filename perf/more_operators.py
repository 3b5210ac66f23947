"""Performance cases: sampled decoding of several continuations of a prompt with speculation trees, over a paged cache.

A prompt's request is forked into its samples (or the beams of a search are dealt anew): full pages are shared by
block tables, and only the page that a request goes on writing in is copied.  The tree that each of them drafts is
verified against the target's distribution by rejection from given random numbers.  As requests come and go
the pages in use scatter over the pool; compaction moves them to its front.

A case's "kind":
  verify   ls_tree_accept_sampled  accepted path, next token and their log probabilities from both models' logits
  fork     ls_page_fork            block tables of forked, reordered and ended requests, and the pages to be copied
  compact  ls_page_compact         pages in use to the front of the pool: tables, free pages, and the pages to be copied
  copy     ls_page_copy            rows of K and V pages of all layers to other pages of the same pool

The plain forms use elementary torch operations; the verification computes in 64 bits, because a token drawn from a
cumulative sum over a vocabulary lies next to a border in 32.  exact() is the verification's definition, distribution by distribution;
the other operators give whole numbers or copies.
"""
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
# (KV heads, head_dim): 8B-class GQA, 7B-class MHA, a small model's heads
HEADS_8B, HEADS_MHA, HEADS_SMALL = (8, 128), (32, 128), (4, 64)


def _verify(name, batch, widths, vocab, dtype, draft_dtype, drawn=True, with_replacement=False, noise=0.7, greedy=0):
    """widths: children of every node, level by level, as text ("4,2,1"); or "beam:4,16,16": nodes of each level, under random nodes
    of the one above.  drawn: the draft's tokens were drawn from its logits (else chosen, and the draft's logits play no part).
    noise: the draft's logits are the target's and so much of a normal value.  greedy: so many requests have temperature 0."""
    return {"name": name, "kind": "verify", "batch": batch, "widths": widths, "vocab": vocab, "dtype": dtype, "draft_dtype": draft_dtype,
            "drawn": drawn, "with_replacement": with_replacement, "noise": noise, "greedy": greedy}


def _fork(name, groups, samples, prompt, tail, page_size, ended=0, short=0):
    """groups of `samples` requests; prompt[0] to prompt[1] rows that a group shares, then `tail` rows of each member (0: only the first
    member of each group is there yet).  The last `ended` groups end.  short: so many pages are missing for the copies."""
    return {"name": name, "kind": "fork", "groups": groups, "samples": samples, "prompt_lo": prompt[0], "prompt_hi": prompt[1],
            "tail": tail, "page_size": page_size, "ended": ended, "short": short}


def _compact(name, batch, rows, page_size, n_pages, samples=1):
    """batch requests of rows[0] to rows[1] rows anywhere in the pool; `samples` of them in a row share all but their last page."""
    return {"name": name, "kind": "compact", "batch": batch, "rows_lo": rows[0], "rows_hi": rows[1], "page_size": page_size,
            "n_pages": n_pages, "samples": samples}


def _copy(name, copies, layers, heads, page_size, dtype, n_pages, whole=False, token_major=False):
    """whole: all rows of each page, as after compaction; else a random part, as after a fork."""
    return {"name": name, "kind": "copy", "copies": copies, "layers": layers, "n_kv_heads": heads[0], "head_dim": heads[1],
            "page_size": page_size, "dtype": dtype, "n_pages": n_pages, "whole": whole, "token_major": token_major}


def listed():
    return [
        # One chat, a small tree over a vocabulary of 32000: latency.
        _verify("verify_chat", 1, "3,2,1,1", 32000, "f16", "f16"),
        # The beam tree of 69 nodes, whose tokens are chosen and not drawn; logits in float as a head leaves them that is not cast.
        _verify("verify_beam", 4, "beam:4,16,16,16,16", 32000, "f32", "f32", drawn=False),
        # Plain speculative sampling of a serving batch: a chain of five tokens, large vocabulary.
        _verify("verify_chain", 48, "1,1,1,1,1", 128256, "bf16", "bf16", noise=0.5),
        # Trees of drawn tokens for a batch of requests over the largest vocabulary.
        _verify("verify_trees", 16, "4,3,2,1", 152064, "bf16", "bf16"),
        # An odd vocabulary (no row but the first is aligned), float draft logits, independent draws, three of the requests greedy.
        _verify("verify_odd", 11, "3,2,2", 50257, "f16", "f32", with_replacement=True, noise=1.0, greedy=3),
        # Eight prompts become eight samples each.
        _fork("fork_samples", 8, 8, (1003, 8111), 0, 16),
        # A step of beam search, 4 beams for each of 64 requests: every beam goes on from one of its group.
        _fork("fork_beams", 64, 4, (211, 4001), 333, 16, ended=3),
        # A server's pool, half empty and scattered.
        _compact("compact_server", 64, (37, 8111), 16, 40000),
        # A large pool of small pages with shared prompts.
        _compact("compact_large", 512, (500, 6007), 16, 262144, samples=4),
        # The partly filled pages after one prompt was forked, two layers at a time: latency.
        _copy("copy_few", 3, 2, HEADS_8B, 16, "bf16", 64),
        # The copies of a step of beam search through all layers of a small model in float, rows token after token.
        _copy("copy_beams", 150, 16, HEADS_SMALL, 32, "f32", 500, token_major=True),
        # Whole pages after a compaction.
        _copy("copy_compact", 900, 8, HEADS_8B, 16, "bf16", 2048, whole=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case of the same ranges.  What would cost more than the largest listed case of its kind is drawn again."""
    most = {}
    for case in listed():
        most[case["kind"]] = max(most.get(case["kind"], 0), work(case)["bytes"])
    while True:
        kind = rng.choice(["verify", "verify", "verify", "fork", "compact", "copy"])
        page_size = rng.choice([16, 16, 32, 64, 128])
        if kind == "verify":
            widths = rng.choice(["1,1", "1,1,1,1,1,1,1", "2,2,2,1,1", "4,3,2,1", "8,2", "16,1,1", "5", "beam:4,16,16,16,16", "beam:3,7,11", "0"])
            drawn = not widths.startswith("beam") and rng.random() < 0.8
            batch = _log_int(rng, 1, 64)
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            vocab = rng.choice([32000, 32003, 50257, 64000, 128256, 152064, _log_int(rng, 1000, 200000)])
            case = _verify("", batch, widths, vocab, dtype, rng.choice([dtype, dtype, "f32"]), drawn=drawn,
                           with_replacement=rng.random() < 0.4, noise=rng.choice([0.2, 0.7, 1.5]), greedy=rng.choice([0, 0, batch // 3]))
            if batch * _nodes(case) * vocab > 250_000_000:
                continue
        elif kind == "fork":
            groups, samples = _log_int(rng, 1, 120), rng.choice([1, 2, 3, 4, 8, 16])
            lo = _log_int(rng, 1, 3000)
            case = _fork("", groups, samples, (lo, lo + _log_int(rng, 1, 6000)), rng.choice([0, 0, _log_int(rng, 1, 900)]), page_size,
                         ended=rng.choice([0, 0, groups // 5]), short=rng.choice([0, 0, 0, groups // 2]))
        elif kind == "compact":
            batch, lo = _log_int(rng, 1, 600), _log_int(rng, 1, 1500)
            hi = lo + _log_int(rng, 1, 6000)
            n_pages = (hi // page_size + 2) * batch
            n_pages = int(n_pages * rng.choice([1.0, 1.2, 2.0]))
            case = _compact("", batch, (lo, hi), page_size, n_pages, samples=rng.choice([1, 1, 2, 4]))
            if n_pages > 300_000:
                continue
        else:
            heads = rng.choice([HEADS_8B, HEADS_8B, HEADS_MHA, HEADS_SMALL])
            copies = _log_int(rng, 1, 900)
            case = _copy("", copies, _log_int(rng, 1, 32), heads, page_size, rng.choice(["bf16", "bf16", "f16", "f32"]),
                         2 * copies + rng.randint(1, 100), whole=rng.random() < 0.5, token_major=rng.random() < 0.4)
            if _pool_bytes(case) > 3 << 30:
                continue
        del case["name"]
        if work(case)["bytes"] <= most[kind]:
            return case


def _pool_bytes(case):
    return 2 * case["layers"] * case["n_pages"] * case["n_kv_heads"] * case["page_size"] * case["head_dim"] * BYTES[case["dtype"]]


def _levels(case):
    """Nodes of each level below the root, and the most children that a node may have."""
    text = case["widths"]
    numbers = [int(n) for n in text.removeprefix("beam:").split(",")]
    if text.startswith("beam:"):
        return numbers, max(numbers)
    nodes, at = [], 1
    for n in numbers:
        at *= n
        if at:
            nodes.append(at)
    return nodes, max(numbers)


def _nodes(case):
    return 1 + sum(_levels(case)[0])


def _rows_of(lo, hi, n):
    """n lengths between the two, in an order that belongs to them."""
    rows = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    random.Random(1000 * n + lo).shuffle(rows)
    return rows


def _pages(rows, size):
    return (rows + size - 1) // size


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    """The inputs, the buffers that a program reuses, and its descriptor and workspace."""
    st = {"verify": _verify_inputs, "fork": _fork_inputs, "compact": _compact_inputs, "copy": _copy_inputs}[case["kind"]](case, seed)
    st["case"] = case
    if not own:
        return st
    from paper_2502_17421_amd import binding as ls
    if case["kind"] == "verify":
        st["desc"] = ls.make_sample_desc(st["target"], st["draft"], with_replacement=case["with_replacement"])
        size = ls.ls_sample_workspace_bytes(st["desc"])
    elif case["kind"] == "fork":
        st["desc"] = ls.make_page_desc(st["table"], n_tokens=0, page_size=case["page_size"], n_pages=st["n_pages"])
        size = ls.ls_page_fork_workspace_bytes(st["desc"])
    elif case["kind"] == "compact":
        st["desc"] = ls.make_page_desc(st["table"], n_tokens=0, page_size=case["page_size"], n_pages=case["n_pages"])
        size = ls.ls_page_compact_workspace_bytes(st["desc"])
    else:
        st["desc"] = ls.make_copy_desc(st["k"], st["v"], max_copies=case["copies"])
        size = 0
    st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return st


def _tree(case, rng):
    """Parents of one tree, level by level: all nodes of a level have as many children, or they hang under random ones."""
    nodes, _ = _levels(case)
    parents, above = [-1], [0]
    for n in nodes:
        first = len(parents)
        if case["widths"].startswith("beam:"):
            parents += sorted(rng.choice(above) for _ in range(n))
        else:
            parents += [p for p in above for _ in range(n // len(above))]
        above = list(range(first, first + n))
    return parents


def _verify_inputs(case, seed):
    gen, rng = _generator(seed), random.Random(seed)
    b, t, v = case["batch"], _nodes(case), case["vocab"]
    parents = _ints([_tree(case, rng) for _ in range(b)])
    # logits as peaked as a language model's: the likeliest token has a tenth of the weight or more
    base = torch.randn((b, t, v), generator=gen, device="cuda", dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16) * 4
    target = base.to(DTYPES[case["dtype"]])
    temperature = 0.6 + 0.6 * torch.rand(b, generator=gen, device="cuda")
    draft = None
    if case["drawn"]:
        draft = (base + case["noise"] * torch.randn(base.shape, generator=gen, device="cuda", dtype=base.dtype)).to(DTYPES[case["draft_dtype"]])
        del base
    tokens = torch.randint(0, v, (b, t), generator=gen, device="cuda")
    kids, there = _children(parents, max(1, _levels(case)[1]))
    for i in range(b):  # a request's tokens: drawn from the draft's distribution at their parent, or the likeliest
        inner = there[i].any(-1)
        rows = (target if draft is None else draft)[i][inner].float()
        if not rows.numel():
            continue
        if draft is None:
            drawn = rows.topk(kids.shape[-1]).indices
        else:
            drawn = torch.multinomial(torch.softmax(rows / temperature[i], -1), kids.shape[-1], case["with_replacement"], generator=gen)
        ours = there[i][inner]
        tokens[i, kids[i][inner][ours]] = drawn[ours]
    # a few requests whose temperature is 0 among the others
    temperature[torch.randperm(b, generator=gen, device="cuda")[:case["greedy"]]] = 0
    out = {"path": torch.zeros((b, t), dtype=torch.int32, device="cuda"), "len": _ints([0] * b), "next": _ints([0] * b),
           "logprobs": torch.zeros((b, t), device="cuda"), "err": _ints([0] * b)}
    return {"parents": parents, "tokens": tokens.to(torch.int32), "target": target, "draft": draft, "temperature": temperature,
            "draft_temperature": torch.where(temperature > 0, temperature, 1.0),
            "accept_uniforms": torch.rand((b, t), generator=gen, device="cuda"),
            "sample_uniforms": torch.rand(b, generator=gen, device="cuda"), "out": out}


def _scattered(entries, n_pages, seed):
    """Pages for so many entries in random order, and the others: a stack of free ones, as long as the pool."""
    order = torch.randperm(n_pages, generator=_generator(seed), device="cuda").to(torch.int32)
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - entries] = order[entries:]
    return order[:entries], free


def _shared_table(shared, pages, samples, width):
    """Which entry of a list of pages each place of a table holds: `samples` requests in a row share their first `shared` pages.
    Returns the places [batch, width] (-1: none) and the length of the list."""
    places, at = [], 0
    for b, (s, n) in enumerate(zip(shared, pages)):
        s = min(s, n)
        if b % samples == 0:
            first, at = at, at + s
        places.append(list(range(first, first + s)) + list(range(at, at + n - s)) + [-1] * (width - n))
        at += n - s
    return torch.tensor(places, device="cuda"), at


def _fork_rows(case):
    """Rows of every request before, and of its group's prompt."""
    size, n = case["samples"], case["groups"]
    prompt = [r for r in _rows_of(case["prompt_lo"], case["prompt_hi"], n) for _ in range(size)]
    rows = [p + case["tail"] if case["tail"] or b % size == 0 else 0 for b, p in enumerate(prompt)]
    return rows, prompt


def _fork_inputs(case, seed):
    size, samples, b = case["page_size"], case["samples"], case["groups"] * case["samples"]
    rows, prompt = _fork_rows(case)
    held = [_pages(r, size) for r in rows]
    width = max(held) + 2
    places, used = _shared_table([p // size for p in prompt], held, samples, width)
    spare = max(0, b - case["short"])
    pages, free = _scattered(used, used + spare + 7, seed)
    table = torch.where(places >= 0, pages[places.clamp(min=0)], 0)
    rng = random.Random(seed)
    sources = [-1 if i // samples >= case["groups"] - case["ended"] else i // samples * samples + (rng.randrange(samples) if case["tail"] else 0)
               for i in range(b)]
    count = max(0, spare - case["short"])
    out = {"table": torch.zeros_like(table), "kv_lens": _ints([0] * b), "held": _ints([0] * b), "free_count": _ints([0]),
           "copies": torch.full((b, 4), -1, dtype=torch.int32, device="cuda"), "n_copies": _ints([0]), "err": _ints([0] * b)}
    return {"table": table, "kv_lens": _ints(rows), "held": _ints(held), "sources": _ints(sources), "free": free, "free_count": _ints([count]),
            "n_pages": free.numel(), "out": out}


def _compact_rows(case):
    return _rows_of(case["rows_lo"], case["rows_hi"], case["batch"])


def _compact_inputs(case, seed):
    size = case["page_size"]
    held = [_pages(r, size) for r in _compact_rows(case)]
    first = [held[b // case["samples"] * case["samples"]] - 1 for b in range(case["batch"])]
    places, used = _shared_table(first, held, case["samples"], max(held) + 1)
    pages, free = _scattered(used, case["n_pages"], seed)
    table = torch.where(places >= 0, pages[places.clamp(min=0)], 0)
    out = {"table": torch.zeros_like(table), "free_count": _ints([0]), "n_copies": _ints([0]),
           "copies": torch.full((case["n_pages"] // 2 + 1, 4), -1, dtype=torch.int32, device="cuda")}
    return {"table": table, "held": _ints(held), "free": free, "out": out}


def _copy_inputs(case, seed):
    gen = _generator(seed)
    hkv, size, d, dtype = case["n_kv_heads"], case["page_size"], case["head_dim"], DTYPES[case["dtype"]]
    shape = (case["layers"], case["n_pages"], size, hkv, d) if case["token_major"] else (case["layers"], case["n_pages"], hkv, size, d)
    pools = [torch.randn(shape, generator=gen, device="cuda", dtype=dtype) for _ in range(2)]
    pools = [p.transpose(2, 3) if case["token_major"] else p for p in pools]
    n = case["copies"]
    order = torch.randperm(case["n_pages"], generator=gen, device="cuda").to(torch.int32)
    rows = torch.full((n,), size, device="cuda") if case["whole"] else torch.randint(1, size, (n,), generator=gen, device="cuda")
    copies = torch.stack([order[:n], order[n:2 * n], rows.to(torch.int32), torch.arange(n, device="cuda", dtype=torch.int32)], 1)
    return {"k": pools[0], "v": pools[1], "copies": copies.contiguous(), "n_copies": _ints([n])}


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"verify": _plain_verify, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy}[st["case"]["kind"]](st)


def _run_own(st):
    from paper_2502_17421_amd import binding as ls
    kind, out = st["case"]["kind"], st.get("out")
    if kind == "verify":
        ls.ls_tree_accept_sampled(st["desc"], st["parents"], st["tokens"], st["target"], st["draft"], st["temperature"],
                                  st["draft_temperature"], st["accept_uniforms"], st["sample_uniforms"], out["path"], out["len"],
                                  out["next"], out["logprobs"], out["err"], st["workspace"])
        return out
    if kind == "fork":
        ls.ls_page_fork(st["desc"], st["sources"], None, st["kv_lens"], st["held"], st["table"], st["free"], st["free_count"],
                        out["table"], out["kv_lens"], out["held"], out["free_count"], out["copies"], out["n_copies"], out["err"],
                        st["workspace"])
        return {**out, "free": st["free"]}
    if kind == "compact":
        ls.ls_page_compact(st["desc"], st["held"], st["table"], out["table"], st["free"], out["free_count"], out["copies"],
                           out["n_copies"], st["workspace"])
        return {**out, "free": st["free"]}
    ls.ls_page_copy(st["desc"], st["copies"], st["n_copies"], st["k"], st["v"])
    return [st["k"], st["v"]]


def _children(parents, most):
    """[batch, node, most]: the children of each node in the order of their indices, and which of these places are taken."""
    b, t = parents.shape
    node = torch.arange(t, device="cuda")
    older = ((parents[:, :, None] == parents[:, None, :]) & (node[:, None] > node)).sum(-1)  # siblings before a node
    kids = torch.full((b, t + 1, most + 1), -1, device="cuda")
    above = torch.where(parents < 0, t, parents).long()
    kids[torch.arange(b, device="cuda")[:, None], above, older.clamp(max=most)] = node.expand(b, t)
    kids = kids[:, :t, :most]
    return kids, kids >= 0


def _plain_verify(st):
    """All requests walk their trees together.  With the target's probabilities p, the draft's q, and the children of a node in
    their order, a child of token x is accepted if p(x) - a q(x) > u q(x) S / W, where S = sum max(p - a q, 0) and W = the mass of q left;
    otherwise a grows by S / W.  The next token is drawn from max(p - a q, 0)."""
    case, parents, tokens = st["case"], st["parents"], st["tokens"].long()
    b, t = parents.shape
    nodes, most = _levels(case)
    request = torch.arange(b, device="cuda")
    kids, there = _children(parents, most)
    greedy = st["temperature"] == 0
    heat = torch.where(greedy, 1.0, st["temperature"]).double()[:, None]
    current, on_the_way = torch.zeros_like(request), torch.ones_like(greedy)
    path = torch.full((b, t), -1, device="cuda")
    path[:, 0] = 0
    length, following = torch.ones_like(request), torch.zeros_like(request)
    logprobs = torch.zeros((b, t), dtype=torch.float64, device="cuda")
    for _ in range(len(nodes) + 1):
        logits = st["target"][request, current].double() / heat
        log_p = logits - logits.amax(-1, keepdim=True)
        log_p = log_p - log_p.exp().sum(-1, keepdim=True).log()
        p = log_p.exp()
        best = torch.zeros_like(p).scatter_(1, logits.argmax(-1, keepdim=True), 1.0)
        p = torch.where(greedy[:, None], best, p)
        if st["draft"] is not None:
            q = st["draft"][request, current].double() / st["draft_temperature"].double()[:, None]
            q = (q - q.amax(-1, keepdim=True)).exp()
            q = q / q.sum(-1, keepdim=True)
            q = torch.where(greedy[:, None], 0.0, q)
        else:
            q = torch.zeros_like(p)
        chosen = greedy if st["draft"] is not None else torch.ones_like(greedy)  # a token that was not drawn: q is 1 there
        a, mass, left = torch.zeros_like(heat), torch.ones_like(heat), torch.ones_like(heat)
        next_node = torch.full_like(current, -1)
        for rank in range(most):
            child, is_child = kids[request, current, rank], there[request, current, rank]
            token = tokens[request, child.clamp(min=0)][:, None]
            u = st["accept_uniforms"][request, child.clamp(min=0)].double()[:, None]
            px, qx = p.gather(1, token), q.gather(1, token)
            qx = torch.where(chosen[:, None], 1.0, qx)
            gain = torch.where(chosen[:, None], px, px - a * qx)
            passed = (gain * left > u * qx * mass)[:, 0] & is_child & (next_node < 0)
            next_node = torch.where(passed, child, next_node)
            refused = (is_child & (next_node < 0))[:, None]
            a = torch.where(refused & ~chosen[:, None], a + mass / left, a)
            p = torch.where(refused, p.scatter(1, token, 0.0), p)
            q = torch.where(refused, q.scatter(1, token, 0.0), q)
            if not case["with_replacement"]:
                left = torch.where(refused & ~chosen[:, None], q.sum(-1, keepdim=True), left)
            mass = torch.where(refused, (p - a * q).clamp(min=0).sum(-1, keepdim=True), mass)
        residual = (p - a * q).clamp(min=0)
        border = residual.cumsum(-1)
        drawn = (border > st["sample_uniforms"].double()[:, None] * border[:, -1:]).to(torch.int8).argmax(-1)
        ends, goes_on = on_the_way & (next_node < 0), on_the_way & (next_node >= 0)
        following = torch.where(ends, drawn, following)
        emitted = torch.where(next_node >= 0, tokens[request, next_node.clamp(min=0)], drawn)[:, None]
        at = (length - 1)[:, None]
        logprobs = torch.where(on_the_way[:, None], logprobs.scatter(1, at, log_p.gather(1, emitted)), logprobs)
        path = torch.where(goes_on[:, None], path.scatter(1, length.clamp(max=t - 1)[:, None], next_node[:, None]), path)
        length = length + goes_on
        current = torch.where(goes_on, next_node, current)
        on_the_way = goes_on
    return {"path": path.to(torch.int32), "len": length.to(torch.int32), "next": following.to(torch.int32), "logprobs": logprobs.float(),
            "err": torch.zeros_like(length).to(torch.int32)}


def _plain_fork(st):
    """Request b goes on from the rows of request sources[b].  Full pages are shared.  A page that is partly filled stays with the lowest
    request that goes on in it, unless another one holds it as a full page; the others get a page of their own, and a copy."""
    size, table = st["case"]["page_size"], st["table"].long()
    b, width = table.shape
    n_pages, request, column = st["n_pages"], torch.arange(b, device="cuda"), torch.arange(width, device="cuda")
    from_ = st["sources"].long()
    rows = torch.where(from_ >= 0, st["kv_lens"].long()[from_.clamp(min=0)], 0)
    full, part = rows // size, rows % size
    new = table[from_.clamp(min=0)]
    kept = column < full[:, None]
    as_full = torch.bincount(new[kept], minlength=n_pages)
    has_part = part > 0
    page = new.gather(1, full.clamp(max=width - 1)[:, None])[:, 0]
    heir = torch.full((n_pages + 1,), b, device="cuda").scatter_reduce(0, torch.where(has_part, page, n_pages), request, "amin")
    keeps = has_part & (as_full[page] == 0) & (heir[page] == request)
    copies = has_part & ~keeps
    still = as_full > 0
    still[page[keeps]] = True
    # pages that nobody holds any more, in the order in which the requests held them
    old = table[column < st["held"][:, None]]
    place = torch.arange(old.numel(), device="cuda")
    first = torch.full((n_pages,), old.numel(), device="cuda").scatter_reduce(0, old, place, "amin")
    given = old[~still[old] & (first[old] == place)]
    free, count = st["free"].clone(), st["free_count"].long()
    free[count + torch.arange(given.numel(), device="cuda")] = given.to(torch.int32)
    top = count + given.numel()
    order = copies.cumsum(0)
    refused = copies & (order > top)
    copies = copies & ~refused
    fresh = free[(top - order).clamp(min=0)].long()
    holds = full + (has_part & ~refused)
    out = torch.zeros_like(table)
    out[kept] = new[kept]
    has = holds > full
    out[request[has], full[has]] = torch.where(copies, fresh, page)[has]
    entries = torch.full((b, 4), -1, dtype=torch.int32, device="cuda")
    n = copies.sum()
    entries[:n] = torch.stack([page, fresh, part, request], 1)[copies].to(torch.int32)
    whole = {"table": out, "kv_lens": torch.where(refused, full * size, rows), "held": holds, "free_count": top - n, "copies": entries,
             "n_copies": n[None], "err": refused, "free": free}
    return {key: x.to(torch.int32) for key, x in whole.items()}


def _plain_compact(st):
    """The pages in use keep their number if it is below their count n; the others, in ascending order, get those below n that are free."""
    table, n_pages = st["table"].long(), st["case"]["n_pages"]
    inside = torch.arange(table.shape[1], device="cuda") < st["held"][:, None]
    used = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    used[table[inside]] = True
    n, page = used.sum(), torch.arange(n_pages, device="cuda")
    from_, to = page[used & (page >= n)], page[~used & (page < n)]
    number = page.clone()
    number[from_] = to
    out = torch.zeros_like(table)
    out[inside] = number[table[inside]]
    entries = torch.full((n_pages // 2 + 1, 4), -1, dtype=torch.int32, device="cuda")
    entries[:from_.numel()] = torch.stack([from_, to, torch.full_like(to, st["case"]["page_size"]), torch.full_like(to, -1)], 1).to(torch.int32)
    free = st["free"].clone()
    free[:n_pages - n] = page[n:].flip(0).to(torch.int32)
    whole = {"table": out, "free_count": (n_pages - n)[None], "n_copies": torch.tensor([from_.numel()], device="cuda"), "copies": entries,
             "free": free}
    return {key: x.to(torch.int32) for key, x in whole.items()}


def _plain_copy(st):
    from_, to, rows = (st["copies"][:, i].long() for i in range(3))
    size = st["case"]["page_size"]
    copied = (torch.arange(size, device="cuda") < rows[:, None])[:, None, :, None]
    for pool in (st["k"], st["v"]):
        pool[:, to] = torch.where(copied, pool[:, from_], pool[:, to])
    return [st["k"], st["v"]]


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definition

def exact(case, seed):
    if case["kind"] != "verify":
        return None  # whole numbers, or values that are only moved
    st = _verify_inputs(case, seed)
    b, t = st["parents"].shape
    path = torch.full((b, t), -1, dtype=torch.int32)
    length, following = torch.zeros(b, dtype=torch.int32), torch.zeros(b, dtype=torch.int32)
    logprobs = torch.zeros((b, t), dtype=torch.float64)
    for i in range(b):
        nodes, token, logs = _walk(st, i, case["with_replacement"])
        path[i, :len(nodes)] = torch.tensor(nodes, dtype=torch.int32)
        length[i], following[i] = len(nodes), token
        logprobs[i, :len(logs)] = torch.tensor(logs, dtype=torch.float64)
    return {"path": path, "len": length, "next": following, "logprobs": logprobs, "err": torch.zeros(b, dtype=torch.int32)}


def _walk(st, i, with_replacement):
    """One request: at each node the children are tried in turn against the target's distribution, which a refused child replaces by
    the normalised positive part of target - draft; without replacement the draft's loses that token."""
    parents, tokens, accept = st["parents"][i].tolist(), st["tokens"][i].tolist(), st["accept_uniforms"][i].tolist()
    heat = st["temperature"][i].double()
    nodes, logs = [0], []
    while True:
        row = st["target"][i, nodes[-1]].double()
        log_p = torch.log_softmax(row / heat if heat > 0 else row, 0)
        if heat > 0:
            p = torch.softmax(row / heat, 0)
        else:
            p = torch.zeros_like(row)
            p[row.argmax()] = 1
        drawn = st["draft"] is not None and bool(heat > 0)
        q = torch.softmax(st["draft"][i, nodes[-1]].double() / st["draft_temperature"][i].double(), 0) if drawn else None
        found = None
        for child in (c for c, above in enumerate(parents) if above == nodes[-1]):
            x = tokens[child]
            if accept[child] < (p[x] / q[x] if drawn else p[x]):
                found = child
                break
            if drawn:
                p = (p - q).clamp(min=0)
                if not with_replacement:
                    q = q.clone()
                    q[x] = 0
                    q = q / q.sum()
            else:
                p = p.clone()
                p[x] = 0
            p = p / p.sum()
        if found is None:
            border = torch.cumsum(p, 0)
            token = int(torch.searchsorted(border, st["sample_uniforms"][i].double() * border[-1], right=True))
            return nodes, token, logs + [float(log_p[token])]
        nodes.append(found)
        logs.append(float(log_p[tokens[found]]))


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "verify":
        # Only the rows of nodes that are reached have to be read: the root's and, at about two levels in three, one more; of the last
        # node, if it is a leaf, the target's alone.
        levels = len(_levels(case)[0])
        reached = 1 + 2 * levels / 3
        row = BYTES[case["dtype"]] + (BYTES[case["draft_dtype"]] if case["drawn"] and levels else 0)
        t = _nodes(case)
        n = case["batch"]
        return {"bytes": n * (reached * case["vocab"] * row + 4 * (5 * t + 6)), "flops": n * reached * case["vocab"] * 6}
    if case["kind"] == "fork":
        # the table's entries in and out, and what there is per request
        rows, _ = _fork_rows(case)
        size, left = case["samples"], (case["groups"] - case["ended"]) * case["samples"]
        before = sum(_pages(r, case["page_size"]) for r in rows)
        after = sum(_pages(rows[b // size * size], case["page_size"]) for b in range(left))
        return {"bytes": 4 * (before + after + 11 * len(rows)), "flops": 0}
    if case["kind"] == "compact":
        # the table's entries in and out, the free pages, about a quarter of the pages moved
        entries = sum(_pages(r, case["page_size"]) for r in _compact_rows(case))
        return {"bytes": 4 * (2 * entries + case["batch"] + case["n_pages"]), "flops": 0}
    rows = case["page_size"] * (1.0 if case["whole"] else 0.5)
    row = case["n_kv_heads"] * case["head_dim"] * BYTES[case["dtype"]]
    return {"bytes": 4 * case["copies"] * case["layers"] * rows * row + 16 * case["copies"], "flops": 0}
