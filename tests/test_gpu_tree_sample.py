"""Acceptance of drafted trees at a temperature against its definition in more than 64 bits.

Paths and tokens have to be equal: the kernel's sums are in 64 bits, so that a draw falls on the other side of a border about once in 10^9.
Log probabilities are rounded once to float: 2^-24 of their value, and what 64 bits lose before (1e-12)."""
import numpy as np
import pytest
import torch

import sampling_reference as ref
from paper_2502_17421_amd import binding as ls

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def tree(rng, n, kind):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "forest":  # several roots, and nodes that no path reaches
        return [-1] + [int(rng.integers(-1, i)) for i in range(1, n)]
    return [-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, n)]


class Case:
    def __init__(self, seed, batch, n, vocab, target="bf16", draft="bf16", kind="tree", with_replacement=False, noise=1.0, spread=3.0,
                 temperature=None, draft_temperature=None, on_path=0.5):
        rng = np.random.default_rng(seed)
        self.with_replacement = with_replacement
        self.parents = torch.tensor([tree(rng, n, kind) for _ in range(batch)], dtype=torch.int32)
        base = torch.from_numpy(rng.standard_normal((batch, n, vocab), dtype=np.float32) * spread)
        self.target = base.to(DT[target])
        self.draft = None if draft is None else (base + noise * torch.from_numpy(rng.standard_normal(base.shape, dtype=np.float32))).to(DT[draft])
        self.temperature = torch.tensor([0.5 + rng.random() for _ in range(batch)] if temperature is None else temperature, dtype=torch.float32)
        self.draft_temperature = None if draft_temperature is None else torch.tensor(draft_temperature, dtype=torch.float32)
        # tokens that the draft finds likely, so that paths go on; some anywhere
        self.tokens = torch.randint(0, vocab, (batch, n), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
        likely = (self.target if self.draft is None else self.draft).float().topk(min(4, vocab)).indices
        for b in range(batch):
            for i in range(1, n):
                p = int(self.parents[b, i])
                if p >= 0 and rng.random() < 0.9:
                    self.tokens[b, i] = likely[b, p, rng.integers(likely.shape[2])]
        self.accept_u = torch.from_numpy(rng.random((batch, n), dtype=np.float32))
        self.accept_u[rng.random((batch, n)) < on_path] *= 0.1  # paths of some length
        self.sample_u = torch.from_numpy(rng.random(batch, dtype=np.float32))

    def run(self, stream=None, **changes):
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        b, n = self.parents.shape
        tgt, drf = changes.get("target", dev(self.target)), changes.get("draft", dev(self.draft))
        desc = ls.make_sample_desc(tgt, drf, self.with_replacement)
        self.out = {"path": torch.full((b, n), 77, dtype=torch.int32, device="cuda"), "logprobs": torch.full((b, n), 7.0, device="cuda")}
        self.out |= {k: torch.full((b,), 77, dtype=torch.int32, device="cuda") for k in ("len", "next", "err")}
        o = self.out
        ws = torch.full((ls.ls_sample_workspace_bytes(desc),), 0x5a, dtype=torch.uint8, device="cuda")
        self.args = [desc, dev(self.parents), dev(self.tokens), tgt, drf, dev(self.temperature), dev(self.draft_temperature),
                     dev(self.accept_u), dev(self.sample_u), o["path"], o["len"], o["next"], o["logprobs"], o["err"], ws]
        ls.ls_tree_accept_sampled(*self.args, stream=stream)
        return self.out

    def expect(self):
        b, n = self.parents.shape
        path, logs = np.full((b, n), -1), np.zeros((b, n))
        lens, nexts, errs = (np.zeros(b, dtype=int) for _ in range(3))
        for i in range(b):
            drf = None if self.draft is None else self.draft[i].float().numpy()
            dt = None if self.draft_temperature is None else float(self.draft_temperature[i])
            p, t, lg, e = ref.accept_sampled(self.parents[i].tolist(), self.tokens[i].tolist(), self.target[i].float().numpy(), drf,
                                             float(self.temperature[i]), dt, self.accept_u[i].tolist(), float(self.sample_u[i]), self.with_replacement,
                                             [torch.finfo((self.target if x is None else x).dtype).max for x in (self.target, self.draft)])
            path[i, :len(p)], logs[i, :len(lg)] = p, np.array(lg, dtype=np.float64)
            lens[i], nexts[i], errs[i] = len(p), t, e
        return {"path": path, "len": lens, "next": nexts, "err": errs, "logprobs": logs}

    def check(self, want=None, got=None):
        want, got = want or self.expect(), {k: v.cpu().numpy() for k, v in (got or self.out).items()}
        for k in ("err", "len", "path", "next"):
            assert np.array_equal(got[k], want[k]), (k, got[k], want[k])
        fine = np.isfinite(want["logprobs"])
        assert np.array_equal(got["logprobs"][~fine], want["logprobs"][~fine])
        g, w = got["logprobs"][fine].astype(np.float64), want["logprobs"][fine]
        assert np.all(np.abs(g - w) <= 2.0 ** -24 * np.abs(w) * 1.0001 + 1e-12), np.abs(g - w).max()
        return want


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 511, 513, 4095, 4097, 8191, 8192, 8193, 32000, 50257])
@pytest.mark.parametrize("with_replacement", [False, True])
def test_vocabularies(vocab, with_replacement):
    c = Case(vocab, 5, 17, vocab, with_replacement=with_replacement)
    c.run()
    c.check()


@pytest.mark.parametrize("target,draft", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("vocab", [3, 50, 1021, 4096, 50257])
def test_nan_that_signals(target, draft, vocab):
    """NaN of any bits has no probability, wherever it stands: in front of the largest entries, behind them, at a row's end."""
    c = Case(vocab, 3, 9, vocab, target=target, draft=draft)
    for x in (c.target, c.draft):
        bits = {torch.bfloat16: (0x7f81, 0xff81 - 0x10000), torch.float16: (0x7c01, 0xfc01 - 0x10000), torch.float32: (0x7f800001, 0xff800001 - (1 << 32))}[x.dtype]
        whole = x.view(torch.int32 if x.dtype == torch.float32 else torch.int16)
        whole[..., 1::3] = bits[0]
        whole[..., 4::6] = bits[1]
        whole[1, ..., -1] = bits[1]
    c.run()
    c.check()


@pytest.mark.parametrize("target,draft", [(t, d) for t in DT for d in (*DT, None)])
def test_types(target, draft):
    c = Case(3, 4, 24, 10007, target, draft)
    c.run()
    c.check()


@pytest.mark.parametrize("n,kind", [(1, "chain"), (2, "chain"), (9, "chain"), (64, "chain"), (17, "star"), (300, "star"), (64, "tree"),
                                    (65, "forest"), (512, "tree"), (511, "forest")])
@pytest.mark.parametrize("draft", ["bf16", None])
def test_trees(n, kind, draft):
    c = Case(n, 3, n, 1501, draft=draft, kind=kind, on_path=0.9 if kind == "chain" else 0.2)
    c.run()
    c.check()


@pytest.mark.parametrize("batch,vocab", [(1, 152064), (2, 200001), (70, 20011), (300, 501)])
def test_batches(batch, vocab):
    c = Case(batch, batch, 11, vocab, spread=4.0, noise=0.7)
    c.run()
    c.check()


def test_more_groups_than_there_is_room_for():
    """1500 sequences of several workgroups each, in float: many rounds of the card."""
    c = Case(6, 1500, 2, 20011, "f32", "f32", spread=4.0, noise=0.7)
    assert ls.ls_sample_workspace_bytes(ls.make_sample_desc(c.target, c.draft)) > 1500 * 64
    c.run()
    c.check()


def test_the_largest_batch():
    """65535 sequences: the bits of two calls of half of them each, and the reference for the first and the last."""
    c = Case(7, 64, 3, 11, kind="star")
    b, most = 64, 65535
    for name in ("parents", "target", "draft", "tokens", "temperature"):
        x = getattr(c, name)
        setattr(c, name, x.repeat(most // b + 1, *(1,) * (x.dim() - 1))[:most].contiguous())
    gen = torch.Generator().manual_seed(7)
    c.accept_u, c.sample_u = torch.rand((most, 3), generator=gen), torch.rand(most, generator=gen)
    out = {k: v.clone() for k, v in c.run().items()}
    names = ("parents", "target", "draft", "tokens", "temperature", "accept_u", "sample_u")
    full = {name: getattr(c, name) for name in names}

    def rows(lo, hi):
        for name in names:
            setattr(c, name, full[name][lo:hi])

    for lo, hi in ((0, 32768), (32768, most)):
        rows(lo, hi)
        for k, v in c.run().items():
            assert torch.equal(out[k][lo:hi], v), k
    for lo, hi in ((0, 100), (most - 100, most)):
        rows(lo, hi)
        c.check(got={k: v[lo:hi] for k, v in out.items()})


def test_the_largest_vocabulary():
    c = Case(5, 1, 3, ls.LS_MAX_VOCAB, "f16", "f16", kind="star")
    c.run()
    c.check()


def test_temperatures():
    """Greedy requests among the others, temperatures that are none, sharp and flat ones, drafts at other temperatures."""
    inf, nan = float("inf"), float("nan")
    t = [0.0, 1.0, -1.0, inf, nan, 0.02, 30.0, 1.0, 1.0, 0.0, 1e-30, 3e38, 1e-42]
    d = [1.0, 0.0, 1.0, 1.0, 1.0, 0.5, 2.0, nan, 1.7, 0.0, 1e-30, 3e38, 1.0]
    for draft_temperature in (d, None):
        c = Case(11, len(t), 20, 3001, temperature=t, draft_temperature=draft_temperature)
        c.run()
        c.check()


def test_greedy_is_the_greedy_acceptance():
    """Temperature 0 with equal largest logits: the lowest one, the path and token of ls_tree_accept_greedy."""
    c = Case(21, 6, 40, 9001, "f16", None, temperature=[0.0] * 6)
    c.target[:, ::2, 500], c.target[:, ::2, 8700] = 99.0, 99.0
    likely = c.target.float().argmax(-1).to(torch.int32)
    for b in range(6):
        for i in range(1, 40):
            if (i + b) % 3:
                c.tokens[b, i] = likely[b, max(0, int(c.parents[b, i]))]
    got = c.run()
    c.check()
    path, n, nxt = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((6, 40), (6,), (6,)))
    ls.ls_tree_accept_greedy(c.parents.cuda(), c.tokens.cuda(), likely.cuda(), path, n, nxt)
    assert torch.equal(path, got["path"]) and torch.equal(n, got["len"]) and torch.equal(nxt, got["next"])


@pytest.mark.parametrize("with_replacement", [False, True])
@pytest.mark.parametrize("target,draft", [("bf16", "f32"), ("f16", "f16"), ("f32", "bf16")])
def test_filtered_logits(target, draft, with_replacement):
    """-inf, NaN, +inf and the type's lowest value: rows that a filter has left few tokens of, rows without any."""
    c = Case(31, 12, 15, 9001, target, draft, with_replacement=with_replacement, kind="tree")
    rng = np.random.default_rng(1)
    for b in range(12):
        for i in range(15):
            what = (b + i) % 6
            if what == 0:
                keep = torch.from_numpy(rng.choice(9001, 3, replace=False))
                for x in (c.target, c.draft):
                    row = torch.full((9001,), -torch.inf if b % 2 else torch.finfo(x.dtype).min, dtype=x.dtype)
                    row[keep] = x[b, i, keep]
                    x[b, i] = row
            elif what == 1:
                c.target[b, i, ::7] = float("nan")
                c.draft[b, i, ::5] = -torch.inf
            elif what == 2 and i > 0:
                c.target[b, i] = -torch.inf if b % 2 else float("nan")
            elif what == 3:
                c.target[b, i, 8888] = torch.inf
                c.draft[b, i, 17 + i] = torch.inf
                for k in range(1, 15):  # a child of that token
                    if c.parents[b, k] == i and b % 2:
                        c.tokens[b, k] = 8888
            elif what == 4:
                c.draft[b, i] = -torch.inf
    c.target[3, 0] = -torch.inf
    c.run()
    want = c.check()
    assert {0, 4} <= set(want["err"].tolist())


def test_what_is_left_by_rejection():
    """All children refused, on purpose: equal logits of both models, a draft without the target's tokens, chosen children that cover
    nearly everything."""
    c = Case(41, 4, 9, 4097, "f32", "f32", kind="star", noise=0.0)
    c.accept_u[:] = 1 - 2.0 ** -24
    c.draft[1, 0, :4000] = -torch.inf
    c.target[2, 0, 40:] = -torch.inf
    c.tokens[2] = torch.arange(9)
    c.run()
    c.check()
    c.draft = None
    c.target[:, 0, 9:] = -torch.inf  # eight of nine tokens are children, and all are refused
    c.tokens[:] = torch.arange(9)
    c.accept_u[:] = 1.0
    c.run()
    want = c.check()
    assert (want["next"] == 0).all() and (want["len"] == 1).all()


def test_uniforms_at_their_ends():
    c = Case(43, 6, 12, 3001)
    c.accept_u[::2] = 0.0
    c.sample_u[:] = torch.tensor([0.0, 1 - 2.0 ** -24, 0.0, 1 - 2.0 ** -24, 0.5, 1.0])
    c.run()
    c.check()


def test_trees_that_are_none_and_tokens_outside():
    c = Case(51, 5, 30, 601)
    c.parents[0, 4], c.parents[1, 7], c.parents[2, 0] = 9, -5, 0
    c.tokens[3, 1:9], c.tokens[4, 2], c.tokens[4, 3] = -1, 601, 2 ** 31 - 1
    c.tokens[:, 0] = -7  # the root's is not looked at
    c.run()
    want = c.check()
    assert want["err"].tolist() == [1, 1, 1, 0, 0]


def test_strides_and_unaligned_rows():
    """Rows that start at any element, a stride between sequences of its own, the same row for all nodes."""
    c = Case(61, 3, 8, 5003, "f16", "f32")
    flat_t = torch.zeros(3 * 60000 + 5, dtype=torch.float16, device="cuda").fill_(float("nan"))
    flat_d = torch.zeros(3 * 70000 + 3, dtype=torch.float32, device="cuda").fill_(float("nan"))
    tgt = flat_t[5:].as_strided((3, 8, 5003), (60000, 5007, 1))
    drf = flat_d[3:].as_strided((3, 8, 5003), (70000, 5005, 1))
    tgt.copy_(c.target)
    drf.copy_(c.draft)
    c.run(target=tgt, draft=drf)
    c.check()
    c.draft = c.draft[:, :1].expand(-1, 8, -1)
    c.run(draft=c.draft[:, :1].contiguous().cuda().expand(-1, 8, -1))
    c.check()


def test_outputs_left_out_and_repeats():
    c = Case(71, 4, 20, 9001)
    got = {k: v.clone() for k, v in c.run().items()}
    want = c.check()
    a = list(c.args)
    for _ in range(3):  # the workspace as the call before left it
        ls.ls_tree_accept_sampled(*a)
    assert all(torch.equal(got[k], v) for k, v in c.out.items())
    c.out["logprobs"].fill_(5.0)
    c.out["err"].fill_(5)
    a[12] = a[13] = None
    ls.ls_tree_accept_sampled(*a)
    assert (c.out["logprobs"] == 5).all() and (c.out["err"] == 5).all()
    assert np.array_equal(c.out["path"].cpu().numpy(), want["path"])


def test_another_stream():
    c = Case(73, 4, 20, 30011)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.run()
        other = {k: v.clone() for k, v in c.run(stream=s).items()}
    s.synchronize()
    c.check(got=other)


def test_two_calls_at_once():
    """Calls of their own workspaces on two streams, each of more sequences than the card has room for at a time."""
    cases = [Case(75 + i, 40, 7, 64007, on_path=0.8) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.run()
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            for k in ("path", "next"):
                with torch.cuda.stream(s):
                    c.out[k].fill_(77)
            ls.ls_tree_accept_sampled(*c.args, stream=s)
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_recorded_into_a_graph():
    c = Case(81, 6, 20, 40009)
    c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ls.ls_tree_accept_sampled(*c.args)
    rng = np.random.default_rng(2)
    for _ in range(4):
        c.accept_u = torch.from_numpy(rng.random(c.accept_u.shape, dtype=np.float32))
        c.sample_u = torch.from_numpy(rng.random(6, dtype=np.float32))
        c.args[7].copy_(c.accept_u)
        c.args[8].copy_(c.sample_u)
        for v in c.out.values():
            v.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        c.check()


def test_graphs_that_share_a_workspace():
    """Two recorded calls of different sizes, replayed in turns over one workspace, with calls of their own in between."""
    cases = [Case(83, 5, 20, 40009), Case(84, 9, 7, 90001, "f32", "f16", on_path=0.8)]
    for c in cases:
        c.run()
    shared = torch.full((max(c.args[-1].numel() for c in cases),), 0xff, dtype=torch.uint8, device="cuda")
    graphs = []
    for c in cases:
        c.args[-1] = shared
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ls.ls_tree_accept_sampled(*c.args)
    rng = np.random.default_rng(3)
    for turn in range(6):
        for c, graph in zip(cases, graphs):
            c.accept_u = torch.from_numpy(rng.random(c.accept_u.shape, dtype=np.float32))
            c.args[7].copy_(c.accept_u)
            for v in c.out.values():
                v.fill_(9)
            if turn % 3 == 2:
                ls.ls_tree_accept_sampled(*c.args)
            else:
                graph.replay()
        torch.cuda.synchronize()
        for c in cases:
            c.check()


@pytest.mark.parametrize("with_replacement", [False, True])
def test_the_tokens_are_distributed_as_the_targets(with_replacement):
    """60000 sequences over 6 tokens whose three children are really drawn from the draft: the first new token has the target's
    distribution, within 5 standard deviations."""
    gen = torch.Generator().manual_seed(5)
    n, v = 60000, 6
    target, draft = torch.tensor([1.0, 0.2, -1.0, 0.5, -0.3, 0.0]), torch.tensor([-0.5, 1.0, 0.3, 0.4, -2.0, 0.1])
    q = torch.softmax(draft, 0).expand(n, v)
    tokens = torch.zeros((n, 4), dtype=torch.int32)
    tokens[:, 1:] = torch.multinomial(q, 3, replacement=with_replacement, generator=gen).to(torch.int32)
    c = Case(1, 1, 1, 6)
    c.with_replacement = with_replacement
    c.parents = torch.tensor([[-1, 0, 0, 0]], dtype=torch.int32).repeat(n, 1)
    c.tokens, c.target, c.draft = tokens, target.expand(n, 4, v).contiguous(), draft.expand(n, 4, v).contiguous()
    c.temperature, c.accept_u, c.sample_u = torch.ones(n), torch.rand((n, 4), generator=gen), torch.rand(n, generator=gen)
    got = {k: x.cpu() for k, x in c.run().items()}
    first = torch.where(got["len"] > 1, tokens.gather(1, got["path"][:, 1:2].clamp(min=0).long())[:, 0], got["next"])
    p = torch.softmax(target.double(), 0)
    share = torch.bincount(first.long(), minlength=v).double() / n
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all(), (share, p)


@pytest.fixture
def nobody_waits():
    ls.ls_set_single_launch_polls(0)
    yield
    ls.ls_set_single_launch_polls(-1)


@pytest.mark.parametrize("draft,with_replacement", [("bf16", False), ("f32", True), (None, False)])
def test_walks_alone_give_the_same_bits(nobody_waits, draft, with_replacement):
    """Workgroups that give up on their group at once: one of them does all of the sequence, with the same sums."""
    c = Case(91, 9, 33, 50021, draft=draft, with_replacement=with_replacement, temperature=[0.0] + [0.8] * 8)
    alone = {k: v.clone() for k, v in c.run().items()}
    c.check()
    ls.ls_set_single_launch_polls(-1)
    assert all(torch.equal(v, alone[k]) for k, v in c.run().items())


@pytest.mark.parametrize("polls", [1, 2, 3, 5, 9])
def test_walks_given_up_on_the_way(nobody_waits, polls):
    """Few polls: some groups get to the end, some do not, and both may write."""
    ls.ls_set_single_launch_polls(polls)
    c = Case(93, 60, 9, 30011, on_path=0.9)
    for _ in range(3):
        c.run()
        c.check()
