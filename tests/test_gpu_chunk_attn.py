"""Attention of a step's new tokens over a paged cache against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd.device_batch import torch_dtype
from step_reference import chunk_attention

pytestmark = pytest.mark.gpu


class Step:
    """Packed queries and a pool in which the requests' rows are scattered; rows past a request's length, a page nobody
    holds and unused table entries' page hold NaN."""

    def __init__(self, dtype, heads, news, lens, page_size=16, token_major=False, head_major_q=False, seed=0, peak=1.0, spare_tokens=0):
        hq, hkv, d = heads
        rng = np.random.default_rng(seed)
        dt = torch_dtype(dtype)
        self.dtype, self.heads, self.news, self.lens, self.page_size = dtype, heads, news, lens, page_size
        draw = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt)  # noqa: E731
        self.n_tokens = sum(news) + spare_tokens
        self.q = (draw(max(1, self.n_tokens), hq, d) * peak).to(dt)
        self.k_rows, self.v_rows = [draw(hkv, n, d) for n in lens], [draw(hkv, n, d) for n in lens]
        per = [-(-n // page_size) for n in lens]
        order = rng.permutation(sum(per)) + 1  # page 0: NaN
        width = max(1, max(per)) + 1
        self.table = np.zeros((len(lens), width), np.int32)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.n_pages, self.token_major, self.head_major_q = sum(per) + 1, token_major, head_major_q

    def pages(self, rows):
        hq, hkv, d = self.heads
        x = torch.full((self.n_pages, hkv, self.page_size, d), float("nan"), dtype=self.q.dtype)
        for b, r in enumerate(rows):
            for i in range(-(-self.lens[b] // self.page_size)):
                part = r[:, i * self.page_size:(i + 1) * self.page_size]
                x[self.table[b, i], :, :part.shape[1]] = part
        x = x.cuda()
        return x.transpose(1, 2).contiguous().transpose(1, 2) if self.token_major else x

    def run(self, window=0, scale=0.0, max_new=None, max_kv=None, times=1, stream=None):
        q = self.q.cuda()
        if self.head_major_q:
            q = q.transpose(0, 1).contiguous().transpose(0, 1)
        k, v = self.pages(self.k_rows), self.pages(self.v_rows)
        table = torch.from_numpy(self.table).cuda()
        cu = torch.from_numpy(np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)).cuda()
        lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.out = torch.full_like(q, 7.0)
        self.lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
        desc = ls.make_chunk_desc(q, k, v, table, self.out, max_new or max(1, max(self.news)), max(self.lens) if max_kv is None else max_kv,
                                  window, scale)
        need = ls.ls_chunk_workspace_bytes(desc)
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        kept = None
        for _ in range(times):
            ls.ls_chunk_attn_paged(desc, q, k, v, table, cu, lens, self.out, self.lse, ws[:need], stream=stream)
            torch.cuda.synchronize()
            now = (self.out.cpu(), self.lse.cpu())
            if kept is not None:
                assert torch.equal(kept[0].view(torch.int16), now[0].view(torch.int16)) and torch.equal(kept[1].view(torch.int32), now[1].view(torch.int32))
            kept = now
        assert (ws[need:] == 0xFF).all()
        return kept

    def check(self, window=0, scale=0.0, **options):
        out, lse = self.run(window, scale, **options)
        real = sum(self.news)
        as64 = lambda rows: [r.double() for r in rows]  # noqa: E731
        want, want_lse, bound, lse_bound = chunk_attention(self.q[:real].double(), as64(self.k_rows), as64(self.v_rows), self.news, self.lens,
                                                           window, scale if scale else self.heads[2] ** -0.5, self.dtype)
        assert (out[real:] == 7).all() and (lse[real:] == 7).all(), "tokens nobody owns"
        compare(out[:real].double(), want, bound, "out")
        compare(lse[:real].double(), want_lse, lse_bound, "lse")


def compare(got, want, bound, what):
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), what
    err = (got - want).abs()[finite]
    worst = (err / bound[finite].clamp(min=1e-300)).max() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {float(worst)} of the bound"


HEADS = {"gqa": (8, 2, 128), "mha": (3, 3, 128), "small": (16, 4, 64), "five": (5, 1, 128), "wide": (24, 1, 64), "one": (1, 1, 64)}

NEWS_LENS = [  # new tokens, rows with them
    ([1], [1]), ([1], [33]), ([1, 1, 1], [1, 16, 777]), ([5], [5]), ([64], [64]), ([65], [129]), ([200], [1003]),
    ([1, 90, 1, 7, 0, 300], [500, 90, 31, 1000, 0, 411]), ([0, 3, 0], [10, 20, 0]), ([2] * 40, [40 + 3 * i for i in range(40)]),
    ([1] * 70, [(37 * i) % 300 + 1 for i in range(70)]), ([513, 1], [640, 2049]),
]


@pytest.mark.parametrize("news,lens", NEWS_LENS)
@pytest.mark.parametrize("heads,dtype", [("gqa", "bf16"), ("mha", "f16"), ("small", "f16"), ("five", "bf16"), ("wide", "bf16"), ("one", "f16")])
def test_against_the_definition(heads, dtype, news, lens):
    Step(dtype, HEADS[heads], news, lens, seed=len(news) + lens[0]).check()


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 1000, 5000])
@pytest.mark.parametrize("heads,dtype,page_size", [("gqa", "bf16", 16), ("small", "f16", 64)])
def test_windows(heads, dtype, page_size, window):
    for news, lens in (([1, 90, 1, 7, 0, 300], [500, 90, 31, 1000, 0, 411]), ([400], [1500]), ([1] * 9, [100 * i + 1 for i in range(9)])):
        Step(dtype, HEADS[heads], news, lens, page_size=page_size, seed=window).check(window=window)


@pytest.mark.parametrize("page_size", [16, 32, 256])
@pytest.mark.parametrize("token_major,head_major_q", [(True, False), (False, True), (True, True)])
def test_layouts(page_size, token_major, head_major_q):
    for heads, dtype in (("gqa", "f16"), ("small", "bf16")):
        Step(dtype, HEADS[heads], [1, 77, 3], [800, 333, 3], page_size=page_size, token_major=token_major, head_major_q=head_major_q).check(scale=0.3)


def test_peaked_rows():
    """Scores of some tens: few keys carry a row, and the running maximum moves."""
    for heads, dtype in (("gqa", "bf16"), ("small", "f16")):
        Step(dtype, HEADS[heads], [1, 200, 2], [900, 900, 40], peak=8.0, seed=4).check()


def test_scores_that_rise_along_the_keys():
    """Every tile has a larger maximum than all before it, by more than a half holds."""
    for heads, dtype in (("gqa", "bf16"), ("small", "f16")):
        for news, lens in (([130], [700]), ([1, 1], [2500, 64])):
            st = Step(dtype, HEADS[heads], news, lens, seed=5)
            st.q = st.q.abs()
            for k in st.k_rows:
                k.copy_((k.abs() * torch.linspace(0.1, 6.0, k.shape[1])[None, :, None]).to(k.dtype))
            st.check()


def test_rows_before_the_first_one_see_nothing():
    """More new tokens than rows, and lengths of zero: zeros and -inf."""
    Step("bf16", HEADS["gqa"], [5, 40, 3], [3, 1, 0]).check()
    Step("f16", HEADS["small"], [70, 1, 200], [10, 0, 199]).check(window=4)


def test_lengths_are_clamped():
    """Rows beyond max_kv_len are not there; tokens past max_new_len of a request and past the last request are not written."""
    st = Step("bf16", HEADS["gqa"], [4, 1], [50, 300], spare_tokens=6)
    st.check()
    # the second request cut to 200 rows: its token stands at row 199
    st.run(max_kv=200)
    cut = Step("bf16", HEADS["gqa"], [4, 1], [50, 300], spare_tokens=6)
    out, lse = st.out.cpu(), st.lse.cpu()
    cut.lens = [50, 200]
    cut.k_rows, cut.v_rows = ([r[:, :n] for r, n in zip(rows, cut.lens)] for rows in (cut.k_rows, cut.v_rows))
    want, want_lse, bound, lse_bound = chunk_attention(cut.q[:5].double(), [r.double() for r in cut.k_rows], [r.double() for r in cut.v_rows],
                                                       [4, 1], cut.lens, 0, 128 ** -0.5, "bf16")
    compare(out[:5].double(), want, bound, "out")
    compare(lse[:5].double(), want_lse, lse_bound, "lse")
    whole = st.run()[0]
    out, lse = st.run(max_new=2)
    assert (out[2:4] == 7).all() and (lse[2:4] == 7).all() and torch.isfinite(out[:2].float()).all() and (out[:2] != 7).any()
    compare(out[4:5].double(), whole[4:5].double(), bound[4:5] * 4 + 0.1, "the other request")


@pytest.mark.parametrize("heads,dtype", [("gqa", "bf16"), ("small", "f16")])
@pytest.mark.parametrize("window", [0, 20])
def test_unseen_values_and_keys_have_no_part(heads, dtype, window):
    """Infinities and NaN in rows that a token does not see, inside its own tiles: later new tokens, rows before the window."""
    for news, lens in (([100], [150]), ([40, 1], [40, 300])):
        st = Step(dtype, HEADS[heads], news, lens, seed=8)
        clean = st.run(window)
        bad = Step(dtype, HEADS[heads], news, lens, seed=8)
        at = lens[0] - 30  # a row of the first request's new tokens
        bad.v_rows[0][:, at, 3] = float("inf")
        bad.v_rows[0][:, at, 5] = float("nan")
        bad.k_rows[0][:, at + 3, 1] = float("nan")
        out, lse = bad.run(window)
        first = at - (lens[0] - news[0])  # the token that stands at that row
        end = news[0] if not window else min(news[0], first + window)
        sees_v = torch.zeros(out.shape[0], dtype=torch.bool)
        sees_k = sees_v.clone()
        sees_v[first:end] = True
        sees_k[first + 3:(news[0] if not window else min(news[0], first + 3 + window))] = True
        none = ~sees_v & ~sees_k
        assert torch.equal(out[none], clean[0][none]) and torch.equal(lse[none], clean[1][none])
        only_v = sees_v & ~sees_k
        assert torch.isinf(out[only_v][:, :, 3]).all() and (out[only_v][:, :, 3] > 0).all() and torch.isnan(out[only_v][:, :, 5]).all()
        others = [i for i in range(out.shape[2]) if i not in (3, 5)]
        assert torch.equal(out[only_v][:, :, others], clean[0][only_v][:, :, others])
        assert torch.isnan(out[sees_k]).all() and torch.isnan(lse[sees_k]).all()


def test_keys_that_score_minus_infinity():
    """Keys whose score is -inf weigh nothing, at the beginning, in whole tiles, and where a row sees no other."""
    for heads, dtype in (("gqa", "bf16"), ("small", "f16")):
        for news, lens in (([60], [400]), ([1, 1], [400, 70])):
            st = Step(dtype, HEADS[heads], news, lens, seed=9)
            st.q = st.q.abs() + 0.1
            for k in st.k_rows:
                k[:, :40] = -float("inf")
                k[:, 64:100] = -float("inf")
                k[:, -1] = -float("inf")
            out, lse = st.run()
            keep = [torch.isfinite(k[0, :, 0]) for k in st.k_rows]
            assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
            at = 0
            for b, n in enumerate(news):
                for i in range(0, n, 7):
                    seen = keep[b] & (torch.arange(lens[b]) <= lens[b] - n + i)
                    for h in (0, st.heads[0] - 1):
                        g = h // (st.heads[0] // st.heads[1])
                        s = st.k_rows[b][g][seen].double() @ st.q[at + i, h].double() * st.heads[2] ** -0.5
                        assert abs(float(lse[at + i, h]) - float(torch.logsumexp(s, 0))) < 1e-4
                at += n
    st = Step("bf16", HEADS["gqa"], [3], [3], seed=10)
    st.q = st.q.abs() + 0.1
    st.k_rows[0][:] = -float("inf")
    out, lse = st.run()
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_the_same_inputs_give_the_same_bits():
    Step("bf16", HEADS["gqa"], [1, 300, 1, 1], [3000, 900, 1500, 20], seed=11).run(times=4)
    Step("f16", HEADS["small"], [1] * 5, [4000, 100, 9, 2000, 3000], seed=12).run(times=4)


def test_long_caches():
    """Many tiles per row, and more keys than one pass over them by a single workgroup would do."""
    Step("bf16", HEADS["gqa"], [1, 3], [20011, 7000], seed=13).check()
    Step("f16", HEADS["small"], [2, 1, 60], [1, 30000, 12000], page_size=64, seed=14).check()
    Step("bf16", (4, 1, 128), [70], [9000], seed=15).check(window=6000)


def test_on_another_stream():
    side = torch.cuda.Stream()
    st = Step("bf16", HEADS["gqa"], [1, 100, 1], [700, 300, 50], seed=16)
    plain = st.run()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other = st.run()
    explicit = st.run(stream=side)
    for got in (other, explicit):
        assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])


def test_pool_beyond_4_gb():
    """Pages past 2^32 bytes of a pool of which only a few are touched, and a wide stride between the rows."""
    hq, hkv, d, kv, n = 8, 2, 128, 300, 40
    st = Step("bf16", (hq, hkv, d), [n], [kv], seed=17)
    pool = (5 << 30) // (hkv * 16 * d * 2)
    big = [torch.empty((pool, hkv, 16, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shift = pool - st.n_pages
    for x, rows in zip(big, (st.k_rows, st.v_rows)):
        x[shift:] = st.pages(rows)
    q, table = st.q.cuda(), torch.from_numpy(st.table + shift).cuda()
    out, lse = torch.empty_like(q), torch.empty((n, hq), dtype=torch.float32, device="cuda")
    cu, lens = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([kv], dtype=torch.int32, device="cuda")
    desc = ls.make_chunk_desc(q, *big, table, out, n, kv)
    ws = torch.empty(ls.ls_chunk_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    ls.ls_chunk_attn_paged(desc, q, *big, table, cu, lens, out, lse, ws)
    want = chunk_attention(st.q.double(), [st.k_rows[0].double()], [st.v_rows[0].double()], [n], [kv], 0, d ** -0.5, "bf16")
    compare(out.cpu().double(), want[0], want[2], "out")
    compare(lse.cpu().double(), want[1], want[3], "lse")


LISTED = [  # more requests than a workgroup's lanes: ended ones among them, blocks cut, single tokens
    ([1, 0, 3, 1] * 30, [(97 * i) % 700 + 3 for i in range(120)], 0),
    ([2] * 64 + [0] * 7 + [150, 1, 400], [5 + 11 * i for i in range(64)] + [9] * 7 + [3000, 2500, 400], 0),
    ([70] * 66, [70 + 5 * i for i in range(66)], 100),
    ([0] * 90 + [1, 33], [40] * 90 + [6000, 2000], 0),
]


@pytest.mark.parametrize("news,lens,window", LISTED)
@pytest.mark.parametrize("heads,dtype", [("gqa", "bf16"), ("small", "f16")])
def test_more_requests_than_lanes(heads, dtype, news, lens, window):
    Step(dtype, HEADS[heads], news, lens, seed=18).check(window=window, times=2)


@pytest.mark.parametrize("batch", [65, 300])
def test_more_requests_than_tokens(batch):
    """Most requests of a table idle: a request is a piece whether it has tokens or not."""
    news, lens = [0] * batch, [3 * i % 90 for i in range(batch)]
    news[7], news[batch - 1], lens[7], lens[batch - 1] = 1, 2, 40, 77
    Step("bf16", HEADS["gqa"], news, lens, seed=19).check()


def test_the_largest_batch():
    news = [1 if i % 3 else 0 for i in range(ls.LS_MAX_STEP_BATCH)]
    Step("f16", (2, 1, 64), news, [1 + i % 37 for i in range(len(news))], seed=20).check()
    news[5] = 90
    Step("f16", (2, 1, 64), news, [90 + i % 37 for i in range(len(news))], seed=21).check()


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("n", [15, 16, 17, 31, 32, 33])
def test_around_the_rows_of_a_product(n, d, dtype):
    """16 and 32 rows per KV head are where the kernels change."""
    Step(dtype, (2, 2, d), [n, 1, n], [n, 90, 500 + n], seed=22).check()
    Step(dtype, (2, 2, d), [n], [300 + n], page_size=64, seed=23).check(window=33)


@pytest.mark.parametrize("heads,dtype", [("gqa", "bf16"), ("small", "f16")])
@pytest.mark.parametrize("n", [4, 7])
@pytest.mark.parametrize("window", [0, 2])
def test_unseen_values_and_keys_have_no_part_in_few_rows(heads, dtype, n, window):
    st, bad = (Step(dtype, HEADS[heads], [n, 1], [150, 70], seed=24) for _ in range(2))
    clean = st.run(window)
    at = 150 - 3  # the row of token n - 3
    bad.v_rows[0][:, at, 3] = float("-inf")
    bad.v_rows[0][:, at, 61] = float("nan")
    bad.k_rows[0][:, at + 1, 1] = float("nan")
    bad.v_rows[0][:, 150 - n - 4] = float("inf")  # before every window of two
    out, lse = bad.run(window)
    before, only_v, after = slice(0, n - 3), n - 3, slice(n - 2, n)
    others = [i for i in range(out.shape[2]) if i not in (3, 61)]
    if window:
        assert torch.equal(out[before], clean[0][before]) and torch.equal(lse[before], clean[1][before])
        assert torch.isneginf(out[only_v][:, 3]).all() and torch.equal(out[only_v][:, others], clean[0][only_v][:, others])
        assert torch.isnan(out[after]).all() and torch.isnan(lse[after]).all()
    else:  # all see the infinite row, the last two a key of NaN as well
        assert torch.isposinf(out[before]).all() and torch.equal(lse[before], clean[1][before])
        assert torch.isnan(out[only_v][:, [3, 61]]).all() and torch.isposinf(out[only_v][:, others]).all()
        assert torch.isnan(out[after]).all()
    assert torch.isnan(out[only_v][:, 61]).all() and torch.equal(lse[only_v], clean[1][only_v])
    assert torch.equal(out[n], clean[0][n]) and torch.equal(lse[n], clean[1][n])


@pytest.mark.parametrize("heads", ["gqa", "five", "wide"])
@pytest.mark.parametrize("news,lens", [([1], [9000]), ([1, 1, 1], [20000, 64, 5000]), ([1] * 20, [4000 + 37 * i for i in range(20)]),
                                       ([1] * 70, [3000 if i % 7 == 0 else 40 + i for i in range(70)])])
def test_few_rows_that_are_cut(heads, news, lens):
    """Few requests, whose workgroups have four waves at head_dim 128, and many, whose have eight."""
    Step("bf16" if heads != "gqa" else "f16", HEADS[heads], news, lens, seed=25).check(times=2)
