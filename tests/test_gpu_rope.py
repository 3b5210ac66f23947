"""Rotary positions and the write into pages against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd.device_batch import torch_dtype
from step_reference import rope, rope_bound

pytestmark = pytest.mark.gpu


def table(rows, pairs):
    angle = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(pairs) / pairs)
    return np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)


def inputs(rng, t, heads, d, dtype, layout="packed"):
    """Queries, keys and values as slices of one projection's rows, or stored head by head."""
    hq, hkv = heads
    x = torch.from_numpy(rng.standard_normal((t, hq + 2 * hkv, d)).astype(np.float32)).to(torch_dtype(dtype)).cuda()
    if layout == "head_major":
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def expected(x, positions, cos_sin, sections, interleaved, dtype):
    out, scale = rope(x.double().cpu().numpy(), positions, cos_sin, sections, interleaved)
    return out, rope_bound(out, scale, dtype)


def close(got, want, bound, what):
    err = np.abs(got.double().cpu().numpy() - want)
    worst = float((err / bound).max())
    assert worst <= 1.0, f"{what}: {worst} of the bound"


CASES = [  # dtype, heads, head_dim, rotary_dim, sections, interleaved, tokens, layout
    ("bf16", (32, 8), 128, 128, [64], False, 1, "packed"), ("bf16", (32, 8), 128, 128, [64], False, 37, "head_major"),
    ("f16", (32, 8), 128, 128, [64], True, 24, "packed"), ("f32", (40, 8), 128, 128, [16, 24, 24], False, 65, "packed"),
    ("bf16", (16, 4), 64, 32, [4, 6, 6], True, 301, "packed"), ("f16", (3, 1), 64, 64, [1, 31], False, 7, "packed"),
    ("bf16", (5, 5), 128, 48, [3, 0, 20, 1], False, 33, "head_major"), ("f32", (8, 8), 64, 16, [8], True, 129, "packed"),
    ("bf16", (7, 1), 128, 96, [47, 1], True, 500, "packed"), ("f32", (1, 1), 128, 112, [56], False, 3, "packed"),
]


@pytest.mark.parametrize("dtype,heads,d,rotary,sections,interleaved,t,layout", CASES)
@pytest.mark.parametrize("in_place", [False, True])
def test_rope(dtype, heads, d, rotary, sections, interleaved, t, layout, in_place):
    rng = np.random.default_rng(t + rotary)
    q, k, _ = inputs(rng, t, heads, d, dtype, layout)
    cos_sin = table(3000, rotary // 2)
    positions = rng.integers(0, 3000, (len(sections), t)).astype(np.int32)
    positions[:, 0] = 0
    positions[-1, t // 2] = 5000  # clamped to the last row
    positions[0, -1] = -3
    wq, bq = expected(q, positions, cos_sin, sections, interleaved, dtype)
    wk, bk = expected(k, positions, cos_sin, sections, interleaved, dtype)
    q_out, k_out = (q, k) if in_place else (torch.full_like(q, float("nan")), torch.full_like(k, float("nan")))
    pos, cs = torch.from_numpy(positions).cuda(), torch.from_numpy(cos_sin).cuda()
    desc = ls.make_rope_desc(q, k, None, q_out, k_out, None, None, pos, cs, sections, interleaved)
    ls.ls_rope(desc, q, k, pos, cs, q_out, k_out)
    close(q_out, wq, bq, "q")
    close(k_out, wk, bk, "k")


@pytest.mark.parametrize("dtype,heads,d,rotary,sections,interleaved,t,layout", CASES)
@pytest.mark.parametrize("page_size,token_major", [(16, False), (1, True), (64, True)])
def test_rope_store(dtype, heads, d, rotary, sections, interleaved, t, layout, page_size, token_major):
    rng = np.random.default_rng(t + rotary)
    q, k, v = inputs(rng, t, heads, d, dtype, layout)
    cos_sin = table(500, rotary // 2)
    positions = rng.integers(0, 500, (len(sections), t)).astype(np.int32)
    pool = -(-t // page_size) + 3
    slots = rng.permutation(pool * page_size)[:t].astype(np.int32)
    slots[rng.random(t) < 0.1] = -1
    if t > 5:
        slots[3], slots[4] = pool * page_size, 2 ** 31 - 1  # outside the pool
    pages = [torch.full((pool, page_size, heads[1], d) if token_major else (pool, heads[1], page_size, d), float("nan"),
                        dtype=q.dtype, device="cuda") for _ in range(2)]
    if token_major:
        pages = [x.transpose(1, 2) for x in pages]
    q_out = torch.full_like(q, float("nan"))
    pos, cs, sl = torch.from_numpy(positions).cuda(), torch.from_numpy(cos_sin).cuda(), torch.from_numpy(slots).cuda()
    desc = ls.make_rope_desc(q, k, v, q_out, None, *pages, pos, cs, sections, interleaved)
    ls.ls_rope_store_paged(desc, q, k, v, pos, cs, sl, q_out, *pages)
    wq, bq = expected(q, positions, cos_sin, sections, interleaved, dtype)
    wk, bk = expected(k, positions, cos_sin, sections, interleaved, dtype)
    close(q_out, wq, bq, "q")
    flat = [x.transpose(1, 2).reshape(pool * page_size, heads[1], d) for x in pages]
    real = np.nonzero((slots >= 0) & (slots < pool * page_size))[0]
    at = torch.from_numpy(slots[real]).long().cuda()
    close(flat[0][at], wk[real], bk[real], "k")
    assert torch.equal(flat[1][at], v[torch.from_numpy(real).cuda()])
    other = torch.ones(pool * page_size, dtype=torch.bool, device="cuda")
    other[at] = False
    assert torch.isnan(flat[0][other]).all() and torch.isnan(flat[1][other]).all()  # nothing else is written


def test_queries_alone():
    rng = np.random.default_rng(3)
    q, _, _ = inputs(rng, 19, (8, 2), 128, "bf16")
    cos_sin, positions = table(100, 64), rng.integers(0, 100, (1, 19)).astype(np.int32)
    q_out = torch.empty_like(q)
    pos, cs = torch.from_numpy(positions).cuda(), torch.from_numpy(cos_sin).cuda()
    ls.ls_rope(ls.make_rope_desc(q, None, None, q_out, None, None, None, pos, cs), q, None, pos, cs, q_out, None)
    close(q_out, *expected(q, positions, cos_sin, [64], False, "bf16"), "q")


def test_all_axes_may_share_one_row_of_positions():
    """A stride of 0 between the axes: text, whose three positions are equal, is the one-axis form."""
    rng = np.random.default_rng(4)
    q, k, _ = inputs(rng, 40, (8, 2), 128, "f32")
    cs, pos = torch.from_numpy(table(100, 64)).cuda(), torch.from_numpy(rng.integers(0, 100, (1, 40)).astype(np.int32)).cuda()
    outs = []
    for p, sections in ((pos, [64]), (pos.expand(3, 40), [16, 24, 24])):
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        ls.ls_rope(ls.make_rope_desc(q, k, None, q_out, k_out, None, None, p, cs, sections), q, k, p, cs, q_out, k_out)
        outs.append((q_out, k_out))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_infinities_and_nan_stay_in_their_pair():
    rng = np.random.default_rng(5)
    q, k, v = inputs(rng, 6, (4, 2), 64, "f16")
    q[2, 1, 5], k[3, 0, 40], v[1, 1, 7] = float("inf"), float("nan"), float("nan")
    cs = torch.from_numpy(table(50, 32)).cuda()
    pos, slots = torch.arange(6, dtype=torch.int32, device="cuda")[None] + 1, torch.arange(6, dtype=torch.int32, device="cuda")
    q_out = torch.empty_like(q)
    pages = [torch.zeros((1, 2, 16, 64), dtype=q.dtype, device="cuda") for _ in range(2)]
    ls.ls_rope_store_paged(ls.make_rope_desc(q, k, v, q_out, None, *pages, pos, cs), q, k, v, pos, cs, slots, q_out, *pages)
    assert torch.nonzero(~torch.isfinite(q_out)).tolist() == [[2, 1, 5], [2, 1, 37]]
    assert torch.nonzero(~torch.isfinite(pages[0])).tolist() == [[0, 0, 3, 8], [0, 0, 3, 40]]
    assert torch.nonzero(~torch.isfinite(pages[1])).tolist() == [[0, 1, 1, 7]]


def test_pool_beyond_4_gb():
    """Pages past 2^32 bytes, in a pool of which only the last ones are touched."""
    rng = np.random.default_rng(6)
    q, k, v = inputs(rng, 20, (4, 2), 128, "bf16")
    pool = (5 << 30) // (2 * 16 * 128 * 2)
    pages = [torch.empty((pool, 2, 16, 128), dtype=q.dtype, device="cuda") for _ in range(2)]
    slots = torch.arange(pool * 16 - 20, pool * 16, dtype=torch.int32, device="cuda")
    cs, pos = torch.from_numpy(table(50, 64)).cuda(), torch.arange(20, dtype=torch.int32, device="cuda")[None]
    q_out = torch.empty_like(q)
    ls.ls_rope_store_paged(ls.make_rope_desc(q, k, v, q_out, None, *pages, pos, cs), q, k, v, pos, cs, slots, q_out, *pages)
    rows = torch.cat([pages[0][-2], pages[0][-1]], dim=1)[:, -20:].transpose(0, 1)
    close(rows, *expected(k, pos.cpu().numpy(), table(50, 64), [64], False, "bf16"), "k")
    assert torch.equal(torch.cat([pages[1][-2], pages[1][-1]], dim=1)[:, -20:].transpose(0, 1), v)


@pytest.mark.parametrize("t", [1024, 1025, 1331])
@pytest.mark.parametrize("dtype,heads,d,rotary,sections,interleaved", [
    ("bf16", (32, 8), 128, 128, [64], False), ("f32", (3, 1), 128, 64, [9, 23], True), ("f16", (16, 4), 64, 64, [32], False),
    ("bf16", (5, 5), 64, 48, [8, 8, 8], True)])
def test_many_tokens(t, dtype, heads, d, rotary, sections, interleaved):
    """Around the number of tokens from which few threads share a token."""
    rng = np.random.default_rng(t)
    cos_sin = table(2000, rotary // 2)
    positions = rng.integers(0, 2000, (len(sections), t)).astype(np.int32)
    q, k, v = inputs(rng, t, heads, d, dtype)
    n_pages, page_size = t // 16 + 3, 16
    k_pages = torch.full((n_pages, heads[1], page_size, d), 7.0, dtype=q.dtype, device="cuda")
    v_pages, q_out = k_pages.clone(), torch.empty_like(q)
    slots = rng.permutation(n_pages * page_size)[:t].astype(np.int32)
    slots[t // 2] = -1
    pos, cs, sl = torch.from_numpy(positions).cuda(), torch.from_numpy(cos_sin).cuda(), torch.from_numpy(slots).cuda()
    desc = ls.make_rope_desc(q, k, v, q_out, None, k_pages, v_pages, pos, cs, sections, interleaved)
    ls.ls_rope_store_paged(desc, q, k, v, pos, cs, sl, q_out, k_pages, v_pages)
    want, bound = expected(q, positions, cos_sin, sections, interleaved, dtype)
    close(q_out, want, bound, "q")
    rows = lambda x: x.transpose(1, 2).reshape(n_pages * page_size, heads[1], d)  # noqa: E731
    real = slots >= 0
    want, bound = expected(k, positions, cos_sin, sections, interleaved, dtype)
    close(rows(k_pages)[slots[real]], want[real], bound[real], "k")
    at = torch.from_numpy(slots[real].astype(np.int64)).cuda()
    assert torch.equal(rows(v_pages)[at], v[torch.from_numpy(real).cuda()])
    other = torch.ones(n_pages * page_size, dtype=torch.bool, device="cuda")
    other[at] = False
    assert (rows(k_pages)[other] == 7).all() and (rows(v_pages)[other] == 7).all()


def test_on_another_stream():
    rng = np.random.default_rng(8)
    positions, cos_sin = rng.integers(0, 50, (1, 9)).astype(np.int32), table(50, 64)
    q, k, _ = inputs(rng, 9, (4, 2), 128, "bf16")
    pos, cs = torch.from_numpy(positions).cuda(), torch.from_numpy(cos_sin).cuda()
    want, bound = expected(q, positions, cos_sin, [64], False, "bf16")
    for explicit in (False, True):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            late = torch.zeros_like(q)
            torch.cuda._sleep(2000000)
            late.copy_(q)  # the queries arrive on the side stream
            k_out, desc = torch.empty_like(k), None
            desc = ls.make_rope_desc(late, k, None, late, k_out, None, None, pos, cs)
            if not explicit:
                ls.ls_rope(desc, late, k, pos, cs, late, k_out)
        if explicit:
            ls.ls_rope(desc, late, k, pos, cs, late, k_out, stream=side)
        side.synchronize()
        close(late, want, bound, "q")


@pytest.mark.parametrize("t", [2048, 2049, 2600])
@pytest.mark.parametrize("dtype,heads,rotary,sections,interleaved", [
    ("f16", (16, 4), 64, [32], False), ("bf16", (5, 5), 48, [8, 8, 8], True), ("f32", (33, 3), 32, [16], False)])
def test_many_tokens_of_64(t, dtype, heads, rotary, sections, interleaved):
    test_many_tokens(t, dtype, heads, 64, rotary, sections, interleaved)
