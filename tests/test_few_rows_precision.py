"""Attention of few new tokens rounds nothing but its result to the storage type: the numerators of the softmax take part in the output
product with what their own rounding leaves.  The inputs are made so that this rounding, were it all, would be off by nearly half a
unit in one direction: every query scores its keys 0 or -x, exactly, with exp(-x) close to the middle between two neighbours of the
type, and the keys that score 0 have values of 0."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk_attn import HEADS, Step

BITS = {"bf16": 8, "f16": 11}  # significant ones


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16 if dtype == "bf16" else torch.float16).double().numpy()


def exponents(n, dtype):
    """n values x of the type for which exp(-x) lies farthest from the type's values, in half units of these."""
    x = np.unique(rounded(np.linspace(0.1, 2.5, 20000), dtype))
    p = np.exp(-x)
    off = np.abs(rounded(p, dtype) - p) / 2.0 ** (np.floor(np.log2(p)) - BITS[dtype])
    best = x[np.argsort(-off)[:n]]
    assert off[np.argsort(-off)[n - 1]] > 0.9
    return best


def problem(heads, dtype, news, lens):
    hq, hkv, d = HEADS.get(heads, heads)
    st = Step(dtype, (hq, hkv, d), news, lens, seed=1)
    st.q.zero_()
    st.q[:, :, 0] = torch.from_numpy(exponents(hq, dtype))
    for k, v in zip(st.k_rows, st.v_rows):
        light = torch.arange(k.shape[1]) % 4 != 0  # (every tile has a key that scores 0: the reference of its exponents)
        k.zero_()
        k[:, light, 0] = -1.0
        v.copy_(light[None, :, None] * (1 + torch.arange(d) / d).to(v.dtype))
    return st


def definition(st, numerator=lambda p: p):
    """With scores times 1, in 64 bits; `numerator`: what becomes of the weights in the output product."""
    out = np.zeros((sum(st.news), st.heads[0], st.heads[2]))
    at = 0
    x, values = st.q[0, :, 0].double().numpy(), 1 + np.arange(st.heads[2]) / st.heads[2]
    for n, kv in zip(st.news, st.lens):
        for i in range(n):
            rows = kv - n + i + 1
            zeros = -(-rows // 4)
            p = np.exp(-x)
            weight = (rows - zeros) * numerator(p) / (zeros + (rows - zeros) * p)
            out[at + i] = weight[:, None] * values
        at += n
    return out


def sums(lens):
    return (max(lens) / 4 + 96) * 2.0 ** -24


def bound(st, want):
    """Half a unit of the result; the second operand's rounding, two halves of a unit of each numerator multiplied (and in f16 half the
    least number there is, next to numerators of 0.08 or more); exponentials to 2^-22 and 8 roundings of their exponents, up to 2.5;
    sums in 32 bits, of which one wave of four or eight adds up a quarter of the tiles at most."""
    half = 2.0 ** -BITS[st.dtype]
    unit = 2.0 ** (np.floor(np.log2(np.maximum(want, 1e-30))) - BITS[st.dtype])
    return unit + want * 1.02 * (half * half + 2.0 ** -21 + 2 * (2.0 ** -22 + 8 * 2.5 * 2.0 ** -24) + 2 * sums(st.lens))


CASES = [  # up to 16 query rows, up to 32; cut along the keys
    ("gqa", [1, 1, 1], [40, 300, 77]), ("small", [3, 1], [100, 290]), ("wide", [1, 1], [64, 200]), ((2, 2, 128), [20], [128]),
    ((2, 2, 64), [32, 17], [60, 250]), ("five", [1], [2400]), ("one", [1] * 70, [40 + i for i in range(69)] + [2400]),
]


@pytest.mark.parametrize("heads,news,lens", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_single_rounding_would_show(heads, news, lens, dtype):
    st = problem(heads, dtype, news, lens)
    want = definition(st)
    once = rounded(definition(st, lambda p: rounded(p, dtype)), dtype)
    rest = lambda p: rounded(p, dtype) + rounded(p - rounded(p, dtype), dtype)  # noqa: E731
    twice = rounded(definition(st, rest), dtype)
    limit = bound(st, want)
    assert (np.abs(twice - want) <= limit).all()
    assert (np.abs(once - want) > limit).any(axis=(0, 2)).all(), "every head would show it"


@pytest.mark.gpu
@pytest.mark.parametrize("heads,news,lens", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_few_rows(heads, news, lens, dtype):
    st = problem(heads, dtype, news, lens)
    want = definition(st)
    out, lse = st.run(scale=1.0)
    err = np.abs(out.double().numpy() - want) / bound(st, want)
    assert err.max() <= 1.0, float(err.max())
    x = st.q[0, :, 0].double().numpy()
    rows = np.concatenate([kv - n + 1 + np.arange(n) for n, kv in zip(news, lens)])[:, None]
    zeros = -(-rows // 4)
    want_lse = np.log(zeros + (rows - zeros) * np.exp(-x))
    assert np.abs(lse.double().numpy() - want_lse).max() <= 2.0 ** -22 + 8 * 2.5 * 2.0 ** -24 + sums(lens) + 4 * 2.0 ** -24 * math.log(max(lens))
