"""Tensors that the binding of ls_tree_accept_sampled refuses, on the CPU, through the native module and through ctypes: other types, shapes, orders and
devices than the descriptor's would be read past their ends or as something else."""
import os

import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import build as ls_build
from paper_2502_17421_amd.paged_step import PagedCache

B, N, V = 3, 5, 40
NAMES = ("parents", "draft_tokens", "target_logits", "draft_logits", "temperature", "draft_temperature", "accept_uniforms", "sample_uniforms",
         "accept_path", "accept_len", "next_token", "logprobs", "err_flag")


@pytest.fixture(params=["native", "ctypes"])
def call(request, monkeypatch):
    if not os.path.exists(ls.LIB_PATH):
        ls_build.build_library()
    lib = ls.lib()
    with monkeypatch.context() as m:
        if request.param == "ctypes":
            m.setattr(ls, "CALL_PATH", ls.CALL_PATH + ".missing")
        made = ls._device_calls(lib, addresses=False, names=("ls_tree_accept_sampled",))
    assert (type(made.ls_tree_accept_sampled).__name__ == "Caller") == (request.param == "native")
    monkeypatch.setattr(lib, "call", made)
    monkeypatch.setattr(ls, "_stream", lambda stream: 0)
    return request.param


def tensors():
    both, each = (lambda dtype: torch.zeros((B, N), dtype=dtype)), (lambda dtype: torch.zeros(B, dtype=dtype))
    i, f = torch.int32, torch.float32
    return dict(zip(NAMES, (both(i), both(i), torch.zeros((B, N, V), dtype=torch.bfloat16), torch.zeros((B, N, V)), each(f), each(f), both(f), each(f), both(i),
                            each(i), each(i), both(f), each(i))))


def run(t, desc=None):
    """What the library says: there is no workspace, so that nothing is launched."""
    desc = desc or ls.make_sample_desc(tensors()["target_logits"], tensors()["draft_logits"])
    return ls.ls_tree_accept_sampled(desc, *(t[name] for name in NAMES), None, check=False)


def test_what_fits_reaches_the_library(call):
    assert run(tensors()) == ls.LS_ERR_WORKSPACE
    for name in ("draft_logits", "draft_temperature", "logprobs", "err_flag"):
        assert run(tensors() | {name: None}) == ls.LS_ERR_WORKSPACE
    for name in ("parents", "temperature", "target_logits"):
        assert run(tensors() | {name: None}) == ls.LS_ERR_NULL
    t = tensors()
    assert run(t | {"accept_len": t["accept_len"].view(B, 1), "parents": t["parents"].view(-1)}) == ls.LS_ERR_WORKSPACE
    wide = torch.zeros((B, N + 2, V + 3), dtype=torch.bfloat16)[:, :N, :V]
    assert run(t | {"target_logits": wide}, ls.make_sample_desc(wide, t["draft_logits"])) == ls.LS_ERR_WORKSPACE


@pytest.mark.parametrize("name", NAMES)
def test_what_does_not_fit_is_refused(call, name):
    x = tensors()[name]
    one = x.dim() == 1
    bad = [x.to(torch.int64), x.to(torch.float64), x[:2], torch.cat([x, x[:1]])]
    bad += [x.to(torch.int32 if x.dtype != torch.int32 else torch.float32), torch.zeros((B, 2), dtype=x.dtype)[:, 0] if one else x.transpose(0, 1)]
    if x.dim() == 2:
        bad += [x[:, :4], torch.zeros((B, N + 1), dtype=x.dtype)[:, :N], x.view(N, B)]
    if x.dim() == 3:
        bad += [x[:, :, ::2], x[0], torch.zeros((B, N, V + 2), dtype=x.dtype)[:, :, :V], x.transpose(0, 1).contiguous().transpose(0, 1)]
    for other in bad:
        with pytest.raises(ValueError, match=name):
            run(tensors() | {name: other})


def test_a_cache_refuses_them(call, monkeypatch):
    """Tokens as torch.multinomial gives them, temperatures in double."""
    monkeypatch.setattr(ls, "_check", lambda status, where: None)
    cache, t = PagedCache(B, 1, 1, 64, 4, 16, 32, torch.float32, device="cpu"), tensors()
    accept = lambda **new: cache.accept(*((t | new)[n] for n in NAMES[:5]), *((t | new)[n] for n in NAMES[6:11]))  # noqa: E731
    with pytest.raises(ValueError, match="draft_tokens"):
        accept(draft_tokens=torch.multinomial(torch.ones(B, V), N))
    with pytest.raises(ValueError, match="temperature"):
        accept(temperature=torch.ones(B, dtype=torch.float64))
