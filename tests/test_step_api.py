"""The entry points of a serving step on the CPU: layouts of their descriptors, refusals (nothing is launched), and the
workspace."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import build as ls_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(ls.LIB_PATH):
        ls_build.build_library()
    return ls.lib()


def test_descriptor_layouts_match_c(tmp_path):
    structs = {"ls_page_desc": ls.ls_page_desc, "ls_rope_desc": ls.ls_rope_desc, "ls_chunk_desc": ls.ls_chunk_desc}
    lines = []
    for name, s in structs.items():
        lines.append(f'printf("%zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {field[0]}));' for field in s._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ls_attn.h"\nint main(void){' + "".join(lines) + " return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, s in zip(out, structs.values()):
        assert [int(x) for x in line.split()] == [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]


ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(260)  # never dereferenced: every call here is refused on the host


def page_desc(**changes):
    d = ls.ls_page_desc(4, 16, 16, 100, 8)
    for key, value in changes.items():
        setattr(d, key, value)
    return d


def plan_args(**changes):
    """Distinct stand-ins in the order of the entry point."""
    names = ("kv_lens", "new_lens", "pages_held", "block_table", "free_pages", "free_count", "new_pages_held", "new_free_count",
             "cu_new", "total_lens", "slots", "positions", "err_flag")
    args = {name: ctypes.c_void_p(256 * (i + 1)) for i, name in enumerate(names)}
    args.update(changes)
    return [args[name] for name in names] + [None]


def test_page_plan_refusals():
    call = ls.lib().ls_page_plan
    assert call(None, *plan_args()) == ls.LS_ERR_NULL
    for name in ("kv_lens", "new_lens", "pages_held", "block_table", "free_pages", "free_count", "new_pages_held", "new_free_count",
                 "cu_new", "total_lens", "slots", "positions"):
        assert call(ctypes.byref(page_desc()), *plan_args(**{name: None})) == ls.LS_ERR_NULL, name
    for name in ("new_pages_held", "total_lens", "err_flag"):  # outputs over inputs
        assert call(ctypes.byref(page_desc()), *plan_args(**{name: ctypes.c_void_p(512)})) == ls.LS_ERR_NULL, name
    for field in ("batch", "page_size", "n_pages", "bt_stride"):
        for value in (0, -1):
            assert call(ctypes.byref(page_desc(**{field: value})), *plan_args()) == ls.LS_ERR_SHAPE, field
    assert call(ctypes.byref(page_desc(n_tokens=-1)), *plan_args()) == ls.LS_ERR_SHAPE
    for changes in ({"page_size": 24}, {"batch": ls.LS_MAX_STEP_BATCH + 1}, {"n_pages": 1 << 27}, {"bt_stride": (1 << 18) + 1},
                    {"n_tokens": (1 << 30) + 1}):
        assert call(ctypes.byref(page_desc(**changes)), *plan_args()) == ls.LS_ERR_UNSUPPORTED, changes


def rope_desc(**changes):
    d = ls.ls_rope_desc()
    d.n_tokens, d.n_q_heads, d.n_kv_heads, d.head_dim, d.rotary_dim, d.n_axes = 10, 8, 2, 128, 128, 1
    d.sections[0], d.n_positions, d.dtype, d.page_size, d.n_pages = 64, 1000, ls.LS_BF16, 16, 50
    for f, h in ((d.q_stride, 8), (d.k_stride, 2), (d.v_stride, 2), (d.qo_stride, 8), (d.ko_stride, 2)):
        f[0], f[1] = h * 128, 128
    for f in (d.kc_stride, d.vc_stride):
        f[0], f[1], f[2] = 2 * 16 * 128, 16 * 128, 128
    for key, value in changes.items():
        if isinstance(value, tuple):
            getattr(d, key)[value[0]] = value[1]
        else:
            setattr(d, key, value)
    return d


def test_rope_refusals():
    L = ls.lib()
    store = lambda d, *p: L.ls_rope_store_paged(ctypes.byref(d) if d else None, *p, None)  # noqa: E731
    full = [ONE] * 9
    assert store(None, *full) == ls.LS_ERR_NULL
    for i in range(9):
        assert store(rope_desc(), *full[:i], None, *full[i + 1:]) == ls.LS_ERR_NULL, i
    for i in (0, 1, 2, 4, 6, 7, 8):  # rows and the table of cosines are 16-byte aligned
        assert store(rope_desc(), *full[:i], ODD, *full[i + 1:]) == ls.LS_ERR_STRIDE, i
    plain = lambda d, *p: L.ls_rope(ctypes.byref(d) if d else None, *p, None)  # noqa: E731
    six = [ONE] * 6
    assert plain(None, *six) == ls.LS_ERR_NULL
    for i in range(6):
        assert plain(rope_desc(), *six[:i], None, *six[i + 1:]) == ls.LS_ERR_NULL, i  # k without k_out, and k_out without k
    for changes, status in (({"n_tokens": 0}, "SHAPE"), ({"n_q_heads": 0}, "SHAPE"), ({"n_kv_heads": -1}, "SHAPE"),
                            ({"rotary_dim": 0}, "SHAPE"), ({"rotary_dim": 144}, "SHAPE"), ({"rotary_dim": 64}, "SHAPE"),
                            ({"n_axes": 0}, "SHAPE"), ({"n_axes": 2, "sections": (1, 1)}, "SHAPE"), ({"sections": (0, 63)}, "SHAPE"),
                            ({"n_axes": 2, "sections": (1, -1)}, "SHAPE"),
                            ({"n_positions": 0}, "SHAPE"), ({"dtype": 3}, "DTYPE"), ({"head_dim": 96, "rotary_dim": 64, "sections": (0, 32)}, "UNSUPPORTED"),
                            ({"rotary_dim": 40, "sections": (0, 20)}, "UNSUPPORTED"), ({"n_axes": 5}, "UNSUPPORTED"),
                            ({"q_stride": (0, 132)}, "STRIDE"), ({"q_stride": (1, -128)}, "STRIDE"), ({"qo_stride": (1, 64)}, "STRIDE"),
                            ({"kc_stride": (2, 120)}, "STRIDE"), ({"vc_stride": (0, 0)}, "STRIDE"), ({"page_size": 24}, "UNSUPPORTED"),
                            ({"page_size": 0}, "SHAPE"), ({"n_pages": 0}, "SHAPE"), ({"n_pages": 1 << 27}, "UNSUPPORTED")):
        assert store(rope_desc(**changes), *full) == getattr(ls, "LS_ERR_" + status), changes
    assert plain(rope_desc(ko_stride=(0, 0)), *six) == ls.LS_ERR_STRIDE
    assert plain(rope_desc(n_axes=5), *six) == ls.LS_ERR_UNSUPPORTED


def chunk_desc(**changes):
    d = ls.ls_chunk_desc()
    d.batch, d.n_tokens, d.max_new_len, d.max_kv_len, d.n_q_heads, d.n_kv_heads, d.head_dim = 2, 100, 60, 1000, 8, 2, 128
    d.dtype, d.page_size, d.bt_stride, d.window, d.softmax_scale = ls.LS_BF16, 16, 64, 0, 0.0
    for f in (d.q_stride, d.o_stride):
        f[0], f[1] = 8 * 128, 128
    for f in (d.kc_stride, d.vc_stride):
        f[0], f[1], f[2] = 2 * 16 * 128, 16 * 128, 128
    for key, value in changes.items():
        if isinstance(value, tuple):
            getattr(d, key)[value[0]] = value[1]
        else:
            setattr(d, key, value)
    return d


def test_chunk_refusals():
    L = ls.lib()
    big = 1 << 40
    call = lambda d, p, ws=ONE, n=big: L.ls_chunk_attn_paged(ctypes.byref(d) if d else None, *p, ws, n, None)  # noqa: E731
    full = [ONE] * 8
    assert call(None, full) == ls.LS_ERR_NULL
    for i in range(8):
        assert call(chunk_desc(), full[:i] + [None] + full[i + 1:]) == ls.LS_ERR_NULL, i
    for i in (0, 1, 2, 6):
        assert call(chunk_desc(), full[:i] + [ODD] + full[i + 1:]) == ls.LS_ERR_STRIDE, i
    assert call(chunk_desc(), full, None) == ls.LS_ERR_WORKSPACE
    assert call(chunk_desc(), full, ODD) == ls.LS_ERR_WORKSPACE
    assert call(chunk_desc(), full, ONE, 16) == ls.LS_ERR_WORKSPACE
    for changes, status in (({"batch": 0}, "SHAPE"), ({"n_tokens": 0}, "SHAPE"), ({"max_new_len": 0}, "SHAPE"), ({"max_new_len": 101}, "SHAPE"),
                            ({"max_kv_len": -1}, "SHAPE"), ({"max_kv_len": 1025}, "SHAPE"), ({"n_q_heads": 7}, "SHAPE"), ({"window": -1}, "SHAPE"),
                            ({"page_size": 0}, "SHAPE"), ({"softmax_scale": float("nan")}, "SHAPE"), ({"softmax_scale": -1.0}, "SHAPE"),
                            ({"dtype": 5}, "DTYPE"), ({"dtype": ls.LS_F32}, "UNSUPPORTED"), ({"head_dim": 80}, "UNSUPPORTED"),
                            ({"page_size": 8, "bt_stride": 200}, "UNSUPPORTED"), ({"page_size": 48}, "UNSUPPORTED"),
                            ({"batch": ls.LS_MAX_STEP_BATCH + 1}, "UNSUPPORTED"), ({"n_tokens": 1 << 25}, "UNSUPPORTED"),
                            ({"q_stride": (0, 1028)}, "STRIDE"), ({"q_stride": (1, -128)}, "STRIDE"), ({"o_stride": (1, 64)}, "STRIDE"),
                            ({"kc_stride": (2, 64)}, "STRIDE"), ({"vc_stride": (2, 1 << 24)}, "UNSUPPORTED")):
        assert call(chunk_desc(**changes), full) == getattr(ls, "LS_ERR_" + status), changes
        n = ctypes.c_size_t(0)
        assert L.ls_chunk_workspace_bytes(ctypes.byref(chunk_desc(**changes)), ctypes.byref(n)) == getattr(ls, "LS_ERR_" + status)
    assert L.ls_chunk_workspace_bytes(ctypes.byref(chunk_desc()), None) == ls.LS_ERR_NULL
    assert L.ls_chunk_workspace_bytes(None, ctypes.byref(ctypes.c_size_t(0))) == ls.LS_ERR_NULL


def test_workspace_is_stable_and_aligned():
    for changes in ({}, {"max_new_len": 1, "n_tokens": 2}, {"n_tokens": 5000, "max_new_len": 4000}, {"head_dim": 64}, {"batch": 300, "n_tokens": 300}):
        n = ls.ls_chunk_workspace_bytes(chunk_desc(**changes))
        assert n > 0 and n % 256 == 0 and n == ls.ls_chunk_workspace_bytes(chunk_desc(**changes))


@pytest.mark.parametrize("native", [True, False])
def test_calls_reach_the_library_through_either_binding(native, monkeypatch):
    if not native:
        monkeypatch.setattr(ls, "CALL_PATH", ls.CALL_PATH + ".missing")
    made = ls._device_calls(ls.lib(), addresses=False, names=ls._STEP_CALLS)
    assert (type(made.ls_page_plan).__name__ == "Caller") == native
    some = torch.zeros(4, dtype=torch.int32)
    assert made.ls_page_plan(page_desc(batch=0), *[some] * 13, 0) == ls.LS_ERR_SHAPE
    assert made.ls_rope(rope_desc(n_axes=0), *[some] * 6, 0) == ls.LS_ERR_SHAPE
    assert made.ls_rope_store_paged(rope_desc(), None, *[some] * 8, 0) == ls.LS_ERR_NULL
    assert made.ls_chunk_attn_paged(chunk_desc(window=-1), *[some] * 8, some, some.nbytes, 0) == ls.LS_ERR_SHAPE
    with pytest.raises(TypeError):
        made.ls_page_plan(page_desc())
    if native:
        with pytest.raises(TypeError, match="ls_rope_desc"):
            made.ls_rope(page_desc(), *[some] * 6, 0)
