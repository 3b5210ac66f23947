"""The entry points of sampled decoding on the CPU: layouts of their descriptors, refusals (nothing is launched), workspaces; and
what the plain implementations are held to themselves."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import sampling_reference as ref
from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import build as ls_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(ls.LIB_PATH):
        ls_build.build_library()
    return ls.lib()


def test_descriptor_layouts_match_c(tmp_path):
    structs = {"ls_sample_desc": ls.ls_sample_desc, "ls_copy_desc": ls.ls_copy_desc}
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


def at(i):
    """Stand-ins, never dereferenced: every call here is refused on the host."""
    return ctypes.c_void_p(256 * (i + 1))


BIG = 1 << 40


def sample_desc(**changes):
    d = ls.ls_sample_desc(4, 16, 1000, ls.LS_BF16, ls.LS_F32, 0)
    d.target_stride[:], d.draft_stride[:] = (16000, 1000), (16000, 1000)
    for key, value in changes.items():
        if isinstance(value, tuple):
            getattr(d, key)[value[0]] = value[1]
        else:
            setattr(d, key, value)
    return d


def test_tree_accept_sampled_refusals():
    call = lambda d, *a: ls.lib().ls_tree_accept_sampled(ctypes.byref(d) if d else None, *a, None)  # noqa: E731
    full = [at(i) for i in range(14)] + [BIG]
    assert call(None, *full) == ls.LS_ERR_NULL
    for i in (0, 1, 2, 4, 6, 7, 8, 9, 10):  # draft_logits, draft_temperature, logprobs and err_flag may be missing
        assert call(sample_desc(), *full[:i], None, *full[i + 1:]) == ls.LS_ERR_NULL, i
    assert call(sample_desc(), *full[:2], ctypes.c_void_p(257), *full[3:]) == ls.LS_ERR_STRIDE
    assert call(sample_desc(), *full[:3], ctypes.c_void_p(258), *full[4:]) == ls.LS_ERR_STRIDE
    for workspace, size in ((None, BIG), (ctypes.c_void_p(128), BIG), (at(13), 0)):
        assert call(sample_desc(), *full[:13], workspace, size) == ls.LS_ERR_WORKSPACE
    for changes, status in (({"batch": 0}, "SHAPE"), ({"n_tree": -1}, "SHAPE"), ({"vocab": 0}, "SHAPE"), ({"target_dtype": 3}, "DTYPE"),
                            ({"draft_dtype": -1}, "DTYPE"), ({"batch": 65536}, "UNSUPPORTED"), ({"n_tree": 513}, "UNSUPPORTED"),
                            ({"vocab": ls.LS_MAX_VOCAB + 1}, "UNSUPPORTED"), ({"target_stride": (0, -1)}, "STRIDE"),
                            ({"draft_stride": (1, -8)}, "STRIDE")):
        assert call(sample_desc(**changes), *full) == getattr(ls, "LS_ERR_" + status), changes
        size = ctypes.c_size_t()
        assert ls.lib().ls_sample_workspace_bytes(ctypes.byref(sample_desc(**changes)), ctypes.byref(size)) == getattr(ls, "LS_ERR_" + status)
    assert ls.lib().ls_sample_workspace_bytes(ctypes.byref(sample_desc()), None) == ls.LS_ERR_NULL


def page_desc(**changes):
    d = ls.ls_page_desc(4, 0, 16, 100, 8)
    for key, value in changes.items():
        setattr(d, key, value)
    return d


PAGE_CHANGES = (({"batch": 0}, "SHAPE"), ({"page_size": 0}, "SHAPE"), ({"n_pages": -1}, "SHAPE"), ({"bt_stride": 0}, "SHAPE"),
                ({"page_size": 24}, "UNSUPPORTED"), ({"batch": ls.LS_MAX_STEP_BATCH + 1}, "UNSUPPORTED"),
                ({"n_pages": ls.LS_MAX_POOL_PAGES + 1, "page_size": 1}, "UNSUPPORTED"), ({"n_pages": 1 << 20, "page_size": 1 << 11}, "UNSUPPORTED"),
                ({"bt_stride": (1 << 18) + 1}, "UNSUPPORTED"), ({"bt_stride": 1 << 17, "page_size": 1 << 14}, "UNSUPPORTED"))


def test_page_fork_refusals():
    call = lambda d, *a: ls.lib().ls_page_fork(ctypes.byref(d) if d else None, *a, None)  # noqa: E731
    full = [at(i) for i in range(15)] + [BIG]
    assert call(None, *full) == ls.LS_ERR_NULL
    for i in range(13):
        if i != 1:  # keep_lens may be missing, and err_flag
            assert call(page_desc(), *full[:i], None, *full[i + 1:]) == ls.LS_ERR_NULL, i
    for out in range(7, 14):
        for given in range(7):  # outputs over inputs
            assert call(page_desc(), *full[:out], full[given], *full[out + 1:]) == ls.LS_ERR_NULL, (out, given)
    assert call(page_desc(), *full[:11], ctypes.c_void_p(8), *full[12:]) == ls.LS_ERR_STRIDE
    for workspace, size in ((None, BIG), (ctypes.c_void_p(128), BIG), (at(14), 1000)):
        assert call(page_desc(), *full[:14], workspace, size) == ls.LS_ERR_WORKSPACE
    for changes, status in PAGE_CHANGES:
        assert call(page_desc(**changes), *full) == getattr(ls, "LS_ERR_" + status), changes
        with pytest.raises(ls.LsError):
            ls.ls_page_fork_workspace_bytes(page_desc(**changes))


def test_page_compact_refusals():
    call = lambda d, *a: ls.lib().ls_page_compact(ctypes.byref(d) if d else None, *a, None)  # noqa: E731
    full = [at(i) for i in range(8)] + [BIG]
    assert call(None, *full) == ls.LS_ERR_NULL
    for i in range(7):
        assert call(page_desc(), *full[:i], None, *full[i + 1:]) == ls.LS_ERR_NULL, i
    for out in range(2, 7):
        for given in range(2):
            assert call(page_desc(), *full[:out], full[given], *full[out + 1:]) == ls.LS_ERR_NULL, (out, given)
    assert call(page_desc(), *full[:5], ctypes.c_void_p(8), *full[6:]) == ls.LS_ERR_STRIDE
    for workspace, size in ((None, BIG), (ctypes.c_void_p(128), BIG), (at(7), 200)):
        assert call(page_desc(), *full[:7], workspace, size) == ls.LS_ERR_WORKSPACE
    for changes, status in PAGE_CHANGES:
        assert call(page_desc(**changes), *full) == getattr(ls, "LS_ERR_" + status), changes
        with pytest.raises(ls.LsError):
            ls.ls_page_compact_workspace_bytes(page_desc(**changes))


def copy_desc(**changes):
    d = ls.ls_copy_desc(2, 50, 8, 16, 256, 10)
    for s in (d.k_stride, d.v_stride):
        s[:] = (50 * 8 * 16 * 256, 8 * 16 * 256, 16 * 256, 256)
    for key, value in changes.items():
        if isinstance(value, tuple):
            getattr(d, key)[value[0]] = value[1]
        else:
            setattr(d, key, value)
    return d


def test_page_copy_refusals():
    call = lambda d, *a: ls.lib().ls_page_copy(ctypes.byref(d) if d else None, *a, None)  # noqa: E731
    full = [at(i) for i in range(4)]
    assert call(None, *full) == ls.LS_ERR_NULL
    for i in range(3):
        assert call(copy_desc(), *full[:i], None, *full[i + 1:]) == ls.LS_ERR_NULL, i
    for i in (0, 2, 3):
        assert call(copy_desc(), *full[:i], ctypes.c_void_p(264), *full[i + 1:]) == ls.LS_ERR_STRIDE, i
    for changes, status in (({"n_layers": 0}, "SHAPE"), ({"n_pages": 0}, "SHAPE"), ({"n_kv_heads": -1}, "SHAPE"), ({"page_size": 0}, "SHAPE"),
                            ({"row_bytes": 0}, "SHAPE"), ({"max_copies": 0}, "SHAPE"), ({"row_bytes": 40}, "STRIDE"),
                            ({"row_bytes": 65552}, "UNSUPPORTED"), ({"page_size": 1 << 24}, "UNSUPPORTED"),
                            ({"max_copies": ls.LS_MAX_POOL_PAGES + 1}, "UNSUPPORTED"),
                            ({"k_stride": (3, 248)}, "STRIDE"), ({"k_stride": (1, -4096)}, "STRIDE"), ({"v_stride": (2, 8)}, "STRIDE"),
                            ({"v_stride": (0, 0)}, "STRIDE"), ({"k_stride": (0, 0)}, "STRIDE")):
        assert call(copy_desc(**changes), *full) == getattr(ls, "LS_ERR_" + status), changes


def test_workspaces():
    """Large enough for what the kernels keep there: words per page and the pages given back; a bit and half a word per page."""
    for batch, pages, stride in ((1, 1, 1), (4, 100, 8), (300, 70001, 999)):
        d = page_desc(batch=batch, n_pages=pages, bt_stride=stride)
        assert ls.ls_page_fork_workspace_bytes(d) >= 4 * (2 * pages + batch * stride + 2 * batch)
        assert ls.ls_page_compact_workspace_bytes(d) >= 8 * -(-pages // 64) + 4 * -(-pages // 64) + 8
    assert ls.ls_sample_workspace_bytes(sample_desc()) >= 256


@pytest.mark.parametrize("with_replacement", [False, True])
def test_the_plain_verification_samples_the_target(with_replacement):
    """A node with two children over four tokens, every pair of children and a grid of random numbers: the first new token has the
    target's distribution to the grid's resolution."""
    target = np.array([[0.6, -0.4, 0.9, -1.5]] * 3)
    draft = np.array([[-0.2, 0.8, 0.1, -0.6]] * 3)
    p, q = (ref.softmax(x[0], 1.0)[0].astype(float) for x in (target, draft))
    grid = (np.arange(12) + 0.5) / 12
    mass = np.zeros(4)
    for x in range(4):
        for y in range(4):
            w = q[x] * (q[y] if with_replacement else 0.0 if x == y else q[y] / (1 - q[x]))
            if w == 0:
                continue
            for u1 in grid:
                for u2 in grid:
                    for u3 in grid[1::3]:
                        path, nxt, _, err = ref.accept_sampled([-1, 0, 0], [0, x, y], target, draft, 1.0, None, [0, u1, u2], u3, with_replacement)
                        assert err == 0
                        mass[[x, y][path[1] - 1] if len(path) > 1 else nxt] += w / 12 ** 2 / 4
    # each of the three numbers decides, of all that comes to it, half a step of its grid too much or too little at most
    assert np.abs(mass - p).max() <= 0.5 / 12 + 0.5 / 12 + 0.5 / 4
