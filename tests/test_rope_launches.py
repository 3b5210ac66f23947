"""Rotary positions of more tokens than one launch can have threads for.  On the CPU: the built library with stand-ins for the HIP
calls that its launchers make."""
import os
import subprocess
import sys

from paper_2502_17421_amd import binding as ls
from paper_2502_17421_amd import build as ls_build

STANDIN = r"""
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim;
static dim grid, block;
int launches;
unsigned workgroups[512], threads[512];
void *pointers[512][8];
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int *v, int what, int d) { (void)what; (void)d; *v = 256; return 0; }
int hipGetLastError(void) { return 0; }
int __hipPushCallConfiguration(dim g, dim b, size_t m, void *s) { (void)m; (void)s; grid = g; block = b; return 0; }
int __hipPopCallConfiguration(dim *g, dim *b, size_t *m, void **s)
{
    *g = grid;
    *b = block;
    *m = 0;
    *s = NULL;
    return 0;
}
int hipLaunchKernel(const void *f, dim g, dim b, void **a, size_t m, void *s)
{
    (void)f; (void)m; (void)s;
    workgroups[launches] = g.x;
    threads[launches] = b.x;
    for (int i = 0; i < 8; ++i) pointers[launches][i] = ((void **)a[0])[i];  /* q, k, v, q_out, k_out, v_out, positions, slots */
    ++launches;
    return 0;
}
"""

CHILD = r"""
import ctypes, sys
sys.path.insert(0, sys.argv[3])
standin, lib = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
from paper_2502_17421_amd import binding as ls
vp = ctypes.c_void_p
lib.ls_rope.argtypes, lib.ls_rope_store_paged.argtypes = [vp] * 8, [vp] * 11
where = lambda i: (i + 1) << 44
for d, tokens_of_a_workgroup in ((128, 1), (64, 8)):
    for n in (1000000, 1 << 23, (1 << 24) - 1, 1 << 24, (1 << 25) + 12345, (1 << 31) - 1):
        for paged in (False, True):
            for elem, dtype in ((2, ls.LS_BF16), (4, ls.LS_F32)):
                x = ls.ls_rope_desc()
                x.n_tokens, x.n_q_heads, x.n_kv_heads, x.head_dim, x.rotary_dim, x.n_axes = n, 3, 1, d, d, 1
                x.sections[0], x.n_positions, x.dtype, x.page_size, x.n_pages = d // 2, 100, dtype, 16, 1 << 20
                for f, stride in ((x.q_stride, 5 * d), (x.k_stride, 2 * d), (x.v_stride, 3 * d), (x.qo_stride, 4 * d), (x.ko_stride, d)):
                    f[0], f[1] = stride, d
                for f in (x.kc_stride, x.vc_stride):
                    f[0], f[1], f[2] = 16 * d, 16 * d, d
                ctypes.c_int.in_dll(standin, "launches").value = 0
                q, k, v, positions, cos_sin, slots, q_out, k_out, v_out = (where(i) for i in range(9))
                if paged:
                    assert lib.ls_rope_store_paged(ctypes.byref(x), q, k, v, positions, cos_sin, slots, q_out, k_out, v_out, None) == 0
                else:
                    assert lib.ls_rope(ctypes.byref(x), q, k, positions, cos_sin, q_out, k_out, None) == 0
                done, launches = 0, ctypes.c_int.in_dll(standin, "launches").value
                assert launches <= 512
                for i in range(launches):
                    groups = (ctypes.c_uint * 512).in_dll(standin, "workgroups")[i]
                    assert groups * (ctypes.c_uint * 512).in_dll(standin, "threads")[i] < 1 << 32 and done < n
                    got = [p or 0 for p in ((vp * 8) * 512).in_dll(standin, "pointers")[i]]
                    at = lambda p, stride: p + done * stride * elem
                    want = [at(q, 5 * d), at(k, 2 * d), at(v, 3 * d) if paged else 0, at(q_out, 4 * d), k_out if paged else at(k_out, d),
                            v_out if paged else 0, positions + 4 * done, slots + 4 * done if paged else 0]
                    assert got == want, (d, n, paged, i)
                    done += groups * tokens_of_a_workgroup
                assert n <= done < n + tokens_of_a_workgroup, (d, n, done)
print("all tokens")
"""


def test_every_launch_fits(tmp_path):
    if not os.path.exists(ls.LIB_PATH):
        ls_build.build_library()
    (tmp_path / "standin.c").write_text(STANDIN)
    standin = str(tmp_path / "standin.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-Wall", "-o", standin, str(tmp_path / "standin.c")], check=True)
    r = subprocess.run([sys.executable, "-c", CHILD, standin, ls.LIB_PATH, os.path.dirname(os.path.dirname(os.path.abspath(__file__)))],
                       env=dict(os.environ, LD_PRELOAD=standin), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all tokens" in r.stdout, (r.stdout[-2000:], r.stderr[-2000:])
