"""What the compiler made of the serving step's kernels."""
import os
import re
import subprocess

from paper_2502_17421_amd import build as ls_build


def resources(name):
    if not os.path.exists(ls_build.RESOURCE_REPORT) or ls_build.is_stale():
        ls_build.build_library()
    return {k: v for k, v in ls_build.kernel_resources().items() if name in k}


def test_the_attention_kernels_keep_everything_in_registers():
    """They count their copies in flight (s_waitcnt vmcnt(N)); a spill would add loads and stores of its own to that count.  At most
    256 registers: two waves on a SIMD."""
    kernels = resources("chunk_attn_kernel")
    assert len(kernels) >= 8
    for name, r in kernels.items():
        assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0 and r["VGPRs"] + r["AGPRs"] <= 256, (name, r)


def test_the_other_kernels_use_no_scratch_memory():
    for name, least in (("page_plan_kernel", 2), ("rope_kernel", 12), ("chunk_merge_kernel", 4), ("chunk_list_kernel", 2)):
        kernels = resources(name)
        assert len(kernels) >= least, name
        for full, r in kernels.items():
            assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (full, r)


def test_only_the_copies_touch_m0(tmp_path):
    """The copies to LDS set M0 inside assembly, which cannot declare it clobbered: the compiler has to leave it alone, and each copy
    has to have its own move right before it."""
    asm = tmp_path / "chunk_attn.s"
    flags = [f for f in ls_build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([ls_build.HIPCC, *flags, "-S", "--cuda-device-only", "-o", str(asm), os.path.join(ls_build.CSRC, "ls_chunk_attn.hip")],
                   check=True, stderr=subprocess.DEVNULL)
    lines = [ln.split(";")[0].strip() for ln in asm.read_text().splitlines()]
    lines = [ln for ln in lines if ln]
    copies = [i for i, ln in enumerate(lines) if ln.startswith("global_load_lds_dword")]
    m0 = [i for i, ln in enumerate(lines) if re.search(r"\bm0\b", ln)]
    assert copies and m0 == [i - 2 for i in copies]
    for i in m0:
        assert re.fullmatch(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi|ttmp\d+)", lines[i]) and lines[i + 1] == "s_nop 0", lines[i:i + 3]
