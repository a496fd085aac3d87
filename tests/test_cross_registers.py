"""Registers of the attention kernels over keys of another length: which forms
keep what they hold in registers, and that the others spill no more than is
known. Three workgroups of the query pass share a CU, which 12 waves of at most
168 registers do."""
import os
import re
import shutil
import subprocess

import pytest

PATH = "/opt/rocm/llvm/bin:" + os.environ.get("PATH", "")
OBJDUMP = shutil.which("llvm-objdump", path=PATH)
READELF = shutil.which("llvm-readelf", path=PATH)

# registers that a form spills at most: kernel, type (f: fp32, t: bf16), head dim,
# bias, waves on rows and on the other axis (query pass: workgroups a CU too).
# Key pass: two gradients' sums, fragments and a block's scores pass 256 registers
# at two waves a SIMD; grids that fill the chip take the forms without (t, 64 and
# t, 128: 4, 2; f, 128: 4, 1)
SPILLS = {
    ("kv", "f", 64, 0, "1,4"): 33, ("kv", "f", 64, 0, "2,2"): 21, ("kv", "f", 64, 0, "4,1"): 18,
    ("kv", "f", 128, 1, "4,1"): 4,
    ("kv", "t", 128, 0, "2,2"): 10, ("kv", "t", 128, 1, "2,4"): 53,
    ("q", "t", 128, 1, "1,4,2"): 9, ("q", "t", 128, 1, "2,2,2"): 5,
    ("q", "t", 64, 1, "2,2,3"): 5, ("q", "t", 64, 1, "4,1,3"): 1,
}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_2410_11720_amd import abft
    if OBJDUMP is None or READELF is None:
        pytest.skip("no disassembler")
    at = tmp_path_factory.mktemp("code")
    shutil.copy(abft.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    out = {}
    for f in at.iterdir():
        if "gfx950" not in f.name or not f.stat().st_size:
            continue
        text = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True,
                              text=True).stdout
        for k in re.split(r"\n\s+- \.agpr_count:", text)[1:]:
            number = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", k).group(1))
            m = re.search(r"\.name:\s+\S*cross_(?:bwd_)?(fwd|q|kv|short)_kernelI([ft])((?:L[ib]\d+E)+)E", k)
            if m:
                n = re.findall(r"L[ib](\d+)E", m.group(3))
                out[(m.group(1), m.group(2), int(n[0]), int(n[1]), ",".join(n[2:]))] = (
                    number("vgpr_count"), number("vgpr_spill_count"),
                    number("private_segment_fixed_size"))
    return out


def test_every_form_is_there(kernels):
    count = lambda kind: sum(k[0] == kind for k in kernels)
    # (no fourth wave split for fp32 rows of 512 bytes; three workgroups a CU of
    # the query pass at head dim 64 in bf16; eight waves of the key pass at 128)
    assert (count("fwd"), count("short"), count("q"), count("kv")) == (22, 8, 26, 22)


def test_forward_keeps_its_registers(kernels):
    for k, (_, spilled, scratch) in kernels.items():
        if k[0] in ("fwd", "short"):
            assert spilled == 0 and scratch == 0, (k, spilled, scratch)


def test_backward_spills_no_more_than_known(kernels):
    for k, (_, spilled, scratch) in kernels.items():
        assert spilled <= SPILLS.get(k, 0), (k, spilled)
        assert (scratch > 0) == (spilled > 0), (k, spilled, scratch)
    assert set(SPILLS) <= set(kernels)


def test_three_workgroups_a_cu(kernels):
    three = {k: v[0] for k, v in kernels.items() if k[0] == "q" and k[4].endswith(",3")}
    assert len(three) == 4 and max(three.values()) <= 168, three
