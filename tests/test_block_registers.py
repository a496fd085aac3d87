"""Registers of the kernels of layer norm, dropout and rotary positions: which forms
keep what they hold in registers, and that the others spill no more than is known."""
import os
import re
import shutil
import subprocess

import pytest

PATH = "/opt/rocm/llvm/bin:" + os.environ.get("PATH", "")
OBJDUMP = shutil.which("llvm-objdump", path=PATH)
READELF = shutil.which("llvm-readelf", path=PATH)

# bytes of scratch a lane: type (f: fp32, t: bf16), what stands in front of the norm, how
# rows lie (1: whole chunks). All of rows above 8192 columns, whose lanes hold the sums of
# two chunks in 128 registers; forward, the same rows in fp32 with dropout
SPILLS_FORWARD = {("f", 2, 2): 24}
SPILLS = {("t", 0, 1): 8, ("t", 0, 2): 56, ("t", 0, 0): 52, ("t", 1, 2): 20, ("t", 1, 0): 40,
          ("t", 2, 2): 68, ("t", 2, 0): 140, ("f", 0, 2): 12, ("f", 0, 0): 72, ("f", 1, 1): 20,
          ("f", 1, 2): 132, ("f", 1, 0): 160, ("f", 2, 1): 76, ("f", 2, 2): 180, ("f", 2, 0): 216}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """(name, template arguments, scratch) of each."""
    from paper_2410_11720_amd import abft
    if OBJDUMP is None or READELF is None:
        pytest.skip("no disassembler")
    at = tmp_path_factory.mktemp("code")
    shutil.copy(abft.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    out = []
    for f in at.iterdir():
        if "gfx950" not in f.name or not f.stat().st_size:
            continue
        text = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True,
                              text=True).stdout
        for k in re.split(r"\n\s+- \.agpr_count:", text)[1:]:
            m = re.search(r"\.name:\s+\S*?\d((?:norm_fwd|norm_bwd|norm_join|rotary)_kernel|dropout_(?:flat|rows))"
                          r"(?:I(\S*))?", k)
            if m:
                args = m.group(2) or ""
                numbers = tuple(int(n) for n in re.findall(r"L[ib](\d+)E", args))
                scratch = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", k).group(1))
                out.append((m.group(1), args[:1], numbers, scratch))
    return out


def test_every_form_is_there(kernels):
    count = lambda name: sum(k[0] == name for k in kernels)
    # (seven widths, three things in front, three ways of rows, two types)
    assert count("norm_fwd_kernel") == count("norm_bwd_kernel") == 7 * 3 * 3 * 2
    assert count("norm_join_kernel") == 1
    assert (count("dropout_flat"), count("dropout_rows")) == (8, 4)
    assert count("rotary_kernel") == 4 * 2 * 2 * 2


def test_no_form_spills_but_the_widest(kernels):
    for name, dtype, numbers, scratch in kernels:
        known = {"norm_bwd_kernel": SPILLS, "norm_fwd_kernel": SPILLS_FORWARD}.get(name, {})
        most = known.get((dtype, *numbers[2:]), 0) if numbers[:2] == (0, 2) else 0
        assert scratch <= most, (name, dtype, numbers, scratch)
