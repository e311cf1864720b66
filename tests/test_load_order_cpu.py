"""The order of loads that counted waits rest on, in the code that is built.

In luffy_moe_few's products on 4-bit weights a wave fetches a step's scales by
DMA into LDS, then two steps of eight weight loads, and waits later until all
but its eight newest loads have landed: that covers the scales only while at
least eight loads follow their DMA and none of those has moved before it."""
import os
import re
import shutil
import subprocess

import pytest


def blocks(path):
    """(kernel, the 'dma' and 'load' of a basic block) for the buffer loads of
    every luffy_moe_few product kernel."""
    name, out = None, []
    for line in open(path):
        m = re.match(r"^(\w*few_product_kernel\w*):", line)
        if m:
            name = m.group(1)
            out.append((name, []))
            continue
        if ".Lfunc_end" in line:
            name = None
        if name is None:
            continue
        s = line.split(";")[0].strip()
        if re.match(r"^\.LBB\S+:", s) or s.startswith(("s_cbranch", "s_branch")):
            out.append((name, []))
        elif s.startswith("buffer_load"):
            out[-1][1].append("dma" if s.endswith("lds") else "load")
    return out


def test_scales_are_older_than_the_loads_that_the_wait_leaves_out(tmp_path):
    from paper_2411_15419_amd import build
    if not (os.path.exists(build.HIPCC) or shutil.which(build.HIPCC)):
        pytest.skip("no hipcc")
    asm = tmp_path / "few.s"
    subprocess.run([build.HIPCC, "-w", *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "few.hip"),
                    "-o", str(asm)], check=True)
    seen = set()
    for name, ops in blocks(asm):
        if "dma" not in ops or "load" not in ops:
            continue
        last = len(ops) - 1 - ops[::-1].index("dma")
        assert "load" not in ops[:last], (name, ops)
        assert len(ops) - 1 - last >= 8, (name, ops)
        seen.add(name)
    assert len(seen) == 4, seen    # two products, up to 8 tokens and more
