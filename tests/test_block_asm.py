"""Scratch memory in the kernels of the norms, the dropout and the sequences' losses: by the names in their sources and in the assembly of the current build (no GPU needed)."""
import os
import re

import pytest

from paper_2502_02581_amd import asm_check, build

SOURCES = ["norm.hip", "dropout.hip", "seq_loss.hip"]


@pytest.mark.parametrize("src", SOURCES)
def test_every_kernel_is_checked(src):
    with open(os.path.join(build.CSRC, src)) as f:
        names = re.findall(r"__global__[^;{]*?(\w+)\(", re.sub(r"__launch_bounds__\([^;{]*?\) (?=void)", "", f.read()))
    assert names and src in build.CHECKED
    for name in names:
        lines = [f"_ZN3moe{len(name)}{name}IxEEv:", "\ts_endpgm", "; ScratchSize: 16"]
        assert len(asm_check.check_no_scratch(lines)) == 1, name


@pytest.mark.parametrize("src", SOURCES)
def test_no_kernel_of_the_current_build_has_any(src):
    path = build.device_asm(src)
    if not os.path.exists(path):
        pytest.skip("the build step has not left its device assembly here")
    with open(path) as f:
        sizes = re.findall(r"^; ScratchSize: (\d+)", f.read(), re.M)
    assert sizes and set(sizes) == {"0"}
