"""The kernels of a training step's operators as the compiler leaves them (no GPU): which there are, their registers, LDS and spilled
registers."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2302_02390_amd import build as lib_build


def _kernels(source):
    """{(name, template arguments as they are mangled): (registers, spilled, LDS)} of a source's kernels."""
    cmd = [lib_build.HIPCC] + lib_build.FLAGS + lib_build.LM_FLAGS
    cmd += ["--cuda-device-only", "-S", os.path.join(lib_build.CSRC, "train", source), "-o", "-"]
    asm = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    found = re.findall(r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+_ZN10qsdp_train12_GLOBAL__N_1\d+(\w+?_kernel)(?:I(\S+?)EEv|E)\S+"
                       r".*?\.vgpr_count:\s+(\d+)\s+\.vgpr_spill_count:\s+(\d+)", asm, re.S)
    return {(name, args): (int(registers), int(spilled), int(lds)) for lds, name, args, registers, spilled in found}


@pytest.fixture(scope="module")
def kernels():
    with ThreadPoolExecutor(4) as ex:
        return dict(zip(("norm", "product", "adamw", "blocks"),
                        ex.map(_kernels, [f"train_{n}.hip" for n in ("norm", "product", "adamw", "blocks")])))


def _numbers(args):
    return tuple(int(v) for v in re.findall(r"L[ib](\d+)E", args + "E"))


def test_every_product_is_one_that_calls_reach(kernels):
    """Tiles by whether the weight's blocks are square, the result exact, the sum in parts, and teams: those of 256 in 16 bits alone,
    parts in tiles of 64 alone, which hold four steps (or three, if they are many), or two teams' two where the result is exact."""
    found = kernels["product"]
    tiles = {_numbers(args) for name, args in found if name == "tiles_kernel"}
    both = (0, 1)
    expected = {(64, 64, 32, 32, 2, square, 1, parts, 2) for square in both for parts in both}
    expected |= {(64, 64, 32, 32, 4, square, 0, parts, 1) for square in both for parts in both}
    expected |= {(64, 64, 32, 32, 3, square, 0, 0, 1) for square in both}
    expected |= {(128, 128, 64, 64, 2, square, exact, 0, 1) for square in both for exact in both}
    expected |= {(256, 256, 64, 128, 2, square, 0, 0, 1) for square in both}
    assert tiles == expected
    few = [(_numbers(args)) for name, args in found if name == "few_kernel"]
    assert sorted(few) == sorted([(groups, parts, exact) for groups, parts in ((1, 0), (1, 1), (2, 0)) for exact in (0, 1)] * 3)
    assert len([1 for name, _ in found if name == "few_wide_kernel"]) == 3 * 2 * 2
    assert len([1 for name, _ in found if name == "join_kernel"]) == 3 and len(found) == len(expected) + 18 + 12 + 3


def test_registers_and_lds(kernels):
    """Tiles of 256 by blocks of a row spill four addresses; rows of 32 elements to a thread spill what a step of the loop keeps beside
    both tensors. Nothing else does, but few registers of the longest rows forward."""
    for group, found in kernels.items():
        for (name, args), (registers, spilled, lds) in found.items():
            numbers = _numbers(args)
            allowed = 0
            if name == "tiles_kernel" and numbers[0] == 256:
                allowed = 0 if numbers[5] else 4
            elif name == "norm_backward_kernel" and numbers[-1] == 4:
                allowed = 96 if "3F32" in args else 16
            elif name == "norm_kernel" and numbers[-1] == 4:
                allowed = 8
            assert spilled <= allowed, (name, args, spilled)
            assert registers <= 256 and lds <= 160 * 1024, (name, args, registers, lds)
    for (name, args), (registers, _, lds) in kernels["product"].items():
        if name == "tiles_kernel" and _numbers(args)[0] == 128:
            assert 2 * lds <= 160 * 1024
        if name == "few_wide_kernel" and _numbers(args)[0] == 1:
            assert registers <= 128 and 2 * lds <= 160 * 1024
