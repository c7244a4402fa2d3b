"""The kernels of the operators on logits and on packed weights as the compiler leaves them (no GPU): which there are, their
registers, LDS and spilled registers."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor
from itertools import product

import pytest

from paper_2302_02390_amd import build as lib_build

FORMAT = "BF16"
TEAMS = [(128, 2, 0), (256, 8, 0), (512, 8, 0), (512, 8, 1), (1024, 8, 0), (1024, 8, 1), (1024, 8, 2)]  # threads, pieces, rest
HELD, STREAM = 1, 2


def _kernels(source, *defines):
    """{(name, template arguments as they are mangled): (registers, spilled, LDS)} of a source's kernels."""
    cmd = [lib_build.HIPCC] + lib_build.FLAGS + lib_build.LM_FLAGS + list(defines)
    cmd += ["--cuda-device-only", "-S", os.path.join(lib_build.CSRC, "lm", source), "-o", "-"]
    asm = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    found = re.findall(r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+_ZN7qsdp_lm12_GLOBAL__N_1\d+(\w+?_kernel)I(\S+?)EEv\S+"
                       r".*?\.vgpr_count:\s+(\d+)\s+\.vgpr_spill_count:\s+(\d+)", asm, re.S)
    return {(name, args): (int(registers), int(spilled), int(lds)) for lds, name, args, registers, spilled in found}


@pytest.fixture(scope="module")
def kernels():
    with ThreadPoolExecutor(2) as ex:
        rows = ex.submit(_kernels, "lm_rows.hip", f"-DQSDP_LM_FORMAT={FORMAT}")
        linear = ex.submit(_kernels, "lm_linear.hip")
        return rows.result(), linear.result()


def _row(args):
    """(threads, pieces, rest), further arguments."""
    m = re.fullmatch(rf"NS_\d{FORMAT}ELi(\d+)ELi(\d+)ELNS0_4RestE(\d)E(.*)", args)
    return tuple(int(v) for v in m.groups()[:3]), m.group(4)


def test_every_kernel_on_rows_is_one_that_calls_reach(kernels):
    """Alternatives of many rows alone take the four-workgroup team with LDS; parts are longer than the smallest team's rows."""
    rows, _ = kernels
    score = {_row(args) for name, args in rows if name == "score_kernel"}
    expected = {(t, f"Lb{top:d}ELb{part:d}E") for t, top, part in product(TEAMS, (0, 1), (0, 1))
                if not (t == TEAMS[0] and part) and not (t == TEAMS[3] and (part or not top))}
    assert score == expected
    distill = {_row(args) for name, args in rows if name == "distill_kernel"}
    assert distill == {(t, f"LNS0_6SecondE{more}E") for t, more in product(TEAMS, range(3))}
    assert len([1 for name, _ in rows if name not in ("score_kernel", "distill_kernel")]) == 3 + 2 + 1


def test_rows_stay_in_registers(kernels):
    """64 registers to a lane, so that a compute unit has 2048 threads, and LDS for two workgroups of 1024 or four of 512. The search
    for alternatives spills two registers at most, of what is the same for all rows' elements."""
    rows, _ = kernels
    for (name, args), (registers, spilled, lds) in rows.items():
        assert spilled <= (2 if name == "score_kernel" and "ELb1ELb" in args else 0), (name, args, spilled)
        if name in ("score_kernel", "distill_kernel"):
            (threads, _, rest), _ = _row(args)
            assert registers <= (128 if rest == STREAM else 64), (name, args, registers)
            assert lds <= 160 * 1024 * threads // 2048, (name, args, lds)


def test_registers_of_the_tiles(kernels):
    """256 registers to a lane for 256-wide tiles and 128-wide ones of several buckets, which spill some outside the loop over the
    codes; nothing else does."""
    _, linear = kernels
    for (name, args), (registers, spilled, lds) in linear.items():
        wide = name == "tiles_kernel" and args.startswith("Li256E")
        buckets = name == "tiles_kernel" and args.startswith("Li128E") and "ELb1E" in args
        assert spilled <= (16 if wide else 2 if buckets else 0), (name, args, spilled)
        assert registers <= 256 and lds <= 128 * 1024, (name, args, registers, lds)
    assert len(linear) == 9 + 12 + 24
