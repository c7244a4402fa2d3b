"""The plan of the operators on logits and on packed weights (csrc/lm/lm_plan.hpp, plain C++), compiled and asked without a GPU:
the sizes of the GPU tests reach the kernels that these name, every kernel is reached, and a team holds the rows it is chosen
for."""
import subprocess

import pytest

from paper_2302_02390_amd import build as lib_build

PRODUCTS = ["FEW_16_8", "FEW_16_4", "FEW_32_8", "FEW_32_4", "TILE_64_TEAMS", "TILE_64_DEEP", "TILE_64", "TILE_128", "TILE_256"]
TEAMS = ["T128", "T256", "T512", "T512_LDS", "T1024", "T1024_LDS", "STREAM"]
SOURCE = r"""
#include "lm/lm_plan.hpp"
#include <cstdio>
#include <cstdlib>
using namespace qsdp_lm;
int main(int argc, char** argv) {
    for (int i = 2; i < argc; ++i) {
        unsigned long a[4] = {};
        std::sscanf(argv[i], "%lu,%lu,%lu,%lu", a, a + 1, a + 2, a + 3);
        if (argv[1][0] == 'p') std::printf("%d\n", (int)choose_product(a[0], a[1], a[2], a[3]));       // m, n, k, buckets
        else if (argv[1][0] == 'r') std::printf("%d\n", (int)choose_row(row_pieces(a[0], a[1]), a[2]));  // n, per, four
        else std::printf("%d\n", (int)score_by_four(a[0], (int)a[1]));                                 // rows, top
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", lib_build.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)

    def answers(what, cases):
        args = [",".join(str(int(v)) for v in c) for c in cases]
        out = subprocess.run([str(at / "plan"), what] + args, check=True, capture_output=True, text=True).stdout
        return [int(v) for v in out.split()]
    return answers


def test_products_of_the_gpu_tests(ask):
    import test_gpu_lm_kernels as gpu
    asked = [(m, n, k, -(-k // bucket)) for _, m, n, k, bucket in gpu.PRODUCTS]
    got = [PRODUCTS[v] for v in ask("p", asked)]
    assert got == [c[0] for c in gpu.PRODUCTS]
    reached = {(name, c[3] > 1) for name, c in zip(got, asked)}
    assert reached == {(name, several) for name in PRODUCTS for several in (False, True)} - {("TILE_256", True),
                                                                                             ("TILE_64_TEAMS", False)}


def test_teams_share_a_tile_of_several_buckets_only(ask):
    """A tile of one bucket is faster without, but for weights that are in the caches."""
    sizes = [(m, n, k) for m in (33, 125, 512, 900) for n in (64, 1000, 2048, 16384) for k in (2048, 5000, 8192, 1 << 20)]
    assert all(PRODUCTS[v] != "TILE_64_TEAMS" for v in ask("p", [(m, n, k, 1) for m, n, k in sizes]))
    assert PRODUCTS[ask("p", [(125, 2048, 8192, 8)])[0]] == "TILE_64_TEAMS"


def test_rows_of_the_gpu_tests(ask):
    import test_gpu_lm_kernels as gpu
    for per, name in ((4, "f32"), (8, "16")):
        limits = gpu.LIMITS[name]
        for i, (n, team) in enumerate(limits):
            four = team == "T512_LDS"
            assert [TEAMS[v] for v in ask("r", [(n, per, 1), (n + 1, per, 1)])] == [team, (TEAMS + ["STREAM"])[i + 1]]
            if not four:
                assert TEAMS[ask("r", [(n, per, 0)])[0]] == team
        assert TEAMS[ask("r", [(limits[3][0], per, 0)])[0]] == "T1024"
        parts = {TEAMS[ask("r", [((-(-v // 8) + 7) // 8 * 8, per, 0)])[0]] for d, v in gpu.PARTS if (d == "f32") == (per == 4)}
        assert parts >= {"T1024", "T1024_LDS", "STREAM"}
    assert ask("f", [(511, 1), (512, 1), (1 << 30, 0), (520, 128)]) == [0, 1, 0, 1]


def test_a_team_holds_its_rows(ask):
    """Pieces of 16 bytes that a team's registers and LDS hold, for rows that start one element inside a piece."""
    room = {"T128": 256, "T256": 2048, "T512": 4096, "T512_LDS": 4096 + 2240, "T1024": 8192, "T1024_LDS": 8192 + 4800}
    for per in (4, 8):
        sizes = sorted({max(1, r * per + d) for r in room.values() for d in range(-17, 18)})
        for four in (0, 1):
            for n, v in zip(sizes, ask("r", [(n, per, four) for n in sizes])):
                lead = 1 if per == 8 else 0
                if TEAMS[v] != "STREAM":
                    assert -(-(n + lead) // per) <= room[TEAMS[v]], (n, per, four)
