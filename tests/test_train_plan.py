"""The plan of the training operators (csrc/train/train_plan.hpp, plain C++), compiled and asked without a GPU: the sizes of the GPU
tests reach every kernel, and a team holds the rows it is chosen for."""
import subprocess

import pytest

from paper_2302_02390_amd import build as lib_build

TILES = ["T64", "T128", "T256", "T64_4"]
NORMS = ["T64", "T64_2", "T128_2", "T256_2", "T512_2", "T1024_2", "T1024_4", "SHORT", "STREAM"]
BACKWARD = ["T64", "T128", "T256", "T512", "T1024", "T512_4", "STREAM"]
ROOM = {"T64": 512, "T64_2": 1024, "T128": 1024, "T128_2": 2048, "T256": 2048, "SHORT": 2048, "T256_2": 4096, "T512": 4096,
        "T512_2": 8192, "T1024": 8192, "T512_4": 16384, "T1024_2": 16384, "T1024_4": 32768}
SOURCE = r"""
#include "train/train_plan.hpp"
#include <cstdio>
using namespace qsdp_train;
int main(int argc, char** argv) {
    for (int i = 2; i < argc; ++i) {
        unsigned long a[4] = {};
        std::sscanf(argv[i], "%lu,%lu,%lu,%lu", a, a + 1, a + 2, a + 3);
        switch (argv[1][0]) {
            case 'p': std::printf("%d\n", (int)choose_tile(a[0], a[1], a[2], a[3] != 0)); break;
            case 'f': std::printf("%d\n", (int)choose_few(a[0], a[1])); break;
            case 'P': std::printf("%lu\n", (unsigned long)choose_parts(a[0], a[1], a[2])); break;
            case 'F': std::printf("%lu\n", (unsigned long)choose_few_parts(a[0], a[1])); break;
            case 'n': std::printf("%d\n", (int)choose_norm(a[0], a[1])); break;
            case 'b': std::printf("%d\n", (int)choose_norm_backward(a[0])); break;
            case 'w': std::printf("%lu\n", (unsigned long)norm_workgroups(a[0], a[1])); break;
        }
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


def test_products_of_the_gpu_tests_reach_every_kernel(ask):
    import test_gpu_blocks as gpu
    for exact, expected in ((0, set(TILES)), (1, {"T64", "T128"})):
        assert {TILES[v] for v in ask("p", [(*p, exact) for p in gpu.PRODUCTS])} == expected
    few = [(n, k) for m, n, k in gpu.PRODUCTS if m <= 16]
    kernels = ask("f", few)
    assert set(kernels) == {0, 1, 2}
    wide = [(n, k) for (n, k), v in zip(few, kernels) if v == 2]
    assert any(k <= 2048 for _, k in wide) and any(k > 2048 for _, k in wide) and any(n > 512 * 16 for n, _ in wide)
    assert {1, 2, 4} <= set(ask("P", gpu.PRODUCTS)) and {1, 2, 5} <= set(ask("F", few))


def test_parts_of_a_sum_are_none_empty(ask):
    cases = [(1, n, k) for n in (1, 100, 2048, 4096, 20000) for k in list(range(1, 6000, 127)) + [8192, 12345, 1 << 20]]
    for what, args in (("P", cases), ("F", [c[1:] for c in cases])):
        for (_, n, k), parts in zip(cases, ask(what, args)):
            steps = -(-k // 128)
            each = -(-steps // parts)
            assert 1 <= parts <= steps and (parts - 1) * each < steps and -(-n // 64) * parts <= max(448, -(-n // 64))
    assert ask("P", [(0, 100, 10000)]) == [1]


def test_rows_of_the_gpu_tests_reach_every_kernel(ask):
    import test_gpu_norm as gpu
    sizes = [(rows, n) for rows, n, _, _ in gpu.SHAPES]
    assert {NORMS[v] for v in ask("n", sizes)} == set(NORMS)
    assert {BACKWARD[v] for v in ask("b", [(n,) for _, n in sizes])} == set(BACKWARD)


def test_a_team_holds_its_rows(ask):
    sizes = sorted({n + d for n in ROOM.values() for d in (-1, 0, 1)} | {1})
    for rows in (1, 1 << 20):
        for n, v in zip(sizes, ask("n", [(rows, n) for n in sizes])):
            assert n <= ROOM.get(NORMS[v], 1 << 62)
    for n, v in zip(sizes, ask("b", [(n,) for n in sizes])):
        assert n <= ROOM.get(BACKWARD[v], 1 << 62)


def test_workgroups_of_the_backward_pass(ask):
    assert ask("w", [(0, 100), (1, 100), (16, 512), (17, 512), (1 << 30, 2048), (3, 16384), (1000, 16385), (5, 20000)]) == [
        0, 1, 1, 2, 256, 3, 32, 5]
