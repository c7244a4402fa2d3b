"""The sizes of the GPU tests of tiles that are wider than the matrix take the tiles they are meant for (plain C++, no GPU)."""
from test_train_plan import TILES, ask  # noqa: F401


def test_tiles(ask):  # noqa: F811
    import test_gpu_blocks_tiles as gpu
    for at, exact in ((3, 0), (4, 1)):
        assert [TILES[v] for v in ask("p", [(*c[:3], exact) for c in gpu.CASES])] == [c[at] for c in gpu.CASES]
    assert any(c[0] < 128 and c[3] == "T128" for c in gpu.CASES) and any(c[0] < 256 and c[3] == "T256" for c in gpu.CASES)
