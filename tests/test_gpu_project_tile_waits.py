"""Lost waits of products on the tensor cores, for each way in which blocks share the work: as test_gpu_project_waits.py, at sizes whose way is held against the library's choice."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_project_waits as waits  # noqa: E402
from test_gpu_project_tiles import plan  # noqa: E402

# width of a tile (0: the matrix-vector kernels), blocks that share its columns, whether blocks take several tiles; n, k, b, group, type, gated
CASES = [
    (0, 0, False, 300, 500, 9, 96, "bf16", 0), (0, 0, False, 300, 500, 9, 96, "f32", 1),
    (32, 1, True, 20000, 70, 17, 128, "f16", 0), (32, 4, False, 520, 390, 33, 64, "bf16", 0), (32, 6, False, 777, 700, 9, 128, "f32", 1),
    (64, 1, True, 20000, 130, 33, 128, "f16", 0), (64, 6, False, 130, 2600, 600, 32, "bf16", 0), (64, 3, False, 1500, 260, 33, 64, "f32", 1),
    (128, 1, True, 4000, 70, 1030, 128, "bf16", 0), (128, 3, False, 520, 1500, 1030, 128, "f16", 0), (128, 4, False, 130, 390, 1500, 64, "f32", 0), (128, 5, False, 130, 2600, 1030, 64, "f16", 1),
    (256, 1, True, 9000, 70, 800, 128, "bf16", 0), (256, 1, True, 6000, 70, 520, 32, "f16", 1), (256, 1, True, 20000, 70, 129, 32, "f32", 0),
]


@pytest.mark.parametrize("width,split,rounds,n,k,b,group,dtype,gated", CASES)
def test_cases_reach_what_they_are_for(width, split, rounds, n, k, b, group, dtype, gated):
    p = plan(n, k, b, group, dtype, gated)
    assert (p["width"], p["split"]) == (width, split) and (p["x_tiles"] * p["w_tiles"] > p["held"]) == rounds


@pytest.mark.gpu
@pytest.mark.parametrize("width,split,rounds,n,k,b,group,dtype,gated", CASES)
def test_a_lost_wait_gives_nan_and_says_so(width, split, rounds, n, k, b, group, dtype, gated):
    waits.test_a_lost_wait_gives_nan_and_says_so(n, k, b, group, dtype, bool(gated))
