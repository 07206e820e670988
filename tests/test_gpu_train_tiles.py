"""The gated block in every tile that its products take, whole and in parts, with an end
in every direction, and in the kernels for narrow rows, with each activation.
test_gated_plan.py checks that the calls reach the kernels they are meant for."""
import pytest
import torch

from tests.test_gpu_train_gated import ACTS, KINDS, check, make

pytestmark = pytest.mark.gpu

# rows, in, hidden, out; the tile of gate and up, of down, of the gradients of g and u, of
# dx; tile and parts (more than one) of the weights' gradients of gate and up, of down
TILES = [
    ((153, 71, 66, 66), (3, 3, 3, 3), (3, False), (3, False)),
    ((16_541, 146, 66, 136), (1, 1, 1, 1), (3, True), (3, True)),
    ((58_208, 218, 71, 584), (2, 2, 2, 2), (1, True), (0, True)),
    ((43_561, 312, 146, 491), (0, 1, 0, 0), (0, True), (1, True)),
    ((4945, 738, 922, 1581), (2, 0, 2, 3), (2, True), (2, True)),
    ((133, 531, 3366, 1284), (3, 3, 3, 3), (1, False), (1, False)),
    ((137, 2049, 2535, 3354), (3, 3, 3, 3), (2, False), (2, False)),
    ((788, 940, 2438, 1855), (1, 3, 1, 3), (0, False), (0, False)),
    ((1500, 1100, 4100, 2070), (2, 3, 2, 3), (2, False), (2, False)),
]
# The narrow kernels: 64 and 128 columns in and out.
NARROW = [(33_003, 61, 97, 64), (33_003, 61, 66, 125), (33_003, 128, 31, 50), (33_003, 100, 130, 128)]


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", [t[0] for t in TILES], ids=str)
def test_tiles(G, size, act, kind):
    check(G, *make(*size, KINDS[kind], sum(size)), act)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", NARROW, ids=str)
def test_narrow_rows(G, size, act, kind):
    check(G, *make(*size, KINDS[kind], sum(size)), act)


def test_tiles_of_aligned_widths(G):
    """Tables that are read where they lie, in the same tiles."""
    for size in ((16_541, 144, 72, 136), (58_208, 216, 72, 584), (4945, 736, 920, 1584),
                 (137, 2048, 2536, 3352), (788, 936, 2440, 1856)):
        check(G, *make(*size, torch.bfloat16, sum(size)), "silu")
