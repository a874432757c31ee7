"""What test_gpu_ortho_parts.py holds orthogonalised updates to, looked at on the host: operands in two parts are within it, any of a product's three parts left
out is far outside, and its shapes reach every way that tiles are shared out."""
import pytest

import ortho_parts as O

LEFT_OUT = ["lows"] + [f"{product} {which}" for product in ("gram", "poly", "update") for which in ("hl", "lh")]
# (batch, rows, cols): one launch; tiles of 64; ... cut along a contraction; of 128; ... what is left of them cut
SHAPES = [(2, 40, 56), (1, 64, 128), (3, 13, 90), (1, 100, 130), (2, 333, 200), (1, 1000, 2100), (30, 600, 1100), (36, 640, 650), (4, 2100, 1000)]


@pytest.mark.parametrize("batch,m,n", SHAPES)
def test_parts_left_out_lie_outside(batch, m, n):
    G = O.wide(O.matrices(1, m, n, 5)[0])
    want, tolerance = O.exact(G), O.tolerance_of(m, n, 1)
    assert O.off_by(O.step(G), want) < 0.5 * tolerance
    for name in LEFT_OUT:
        assert O.off_by(O.step(G, (name,)), want) > 10 * tolerance, name


def test_shapes_reach_all_ways_of_sharing_out():
    ways = {(product, *way) for batch, m, n in SHAPES[3:] for product, way in O.tiles(batch, min(m, n), max(m, n)).items()}
    assert ways >= {(product, side, False) for product in ("gram", "poly", "update") for side in (64, 128)}
    assert ways >= {("gram", 64, True), ("poly", 64, True), ("gram", 128, True), ("poly", 128, True), ("update", 128, True)}
