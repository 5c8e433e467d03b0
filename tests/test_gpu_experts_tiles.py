"""The experts' products by tiles where a workgroup takes several, in tiles of 64 and of 128 rows of x, with both acts.

The tests name the form that they mean to reach and see from the library's rule, written out here once more, that a call
of theirs does: the rows of a tile, and more tiles than the 256 workgroups of a launch.
"""
import pytest

from tests.test_gpu_experts_precision import check_kept, exact_experts
from tests.test_gpu_mx4 import torch  # noqa: F401

pytestmark = pytest.mark.gpu

WORKGROUPS, WEIGHT_ROWS = 256, 256


def tile_us(rows, M, groups, outputs, blocks, mx4):
    tiles = M // rows + max(min(groups, M) // 2, 1)
    jobs = tiles * -(-outputs // WEIGHT_ROWS)
    one = 4.9 + 0.62 * -(-blocks // 8) if mx4 else 4 + 0.85 * -(-blocks // 4)
    return -(-jobs // WORKGROUPS) * one * (1 if rows == 64 else 1.2 if mx4 else 1.45)


def tile_rows(*args):
    return 128 if tile_us(128, *args) < tile_us(64, *args) else 64


# tokens, experts, a token's, D, I, ids; rows of a tile of the first product: (bf16, 4 bits)
SHAPES = [(3000, 8, 4, 96, 416, "distinct", (128, 128)), (6000, 8, 4, 544, 416, "bad", (128, 128)),
          (3000, 8, 4, 1056, 416, "distinct", (128, 128)), (2600, 24, 6, 288, 480, "distinct", (64, 128)),
          (5200, 5, 3, 64, 1152, "bad", (128, 128)), (1500, 64, 8, 160, 672, "any", (128, 128)),
          (4800, 300, 4, 416, 96, "any", (64, 64))]


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T,n,K,D,I,kind,rows", SHAPES)
def test_experts_of_several_tiles_a_workgroup(torch, T, n, K, D, I, kind, rows, act):  # noqa: F811
    P, mx4 = T * K, act == "mx4"
    assert P >= 64 * n and tile_rows(P, n, 2 * I, D // 32, mx4) == rows[mx4]
    e = exact_experts(T, n, K, D, I, kind, seed=D + I)
    pairs = int(((e.topk >= 0) & (e.topk < n)).sum())
    assert pairs // rows[mx4] * -(-2 * I // WEIGHT_ROWS) > WORKGROUPS
    check_kept(e, act)
    again = e.run(act)
    assert torch.equal(e.run(act)[:T, :D], again[:T, :D])
