"""Cross attention where a workgroup's tokens are of one head and pass LDS in tiles of their own, which in float are larger than the tiles of
positions: heads of every width, as many tokens as fill such a tile, less and more.  The last channels of the last tokens lie
furthest behind.  Tolerances are those of test_gpu_cross_attn.py."""
import pytest

from test_gpu_cross_attn import run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 32, 97, 40), (1, 1, 1, 32, 128, 40), (1, 3, 1, 32, 130, 9), (2, 2, 2, 32, 257, 33), (2, 2, 2, 31, 120, 17),
                                   (1, 1, 1, 64, 128, 20), (1, 1, 1, 96, 100, 20), (1, 3, 1, 128, 128, 20), (4, 8, 8, 32, 128, 70)], ids=str)
def test_tokens_of_one_head(shape, dtype):
    B, _, _, _, U, T = shape
    run_and_check(*shape, dtype)
    run_and_check(*shape, dtype, lengths=[T - 1] * B, q_lengths=[U - 1] * B, poison=True, seed=1)
