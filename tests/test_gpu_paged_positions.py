"""Positions at the ends of their type: a row sees the tokens j <= position that its sequence holds, whatever the number is."""
import numpy as np
import pytest

from tests.test_gpu_paged import check_attention

pytestmark = pytest.mark.gpu
MOST, LEAST = 2 ** 31 - 1, -2 ** 31


@pytest.mark.parametrize("positions", [[MOST] * 6, [LEAST] * 6, [MOST, LEAST, 0, MOST - 1, LEAST + 1, -1], [MOST - 62, MOST - 63, MOST - 64, 40, MOST, 39]])
@pytest.mark.parametrize("H,G,D", [(8, 2, 128), (4, 4, 64), (16, 1, 128)])
@pytest.mark.parametrize("lens,rows,width,max_keys", [
    ([41, 200, 70], [3, 2, 1], 13, 0),      # whole sequences; their last pages end in tokens that hold anything
    ([41, 3000, 70], [3, 2, 1], 190, 0),    # split
    ([9] * 64, [6] + [0] * 63, 2, 20)])     # by the wave
def test_positions_at_the_ends_of_the_type(positions, H, G, D, lens, rows, width, max_keys):
    check_attention(np.random.RandomState(len(lens) + D), "amxfp4_e5m2", H, G, D, 16, lens, rows, width=width, positions=np.array(positions),
                    max_keys=max_keys)
