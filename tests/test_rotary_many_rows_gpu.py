"""Rotary positions of calls with so many rows that a CTA takes two of them: odd numbers of rows, ragged sequences, rows at
negative positions, a padding slot, both pair layouts, in place and not."""
import pytest

import test_rotary as one
from test_rotary import dp, torch  # noqa: F401  (the fixtures)

pytestmark = pytest.mark.gpu

# rows of each sequence, lengths with them, heads, head dim, rotated dims
SHAPES = [([2501], [70000], 3, 128, 128), ([1301, 1300, 7], [1301, 131072, 5], 2, 128, 64), ([2601], [2600], 1, 64, 64),
          ([901, 0, 900, 33], [134217728, 7, 899, 0], 5, 64, 32), ([2433], [9000], 2, 256, 256), ([2450, 1], [2450, 1], 2, 512, 512),
          ([2435], [5000], 9, 80, 48)]


@pytest.mark.parametrize("ns,lens,H,D,r", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("place", ["apart", "in place", "strided in place"])
def test_rotary(dp, torch, ns, lens, H, D, r, interleaved, place):  # noqa: F811
    # two rows a CTA: from 8 CTAs an SM on, of the most rows that the call may have
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert max(ns) * len(ns) >= 16 * sms and r % 16 == 0 and D % 16 == 0
    one.test_rotary(dp, torch, ns, lens, H, D, r, interleaved, place)
