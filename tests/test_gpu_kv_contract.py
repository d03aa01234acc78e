"""What the header of the key/value cache promises beside the results."""
import math

import pytest
import torch

from test_gpu_kv_cache import Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,d", [(45, 128), (4000, 64)])
def test_padding_rows_may_hold_anything(batq, tokens, d):
    """Rows with a negative slot: NaN and infinities in k, v and q, positions outside the table; the others come out as ever."""
    padding = (0, 7, 8, tokens // 2, tokens - 2, tokens - 1)
    a = Append(batq, tokens, 28, 4, d, 32, rot=d, padding=padding, seed=5)
    x, positions = a.x.cuda(), a.positions.clone()
    for n, i in enumerate(padding):
        x[i] = (math.nan, math.inf, -math.inf)[n % 3]
        positions[i] = (-5, 1 << 30, -(1 << 31), 1 << 20, -1, a.table.shape[0])[n]
    a.run(batq, x=x, positions=positions)
    assert batq.batq_last_device_status() == 0
    a.check()
