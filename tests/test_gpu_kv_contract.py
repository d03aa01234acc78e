"""What the header of the key/value cache promises beside the results."""
import math

import pytest
import torch

from paper_2603_16590_b200 import synth
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


def test_dual_that_fp32_does_not_hold(batq):
    """Factors whose inverses pass fp32: refused as singular, no infinity goes into the queries."""
    t = synth.make_transform(128, 3, "paper")
    for left, right in ((t.left * 1e-39, t.right), (t.left, t.right * 1e-40)):
        small = batq.batq_transform_create(128, left, right)
        with pytest.raises(batq.BatqError) as e:
            batq.batq_transform_create_dual(small)
        assert e.value.status == 6
    assert batq.batq_transform_create_dual(batq.batq_transform_create(128, t.left * 1e-30, t.right * 1e-30)).n == 128
