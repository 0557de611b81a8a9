"""janus_attn_decode_shared where its tiles, copies and fragments end.  Tolerances and the reference as in test_gpu_attn_shared."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B
from test_gpu_attn_shared import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["gqa", "gqa64", "mha192", "mqa", "mqa200"])
@pytest.mark.parametrize("prefix,own", [(0, 128 * 2 + 5), (0, 128 * 6 + 127), (128 * 4 + 1, 0), (131, 128 * 7 + 64), (1, 64 * 9 + 1)])
def test_the_last_tile_behind_whole_ones(layout, prefix, own):
    """Rows of V are cleared in a tile behind whole ones, again and again: the same bits every time, and no token that a session does not see."""
    c = make(own, layout, [prefix + own, prefix + own // 2, prefix + own - 1][: 3 if own > 1 else 1], prefix, 16, junk=math.nan)
    out, lse = call(c)
    check(c, out, lse)
    for _ in range(20):
        again, lse2 = call(c)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    B.check_dev_status()
