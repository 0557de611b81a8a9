"""janus_attn_decode_shared on the latent layout: sessions in pieces."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B
from test_gpu_attn_shared import LAYOUTS, call, exact, make
from test_gpu_attn_shared_edges import slot

pytestmark = pytest.mark.gpu


def test_pieces_of_a_latent_session_that_cancel():
    """Two stretches of 256 tokens whose means are 1 + 2^-9 and -1, every probability the same: what is left is 2^-10.  Probabilities of one are exact, sums of 512
    values of one fp32: the output's own rounding and 2^-20 of the means remain."""
    hq, n, dqk, dv, _ = LAYOUTS["latent"]
    c = make(5, "latent", [512], 0, 64)
    c["q"].zero_()
    c["kp"].zero_()
    for s in range(512):
        c["kp"][slot(c, 0, s)] = 1.0 if s < 256 else -1.0
    c["kp"][slot(c, 0, 100)] = 1.5
    out, lse = call(c)
    want = 0.5 / 512
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want + 2.0 ** -20).all(), float(out.float().min())
    assert ((lse.double() - math.log(512)).abs() <= 2.0 ** -16).all()
    B.check_dev_status()


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("prefix,own", [(0, 40), (0, 700), (300, 1000), (700, 0)])
def test_infinite_entries_of_a_row(prefix, own, sign):
    """Values are part of the keys: an infinite one makes its key's logit infinite.  Minus infinity: the key has no weight, and the other dims are those of the other
    keys.  Plus infinity: nothing is a number."""
    total = prefix + own
    c = make(own, "latent", [total, total], prefix, 16)
    c["q"][..., 5] = sign
    sees = [0, 1] if own == 0 else [0]                              # the last token is the first session's, or of the prefix
    keep = torch.arange(total, device="cuda") != total - 1
    want = [exact(c, b, keep if b in sees else None) for b in (0, 1)]
    c["kp"][slot(c, 0, total - 1)][0, 5] = math.inf
    out, lse = call(c)
    for b in (0, 1):
        if b in sees and sign > 0:
            assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
            continue
        o, mag, l = want[b]
        fine = (out[b].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -13) * mag
        if b in sees:
            fine[:, 5] = True
        assert fine.all() and ((lse[b].double() - l).abs() <= 2.0 ** -16 + 2.0 ** -20 * l.abs()).all(), b
    B.check_dev_status()
