"""janus_attn_decode_shared on the latent layout: sessions in pieces."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B
from test_gpu_attn_shared import LAYOUTS, call, check, exact, make
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


@pytest.mark.parametrize("page", [1, 7, 48, 192, 512])
@pytest.mark.parametrize("prefix,own", [(515, 900), (0, 1025), (1024, 1), (255, 258)])
def test_tables_of_pieces(prefix, own, page):
    """A piece's table holds the pages of its own tokens, the page that the prefix ends in twice where own tokens follow in it."""
    c = make(page, "latent", [prefix + own, prefix, prefix + own // 2], prefix, page)
    out, lse = call(c)
    check(c, out, lse)
    B.check_dev_status()


def test_more_pieces_than_are_made_at_once():
    """300 sessions bounded by 131072 tokens: 256 of them at a time, with tables, lengths and outputs of their own."""
    rng = torch.Generator().manual_seed(6)
    lens = [70 + int(x) for x in torch.randint(0, 600, (300,), generator=rng)]
    lens[3] = lens[299] = 0
    c = make(6, "latent", lens, 70, 64)
    need = B.attn_decode_shared_workspace_size(300, 128, 576, 1, 512, 64, 70, 131072)
    assert need < 3 << 30
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = call(c, max_len=131072, workspace=ws)
    check(c, out, lse, sessions=[0, 1, 3, 100, 254, 255, 256, 257, 298, 299])
    tight, lse2 = call(c)
    assert (tight.float() - out.float()).abs().max() <= 2.0 ** -6 * out.float().abs().max() and torch.allclose(lse[lse > -1e30], lse2[lse > -1e30], atol=2.0 ** -14)
    B.check_dev_status()


def test_values_of_their_own_take_the_general_route():
    """The latent shape with values that are no part of the keys: the other kernel, in the workspace that the same size function gives."""
    c = make(7, "latent", [300, 260, 0, 70], 70, 16)
    c["vp"] = c["kp"][..., :512].clone()
    need = B.attn_decode_shared_workspace_size(4, 128, 576, 1, 512, 16, 70, 300)
    buf = torch.full((need + 65536,), 7, dtype=torch.uint8, device="cuda")
    out, lse = call(c, workspace=buf[:need])
    check(c, out, lse)
    assert (buf[need:] == 7).all()
    B.check_dev_status()
