"""janus_attn_decode_shared where its tiles, copies and fragments end.  Tolerances and the reference as in test_gpu_attn_shared."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B
from test_gpu_attn_shared import call, check, exact, make

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


def slot(c, b, s):
    """Page and place of token s of session b."""
    page = c["page"]
    return (int(c["perm"][s // page]) if s < c["prefix"] else int(c["np_tables"][b][s // page])), s % page


def check_values(c, out, lse):
    """As check(), and what is no number is the definition's: an infinity of its sign, or NaN."""
    for b in range(len(c["np_lens"])):
        if c["np_lens"][b] == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all(), b
            continue
        want, _, want_lse = exact(c, b)
        got = out[b].double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), b
        for sign in (math.inf, -math.inf):
            assert torch.equal(got == sign, want == sign), (b, sign)
        fine = torch.isfinite(want)
        mag = finite_magnitude(c, b)
        err = torch.where(fine, (got - want).abs(), 0.0)
        assert (err <= torch.where(fine, 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -13) * mag, 1.0)).all(), b
        assert ((lse[b].double() - want_lse).abs() <= 2.0 ** -16 + 2.0 ** -20 * want_lse.abs()).all()


def finite_magnitude(c, b):
    vp = c["vp"]
    try:
        c["vp"] = torch.where(torch.isfinite(vp), vp, torch.zeros_like(vp))
        return exact(c, b)[1]
    finally:
        c["vp"] = vp


@pytest.mark.parametrize("layout", ["gqa", "mha", "gqa64", "mha192", "mqa", "mqa200", "seven"])
@pytest.mark.parametrize("prefix,own", [(0, 1), (0, 20), (0, 60), (0, 97), (0, 100), (0, 129), (0, 300), (5, 40), (200, 3), (300, 0), (700, 30)])
def test_infinite_values_among_few_and_many(layout, prefix, own):
    """Lanes that share a row's keys, tiles with few keys, several fragments: an infinite value comes out as such, opposite ones and NaN as NaN."""
    lens = [prefix + own] * 2 + [prefix + own // 2]
    c = make(prefix + own, layout, lens, prefix, 16)
    n, dv = c["vp"].shape[2], min(c["vp"].shape[3], 64)
    for dim, places in enumerate([[(0, math.inf)], [(0.5, -math.inf)], [(1, math.inf)], [(0, math.inf), (1, math.inf)], [(0, math.inf), (1, -math.inf)], [(0.3, math.nan)],
                                  [(0.3, math.nan), (0.9, math.inf)], [(0.7, -math.inf)]]):
        for at, value in places:
            page, within = slot(c, 0, min(int(at * lens[0]), lens[0] - 1))
            c["vp"][page, within, dim % n, dim * 7 % dv] = value
    out, lse = call(c)
    check_values(c, out, lse)
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "mha192", "mqa200"])
@pytest.mark.parametrize("own", [50, 700])
def test_infinite_values_of_little_weight(layout, own):
    """Logits hundreds apart: the weight of most keys is 0 in fp32, by the definition it is positive."""
    c = make(own, layout, [own, own // 2 + 30], 30, 64)
    page, within = slot(c, 0, 10)
    c["kp"].mul_(24.0)
    c["vp"][page, within, 0, 3], c["vp"][slot(c, 0, own - 1)][0, 9] = math.inf, -math.inf
    out, _ = call(c)
    for b in range(2):
        want, _, _ = exact(c, b)
        bad = ~torch.isfinite(want)
        assert torch.equal(out[b].double()[bad], want[bad]) and torch.isfinite(out[b][~bad]).all()
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "mha", "mha192"])
def test_huge_values_without_weight(layout):
    """A key 100 and more below the others in its logit, with values of 3e38: nothing of them is in the sum."""
    c = make(3, layout, [40, 90], 0, 64)
    c["q"].abs_()
    for b in range(2):
        page, within = slot(c, b, 7)
        c["kp"][page, within], c["vp"][page, within] = -30.0, 3e38
    out, lse = call(c)
    check(c, out, lse)
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "mha192", "mqa200"])
def test_a_row_without_a_logit_and_infinite_values(layout):
    """Every logit is minus infinity: zeros, whatever the values are."""
    c = make(4, layout, [33, 150], 0, 64)
    c["q"].fill_(1.0)
    c["kp"][..., 0] = -math.inf
    c["vp"][slot(c, 0, 3)][..., 5], c["vp"][slot(c, 1, 140)][..., 6] = math.inf, math.nan
    out, lse = call(c)
    assert (out == 0).all() and (lse == -math.inf).all()
    B.check_dev_status()


@pytest.mark.parametrize("layout,nb", [("gqa", 40), ("gqa64", 50), ("mqa200", 5), ("mha", 300), ("mha192", 140)])
@pytest.mark.parametrize("factor", [1.0, 24.0])
def test_infinite_values_that_all_sessions_see(layout, nb, factor):
    """Segments of up to 256 rows, of fewer rows and of one session: infinities, a NaN and opposite infinities among the shared tokens and a session's own."""
    prefix = 700
    lens = [prefix + 5 * (b % 9) for b in range(nb)]
    c = make(nb, layout, lens, prefix, 64)
    c["kp"].mul_(factor)
    for h, dim, s, value in ((0, 3, 0, math.inf), (0, 9, 699, -math.inf), (0, 20, 100, math.nan), (0, 33, 5, math.inf), (0, 33, 600, -math.inf), (0, 40, 300, math.inf),
                             (0, 40, 301, math.inf)):
        page, within = slot(c, 0, s)
        c["vp"][page, within, h, dim] = value
    page, within = slot(c, 8 if nb > 8 else 4, prefix + 3)
    c["vp"][page, within, 0, 50] = -math.inf
    out, lse = call(c)
    for b in sorted({0, 1, 4, 8, nb // 2, nb - 1} & set(range(nb))):
        want, _, _ = exact(c, b)
        bad = ~torch.isfinite(want)
        assert torch.equal(torch.isnan(out[b].double()), torch.isnan(want)) and torch.isfinite(out[b][~bad]).all(), b
        there = bad & ~torch.isnan(want)
        assert torch.equal(out[b].double()[there], want[there]), b
    B.check_dev_status()
