"""Rotary positions: what the angle itself may be off by."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_small_angles(interleaved):
    """x = (1, 0) turned by a phase of less than 2^-20 turns gives its sine: the phase is rounded to a multiple of 2^-32 turns, half a step or 2^-33 turns; angle, sine
    and product in fp32 2^-21 of it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    freqs = torch.randint(0, 1 << 44, (64,), device="cuda", generator=g)
    freqs[0], freqs[1], freqs[2] = (1 << 32) - 1, (1 << 31) + 1, (1 << 31) - 1
    x = torch.zeros((1, 1, 128), device="cuda")
    first, second = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, 64), slice(64, None))
    x[..., first] = 1.0
    for pos in (1, 3):
        y = B.janus_rope(x, torch.tensor([pos], device="cuda"), freqs, interleaved=interleaved)
        want = torch.sin(freqs.double() * pos * 2.0 ** -64 * 2 * math.pi)
        err = (y[0, 0, second].double() - want).abs()
        assert (err <= 2 * math.pi * 2.0 ** -33 + 2.0 ** -21 * want).all(), float(err.max())
        assert ((y[0, 0, first].double() - 1.0).abs() <= 2.0 ** -21).all()


def test_append_into_pages_of_keys_and_then_values():
    """One tensor whose pages hold the keys of their tokens and behind them the values, of another width; rows of a fused projection, the queries turned in place."""
    g, n, dk, dv, page, pages, T = torch.Generator(device="cuda").manual_seed(2), 4, 192, 128, 16, 12, 50
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()      # noqa: E731
    arena = rnd(pages, page * n * (dk + dv))
    kp, vp = arena[:, :page * n * dk].view(pages, page, n, dk), arena[:, page * n * dk:].view(pages, page, n, dv)
    fused, v = rnd(T, 8 + n, dk), rnd(T, n, dv)
    q, k = fused[:, :8], fused[:, 8:]
    pos, slots = torch.arange(T, device="cuda") + 70000, torch.randperm(pages * page, device="cuda", generator=g)[:T].contiguous()
    freqs, _ = B.rope_frequencies(64)
    want_k, want_v, want_q = kp.clone(), vp.clone(), B.janus_rope(q, pos, freqs, rot_offset=128)
    want_k.view(-1, n, dk)[slots] = B.janus_rope(k, pos, freqs, rot_offset=128)
    want_v.view(-1, n, dv)[slots] = v
    assert B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, rot_offset=128, q=q, q_out=q) is q
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v) and torch.equal(q, want_q)
    # an output among the other heads of the same tensor
    wide = rnd(T, 16, dk)
    x, out = wide[:, 0::2], wide[:, 1::2]
    want = B.janus_rope(x, pos, freqs)
    B.janus_rope(x, pos, freqs, out=out)
    assert torch.equal(out, want)
    for bad in (wide[:, 1:9], wide[:, 4:12]):
        with pytest.raises(B.JanusError, match="INVALID_ARG"):
            B.janus_rope(wide[:, 0:8], pos, freqs, out=bad)
    B.check_dev_status()
