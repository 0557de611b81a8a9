"""Rotary positions and cache rows against complex products in 64 bits.

Tolerance of a rotated value y = scale (x1 cos a -+ x2 sin a): half a step of its type, and fp32 arithmetic before it: the reduced angle is rounded
to 2^-27 of a turn (2 pi 2^-27 = 0.4 * 2^-23 rad), sine and cosine to 2 units of 2^-24, each product and the sum to 2^-24: below 2^-21 (|x1| + |x2|) scale."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu
FAR = 2 ** 31 - 1


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def turned(x, pos, freqs, scale, interleaved, inverse, off):
    """(the exact rotation, |x1| + |x2| of every element's pair), in fp64; the phase is reduced in whole numbers."""
    rot = 2 * freqs.numel()
    f = [int(v) % 2 ** 64 for v in freqs.tolist()]
    phase = torch.tensor([[(int(p) * v) % 2 ** 64 / 2 ** 64 for v in f] for p in pos.tolist()], dtype=torch.float64, device=x.device) * (2 * math.pi)
    c, s = (torch.cos(phase) * scale)[:, None], (torch.sin(phase) * (-scale if inverse else scale))[:, None]
    y, mag = x.double(), torch.zeros_like(x, dtype=torch.float64)
    y = y.clone()
    part = x[..., off:off + rot].double()
    if interleaved:
        x1, x2 = part[..., 0::2], part[..., 1::2]
        y[..., off:off + rot] = torch.stack((x1 * c - x2 * s, x1 * s + x2 * c), -1).flatten(-2)
        mag[..., off:off + rot] = (x1.abs() + x2.abs()).repeat_interleave(2, -1)
    else:
        x1, x2 = part.chunk(2, -1)
        y[..., off:off + rot] = torch.cat((x1 * c - x2 * s, x1 * s + x2 * c), -1)
        mag[..., off:off + rot] = (x1.abs() + x2.abs()).repeat(1, 1, 2)
    return y, mag


def near(got, want, mag, scale=1.0):
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + 2.0 ** -21 * scale * mag
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25      # half a step of the subnormal numbers
    err = (got.double() - want).abs()
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,H,D,off,rot", [(1, 1, 64, 0, 64), (1, 128, 576, 512, 64), (19, 5, 192, 128, 64), (33, 7, 128, 0, 96), (257, 24, 80, 0, 80), (5, 3, 70, 3, 38),
                                           (9, 2, 8, 2, 2), (700, 33, 128, 0, 128)])
def test_rope(T, H, D, off, rot, dtype, interleaved, inverse):
    g = gen(T + D)
    x = (torch.randn((T, H, D), device="cuda", generator=g) * 3).to(dtype)
    pos = torch.randint(0, 1 << 20, (T,), device="cuda", generator=g)
    pos[0] = 0
    if T > 4:
        pos[1], pos[2] = FAR, 1
    freqs, scale = B.rope_frequencies(rot, scaling={"type": "yarn", "factor": 4.0, "original_max_position": 4096} if rot > 2 else None)
    keep = x.clone()
    want, mag = turned(x, pos, freqs, scale, interleaved, inverse, off)
    out = B.janus_rope(x, pos, freqs, rot_offset=off, interleaved=interleaved, scale=scale, inverse=inverse)
    near(out, want, mag, scale)
    assert torch.equal(x, keep)
    rest = torch.ones(D, dtype=torch.bool, device="cuda")
    rest[off:off + rot] = False
    assert torch.equal(out[..., rest], x[..., rest])
    again = B.janus_rope(x, pos, freqs, rot_offset=off, interleaved=interleaved, scale=scale, inverse=inverse, out=x)
    assert again is x and torch.equal(x, out)


@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_padding_and_placement(interleaved):
    """Heads before rows, slices of a wider tensor at odd addresses, padding rows of the output left as they were, broadcast inputs."""
    g, freqs = gen(1), B.rope_frequencies(32)[0]
    wide = torch.randn((6, 40, 53), device="cuda", generator=g).bfloat16()
    x = wide[:, :, 3:51].transpose(0, 1)                                          # [40, 6, 48]: rows 53 apart, heads 40 * 53
    pos = torch.randint(0, 9999, (40,), device="cuda", generator=g)
    pos[7] = pos[39] = -1
    base = torch.full((6, 40, 60), 5.0, device="cuda", dtype=torch.bfloat16)
    out = base[:, :, 1:49].transpose(0, 1)
    want, mag = turned(x, pos, freqs, 1.0, interleaved, False, 9)
    B.janus_rope(x, pos, freqs, rot_offset=9, interleaved=interleaved, out=out)
    live = pos >= 0
    near(out[live], want[live], mag[live])
    assert (out[~live] == 5).all() and (base[..., 0] == 5).all() and (base[..., 49:] == 5).all()
    one = torch.randn((1, 1, 48), device="cuda", generator=g).bfloat16().expand(40, 6, 48)
    want, mag = turned(one, pos, freqs, 1.0, interleaved, False, 9)
    got = B.janus_rope(one, pos, freqs, rot_offset=9, interleaved=interleaved, out=torch.empty((40, 6, 48), device="cuda", dtype=torch.bfloat16))
    near(got[live], want[live], mag[live])
    with pytest.raises(B.JanusError, match="INVALID_ARG"):
        B.janus_rope(one, pos, freqs, rot_offset=9, interleaved=interleaved, out=one)      # one place for many rows


def test_gradient_is_the_inverse():
    """<dy, R x> has the gradient R^T dy in x: the call's, the formula's, and differences of the exact rotation."""
    g = gen(2)
    freqs, scale = B.rope_frequencies(64, scaling={"type": "yarn", "factor": 8.0, "original_max_position": 4096})
    x, dy = (torch.randn((11, 3, 64), device="cuda", generator=g) for _ in range(2))
    pos = torch.randint(0, 1 << 20, (11,), device="cuda", generator=g)
    dx = B.janus_rope(dy, pos, freqs, scale=scale, inverse=True)
    leaf = x.double().requires_grad_()
    y, _ = turned(leaf, pos, freqs, scale, False, False, 0)
    (y * dy.double()).sum().backward()
    _, mag = turned(dy, pos, freqs, scale, False, True, 0)
    near(dx, leaf.grad, mag, scale)
    step = torch.randn(x.shape, device="cuda", generator=g, dtype=torch.float64)
    up, down = (turned(x.double() + h * step, pos, freqs, scale, False, False, 0)[0] for h in (1e-4, -1e-4))
    assert abs(float(((up - down) * dy).sum() / 2e-4) - float((dx.double() * step).sum())) < 1e-4      # 11 * 3 * 64 values, each 2^-22 off: 2e-5


def test_infinities_and_nan_stay_in_their_pairs():
    freqs = B.rope_frequencies(8)[0]
    x = torch.ones((2, 1, 16), device="cuda")
    x[0, 0, 1], x[1, 0, 12] = float("inf"), float("nan")
    y = B.janus_rope(x, torch.tensor([3, 5], device="cuda"), freqs)
    bad = ~torch.isfinite(y)
    assert bad[0, 0].nonzero().flatten().tolist() == [1, 5] and bad[1, 0].nonzero().flatten().tolist() == [12]


def test_nothing_to_do():
    freqs = B.rope_frequencies(8)[0]
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert B.janus_rope(torch.zeros((0, 4, 8), device="cuda"), none, freqs).shape == (0, 4, 8)
    assert B.janus_rope(torch.zeros((0, 0, 8), device="cuda"), none, freqs).shape == (0, 0, 8)


# ---- rows into the cache ------------------------------------------------------------------------------------------------
LAYOUTS = {"latent": (128, 1, 576, None), "gqa": (32, 4, 128, 128), "mha": (8, 8, 128, 128), "wide": (6, 2, 192, 64), "short": (3, 3, 8, 16)}


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout,T,page,rot,off", [("latent", 1, 64, 64, 512), ("latent", 300, 16, 64, 512), ("gqa", 12, 64, 128, 0), ("gqa", 777, 48, 20, 6), ("mha", 33, 1, 64, 64),
                                                   ("wide", 65, 128, 64, 128), ("short", 9, 3, 4, 2), ("gqa", 3000, 16, 64, 0)])
def test_append(layout, T, page, rot, off, interleaved):
    hq, n, dqk, dv = LAYOUTS[layout]
    g = gen(T)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()      # noqa: E731
    pages = 2 * (T // page + 1)
    q, k, v = rnd(T, hq, dqk), rnd(T, n, dqk), rnd(T, n, dv) if dv else None
    kp, vp = rnd(pages, page, n, dqk), rnd(pages, page, n, dv) if dv else None
    pos = torch.randint(0, 200000, (T,), device="cuda", generator=g)
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:T].contiguous()
    if T > 8:
        slots[-3:] = -1
        pos[-2:] = -1
        slots[4] = -1
    freqs, scale = B.rope_frequencies(rot)
    k_want, v_want = kp.clone(), None if vp is None else vp.clone()
    turned_k = B.janus_rope(k, pos.clamp(min=0), freqs, rot_offset=off, interleaved=interleaved, scale=scale)
    live = slots >= 0
    k_want.view(-1, n, dqk)[slots[live]] = turned_k[live]
    if dv:
        v_want.view(-1, n, dv)[slots[live]] = v[live]
    q_out = torch.full_like(q, 3.0)
    got = B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, rot_offset=off, interleaved=interleaved, scale=scale, q=q, q_out=q_out)
    assert got is q_out and torch.equal(kp, k_want) and (vp is None or torch.equal(vp, v_want))
    want, mag = turned(q, pos.clamp(min=0), freqs, scale, interleaved, False, off)
    ok = pos >= 0
    near(q_out[ok], want[ok], mag[ok])
    assert (q_out[~ok] == 3).all()
    assert B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, rot_offset=off, interleaved=interleaved, scale=scale) is None
    fresh = B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, rot_offset=off, interleaved=interleaved, scale=scale, q=q)
    assert torch.equal(fresh[ok], q_out[ok])
    assert B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, rot_offset=off, interleaved=interleaved, scale=scale, q=q, q_out=q) is q
    assert torch.equal(q[ok], q_out[ok]) and torch.equal(kp, k_want)
    B.check_dev_status()


def test_append_into_strided_pools():
    """Keys and values of one pool beside each other, heads outermost, rows of a fused projection."""
    g, n, d, page, pages, T = gen(4), 4, 64, 16, 12, 50
    both = torch.randn((n, pages, page, 2 * d), device="cuda", generator=g).bfloat16()
    kp, vp = both[..., :d].permute(1, 2, 0, 3), both[..., d:].permute(1, 2, 0, 3)
    fused = torch.randn((T, 8 + 4 + 4, d), device="cuda", generator=g).bfloat16()
    q, k, v = fused[:, :8], fused[:, 8:12], fused[:, 12:]
    pos, slots = torch.arange(T, device="cuda") + 70000, torch.randperm(pages * page, device="cuda", generator=g)[:T].contiguous()
    freqs, _ = B.rope_frequencies(d)
    want = both.clone()
    flat_k, flat_v = want[..., :d].reshape(n, -1, d), want[..., d:].reshape(n, -1, d)
    flat_k[:, slots] = B.janus_rope(k, pos, freqs).transpose(0, 1)
    flat_v[:, slots] = v.transpose(0, 1)
    want = torch.cat((flat_k.view(n, pages, page, d), flat_v.view(n, pages, page, d)), -1)
    q_want = B.janus_rope(q, pos, freqs)
    B.janus_rope_append(k, v, pos, slots, freqs, kp, vp, q=q, q_out=q)
    assert torch.equal(both, want) and torch.equal(q, q_want)
    B.check_dev_status()


def test_append_reports_places_that_are_not_there():
    g, freqs = gen(5), B.rope_frequencies(8)[0]
    k = torch.randn((4, 2, 8), device="cuda", generator=g).bfloat16()
    pool = torch.zeros((3, 4, 2, 8), device="cuda", dtype=torch.bfloat16)
    for pos, slots in (([0, 1, 2, 3], [0, 12, 5, 1 << 40]), ([0, -1, 2, -1], [0, 3, 5, -1])):
        pool.zero_()
        B.janus_rope_append(k, None, torch.tensor(pos, device="cuda"), torch.tensor(slots, device="cuda"), freqs, pool, None)
        with pytest.raises(B.JanusError, match="INDEX_OUT_OF_RANGE"):
            B.check_dev_status()
        assert pool.view(12, 16).any(-1).nonzero().flatten().tolist() == [0, 5]


def test_far_offsets_in_a_large_pool():
    """A pool of more than 2^32 bytes: the last page is reached, and nothing before it."""
    freqs, page, d = B.rope_frequencies(64)[0], 64, 576
    pages = (5 << 30) // (page * d * 2)
    pool = torch.zeros((pages, page, 1, d), device="cuda", dtype=torch.bfloat16)
    k = torch.ones((2, 1, d), device="cuda", dtype=torch.bfloat16)
    slots = torch.tensor([pages * page - 1, (pages - 1) * page], device="cuda")
    B.janus_rope_append(k, None, torch.zeros(2, dtype=torch.int64, device="cuda"), slots, freqs, pool, None, rot_offset=512)
    assert (pool[-1, -1] == 1).all() and (pool[-1, 0] == 1).all() and float(pool.sum(dtype=torch.float32)) == 2 * d
    B.check_dev_status()
