"""Plans, rotary positions, cache rows and shared-prefix attention: what the C boundary and the binding refuse on the host, and the
frequency table (no GPU needed)."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

from paper_2609_36938_b200 import binding as B
from paper_2609_36938_b200 import build

INVALID, UNSUPPORTED, TOO_SMALL = 1, 2, 3
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


def test_batch_plan_refusals(lib):
    names = ("cached", "new", "tables", "free", "ro", "kv", "to", "pt", "rs", "pos", "slots", "counts", "other")
    at = {n: ctypes.c_void_p(0x10000 * (i + 1)) for i, n in enumerate(names)}      # each in memory of its own

    def call(**kw):
        a = dict({n: at[n] for n in names}, B=4, page=64, ld=16, width=16, n_free=8, n_phys=100, key=None, cap=64, kr=None, rows=8)
        a.update(kw)
        return lib.janus_batch_plan(a["cached"], a["new"], a["B"], a["page"], a["tables"], a["ld"], a["width"], a["free"], a["n_free"], a["n_phys"], a["key"], a["ro"],
                                    a["kv"], a["to"], a["pt"], a["cap"], a["rs"], a["pos"], a["slots"], a["kr"], a["rows"], a["counts"], None, None)

    for bad in (dict(B=-1), dict(page=0), dict(ld=15), dict(width=-1), dict(n_free=-1), dict(cap=-1), dict(rows=-1), dict(n_phys=-1), dict(cached=None),
                dict(new=None), dict(tables=None), dict(free=None), dict(ro=None), dict(kv=None), dict(to=None), dict(pt=None), dict(rs=None), dict(pos=None),
                dict(slots=None), dict(counts=None), dict(key=at["other"]), dict(kr=at["other"]), dict(n_phys=1 << 31), dict(rows=1 << 31)):
        assert call(**bad) == INVALID, bad
    # outputs that share memory with an input, or with one another
    for bad in (dict(kv=at["cached"]), dict(kv=at["new"]), dict(pos=at["slots"]), dict(tables=at["free"]), dict(ro=at["to"]), dict(pt=at["tables"]),
                dict(kv=ctypes.c_void_p(at["cached"].value + 24)), dict(counts=ctypes.c_void_p(at["ro"].value + 32)), dict(key=at["slots"], kr=at["other"]),
                dict(rs=ctypes.c_void_p(at["tables"].value + 4 * 63))):
        assert call(**bad) == INVALID, bad
    assert call(B=8193) == UNSUPPORTED
    assert call(B=8192, width=1 << 18, ld=1 << 18) == UNSUPPORTED      # 2^31 pages


def test_rope_refusals(lib):
    def call(**kw):
        a = dict(x=FAKE, xr=1024, xh=128, T=4, H=8, D=128, pos=FAKE, f=FAKE, off=0, rot=64, il=0, inv=0, dt=0, out=ctypes.c_void_p(0x900000), outr=1024, outh=128)
        a.update(kw)
        return lib.janus_rope(a["x"], a["xr"], a["xh"], a["T"], a["H"], a["D"], a["pos"], a["f"], a["off"], a["rot"], a["il"], 1.0, a["inv"], a["dt"], a["out"],
                              a["outr"], a["outh"], None)

    for bad in (dict(T=-1), dict(H=-1), dict(D=0), dict(rot=0), dict(rot=63), dict(off=-2), dict(off=65), dict(x=None), dict(out=None), dict(pos=None), dict(f=None),
                dict(x=ODD), dict(out=ODD), dict(xr=-8), dict(outh=127), dict(outr=1023), dict(outr=0), dict(outh=0),
                dict(x=FAKE, out=FAKE, outr=2048), dict(x=FAKE, out=FAKE, xh=256)):
        assert call(**bad) == INVALID, bad
    assert call(dt=3) == UNSUPPORTED
    assert call(T=0) == 0 and call(H=0) == 0
    assert call(T=0, x=None, out=None) == 0


def test_rope_append_refusals(lib):
    def call(**kw):
        a = dict(q=None, qr=0, qh=0, H=0, k=FAKE, kr=512, kh=128, n=4, dqk=128, v=FAKE, vr=512, vh=128, dv=128, T=4, pos=FAKE, slots=FAKE, f=FAKE, off=0, rot=64,
                 qo=None, qor=0, qoh=0, kp=FAKE, kps=32768, kts=512, khs=128, vp=ctypes.c_void_p(0x900000), vps=32768, vts=512, vhs=128, page=64, phys=16)
        a.update(kw)
        return lib.janus_rope_append(a["q"], a["qr"], a["qh"], a["H"], a["k"], a["kr"], a["kh"], a["n"], a["dqk"], a["v"], a["vr"], a["vh"], a["dv"], a["T"], a["pos"],
                                     a["slots"], a["f"], a["off"], a["rot"], 0, 1.0, a["qo"], a["qor"], a["qoh"], a["kp"], a["kps"], a["kts"], a["khs"], a["vp"],
                                     a["vps"], a["vts"], a["vhs"], a["page"], a["phys"], None, None)

    q = dict(q=FAKE, qr=1024, qh=128, H=8, qo=FAKE, qor=1024, qoh=128)
    for bad in (dict(T=-1), dict(n=0), dict(dqk=0), dict(page=0), dict(phys=-1), dict(rot=65), dict(off=72), dict(k=None), dict(kp=None), dict(pos=None), dict(slots=None),
                dict(f=None), dict(v=None), dict(vp=None), dict(vp=FAKE), dict(kts=504), dict(khs=64), dict(k=ODD), dict(kps=32769), dict(kr=513), dict(kr=-512),
                dict(q, qo=None), dict(q, q=None), dict(q, H=0), dict(q, qor=2048), dict(q, qo=ctypes.c_void_p(0x900000), qoh=64), dict(q, qr=1028, qor=1028)):
        assert call(**bad) == INVALID, bad
    assert call(dqk=100, kr=400, kh=100) == UNSUPPORTED
    assert call(dv=100) == UNSUPPORTED
    assert call(T=0) == 0


def test_attn_decode_shared_refusals(lib):
    need = lib.janus_attn_decode_shared_workspace_size(4, 32, 128, 4, 128, 64, 1000, 3000)
    assert need > 0

    def call(**kw):
        a = dict(q=FAKE, B=4, H=32, dqk=128, kp=FAKE, kps=32768, kts=512, khs=128, vp=ctypes.c_void_p(0x900000), vps=32768, vts=512, vhs=128, n=4, dv=128, page=64,
                 phys=100, pt=FAKE, P=1000, tables=FAKE, off=FAKE, lens=FAKE, most=3000, scale=0.1, out=FAKE, ws=FAKE, bytes=need)
        a.update(kw)
        return lib.janus_attn_decode_shared(a["q"], a["B"], a["H"], a["dqk"], a["kp"], a["kps"], a["kts"], a["khs"], a["vp"], a["vps"], a["vts"], a["vhs"], a["n"],
                                            a["dv"], a["page"], a["phys"], a["pt"], a["P"], a["tables"], a["off"], a["lens"], a["most"], a["scale"], a["out"], None,
                                            a["ws"], a["bytes"], None, None)

    for bad in (dict(B=-1), dict(H=0), dict(H=30), dict(dqk=0), dict(n=0), dict(page=0), dict(P=-1), dict(most=999), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=math.nan), dict(scale=math.inf), dict(q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(lens=None), dict(pt=None), dict(tables=None),
                dict(off=None), dict(q=ODD), dict(kp=ODD), dict(out=ODD), dict(ws=ODD), dict(kps=32769), dict(vts=513), dict(vp=FAKE, dv=136), dict(vp=FAKE, vps=65536), dict(phys=0), dict(kts=0), dict(vhs=-128), dict(kps=-32768)):
        assert call(**bad) == INVALID, bad
    assert call(dqk=132) == UNSUPPORTED and call(dqk=640) == UNSUPPORTED and call(dv=520) == UNSUPPORTED
    assert call(most=(1 << 31) - 100) == UNSUPPORTED and call(B=65536, bytes=1 << 60) == UNSUPPORTED
    assert call(bytes=need - 1) == TOO_SMALL
    assert call(B=0) == 0


def test_workspace_of_nothing_is_nothing(lib):
    assert lib.janus_attn_decode_shared_workspace_size(0, 32, 128, 4, 128, 64, 1000, 3000) == 0
    assert lib.janus_attn_decode_shared_workspace_size(4, 32, 128, 4, 128, 64, 1000, 999) == 0
    # latent sessions that are all empty go by the general route, which keeps an offset for each
    assert lib.janus_attn_decode_shared_workspace_size(1000, 128, 576, 1, 512, 64, 0, 0) >= 8 * 1001


def test_binding_refuses(lib):
    x, pos = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int64)
    f, _ = B.rope_frequencies(64, device="cpu")
    with pytest.raises(B.JanusError, match="bfloat16, float16 or float32"):
        B.janus_rope(x.double(), pos, f)
    with pytest.raises(B.JanusError, match="adjacent"):
        B.janus_rope(x.transpose(1, 2), pos, f)
    with pytest.raises(B.JanusError, match="shape and type"):
        B.janus_rope(x, pos, f, out=torch.zeros(2, 4, 32))
    with pytest.raises(B.JanusError, match="positions"):
        B.janus_rope(x, pos.int(), f)
    with pytest.raises(ValueError, match="dimensions"):
        B.janus_rope(x[0], pos, f)
    with pytest.raises(B.JanusError, match="CUDA tensor"):
        B.janus_rope(x, pos, f)
    k, pool = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 8, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(B.JanusError, match="go together"):
        B.janus_rope_append(k, None, pos, pos, f, pool, pool)
    with pytest.raises(B.JanusError, match="heads and dims"):
        B.janus_rope_append(k, None, pos, pos, f, pool[..., :32], None)
    with pytest.raises(B.JanusError, match="goes with q"):
        B.janus_rope_append(k, None, pos, pos, f, pool, None, q_out=k)
    with pytest.raises(B.JanusError, match="must be bfloat16"):
        B.janus_rope_append(k.float(), None, pos, pos, f, pool, None)
    lens, table = torch.zeros(2, dtype=torch.int64), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(B.JanusError, match="number of sessions"):
        B.janus_batch_plan(lens, lens[:1], table, table[0], page_size=8, n_phys_pages=4, max_rows=2, out={})
    with pytest.raises(KeyError):
        B.janus_batch_plan(lens, lens, table, table[0], page_size=8, n_phys_pages=4, max_rows=2, out={})
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    args = dict(prefix_table=table[0], prefix_len=8, page_tables=table[0], table_offsets=torch.zeros(3, dtype=torch.int64), kv_lens=lens, max_len=24, page_size=8,
                softmax_scale=1.0, d_v=64)
    with pytest.raises(B.JanusError, match="page_size"):
        B.janus_attn_decode_shared(q, pool, pool, **dict(args, page_size=16))
    with pytest.raises(B.JanusError, match="cover prefix_len"):
        B.janus_attn_decode_shared(q, pool, pool, **dict(args, prefix_len=25, max_len=30))
    with pytest.raises(B.JanusError, match="shorter than the heads"):
        B.janus_attn_decode_shared(q, pool, pool, **dict(args, d_v=72))
    with pytest.raises(B.JanusError, match="contiguous"):
        B.janus_attn_decode_shared(q.transpose(0, 1).contiguous().transpose(0, 1), pool, pool, **args)
    with pytest.raises(TypeError):
        B.janus_attn_decode_shared(q, pool, pool, **dict(args, max_len=24.0))


@pytest.mark.parametrize("scaling", [None, {"type": "linear", "factor": 8.0}, {"type": "ntk", "factor": 4.0},
                                     {"type": "yarn", "factor": 8.0, "original_max_position": 4096},
                                     {"type": "wavelength", "factor": 8.0, "low_freq_factor": 1.0, "high_freq_factor": 4.0, "original_max_position": 8192}])
@pytest.mark.parametrize("rot", [2, 64, 96, 128])
def test_frequency_table(rot, scaling):
    """Every entry is the pair's turns per position to 2^-50 of itself (fp64 arithmetic), and what stretches long wavelengths leaves the shortest."""
    f, scale = B.rope_frequencies(rot, scaling=scaling, device="cpu")
    assert f.dtype == torch.int64 and f.shape == (rot // 2,)
    got = [Fraction(int(x) % 2 ** 64, 2 ** 64) for x in f]
    plain = [10000.0 ** (-2 * i / rot) / (2 * math.pi) for i in range(rot // 2)]
    kind = scaling and scaling["type"]
    if kind is None or kind == "linear":
        want = [p / (scaling["factor"] if kind else 1.0) for p in plain]
        assert all(abs(float(g) - w) <= 2.0 ** -50 * w + 2.0 ** -64 for g, w in zip(got, want))
    else:
        want_end = plain[-1] / scaling["factor"]
        assert abs(float(got[0]) - plain[0]) <= 2.0 ** -50 * plain[0] or rot == 2
        if rot >= 64:
            assert abs(float(got[-1]) - want_end) <= 2.0 ** -45 * want_end
            assert all(a >= b for a, b in zip(got, got[1:]))
            assert all(p / scaling["factor"] * (1 - 1e-9) <= float(g) <= p * (1 + 1e-9) for g, p in zip(got, plain))
    assert scale == (pytest.approx(0.1 * math.log(8.0) + 1.0) if kind == "yarn" else 1.0)


def test_frequency_table_refuses():
    for bad in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=64, base=0.0), dict(rot_dim=64, scaling={"type": "other"}), dict(rot_dim=64, scaling={"type": "linear"}),
                dict(rot_dim=64, scaling={"type": "linear", "factor": 0.5}), dict(rot_dim=64, scaling={"type": "yarn", "factor": 2.0}),
                dict(rot_dim=64, scaling={"type": "linear", "factor": 2.0, "more": 1})):
        with pytest.raises(ValueError):
            B.rope_frequencies(device="cpu", **bad)
