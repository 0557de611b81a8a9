"""janus_attn_decode_shared against softmax in 64 bits, session by session.

Tolerance.  With A = sum of softmax * |v|: the probabilities are rounded to bf16 (2^-8 of each) and so is the output (2^-8 of it); logits in fp32 are off by at
most d 2^-22 of sum |q||k| (sum of d products), which for the inputs here stays below 2^-13 of A.  lse: the logits' error and 2^-20 of the arithmetic."""
import math

import numpy as np
import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu
LAYOUTS = {"latent": (128, 1, 576, 512, True), "mha": (8, 8, 128, 128, False), "gqa": (32, 4, 128, 128, False), "gqa64": (24, 4, 64, 64, False), "mha192": (4, 4, 192, 128, False),
           "mqa": (40, 1, 128, 64, False), "mqa200": (200, 1, 64, 128, False), "odd": (6, 2, 96, 32, False), "seven": (14, 2, 128, 128, False), "alias": (8, 2, 128, 64, True)}


def make(seed, layout, lens, prefix, page, spread=1.0, junk=None):
    """Pools, tables and lengths; `junk` fills every token that no session may see."""
    hq, n, dqk, dv, alias = LAYOUTS[layout]
    g, rng, nb = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed), len(lens)
    pages_b = [-(-int(t) // page) for t in lens]
    own = [max(p - prefix // page, 0) for p in pages_b]
    n_prefix = -(-prefix // page)
    n_phys = n_prefix + sum(own) + 2
    perm = rng.permutation(n_phys).astype(np.int32)
    tables, at = [], n_prefix
    for b in range(nb):
        shared = min(prefix // page, pages_b[b])
        tables.append(np.concatenate([perm[:shared], perm[at:at + own[b]]]))
        at += own[b]
    rnd = lambda d: (torch.randn((n_phys, page, n, d), device="cuda", generator=g) * spread).bfloat16()      # noqa: E731
    kp = rnd(dqk)
    vp = kp if alias else rnd(dv)
    if junk is not None:
        seen = torch.zeros((n_phys * page,), dtype=torch.bool, device="cuda")
        for b in range(nb):
            seen[torch.from_numpy(slots_of(perm, tables[b], prefix, int(lens[b]), page)).cuda()] = True
        kp.view(n_phys * page, -1)[~seen] = junk
        vp.view(n_phys * page, -1)[~seen] = junk
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()      # noqa: E731
    return {"q": torch.randn((nb, hq, dqk), device="cuda", generator=g).bfloat16(), "kp": kp, "vp": vp, "prefix_table": dev(perm[:n_prefix], torch.int32),
            "tables": dev(np.concatenate(tables) if nb else [], torch.int32), "offsets": dev(np.concatenate([[0], np.cumsum([len(t) for t in tables])]), torch.int64),
            "lens": dev(lens, torch.int64), "prefix": prefix, "page": page, "np_tables": tables, "perm": perm, "np_lens": [int(t) for t in lens], "layout": layout,
            "max_len": max([prefix] + [int(t) for t in lens])}


def slots_of(perm, table, prefix, length, page):
    s = np.arange(length)
    if length == 0:
        return s
    shared, mine = s[s < prefix], s[s >= prefix]
    return np.concatenate([perm[shared // page].astype(np.int64) * page + shared % page, table[mine // page].astype(np.int64) * page + mine % page])


def call(c, **kw):
    hq, n, dqk, dv, alias = LAYOUTS[c["layout"]]
    a = dict(prefix_table=c["prefix_table"], prefix_len=c["prefix"], page_tables=c["tables"], table_offsets=c["offsets"], kv_lens=c["lens"], max_len=c["max_len"],
             page_size=c["page"], softmax_scale=1 / math.sqrt(dqk), d_v=dv)
    a.update(kw)
    return B.janus_attn_decode_shared(c.get("q_view", c["q"]), c["kp"], c["vp"], **a)


def exact(c, b, keep=None):
    """(out, A, lse) of session b in fp64; keep: which tokens count (all)."""
    hq, n, dqk, dv, alias = LAYOUTS[c["layout"]]
    slots = torch.from_numpy(slots_of(c["perm"], c["np_tables"][b], c["prefix"], c["np_lens"][b], c["page"])).cuda()
    if keep is not None:
        slots = slots[keep]
    pages, within = slots // c["page"], slots % c["page"]
    out, mag, lse = (torch.zeros((hq, x), dtype=torch.float64, device="cuda") for x in (dv, dv, 1))
    for h in range(n):
        k, v = c["kp"][pages, within, h].double(), c["vp"][pages, within, h, :dv].double()
        rows = slice(h * hq // n, (h + 1) * hq // n)
        logits = c["q"][b, rows].double() @ k.t() / math.sqrt(dqk)
        p = torch.softmax(logits, -1)
        out[rows], mag[rows], lse[rows] = p @ v, p @ v.abs(), torch.logsumexp(logits, -1, keepdim=True)
    return out, mag, lse[:, 0]


def check(c, out, lse, sessions=None, keep=None):
    for b in range(len(c["np_lens"])) if sessions is None else sessions:
        if c["np_lens"][b] == 0:
            assert (out[b] == 0).all() and (lse is None or (lse[b] == -math.inf).all()), b
            continue
        want, mag, want_lse = exact(c, b, None if keep is None else keep.get(b))
        err, tol = (out[b].double() - want).abs(), 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -13) * mag
        assert (err <= tol).all(), (b, float((err / tol).max()))
        if lse is not None:
            assert ((lse[b].double() - want_lse).abs() <= 2.0 ** -16 + 2.0 ** -20 * want_lse.abs()).all(), (b, float((lse[b].double() - want_lse).abs().max()))


def lengths(n, prefix, own, seed=0):
    rng = np.random.default_rng(seed)
    out = prefix + np.exp(rng.uniform(0, math.log(own + 1), n)).astype(np.int64) - 1
    out[0] = prefix + own
    if n > 3:
        out[1], out[2] = prefix, 0
    return out


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("n,prefix,own,page", [(1, 0, 1, 64), (1, 1, 0, 64), (1, 64, 64, 64), (2, 127, 130, 64), (3, 129, 1, 16), (5, 1000, 300, 48), (9, 640, 777, 128),
                                               (17, 2111, 65, 16), (40, 515, 260, 64), (7, 100, 40, 1), (6, 77, 90, 7), (5, 300, 500, 192)])
def test_against_64_bits(layout, n, prefix, own, page):
    lens = np.maximum(lengths(n, prefix, own, seed=page), 0)
    c = make(n + page, layout, lens, prefix, page)
    out, lse = call(c)
    check(c, out, lse)
    B.check_dev_status()


@pytest.mark.parametrize("layout,n,prefix,own", [("gqa", 64, 8000, 500), ("gqa", 3, 30000, 9000), ("mha", 300, 700, 100), ("gqa64", 100, 3001, 130), ("mqa200", 20, 2000, 300),
                                                 ("latent", 20, 3000, 400), ("mha192", 130, 600, 200)])
def test_larger(layout, n, prefix, own):
    c = make(n, layout, lengths(n, prefix, own), prefix, 64)
    out, lse = call(c)
    check(c, out, lse, sessions=sorted({0, 1, 2, n // 2, n - 1}))
    B.check_dev_status()


def test_more_sessions_than_a_launch_takes():
    """1100 sessions: two launches, each with its own part of the tables, lengths and outputs."""
    c = make(31, "seven", lengths(1100, 130, 70), 130, 16)
    out, lse = call(c)
    check(c, out, lse, sessions=[0, 1, 2, 500, 1022, 1023, 1024, 1025, 1099])
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "latent", "odd"])
def test_a_batch_that_stands_empty(layout):
    """No session has a token and none can have one: zeros and -inf, and nothing is written behind the workspace."""
    hq, n, dqk, dv, _ = LAYOUTS[layout]
    c = make(8, layout, np.full(700, 3), 0, 16)
    c["lens"].zero_()
    need = B.attn_decode_shared_workspace_size(700, hq, dqk, n, dv, 16, 0, 0)
    buf = torch.full((need + 65536,), 7, dtype=torch.uint8, device="cuda")
    out, lse = call(c, max_len=0, workspace=buf[:need], want_lse=True)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all() and (buf[need:] == 7).all()


def test_lengths_far_below_their_bound():
    """max_len is a bound only: a bound of 2^20 tokens over short sessions changes no bit of a row's sums beyond their order."""
    for layout in ("gqa", "latent"):
        c = make(32, layout, [300, 77, 0, 150], 70, 16)
        out, lse = call(c, max_len=1 << 20)
        check(c, out, lse)
    B.check_dev_status()


def test_a_call_on_another_stream_while_one_runs():
    """Two calls with workspaces of their own, on two streams at once."""
    cs = [make(33 + i, layout, lengths(24, 900, 700, seed=i), 900, 64) for i, layout in enumerate(("gqa", "mha"))]
    want = [call(c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cs, streams)):
            with torch.cuda.stream(s):
                got[i].append(call(c))
    torch.cuda.synchronize()
    for g, (o, l) in zip(got, want):
        assert all(torch.equal(x, o) and torch.equal(y, l) for x, y in g)
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "latent", "mha192", "odd"])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf, 3e38])
@pytest.mark.parametrize("prefix,own,page", [(100, 77, 64), (0, 5, 16), (130, 0, 64), (64, 1, 64)])
def test_what_no_session_sees_does_not_count(layout, junk, prefix, own, page):
    """Tokens behind the prefix in its last page, behind a session's last token, before its first own token: NaN and infinities there change nothing."""
    lens = [prefix + own, prefix + own // 2, prefix + own, 0][: 4 if prefix + own // 2 > 0 else 1]
    c = make(5, layout, lens, prefix, page, junk=junk)
    out, lse = call(c)
    check(c, out, lse)
    B.check_dev_status()


@pytest.mark.parametrize("layout", ["gqa", "mha", "latent"])
def test_large_logits(layout):
    """Logits of some hundred: the running maximum moves, far values vanish; the sums stay exact."""
    c = make(11, layout, [900, 1500, 800], 700, 64, spread=8.0)
    out, lse = call(c)
    for b in range(3):
        want, mag, want_lse = exact(c, b)
        # logits up to 600, each off by up to 2^-16 of themselves in fp32 (products of 7 bits summed): 2^-6 of a probability at most
        assert ((out[b].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -6) * mag).all()
        assert ((lse[b].double() - want_lse).abs() <= 2.0 ** -16 * want_lse.abs() + 2.0 ** -16).all()
    B.check_dev_status()


def test_values_that_are_not_numbers_come_through():
    for layout in ("gqa", "latent"):
        c = make(12, layout, [300, 260, 290], 200, 64)
        slot = slots_of(c["perm"], c["np_tables"][1], 200, 260, 64)[230]
        c["kp"].view(-1, *c["kp"].shape[2:])[int(slot)] = math.nan       # a key of session 1 alone
        out, lse = call(c)
        check(c, out, lse, sessions=[0, 2])
        assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    c = make(13, "gqa", [300, 260], 200, 64)
    c["vp"].view(-1, 4, 128)[int(slots_of(c["perm"], c["np_tables"][0], 200, 300, 64)[5]), 1, 7] = math.inf      # a value that all sessions see
    out, lse = call(c)
    bad = ~torch.isfinite(out)
    assert bad[:, 8:16, 7].all() and int(bad.sum()) == 2 * 8 and (out[:, 8:16, 7] == math.inf).all()


@pytest.mark.parametrize("layout", ["gqa", "latent", "odd"])
def test_bad_pages_and_lengths_are_reported_and_skipped(layout):
    prefix, page = 200, 16
    c = make(14, layout, [300, 260, 290, 250], prefix, page)

    def reported():
        with pytest.raises(B.JanusError, match="INDEX_OUT_OF_RANGE"):
            B.check_dev_status()

    table, offs = c["tables"].clone(), c["offsets"].tolist()
    gone = {0: 208 // page, 2: 272 // page}
    c["tables"][offs[0] + gone[0]] = -1
    c["tables"][offs[2] + gone[2]] = c["kp"].shape[0]
    out, lse = call(c)
    reported()
    keep = {b: torch.tensor([s // page != j for s in range(c["np_lens"][b])], device="cuda") for b, j in gone.items()}
    check(c, out, lse, keep=keep)
    c["tables"].copy_(table)
    prefix_table = c["prefix_table"].clone()
    c["prefix_table"][3] = 1 << 30
    out, lse = call(c)
    reported()
    check(c, out, lse, keep={b: torch.tensor([s // page != 3 or s >= prefix for s in range(c["np_lens"][b])], device="cuda") for b in range(4)})
    c["prefix_table"].copy_(prefix_table)
    # a length below the prefix empties its entry, a negative one too, one above max_len is cut
    lens = c["lens"].clone()
    c["lens"][1], c["lens"][3] = 150, -4
    out, lse = call(c, max_len=280)
    reported()
    c["np_lens"] = [280, 0, 280, 0]
    check(c, out, lse)
    # a table shorter than its session: what it does not cover is skipped
    c["lens"].copy_(lens)
    c["np_lens"] = lens.tolist()
    c["offsets"][4] = c["offsets"][3] + 15
    out, lse = call(c)
    reported()
    check(c, out, lse, keep={3: torch.arange(250, device="cuda") < 240})


def test_shapes_of_the_pools():
    """Keys and values in one tensor, heads outermost, tokens of a page apart; a batch with nothing in it."""
    hq, n, dqk, dv, _ = LAYOUTS["gqa"]
    c = make(15, "gqa", [300, 333], 256, 64)
    both = torch.zeros((n, c["kp"].shape[0], 64, dqk + dv), device="cuda", dtype=torch.bfloat16)
    both[..., :dqk], both[..., dqk:] = c["kp"].permute(2, 0, 1, 3), c["vp"].permute(2, 0, 1, 3)
    out, lse = call(c)
    c["kp"], c["vp"] = both[..., :dqk].permute(1, 2, 0, 3), both[..., dqk:].permute(1, 2, 0, 3)
    again, lse2 = call(c)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    check(c, again, lse2)
    none = make(16, "gqa", [], 256, 64)
    out, lse = call(none)
    assert out.shape == (0, 32, 128)
    c = make(17, "gqa", [0, 0], 0, 64)
    out, lse = call(c, max_len=0, prefix_table=None, page_tables=None, table_offsets=None)
    check(c, out, lse)
    c = make(18, "gqa", [128, 0, 128], 128, 64)
    out, lse = call(c, page_tables=None, table_offsets=None, want_lse=False)
    assert lse is None
    check(c, out, None)
    B.check_dev_status()


def test_streams_graphs_and_the_same_bits():
    """Two calls give the same bits; on another stream; captured and replayed with other lengths; two graphs with workspaces of their own."""
    c = make(19, "gqa", lengths(20, 1000, 800), 1000, 64)
    first, lse = call(c)
    second, lse2 = call(c)
    assert torch.equal(first, second) and torch.equal(lse, lse2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    need = B.attn_decode_shared_workspace_size(20, 32, 128, 4, 128, 64, 1000, c["max_len"])
    graphs, outs, spaces = [], [], []
    with torch.cuda.stream(side):
        out, _ = call(c)
        side.synchronize()
        assert torch.equal(out, first)
        for _ in range(2):
            spaces.append(torch.empty(need, dtype=torch.uint8, device="cuda"))
            outs.append(torch.empty_like(first))
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                call(c, out=outs[-1], workspace=spaces[-1], want_lse=False)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    lens = c["lens"].clone()
    c["lens"].copy_(torch.where(lens > 1000, 1000 + (lens - 1000) // 2, lens))
    c["np_lens"] = c["lens"].tolist()
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    check(c, outs[0], None)
    B.check_dev_status()


def test_far_pages():
    """Pages beyond 2^32 bytes of the pool."""
    hq, n, dqk, dv, _ = LAYOUTS["gqa"]
    c = make(20, "gqa", [300, 200], 150, 64)
    pages = (9 << 29) // (64 * n * dqk * 2) + 40
    kp, vp = (torch.empty((pages, 64, n, dqk), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    shift = pages - c["kp"].shape[0]
    kp[shift:], vp[shift:] = c["kp"], c["vp"]
    out, lse = call(c)
    c["kp"], c["vp"] = kp, vp
    again, lse2 = call(c, prefix_table=c["prefix_table"] + shift, page_tables=c["tables"] + shift)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    B.check_dev_status()


def test_a_step_from_plan_to_attention():
    """As a serving loop makes it: plan, rows into the cache, dense attention, and the sparse calls on the same tables; then the next step."""
    hq, n, dqk, dv, _ = LAYOUTS["gqa"]
    page, prefix, nb, width = 16, 100, 6, 24
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()      # noqa: E731
    n_phys = 200
    kp, vp = rnd(n_phys, page, n, dqk), rnd(n_phys, page, n, dv)
    perm = torch.randperm(n_phys, device="cuda", generator=g).int()
    prefix_table, free = perm[:7], perm[7:]
    tables = torch.full((nb, width), -1, dtype=torch.int32, device="cuda")
    tables[:, :6] = prefix_table[:6]                                            # whole pages are shared ...
    tables[:, 6] = free[:nb]                                                    # ... the one in which the prefix ends is copied
    free = free[nb:]
    for p in (kp, vp):
        p[tables[:, 6].long()] = p[prefix_table[6:7].long()].expand(nb, -1, -1, -1).clone()
    cached = torch.full((nb,), prefix, dtype=torch.int64, device="cuda")
    freqs, scale = B.rope_frequencies(64)
    history = [[] for _ in range(nb)]
    for step in range(3):
        new = torch.tensor([[30, 1, 0, 17, 5, 64], [1, 1, 1, 1, 1, 1], [1, 40, 1, 1, 16, 1]][step], device="cuda")
        T = int(new.sum())
        plan = B.janus_batch_plan(cached, new, tables, free, page_size=page, n_phys_pages=n_phys, max_rows=T + 3)
        free = free[int(plan["counts"][0]):].contiguous()
        q, k, v = rnd(T + 3, hq, dqk), rnd(T + 3, n, dqk), rnd(T + 3, n, dv)
        qr = B.janus_rope_append(k, v, plan["positions"], plan["slots"], freqs, kp, vp, rot_offset=64, scale=scale, q=q)
        last = plan["row_offsets"][1:] - 1                                      # the last new token of every session asks
        ask = qr[last.clamp(min=0)].contiguous()
        out, lse = B.janus_attn_decode_shared(ask, kp, vp, prefix_table=prefix_table, prefix_len=prefix, page_tables=plan["page_tables"], table_offsets=plan["table_offsets"],
                                              kv_lens=plan["kv_lens"], max_len=width * page, page_size=page, softmax_scale=0.1, d_v=dv)
        kt = B.janus_rope(k, plan["positions"], freqs, rot_offset=64, scale=scale)
        rows = plan["row_offsets"].tolist()
        top = int(plan["kv_lens"].max())
        idx = torch.full((nb, top), -1, dtype=torch.int32, device="cuda")
        for b in range(nb):
            history[b] += [(kt[r], v[r]) for r in range(rows[b], rows[b + 1])]
            at = torch.arange(prefix, device="cuda")
            ks = torch.cat((kp[prefix_table.long()].flatten(0, 1)[at], torch.stack([x for x, _ in history[b]]) if history[b] else kt[:0])).double()
            vs = torch.cat((vp[prefix_table.long()].flatten(0, 1)[at], torch.stack([x for _, x in history[b]]) if history[b] else v[:0])).double()
            assert ks.shape[0] == int(plan["kv_lens"][b])
            idx[b, :ks.shape[0]] = torch.arange(ks.shape[0], device="cuda", dtype=torch.int32)
            for h in range(n):
                hs = slice(h * hq // n, (h + 1) * hq // n)
                logits = ask[b, hs].double() @ ks[:, h].t() * 0.1
                p = torch.softmax(logits, -1)
                err, mag = (out[b, hs].double() - p @ vs[:, h]).abs(), p @ vs[:, h].abs()
                assert (err <= 2.0 ** -8 * (p @ vs[:, h]).abs() + (2.0 ** -8 + 2.0 ** -13) * mag).all()
        # the sparse call with everything selected sees the same cache through the same tables
        sp, sp_lse = B.janus_sparse_attn_decode(ask, kp, vp, idx, page_tables=plan["page_tables"], table_offsets=plan["table_offsets"], page_size=page, softmax_scale=0.1, d_v=dv)
        assert (sp_lse - lse).abs().max() < 1e-4 and (sp.float() - out.float()).abs().max() < 2.0 ** -6
        cached = plan["kv_lens"].clone()
    B.check_dev_status()
