"""The operators around the cache of a serving step, as cases that can be timed and whose outputs can be compared.

Four kinds of call of ``paper_2609_36938_b200.binding``, in the order in which a step makes them:

  plan     ``janus_batch_plan``: from the lengths of a batch of sessions the page tables, the rows of the new tokens, their positions
           and their places in the cache
  rope     ``janus_rope``: rotary positions on part of every head
  append   ``janus_rope_append``: new keys rotated and written with their values into the paged cache, queries rotated beside them
  attn     ``janus_attn_decode_shared``: one query token per session over a prefix that all sessions share and each session's own tokens

Inputs are drawn on the device from the seed.  Buffers that a serving loop keeps (plans, outputs, workspace, frequency table) are made in
``prepare``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

#: attention layouts: query heads, key/value heads, key dim, value dim, values alias the keys
LAYOUTS = {
    "latent": (128, 1, 576, 512, True),     # one shared 512 + 64 latent row per token
    "mha": (8, 8, 128, 128, False),         # one query head per key/value head
    "gqa": (32, 4, 128, 128, False),        # eight query heads per key/value head
    "gqa64": (24, 4, 64, 64, False),        # six query heads per key/value head, short rows
    "mha192": (16, 16, 192, 128, False),    # keys with 64 rotated dims beside 128 plain ones
}

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- the cases ------------------------------------------------------------------------------------------------------------
def listed():
    def attn(name, B, layout, prefix, own_max, page=64):
        return {"name": name, "kind": "attn", "B": B, "layout": layout, "prefix": prefix, "own": own_max, "page": page}

    return [
        # a decode step of a small batch: the smallest plan there is, made before every step
        {"name": "plan_decode_12", "kind": "plan", "B": 12, "cached": 50021, "new": 1, "page": 64},
        # decoding sessions beside sessions that append chunks, small pages, entries of the batch that stand empty
        {"name": "plan_mixed_203", "kind": "plan", "B": 203, "cached": 20011, "new": 777, "page": 16},
        # a full server: a thousand sessions of up to 128K tokens
        {"name": "plan_decode_1024", "kind": "plan", "B": 1024, "cached": 131072, "new": 1, "page": 64},
        # the queries of one long append on the latent layout: the last 64 of 576 dims, neighbours paired, stretched for long contexts
        {"name": "rope_latent_q_4096", "kind": "rope", "T": 4096, "H": 128, "row": 576, "offset": 512, "rot": 64, "dtype": "bf16", "interleaved": True,
         "scaling": "yarn", "inverse": False, "positions": 135168},
        # whole heads in halves, in fp32, turned back, at far positions
        {"name": "rope_half_fp32_777", "kind": "rope", "T": 777, "H": 32, "row": 128, "offset": 0, "rot": 128, "dtype": "fp32", "interleaved": False,
         "scaling": "linear", "inverse": True, "positions": 1048576},
        # one decode step of a small batch, latent rows, queries in the same call: latency
        {"name": "append_decode_12", "kind": "append", "T": 12, "layout": "latent", "page": 64, "rot": 64, "interleaved": True, "scaling": "yarn"},
        # the rows of a long append of a grouped layout
        {"name": "append_gqa_4096", "kind": "append", "T": 4096, "layout": "gqa", "page": 64, "rot": 128, "interleaved": False, "scaling": None},
        # one session with a short history: the smallest attention there is
        attn("attn_gqa_1", 1, "gqa", 1000, 2000),
        # a serving batch over a common system prompt, ragged histories behind it
        attn("attn_gqa_16", 16, "gqa", 8192, 4096),
        # a full batch over a long common document
        attn("attn_gqa_96", 96, "gqa", 65536, 2048),
        # one query head per kv head, odd lengths, small pages
        attn("attn_mha_37", 37, "mha", 20011, 777, page=16),
        # the latent layout, 128 heads over one row per token
        attn("attn_latent_24", 24, "latent", 8192, 1024),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "rope", "append", "attn", "attn", "attn"])
    if kind == "plan":
        return {"kind": kind, "B": _spread(rng, 1, 1024), "cached": _spread(rng, 64, 131072), "new": rng.choice([1, _spread(rng, 1, 512)]),
                "page": rng.choice([1, 16, 48, 64, 128])}
    if kind == "rope":
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rot = rng.choice([32, 64, 96, 128])
        row = rng.choice([r for r in (64, 96, 128, 192, 576) if r >= rot])
        return {"kind": kind, "T": _spread(rng, 1, 2048), "H": rng.choice([1, 4, 24, 32, 64, 128]), "row": row, "offset": rng.choice([0, row - rot]), "rot": rot,
                "dtype": dtype, "interleaved": rng.random() < 0.5, "scaling": rng.choice([None, "linear", "yarn"]), "inverse": rng.random() < 0.4,
                "positions": _spread(rng, 4096, 1048576)}
    if kind == "append":
        layout = rng.choice(sorted(LAYOUTS))
        return {"kind": kind, "T": _spread(rng, 1, 2048), "layout": layout, "page": rng.choice([1, 16, 48, 64, 128]), "rot": rng.choice([32, 64]),
                "interleaved": rng.random() < 0.5, "scaling": rng.choice([None, "linear", "yarn"])}
    while True:
        layout = rng.choice(["latent", "mha", "gqa", "gqa", "gqa64", "mha192"])
        case = {"kind": kind, "B": _spread(rng, 1, 128), "layout": layout, "prefix": _spread(rng, 64, 65536), "own": _spread(rng, 1, 8192),
                "page": rng.choice([16, 64, 64, 128])}
        w, most = work(case), work({"kind": "attn", "B": 96, "layout": "gqa", "prefix": 65536, "own": 2048, "page": 64})
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _lengths(rng, n, hi):
    """n lengths between 0 and hi: most spread over their logarithm, the longest among them, some very short."""
    out = np.exp(rng.uniform(0, np.log(hi + 1), n)).astype(np.int64)
    out[rng.random(n) < 0.3] = rng.integers(max(hi // 2, 1), hi + 1)
    out[int(rng.integers(n))] = hi
    return np.minimum(out, hi)


def _rng(case, seed):
    return np.random.default_rng([seed, sum(map(ord, case["kind"]))])


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _frequencies(rot, scaling):
    """Radians per position of every pair, in 64 bits, and the factor on the rotated values."""
    base, factor, old = 10000.0, 8.0, 4096
    i = np.arange(rot // 2, dtype=np.float64)
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":      # fast pairs stay, slow ones are stretched, a ramp between 32 and 1 turns over the old context
        def pair_of(turns):
            return rot * math.log(old / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
        ramp = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f / factor * ramp + f * (1.0 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


_SCALING = {None: None, "linear": {"type": "linear", "factor": 8.0}, "yarn": {"type": "yarn", "factor": 8.0, "original_max_position": 4096}}


def _row_budget(case):
    """Rows that the buffers of a step have room for: a whole number of 64, or one for each session where all decode."""
    return case["B"] if case["new"] == 1 else -(-max(case["B"], case["B"] * case["new"] // 6) // 64) * 64


def _plan_lengths(case, seed):
    rng = _rng(case, seed)
    n, most = case["B"], case["new"]
    cached = _lengths(rng, n, case["cached"])
    if most == 1:
        new = np.ones(n, dtype=np.int64)
    else:
        new = np.where(rng.random(n) < 0.5, 1, _lengths(rng, n, most))
        new = np.diff(np.minimum(np.cumsum(new), _row_budget(case)), prepend=0)      # a step takes so many tokens and no more
    if n >= 8:      # entries of the batch that stand empty
        cached[n // 3] = new[n // 3] = 0
        new[n // 2] = 0
    return cached, new


def prepare(case, seed):
    if own:
        from paper_2609_36938_b200 import binding
    g, kind = _gen(seed), case["kind"]
    if kind == "plan":
        cached, new = _plan_lengths(case, seed)
        n, page = case["B"], case["page"]
        width = -(-(case["cached"] + case["new"]) // page)
        held, total = -(-cached // page), -(-(cached + new) // page)
        n_new = int((total - held).sum())
        n_phys = int(held.sum()) + n_new + 64
        perm = torch.randperm(n_phys, device="cuda", generator=g).to(torch.int32)
        tables = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        cols = torch.arange(width, device="cuda")
        tables[cols < torch.from_numpy(held).cuda()[:, None]] = perm[:int(held.sum())]
        capacity, rows = n * width, _row_budget(case)
        state = {"case": case, "cached": torch.from_numpy(cached).cuda(), "new": torch.from_numpy(new).cuda(), "tables": tables,
                 "free": perm[int(held.sum()):].contiguous(), "n_phys": n_phys, "rows": rows, "capacity": capacity,
                 "key_offsets": torch.arange(n + 1, device="cuda", dtype=torch.int64) * (-(-(case["cached"] + case["new"]) // 4) * 4)}
        if own:
            state["out"] = binding.batch_plan_buffers(n, rows, capacity, want_key_rows=True)
            state["out"]["page_tables"].fill_(-1)
        else:
            state["page_tables"] = torch.full((capacity,), -1, dtype=torch.int32, device="cuda")
        return state
    if kind == "rope":
        T, H, row, off, rot = case["T"], case["H"], case["row"], case["offset"], case["rot"]
        dtype = TYPES[case["dtype"]]
        state = {"case": case, "x": torch.randn((T, H, row), device="cuda", generator=g).to(dtype)[:, :, off:off + rot],
                 "out": torch.empty((T, H, row), device="cuda", dtype=dtype)[:, :, off:off + rot],
                 "pos": torch.randint(0, case["positions"], (T,), device="cuda", generator=g)}
        state["freqs"] = binding.rope_frequencies(rot, scaling=_SCALING[case["scaling"]]) if own else _frequencies_on_device(case)
        return state
    if kind == "append":
        T, page = case["T"], case["page"]
        hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
        n_pages = 2 * (-(-T // page)) + 1
        state = {"case": case, "q": torch.randn((T, hq, d_qk), device="cuda", generator=g).bfloat16(),
                 "k": torch.randn((T, n_kv, d_qk), device="cuda", generator=g).bfloat16(),
                 "v": None if alias else torch.randn((T, n_kv, d_v), device="cuda", generator=g).bfloat16(),
                 "k_pool": torch.randn((n_pages, page, n_kv, d_qk), device="cuda", generator=g).bfloat16(),
                 "v_pool": None if alias else torch.randn((n_pages, page, n_kv, d_v), device="cuda", generator=g).bfloat16(),
                 "pos": torch.randint(0, 131072, (T,), device="cuda", generator=g),
                 "slots": torch.randperm(n_pages * page, device="cuda", generator=g)[:T].contiguous(),
                 "q_out": torch.empty((T, hq, d_qk), device="cuda", dtype=torch.bfloat16)}
        if T >= 8:      # rows that stand empty at the end of a padded batch
            state["slots"][T - T // 8:] = -1
            state["pos"][T - T // 8:] = -1
            state["q_out"][T - T // 8:] = 0
        state["freqs"] = binding.rope_frequencies(case["rot"], scaling=_SCALING[case["scaling"]]) if own else _frequencies_on_device(case)
        return state
    n, page, prefix = case["B"], case["page"], case["prefix"]
    hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
    lens = _attn_lengths(case, seed)
    n_pages_b = -(-lens // page)
    n_prefix = -(-prefix // page)
    own_pages = np.maximum(n_pages_b - prefix // page, 0)      # a page that the prefix ends in is the session's own copy
    n_phys = n_prefix + int(own_pages.sum()) + 3
    perm = np.random.default_rng(seed).permutation(n_phys).astype(np.int32)
    tables, at = [], n_prefix
    for b in range(n):
        shared = min(prefix // page, int(n_pages_b[b]))
        tables.append(np.concatenate([perm[:shared], perm[at:at + int(own_pages[b])]]))
        at += int(own_pages[b])
    offsets = np.concatenate([[0], np.cumsum([len(t) for t in tables])]).astype(np.int64)
    k_pool = torch.randn((n_phys, page, n_kv, d_qk), device="cuda", generator=g, dtype=torch.bfloat16)
    state = {"case": case, "q": torch.randn((n, hq, d_qk), device="cuda", generator=g).bfloat16(), "k_pool": k_pool,
             "v_pool": k_pool if alias else torch.randn((n_phys, page, n_kv, d_v), device="cuda", generator=g, dtype=torch.bfloat16),
             "prefix_table": torch.from_numpy(perm[:n_prefix].copy()).cuda(), "tables": torch.from_numpy(np.concatenate(tables)).cuda(),
             "offsets": torch.from_numpy(offsets).cuda(), "lens": torch.from_numpy(lens).cuda(), "max_len": prefix + case["own"],
             "out": torch.empty((n, hq, d_v), device="cuda", dtype=torch.bfloat16)}
    if own:
        need = binding.attn_decode_shared_workspace_size(n, hq, d_qk, n_kv, d_v, page, prefix, state["max_len"])
        state["ws"] = torch.empty((max(need, 16),), dtype=torch.uint8, device="cuda")
    return state


def _attn_lengths(case, seed):
    lens = case["prefix"] + _lengths(_rng(case, seed), case["B"], case["own"])
    if case["B"] >= 8:
        lens[case["B"] // 3] = 0                        # an entry of the batch that stands empty
        lens[case["B"] // 2] = case["prefix"]           # a session with nothing of its own yet
    return lens


def _frequencies_on_device(case):
    f, scale = _frequencies(case["rot"], case["scaling"])
    return torch.from_numpy(f).cuda(), scale


# ---- one pass -----------------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2609_36938_b200 import binding

    case = s["case"]
    if case["kind"] == "plan":
        out = binding.janus_batch_plan(s["cached"], s["new"], s["tables"], s["free"], page_size=case["page"], n_phys_pages=s["n_phys"],
                                       max_rows=s["rows"], key_offsets=s["key_offsets"], out=s["out"])
        return {**out, "block_tables": s["tables"]}
    if case["kind"] == "rope":
        freqs, scale = s["freqs"]
        return binding.janus_rope(s["x"], s["pos"], freqs, interleaved=case["interleaved"], scale=scale, inverse=case["inverse"], out=s["out"])
    if case["kind"] == "append":
        freqs, scale = s["freqs"]
        d_qk = LAYOUTS[case["layout"]][2]
        q = binding.janus_rope_append(s["k"], s["v"], s["pos"], s["slots"], freqs, s["k_pool"], s["v_pool"], rot_offset=d_qk - case["rot"],
                                      interleaved=case["interleaved"], scale=scale, q=s["q"], q_out=s["q_out"])
        return {"q": q, "k_pool": s["k_pool"], **({} if s["v_pool"] is None else {"v_pool": s["v_pool"]})}
    hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
    out, lse = binding.janus_attn_decode_shared(s["q"], s["k_pool"], s["v_pool"], prefix_table=s["prefix_table"], prefix_len=case["prefix"],
                                                page_tables=s["tables"], table_offsets=s["offsets"], kv_lens=s["lens"], max_len=s["max_len"],
                                                page_size=case["page"], softmax_scale=1 / math.sqrt(d_qk), d_v=d_v, out=s["out"], workspace=s["ws"])
    return {"out": out, "lse": lse}


def _rotate(x, pos, freqs, scale, interleaved, inverse):
    """x [T, H, rot] in fp32, angles in fp64."""
    a = pos.double()[:, None] * freqs
    a = torch.where(pos[:, None] < 0, 0.0, a)
    c, s = (torch.cos(a) * scale).float()[:, None], (torch.sin(a) * (-scale if inverse else scale)).float()[:, None]
    if interleaved:
        x1, x2 = x[..., 0::2].float(), x[..., 1::2].float()
        return torch.stack((x1 * c - x2 * s, x1 * s + x2 * c), -1).flatten(-2)
    half = x.shape[-1] // 2
    x1, x2 = x[..., :half].float(), x[..., half:].float()
    return torch.cat((x1 * c - x2 * s, x1 * s + x2 * c), -1)


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "plan":
        return _plan_plain(s)
    if case["kind"] == "rope":
        freqs, scale = s["freqs"]
        s["out"].copy_(_rotate(s["x"], s["pos"], freqs, scale, case["interleaved"], case["inverse"]).to(s["x"].dtype))
        return s["out"]
    if case["kind"] == "append":
        freqs, scale = s["freqs"]
        off = s["q"].shape[-1] - case["rot"]
        live = s["slots"] >= 0
        for x, where in ((s["q"], "q"), (s["k"], "k")):
            y = x.clone()
            y[..., off:] = _rotate(x[..., off:], s["pos"], freqs, scale, case["interleaved"], False).to(x.dtype)
            if where == "q":
                s["q_out"][live] = y[live]
            else:
                s["k_pool"].view(-1, *x.shape[1:])[s["slots"][live]] = y[live]
        if s["v"] is not None:
            s["v_pool"].view(-1, *s["v"].shape[1:])[s["slots"][live]] = s["v"][live]
        return {"q": s["q_out"], "k_pool": s["k_pool"], **({} if s["v_pool"] is None else {"v_pool": s["v_pool"]})}
    return _attn_plain(s)


def _plan_plain(s):
    page, cached, new, tables = s["case"]["page"], s["cached"], s["new"], s["tables"]
    n, width = tables.shape
    dev = tables.device

    def exclusive(x):
        return torch.cat((torch.zeros(1, dtype=torch.int64, device=dev), torch.cumsum(x, 0)))

    lens = cached + new
    held, total = (cached + page - 1) // page, (lens + page - 1) // page
    row_offsets, table_offsets, taken = exclusive(new), exclusive(total), exclusive(total - held)
    cols = torch.arange(width, device=dev)
    fresh = (cols >= held[:, None]) & (cols < total[:, None])
    rank = (taken[:-1, None] + cols - held[:, None]).clamp(0, max(s["free"].numel() - 1, 0))
    tables.copy_(torch.where(fresh, s["free"][rank], tables))
    page_tables = s["page_tables"]
    flat = tables[cols < total[:, None]]
    page_tables[:flat.numel()] = flat
    rows = torch.arange(s["rows"], device=dev)
    live = rows < row_offsets[-1]
    b = (torch.searchsorted(row_offsets, rows, right=True) - 1).clamp(0, n - 1)
    pos = cached[b] + rows - row_offsets[b]
    slot = tables[b, (pos // page).clamp(0, width - 1)].long() * page + pos % page
    counts = torch.stack((taken[-1], table_offsets[-1], row_offsets[-1]))
    return {"row_offsets": row_offsets, "kv_lens": lens, "table_offsets": table_offsets, "page_tables": page_tables,
            "row_sessions": torch.where(live, b, -1).int(), "positions": torch.where(live, pos, -1), "slots": torch.where(live, slot, -1), "counts": counts,
            "key_rows": torch.where(live, s["key_offsets"][b] + pos, -1), "block_tables": tables}


def _attn_plain(s):
    case = s["case"]
    hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
    n, page, prefix, group = case["B"], case["page"], case["prefix"], hq // n_kv
    dev, scale = s["q"].device, 1 / math.sqrt(d_qk)
    q = s["q"].float().view(n, n_kv, group, d_qk)
    k_rows, v_rows = s["k_pool"].view(-1, n_kv, d_qk), s["v_pool"].view(-1, n_kv, s["v_pool"].shape[-1])
    at = torch.arange(prefix, device=dev)
    shared = s["prefix_table"][at // page].long() * page + at % page
    pos = prefix + torch.arange(case["own"], device=dev)
    mine = pos < s["lens"][:, None]
    entry = (s["offsets"][:-1, None] + pos // page).clamp(0, max(s["tables"].numel() - 1, 0))
    rows = torch.where(mine, s["tables"][entry].long() * page + pos % page, 0)
    lse = torch.empty((n, n_kv, group), device=dev)
    empty = (s["lens"] == 0)[:, None, None]
    out = s["out"].view(n, n_kv, group, d_v)
    for h in range(n_kv):
        kp, vp = k_rows[shared, h].float(), v_rows[shared, h, :d_v].float()
        a = torch.matmul(q[:, h].reshape(n * group, d_qk), kp.t()).view(n, group, prefix) * scale
        c = torch.matmul(q[:, h], k_rows[rows, h].float().transpose(1, 2)) * scale
        c = c.masked_fill(~mine[:, None], -math.inf)
        top = torch.maximum(a.amax(-1), c.amax(-1))[..., None]
        a, c = torch.exp(a - top), torch.exp(c - top)
        total = a.sum(-1) + c.sum(-1)
        o = torch.matmul(a.view(n * group, prefix), vp).view(n, group, d_v) + torch.matmul(c, v_rows[rows, h, :d_v].float())
        out[:, h] = torch.where(empty, 0.0, o / total[..., None]).to(out.dtype)
        lse[:, h] = torch.where(empty[..., 0], -math.inf, top[..., 0] + torch.log(total))
    return {"out": s["out"], "lse": lse.view(n, hq)}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------
def _turned(x, pos, case, inverse):
    """Rotation of x's last axis as a product of complex numbers, in 64 bits."""
    f, scale = _frequencies(case["rot"], case["scaling"])
    a = pos.double().clamp(min=0)[:, None, None] * torch.from_numpy(f).cuda()
    z = x.double()
    z = torch.view_as_complex(z.unflatten(-1, (-1, 2)).contiguous()) if case["interleaved"] else torch.complex(*z.chunk(2, -1))
    z = z * torch.polar(torch.full_like(a, scale), -a if inverse else a)
    return torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat((z.real, z.imag), -1)


def exact(case, seed):
    if case["kind"] == "plan":
        return None      # whole numbers only
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _turned(s["x"], s["pos"], case, case["inverse"])
    if case["kind"] == "append":
        off = s["q"].shape[-1] - case["rot"]
        res = {"q": s["q_out"].double(), "k_pool": s["k_pool"].double()}
        q, k = (torch.cat((x[..., :off].double(), _turned(x[..., off:], s["pos"], case, False)), -1) for x in (s["q"], s["k"]))
        n = int((s["slots"] >= 0).sum())
        res["q"][:n] = q[:n]
        where = s["slots"][:n]
        res["k_pool"][where // case["page"], where % case["page"]] = k[:n]
        if s["v"] is not None:
            res["v_pool"] = s["v_pool"].double()
            res["v_pool"][where // case["page"], where % case["page"]] = s["v"][:n].double()
        return res
    hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
    n, group, page = case["B"], hq // n_kv, case["page"]
    out = torch.zeros((n, hq, d_v), dtype=torch.float64, device="cuda")
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
    lens, offsets = s["lens"].tolist(), s["offsets"].tolist()
    for b in range(n):
        if lens[b] == 0:
            continue
        table = s["tables"][offsets[b]:offsets[b + 1]].long()
        ids = torch.cat((s["prefix_table"].long(), table[case["prefix"] // page:]))
        rest = case["prefix"] % page
        k, v = s["k_pool"][ids], s["v_pool"][ids][..., :d_v]
        k, v = k.flatten(0, 1), v.flatten(0, 1)
        if rest and lens[b] > case["prefix"]:      # the last page of the prefix holds only its first tokens; the session's copy the ones after them
            end = len(s["prefix_table"]) * page
            keep = torch.cat((torch.arange(case["prefix"], device="cuda"), torch.arange(end + rest, k.shape[0], device="cuda")))
            k, v = k[keep], v[keep]
        k, v = k[:lens[b]], v[:lens[b]]
        for h in range(n_kv):
            logits = s["q"][b, h * group:(h + 1) * group].double() @ k[:, h].double().t() / math.sqrt(d_qk)
            lse[b, h * group:(h + 1) * group] = torch.logsumexp(logits, -1)
            out[b, h * group:(h + 1) * group] = torch.softmax(logits, -1) @ v[:, h].double()
    return {"out": out, "lse": lse}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "plan":
        cached, new = _plan_lengths(case, 0)
        page = case["page"]
        held, total = -(-cached // page), -(-(cached + new) // page)
        # lengths, offsets of the keys; held pages and fresh ones in, all out, fresh ones into the block tables; rows; offsets and lengths
        moved = 24 * case["B"] + 4 * int(total.sum()) * 2 + 4 * int((total - held).sum()) + 28 * int(new.sum()) + 24 * case["B"]
        return {"bytes": float(moved), "flops": float(10 * case["B"])}
    if kind == "rope":
        size = torch.empty(0, dtype=TYPES[case["dtype"]]).element_size()
        n = case["T"] * case["H"] * case["rot"]
        return {"bytes": float(2 * n * size + 8 * case["T"]), "flops": float(3 * n)}
    hq, n_kv, d_qk, d_v, alias = LAYOUTS[case["layout"]]
    if kind == "append":
        T = case["T"] - (case["T"] // 8 if case["T"] >= 8 else 0)
        row = hq * d_qk + n_kv * (d_qk + (0 if alias else d_v))
        return {"bytes": float(T * (4 * row + 16)), "flops": float(3 * T * (hq + n_kv) * case["rot"])}
    lens = _attn_lengths(case, 0)
    own_tokens, live = int(np.maximum(lens - case["prefix"], 0).sum()), int((lens > 0).sum())
    row = 2 * n_kv * (d_qk + (0 if alias else d_v))
    moved = (case["prefix"] + own_tokens) * row + case["B"] * hq * (2 * d_qk + 2 * d_v + 4)
    return {"bytes": float(moved), "flops": float(2 * hq * (d_qk + d_v) * (live * case["prefix"] + own_tokens))}
