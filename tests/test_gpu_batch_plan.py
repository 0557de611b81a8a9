"""janus_batch_plan against the definition in whole numbers."""
import numpy as np
import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu


def reference(cached, new, tables, free, page, n_phys, max_rows, capacity, key_offsets):
    """The header's definition, one session after the other; also the status that is reported (0, 101 or 102, the first one wins nowhere here)."""
    n, width = tables.shape
    tables = tables.copy()
    room, conditions = width * page, set()
    row_off, tab_off, lens, pt, rows, taken = [0], [0], [], [], [], 0
    for b in range(n):
        c, m = int(cached[b]), int(new[b])
        if c < 0 or m < 0:
            conditions.add(101)
        c, m = max(c, 0), max(m, 0)
        if c > room or c + m > room:
            conditions.add(102)
        held, total = -(-min(c, room) // page), -(-min(c + m, room) // page)
        ids = []
        for j in range(total):
            if j < held:
                pid = int(tables[b, j])
            elif taken < len(free):
                pid = int(free[taken])
            else:
                pid = None
                conditions.add(102)
            if j >= held:
                taken += 1
            if pid is not None and not 0 <= pid < n_phys:
                conditions.add(101)
                pid = None
            pid = -1 if pid is None else pid
            if j >= held:
                tables[b, j] = pid
            ids.append(pid)
        pt += ids
        for i in range(min(m, max_rows + 1)):
            pos = c + i if c <= room else c + i
            j = pos // page
            slot = ids[j] * page + pos % page if j < len(ids) and ids[j] >= 0 else -1
            rows.append((b, pos, slot, -1 if slot < 0 else int(key_offsets[b]) + pos))
        row_off.append(row_off[-1] + m)
        tab_off.append(tab_off[-1] + total)
        lens.append(min(c + m, room))
    if row_off[-1] > max_rows or tab_off[-1] > capacity:
        conditions.add(102)
    counts = [taken, tab_off[-1], row_off[-1]]
    rows = (rows + [(-1, -1, -1, -1)] * max_rows)[:max_rows]
    return {"row_offsets": np.minimum(row_off, max_rows), "table_offsets": np.minimum(tab_off, capacity), "kv_lens": np.array(lens), "page_tables": np.array(pt[:capacity]),
            "row_sessions": np.array([r[0] for r in rows]), "positions": np.array([r[1] for r in rows]), "slots": np.array([r[2] for r in rows]),
            "key_rows": np.array([r[3] for r in rows]), "counts": np.array(counts), "block_tables": tables}, conditions


def make(seed, n, page, most, new_most, spare=7):
    rng = np.random.default_rng(seed)
    cached = np.exp(rng.uniform(0, np.log(most + 1), n)).astype(np.int64) - 1
    new = np.where(rng.random(n) < 0.5, 1, rng.integers(0, new_most + 1, n)).astype(np.int64)
    if n > 3:
        cached[1] = new[1] = 0
        new[2] = 0
    width = max(1, -(-(most + new_most) // page))
    held, total = -(-cached // page), -(-(cached + new) // page)
    n_phys = int(total.sum()) + spare
    perm = rng.permutation(n_phys).astype(np.int32)
    tables, at = np.full((n, width), -1, np.int32), 0
    for b in range(n):
        tables[b, :held[b]] = perm[at:at + held[b]]
        at += int(held[b])
    return cached, new, tables, perm[at:], n_phys, np.arange(n + 1, dtype=np.int64) * (most + new_most + 4) // 4 * 4


def check(got, want, tables_dev):
    for name, w in want.items():
        g = tables_dev.cpu().numpy() if name == "block_tables" else got[name].cpu().numpy()
        assert np.array_equal(g[:len(w)] if name == "page_tables" else g, w), name
    assert (got["page_tables"].cpu().numpy()[len(want["page_tables"]):] == -7).all()      # behind the last table: as it was


def run(cached, new, tables, free, page, n_phys, max_rows, capacity, key_offsets, dev_tables=None):
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (cached, new, free, key_offsets)]
    t = torch.from_numpy(tables).cuda() if dev_tables is None else dev_tables
    out = B.batch_plan_buffers(len(cached), max_rows, capacity, want_key_rows=True)
    out["page_tables"].fill_(-7)
    got = B.janus_batch_plan(dev[0], dev[1], t, dev[2], page_size=page, n_phys_pages=n_phys, max_rows=max_rows, key_offsets=dev[3], out=out)
    assert got is out
    return got, t


@pytest.mark.parametrize("n,page,most,new_most", [(1, 64, 1, 1), (1, 1, 300, 40), (2, 64, 4096, 1), (12, 64, 50021, 1), (37, 48, 3000, 500), (203, 16, 2011, 77),
                                                  (512, 64, 1000, 1), (513, 128, 1000, 3), (1024, 64, 9000, 1), (3001, 16, 100, 2)])
def test_plan(n, page, most, new_most):
    cached, new, tables, free, n_phys, keys = make(n + page, n, page, most, new_most)
    max_rows = int(new.sum()) + 5
    want, cond = reference(cached, new, tables, free, page, n_phys, max_rows, n * tables.shape[1], keys)
    assert not cond
    got, t = run(cached, new, tables, free, page, n_phys, max_rows, n * tables.shape[1], keys)
    check(got, want, t)
    B.check_dev_status()


def test_largest_batch():
    n = 8192
    cached, new, tables, free, n_phys, keys = make(5, n, 64, 500, 1)
    want, cond = reference(cached, new, tables, free, 64, n_phys, n, 70000, keys)
    assert not cond
    got, t = run(cached, new, tables, free, 64, n_phys, n, 70000, keys)
    check(got, want, t)
    B.check_dev_status()
    with pytest.raises(B.JanusError, match="UNSUPPORTED"):
        z = torch.zeros(8193, dtype=torch.int64, device="cuda")
        B.janus_batch_plan(z, z, torch.zeros((8193, 1), dtype=torch.int32, device="cuda"), z.int(), page_size=64, n_phys_pages=4, max_rows=1)


def expect(code, got, want, t):
    with pytest.raises(B.JanusError, match=B.DEV_NAMES[code]):
        B.check_dev_status()
    check(got, want, t)


def test_lists_that_are_too_short():
    cached, new, tables, free, n_phys, keys = make(3, 20, 16, 900, 100)
    full, total = int(new.sum()), int((-(-(cached + new) // 16)).sum())
    for kw in (dict(free=free[:5]), dict(max_rows=full // 2), dict(capacity=total // 2), dict(free=free[:0], max_rows=0, capacity=0)):
        a = dict(dict(free=free, max_rows=full, capacity=total), **kw)
        want, cond = reference(cached, new, tables, a["free"], 16, n_phys, a["max_rows"], a["capacity"], keys)
        assert cond == {102}
        got, t = run(cached, new, tables, a["free"], 16, n_phys, a["max_rows"], a["capacity"], keys)
        expect(102, got, want, t)


def test_sessions_longer_than_their_table():
    cached, new, tables, free, n_phys, keys = make(4, 9, 16, 900, 100)
    cached[3], new[3] = tables.shape[1] * 16 - 3, 10          # the last tokens have no page
    cached[4], new[4] = tables.shape[1] * 16 + 5, 4           # nor do these, cached ones included
    new[5] = 1 << 40                                          # more rows than any buffer
    tables[3] = tables[4] = np.arange(tables.shape[1]) % n_phys
    free = np.arange(400, dtype=np.int32) % n_phys
    want, cond = reference(cached, new, tables, free, 16, n_phys, 300, 4000, keys)
    assert cond == {102}
    want["counts"][2] = int(new.sum()) - new[5] + 2 ** 31 - 1      # (a session's rows count up to 2^31 - 1)
    got, t = run(cached, new, tables, free, 16, n_phys, 300, 4000, keys)
    expect(102, got, want, t)


def test_bad_lengths_and_pages():
    cached, new, tables, free, n_phys, keys = make(6, 11, 16, 900, 100)
    cached[4], new[6] = -5, -1
    tables[7, 0], tables[8, 0] = n_phys, -3
    cached[7] = cached[8] = 40
    tables[7, 1:3] = tables[8, 1:3] = 1
    free = free.copy()
    free[1] = 1 << 30
    want, cond = reference(cached, new, tables, free, 16, n_phys, 700, 4000, keys)
    assert 101 in cond
    if 102 in cond:
        pytest.fail("the case is to have one condition")
    got, t = run(cached, new, tables, free, 16, n_phys, 700, 4000, keys)
    expect(101, got, want, t)


def test_no_sessions():
    z, t = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros((0, 4), dtype=torch.int32, device="cuda")
    got = B.janus_batch_plan(z, z, t, z.int(), page_size=64, n_phys_pages=0, max_rows=3)
    assert got["row_offsets"].tolist() == [0] and got["table_offsets"].tolist() == [0] and got["counts"].tolist() == [0, 0, 0]
    assert got["slots"].tolist() == [-1] * 3 and got["row_sessions"].tolist() == [-1] * 3
    B.check_dev_status()


def test_buffers_that_are_too_short_are_refused():
    lens, table = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(B.JanusError, match="at least 5"):
        B.janus_batch_plan(lens, lens, table, table[0], page_size=8, n_phys_pages=4, max_rows=5, out=B.batch_plan_buffers(2, 4, 6))
    with pytest.raises(B.JanusError, match="adjacent columns"):
        B.janus_batch_plan(lens, lens, torch.zeros(3, 2, dtype=torch.int32, device="cuda").t(), table[0], page_size=8, n_phys_pages=4, max_rows=5)
    with pytest.raises(B.JanusError, match="INVALID_ARG"):
        B.janus_batch_plan(lens, lens, table[:1].expand(2, 3), table[0], page_size=8, n_phys_pages=4, max_rows=5)


def test_strided_tables_other_stream_and_replay():
    """Rows of a wider table; a graph that is replayed with other lengths and another free list."""
    n, page = 24, 16
    cached, new, tables, free, n_phys, keys = make(8, n, page, 900, 60)
    wide = torch.full((n, tables.shape[1] + 5), 99, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = torch.from_numpy(tables).cuda()
    view, max_rows, capacity = wide[:, :tables.shape[1]], 1500, 3000
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (cached, new, free, keys)]
    out = B.batch_plan_buffers(n, max_rows, capacity, want_key_rows=True)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        def step():
            B.janus_batch_plan(dev[0], dev[1], view, dev[2], page_size=page, n_phys_pages=n_phys, max_rows=max_rows, key_offsets=dev[3], out=out)
        step()
        side.synchronize()
        with torch.cuda.graph(g, stream=side):
            step()
    for seed in (8, 9, 10):
        rng = np.random.default_rng(seed)
        c, m = (cached, new) if seed == 8 else (np.minimum(cached, rng.integers(0, 900, n)), rng.integers(0, 60, n))
        f = rng.permutation(free)
        view.copy_(torch.from_numpy(tables))
        out["page_tables"].fill_(-7)
        for d, x in zip(dev, (c, m, f)):
            d.copy_(torch.from_numpy(np.ascontiguousarray(x)))
        want, cond = reference(c, m, tables, f, page, n_phys, max_rows, capacity, keys)
        g.replay()
        torch.cuda.synchronize()
        assert cond <= {102}
        if cond:
            expect(102, out, want, view)
        else:
            check(out, want, view)
            B.check_dev_status()
    assert (wide[:, tables.shape[1]:] == 99).all()
