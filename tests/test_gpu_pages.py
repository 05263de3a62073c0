"""A step's tables (update_pages) against a plain program: whole numbers, all equal."""
import pytest
import torch

import paper_2607_13500_amd as tr
from test_gpu_rotate import DEV, gen, say

pytestmark = pytest.mark.gpu

I32, I64 = torch.int32, torch.int64
FULL = 2 ** 31 - 1


def pages_for(n, size):
    return -(-n // size)


def plain(change, kv, table, ring, state, size, rows):
    """Everything that a call returns or writes, from lists."""
    table, ring, pages, width = [list(r) for r in table], list(ring), len(ring), len(table[0]) if table else 0
    after = [max(0, n + c) for n, c in zip(kv, change)]
    held, need = [pages_for(n, size) for n in kv], [pages_for(n, size) for n in after]
    fresh = sum(max(c, 0) for c in change)
    first, free = state
    lack = max(0, sum(max(0, b - a) for a, b in zip(held, need)) - free)
    if any(n > width for n in need) or fresh > rows:
        lack = FULL
    slots, pos, q_start = [-1] * rows, [0] * rows, [0] * (len(kv) + 1)
    if lack:
        return dict(q_start=q_start, kv_len=list(kv), table=table, slots=slots, pos=pos, ring=ring, state=list(state), short=[lack])
    end = first + free
    for b in range(len(kv)):
        for i in range(held[b], need[b]):
            table[b][i] = ring[first % pages]
            first += 1
        for i in range(need[b], held[b]):
            ring[end % pages] = table[b][i]
            end += 1
        q_start[b + 1] = q_start[b] + max(change[b], 0)
        for i in range(max(change[b], 0)):
            p = after[b] - change[b] + i
            slots[q_start[b] + i], pos[q_start[b] + i] = table[b][p // size] * size + p % size, p
    return dict(q_start=q_start, kv_len=after, table=table, slots=slots, pos=pos, ring=ring, state=[first % pages, end - first], short=[0])


def state_of(g, kv, size, width, spare, pad=0):
    """A table, a ring and its state for sequences of kv tokens and `spare` free pages."""
    counts = [pages_for(n, size) for n in kv]
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=g).tolist()
    table = torch.full((len(kv), width + pad), -7, dtype=I32)
    r = 0
    for b, c in enumerate(counts):
        table[b, :c] = torch.tensor(order[r:r + c], dtype=I32)
        r += c
    pages = max(pages, 1)
    ring, first = torch.full((pages,), -9, dtype=I32), int(torch.randint(0, pages, (1,), generator=g))
    for i, p in enumerate(order[r:]):
        ring[(first + i) % pages] = p
    return table, ring, torch.tensor([first, spare], dtype=I32)


def check(change, kv, table, ring, state, size, rows, width, in_place=False, what=""):
    dev = [t.to(DEV) for t in (torch.tensor(change, dtype=I32), torch.tensor(kv, dtype=I32), table, ring, state)]
    want = plain(change, kv, table[:, :width].tolist(), ring.tolist(), state.tolist(), size, rows)
    view = dev[2][:, :width]
    u = tr.update_pages(dev[0], dev[1], view, tr.PagePool(dev[3], dev[4]), size, rows, in_place=in_place)
    got = dict(q_start=u.step.q_start, kv_len=u.step.kv_len, table=u.step.table, slots=u.slots, pos=u.pos, ring=u.pool.ring, state=u.pool.state, short=u.short)
    for name, t in got.items():
        assert t.dtype == (I64 if name == "slots" else I32) and t.tolist() == want[name], (what, name)
    assert torch.equal(dev[2][:, width:].cpu(), table[:, width:])          # what lies between the table's rows
    assert torch.equal(dev[0].cpu(), torch.tensor(change, dtype=I32))
    if in_place:
        assert u.step.kv_len.data_ptr() == dev[1].data_ptr() and u.pool.state.data_ptr() == dev[4].data_ptr()
    else:
        assert dev[1].tolist() == list(kv) and dev[4].tolist() == state.tolist()
    return u


def lengths(g, n, most):
    return torch.randint(0, most + 1, (n,), generator=g).tolist()


@pytest.mark.parametrize("seqs", [1, 2, 63, 64, 65, 300, 1024, 1025, 2500])
@pytest.mark.parametrize("size", [1, 16, 48])
def test_steps(seqs, size):
    """Sequences that grow by one token, by many, shrink, end and stay, in and out of place."""
    for n, (most, new, back) in enumerate([(40, 1, 0), (100, 70, 30), (200, 0, 220), (0, 9, 0), (64, 20, 5)]):
        say("pages", seqs, size, n)
        g = gen(seqs + 31 * n + size)
        kv = lengths(g, seqs, most)
        change = [int(torch.randint(-back, new + 1, (1,), generator=g)) for _ in range(seqs)]
        width = max(1, max(pages_for(max(a, a + c), size) for a, c in zip(kv, change)))
        spare = sum(max(0, pages_for(a + c, size) - pages_for(a, size)) for a, c in zip(kv, change)) + n % 3
        fresh = sum(max(c, 0) for c in change)
        for in_place, pad, more in ((False, 0, 3), (True, 5, 0), (True, 0, 5000)):
            check(change, kv, *state_of(g, kv, size, width, spare, pad), size, fresh + more, width, in_place, (seqs, size, n))


def test_many_pages_and_tokens():
    """More pages and tokens than a workgroup's threads, of few and of one sequence."""
    say("many")
    g = gen(4)
    for kv, change, size in (([0], [70000], 1), ([70000, 5], [-70000, 30000], 1), ([100000, 0, 17], [1, 18432, -17], 16), ([20000] * 40, [-20000] * 20 + [40] * 20, 8)):
        width = max(pages_for(max(a, a + c), size) for a, c in zip(kv, change))
        spare = sum(max(0, pages_for(a + c, size) - pages_for(a, size)) for a, c in zip(kv, change))
        for in_place in (False, True):
            check(change, kv, *state_of(g, kv, size, width, spare), size, sum(max(c, 0) for c in change) + 1, width, in_place)


def test_pages_that_are_lacking():
    """Too few free pages, rows or entries of the table: nothing changes but `short`."""
    for seqs in (3, 1500):
        for in_place in (False, True):
            say("lacking", seqs, in_place)
            g = gen(seqs)
            kv, change = lengths(g, seqs, 60), lengths(g, seqs, 40)
            change[0] = -3
            width = max(pages_for(max(a, a + c), 16) for a, c in zip(kv, change))
            take = sum(max(0, pages_for(a + c, 16) - pages_for(a, 16)) for a, c in zip(kv, change))
            fresh = sum(max(c, 0) for c in change)
            u = check(change, kv, *state_of(g, kv, 16, width, take - 1), 16, fresh, width, in_place)
            assert u.short.tolist() == [1]
            u = check(change, kv, *state_of(g, kv, 16, width, 0), 16, fresh, width, in_place)
            assert u.short.tolist() == [take]
            u = check(change, kv, *state_of(g, kv, 16, width, take), 16, fresh - 1, width, in_place)
            assert u.short.tolist() == [FULL]
            big = list(change)
            big[-1] = width * 16 + 1 - kv[-1]
            u = check(big, kv, *state_of(g, kv, 16, width, take + width), 16, fresh + width * 16, width, in_place)
            assert u.short.tolist() == [FULL]
            check(change, kv, *state_of(g, kv, 16, width, take), 16, fresh, width, in_place)       # exactly enough


def test_lengths_near_2_31():
    say("near 2^31")
    size = 1 << 24
    kv, change = [FULL - 10, FULL, 5], [10, -FULL, FULL - 5]
    g = gen(2)
    width = 128
    table, ring, state = state_of(g, kv, size, width, 130)
    dev = [t.to(DEV) for t in (torch.tensor(change, dtype=I32), torch.tensor(kv, dtype=I32), table, ring, state)]
    u = tr.update_pages(dev[0], dev[1], dev[2], tr.PagePool(dev[3], dev[4]), size, 20)
    assert u.short.tolist() == [FULL] and u.step.kv_len.tolist() == kv            # more new tokens than rows
    dev[0].copy_(torch.tensor([10, -FULL, 0], dtype=I32))
    u = tr.update_pages(dev[0], dev[1], dev[2], tr.PagePool(dev[3], dev[4]), size, 20)
    assert u.short.tolist() == [0] and u.step.kv_len.tolist() == [FULL, 0, 5] and u.pos.tolist()[:10] == [FULL - 10 + i for i in range(10)]
    page = int(table[0, 127])
    assert u.slots.tolist()[:10] == [page * size + (FULL - 10 + i) % size for i in range(10)]
    dev[0].copy_(torch.tensor([11, 0, 0], dtype=I32))                              # past 2^31 - 1 tokens
    u = tr.update_pages(dev[0], dev[1], dev[2], tr.PagePool(dev[3], dev[4]), size, 20)
    assert u.short.tolist() == [FULL]


def test_no_sequences():
    say("none")
    e = torch.zeros(0, dtype=I32, device=DEV)
    ring, state = torch.arange(4, dtype=I32, device=DEV), torch.tensor([1, 2], dtype=I32, device=DEV)
    u = tr.update_pages(e, e, torch.zeros(0, 3, dtype=I32, device=DEV), tr.PagePool(ring, state), 16, 5)
    assert u.step.q_start.tolist() == [0] and u.slots.tolist() == [-1] * 5 and u.pos.tolist() == [0] * 5
    assert u.pool.state.tolist() == [1, 2] and u.short.tolist() == [0]


def test_a_life_of_a_cache():
    """Steps one after another, recorded once and replayed: no page is lost or held twice."""
    say("life")
    g = gen(11)
    seqs, size, width, pages = 40, 16, 12, 80
    kv = torch.zeros(seqs, dtype=I32, device=DEV)
    change = torch.zeros(seqs, dtype=I32, device=DEV)
    table = torch.full((seqs, width), -1, dtype=I32, device=DEV)
    pool = tr.PagePool(torch.randperm(pages, generator=g).to(I32).to(DEV), torch.tensor([0, pages], dtype=I32, device=DEV))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        tr.update_pages(change, kv, table, pool, size, 400, in_place=True)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u = tr.update_pages(change, kv, table, pool, size, 400, in_place=True)
    lacked = 0
    for i in range(60):
        most = (20, 9, 1, 3)[i % 4]
        new = torch.randint(-most, most + 1, (seqs,), generator=g)
        if i % 7 == 6:
            new[torch.randperm(seqs, generator=g)[:5]] = -1000
        change.copy_(new.to(I32))
        torch.cuda.synchronize()
        want = plain(new.tolist(), kv.tolist(), table.tolist(), pool.ring.tolist(), pool.state.tolist(), size, 400)
        graph.replay()
        torch.cuda.synchronize()
        got = dict(q_start=u.step.q_start, kv_len=kv, table=table, slots=u.slots, pos=u.pos, ring=pool.ring, state=pool.state, short=u.short)
        for name, t in got.items():
            assert t.tolist() == want[name], (i, name)
        lacked += want["short"] != [0]
        held = [p for r, n in zip(table.tolist(), kv.tolist()) for p in r[:pages_for(n, size)]]
        first, free = pool.state.tolist()
        held += [pool.ring.tolist()[(first + j) % pages] for j in range(free)]
        assert sorted(held) == list(range(pages))
    assert 0 < lacked < 60


def test_other_streams():
    """A call on a stream of its own, beside work on the current one."""
    g = gen(5)
    kv, change = lengths(g, 50, 90), lengths(g, 50, 9)
    width, take = 8, sum(pages_for(a + c, 16) - pages_for(a, 16) for a, c in zip(kv, change))
    table, ring, state = state_of(g, kv, 16, width, take)
    dev = [t.to(DEV) for t in (torch.tensor(change, dtype=I32), torch.tensor(kv, dtype=I32), table, ring, state)]
    want = plain(change, kv, table.tolist(), ring.tolist(), state.tolist(), 16, sum(change))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    u = tr.update_pages(dev[0], dev[1], dev[2], tr.PagePool(dev[3], dev[4]), 16, sum(change), stream=side)
    side.synchronize()
    assert u.slots.tolist() == want["slots"] and u.step.table.tolist() == want["table"]


def test_refusals():
    kv = torch.zeros(3, dtype=I32, device=DEV)
    table, ring, state = torch.zeros(3, 4, dtype=I32, device=DEV), torch.arange(9, dtype=I32, device=DEV), torch.tensor([0, 9], dtype=I32, device=DEV)
    pool = tr.PagePool(ring, state)
    bad = [lambda: tr.update_pages(kv.long(), kv, table, pool, 16, 4), lambda: tr.update_pages(kv[:2], kv, table, pool, 16, 4),
           lambda: tr.update_pages(kv, kv.cpu(), table, pool, 16, 4), lambda: tr.update_pages(kv, kv, table[:2], pool, 16, 4),
           lambda: tr.update_pages(kv, kv, table.t()[:3, :3], pool, 16, 4), lambda: tr.update_pages(kv, kv, table[:1].expand(3, 4), pool, 16, 4),
           lambda: tr.update_pages(kv, kv, table, pool, 0, 4), lambda: tr.update_pages(kv, kv, table, pool, 16, -1),
           lambda: tr.update_pages(kv, kv, table, pool, (1 << 32) + 16, 4), lambda: tr.update_pages(kv, kv, table, pool, 16, 1 << 31),
           lambda: tr.update_pages(kv, kv, table, tr.PagePool(ring[:0], state), 16, 4), lambda: tr.update_pages(kv, kv, table, tr.PagePool(ring.long(), state), 16, 4),
           lambda: tr.update_pages(kv, kv, table, tr.PagePool(ring, state[:1]), 16, 4), lambda: tr.update_pages(kv, kv, table, tr.PagePool(ring[::2], state), 16, 4)]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, tr.TRError)):
            f()
            print("not refused:", i)
