"""Block tables and slot maps of a step against the definition, request by request in Python: integers, equal in every place."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def oracle(seq_len, new_len, table, free, count, block, rows):
    """table and free are changed; returns (seq_len, count, start, q_start, positions, slots, bad)."""
    B, width, cap, bad = len(seq_len), len(table[0]), len(free), 0
    count = min(max(count, 0), cap)
    old = [min(max(n, 0), width * block) for n in seq_len]
    blocks = [-(-n // block) for n in old]
    for b in range(B):
        if new_len[b] < 0:
            bad += count + blocks[b] > cap
            for j in range(blocks[b]):
                if count + j < cap:
                    free[count + j] = table[b][j]
            count += blocks[b]
    count = min(count, cap)
    asked, taken, row = 0, 0, 0
    out, start, q_start, pos, slots = list(old), [], [], [0] * rows, [-1] * rows
    grants = []
    for b in range(B):
        q_start.append(min(row, rows))
        n = new_len[b]
        start.append(-1)
        if n < 0:
            out[b] = 0
            continue
        row += n
        need = -(-(old[b] + n) // block)
        if need > width or row > rows:
            bad += 1
            continue
        want = need - blocks[b]
        asked += want
        if want and asked > count:
            bad += 1
            continue
        grants.append((b, blocks[b], want, asked - want))
        taken = max(taken, asked if want else 0)
        out[b], start[b] = old[b] + n, old[b]
    for b, have, want, before in grants:
        for j in range(want):
            table[b][have + j] = free[count - 1 - before - j]
    q_start.append(min(row, rows))
    for b in range(B):
        if start[b] >= 0:
            for i in range(new_len[b]):
                p = old[b] + i
                pos[q_start[b] + i] = p
                slots[q_start[b] + i] = table[b][p // block] * block + p % block
    return out, count - taken, start, q_start, pos, slots, bad


def check(seq_len, new_len, table, free, count, block, rows, in_place=False, pad=0):
    from paper_2504_12285_amd import binding as bl
    dev = "cuda:0"

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)
    tab = t([r + [77] * pad for r in table])
    args = [t(seq_len), t(new_len), tab[:, :len(table[0])] if pad else tab, t(free), t([count])]
    h = bl.KVTables(*args, block, rows, in_place=in_place)
    h.run()
    got = [x.tolist() for x in (h.seq_len_out, h.free_count_out, h.start, h.q_start, h.positions, h.slots, h.bad)]
    table, free = [list(r) for r in table], list(free)
    want = oracle(seq_len, new_len, table, free, count, block, rows)
    want = [want[0], [want[1]], *want[2:6], [want[6]]]
    for name, g, w in zip(("seq_len", "free_count", "start", "q_start", "positions", "slots", "bad"), got, want):
        assert g == w, name
    assert tab.tolist() == [r + [77] * pad for r in table]
    assert args[3].tolist() == free
    return h, want


def batch(seed, B, longest, block, width, rows=None, supply=1.0, ends=0.15, cap_slack=0):
    r = random.Random(seed)
    seq = [r.choice([0, 1, block - 1, block, block + 1, r.randrange(longest + 1)]) for _ in range(B)]
    seq = [min(n, width * block) for n in seq]
    new = [-1 if r.random() < ends else r.choice([0, 1, 1, 1, r.randrange(2 * block + 1), r.randrange(longest + 1)]) for _ in range(B)]
    used = [-(-n // block) for n in seq]
    demand = sum(max(0, -(-(s + n) // block) - u) for s, n, u in zip(seq, new, used) if n >= 0)
    count = int(demand * supply)
    ids = list(range(sum(used) + count))
    r.shuffle(ids)
    table = []
    for u in used:
        table.append([ids.pop() for _ in range(u)] + [-1] * (width - u))
    free = ids + [-1] * (sum(used) + cap_slack)
    return seq, new, table, free, count, block, (sum(max(0, n) for n in new) + 3 if rows is None else rows)


@pytest.mark.parametrize("seed, B, longest, block, width", [
    (1, 1, 40, 16, 8), (2, 2, 100, 32, 8), (3, 7, 200, 16, 40), (4, 64, 300, 64, 12), (5, 65, 500, 128, 9), (6, 257, 90, 16, 12),
    (7, 1023, 40, 32, 5), (8, 1025, 50, 16, 8), (9, 4096, 30, 16, 5), (10, 3, 6000, 16, 900)])
@pytest.mark.parametrize("supply", [2.0, 0.6])
def test_random_batches(seed, B, longest, block, width, supply):
    check(*batch(seed, B, longest, block, width, supply=supply))


@pytest.mark.parametrize("in_place", [False, True])
def test_in_place_and_wide_tables(in_place):
    check(*batch(11, 33, 100, 16, 20), in_place=in_place, pad=5)


def test_rows_that_do_not_fit_are_refused():
    for rows in (1, 5, 40, 5000):
        check(*batch(12, 40, 60, 16, 10, rows=rows))


def test_more_rows_than_the_table_kernel_writes_itself():
    check(*batch(13, 20, 2000, 32, 150, supply=1.0))
    check(*batch(13, 20, 2000, 32, 150, supply=0.5, rows=9000))


def test_lengths_and_counts_out_of_range():
    check([-5, 1000, 3], [1, 1, 1], [[0, -1], [1, 2], [3, -1]], [9, 8, 7], 50, 16, 5)
    check([0, 0], [2**31 - 1, 1], [[-1, -1], [-1, -1]], [4, 5], 2, 16, 4)
    check([16, 16], [-1, 1], [[3, 9], [4, 9]], [], 0, 16, 4)                 # a stack of no entries: what comes back is dropped
    check([16, 16], [-1, -1], [[3, 9], [4, 9]], [7, 6], 1, 16, 4)
    check([0], [0], [[-1]], [1], -3, 128, 1)


def test_ended_requests_blocks_serve_the_same_step():
    _, want = check([40, 0], [-1, 40], [[5, 6, 7], [-1, -1, -1]], [-1, -1, -1], 0, 16, 40)
    assert want[2] == [-1, 0] and want[6] == [0]


def test_replayed_steps_keep_their_own_books():
    """In place, captured once: every replay is the next step of the same requests."""
    from paper_2504_12285_amd import binding as bl
    dev = "cuda:0"
    B, block, width = 5, 16, 6
    seq, table, free, count = [3, 16, 0, 31, 15], [[0] + [-1] * 5, [1] + [-1] * 5, [-1] * 6, [2, 3] + [-1] * 4, [4] + [-1] * 5], list(range(5, 20)) + [-1] * 10, 15
    t = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    h = bl.KVTables(t(seq), t([0] * B), t(table), t(free), t([count]), block, 12, in_place=True)
    h.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.run()
    r = random.Random(4)
    for step in range(30):
        new = [r.choice([-1, 1, 1, 2, 0]) if step % 3 else 1 for _ in range(B)]
        h.new_len.copy_(t(new))
        g.replay()
        torch.cuda.synchronize()
        seq, count, start, q_start, pos, slots, bad = oracle(seq, new, table, free, count, block, 12)
        assert h.seq_len.tolist() == seq and h.free_count.tolist() == [count] and h.slots.tolist() == slots and h.bad.tolist() == [bad]
        assert h.table.tolist() == table and h.free_list.tolist() == free


@pytest.mark.parametrize("block", [16, 128])
def test_entries_that_name_no_block(block):
    """Neither a negative entry nor one whose slots pass 31 bits becomes the slot of another block (or -1: a row that goes nowhere)."""
    from paper_2504_12285_amd import binding as bl

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda:0")
    entries = [-1, 2**31 // block, 2**31 - 1, -2**31, 2**31 // block - 1, 2**32 // block]
    h = bl.KVTables(t([block - 1] * 6), t([1] * 6), t([[e, 5] for e in entries]), t([0]), t([0]), block, 7)
    h.run()
    assert h.slots.tolist() == [-2, -2, -2, -2, 2**31 - 1, -2, -1] and h.bad.tolist() == [0]


@pytest.mark.parametrize("B, most", [(5, 3), (200, 40), (300, 17), (1100, 6), (4096, 1)])
def test_requests_of_more_tokens_than_the_limit_are_refused(B, most):
    """Against the definition where nothing else refuses: the pool, the table and the batch are large enough for all."""
    from paper_2504_12285_amd import binding as bl

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda:0")
    r, block, width = random.Random(B), 16, 12
    old = [r.randrange(60) for _ in range(B)]
    new = [r.choice([-1, 0, 1, most, most + 1, most + 30]) for _ in range(B)]
    held = [-(-n // block) for n in old]
    ids = list(range(sum(held) + 8 * B))
    r.shuffle(ids)
    table = [[ids.pop() for _ in range(u)] + [-1] * (width - u) for u in held]
    rows, count = sum(max(0, n) for n in new) + 2, len(ids)
    h = bl.KVTables(t(old), t(new), t(table), t(ids + [-1] * sum(held)), t([count]), block, rows, max_new=most)
    h.run()
    good = [0 <= n <= most for n in new]
    want = [-(-(o + n) // block) - u if g else -u if n < 0 else 0 for o, n, u, g in zip(old, new, held, good)]
    start, slots, after, q_start, bad = h.start.tolist(), h.slots.tolist(), h.table.tolist(), h.q_start.tolist(), h.bad.tolist()
    assert start == [o if g else -1 for o, g in zip(old, good)] and bad == [sum(n > most for n in new)]
    assert h.seq_len_out.tolist() == [0 if n < 0 else o + n if g else o for o, n, g in zip(old, new, good)]
    assert h.free_count_out.tolist() == [count - sum(want)]
    at, used = 0, []
    for b in range(B):
        assert q_start[b] == at
        for i in range(max(0, new[b])):
            p = old[b] + i
            assert slots[at + i] == (after[b][p // block] * block + p % block if good[b] else -1)
        at += max(0, new[b])
        assert good[b] or after[b] == table[b]
        if new[b] >= 0:
            used += after[b][:held[b] + max(0, want[b])]
    assert q_start[B] == at and slots[at:] == [-1] * (rows - at) and len(set(used)) == len(used)
