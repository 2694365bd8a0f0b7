"""Block tables whose requests hold blocks of another's: the definition of test_gpu_kv_tables, with rows of ended requests that begin behind what they hold."""
import random

import pytest

torch = pytest.importorskip("torch")
from test_gpu_kv_tables import batch, oracle  # noqa: E402

pytestmark = pytest.mark.gpu


def check(seq_len, new_len, table, free, count, block, rows, held, in_place=False):
    from paper_2504_12285_amd import binding as bl
    dev, B = "cuda:0", len(seq_len)

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)
    tab, lst = t(table), t(free)
    h = bl.KVTables(t(seq_len), t(new_len), tab, lst, t([count]), block, rows, in_place=in_place, held=t(held))
    h.run()
    got = [x.tolist() for x in (h.seq_len_out, h.free_count_out, h.start, h.q_start, h.positions, h.slots, h.bad)]
    width = len(table[0])
    keep = [max(0, min(n, width)) if new_len[b] < 0 else 0 for b, n in enumerate(held)]
    shifted = [row[k:] + [-5] * k for row, k in zip(table, keep)]
    lens = [max(0, min(n, width * block) - k * block) if k else n for n, k in zip(seq_len, keep)]
    free = list(free)
    want = oracle(lens, new_len, shifted, free, count, block, rows)
    want = [want[0], [want[1]], *want[2:6], [want[6]]]
    for name, g, w in zip(("seq_len", "free_count", "start", "q_start", "positions", "slots", "bad"), got, want):
        assert g == w, name
    assert tab.tolist() == [table[b] if new_len[b] < 0 else shifted[b] for b in range(B)]
    assert lst.tolist() == free


@pytest.mark.parametrize("B", [1, 7, 64, 65, 300, 1500])
@pytest.mark.parametrize("in_place", [False, True])
def test_steps(B, in_place):
    for seed in range(4):
        args = batch(seed, B, 400, 16, 30, supply=(1.0, 0.6, 1.0, 0.3)[seed], ends=0.4)
        r = random.Random(seed)
        held = [r.choice([0, 0, 1, 2, 5, 30, 1000, -3]) for _ in range(B)]
        check(*args, held=held, in_place=in_place)


def test_a_stack_that_is_full_and_a_limit():
    """Only what is given back can be dropped; max_new refuses as without held blocks."""
    table = [[0, 1, 2, 3], [0, 1, 4, 5], [0, 1, 6, 7]]
    check([64, 60, 50], [-1, -1, -1], table, [-1] * 3, 0, 16, 4, [2, 2, 2])
    from paper_2504_12285_amd import binding as bl

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda:0")
    h = bl.KVTables(t([32, 32, 32]), t([1, 3, 2]), t(table), t([9, 10, 11]), t([3]), 16, 8, max_new=2, held=t([2, 2, 2]))
    h.run()
    assert h.bad.item() == 1 and h.start.tolist() == [32, -1, 32] and h.seq_len_out.tolist() == [33, 32, 34] and h.q_start.tolist() == [0, 1, 4, 6]
    assert h.table.tolist() == [[0, 1, 11, 3], [0, 1, 4, 5], [0, 1, 10, 7]] and h.free_count_out.item() == 1
    assert h.positions.tolist()[:1] + h.positions.tolist()[4:6] == [32, 32, 33] and h.slots.tolist()[:6] == [176, -1, -1, -1, 160, 161]


def test_requests_that_share_a_prefix_come_and_go():
    """A prompt fills two blocks; three requests take its row, answer and end: the pool has again what it had, and the prompt's blocks were never in it."""
    from paper_2504_12285_amd import binding as bl
    dev = "cuda:0"

    def t(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)
    seq, new, held, table = t([0, 0, 0, 0]), t([32, 0, 0, 0]), t([0, 0, 0, 0]), t([[-1] * 6] * 4)
    free, count = t(list(range(12))), t([12])
    h = bl.KVTables(seq, new, table, free, count, 16, 40, in_place=True, held=held)
    h.run()
    assert count.item() == 10
    prefix = table[0, :2].tolist()
    for turn in range(3):
        table[1:, :2] = table[0, :2]
        seq[1:], held[1:] = 32, 2
        for step in range(20):
            new.copy_(t([0, 1, 1, 1]))
            h.run()
            assert h.positions[:3].tolist() == [32 + step] * 3 and h.bad.item() == 0
        assert count.item() == 10 - 6
        own = table[1:, 2:4].flatten().tolist()
        assert len(set(own)) == 6 and not set(own) & set(prefix)
        new.copy_(t([0, -1, -1, -1]))
        h.run()
        assert count.item() == 10 and not set(free[:10].tolist()) & set(prefix) and len(set(free[:10].tolist())) == 10
    new.copy_(t([-1, 0, 0, 0])), held.zero_()
    h.run()
    assert count.item() == 12 and sorted(free.tolist()) == list(range(12))
