"""Attention of requests that share prefixes, against the definition in 64 bits over whole tables and within the bounds of test_gpu_attn (the
join of the two parts is a few more fp32 steps of its 2^-16)."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_attn import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["int8", "e4m3"]
FAR = 1000000                       # as a hint of the length: nothing is short enough for kernels that read the prefix once a request


class Shared(Batch):
    """Requests (tokens in all, new ones), the blocks of each group's prefix, and the group of each request.  A request's row of the table begins with
    its group's blocks."""

    def __init__(self, reqs, prefix, group, heads, block, kind, seed=0, width=None, **more):
        most = max(prefix)
        super().__init__(reqs, heads, block, kind, seed=seed, spare=sum(prefix) + 3,
                         width=max(width or 1, max(-(-t // block) for t, _ in reqs), max([prefix[g] for g in group if 0 <= g < len(prefix)] or [1])), **more)
        rows, at = [], 0
        for n in prefix:
            rows.append(self.unused[at:at + n] + [-1] * (most - n))
            at += n
        self.shared_table = torch.tensor(rows, dtype=torch.int32, device=DEV)
        self.shared_blocks = torch.tensor(prefix, dtype=torch.int32, device=DEV)
        self.group = torch.tensor(group, dtype=torch.int32, device=DEV)
        for b, g in enumerate(group):
            if 0 <= g < len(prefix):
                self.table[b, :prefix[g]] = self.shared_table[g, :prefix[g]]

    def handle(self, max_q=None, max_len=FAR, **more):
        from paper_2504_12285_amd import binding as bl
        most = max(1, max(n for _, n in self.reqs))
        return bl.KVSharedAttention(bl.KVCache(self.k, self.v, self.ks, self.vs), self.q, self.q_start, self.seq_len, self.table, self.group, self.shared_table,
                                    self.shared_blocks, n_q=self.heads[0], max_q=most if max_q is None else max_q, max_len=max_len, **more)

    def check(self, window=0, **more):
        """The kernels of shared prefixes, and those that the sizes themselves lead to."""
        for far in ({}, dict(max_len=0)):
            h = self.handle(window=window, **dict(far, **more))
            h.out.fill_(math.nan), h.workspace.fill_(255)
            h.run()
            self.compare(h.out, window, h.desc.attn.softmax_scale)


def dealt(prefix, own, block, groups, new=1, lone=()):
    """Requests dealt over the groups in turn: (tokens in all, new ones), group."""
    group = [-1 if b in lone else b % groups for b in range(len(own))]
    return [((prefix[g] * block if g >= 0 else 0) + n, min(n, new)) for g, n in zip(group, own)], group


OWN = [1, 2, 15, 16, 17, 63, 64, 65, 130, 200, 33, 700]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [(20, 5, 128), (4, 4, 64), (16, 1, 128), (6, 2, 64)])
def test_one_token_a_request(kind, block, heads):
    prefix = [5, 1, 22]
    reqs, group = dealt(prefix, OWN, block, 3, lone=(4, 9))
    Shared(reqs, prefix, group, heads, block, kind, seed=block).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads, new", [((20, 5, 128), 4), ((8, 8, 64), 16), ((12, 4, 128), 7), ((16, 2, 64), 40), ((18, 1, 128), 3), ((32, 1, 64), 1)])
def test_several_tokens_a_request(kind, heads, new):
    """Few and many rows of a request, also in one batch; groups of more heads than the kernel of few rows has."""
    prefix = [9, 3]
    reqs, group = dealt(prefix, OWN, 32, 2, new, lone=(2,))
    reqs = [(t, n if b % 3 else 1) for b, (t, n) in enumerate(reqs)]
    Shared(reqs, prefix, group, heads, 32, kind, seed=new).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads, block", [((20, 5, 128), 64), ((8, 2, 64), 16), ((16, 16, 64), 128)])
def test_windows(kind, heads, block):
    """Windows that end inside the prefix, behind it, and that leave nothing of it."""
    prefix = [13, 4]
    for window in (1, 50, 129, 400, 5000):
        reqs, group = dealt(prefix, OWN, block, 2, 5)
        Shared(reqs, prefix, group, heads, block, kind, seed=window).check(window=window)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", [(20, 5, 128), (8, 2, 64)])
def test_queries_inside_the_prefix(kind, heads):
    """Requests shorter than their group's prefix, ended ones, queries on both sides of its end, and more of them than tokens."""
    block, prefix = 32, [6, 3]
    reqs = [(100, 3), (192, 1), (193, 1), (200, 20), (0, 0), (50, 50), (3, 3), (96, 96), (97, 40), (1, 1), (40, 60), (0, 2)]
    Shared(reqs, prefix, [b % 2 for b in range(12)], heads, block, kind).check_finite(kind)


def _check_finite(self, kind):
    h = self.handle()
    h.out.fill_(math.nan), h.workspace.fill_(255)
    h.run()
    out = h.out.view(-1, *h.out.shape[1:])
    # the definition of requests with more queries than tokens: the first of them see nothing and are zeros
    keep = self.reqs, self.starts
    for b, (t, n) in enumerate(self.reqs):
        if n > t:
            assert bool((out[self.starts[b]:self.starts[b] + n - t] == 0).all())
    self.reqs = [(t, min(t, n)) for t, n in self.reqs]
    self.starts = [s + max(0, n - t) for s, (t, n) in zip(self.starts, keep[0])]
    self.compare(h.out)


Shared.check_finite = _check_finite


@pytest.mark.parametrize("kind", KINDS)
def test_many_requests_and_groups(kind):
    """More than 64 of each, a group whose rows fill several tiles, groups without requests or blocks, requests of groups that are none."""
    B = 150
    prefix = [70] + [(3 * g) % 11 for g in range(1, 90)]
    group = [0 if b % 2 else (b * 7) % 95 - 2 for b in range(B)]
    own = [(b * 37) % 90 + 1 for b in range(B)]
    reqs = [((prefix[g] * 16 if 0 <= g < 90 else 0) + n, 1 if b % 5 else min(n, 3)) for b, (g, n) in enumerate(zip(group, own))]
    Shared(reqs, prefix, group, (8, 2, 64), 16, kind).check()


@pytest.mark.parametrize("new", [1, 3, 30, 70])
@pytest.mark.parametrize("B, groups", [(300, 4), (40, 270), (257, 257)])
def test_more_requests_or_groups_than_threads(B, groups, new):
    """One token each, a few, and requests of many rows among them that are of their groups (30 of 2 heads) or apart (70)."""
    prefix = [(5 * g) % 7 for g in range(groups)]
    reqs, group = dealt(prefix, [(b * 37) % 50 + 1 + (new if b % 60 == 7 else 0) for b in range(B)], 16, groups)
    reqs = [(t, min(t, new) if b % 60 == 7 else 1 + b % min(new, 2)) for b, (t, n) in enumerate(reqs)]
    reqs = [(max(t, n), n) for t, n in reqs]
    Shared(reqs, prefix, group, (4, 2, 64), 16, "int8", seed=new).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads, counts", [((20, 5, 128), (1, 4, 5, 20, 31)), ((20, 5, 128), (1, 4, 5, 31, 32, 40, 200)), ((8, 8, 64), (16, 17, 127, 1)), ((8, 8, 64), (16, 17, 127, 128, 1, 260)),
                                           ((34, 2, 64), (1, 2, 7)), ((34, 2, 64), (1, 8, 30))])
def test_many_and_few_rows_in_one_batch(kind, heads, counts):
    """Numbers of rows on both sides of what a few, a group's and a prompt's are."""
    prefix = [20, 6]
    reqs = [(prefix[b % 2] * 32 + n + 10 * b, n) for b, n in enumerate(counts * 2)]
    Shared(reqs, prefix, [b % 2 if b != 3 else -1 for b in range(len(reqs))], heads, 32, kind, seed=len(counts)).check()
    Shared(reqs, prefix, [b % 2 for b in range(len(reqs))], heads, 32, kind, seed=len(counts)).check(window=300, max_own=1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads, block", [((20, 5, 128), 64), ((32, 8, 64), 128)])
def test_long_prefixes(kind, heads, block):
    n = 5000 // block
    reqs, group = dealt([n], [100, 3, 900, 40, 1], block, 1)
    Shared(reqs, [n], group, heads, block, kind).check(max_len=6000, max_own=900)


@pytest.mark.parametrize("kind", KINDS)
def test_hints_and_a_wide_table_change_nothing_that_counts(kind):
    prefix = [9, 3]
    for more in (dict(max_len=1), dict(max_len=10**6), dict(max_own=1), dict(max_own=10**6)):
        reqs, group = dealt(prefix, OWN, 32, 2, 3)
        Shared(reqs, prefix, group, (8, 2, 128), 32, kind, width=900).check(**more)


def test_entries_that_name_no_block():
    """Holes in a group's row and in a request's: their tokens are not seen."""
    prefix = [8, 2]
    reqs, group = dealt(prefix, OWN, 32, 2, 2)
    b = Shared(reqs, prefix, group, (8, 2, 64), 32, "int8")
    b.shared_table[0, 3], b.shared_table[0, 7], b.shared_table[1, 1] = -1, 10**9, b.k.shape[0]
    for i, g in enumerate(group):
        b.table[i, :prefix[g]] = b.shared_table[g, :prefix[g]]
    b.table[11, prefix[1] + 2] = -3
    b.check()


def test_counts_outside_the_table_are_the_nearer_end():
    prefix = [4, 4, 4]
    reqs, group = dealt([4, 4, 0], OWN, 32, 3)
    b = Shared(reqs, [4, 4, 0], group, (8, 2, 64), 32, "e4m3")
    b.shared_blocks.copy_(torch.tensor([10**9, 4, -5], dtype=torch.int32, device=DEV))
    assert b.shared_table.shape[1] == prefix[0]
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [1, 6])
def test_memory_that_nobody_has_written(kind, new):
    """NaN codes and scales wherever no token of the batch lies: behind the last tokens, in blocks of nobody, in front of the windows."""
    prefix, block = [9, 3], 16
    for window in (0, 70):
        reqs, group = dealt(prefix, OWN, block, 2, new)
        b = Shared(reqs, prefix, group, (8, 2, 128), block, kind)
        clean = [t.clone() for t in (b.k, b.v, b.ks, b.vs)]
        if kind == "e4m3":
            k, v = b.k.view(torch.uint8), b.v.view(torch.uint8)
            own = set()
            for r, (t, n) in enumerate(reqs):
                low = max(0, t - n + 1 - window) if window else 0
                for p in range(-(-t // block)):
                    page = int(b.table[r, p])
                    if p * block + block > low:
                        own.add(page)
                    if t - p * block < block:
                        k[page, :, t - p * block:] = 0x7f
                        v[page, :, :, t - p * block:] = 0x7f
            for page in set(range(b.k.shape[0])) - own:
                k[page], v[page] = 0x7f, 0x7f
                b.ks[page] = b.vs[page] = math.nan
        h = b.handle(window=window)
        h.out.fill_(math.nan), h.workspace.fill_(255)
        h.run()
        b.k, b.v, b.ks, b.vs = clean                          # (the definition sums over all tokens of a request, with weights of 0)
        b.compare(h.out, window)


def test_rows_of_no_request_and_requests_of_too_many_queries():
    prefix = [4]
    reqs, group = dealt(prefix, [40, 3, 60], 32, 1)
    b = Shared([(reqs[0][0], 1), (reqs[1][0], 1), (reqs[2][0], 30)], prefix, group, (8, 2, 64), 32, "int8")
    h = b.handle(max_q=1)
    h.out.fill_(7.0)
    h.run()
    assert bool(h.out[2:].isnan().all())
    b.reqs = [b.reqs[0], b.reqs[1], (reqs[2][0], 0)]
    b.compare(h.out)
    # rows in front of the first request and behind the last stay as they are
    b = Shared([(200, 2), (140, 1)], prefix, [0, 0], (8, 2, 64), 32, "int8")
    q = torch.cat([b.q, b.q, b.q])
    b.q, b.starts = q, [4, 6, 7]
    b.q_start.copy_(torch.tensor(b.starts, dtype=torch.int32, device=DEV))
    h = b.handle()
    h.out.fill_(7.0)
    h.run()
    assert bool((h.out[:4] == 7).all()) and bool((h.out[7:] == 7).all())
    b.compare(h.out)


def test_a_number_that_is_none_in_q_spoils_its_row_and_head():
    prefix = [6]
    reqs, group = dealt(prefix, OWN, 32, 1, 2)
    b = Shared(reqs, prefix, group, (8, 2, 64), 32, "int8")
    want = b.handle()
    want.run()
    for odd in (math.nan, math.inf):
        b.q[3, 5, 7] = odd
        h = b.handle()
        h.run()
        x, y = h.out.view(-1, 8, 64), want.out.view(-1, 8, 64)
        assert bool(x[3, 5].isnan().all())
        x[3, 5] = y[3, 5]
        assert torch.equal(x, y)


@pytest.mark.parametrize("kind", KINDS)
def test_blocks_rows_and_tables_that_lie_apart(kind):
    prefix = [5, 2]
    reqs, group = dealt(prefix, OWN, 64, 2, 3)
    b = Shared(reqs, prefix, group, (8, 2, 64), 64, kind, strided=True)
    wide = torch.full((2, 11), 10**9, dtype=torch.int32, device=DEV)
    wide[:, :5] = b.shared_table
    b.shared_table = wide[:, :5]
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_the_same_bits_every_time(kind):
    prefix = [40, 7]
    reqs, group = dealt(prefix, OWN, 32, 2, 6)
    b = Shared(reqs, prefix, group, (8, 2, 128), 32, kind)
    h = b.handle()
    h.run()
    want = h.out.clone()
    for _ in range(3):
        h.out.fill_(math.nan), h.workspace.fill_(255)
        h.run()
        assert torch.equal(h.out, want)


def test_captured_and_on_another_stream():
    """Replays follow the lengths, the groups and the queries of their time."""
    prefix = [5, 12]
    reqs, group = dealt(prefix, [40, 9, 100, 30], 32, 2)
    b = Shared(reqs, prefix, group, (8, 2, 64), 32, "int8", width=20)
    h = b.handle(max_own=200)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        h.run()
    s.synchronize()
    b.compare(h.out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.run()
    for step in range(4):
        lens = [reqs[0][0] - 9 * step, reqs[1][0] - step, 1 + step, reqs[3][0]]
        b.seq_len.copy_(torch.tensor(lens, dtype=torch.int32, device=DEV))
        b.q.copy_(torch.randn_like(b.q))
        if step == 3:
            b.shared_blocks.copy_(torch.tensor([4, 12], dtype=torch.int32, device=DEV))
        g.replay()
        torch.cuda.synchronize()
        b.reqs = [(t, 1) for t in lens]
        b.compare(h.out)
        eager = b.handle(max_own=200)
        eager.run()
        assert torch.equal(eager.out, h.out)


@pytest.mark.parametrize("new", [1, 20])
def test_without_groups_it_is_the_attention_of_its_tables(new):
    reqs = [(t + 20, min(t, new)) for t in OWN]
    b = Shared(reqs, [3], [-1, 1, 5, -9] * 3, (8, 2, 64), 32, "int8")
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block, heads", [(16, (8, 2, 128)), (64, (20, 5, 128)), (128, (8, 2, 64))])
@pytest.mark.parametrize("new", [1, 6, 40])
def test_scales_and_codes_of_nobody_s_blocks(kind, block, heads, new):
    """Blocks of no request have NaN for scales and the lowest codes, block 0 among them, whose scales stand in where a tile has no block; so have places
    behind the last tokens the lowest codes.  (e4m3: 0xff, a NaN.)"""
    prefix = [9, 3] if block < 64 else [3, 1]
    low = -128 if kind == "int8" else 0xff
    for window, far in ((0, FAR), (70, FAR), (0, 0), (70, 0)):
        reqs, group = dealt(prefix, OWN, block, 2, new, lone=(3,))
        b = Shared(reqs, prefix, group, heads, block, kind, seed=new)
        clean = [t.clone() for t in (b.k, b.v, b.ks, b.vs)]
        k, v = (t.view(torch.int8 if kind == "int8" else torch.uint8) for t in (b.k, b.v))
        seen = set()
        for r, (t, n) in enumerate(reqs):
            first = max(0, t - n + 1 - window) if window else 0
            for p in range(-(-t // block)):
                page = int(b.table[r, p])
                if p * block + block > first:
                    seen.add(page)
                if t - p * block < block:
                    k[page, :, t - p * block:], v[page, :, :, t - p * block:] = low, low
        nobody = set(range(k.shape[0])) - seen
        if 0 in seen:                                         # (another block takes its place)
            other = max(nobody)
            for x in (k, v, b.ks, b.vs, *(x.view(torch.uint8) if x.element_size() == 1 else x for x in clean)):
                x[other] = x[0].clone()
            for x in (b.table, b.shared_table):
                x[x == 0] = other
            nobody = nobody - {other} | {0}
        for page in nobody:
            k[page], v[page] = low, low
            b.ks[page] = b.vs[page] = math.nan
        h = b.handle(window=window, max_len=far)
        h.out.fill_(math.nan), h.workspace.fill_(255)
        h.run()
        b.k, b.v, b.ks, b.vs = clean
        b.compare(h.out, window)
