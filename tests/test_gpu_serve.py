"""Requests served through layers with their cache: the step's attention against the definition over what the caches hold,
its tables against the lengths, and captured steps against eager ones."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_attn import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def model():
    from paper_2504_12285_amd import serve
    return serve.random_layers(2, torch.device(DEV), seed=3)


def served(model, requests, rows, kind=0, **more):
    from paper_2504_12285_amd import serve
    return serve.CachedLayers(*model, requests, rows, max_blocks=8, n_blocks=30, device=torch.device(DEV), block=32, kind=kind, **more)


def check_attention(layers, lens, new, kind):
    """Each layer's attention is the last one's buffers: the last layer's, against its cache."""
    b = object.__new__(Batch)
    c = layers.caches[-1]
    b.reqs, b.heads, b.block, b.kind = list(zip(lens, new)), (20, 5, 128), 32, ("int8", "e4m3")[kind]
    b.k, b.v, b.ks, b.vs, b.table, b.q = c.k, c.v, c.k_scale, c.v_scale, layers.table, layers.attend[-1].q
    b.starts = layers.tables.q_start.tolist()
    b.compare(layers.attend[-1].out)


@pytest.mark.parametrize("kind", [0, 1])
def test_prompts_decode_steps_and_ends(model, kind):
    layers = served(model, 3, 90, kind)
    g = torch.Generator(device=DEV).manual_seed(kind)
    lens = [0, 0, 0]
    for new in ([40, 33, 1], [1, 1, 1], [1, -1, 60], [1, 70, 1], [0, 1, 1], [1, 1, 0]):
        y = layers.step(torch.randn(90, 2560, generator=g, device=DEV), torch.tensor(new, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        lens = [0 if n < 0 else t + n for t, n in zip(lens, new)]
        assert layers.seq_len.tolist() == lens and int(layers.tables.bad) == 0 and int(layers.bad) == 0
        used = sum(-(-t // 32) for t in lens)
        assert int(layers.free_count) == 30 - used
        held = [layers.table[b, :-(-t // 32)].tolist() for b, t in enumerate(lens)]
        assert len({x for h in held for x in h}) == used and not {x for h in held for x in h} & set(layers.free_list[:30 - used].tolist())
        assert torch.isfinite(y[:sum(max(n, 0) for n in new)]).all()
        check_attention(layers, lens, [max(n, 0) for n in new], kind)


@pytest.mark.parametrize("few_rows, new", [(1, (1, 0)), (10, (6, 4))])
def test_every_route_of_the_products_gives_the_same_rows(model, few_rows, new):
    """The same tokens through steps of few rows (products with their producers inside, or the grouped product) and of many (the
    prefill product): the arithmetic is the same bit for bit up to the attention, so the first layer's codes and scales are too."""
    few, many = served(model, 2, few_rows), served(model, 2, 100)
    g = torch.Generator(device=DEV).manual_seed(9)
    x = torch.randn(few_rows, 2560, generator=g, device=DEV)
    n = torch.tensor(new, dtype=torch.int32, device=DEV)
    few.step(x, n)
    many.step(torch.cat([x, torch.zeros(100 - few_rows, 2560, device=DEV)]), n)
    a, b = few.caches[0], many.caches[0]
    for name in ("k_scale", "v_scale"):
        for r in range(2):
            assert new[r] == 0 or torch.equal(getattr(a, name)[int(few.table[r, 0])], getattr(b, name)[int(many.table[r, 0])])
    for r in range(2):
        if new[r] == 0:
            continue
        i, j = int(few.table[r, 0]), int(many.table[r, 0])
        assert torch.equal(a.k[i, :, :new[r]], b.k[j, :, :new[r]]) and torch.equal(a.v[i, :, :, :new[r]], b.v[j, :, :, :new[r]])
    check_attention(few, list(new), list(new), 0)
    check_attention(many, list(new), list(new), 0)


def test_captured_steps_are_the_eager_ones(model):
    eager, captured = served(model, 4, 4, max_new=1), served(model, 4, 4, max_new=1)
    g = torch.Generator(device=DEV).manual_seed(2)
    ones = torch.ones(4, dtype=torch.int32, device=DEV)
    x = torch.randn(4, 2560, generator=g, device=DEV)
    for layers in (eager, captured):
        layers.step(x, ones)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for step in range(40):                               # over a block's end
        x = torch.randn(4, 2560, generator=g, device=DEV)
        new = ones if step != 20 else torch.tensor([1, -1, 1, 1], dtype=torch.int32, device=DEV)
        y = eager.step(x, new)
        captured.x.copy_(x)
        captured.new_len.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        rows = 4 if step != 20 else 3
        assert torch.equal(captured.buffers.x_next[:rows], y[:rows]), step
        assert torch.equal(captured.seq_len, eager.seq_len) and torch.equal(captured.table, eager.table)


def test_a_pool_that_runs_dry_refuses(model):
    layers = served(model, 3, 700)
    new = torch.tensor([250, 250, 200], dtype=torch.int32, device=DEV)
    layers.step(torch.randn(700, 2560, device=DEV), new)
    assert layers.seq_len.tolist() == [250, 250, 200] and int(layers.tables.bad) == 0 and int(layers.free_count) == 30 - 23
    layers.step(torch.randn(700, 2560, device=DEV), torch.tensor([7, -1, 50], dtype=torch.int32, device=DEV))
    assert layers.seq_len.tolist() == [250, 0, 250]        # the first would need a ninth block
    assert layers.tables.start.tolist() == [-1, -1, 200] and int(layers.tables.bad) == 1
    assert layers.tables.slots[:7].eq(-1).all() and int(layers.bad) == 0


def test_a_request_of_more_tokens_than_max_new_is_refused(model):
    """Five tokens where four are the most: nothing of them reaches the caches or the lengths, and the others' rows are those of a step
    without them."""
    layers, alone = served(model, 3, 12, max_new=4), served(model, 3, 12, max_new=4)
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn(12, 2560, generator=g, device=DEV)
    y = layers.step(x, torch.tensor([3, 5, 4], dtype=torch.int32, device=DEV)).clone()
    assert layers.seq_len.tolist() == [3, 0, 4] and layers.tables.start.tolist() == [0, -1, 0]
    assert int(layers.tables.bad) == 1 and int(layers.bad) == 0 and int(layers.free_count) == 28
    rest = torch.cat([x[:3], x[8:], x[:5]])
    z = alone.step(rest, torch.tensor([3, 0, 4], dtype=torch.int32, device=DEV))
    assert int(alone.tables.bad) == 0
    assert torch.equal(y[:3], z[:3]) and torch.equal(y[8:12], z[3:7])


def test_rows_of_refused_requests_and_padding_are_zeros(model):
    """Too many tokens, and too little of the pool; a captured step too."""
    layers = served(model, 3, 700, max_new=300)
    x = torch.randn(700, 2560, generator=torch.Generator(device=DEV).manual_seed(8), device=DEV)
    y = layers.step(x, torch.tensor([250, 301, 100], dtype=torch.int32, device=DEV))
    assert layers.tables.start.tolist() == [0, -1, 0]
    assert bool(y[:250].abs().amax(1).gt(0).all()) and not y[250:551].any() and bool(y[551:651].abs().amax(1).gt(0).all()) and not y[651:].any()
    y = layers.step(x, torch.tensor([7, 200, 30], dtype=torch.int32, device=DEV))
    assert layers.tables.start.tolist() == [-1, 0, 100]          # the first would need a ninth block
    assert not y[:7].any() and bool(y[7:237].abs().amax(1).gt(0).all()) and not y[237:].any()
    small = served(model, 2, 3, max_new=1)
    small.step(x[:3], torch.tensor([1, 1], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small.run()
    for new, zeros in (([1, 1], [2]), ([2, 1], [0, 1]), ([0, 1], [1, 2]), ([1, 2], [1, 2])):
        small.new_len.copy_(torch.tensor(new, dtype=torch.int32, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert [i for i in range(3) if not small.buffers.x_next[i].any()] == zeros
