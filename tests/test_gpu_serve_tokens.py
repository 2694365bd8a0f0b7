"""From token ids to token ids: the vocabulary's lookup and head around layers with norms of Q and K, and requests that share a prefix."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_f8 import check  # noqa: E402
from test_gpu_serve import check_attention  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WORDS = 1000


@pytest.fixture(scope="module")
def model():
    from paper_2504_12285_amd import binding as bl
    from paper_2504_12285_amd import serve
    weights, gains = serve.random_layers(2, torch.device(DEV), seed=3)
    g = torch.Generator(device=DEV).manual_seed(4)
    qk = [tuple(1 + 0.2 * torch.randn(128, generator=g, device=DEV) for _ in range(2)) for _ in range(2)]
    return weights, gains, qk, bl.F8Matrix.quantise(torch.randn(WORDS, 2560, generator=g, device=DEV) * 0.02)


def served(model, requests, rows, groups=0, kind=0, n_blocks=30, **more):
    from paper_2504_12285_amd import serve
    weights, gains, qk, words = model
    layers = serve.CachedLayers(weights, gains, requests, rows, max_blocks=8, n_blocks=n_blocks, device=torch.device(DEV), block=32, kind=kind, qk_gains=qk, groups=groups, **more)
    return layers, serve.TokenLayers(layers, words, multiplier=50.0)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def some_ids(n, rows, seed):
    ids = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    ids[:n] = torch.randint(0, WORDS, (n,), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV, dtype=torch.int32)
    return ids


def check_step(layers, tokens, lens, new, kind):
    """Lengths, the last layer's attention over its cache, the logits of the hidden states, and the ids of the largest."""
    torch.cuda.synchronize()
    assert layers.seq_len.tolist() == lens and int(layers.tables.bad) == 0 and int(layers.bad) == 0 and int(tokens.bad) == 0
    check_attention(layers, lens, new, kind)
    check(tokens.head, tokens.head.matrix.codes, tokens.head.matrix.scale, tokens.hidden, norm=True, eps=float(torch.tensor(1e-5)))
    for b, n in enumerate(new):
        if n:
            assert torch.equal(tokens.hidden[b], layers.buffers.x_next[int(layers.tables.q_start[b + 1]) - 1])
            assert int(tokens.next[b]) == int(torch.argmax(tokens.logits[b]))
        else:
            assert int(tokens.next[b]) == -1


@pytest.mark.parametrize("kind", [0, 1])
def test_prompts_and_decode_steps(model, kind):
    layers, tokens = served(model, 3, 90, kind=kind)
    lens = [0, 0, 0]
    for i, new in enumerate(([40, 33, 1], [1, 0, 1], [1, 1, 60])):
        tokens.step(some_ids(sum(new), 90, i), ints(new))
        lens = [a + b for a, b in zip(lens, new)]
        check_step(layers, tokens, lens, new, kind)


@pytest.mark.parametrize("kind", [0, 1])
def test_requests_behind_a_prompt(model, kind):
    """A prompt of 70 tokens, two blocks of which three others begin behind; the same tokens in a row of their own leave the same first layer's cache."""
    layers, tokens = served(model, 4, 100, groups=2, kind=kind)
    prompt = some_ids(70, 100, 7)
    tokens.step(prompt, ints([70, 0, 0, 0]))
    layers.share(1, 0, 2)
    for place in (1, 2, 3):
        layers.join(place, 1)
    lens = [70, 64, 64, 64]
    asked = [5, 20, 1]
    for i, new in enumerate(([1, *asked], [1, 1, 1, 1], [0, 3, 1, 0])):
        ids = some_ids(sum(new), 100, 10 + i)
        if i == 0:
            question = ids[1:6].clone()
        tokens.step(ids, ints(new))
        lens = [a + b for a, b in zip(lens, new)]
        check_step(layers, tokens, lens, new, kind)
    used = 3 + 3 * 1                                          # the prompt's three blocks, and one for each of the others
    assert int(layers.free_count) == 30 - used and layers.group.tolist() == [1, 1, 1, 1] and layers.held.tolist() == [2, 2, 2, 2]
    alone, alone_tokens = served(model, 1, 100, kind=kind)
    ids = some_ids(0, 100, 0)
    ids[:64], ids[64:69] = prompt[:64], question
    alone_tokens.step(ids, ints([69]))
    a, b = layers.caches[0], alone.caches[0]
    for p in range(2):
        i, j = int(layers.table[1, p]), int(alone.table[0, p])
        for name in ("k", "v", "k_scale", "v_scale"):
            x, y = (getattr(c, name) for c in (a, b))
            assert torch.equal(x[i].view(torch.uint8) if x.element_size() == 1 else x[i], y[j].view(torch.uint8) if y.element_size() == 1 else y[j])
    # they end one after the other; the prefix outlives its own request, until it is given back
    tokens.step(some_ids(2, 100, 20), ints([-1, 1, -1, 1]))
    lens = [0, lens[1] + 1, 0, lens[3] + 1]
    check_step(layers, tokens, lens, [0, 1, 0, 1], kind)
    assert layers.group.tolist() == [-1, 1, -1, 1] and layers.held.tolist() == [0, 2, 0, 2] and int(layers.free_count) == 30 - 4
    layers.join(2, 1)
    tokens.step(some_ids(36, 100, 21), ints([33, 1, 2, 0]))   # a prompt of its own in the first place, a new one behind the prefix in the third
    lens = [33, lens[1] + 1, 66, lens[3]]
    check_step(layers, tokens, lens, [33, 1, 2, 0], kind)
    tokens.step(some_ids(0, 100, 0), ints([-1, -1, -1, -1]))
    assert int(layers.free_count) == 28
    layers.release(1)
    with pytest.raises(ValueError):
        layers.join(0, 1)
    assert int(layers.free_count) == 30 and sorted(layers.free_list.tolist()) == list(range(30)) and layers.shared_blocks.tolist() == [0, 0]
    tokens.step(some_ids(40, 100, 22), ints([0, 40, 0, 0]))
    layers.share(1, 1, 1)


def test_refusals(model):
    layers, tokens = served(model, 2, 10, groups=1)
    for blocks in (0, 9):
        with pytest.raises(ValueError):
            layers.share(0, 0, blocks)
    with pytest.raises(ValueError):
        tokens.step(ints([1, 2]), ints([1, 1]))
    tokens.step(ints([3, WORDS, -1, -1, -1, -1, -1, -1, -1, -1]), ints([1, 1]))
    assert int(tokens.bad) == 1


def test_groups_are_what_they_are_made_for(model):
    """A prefix is of whole blocks of a request that is in no group; places are joined empty, to a group with a prefix, which is given back when nobody is in it."""
    layers, tokens = served(model, 3, 80, groups=2)
    tokens.step(some_ids(75, 80, 5), ints([70, 5, 0]))
    for group, place, blocks in ((0, 0, 3), (0, 1, 1), (0, 2, 1)):
        with pytest.raises(ValueError):
            layers.share(group, place, blocks)
    layers.share(0, 0, 2)
    for call in (lambda: layers.share(0, 1, 1), lambda: layers.share(1, 0, 1), lambda: layers.join(1, 0), lambda: layers.join(2, 1), lambda: layers.release(0)):
        with pytest.raises(ValueError):
            call()
    layers.join(2, 0)
    assert layers.seq_len.tolist() == [70, 5, 64] and layers.group.tolist() == [0, -1, 0] and layers.held.tolist() == [2, 0, 2]


def test_captured_generation_is_the_eager_one(model):
    """Five requests behind a prompt feed their own ids back, eagerly and from a graph that is replayed between other work."""
    both = []
    for _ in range(2):
        layers, tokens = served(model, 5, 64, groups=1)
        tokens.step(some_ids(64, 64, 3), ints([64, 0, 0, 0, 0]))
        step, ids = served(model, 5, 5, groups=1, max_new=1)
        for name in ("seq_len", "table", "free_list", "free_count"):
            getattr(step, name).copy_(getattr(layers, name))
        for a, b in zip(step.caches, layers.caches):
            for name in ("k", "v", "k_scale", "v_scale"):
                getattr(a, name).copy_(getattr(b, name))
        step.share(0, 0, 2)
        for place in range(1, 5):
            step.join(place, 0)
        ids.step(ints([1, 2, 3, 4, 5]), ints([1] * 5))
        both.append((step, ids))
    (step, eager), (_, other) = both
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    other.ids.copy_(other.next)
    with torch.cuda.graph(graph):
        other.ids.copy_(other.run())
    torch.cuda.synchronize()
    ids = eager.next.clone()
    for _ in range(12):
        ids = eager.step(ids, ints([1] * 5)).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(other.ids, ids) and torch.equal(other.logits, eager.logits)
    check_attention(step, [64 + 13] * 5, [1] * 5, 0)
