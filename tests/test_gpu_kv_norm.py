"""The append with norms of Q and K against its definition in numpy: the mean square in 64 bits, every other step one rounded fp32 operation,
so codes, scales and queries are compared bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_kv_append import encode, oracle  # noqa: E402

pytestmark = pytest.mark.gpu
F = np.float32


def normed(x, gain, eps):
    """x [T][heads][D]"""
    with np.errstate(all="ignore"):
        r = (1.0 / np.sqrt((x.astype(np.float64) ** 2).sum(-1, keepdims=True) / x.shape[-1] + np.float64(F(eps)))).astype(F)
        y = (x * r).astype(F)
        return y if gain is None else (y * gain).astype(F)


def run(kind, source, heads, block, runs, seed=0, rotate=True, gains=(True, True), eps=1e-6, extra=(), spoil=None, strided=False, captured=False):
    from paper_2504_12285_amd import binding as bl
    n_q, H, D = heads
    r = np.random.RandomState(seed)
    T = sum(n for _, n in runs)
    N = max(s // block for s, _ in runs) + 4
    slots = np.concatenate([np.arange(s, s + n) for s, n in runs]).astype(np.int32)
    positions = np.concatenate([np.arange(n) + r.randint(0, 50) for _, n in runs]).astype(np.int32)
    for row, slot, pos in extra:
        slots[row], positions[row] = slot, pos
    x = r.randn(T, n_q + 2 * H, D).astype(F) * np.exp(2 * r.randn(T, n_q + 2 * H, 1)).astype(F)
    x[0, 0] = 0                                              # a head of zeros
    if spoil:
        spoil(x)
    xt = torch.from_numpy(x.reshape(T, -1)).to(torch.float32 if source == "f32" else torch.bfloat16)
    x = xt.float().numpy().reshape(x.shape).copy()
    angle = r.rand(400, D // 2) * 6.3
    cos, sin = np.cos(angle).astype(F), np.sin(angle).astype(F)
    k, v = (encode(r.randn(N, H, *s).astype(F) * F(40), kind) for s in ((block, D), (D, block)))
    ks, vs = ((np.exp(r.randn(N, H)) * 0.02).astype(F) for _ in range(2))
    qg, kg = ((1 + 0.3 * r.randn(D)).astype(F) if g else None for g in gains)
    dev = "cuda:0"
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn

    def t(a):
        return None if a is None else torch.from_numpy(a).to(dev)
    tk, tv, tks, tvs = t(k).view(dtype), t(v).view(dtype), t(ks), t(vs)
    qkv = xt.to(dev)
    if strided:
        wide = torch.zeros((T, xt.shape[1] + 24), dtype=xt.dtype, device=dev)
        wide[:, :xt.shape[1]] = qkv
        qkv = wide[:, :xt.shape[1]]
    bad = torch.zeros(1, dtype=torch.int32, device=dev)
    h = bl.KVNormAppend(bl.KVCache(tk, tv, tks, tvs), qkv, n_q, t(slots), t(positions), t(cos) if rotate else None, t(sin) if rotate else None, bad=bad,
                        q_gain=t(qg), k_gain=t(kg), eps=eps)
    if captured:
        keep = [a.clone() for a in (tk.view(torch.uint8), tv.view(torch.uint8), tks, tvs)]
        h.run()                                              # (nothing is compiled or resolved inside the capture)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.run()
        for _ in range(3):
            for a, b in zip((tk.view(torch.uint8), tv.view(torch.uint8), tks, tvs), keep):
                a.copy_(b)
            bad.zero_()
            graph.replay()
            torch.cuda.synchronize()
    else:
        h.run()
    y = x.copy()
    y[:, :n_q], y[:, n_q:n_q + H] = normed(x[:, :n_q], qg, eps), normed(x[:, n_q:n_q + H], kg, eps)
    q, n_bad = oracle((k, v, ks, vs), y, n_q, slots, positions, cos if rotate else None, sin, kind)
    assert np.array_equal(tks.cpu().numpy(), ks, equal_nan=True) and np.array_equal(tvs.cpu().numpy(), vs, equal_nan=True)
    assert np.array_equal(tk.view(torch.uint8).cpu().numpy(), k)
    assert np.array_equal(tv.view(torch.uint8).cpu().numpy(), v)
    if n_q and not spoil:
        assert np.array_equal(h.q.view(torch.int16).cpu().numpy(), q)
    assert bad.item() == n_bad
    return h


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("source", ["f32", "bf16"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [(4, 2, 64), (20, 5, 128)])
def test_tokens_of_decode_steps_and_prompts(kind, source, block, heads):
    run(kind, source, heads, block, [(5, 1), (3 * block, 1), (4 * block + block - 1, 1), (6 * block + 3, 2 * block + 5), (10 * block, block),
                                     (12 * block + 1, block - 1), (14 * block, 2)], seed=block)


@pytest.mark.parametrize("heads", [(3, 1, 128), (0, 2, 64), (8, 8, 64), (5, 5, 128)])
@pytest.mark.parametrize("gains", [(True, False), (False, True), (False, False)])
def test_head_layouts_and_gains(heads, gains):
    run("int8", "f32", heads, 32, [(7, 20), (64, 33), (130, 1)], seed=3, gains=gains)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_without_rotation_and_with_strides(kind):
    run(kind, "bf16", (4, 2, 128), 16, [(3, 40), (100, 1)], rotate=False)
    run(kind, "f32", (4, 2, 64), 64, [(3, 140), (400, 1), (449, 63)], strided=True)
    run(kind, "bf16", (4, 2, 128), 64, [(3, 140), (400, 1), (449, 63)], strided=True, eps=0.5)


def test_rows_that_go_nowhere():
    for row, slot, pos in ((0, -1, 0), (7, -1, 0), (7, -9, 3), (7, 10**6, 3), (7, 23, 400), (7, 23, -1), (49, 2**31 - 1, 0), (20, 20, 2**31 - 1)):
        run("int8", "f32", (4, 2, 64), 16, [(16, 50)], extra=[(row, slot, pos)])


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_numbers_that_are_none_spoil_their_head(kind):
    """A NaN makes its head NaN (codes of -T in the cache), an infinity zeros and one such code; the other heads and tokens do not move."""
    def nan(x):
        x[5, 1, 7] = np.nan                                   # a Q head
        x[6, 4, 60] = np.nan                                  # a K head
    run(kind, "f32", (4, 2, 64), 16, [(3, 20)], spoil=nan)

    def inf(x):
        x[6, 4, 3] = np.inf
    run(kind, "f32", (4, 2, 64), 16, [(3, 20)], spoil=inf)


def test_large_and_small_numbers():
    """Squares that fp32 does not hold."""
    def far(x):
        x[:, ::2] *= F(1e25)
        x[:, 1::2] *= F(1e-25)
    run("int8", "f32", (4, 2, 64), 32, [(3, 20), (70, 1)], spoil=far, eps=1e-30)


def test_captured():
    run("e4m3", "bf16", (20, 5, 128), 64, [(3, 20), (70, 1), (200, 64)], captured=True)


def nan_in_queries(x):
    x[5, 1, 7] = np.nan


def infinity_in_queries(x):
    x[6, 2, 40] = -np.inf
    x[7, 0, 3] = np.inf


def none_in_keys(x):
    x[6, 4, 60] = np.nan
    x[8, 5, 1] = np.inf


def beyond_squares(x):
    x[:, ::2] *= F(1e25)
    x[:, 1::2] *= F(1e-25)


@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("rotate", [True, False])
@pytest.mark.parametrize("spoil", [nan_in_queries, infinity_in_queries, none_in_keys, beyond_squares])
def test_queries_beside_numbers_that_are_none_and_of_far_ones(spoil, rotate, heads):
    """Every query bit for bit, but for the NaN's own bits: what spoils a head reaches no other head and no other token."""
    from paper_2504_12285_amd import binding as bl
    n_q, H, D = heads
    r = np.random.RandomState(D)
    T, eps = 23, 1e-30
    x = r.randn(T, n_q + 2 * H, D).astype(F)
    spoil(x)
    angle = r.rand(60, D // 2) * 6.3
    cos, sin = np.cos(angle).astype(F), np.sin(angle).astype(F)
    positions, slots = r.randint(0, 60, T).astype(np.int32), np.arange(5, 5 + T, dtype=np.int32)
    qg, kg = ((1 + 0.3 * r.randn(D)).astype(F) for _ in range(2))

    def t(a):
        return torch.from_numpy(a).cuda()
    h = bl.KVNormAppend(bl.KVCache.empty(4, H, 16, D, torch.device("cuda:0")), t(x.reshape(T, -1)), n_q, t(slots), t(positions), t(cos) if rotate else None,
                        t(sin) if rotate else None, q_gain=t(qg), k_gain=t(kg), eps=eps)
    h.q.fill_(7.0)
    h.run()
    y = normed(x[:, :n_q], qg, eps)
    if rotate:
        c, s = cos[positions][:, None], sin[positions][:, None]
        a, b = y[..., :D // 2], y[..., D // 2:]
        with np.errstate(all="ignore"):
            y = np.concatenate([a * c - b * s, b * c + a * s], -1)
    want = torch.from_numpy(y).to(torch.bfloat16).view(T, -1)
    got = h.q.cpu().view(T, -1)
    none = want.isnan()
    assert bool(none.any()) == (spoil in (nan_in_queries, infinity_in_queries))
    assert torch.equal(got.isnan(), none)
    assert torch.equal(got.view(torch.int16)[~none], want.view(torch.int16)[~none])
