"""The rotary append against its definition, token by token in numpy: every fp32 step is one rounded operation on both
sides, so codes, scales and the bf16 queries are compared bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F = np.float32


def e4m3(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=F)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def e4m3_value(c):
    return torch.from_numpy(np.ascontiguousarray(c)).view(torch.float8_e4m3fn).float().numpy()


def encode(y, kind):
    top = F(127 if kind == "int8" else 448)
    y = np.minimum(np.maximum(np.where(np.isnan(y), -top, y), -top), top).astype(F)
    return np.rint(y).astype(np.int8).view(np.uint8) if kind == "int8" else e4m3(y)


def value(c, kind):
    return c.view(np.int8).astype(F) if kind == "int8" else e4m3_value(c)


def oracle(cache, x, n_q, slots, positions, cos, sin, kind):
    """cache: k, v (uint8), k_scale, v_scale, changed in place.  x fp32 [T][heads][D].  Returns (q bits, bad)."""
    k, v, ks, vs = cache
    N, H, bs, D = k.shape
    T, top, bad = len(x), F(127 if kind == "int8" else 448), 0
    q = np.zeros((T, n_q, D), F)
    ok = []
    for t in range(T):
        turned = x[t].copy()
        here = True
        if cos is not None:
            here = 0 <= positions[t] < len(cos)
            if here:
                c, s = cos[positions[t]], sin[positions[t]]
                a, b = x[t, :n_q + H, :D // 2], x[t, :n_q + H, D // 2:]
                with np.errstate(all="ignore"):
                    turned[:n_q + H, :D // 2] = a * c - b * s
                    turned[:n_q + H, D // 2:] = b * c + a * s
        if here:
            q[t] = turned[:n_q]
        x[t] = turned
        outside = slots[t] < -1 or slots[t] >= N * bs
        bad += (not here) or outside
        ok.append(here and not outside and slots[t] >= 0)
    for t in range(T):
        blk, off = slots[t] // bs, slots[t] % bs
        if not ok[t] or any(t >= j and ok[t - j] and slots[t - j] == slots[t] - j for j in range(1, off + 1)):
            continue
        rows = [t + j for j in range(bs - off) if t + j < T and ok[t + j] and slots[t + j] == slots[t] + j]
        at = off + np.array(rows) - t
        for codes, scales, first in ((k, ks, n_q), (v, vs, n_q + H)):
            for h in range(H):
                y = x[rows, first + h]
                most = F(np.nanmax(np.abs(y))) if not np.isnan(y).all() else F(0)
                s = max(most, F(1e-5)) * (F(1) / top)
                held = codes[blk, h, :off] if codes is k else codes[blk, h, :, :off]
                if off:
                    old = scales[blk, h]
                    if s > old:
                        held[...] = encode(value(held.copy(), kind) * (old / s), kind)
                    else:
                        s = old
                scales[blk, h] = s
                with np.errstate(all="ignore"):
                    z = encode(y * (F(1) / s), kind)
                if codes is k:
                    codes[blk, h, at] = z
                else:
                    codes[blk, h][:, at] = z.T
    bits = torch.from_numpy(q).to(torch.bfloat16).view(torch.int16).numpy()
    return bits.reshape(T, -1), bad


def run(kind, source, heads, block, runs, seed=0, rotate=True, spoil=None, extra=(), strided=False, N=None, check_q=True):
    """runs: (first slot, tokens) in order of the rows; extra: (row, slot, position) put in place afterwards."""
    from paper_2504_12285_amd import binding as bl
    n_q, H, D = heads
    r = np.random.RandomState(seed)
    T = sum(n for _, n in runs)
    N = N or max(s // block for s, _ in runs) + 3
    slots = np.concatenate([np.arange(s, s + n) for s, n in runs]).astype(np.int32)
    positions = np.concatenate([np.arange(n) + r.randint(0, 50) for _, n in runs]).astype(np.int32)
    for row, slot, pos in extra:
        slots[row], positions[row] = slot, pos
    x = r.randn(T, n_q + 2 * H, D).astype(F) * np.exp(r.randn(T, 1, 1)).astype(F)
    if spoil:
        spoil(x)
    xt = torch.from_numpy(x.reshape(T, -1)).to(torch.float32 if source == "f32" else torch.bfloat16)
    x = xt.float().numpy().reshape(x.shape).copy()
    angle = r.rand(400, D // 2) * 6.3
    cos, sin = np.cos(angle).astype(F), np.sin(angle).astype(F)
    k, v = (encode(r.randn(N, H, *s).astype(F) * F(40), kind) for s in ((block, D), (D, block)))
    ks, vs = ((np.exp(r.randn(N, H)) * 0.02).astype(F) for _ in range(2))
    dev = "cuda:0"
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn

    def layer(a):                                     # a view whose blocks lie apart, or the tensor itself
        t = torch.from_numpy(a).to(dev)
        if not strided:
            return t
        pool = torch.full((a.shape[0], 3) + a.shape[1:], 7, dtype=t.dtype, device=dev)
        pool[:, 1] = t
        return pool[:, 1]
    tk, tv, tks, tvs = layer(k).view(dtype), layer(v).view(dtype), layer(ks), layer(vs)
    qkv = xt.to(dev)
    if strided:
        wide = torch.zeros((T, xt.shape[1] + 24), dtype=xt.dtype, device=dev)
        wide[:, :xt.shape[1]] = qkv
        qkv = wide[:, :xt.shape[1]]
    bad = torch.zeros(1, dtype=torch.int32, device=dev)
    h = bl.KVAppend(bl.KVCache(tk, tv, tks, tvs), qkv, n_q, torch.from_numpy(slots).to(dev), torch.from_numpy(positions).to(dev),
                    torch.from_numpy(cos).to(dev) if rotate else None, torch.from_numpy(sin).to(dev) if rotate else None, bad=bad)
    h.run()
    q, n_bad = oracle((k, v, ks, vs), x, n_q, slots, positions, cos if rotate else None, sin, kind)
    assert np.array_equal(tks.cpu().numpy(), ks, equal_nan=True) and np.array_equal(tvs.cpu().numpy(), vs, equal_nan=True)
    assert np.array_equal(tk.view(torch.uint8).cpu().numpy(), k)
    assert np.array_equal(tv.view(torch.uint8).cpu().numpy(), v)
    if n_q and check_q:
        assert np.array_equal(h.q.view(torch.int16).cpu().numpy(), q)
    assert bad.item() == n_bad
    return h


HEADS = [(4, 2, 64), (20, 5, 128), (3, 1, 128), (0, 2, 64), (8, 8, 64)]


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("source", ["f32", "bf16"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", HEADS[:2])
def test_tokens_of_decode_steps_and_prompts(kind, source, block, heads):
    run(kind, source, heads, block, [(5, 1), (3 * block, 1), (4 * block + block - 1, 1), (6 * block + 3, 2 * block + 5), (10 * block, block), (12 * block + 1, block - 1),
                                     (14 * block, 2)], seed=block)


@pytest.mark.parametrize("heads", HEADS[2:])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_head_layouts(kind, heads):
    run(kind, "f32", heads, 32, [(7, 20), (64, 33), (130, 1)], seed=3)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_without_rotation_and_with_strides(kind):
    run(kind, "bf16", (4, 2, 128), 16, [(3, 40), (100, 1)], rotate=False)
    run(kind, "f32", (4, 2, 64), 64, [(3, 140), (400, 1), (449, 63)], strided=True)
    run(kind, "bf16", (4, 2, 128), 64, [(3, 140), (400, 1), (449, 63)], strided=True)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_rows_that_go_nowhere(kind):
    """Padding, slots outside the cache and positions outside the table, in the middle of runs and at their ends."""
    for row, slot, pos in ((0, -1, 0), (7, -1, 0), (7, -9, 3), (7, 10**6, 3), (7, 23, 400), (7, 23, -1), (49, 2**31 - 1, 0), (20, 20, 2**31 - 1)):
        run(kind, "f32", (4, 2, 64), 16, [(16, 50)], extra=[(row, slot, pos)])
    run(kind, "f32", (4, 2, 64), 16, [(16, 50)], extra=[(i, -1, 0) for i in range(50)])


def test_a_scale_that_grows_token_by_token_stays_near():
    """Sixteen tokens, each larger than the last, one call each: every step moves the block.  A code is off by half a step
    of the scale of its time for its own rounding and half a step of every later scale, so by (17 - t) / 2 steps of the last at most."""
    from paper_2504_12285_amd import binding as bl
    dev, D, bs = "cuda:0", 64, 16
    g = torch.Generator().manual_seed(5)
    x = torch.randn(bs, 3 * D, generator=g) * (1.2 ** torch.arange(bs))[:, None]
    c = bl.KVCache.empty(2, 1, bs, D, dev)
    c.k.zero_(), c.v.zero_(), c.k_scale.fill_(1e9), c.v_scale.fill_(1e9)
    for t in range(bs):
        bl.KVAppend(c, x[t:t + 1].to(dev), 1, torch.tensor([bs + t], dtype=torch.int32, device=dev)).run()
    for codes, scale, part in ((c.k[1, 0], c.k_scale[1, 0], x[:, D:2 * D]), (c.v[1, 0].t(), c.v_scale[1, 0], x[:, 2 * D:])):
        s = scale.item()
        assert s == F(part.abs().max().item()) * (F(1) / F(127))
        off = (codes.cpu().double() * s - part.double()).abs().amax(1) / s
        assert bool((off <= (17 - torch.arange(bs)) / 2 * (1 + 1e-5)).all())
    assert c.k_scale[0, 0].item() == F(1e9)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_values_that_are_not_numbers_and_rows_of_zeros(kind):
    def nan(x):
        x[3, :, 5] = np.nan
    run(kind, "f32", (2, 1, 64), 16, [(0, 12)], spoil=nan, check_q=False, rotate=False)

    def zeros(x):
        x[:] = 0
    run(kind, "f32", (2, 1, 64), 16, [(0, 12), (33, 2)], spoil=zeros)

    def tiny(x):
        x[:] *= F(1e-9)
    run(kind, "f32", (2, 1, 64), 16, [(0, 12)], spoil=tiny)

    def huge(x):
        x[:] *= F(1e36)
    run(kind, "f32", (2, 1, 64), 16, [(0, 12), (20, 3)], spoil=huge, rotate=False)


def test_an_infinity_spoils_its_block_and_head_only():
    from paper_2504_12285_amd import binding as bl
    dev = "cuda:0"
    x = torch.randn(40, 4 * 64, device=dev)
    x[5, 1 * 64 + 3] = float("inf")                     # K of head 0
    got = []
    for y in (x, torch.where(x.isinf(), 0.0, x)):
        c = bl.KVCache.empty(3, 1, 16, 64, dev)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.zero_()
        bl.KVAppend(c, y[:, :3 * 64].contiguous(), 1, torch.arange(40, dtype=torch.int32, device=dev)).run()
        got.append(c)
    a, b = got
    assert a.k_scale[0, 0].isinf() and torch.equal(a.k_scale[1:], b.k_scale[1:]) and torch.equal(a.k[1:], b.k[1:])
    assert torch.equal(a.v, b.v) and torch.equal(a.v_scale, b.v_scale)


def test_more_rows_than_a_window_each():
    """Enough rows that a workgroup looks at several: runs that start anywhere in a window, long and single."""
    r = np.random.RandomState(9)
    runs, at = [], 0
    while sum(n for _, n in runs) < 3000:
        n = int(r.choice([1, 1, 2, 15, 16, 17, 40]))
        at = (at // 16 + 1) * 16 + int(r.randint(16))
        runs.append((at, n))
        at += n
    run("int8", "f32", (1, 1, 64), 16, runs, seed=2)
    run("e4m3", "bf16", (1, 1, 64), 16, runs, seed=2)


def test_blocks_beyond_four_gigabytes():
    """Blocks 1.5 GiB apart: offsets of the last pass 32 bits."""
    from paper_2504_12285_amd import binding as bl
    dev, far, D = "cuda:0", 3 << 29, 64
    pools = [torch.empty(3 * far + 16 * D, dtype=torch.int8, device=dev) for _ in range(2)]
    k = torch.as_strided(pools[0], (4, 1, 16, D), (far, 16 * D, D, 1))
    v = torch.as_strided(pools[1], (4, 1, D, 16), (far, 16 * D, 16, 1))
    near = bl.KVCache.empty(4, 1, 16, D, dev)
    c = bl.KVCache(k, v, torch.zeros(4, 1, device=dev), torch.zeros(4, 1, device=dev))
    x = torch.randn(64, 3 * D, device=dev)
    for cache in (c, near):
        bl.KVAppend(cache, x, 1, torch.arange(64, dtype=torch.int32, device=dev)).run()
    for b in range(4):
        assert torch.equal(c.k[b], near.k[b]) and torch.equal(c.v[b], near.v[b])


def test_captured_and_on_another_stream():
    from paper_2504_12285_amd import binding as bl
    dev = "cuda:0"
    qkv, slots = torch.zeros(4, 3 * 64, device=dev), torch.zeros(4, dtype=torch.int32, device=dev)
    a, b = (bl.KVCache.empty(8, 1, 16, 64, dev) for _ in range(2))
    for c in (a, b):
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.zero_()
    captured, eager = (bl.KVAppend(c, qkv, 1, slots) for c in (a, b))
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    slots.fill_(-1)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        captured.run()
    s.synchronize()
    with torch.cuda.graph(g):
        captured.run()
    for step in range(4):
        qkv.copy_(torch.randn(4, 3 * 64, device=dev) * (step + 1))
        slots.copy_(torch.arange(4, dtype=torch.int32, device=dev) * 32 + step)
        g.replay()
        eager.run()
        torch.cuda.synchronize()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale), (captured.q, eager.q)):
            assert torch.equal(x, y)
