"""The 8-bit float matrix: its product and its lookup against their definitions.

The row codes and their scales follow the definition step by step (every one a rounded fp32 operation), so a matrix that picks single
features gives them back bit for bit.  For a product in 64 bits over the same codes, A = sum_b s_b ws_b sum_k |c w| a row and column:
  sums inside a block             127 additions of at most two rounding units (an adder that cuts instead of rounding): 2 * 127 * 2^-24 of A
  scales and the sum over blocks  one product, one fused step a block and the joins of a split loop: (nb + 18) * 2^-24 of A
  the output                      fp32: contained; bf16: 2^-8 of the value
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn


def matrix(N, K, seed=0, gap=0):
    """Codes of all sizes, scales that differ from block to block."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    codes = (torch.randn(N, K + gap, generator=g, device=DEV) * torch.exp2(torch.randint(-3, 6, (N, 1), generator=g, device=DEV).float())).clamp(-448, 448).to(E4M3)
    scale = torch.exp(torch.randn(-(-N // 128), -(-K // 128), generator=g, device=DEV)) * 1e-3
    if gap:
        codes.view(torch.uint8)[:, K:] = 0x7f                 # NaN between the rows
        wide = torch.full((scale.shape[0], scale.shape[1] + 3), math.nan, device=DEV)
        wide[:, :scale.shape[1]] = scale
        scale = wide[:, :scale.shape[1]]
    return codes[:, :K], scale


def rows(M, K, seed=0, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed + 77)
    x = torch.randn(M, K, generator=g, device=DEV) * torch.exp(torch.randn(M, 1, generator=g, device=DEV))
    x[:, 3::50] *= 20
    x[:, 128:256] *= 1e-7                                     # a group below the floor of the scale
    if M > 2:
        x[1] = 0
    return x.to(dtype)


def row_codes(x, norm, gain, eps):
    """Codes (as fp32) and scales [M][nb] of rows, from their definition."""
    t = x.float()
    if norm:
        r = (1.0 / ((t.double() ** 2).sum(1, keepdim=True) / t.shape[1] + eps).sqrt()).float()
        t = t * r
        if gain is not None:
            t = t * gain
    M, K = t.shape
    nb = -(-K // 128)
    t = torch.nn.functional.pad(t.to(torch.bfloat16).float(), (0, nb * 128 - K)).view(M, nb, 128)
    s = torch.clamp(t.abs().amax(2), min=1e-5) * torch.tensor(1 / 448.0, device=DEV)
    return (t * (1.0 / s)[..., None]).to(E4M3).float(), s


def check(h, codes, scale, x, norm=False, gain=None, eps=2.0 ** -17):
    c, s = row_codes(x, norm, gain, eps)
    N, K = codes.shape
    M, nb = s.shape
    want, A = torch.zeros(M, N, dtype=torch.float64, device=DEV), torch.zeros(M, N, dtype=torch.float64, device=DEV)
    ws = scale.double().repeat_interleave(128, 0)[:N]
    for b in range(nb):
        w = codes[:, 128 * b:128 * b + 128].double()
        f = s[:, b].double()[:, None] * ws[:, b][None]
        want += (c[:, b, :w.shape[1]].double() @ w.T) * f
        A += (c[:, b, :w.shape[1]].double().abs() @ w.abs().T) * f
    y = h.y.double()
    assert torch.isfinite(y).all()
    most = (2 * 127 + nb + 18) * 2.0 ** -24 * A
    if h.y.dtype == torch.bfloat16:
        most = most * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    off = (y - want).abs()
    assert bool((off <= most).all()), "%g of what is allowed" % float((off / most.clamp(min=1e-300)).max())


def linear(M, N, K, dtype=torch.float32, out=torch.float32, norm=False, gain=True, gap=0, seed=0, **more):
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(N, K, seed, gap)
    x = rows(M, K, seed, dtype)
    g = None
    if norm and gain:
        g = 1 + 0.3 * torch.randn(K, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    h = bl.F8Linear(bl.F8Matrix(codes, scale), x, dtype=out, norm=norm, gain=g, eps=2.0 ** -17, **more)
    h.y.fill_(math.nan), h.workspace.fill_(255)
    h.run()
    check(h, codes, scale, x, norm, g)
    return h


@pytest.mark.parametrize("K", [64, 128, 192, 1088, 2560, 6912])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 48, 64, 65, 130])
def test_rows_and_lengths(M, K):
    linear(M, 300, K, seed=M)
    linear(M, 129, K, out=torch.bfloat16, dtype=torch.bfloat16, norm=M % 2 == 0, seed=K)


@pytest.mark.parametrize("N", [1, 3, 15, 16, 17, 127, 128, 130, 255, 257, 1000, 5003])
def test_outputs_of_every_width(N):
    for M in (1, 5, 40, 150):
        linear(M, N, 320, seed=N, out=torch.bfloat16 if M == 5 else torch.float32)


@pytest.mark.parametrize("M", [1, 7, 20, 64, 200])
def test_norms_and_producers(M):
    from paper_2504_12285_amd import binding as bl
    linear(M, 200, 1344, norm=True)
    linear(M, 200, 1344, norm=True, gain=False, dtype=torch.bfloat16)
    codes, scale = matrix(200, 640)
    a, b = rows(M, 640, 1), rows(M, 640, 2)
    aux = torch.empty_like(a)
    h = bl.F8Linear(bl.F8Matrix(codes, scale), prod=bl.make_producer(bl.BL_PROD_RESIDUAL, a, b, aux, norm=True, eps=2.0 ** -17), M=M)
    h.run()
    assert torch.equal(aux, a + b)
    check(h, codes, scale, a + b, True)
    gu = torch.cat([a, b], 1).contiguous()
    h = bl.F8Linear(bl.F8Matrix(codes, scale), prod=bl.make_producer(bl.BL_PROD_RELU2_GATE, gu), M=M)
    h.run()
    check(h, codes, scale, (a.clamp(min=0) * a.clamp(min=0)) * b)
    qkv = rows(M, 640 + 2 * 128, 3)
    h = bl.F8Linear(bl.F8Matrix(codes, scale), prod=bl.make_producer(bl.BL_PROD_ATTN_V, qkv, n_q=10, n_kv=2, head_dim=64), M=M)
    h.run()
    v = qkv[:, 640 + 128:].view(M, 2, 1, 64).expand(M, 2, 5, 64).reshape(M, 640)
    check(h, codes, scale, v)


@pytest.mark.parametrize("M", [1, 16, 100])
def test_long_rows(M):
    linear(M, 140, 20480)
    linear(M, 70, 9024, norm=True, out=torch.bfloat16)


def test_many_rows_and_columns():
    linear(777, 2000, 1216, dtype=torch.bfloat16, out=torch.bfloat16)
    linear(1025, 1409, 704)
    for M in (48, 49, 64, 65):                                # (the widest choices of each kind of kernel)
        linear(M, 8300, 2560, out=torch.bfloat16)
        linear(M, 8192, 4096, norm=True)
    for K in (1344, 1408, 1472, 1536):
        linear(200, 300, K, dtype=torch.bfloat16, norm=K == 1408)


@pytest.mark.parametrize("M", [1, 20, 70])
def test_rows_that_lie_apart(M):
    """NaN between the rows of codes and of scales is not read; outputs stand between others that stay."""
    for out, N in ((torch.float32, 210), (torch.bfloat16, 333)):
        y = torch.full((M, N + 11), 7.0, dtype=out, device=DEV)
        h = linear(M, N, 448, gap=64, y=y[:, 3:N + 3], out=out)
        keep = y.clone()
        keep[:, 3:N + 3] = 7
        assert h.y.data_ptr() == y.data_ptr() + 3 * y.element_size() and bool((keep == 7).all())


@pytest.mark.parametrize("M", [1, 3, 16, 40, 64, 100])
@pytest.mark.parametrize("norm", [False, True])
def test_row_codes_bit_for_bit(M, norm):
    """The matrix of single features: every output is one code times its scale."""
    from paper_2504_12285_amd import binding as bl
    K = 704
    codes = torch.eye(K, device=DEV).to(E4M3)
    x = rows(M, K, 5)
    h = bl.F8Linear(bl.F8Matrix(codes, torch.ones(6, 6, device=DEV)), x, norm=norm, eps=2.0 ** -17)
    h.run()
    c, s = row_codes(x, norm, None, 2.0 ** -17)
    assert torch.equal(h.y, (c * s[..., None]).view(M, -1)[:, :K])


@pytest.mark.parametrize("M", [2, 30, 70])
def test_numbers_that_are_none_spoil_their_row_and_nothing_else(M):
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(200, 448)
    x = rows(M, 448)
    clean = bl.F8Linear(bl.F8Matrix(codes, scale), x)
    clean.run()
    for k, odd in ((0, math.nan), (447, math.inf), (200, -math.inf)):
        bad = x.clone()
        bad[1, k] = odd
        h = bl.F8Linear(bl.F8Matrix(codes, scale), bad)
        h.run()
        assert bool(h.y[1].isnan().all())
        h.y[1] = clean.y[1]
        assert torch.equal(h.y, clean.y)
    codes.view(torch.uint8)[150, 5] = 0x7f                     # a NaN among the weights: its column
    h = bl.F8Linear(bl.F8Matrix(codes, scale), x)
    h.run()
    assert bool(h.y[:, 150].isnan().all())
    h.y[:, 150] = clean.y[:, 150]
    assert torch.equal(h.y, clean.y)


def test_the_same_bits_every_time():
    from paper_2504_12285_amd import binding as bl
    for M, N, K in ((1, 3000, 2560), (40, 500, 8192), (64, 130, 20480), (300, 260, 2048)):
        codes, scale = matrix(N, K)
        h = bl.F8Linear(bl.F8Matrix(codes, scale), rows(M, K), norm=True)
        h.run()
        want = h.y.clone()
        for _ in range(3):
            h.y.fill_(math.nan), h.workspace.fill_(255)
            h.run()
            assert torch.equal(h.y, want)


@pytest.mark.parametrize("M", [1, 20, 200])
def test_captured_and_on_another_stream(M):
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(400, 1280)
    x = rows(M, 1280)
    h = bl.F8Linear(bl.F8Matrix(codes, scale), x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        h.run()
    s.synchronize()
    check(h, codes, scale, x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.run()
    for step in range(4):
        x.copy_(rows(M, 1280, step))
        g.replay()
        torch.cuda.synchronize()
        eager = bl.F8Linear(bl.F8Matrix(codes, scale), x)
        eager.run()
        assert torch.equal(eager.y, h.y)
        check(h, codes, scale, x)


def test_a_matrix_beyond_four_gigabytes():
    """Rows so far apart that the last ones' offsets pass 32 bits; outputs too."""
    from paper_2504_12285_amd import binding as bl
    N, K, far = 300, 256, 16 << 20
    codes, scale = matrix(N, K)
    pool = torch.empty((N - 1) * far + K, dtype=torch.uint8, device=DEV)
    apart = torch.as_strided(pool, (N, K), (far, 1)).view(E4M3)
    apart.view(torch.uint8).copy_(codes.view(torch.uint8))
    ids = torch.tensor([299, 0, 257], dtype=torch.int32, device=DEV)
    for M in (1, 20, 130):
        x = rows(M, K)
        y = torch.as_strided(torch.empty((M - 1) * 9_000_000 + N, device=DEV), (M, N), (9_000_000, 1))
        h = bl.F8Linear(bl.F8Matrix(apart, scale), x, y=y)
        h.run()
        check(h, codes, scale, x)
    a, b = bl.F8Embedding(bl.F8Matrix(apart, scale), ids), bl.F8Embedding(bl.F8Matrix(codes, scale), ids)
    a.run(), b.run()
    assert torch.equal(a.out, b.out)


# ---- lookup ----

@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T, N, K", [(1, 1, 64), (5, 300, 192), (1000, 700, 2560), (3, 129, 6912), (70, 128, 128)])
def test_lookup(out, T, N, K):
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(N, K, gap=64 if K == 192 else 0)
    ids = torch.randint(0, N, (T,), generator=torch.Generator(device=DEV).manual_seed(T), device=DEV, dtype=torch.int32)
    ids[-1] = N - 1
    h = bl.F8Embedding(bl.F8Matrix(codes, scale), ids, dtype=out, multiplier=50.6)
    h.out.fill_(math.nan)
    h.run()
    i = ids.long()
    factor = scale[i // 128].repeat_interleave(128, 1)[:, :K]
    assert torch.equal(h.out, ((codes.contiguous().view(torch.uint8)[i].view(E4M3).float() * factor) * torch.tensor(50.6, device=DEV)).to(out))


def test_lookup_of_ids_that_name_no_row():
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(200, 128)
    ids = torch.tensor([5, -1, 200, -2, 2**31 - 1, -2**31, 199, 5], dtype=torch.int32, device=DEV)
    bad = torch.full((1,), 10, dtype=torch.int32, device=DEV)
    out = torch.full((8, 160), 3.0, device=DEV)
    h = bl.F8Embedding(bl.F8Matrix(codes, scale), ids, out=out[:, :128], bad=bad)
    h.run()
    assert bad.item() == 14 and bool((out[1:6, :128] == 0).all()) and bool((out[:, 128:] == 3).all())
    assert torch.equal(out[0], out[7]) and bool((out[0, :128] != 0).any()) and bool((out[6, :128] != 0).any())


def test_quantised_matrix_stands_for_its_numbers():
    """A code is off by half a step: 2^-4 of the value, or half of the smallest step, 2^-10 of the block's scale; the scale and the quotient add 2^-23."""
    from paper_2504_12285_amd import binding as bl
    g = torch.Generator(device=DEV).manual_seed(1)
    W = torch.randn(300, 320, generator=g, device=DEV) * torch.exp(torch.randn(300, 1, generator=g, device=DEV))
    m = bl.F8Matrix.quantise(W)
    h = bl.F8Embedding(m, torch.arange(300, dtype=torch.int32, device=DEV))
    h.run()
    step = m.scale.repeat_interleave(128, 0)[:300].repeat_interleave(128, 1)[:, :320]
    assert bool(((h.out - W).abs() <= (2.0 ** -4 + 2.0 ** -22) * W.abs() + 2.0 ** -10 * step).all())


@pytest.mark.parametrize("K", [8192, 8256, 9024, 20480])
@pytest.mark.parametrize("M", [1, 3, 20, 100])
def test_the_sum_that_a_producer_leaves_is_whole(M, K):
    """Rows on both sides of the 8192 values that a workgroup keeps between their norm and their codes: every value of the sum is written."""
    from paper_2504_12285_amd import binding as bl
    codes, scale = matrix(70, K)
    a, b = rows(M, K, 1), rows(M, K, 2)
    for norm in (True, False):
        aux = torch.full_like(a, math.nan)
        h = bl.F8Linear(bl.F8Matrix(codes, scale), prod=bl.make_producer(bl.BL_PROD_RESIDUAL, a, b, aux, norm=norm, eps=2.0 ** -17), M=M)
        h.run()
        assert torch.equal(aux, a + b)
        check(h, codes, scale, a + b, norm)
