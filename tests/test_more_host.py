"""Calls of the 8-bit float matrix, of shared prefixes and of the append with norms on the host: every refusal comes before any GPU work, sizes are
right, and the binding takes only tensors that a descriptor can stand for.  Needs no GPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2504_12285_amd import binding as bl
from paper_2504_12285_amd import build as hip_build
from test_kv_host import ALIGN, BAD_ATTENTION, BAD_CACHES, NULL, P, SHAPE, VALUE, WORKSPACE, attention, cache, lib, tables, tokens  # noqa: F401

torch = pytest.importorskip("torch")


def held(batch=None, **more):
    return bl.KVHeldBatchDesc(**dict(dict(batch=batch or tables(), max_new=0, held=P), **more))


@pytest.mark.parametrize("d, status", [(dict(held=None), NULL), (dict(held=P + 2), ALIGN), (dict(max_new=-1), SHAPE), (dict(batch=tables(B=0)), SHAPE),
                                       (dict(batch=tables(bad=None)), NULL)])
def test_held_tables_refuse(lib, d, status):  # noqa: F811
    assert lib.bl_kv_tables_held(ctypes.byref(held(**d)), None) == status
    assert lib.bl_kv_tables_held(None, None) == NULL


def norm(t=None, **more):
    return bl.KVNormTokensDesc(**dict(dict(tokens=t or tokens(), q_gain=P, k_gain=P, eps=1e-5), **more))


@pytest.mark.parametrize("d, status", [(dict(eps=0.0), VALUE), (dict(eps=-1.0), VALUE), (dict(eps=float("nan")), VALUE), (dict(eps=float("inf")), VALUE),
                                       (dict(q_gain=P + 4), ALIGN), (dict(k_gain=P + 8), ALIGN), (dict(t=tokens(T=0)), SHAPE), (dict(t=tokens(qkv=None)), NULL),
                                       (dict(t=tokens(qkv_stride=30 * 128 - 4)), SHAPE)])
def test_append_with_norms_refuses(lib, d, status):  # noqa: F811
    assert lib.bl_kv_append_norm(ctypes.byref(norm(**d)), None) == status
    assert lib.bl_kv_append_norm(None, None) == NULL


def shared(a=None, **more):
    return bl.AttnSharedDesc(**dict(dict(attn=a or attention(), group=P, shared_blocks=P, shared_table=P, shared_stride=6, n_groups=3, max_shared=6, max_own=0), **more))


@pytest.mark.parametrize("d, status", [(dict(group=None), NULL), (dict(shared_blocks=None), NULL), (dict(shared_table=None), NULL), (dict(n_groups=0), SHAPE),
                                       (dict(n_groups=4097), SHAPE), (dict(max_shared=0), SHAPE), (dict(max_shared=7), SHAPE), (dict(max_own=-1), SHAPE),
                                       (dict(max_shared=1 << 25, shared_stride=1 << 25), SHAPE), (dict(group=P + 2), ALIGN), (dict(shared_table=P + 1), ALIGN),
                                       (dict(shared_blocks=P + 3), ALIGN)])
def test_shared_attention_refuses(lib, d, status):  # noqa: F811
    s = shared(**d)
    assert lib.bl_attn_kv8_shared(ctypes.byref(s), None) == status
    assert lib.bl_attn_shared_workspace_bytes(ctypes.byref(s)) == 0
    assert lib.bl_attn_kv8_shared(None, None) == NULL


@pytest.mark.parametrize("more, status", BAD_ATTENTION)
def test_shared_attention_refuses_what_attention_does(lib, more, status):  # noqa: F811
    assert lib.bl_attn_kv8_shared(ctypes.byref(shared(attention(**more))), None) == status


@pytest.mark.parametrize("more, status", BAD_CACHES)
def test_a_bad_cache_is_refused(lib, more, status):  # noqa: F811
    assert lib.bl_attn_kv8_shared(ctypes.byref(shared(attention(cache(**more)))), None) == status
    assert lib.bl_kv_append_norm(ctypes.byref(norm(tokens(cache(**more)))), None) == status


def test_shared_attention_wants_its_workspace(lib):  # noqa: F811
    assert lib.bl_attn_kv8_shared(ctypes.byref(shared(attention(workspace=None))), None) == WORKSPACE
    assert lib.bl_attn_kv8_shared(ctypes.byref(shared(attention(workspace=P + 16))), None) == ALIGN
    one, few, more = (lib.bl_attn_shared_workspace_bytes(ctypes.byref(shared(**d))) for d in (dict(), dict(a=attention(max_len=10**6)), dict(a=attention(max_len=10**6), max_shared=500, shared_stride=500)))
    assert 0 < one < few < more


def test_shared_attention_s_workspace_stays_small_beside_a_prompt(lib):  # noqa: F811
    """Partial results stand for the rows that have some: a prompt of thousands of rows beside seven decoding requests takes what its own pieces need."""
    a = attention(B=8, T=8192 + 7, max_q=8192, max_len=30000)
    n = lib.bl_attn_shared_workspace_bytes(ctypes.byref(shared(a, max_own=9000)))
    assert 0 < n <= (a.T * a.n_q + 60 * a.B * a.cache.n_kv * 16) * 130 * 4 + a.T * 8 + 512
    a = attention(B=4096, T=4200, max_q=50, max_len=30000)
    n = lib.bl_attn_shared_workspace_bytes(ctypes.byref(shared(a, max_own=100)))
    assert 0 < n <= 3 * a.T * a.n_q * 130 * 4 + a.T * 8 + 512


def matrix(**more):
    return bl.F8MatrixDesc(**dict(dict(codes=P, scale=P, N=200, K=192, stride=192, scale_stride=2), **more))


BAD_MATRICES = [(dict(codes=None), NULL), (dict(scale=None), NULL), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=200, stride=256), SHAPE), (dict(K=32), SHAPE),
                (dict(stride=128), SHAPE), (dict(scale_stride=1), SHAPE), (dict(N=(1 << 24) + 1), SHAPE), (dict(codes=P + 8), ALIGN), (dict(stride=200), ALIGN),
                (dict(scale=P + 2), ALIGN)]


def product(w=None, prod=None, **more):
    d = dict(w=w or matrix(), prod=prod or bl.Producer(kind=bl.BL_PROD_F32, in0=P), M=3, y_stride=200, y=P, y_kind=0, workspace=P)
    return bl.F8ProductDesc(**dict(d, **more))


def lookup(w=None, **more):
    return bl.F8LookupDesc(**dict(dict(w=w or matrix(), ids=P, T=4, out_stride=192, out=P, out_kind=0, multiplier=1.0, bad=P), **more))


@pytest.mark.parametrize("more, status", BAD_MATRICES)
def test_a_bad_matrix_is_refused(lib, more, status):  # noqa: F811
    assert lib.bl_f8_linear(ctypes.byref(product(matrix(**more))), None) == status
    assert lib.bl_f8_workspace_bytes(ctypes.byref(product(matrix(**more)))) == 0
    assert lib.bl_f8_embed(ctypes.byref(lookup(matrix(**more))), None) == status


@pytest.mark.parametrize("d, status", [(dict(y=None), NULL), (dict(prod=bl.Producer(kind=bl.BL_PROD_F32)), NULL), (dict(prod=bl.Producer(kind=9, in0=P)), VALUE),
                                       (dict(prod=bl.Producer(kind=bl.BL_PROD_RESIDUAL, in0=P)), VALUE), (dict(prod=bl.Producer(kind=bl.BL_PROD_F32, in0=P + 4)), VALUE),
                                       (dict(prod=bl.Producer(kind=bl.BL_PROD_F32, in0=P, norm=1, eps=-1.0)), VALUE), (dict(y_kind=2), VALUE), (dict(M=0), SHAPE),
                                       (dict(M=(1 << 24) + 1), SHAPE), (dict(y_stride=199), SHAPE), (dict(y=P + 2), ALIGN), (dict(y=P + 1, y_kind=1), ALIGN),
                                       (dict(w=matrix(N=1 << 24), M=1 << 24, y_stride=1 << 24), SHAPE), (dict(workspace=P + 16), ALIGN)])
def test_product_refuses(lib, d, status):  # noqa: F811
    assert lib.bl_f8_linear(ctypes.byref(product(**d)), None) == status
    assert lib.bl_f8_linear(None, None) == NULL


def test_product_wants_its_workspace(lib):  # noqa: F811
    p = product(M=300, workspace=None)
    assert lib.bl_f8_workspace_bytes(ctypes.byref(p)) >= 300 * 256 and lib.bl_f8_linear(ctypes.byref(p), None) == WORKSPACE


@pytest.mark.parametrize("d, status", [(dict(ids=None), NULL), (dict(out=None), NULL), (dict(T=0), SHAPE), (dict(T=(1 << 24) + 1), SHAPE), (dict(out_stride=128), SHAPE),
                                       (dict(out_kind=3), VALUE), (dict(out=P + 8), ALIGN), (dict(out_stride=194), ALIGN), (dict(out_stride=196, out_kind=1), ALIGN),
                                       (dict(ids=P + 2), ALIGN), (dict(bad=P + 1), ALIGN)])
def test_lookup_refuses(lib, d, status):  # noqa: F811
    assert lib.bl_f8_embed(ctypes.byref(lookup(**d)), None) == status
    assert lib.bl_f8_embed(None, None) == NULL


def test_descriptors_have_the_size_of_the_header_s():
    assert [ctypes.sizeof(c) for c in (bl.KVHeldBatchDesc, bl.KVNormTokensDesc, bl.AttnSharedDesc, bl.F8MatrixDesc, bl.F8ProductDesc, bl.F8LookupDesc)] == \
        [152, 200, 240, 48, 152, 96]


def test_the_binding_takes_what_a_descriptor_can_stand_for(lib):  # noqa: F811
    f8, i32 = torch.float8_e4m3fn, torch.int32
    pool = torch.zeros(200, 256, dtype=torch.uint8).view(f8)
    m = bl.F8Matrix(pool[:, :192], torch.zeros(2, 2))
    assert (m.desc.N, m.desc.K, m.desc.stride, m.desc.scale_stride) == (200, 192, 256, 2)
    for bad in ((pool.view(torch.int8), torch.zeros(2, 2)), (pool, torch.zeros(2, 3)), (pool, torch.zeros(2, 2).double()), (pool.view(torch.uint8).t().view(f8), torch.zeros(2, 2))):
        with pytest.raises((TypeError, ValueError)):
            bl.F8Matrix(*bad)
    x = torch.zeros(20, 192)
    h = bl.F8Linear(m, x, dtype=torch.bfloat16)
    assert h.y.shape == (20, 200) and h.desc.y_kind == bl.BL_F8_OUT_BF16 and h.workspace.numel() >= 20 * 256
    assert bl.F8Linear(m, x, y=torch.zeros(20, 208)[:, :200], workspace=h.workspace).desc.y_stride == 208
    for more in (dict(x=x.half()), dict(x=x[:, :128]), dict(x=x.t()), dict(), dict(x=x, prod=bl.Producer()), dict(prod=bl.Producer()), dict(x=x, y=torch.zeros(20, 100)),
                 dict(x=x, gain=torch.zeros(3)), dict(x=x, dtype=torch.float16), dict(x=x, workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            bl.F8Linear(m, **more)
    ids = torch.zeros(5, dtype=i32)
    assert bl.F8Embedding(m, ids).out.shape == (5, 192)
    for more in (dict(ids=ids.long()), dict(ids=ids, out=torch.zeros(5, 200)), dict(ids=ids, bad=torch.zeros(2, dtype=i32)), dict(ids=ids, dtype=torch.int8)):
        with pytest.raises((TypeError, ValueError)):
            bl.F8Embedding(m, **more)
    c = bl.KVCache.empty(6, 2, 16, 64, "cpu")
    n, q, table = torch.zeros(3, dtype=i32), torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=i32)
    args = dict(cache=c, q=q, q_start=torch.zeros(4, dtype=i32), seq_len=n, table=table, group=n, shared_table=torch.zeros(2, 3, dtype=i32),
                shared_blocks=torch.zeros(2, dtype=i32))
    h = bl.KVSharedAttention(**args)
    assert (h.desc.n_groups, h.desc.max_shared, h.desc.shared_stride) == (2, 3, 3)
    for more in (dict(group=n[:2]), dict(group=n.long()), dict(shared_blocks=n), dict(shared_table=n), dict(workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            bl.KVSharedAttention(**dict(args, **more))
    a = dict(cache=c, qkv=torch.zeros(3, 6 * 64), n_q=2, slots=n)
    assert bl.KVNormAppend(**a, q_gain=torch.zeros(64)).desc.k_gain is None
    for more in (dict(q_gain=torch.zeros(32)), dict(k_gain=torch.zeros(64).double())):
        with pytest.raises((TypeError, ValueError)):
            bl.KVNormAppend(**a, **more)
    t = bl.KVTables(n, n, table, torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5, held=n, max_new=3)
    assert t.desc.max_new == 3 and t._where == "bl_kv_tables_held"
    for more in (dict(held=n[:2]), dict(held=n, max_new=0)):
        with pytest.raises((TypeError, ValueError)):
            bl.KVTables(n, n, table, torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5, **more)


def test_a_producer_keeps_its_tensors():
    import gc
    import weakref
    tensors = [torch.zeros(3, 192) for _ in range(4)]
    refs = [weakref.ref(t) for t in tensors]
    p = bl.make_producer(bl.BL_PROD_RESIDUAL, tensors[0], tensors[1], tensors[2], norm=True, gain=tensors[3])
    del tensors
    gc.collect()
    assert all(r() is not None for r in refs)
    del p
    gc.collect()
    assert all(r() is None for r in refs)


def test_product_refuses_to_write_what_it_reads(lib):  # noqa: F811
    """Addresses far apart, then one of them moved into another's bytes: every pair of a written and a read one, ends included."""
    at = {k: P + (i << 32) for i, k in enumerate(("in0", "in1", "aux", "gain", "codes", "scale", "y", "space"))}

    def call(**moved):
        a = dict(at, **moved)
        prod = bl.Producer(kind=bl.BL_PROD_RESIDUAL, in0=a["in0"], in1=a["in1"], aux_out=a["aux"], norm=1, gain=a["gain"], eps=1e-5)
        return lib.bl_f8_linear(ctypes.byref(product(matrix(codes=a["codes"], scale=a["scale"], K=192), prod, M=300, y=a["y"], workspace=a["space"])), None)

    length = dict(in0=300 * 192 * 4, in1=300 * 192 * 4, aux=300 * 192 * 4, gain=192 * 4, codes=200 * 192, scale=16, y=300 * 200 * 4)
    for out in ("aux", "y", "space"):
        for other in at:
            if other == out or other == "space":
                continue
            assert call(**{out: at[other]}) == VALUE, (out, other)
            last = at[other] + length[other] - 1
            assert call(**{out: last - last % 256}) == VALUE or last - last % 256 < at[other], (out, other)


def layers_of_nothing(**more):
    """The tables and groups of served layers, without a layer: three places, the first with a request of 70 tokens in blocks of 32."""
    from paper_2504_12285_amd import serve
    layers = serve.CachedLayers([], [], 3, 80, max_blocks=8, n_blocks=30, device=torch.device("cpu"), block=32, **more)
    layers.seq_len[0] = 70
    layers.table[0, :3] = torch.tensor([7, 8, 9], dtype=torch.int32)
    layers.free_count[0] = 27
    return layers


def state(layers):
    return [t.clone() for t in (layers.seq_len, layers.table, layers.held, layers.group, layers.shared_table, layers.shared_blocks, layers.free_list, layers.free_count)]


def test_groups_and_places_are_the_layers_own():
    """Numbers outside the groups and places are refused, negative ones too (they would be those of another), and change nothing."""
    layers = layers_of_nothing(groups=2)
    before = state(layers)
    for group, place in ((-1, 0), (2, 0), (-2, 0), (0, -1), (0, -3), (0, 3), (1, 10)):
        with pytest.raises(ValueError):
            layers.share(group, place, 2)
    assert all(torch.equal(a, b) for a, b in zip(before, state(layers))) and layers.prefix == [0, 0]
    layers.share(1, 0, 2)
    assert layers.group.tolist() == [1, -1, -1] and layers.prefix == [0, 2]
    before = state(layers)
    for group, place in ((-1, 1), (3, 1), (1, -1), (1, -2), (1, 3)):
        with pytest.raises(ValueError):
            layers.join(place, group)
    for group in (-1, -2, 2, 10):
        with pytest.raises(ValueError):
            layers.release(group)
    assert all(torch.equal(a, b) for a, b in zip(before, state(layers))) and layers.prefix == [0, 2]
    layers.join(2, 1)
    assert layers.seq_len.tolist() == [70, 0, 64] and layers.table[2, :2].tolist() == [7, 8] and layers.held.tolist() == [2, 0, 2]


def test_layers_without_groups_share_nothing():
    layers = layers_of_nothing()
    for call in (lambda: layers.share(0, 0, 1), lambda: layers.join(1, 0), lambda: layers.release(0)):
        with pytest.raises(ValueError):
            call()


PRODUCERS = [                              # kind, what it reads and writes of 3 rows of 192 values: name, type, values a row
    (bl.BL_PROD_BF16, dict(in0=(torch.bfloat16, 192)), {}),
    (bl.BL_PROD_F32, dict(in0=(torch.float32, 192)), {}),
    (bl.BL_PROD_RESIDUAL, dict(in0=(torch.float32, 192), in1=(torch.float32, 192), aux_out=(torch.float32, 192)), {}),
    (bl.BL_PROD_RELU2_GATE, dict(in0=(torch.float32, 384)), {}),
    (bl.BL_PROD_ATTN_V, dict(in0=(torch.float32, 320)), dict(n_q=3, n_kv=1, head_dim=64)),
]


@pytest.mark.parametrize("kind, parts, more", PRODUCERS)
def test_product_takes_producers_of_its_rows(lib, kind, parts, more):  # noqa: F811
    """A producer's tensors against the matrix and M: nothing is taken that would be read, or written, past its end, as another type or in another order."""
    m = bl.F8Matrix(torch.zeros(200, 192, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(2, 2))

    def call(M=3, gain=None, norm=True, **other):
        tensors = {name: torch.zeros(3, width, dtype=dtype) for name, (dtype, width) in parts.items()}
        tensors.update(other)
        return bl.F8Linear(m, prod=bl.make_producer(kind, norm=norm, gain=gain, **tensors, **more), M=M)
    assert call().y.shape == (3, 200) and call(M=1).y.shape == (1, 200) and call(gain=torch.zeros(192)).desc.prod.gain
    for bad in (dict(M=4), dict(gain=torch.zeros(191)), dict(gain=torch.zeros(192).double())):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)
    for name, (dtype, width) in parts.items():
        for shape in ((5, width), (width * 3,), (1, 3, width), (3, width // 64, 64)):     # (more rows than are used, and the same values in other shapes)
            call(**{name: torch.zeros(shape, dtype=dtype)})
        wrong = [torch.zeros(2, width, dtype=dtype), torch.zeros(3, width + 64, dtype=dtype), torch.zeros(4, width - 16, dtype=dtype), torch.zeros(width * 3 - 1, dtype=dtype),
                 torch.zeros(3, width + 64, dtype=dtype)[:, :width], torch.zeros(width, 3, dtype=dtype).t(), torch.zeros(1, width, dtype=dtype).expand(3, width),
                 torch.zeros(3, width, dtype=torch.float16), torch.zeros(3, width, dtype=torch.float32 if dtype == torch.bfloat16 else torch.bfloat16)]
        for t in wrong:
            with pytest.raises((TypeError, ValueError)):
                call(**{name: t})
    if "aux_out" in parts:
        call(aux_out=None)


def test_producers_without_tensors_and_refused_ones_are_the_call_s_own(lib):  # noqa: F811
    """What the call itself refuses, with its status, is left to it; so is a descriptor that was filled in by hand."""
    m = bl.F8Matrix(torch.zeros(200, 192, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(2, 2))
    x = torch.zeros(3, 192)
    for prod in (bl.make_producer(9, x), bl.make_producer(bl.BL_PROD_RESIDUAL, x), bl.make_producer(bl.BL_PROD_ATTN_V, x, n_q=3, n_kv=1, head_dim=32)):
        assert lib.bl_f8_linear(ctypes.byref(bl.F8Linear(m, prod=prod, M=3).desc), None) == VALUE
    bl.F8Linear(m, prod=bl.Producer(kind=bl.BL_PROD_F32, in0=x.data_ptr()), M=3)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("kind, parts, more", PRODUCERS)
def test_the_quantiser_s_tensors_hold_its_rows(monkeypatch, native, kind, parts, more):
    """What would be read or written behind the memory of a tensor is refused before anything else, by the native form as by the Python form; views into
    longer memory are taken as before."""
    monkeypatch.setattr(bl, "_native", None if native else bl._PythonForm())
    def call(M=3, gain=None, **other):
        tensors = {name: torch.zeros(3, width, dtype=dtype) for name, (dtype, width) in parts.items()}
        tensors.update((k, other.pop(k)) for k in list(other) if k in tensors)
        bl.bl_quant_act_ex(bl.make_producer(kind, norm=True, gain=gain, **tensors, **more), M, 192, "cpu", **other)
    wrong = [dict(M=4), dict(gain=torch.zeros(191)), dict(q=torch.zeros(2, 192, dtype=torch.int8)), dict(scale=torch.zeros(2)), dict(rowsum=torch.zeros(2, dtype=torch.int32))]
    wrong += [{name: t} for name, (dtype, width) in parts.items()
              for t in (torch.zeros(2, width, dtype=dtype), torch.zeros(3 * width - 1, dtype=dtype), torch.zeros(1, width, dtype=dtype).expand(3, width),
                        torch.zeros(4, width, dtype=dtype)[2:])]
    for bad in wrong:
        with pytest.raises(ValueError, match="bytes"):
            call(**bad)
    hold = (bl._native or bl._first_native()).holds
    x = torch.zeros(9, 4)
    for fits in ((), (None, 5), (x, 144, None, 1 << 40), (x[3:], 96), (x[:, :2], 144), (x[:3], 144)):
        assert hold(*fits) == (-1 if native else NotImplemented) and bl._hold("ab", *fits) is None
    with pytest.raises(ValueError, match="b has 96 bytes, 97"):
        bl._hold("ab", x, 1, x[3:], 97)


@pytest.mark.parametrize("source", [s for s in hip_build.SOURCES if s.endswith(".hip")])
def test_vectors_have_the_alignment_that_their_types_say(source):
    """No kernel hands an address of a lower alignment to an access of a higher one (outputs may begin at any value)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    done = subprocess.run([hipcc, "--offload-arch=gfx950", "-std=c++17", "--cuda-device-only", "-fsyntax-only", "-Werror=align-mismatch", "-I", hip_build.INCLUDE,
                           "-I", hip_build.CSRC, os.path.join(hip_build.CSRC, source)], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-2000:]
