"""Key/value cache calls on the host: every refusal comes before any GPU work, sizes are right, and the binding takes
only tensors that a descriptor can stand for.  Needs no GPU."""
import ctypes
import os

import pytest

from paper_2504_12285_amd import binding as bl
from paper_2504_12285_amd import build as hip_build

torch = pytest.importorskip("torch")
NULL, SHAPE, ALIGN, VALUE, WORKSPACE = 1, 2, 4, 5, 7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hip_build.LIB_PATH):
        hip_build.build()
    return bl.load()


BUF = (ctypes.c_char * 8192)()
P = (ctypes.addressof(BUF) + 255) & ~255          # an aligned host address, never dereferenced on a refusal


def cache(**more):
    d = dict(kind=bl.BL_KV_INT8, block=64, n_kv=5, head_dim=128, n_blocks=10, k=P, v=P, k_scale=P, v_scale=P, k_stride=5 * 64 * 128,
             v_stride=5 * 64 * 128, scale_stride=5)
    d.update(more)
    return bl.KVCacheDesc(**d)


BAD_CACHES = [(dict(k=None), NULL), (dict(v_scale=None), NULL), (dict(kind=2), VALUE), (dict(block=48), SHAPE), (dict(block=8), SHAPE), (dict(block=256), SHAPE),
              (dict(head_dim=96), SHAPE), (dict(n_kv=0), SHAPE), (dict(n_blocks=0), SHAPE), (dict(n_blocks=1 << 25), SHAPE),
              (dict(k_stride=5 * 64 * 128 - 16), SHAPE), (dict(v_stride=0), SHAPE), (dict(scale_stride=4), SHAPE), (dict(k=P + 8), ALIGN),
              (dict(v_stride=5 * 64 * 128 + 8), ALIGN), (dict(k_scale=P + 2), ALIGN)]


def tables(**more):
    d = dict(B=4, rows=8, table_stride=6, free_cap=10, block=64, max_blocks=6, **{n: P for n in (
        "seq_len", "new_len", "free_count", "table", "free_list", "seq_len_out", "free_count_out", "start", "q_start", "positions", "slots", "bad")})
    d.update(more)
    return bl.KVBatchDesc(**d)


@pytest.mark.parametrize("more, status", [(dict(seq_len=None), NULL), (dict(bad=None), NULL), (dict(table=None), NULL), (dict(block=24), SHAPE), (dict(B=0), SHAPE),
                                          (dict(B=4097), SHAPE), (dict(rows=0), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(max_blocks=0), SHAPE),
                                          (dict(max_blocks=7), SHAPE), (dict(free_cap=-1), SHAPE), (dict(max_blocks=1 << 26, table_stride=1 << 26), SHAPE),
                                          (dict(slots=P + 1), ALIGN), (dict(free_list=P + 2), ALIGN)])
def test_tables_refuses(lib, more, status):
    assert lib.bl_kv_tables(ctypes.byref(tables(**more)), None) == status
    assert lib.bl_kv_tables(None, None) == NULL


def tokens(c=None, **more):
    d = dict(cache=c or cache(), qkv=P, qkv_stride=30 * 128, q_stride=20 * 128, T=3, n_pos=100, qkv_kind=0, n_q=20, positions=P, slots=P, cos=P,
             sin=P, q_out=P, bad=P)
    d.update(more)
    return bl.KVTokensDesc(**d)


@pytest.mark.parametrize("more, status", [(dict(qkv=None), NULL), (dict(slots=None), NULL), (dict(cos=None), NULL), (dict(positions=None), NULL), (dict(qkv_kind=2), VALUE),
                                          (dict(T=0), SHAPE), (dict(T=(1 << 24) + 1), SHAPE), (dict(n_q=-1), SHAPE), (dict(qkv_stride=30 * 128 - 4), SHAPE),
                                          (dict(n_pos=0), SHAPE), (dict(q_stride=20 * 128 - 8), SHAPE), (dict(n_q=0), SHAPE), (dict(qkv=P + 8), ALIGN),
                                          (dict(qkv_stride=30 * 128 + 2), ALIGN), (dict(qkv_kind=1, qkv_stride=30 * 128 + 4), ALIGN), (dict(q_out=P + 8), ALIGN),
                                          (dict(q_stride=20 * 128 + 4), ALIGN), (dict(slots=P + 2), ALIGN), (dict(cos=P + 4), ALIGN)])
def test_append_refuses(lib, more, status):
    assert lib.bl_kv_append(ctypes.byref(tokens(**more)), None) == status
    assert lib.bl_kv_append(None, None) == NULL


def attention(c=None, **more):
    d = dict(cache=c or cache(), q=P, q_stride=20 * 128, out_stride=20 * 128, table_stride=6, B=4, T=7, q_start=P, seq_len=P, table=P, n_q=20,
             max_blocks=6, max_q=4, max_len=0, window=0, softmax_scale=0.1, out=P, workspace=P)
    d.update(more)
    return bl.AttnDesc(**d)


BAD_ATTENTION = [(dict(q=None), NULL), (dict(q_start=None), NULL), (dict(seq_len=None), NULL), (dict(table=None), NULL), (dict(out=None), NULL), (dict(B=0), SHAPE),
                 (dict(B=4097), SHAPE), (dict(T=0), SHAPE), (dict(n_q=18), SHAPE), (dict(n_q=0), SHAPE), (dict(max_blocks=7), SHAPE), (dict(max_blocks=0), SHAPE),
                 (dict(max_blocks=1 << 25, table_stride=1 << 25), SHAPE), (dict(max_q=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(window=-1), SHAPE),
                 (dict(q_stride=20 * 128 - 8), SHAPE), (dict(out_stride=0), SHAPE), (dict(softmax_scale=0.0), VALUE), (dict(softmax_scale=-1.0), VALUE),
                 (dict(softmax_scale=float("nan")), VALUE), (dict(softmax_scale=float("inf")), VALUE), (dict(q=P + 8), ALIGN), (dict(out=P + 2), ALIGN),
                 (dict(q_stride=20 * 128 + 4), ALIGN), (dict(seq_len=P + 1), ALIGN)]


@pytest.mark.parametrize("more, status", BAD_ATTENTION)
def test_attention_refuses(lib, more, status):
    a = attention(**more)
    assert lib.bl_attn_kv8(ctypes.byref(a), None) == status
    assert lib.bl_attn_workspace_bytes(ctypes.byref(a)) == 0
    assert lib.bl_attn_kv8(None, None) == NULL


def test_attention_wants_its_workspace(lib):
    assert lib.bl_attn_kv8(ctypes.byref(attention(workspace=None)), None) == WORKSPACE
    assert lib.bl_attn_kv8(ctypes.byref(attention(workspace=P + 16)), None) == ALIGN
    few, split = (lib.bl_attn_workspace_bytes(ctypes.byref(attention(**m))) for m in (dict(), dict(max_q=7, max_blocks=500, table_stride=500)))
    assert 0 < few < split


@pytest.mark.parametrize("more, status", BAD_CACHES)
def test_a_bad_cache_is_refused_by_both_of_its_users(lib, more, status):
    assert lib.bl_kv_append(ctypes.byref(tokens(cache(**more))), None) == status
    assert lib.bl_attn_kv8(ctypes.byref(attention(cache(**more))), None) == status


def test_descriptors_have_the_size_of_the_header_s():
    assert [ctypes.sizeof(c) for c in (bl.KVCacheDesc, bl.KVBatchDesc, bl.KVTokensDesc, bl.AttnDesc)] == [80, 136, 176, 192]


def test_the_binding_takes_what_a_descriptor_can_stand_for(lib):
    i32 = torch.int32
    k, s = torch.zeros(6, 2, 16, 64, dtype=torch.int8), torch.zeros(6, 2)
    v = torch.zeros(6, 2, 64, 16, dtype=torch.int8)
    c = bl.KVCache(k, v, s, s.clone())
    assert (c.desc.k_stride, c.desc.v_stride, c.desc.scale_stride) == (2048, 2048, 2)
    pool = torch.zeros(6, 3, 2, 16, 64, dtype=torch.int8)                     # three layers' blocks side by side
    assert bl.KVCache(pool[:, 1], v, s, s.clone()).desc.k_stride == 3 * 2048
    for bad in ((v, v, s, s), (k, k, s, s), (k, v, s.double(), s), (k.transpose(2, 3), v, s, s), (k[:, :1], v[:, :1], s[:, :1], s[:, :1].clone().t()),
                (k.float(), v, s, s), (k, v.to(torch.uint8), s, s), (k[:, :, ::2], v, s, s)):
        with pytest.raises((TypeError, ValueError)):
            bl.KVCache(*bad)
    n = torch.zeros(3, dtype=i32)
    table = torch.zeros(3, 4, dtype=i32)
    t = bl.KVTables(n, n, table, torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5)
    assert t.seq_len_out is not n and t.q_start.shape == (4,) and t.slots.shape == (5,)
    assert bl.KVTables(n, n, table, torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5, in_place=True).seq_len_out is n
    with pytest.raises(TypeError):
        bl.KVTables(n.long(), n, table, torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5)
    with pytest.raises(ValueError):
        bl.KVTables(n, n, table[:2], torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5)
    qkv = torch.zeros(5, 8 * 64)
    slots = torch.zeros(5, dtype=i32)
    assert bl.KVAppend(c, qkv, 4, slots).q.shape == (5, 256)
    wide = torch.zeros(5, 600)[:, :512]
    assert bl.KVAppend(c, wide, 4, slots).desc.qkv_stride == 600
    cos = torch.zeros(7, 32)
    for bad in ((c, qkv, 3, slots), (c, qkv.half(), 4, slots), (c, qkv, 4, slots.long()), (c, qkv, 4, slots[:4]), (c, qkv, 4, slots, slots, cos, None),
                (c, qkv, 4, slots, None, cos, cos), (c, qkv, 4, slots, slots, cos[:, :31], cos)):
        with pytest.raises((TypeError, ValueError)):
            bl.KVAppend(*bad)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    start = torch.zeros(4, dtype=i32)
    a = bl.KVAttention(c, q, start, n, table, max_q=3)
    assert a.out.shape == (5, 256) and a.desc.n_q == 4 and abs(a.desc.softmax_scale - 0.125) < 1e-9
    assert bl.KVAttention(c, q.view(5, 256), start, n, table, n_q=4).desc.q_stride == 256
    for bad in (dict(q=q.float()), dict(q_start=n), dict(q=q[..., ::2]), dict(table=table[:2]), dict(seq_len=n.long()), dict(out=q),
                dict(workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            bl.KVAttention(**dict(dict(cache=c, q=q, q_start=start, seq_len=n, table=table), **bad))


@pytest.mark.parametrize("limit, more, status", [(0, {}, SHAPE), (-3, {}, SHAPE), (1, dict(seq_len=None), NULL), (1, dict(B=0), SHAPE), (1 << 40, dict(block=24), SHAPE),
                                                 (5, dict(slots=P + 1), ALIGN)])
def test_tables_with_a_limit_refuse(lib, limit, more, status):
    assert lib.bl_kv_tables_limited(ctypes.byref(bl.KVLimitedBatchDesc(tables(**more), limit)), None) == status
    assert lib.bl_kv_tables_limited(None, None) == NULL


def test_a_limit_stands_in_the_handle_and_in_the_layers(lib):
    from paper_2504_12285_amd import serve
    i32 = torch.int32
    n = torch.zeros(3, dtype=i32)
    args = (n, n, torch.zeros(3, 4, dtype=i32), torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5)
    assert ctypes.sizeof(bl.KVLimitedBatchDesc) == 144
    assert isinstance(bl.KVTables(*args).desc, bl.KVBatchDesc)
    h = bl.KVTables(*args, max_new=2)
    assert h.desc.max_new == 2 and h.desc.batch.rows == 5 and h._where == "bl_kv_tables_limited"
    layers = serve.CachedLayers([{}], [{}], requests=2, rows=6, max_blocks=3, n_blocks=6, device="cpu", max_new=4)
    assert layers.tables.desc.max_new == 4 and layers.attend[0].desc.max_q == 4
    free = serve.CachedLayers([{}], [{}], requests=2, rows=6, max_blocks=3, n_blocks=6, device="cpu")
    assert isinstance(free.tables.desc, bl.KVBatchDesc) and free.attend[0].desc.max_q == 6


def test_the_time_of_prompts_is_that_of_their_step_alone(monkeypatch):
    """What the places held ends, and is waited for, before the clock is read: the time between its two readings holds one step, the prompts'."""
    from paper_2504_12285_amd import serve
    log = []

    class Layers:
        def step(self, x, new_len):
            log.append(new_len.tolist())
            return x

    def clock():
        log.append("clock")
        return 3.0 * log.count("clock")
    monkeypatch.setattr(serve.torch.cuda, "synchronize", lambda: log.append("wait"))
    monkeypatch.setattr(serve.time, "perf_counter", clock)
    x, lens = torch.zeros(7, 2560), torch.tensor([4, 3], dtype=torch.int32)
    seconds, y = serve.time_prompts(Layers(), x, lens)
    assert log == [[-1, -1], "wait", "clock", [4, 3], "wait", "clock"] and seconds == 3.0 and y is x


@pytest.mark.parametrize("more", [dict(), dict(window=100, max_blocks=500, table_stride=500), dict(max_q=7, max_len=300)])
def test_items_need_no_room_for_partial_results(lib, more):
    """Short contexts and short windows leave nothing to join: 256 bytes, and a split's own pieces where there is one."""
    a = attention(**more)
    T, n_q, D = a.T, a.n_q, a.cache.head_dim
    assert (lib.bl_attn_workspace_bytes(ctypes.byref(a)) - 256) % (T * n_q * (D + 2) * 4) == 0
    assert lib.bl_attn_workspace_bytes(ctypes.byref(a)) < 1 << 20
    streams = attention(max_blocks=500, table_stride=500)
    assert lib.bl_attn_workspace_bytes(ctypes.byref(streams)) == 256 + 2048 * 2 * 16 * 130 * 4


def test_calls_without_rows_are_refused_as_others_are(lib):
    """No token, no request, no block: the handle stands, and the call says that it is refused."""
    i32 = torch.int32

    def new(n):
        return [torch.zeros(n, 2, 16, 64, dtype=torch.int8), torch.zeros(n, 2, 64, 16, dtype=torch.int8), torch.zeros(n, 2), torch.zeros(n, 2)]
    none, c = torch.zeros(0, dtype=i32), bl.KVCache(*new(3))
    t = bl.KVTables(none, none, torch.zeros(0, 4, dtype=i32), torch.zeros(9, dtype=i32), torch.zeros(1, dtype=i32), 16, 5)
    assert lib.bl_kv_tables(ctypes.byref(t.desc), None) in (NULL, SHAPE)
    a = bl.KVAppend(c, torch.zeros(0, 8 * 64), 4, none)
    assert lib.bl_kv_append(ctypes.byref(a.desc), None) in (NULL, SHAPE)
    a = bl.KVAppend(bl.KVCache(*new(0)), torch.zeros(2, 8 * 64), 4, torch.zeros(2, dtype=i32))
    assert lib.bl_kv_append(ctypes.byref(a.desc), None) in (NULL, SHAPE)
    for q, b in ((0, 3), (5, 0)):
        h = bl.KVAttention(c, torch.zeros(q, 4, 64, dtype=torch.bfloat16), torch.zeros(b + 1, dtype=i32), torch.zeros(b, dtype=i32), torch.zeros(b, 4, dtype=i32))
        assert lib.bl_attn_kv8(ctypes.byref(h.desc), None) in (NULL, SHAPE)


@pytest.mark.parametrize("x, new_len", [((1, 2560), (2,)), ((2560,), (2,)), ((6, 1), (2,)), ((6, 2560), (1,)), ((6, 2560), ()), ((5, 2560), (2,)), ((6, 2560), (3,))])
def test_a_step_of_other_shapes_is_refused(lib, x, new_len):
    """One row is no batch: it is not repeated for all of them."""
    from paper_2504_12285_amd import serve
    layers = serve.CachedLayers([{}], [{}], requests=2, rows=6, max_blocks=3, n_blocks=6, device="cpu")
    with pytest.raises(ValueError):
        layers.step(torch.ones(x), torch.ones(new_len, dtype=torch.int32))
    assert not layers.x.any() and not layers.new_len.any()


def test_a_limit_of_none_stays_none(lib):
    from paper_2504_12285_amd import serve
    layers = serve.CachedLayers([{}], [{}], requests=2, rows=6, max_blocks=3, n_blocks=6, device="cpu", max_new=0)
    assert isinstance(layers.tables.desc, bl.KVBatchDesc) and layers.attend[0].desc.max_q == 6
