"""Refusals of the paged 4-bit cache's calls, before anything reaches a device (no GPU needed)."""
import ctypes as C
import struct

import numpy as np
import pytest
import torch

from paper_2408_08146_b200 import KoalaError, PagedKV4
from paper_2408_08146_b200 import kv4 as m
from tests.kv4_reference import floor_bf16, quantise

INVALID, UNSUPPORTED, CAPACITY = 1, 2, 3


def cache_c(**kw):
    f = {"n_layers": 2, "n_kv_heads": 4, "head_dim": 128, "page_size": 16, "n_pages": 8, "pages": 1 << 20}
    f.update(kw)
    return m.koala_kv4(C.sizeof(m.koala_kv4), *(f[n] for n in ("n_layers", "n_kv_heads", "head_dim", "page_size", "n_pages", "pages")))


def rows_c(**kw):
    f = {"B": 2, "total": 2, "max_rows": 1, "table_stride": 4, "page_table": 4096, "ctx_len": 4096, "row_start": None, "kv_len": None, "slot": None,
         "mask": None, "status": None}
    f.update(kw)
    return m.koala_kv4_rows(C.sizeof(m.koala_kv4_rows), *(f[n] for n, _ in m.koala_kv4_rows._fields_[1:]))


def tensors(*t):
    return struct.pack(f"{3 * len(t)}q", *[x for one in t for x in one])


GOOD = (4096, 512, 128)


def append(c, r, dtype=1, t=(GOOD, GOOD, GOOD, GOOD), layer=0, heads=4, rope=4096, n_pos=9):
    return m._library().koala_kv4_append(C.byref(c), layer, C.byref(r), dtype, tensors(*t), heads, rope, n_pos, None, None)


def attention(c, r, dtype=1, t=(GOOD, GOOD), layer=0, heads=4, scale=0.1):
    return m._library().koala_kv4_attention(C.byref(c), layer, C.byref(r), dtype, tensors(*t), heads, scale, None, 0, None)


def test_bytes_of_a_cache():
    n = lambda **kw: int(m._library().koala_kv4_bytes(C.byref(cache_c(**kw))))
    assert n() == 2 * 8 * 4 * (16 * 128 + 128)
    assert n(head_dim=64, page_size=64) == 2 * 8 * 4 * 4 * (16 * 64 + 128)
    for bad in ({"head_dim": 96}, {"page_size": 8}, {"page_size": 48}, {"page_size": 2048}, {"n_layers": 0}, {"n_kv_heads": 0}, {"n_pages": 0}):
        assert n(**bad) == 0, bad
    c = cache_c()
    c.struct_size -= 4
    assert int(m._library().koala_kv4_bytes(C.byref(c))) == 0
    assert int(m._library().koala_kv4_bytes(None)) == 0


@pytest.mark.parametrize("call", [append, attention])
def test_bad_descriptions_are_refused(call):
    for bad in ({"pages": None}, {"pages": (1 << 20) + 64}, {"head_dim": 80}, {"page_size": 24}):
        assert call(cache_c(**bad), rows_c()) == INVALID, bad
    for bad in ({"page_table": None}, {"ctx_len": None}, {"B": 0}, {"total": -1}, {"max_rows": 0}, {"table_stride": 0}, {"total": 3}, {"table_stride": 1 << 29},
                {"B": 65535, "total": 65535}, {"mask": 4100}):
        assert call(cache_c(), rows_c(**bad)) == INVALID, bad
    for extra in ("slot", "mask"):
        assert call(cache_c(), rows_c(max_rows=129, total=258, **{extra: 4096})) == UNSUPPORTED
    for layer in (-1, 2):
        assert call(cache_c(), rows_c(), layer=layer) == INVALID
    for dtype in (-1, 3):
        assert call(cache_c(), rows_c(), dtype=dtype) == INVALID
    n = 4 if call is append else 2
    for bad in ((0, 512, 128), (4098, 512, 128), (4096, 510, 128), (4096, 512, 126)):
        for i in range(n):
            if call is append and i == 2 and bad[0] == 0:
                continue                                   # no queries
            t = [GOOD] * n
            t[i] = bad
            assert call(cache_c(), rows_c(), t=t) == INVALID, (i, bad)
    assert call(cache_c(), rows_c(), heads=0) == INVALID
    assert call(cache_c(), rows_c(), dtype=0, t=[(4104, 512, 128)] + [GOOD] * (n - 1)) == INVALID       # fp32: 16 bytes


def test_more_refusals():
    assert append(cache_c(), rows_c(), n_pos=0) == INVALID
    assert append(cache_c(), rows_c(), rope=4100) == INVALID
    assert attention(cache_c(), rows_c(), heads=6) == INVALID          # not a multiple of the kv heads
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attention(cache_c(), rows_c(), scale=scale) == INVALID
    lib = m._library()
    assert lib.koala_kv4_read(C.byref(cache_c()), 2, C.byref(rows_c()), 1, tensors(GOOD, GOOD), None, None) == INVALID
    assert lib.koala_kv4_read(C.byref(cache_c()), -1, C.byref(rows_c()), 1, tensors(GOOD, GOOD), None, None) == INVALID      # no layer strides
    move = lambda **kw: lib.koala_kv4_move(*[{"c": C.byref(cache_c()), "B": 1, "table": 4096, "stride": 4, "n": 2, "src": 4096, "dst": 4096,
                                             "status": None, "stream": None, **kw}[x] for x in ("c", "B", "table", "stride", "n", "src", "dst", "status", "stream")])
    assert move(B=0) == INVALID and move(table=None) == INVALID and move(n=-1) == INVALID and move(src=None) == INVALID and move(dst=None) == INVALID
    assert move(n=129) == UNSUPPORTED
    # nothing to do is no error
    assert move(n=0) == 0
    empty = rows_c(total=0, row_start=4096)
    assert append(cache_c(), empty) == 0 and attention(cache_c(), empty) == 0
    assert lib.koala_kv4_read(C.byref(cache_c()), 0, C.byref(empty), 1, tensors(GOOD, GOOD), None, None) == 0


def test_scratch_of_the_attention():
    lib = m._library()
    n = lambda heads=4, **kw: int(lib.koala_kv4_attention_scratch_bytes(C.byref(cache_c()), C.byref(rows_c(**kw)), heads))
    assert n() > 0 and n(total=0, row_start=4096) == 0 and n(heads=6) == 0 and n(B=0) == 0
    call = lambda at, size: lib.koala_kv4_attention(C.byref(cache_c()), 0, C.byref(rows_c()), 1, tensors(GOOD, GOOD), 4, 0.1, at, size, None)
    assert call(None, n()) == CAPACITY and call(4096, n() - 1) == CAPACITY and call(4100, n()) == INVALID
    assert lib.koala_kv4_attention(C.byref(cache_c()), 0, C.byref(rows_c(max_rows=1 << 20, total=1, row_start=4096)), 1, tensors(GOOD, GOOD), 4, 0.1, 4096, 1 << 40, None) == UNSUPPORTED


def test_no_rows_need_no_tensors():
    """A step without rows passes, whatever an empty tensor's address is; what else is wrong is still refused."""
    none, empty = (0, 512, 128), rows_c(total=0, row_start=4096)
    assert append(cache_c(), empty, t=(none, none, none, none)) == 0
    assert attention(cache_c(), empty, t=(none, none)) == 0
    assert m._library().koala_kv4_read(C.byref(cache_c()), 0, C.byref(empty), 1, tensors(none, none), None, None) == 0
    move = lambda n, at: m._library().koala_kv4_move(C.byref(cache_c()), 2, 4096, 4, n, at, at, None, None)
    assert move(0, None) == 0 and move(1, None) == INVALID
    assert append(cache_c(), empty, t=(none,) * 4, layer=2) == INVALID
    assert attention(cache_c(), empty, t=(none, none), heads=3) == INVALID


def test_more_work_than_is_counted():
    """Units of work are counted in 32 bits."""
    for c, r in ((cache_c(n_kv_heads=1), rows_c(B=60000, total=60000, table_stride=1 << 26)),
                 (cache_c(n_kv_heads=1), rows_c(B=1, total=1 << 30, max_rows=1 << 30)),
                 (cache_c(n_kv_heads=8), rows_c(B=8000, total=8000 * 128, max_rows=128, table_stride=1 << 18))):      # 64000 heads, 2 tiles, 65544 units
        assert attention(c, r, heads=c.n_kv_heads) == UNSUPPORTED
        assert int(m._library().koala_kv4_attention_scratch_bytes(C.byref(c), C.byref(r), c.n_kv_heads)) == 0
    # as many sequences of as many slots are fine one by one
    assert attention(cache_c(n_kv_heads=1), rows_c(B=60000, total=60000, table_stride=16), heads=1) == CAPACITY       # (no scratch)
    assert attention(cache_c(n_kv_heads=1), rows_c(B=1, total=1, table_stride=1 << 26), heads=1) == CAPACITY


def test_rows_belong_to_caches_of_one_shape():
    memory = torch.zeros(1 << 16, dtype=torch.uint8)
    memory = memory[-memory.data_ptr() % 128:]
    make = lambda **kw: PagedKV4(**{**dict(n_layers=1, n_kv_heads=2, head_dim=64, page_size=16, n_pages=4, device="cpu", pages=memory), **kw})
    table, ctx = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    rows = make().rows(table, ctx)
    for other in (make(n_kv_heads=4), make(head_dim=128), make(page_size=32)):
        shape = torch.zeros(1, other.n_kv_heads, other.head_dim)
        with pytest.raises(ValueError):
            other.append(0, rows, shape, shape)
        with pytest.raises(ValueError):
            other.attention(0, rows, shape)
        with pytest.raises(ValueError):
            other.read(rows)


def test_the_binding_checks_its_tensors():
    with pytest.raises(KoalaError):
        PagedKV4(1, 2, 100, 16, 4, device="cpu")
    with pytest.raises(ValueError, match="pages"):
        PagedKV4(1, 2, 64, 16, 4, device="cpu", pages=torch.zeros(100, dtype=torch.uint8))
    n = 4 * 2 * (16 * 64 + 128)
    memory = torch.zeros(n + 128, dtype=torch.uint8)
    at = -memory.data_ptr() % 128
    c = PagedKV4(1, 2, 64, 16, 4, device="cpu", pages=memory[at:at + n])
    ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    with pytest.raises(ValueError, match="page_table"):
        c.rows(ints(2), ints(2))
    with pytest.raises(ValueError, match="ctx_len"):
        c.rows(ints(2, 3), ints(3))
    with pytest.raises(ValueError, match="total"):
        c.rows(ints(2, 3), ints(2), row_start=ints(3))
    with pytest.raises(ValueError, match="total"):
        c.rows(ints(2, 3), ints(2), total=5, max_rows=2)
    with pytest.raises(ValueError, match="128"):
        c.rows(ints(2, 3), ints(2), max_rows=200, slot=ints(400))
    with pytest.raises(ValueError, match="mask"):
        c.rows(ints(2, 3), ints(2), max_rows=2, mask=ints(4, 2))
    rows = c.rows(ints(2, 3), ints(2), max_rows=2)
    assert rows.total == 4
    x = torch.zeros(4, 2, 64)
    for k, v in ((x[:3], x), (x, x.bfloat16()), (x.transpose(0, 1), x), (torch.zeros(4, 2, 128)[..., ::2], x), (x.double(), x.double()),
                 (torch.zeros(4, 2, 66)[..., 1:65], x)):
        with pytest.raises(ValueError):
            c.append(0, rows, k, v)
    with pytest.raises(ValueError, match="rope"):
        c.append(0, rows, x, x, rope=torch.zeros(9, 64, 2))
    with pytest.raises(ValueError):
        c.attention(0, rows, x[:, :, :32])
    with pytest.raises(ValueError):
        c.move(ints(1, 3), ints(1, 200), ints(1, 200))


def test_the_reference_quantisation():
    """Half a step: every finite value lies within scale / 2 (and fp32 rounding) of what it is held as, whatever the offset."""
    rng = np.random.default_rng(0)
    for off, size in ((0, 1), (100, 1), (-1e4, 3), (1e-30, 1e-30), (3e38, 1e37), (0, 0)):
        x = (off + size * rng.standard_normal((50, 64))).astype(np.float32)
        code, zero, scale, value = quantise(x)
        assert (np.abs(value - x) <= 0.5 * scale * (1 + 2.0 ** -20) + 2.0 ** -22 * np.abs(x) + 2.0 ** -96).all()
        assert (zero <= x.min(-1, keepdims=True)).all() and ((zero + 15 * scale) >= x.max(-1, keepdims=True) * (1 - np.sign(x.max(-1, keepdims=True)) * 2.0 ** -22) - 2.0 ** -96).all()
    assert (floor_bf16(np.float32([1.0, 1.001, -1.001, 0.0])) == np.float32([1.0, 1.0, -1.0078125, 0.0])).all()
    for bad in (np.inf, -np.inf, np.nan):
        x = np.zeros((1, 64), np.float32)
        x[0, 5] = bad
        assert np.isnan(quantise(x)[3]).all()
    assert np.isnan(quantise(np.float32([[-3e38, 3e38] * 32]))[3]).all()
