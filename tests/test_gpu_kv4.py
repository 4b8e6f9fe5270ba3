"""The paged 4-bit cache on the GPU: append, read and move bit for bit, attention within its error bound of 64 bits."""
import numpy as np
import pytest
import torch

from paper_2408_08146_b200 import PagedKV4, rope_table
from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class World:
    """A cache of garbage pages, a random page table, and what every slot should hold."""

    more_slots = 0                                       # that a row of the page table has, without a page

    def __init__(self, B, layers, hk, dh, page, capacity, seed=0, first_page=0):
        self.rng = np.random.default_rng(seed)
        self.B, self.L, self.hk, self.dh, self.page, self.cap = B, layers, hk, dh, page, capacity
        per = -(-capacity // page)
        n = B * per + 2 + first_page
        self.cache = PagedKV4(layers, hk, dh, page, n, device=DEV)
        self.cache.pages.fill_(0xFF)                     # codes 15, parameters NaN
        self.table_np = (first_page + self.rng.permutation(B * per + 2)[:B * per].reshape(B, per)).astype(np.int32)
        self.table = ints(np.pad(self.table_np, ((0, 0), (0, self.more_slots // page)), constant_values=-1))
        part = lambda w: np.full((layers, B, per * page, hk, w), np.nan, np.float32)
        self.K, self.V = [part(dh), part(1), part(1), part(dh)], [part(dh), part(1), part(1), part(dh)]
        self.gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.gen, device=DEV).to(dtype)

    def put(self, layer, seq, slot, k, v):
        for store, x in ((self.K, k), (self.V, v)):
            for part, new in zip(store, ref.quantise(x)):
                part[layer, seq, slot] = new

    def plan(self, ctx, count, **kw):
        start = np.concatenate([[0], np.cumsum(count)])
        kw.setdefault("total", int(start[-1]))
        return self.cache.rows(self.table, ints(ctx), row_start=ints(start), max_rows=max(1, max(count)), **kw)

    def where(self, ctx, count):
        seq = np.repeat(np.arange(self.B), count)
        i = np.concatenate([np.arange(n) for n in count]).astype(int)
        return seq, np.asarray(ctx)[seq] + i, i

    def fill(self, ctx, dtype=torch.bfloat16, layers=None, tweak=None):
        """ctx[b] slots of every sequence, without rotation, in parts."""
        for layer in range(self.L) if layers is None else layers:
            n = sum(ctx)
            k, v = self.normal(n, self.hk, self.dh, dtype=dtype), self.normal(n, self.hk, self.dh, dtype=dtype)
            if tweak is not None:
                k, v = tweak(k, v)
            zero = [0] * self.B
            self.cache.append(layer, self.plan(zero, ctx), k, v)
            seq, slot, _ = self.where(zero, ctx)
            self.put(layer, seq, slot, k.float().cpu().numpy(), v.float().cpu().numpy())

    def check_attention(self, layer, q, out, ctx, count, scale, masks=None, kv=None, what=""):
        first, worst = 0, 0.0
        for b in range(self.B):
            n = count[b]
            S = ctx[b] + n if kv is None else kv[b]
            sees = np.zeros((n, S), bool)
            sees[:, :min(ctx[b], S)] = True
            for i in range(n):
                if masks is None:
                    sees[i, :ctx[b] + i + 1] = True
                else:
                    w = min(S - ctx[b], n)
                    if w > 0:
                        sees[i, ctx[b]:ctx[b] + w] = masks[b][i, :w]
            K, V = ([part[layer, b, :S] for part in store] for store in (self.K, self.V))
            r = ref.attention(q[first:first + n].float().cpu().numpy(), K, V, scale, sees)
            worst = max(worst, ref.check(out[first:first + n], *r, q.dtype, f"{what} sequence {b}"))
            first += n
        return worst


@pytest.fixture(params=[0, 1 << 17], ids=["short_tables", "long_tables"])
def tables(request, monkeypatch):
    """Which kernel attends goes by the slots that a page-table row names: just those in use, or many more."""
    monkeypatch.setattr(World, "more_slots", request.param)


def same(got, want, what):
    got, want = got.float().cpu().numpy(), np.asarray(want, np.float32)
    ok = (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), f"{what}: {(~ok).sum()} of {ok.size} differ, first at {np.argwhere(~ok)[:3].tolist()}"


@pytest.mark.parametrize("dh,page,hq,hk,ctx,count,dtype", [
    (128, 16, 8, 2, [0, 5, 40], [1, 33, 17], "bf16"),
    (64, 32, 4, 4, [31, 0], [2, 70], "fp16"),
    (128, 64, 3, 3, [100], [1], "fp32"),
    (64, 16, 6, 1, [15, 16, 17, 0], [1, 0, 16, 3], "bf16"),
    (128, 1024, 2, 1, [1000, 3], [50, 1], "fp32"),
])
def test_append_and_read_bit_for_bit(dh, page, hq, hk, ctx, count, dtype):
    t = TYPES[dtype]
    w = World(len(ctx), 2, hk, dh, page, max(a + n for a, n in zip(ctx, count)) + 1)
    total = sum(count)
    # q, k and v as parts of one wider row, as a Q/K/V multiply leaves them
    wide = w.normal(total, (hq + 2 * hk) * dh + 8, dtype=t)
    q, k, v = (wide[:, a * dh:b * dh].unflatten(1, (-1, dh)) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    table = rope_table(3000, dh, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rows = w.plan(ctx, count, status=status)
    seq, slot, _ = w.where(ctx, count)
    pos = (slot * 2 + 7) % 3000
    qn, kn, vn = (x.float().cpu().numpy() for x in (q, k, v))
    tab = table.cpu().numpy()
    for p, given in ((pos, ints(pos)), (slot, None)):
        out = w.cache.append(1, rows, k, v, rope=table, pos=given, q=q)
        same(out, torch.from_numpy(ref.rotate(qn, tab, p)).to(t).float().numpy(), "queries")
        w.put(1, seq, slot, ref.rotate(kn, tab, p), vn)
        for rt in (torch.float32, torch.bfloat16, torch.float16):
            gk, gv = w.cache.read(rows, layer=1, dtype=rt)
            same(gk, torch.from_numpy(w.K[3][1, seq, slot]).to(rt).float().numpy(), "keys")
            same(gv, torch.from_numpy(w.V[3][1, seq, slot]).to(rt).float().numpy(), "values")
    # in place, and nothing rotated
    before = q.clone()
    w.cache.append(0, rows, k, v, q=q, q_out=q)
    same(q, before.float().cpu().numpy(), "queries without a table")
    w.put(0, seq, slot, kn, vn)
    out = w.cache.append(1, rows, k, v, rope=table, q=q, q_out=q)
    assert out is q
    same(q, torch.from_numpy(ref.rotate(qn, tab, slot)).to(t).float().numpy(), "queries in place")
    # both layers at once
    gk, gv = w.cache.read(rows, dtype=torch.float32)
    for layer in range(2):
        same(gk[layer], w.K[3][layer, seq, slot], "keys of every layer")
        same(gv[layer], w.V[3][layer, seq, slot], "values of every layer")
    assert int(status) == 0


def test_odd_vectors():
    """Constant, zero, tiny, huge, far off zero; infinities and NaN make their vector NaN and no other."""
    for dh in (64, 128):
        w = World(1, 1, 2, dh, 16, 40)
        x = w.normal(20, 2, dh)
        x[0], x[1], x[2] = 0.0, 1.25, -3.1415927
        x[3] *= 1e-38
        x[4] *= 1e-30
        x[5] *= 1e37
        x[6] = x[6] + 1000
        x[7] = x[7] - 1e5
        x[8, 0, 3], x[9, 1, dh - 1], x[10, 0, 0] = float("inf"), float("nan"), float("-inf")
        x[11, :, 0], x[11, :, 1] = 3e38, -3e38
        x[12] = -0.0
        x[13] = torch.where(x[13] > 0, 1.0, -1.0)
        x[14, 0] = 1e-44
        v = x.flip(0).contiguous()
        rows = w.plan([3], [20])
        w.cache.append(0, rows, x, v)
        w.put(0, np.zeros(20, int), np.arange(3, 23), x.cpu().numpy(), v.cpu().numpy())
        gk, gv = w.cache.read(rows, layer=0, dtype=torch.float32)
        same(gk, w.K[3][0, 0, 3:23], "keys")
        same(gv, w.V[3][0, 0, 3:23], "values")
        assert np.isnan(w.K[3][0, 0, 3 + 8, 0]).all() and not np.isnan(w.K[3][0, 0, 3 + 8, 1]).any()


@pytest.mark.parametrize("dh", [64, 128])
def test_codes_and_scales_are_those_of_a_division(dh):
    """Ranges of every size, and numbers half way between two codes or next to it: the kernel's quotients round as a division does."""
    n, hk = 1500, 3
    w = World(1, 1, hk, dh, 64, n)
    rng = np.random.default_rng(dh)
    size = np.exp2(rng.uniform(-98, 120, (2, n, hk, 1)))
    x = (rng.uniform(-1, 1, (2, n, hk, dh)) * size + rng.uniform(-4, 4, (2, n, hk, 1)) * size * (rng.random((2, n, hk, 1)) < 0.5)).astype(np.float32)
    # the second half: half-way numbers of the vector's own grid, moved by up to two units in the last place; the ends stay
    _, zero, scale, _ = ref.quantise(x[:, n // 2:])
    half = (zero + scale * (rng.integers(0, 15, x[:, n // 2:].shape) + np.float32(0.5))).astype(np.float32)
    half = np.where(half == 0, half, (half.view(np.int32) + rng.integers(-2, 3, half.shape).astype(np.int32)).view(np.float32))
    lo, hi = x[:, n // 2:].min(-1, keepdims=True), x[:, n // 2:].max(-1, keepdims=True)
    half = np.clip(half, lo, hi)
    half[..., :1], half[..., 1:2] = lo, hi
    x[:, n // 2:] = half
    k, v = (torch.from_numpy(np.ascontiguousarray(t)).to(DEV) for t in x)
    rows = w.plan([0], [n])
    w.cache.append(0, rows, k, v)
    w.put(0, np.zeros(n, int), np.arange(n), x[0], x[1])
    gk, gv = w.cache.read(rows, layer=0, dtype=torch.float32)
    same(gk, w.K[3][0, 0, :n], "keys")
    same(gv, w.V[3][0, 0, :n], "values")


def test_slots_of_their_own():
    """Rows at given slots: negative ones are left out, of two with the same slot the last one is kept."""
    w = World(2, 1, 2, 128, 16, 64)
    count, slot = [5, 6], [7, 3, -1, 7, 20, 0, 63, 0, 0, -5, 31]
    k, v, q = w.normal(11, 2, 128), w.normal(11, 2, 128), w.normal(11, 4, 128)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rows = w.plan([0, 0], count, slot=ints(slot), status=status)
    q_out = torch.full_like(q, 9.0)
    w.cache.append(0, rows, k, v, q=q, q_out=q_out)
    kept = {}
    for r in range(11):
        if slot[r] >= 0:
            kept[(0 if r < 5 else 1, slot[r])] = r
    gk, gv = w.cache.read(rows, layer=0, dtype=torch.float32, k_out=torch.full_like(k, 5.0), v_out=torch.full_like(v, 5.0))
    for r in range(11):
        if slot[r] < 0:
            assert (gk[r] == 5).all() and (gv[r] == 5).all() and (q_out[r] == 9).all()
        else:
            src = kept[(0 if r < 5 else 1, slot[r])]
            same(gk[r], ref.quantise(k[src].cpu().numpy())[3], f"row {r}")
            same(gv[r], ref.quantise(v[src].cpu().numpy())[3], f"row {r}")
            assert (q_out[r] == q[r]).all()
    assert int(status) == 0


def test_rows_out_of_range_are_left_out_and_reported():
    w = World(2, 1, 1, 64, 16, 32)
    k = w.normal(4, 1, 64)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def run(table, ctx, start, total=4, max_rows=2, rope=None, pos=None, slot=None):
        before = w.cache.pages.clone()
        status.zero_()
        rows = w.cache.rows(ints(table), ints(ctx), row_start=ints(start), total=total, max_rows=max_rows, status=status, slot=slot)
        w.cache.append(0, rows, k, k, rope=rope, pos=pos)
        changed = int((w.cache.pages != before).any())
        return int(status), changed, rows

    good = w.table_np
    assert run(good, [0, 0], [0, 2, 4])[:2] == (0, 1)
    w.cache.pages.fill_(0xFF)
    assert run(good, [31, 32], [0, 1, 1], max_rows=1)[:2] == (0, 1)          # the last slot; a sequence without rows
    w.cache.pages.fill_(0xFF)
    assert run(good, [32, 32], [0, 2, 4])[:2] == (1, 0)                       # behind the table
    assert run(good, [-7, -7], [0, 2, 4])[:2] == (1, 0)
    assert run([[-1, 2], [99, 1]], [0, 0], [0, 2, 4])[:2] == (1, 0)          # no such page
    assert run(good, [0, 0], [0, 3, 3])[:2] == (1, 0)                         # more rows than max_rows
    assert run(good, [0, 0], [2, 1, 1])[:2] == (1, 0)
    assert run(good, [0, 0], [5, 9, 9], max_rows=9)[:2] == (1, 0)             # rows that the tensors do not have
    table = rope_table(4, 64, device=DEV)
    assert run(good, [0, 0], [0, 2, 4], rope=table, pos=ints([4, 4, -1, 7]))[:2] == (1, 0)
    # reading and attending
    _, _, rows = run([[-1, 2], [99, 1]], [0, 0], [0, 2, 4])
    status.zero_()
    out = torch.full_like(k, 3.0)
    w.cache.read(rows, layer=0, k_out=out, v_out=out)
    assert int(status) == 1 and (out == 3).all()
    status.zero_()
    assert (w.cache.attention(0, rows, k) == 0).all() and int(status) == 1    # no slot can be read
    rows = w.cache.rows(w.table, ints([-3, 0]), max_rows=2, status=status)
    status.zero_()
    assert (w.cache.attention(0, rows, k)[:2] == 0).all() and int(status) == 1


ATTENTION = [
    # heads, kv heads, dh, page, context, rows, type, tree
    (4, 4, 128, 16, [0], [1], "bf16", False),
    (4, 4, 128, 16, [577], [1], "bf16", False),
    (8, 2, 64, 32, [1, 15, 16, 17, 300], [1, 1, 1, 1, 1], "fp16", False),
    (32, 8, 128, 64, [3000, 0, 130], [1, 1, 1], "bf16", False),
    (8, 1, 128, 128, [4500], [1], "fp32", False),
    (16, 1, 64, 16, [700, 64], [1, 2], "fp32", False),
    (5, 5, 128, 16, [200, 33], [7, 3], "fp32", False),
    (4, 2, 128, 32, [90], [8], "fp16", False),
    (12, 4, 64, 64, [1000, 0, 20], [4, 5, 0], "bf16", True),
    (2, 2, 128, 16, [511, 48], [60, 64], "fp32", True),
    (3, 3, 128, 64, [1, 640, 63], [64, 128, 17], "bf16", True),
    (2, 1, 64, 16, [100], [128], "fp16", True),
    (8, 2, 128, 32, [260, 0], [150, 77], "bf16", False),
    (4, 4, 64, 16, [33], [200], "fp16", False),
    (28, 4, 128, 16, [127, 640], [20, 31], "fp32", False),
    (1, 1, 128, 16, [16000], [1], "fp16", False),
    (2, 2, 128, 64, [5000], [33], "bf16", True),
    (40, 40, 128, 16, [95, 300, 64, 8], [18, 18, 18, 18], "bf16", True),
    (4, 4, 64, 16, [200, 3], [20, 50], "bf16", True),
    (6, 2, 64, 32, [129], [31], "fp32", True),
    (4, 4, 64, 64, [1000], [40], "fp16", False),
    (1, 1, 64, 16, [0, 63, 64, 65], [17, 17, 1, 64], "fp32", False),
    (64, 64, 128, 16, [30, 2, 70, 0, 17, 90, 64, 1, 33, 5] * 4, [1] * 40, "bf16", False),      # more items than are resident at once
    (16, 8, 128, 16, [127] * 9 + [3], [8] * 10, "fp16", True),
    (2, 2, 128, 16, [250], [16], "fp32", True),                                               # every size of a cluster
    (2, 2, 64, 16, [100], [3], "bf16", True),
]


@pytest.mark.parametrize("hq,hk,dh,page,ctx,count,dtype,tree", ATTENTION)
@pytest.mark.usefixtures("tables")
def test_attention(hq, hk, dh, page, ctx, count, dtype, tree):
    t = TYPES[dtype]
    w = World(len(ctx), 1, hk, dh, page, max(a + n for a, n in zip(ctx, count)))
    # keys with channels of different size and an offset, values far off zero in one head: codes are not centred
    w.fill([a + n for a, n in zip(ctx, count)], tweak=lambda k, v: ((k * torch.linspace(0.3, 2, dh, device=DEV) + 0.5).bfloat16(), (v + 3 * (torch.arange(hk, device=DEV) == 0)[:, None]).bfloat16()))
    total = sum(count)
    q = w.normal(total, hq + 1, dh, dtype=t)[:, :hq]                # a stride wider than the heads
    masks = words = None
    if tree:
        both = [ref.tree_masks(n, w.rng) for n in count if n]
        masks = [np.zeros((0, 0), bool)] * len(count)
        for b, m in zip([b for b, n in enumerate(count) if n], both):
            masks[b] = m[0]
        words = torch.from_numpy(np.concatenate([m[1] for m in both])).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rows = w.plan(ctx, count, mask=words, status=status)
    out = torch.full((total + 3, hq, dh), 7.0, dtype=t, device=DEV)
    w.cache.attention(0, rows, q, out=out[:total])
    w.check_attention(0, q, out[:total], ctx, count, dh ** -0.5, masks, what="attention")
    assert (out[total:] == 7).all() and int(status) == 0
    # once more into the queries' own memory: the same bits
    w.cache.attention(0, rows, q, out=q)
    assert torch.equal(q, out[:total])


@pytest.mark.parametrize("hq,hk,dh,n", [(2, 2, 128, 5), (8, 1, 64, 3), (2, 2, 128, 40), (4, 1, 128, 100)])
@pytest.mark.usefixtures("tables")
def test_masks_that_leave_nothing(hq, hk, dh, n):
    """No context and an empty mask: 0.  Slots that a row does not see may hold NaN and infinities."""
    w = World(2, 1, hk, dh, 16, 160)
    ctx = [0, 20]
    w.fill([0, 20])
    kv = [n, 20 + n]
    k, v = w.normal(2 * n, hk, dh), w.normal(2 * n, hk, dh)
    k[1], v[1], k[n + 2], v[n + 2] = float("nan"), float("inf"), float("inf"), float("nan")
    rows = w.plan(ctx, [n, n])
    w.cache.append(0, rows, k, v)
    seq, slot, _ = w.where(ctx, [n, n])
    w.put(0, seq, slot, k.cpu().numpy(), v.cpu().numpy())
    see = [np.eye(n, dtype=bool), np.eye(n, dtype=bool)]
    see[0][0, 0] = False                                             # row 0 of sequence 0: nothing
    see[0][1, 1] = False                                             # row 1: not its own NaN either
    see[1][2, 2] = False
    words = np.zeros((2 * n, 128), bool)
    words[:n, :n], words[n:, :n] = see
    mask = torch.from_numpy(np.packbits(words, axis=1, bitorder="little").view(np.int64)).to(DEV)
    for dtype in TYPES.values():
        q = w.normal(2 * n, hq, dh, dtype=dtype)
        out = w.cache.attention(0, w.plan(ctx, [n, n], mask=mask), q)
        assert (out[0] == 0).all() and (out[1] == 0).all() and torch.isfinite(out).all()
        w.check_attention(0, q, out, ctx, [n, n], dh ** -0.5, see, what=str(dtype))
        # a row that does see a NaN vector is NaN, the others keep their bits
        bits = mask.clone()
        bits[0, 0] |= 2
        other = w.cache.attention(0, w.plan(ctx, [n, n], mask=bits), q)
        assert torch.isnan(other[0]).all() and torch.equal(other[1:], out[1:])


@pytest.mark.usefixtures("tables")
def test_lengths_and_unused_rows():
    """kv_len cuts a sequence (to nothing as well); rows with a negative slot give 0; rows behind the last sequence stay."""
    w = World(3, 1, 2, 128, 16, 80)
    w.fill([80, 80, 80])
    for kv in ([0, 1, 80], [16, 17, 15], [33, 70, 64]):
        q = w.normal(12, 4, 128)
        out = torch.full_like(q, 4.0)
        slot = ints([70, 71, -1, 73, 70, -2, 72, 73, 70, 71, 72, 73])
        ctx, count = [70, 70, 70], [4, 4, 4]
        w.cache.attention(0, w.plan(ctx, count, kv_len=ints(kv), slot=slot), q, out=out)
        want = out.clone()
        assert (out[2] == 0).all() and (out[5] == 0).all()
        used = [0, 1, 3, 4, 6, 7, 8, 9, 10, 11]
        plain = w.cache.attention(0, w.plan(ctx, count, kv_len=ints(kv)), q)
        assert torch.equal(plain[used], want[used])
        w.check_attention(0, q, plain, ctx, count, 128 ** -0.5, kv=kv, what=str(kv))
    q = w.normal(9, 2, 128)
    out = torch.full_like(q, 4.0)
    start = ints([2, 3, 3, 7])
    w.cache.attention(0, w.cache.rows(w.table, ints([10, 0, 20]), row_start=start, total=9, max_rows=4), q, out=out)
    assert (out[:2] == 4).all() and (out[7:] == 4).all() and not (out[2:7] == 4).any()


@pytest.mark.parametrize("hq,hk,dh,rows", [(1, 1, 128, 1), (4, 1, 64, 1), (2, 2, 128, 24)])
@pytest.mark.usefixtures("tables")
def test_scores_and_scales_that_grow(hq, hk, dh, rows):
    """Keys whose scores rise along the context and values whose scale jumps by 2^40: references are raised on the way."""
    n = 900
    w = World(1, 1, hk, dh, 16, n + rows)
    q = w.normal(rows, hq, dh)
    q[:] = q[0, 0].abs() + 0.1
    ramp = torch.linspace(-60, 60, n + rows, device=DEV)[:, None, None]
    big = torch.ones(n + rows, device=DEV)
    big[:300], big[300:600] = 2.0 ** -30, 2.0 ** -10
    def tweak(k, v):
        k = k.float() * 0.02 + ramp * q[0, 0] / (q[0, 0].square().sum() * dh ** -0.5)
        return k, v.float() * big[:, None, None]
    w.fill([n + rows], dtype=torch.float32, tweak=tweak)
    for dtype in TYPES.values():
        x = q.to(dtype)
        out = w.cache.attention(0, w.plan([n], [rows]), x)
        w.check_attention(0, x, out, [n], [rows], dh ** -0.5, what=str(dtype))
    # the other way round: the largest first
    w.fill([n + rows], dtype=torch.float32, tweak=lambda k, v: tuple(x.flip(0).contiguous() for x in tweak(k, v)))
    out = w.cache.attention(0, w.plan([n], [rows]), q)
    w.check_attention(0, q, out, [n], [rows], dh ** -0.5, what="falling")


@pytest.mark.usefixtures("tables")
def test_extreme_queries_and_scale():
    w = World(1, 1, 1, 128, 16, 70)
    w.fill([70])
    q = w.normal(6, 1, 128)
    q[0] = 0
    q[1] *= 1e-30
    q[2] *= 30
    q[3, 0, 1:] = 0
    q[4] *= torch.logspace(-30, 0, 128, device=DEV)
    out = w.cache.attention(0, w.plan([64], [6]), q, scale=0.5)
    w.check_attention(0, q, out, [64], [6], 0.5)
    q[5, 0, 7] = float("nan")
    bad = w.cache.attention(0, w.plan([64], [6]), q, scale=0.5)
    assert torch.isnan(bad[5]).all() and torch.equal(bad[:5], out[:5])


def test_attention_of_a_long_cache_behind_4_gb():
    """Pages past 2^32 bytes of a layer, a second layer behind them, 70 000 slots."""
    first = 2 * 1024 * 1024 // 2 + 1000
    w = World(1, 2, 1, 128, 64, 70000 + 1, first_page=first // 2)
    assert w.cache.pages.numel() > 2 ** 33
    w.fill([70000], layers=[1])
    k, v, q = w.normal(1, 1, 128), w.normal(1, 1, 128), w.normal(1, 4, 128)
    rows = w.plan([70000], [1])
    w.cache.append(1, rows, k, v)
    w.put(1, np.array([0]), np.array([70000]), k.cpu().numpy(), v.cpu().numpy())
    for dtype in (torch.float32, torch.float16):
        x = q.to(dtype)
        w.check_attention(1, x, w.cache.attention(1, rows, x), [70000], [1], 128 ** -0.5)
    src, dst = ints([[69999, 5]]), ints([[69000, 70000]])
    w.cache.move(w.table, src, dst)
    gk, _ = w.cache.read(w.cache.rows(w.table, ints([0]), row_start=ints([0, 2]), total=2, max_rows=2, slot=dst.view(-1)), layer=1, dtype=torch.float32)
    same(gk, w.K[3][1, 0, [69999, 5]], "moved")


@pytest.mark.parametrize("dh,page,n", [(128, 16, 5), (64, 64, 128), (128, 32, 1)])
def test_moves(dh, page, n):
    """Chains and swaps of slots, repeated destinations (the last is kept), entries left out, every layer."""
    cap = 200
    w = World(3, 3, 2, dh, page, cap)
    w.fill([cap] * 3)
    src = w.rng.integers(0, cap, (3, n))
    dst = np.stack([w.rng.permutation(cap)[:n] for _ in range(3)])
    if n > 4:
        src[0, :3], dst[0, :3] = [1, 2, 0], [0, 1, 2]                   # a cycle
        dst[1, 4] = dst[1, 0]
        dst[1, 3], src[2, 2], dst[2, 1] = -1, -4, src[2, 1]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    w.cache.move(w.table, ints(src), ints(dst), status=status)
    K, V = w.K[3].copy(), w.V[3].copy()
    for b in range(3):
        for s, d in zip(src[b], dst[b]):
            if s >= 0 and d >= 0:
                K[:, b, d], V[:, b, d] = w.K[3][:, b, s], w.V[3][:, b, s]
    gk, gv = w.cache.read(w.plan([0] * 3, [cap] * 3), dtype=torch.float32)
    for layer in range(3):
        same(gk[layer], K[layer, :, :cap].reshape(-1, 2, dh), "keys")
        same(gv[layer], V[layer, :, :cap].reshape(-1, 2, dh), "values")
    assert int(status) == 0
    w.cache.move(w.table, ints([[0], [0], [1 << 28]]), ints([[1 << 20], [3], [0]]), status=status)
    assert int(status) == 1
    after = w.cache.read(w.plan([0] * 3, [cap] * 3), layer=0, dtype=torch.float32)[0].view(3, cap, 2, dh)
    same(after[[0, 2]], gk[0].view(3, cap, 2, dh)[[0, 2]].cpu().numpy(), "untouched")
    same(after[1, 3], gk[0].view(3, cap, 2, dh)[1, 0].cpu().numpy(), "moved")


@pytest.mark.usefixtures("tables")
def test_the_calls_together_as_a_step_of_decoding():
    """Prompt, tree, acceptance, next token: what a serving loop runs, on two layers, against the definition."""
    B, hq, hk, dh = 2, 8, 4, 128
    w = World(B, 2, hk, dh, 16, 260)
    table, tab = rope_table(300, dh, device=DEV), rope_table(300, dh, device=DEV).cpu().numpy()
    held = [0, 0]

    def forward(count, positions=None, masks=None, words=None):
        rows = w.plan(held, count, mask=words)
        seq, slot, _ = w.where(held, count)
        p = slot if positions is None else positions
        for layer in range(2):
            k, v, q = (w.normal(sum(count), h, dh, dtype=torch.bfloat16) for h in (hk, hk, hq))
            rot = w.cache.append(layer, rows, k, v, rope=table, pos=None if positions is None else ints(p), q=q)
            w.put(layer, seq, slot, ref.rotate(k.float().cpu().numpy(), tab, p), v.float().cpu().numpy())
            out = w.cache.attention(layer, rows, rot)
            w.check_attention(layer, rot, out, held, count, dh ** -0.5, masks, what=f"layer {layer}")

    forward([100, 37])
    held = [100, 37]
    for step in range(3):
        both = [ref.tree_masks(n, w.rng) for n in (20, 9)]
        depth = np.concatenate([m[0].sum(1) - 1 for m in both])
        seq, _, _ = w.where(held, [20, 9])
        forward([20, 9], np.asarray(held)[seq] + depth, [m[0] for m in both], torch.from_numpy(np.concatenate([m[1] for m in both])).to(DEV))
        paths = [np.nonzero(m[0][-1])[0] for m in both]                 # the last node's path is accepted
        src, dst = np.full((B, 20), -1), np.full((B, 20), -1)
        for b, path in enumerate(paths):
            src[b, :len(path)], dst[b, :len(path)] = held[b] + path, held[b] + np.arange(len(path))
        w.cache.move(w.table, ints(src), ints(dst))
        for b, path in enumerate(paths):
            for store in (w.K, w.V):
                for part in store:
                    part[:, b, held[b]:held[b] + len(path)] = part[:, b, held[b] + path]
        held = [held[b] + len(path) for b, path in enumerate(paths)]
        forward([1, 1])
        held = [n + 1 for n in held]


@pytest.mark.parametrize("hq,hk,rows", [(4, 4, 1), (4, 4, 30), (2, 1, 1)])
@pytest.mark.usefixtures("tables")
def test_captured_and_replayed_and_on_another_stream(hq, hk, rows):
    """A step captured into graphs gives the eager bits, with new data in the same buffers; two graphs share a plan; another stream."""
    w = World(2, 1, hk, 128, 64, 4000)
    ctx = [3900, 200]
    w.fill([3950, 250])
    table = rope_table(4000, 128, device=DEV)
    n = 2 * rows
    k, v, q = (w.normal(n, h, 128, dtype=torch.bfloat16) for h in (hk, hk, hq))
    lens = ints(ctx)
    plan = w.cache.rows(w.table, lens, max_rows=rows)
    q_out, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        w.cache.append(0, plan, k, v, rope=table, q=q, q_out=q_out)
        w.cache.attention(0, plan, q_out, out=out)

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for i in range(4):
        for x in (k, v, q):
            x.copy_(w.normal(*x.shape, dtype=torch.bfloat16))
        lens.copy_(ints([3900 - 17 * i, 200 + 3 * i]))
        step()
        want = out.clone()
        out.fill_(0)
        graphs[i % 2].replay()
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = w.cache.attention(0, plan, q_out)
    # two streams at once, each with an output of its own
    here = [w.cache.attention(0, plan, q_out) for _ in range(8)]
    with torch.cuda.stream(side):
        there = [w.cache.attention(0, plan, q_out) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in [again] + here + there)
