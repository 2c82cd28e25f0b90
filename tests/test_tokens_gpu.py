"""New tokens into the bf16 and the 8-bit cache, and rows of the 8-bit cache read back, against 64-bit forms.

Error bound of a prepared query or key (roundings are half a step: fp32 2^-24, bf16 2^-8 relative).  Norm: 128 additions of squares,
2^-17 of their sum, so 2^-18 of its root; the reciprocal root (2 ulp), two products: below 1.2 * 2^-18 of the value.  Rotation: cosine
and sine are off by 2^-22 (2 ulp, an angle held to 2^-28 turns, a factor) and by the angle's own three fp64 roundings, 2^-51 |angle|;
two roundings of the sum: (2^-17 + 2^-51 |angle|) (|a| + |b|) in all.  The result's rounding: 2^-8 |y|, and 2^-134.
"""
import math

import numpy as np
import pytest
import torch

from paper_2602_08329_b200 import binding as P
from tests.test_byte_cache_gpu import DTYPE, Cache, np64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


class Batch:
    """New tokens of a ragged batch, packed, with a bf16 cache; what holds nothing is NaN."""

    def __init__(self, dev, lens, new, kv_heads, group, paged, pad_rows=3, seed=0, amp=1.0):
        g = torch.Generator().manual_seed(seed)
        self.dev, self.lens, self.new, self.H, self.G, self.paged = dev, lens, new, kv_heads, group, paged
        self.B, self.Hq = len(lens), kv_heads * group
        self.starts = [sum(new[:b]) for b in range(self.B + 1)]
        self.rows = self.starts[-1] + pad_rows
        heads = self.Hq + 2 * kv_heads
        # rows further apart than their heads need
        buf = (torch.randn(self.rows, heads * 128 + 40, generator=g) * amp).to(BF)
        buf[self.starts[-1]:] = math.nan
        self.x = buf.to(dev)[:, :heads * 128].unflatten(1, (heads, 128))
        self.q, self.k, self.v = self.x[:, :self.Hq], self.x[:, self.Hq:self.Hq + kv_heads], self.x[:, self.Hq + kv_heads:]
        self.cap = -(-max(max(lens), 1) // 16) * 16
        nb = self.cap // 16
        self.table = None
        shape = (self.B, kv_heads, self.cap, 128)
        if paged:
            pool = self.B * nb + 2
            self.table = torch.randperm(pool, generator=g)[:self.B * nb].view(self.B, nb).to(torch.int32).to(dev)
            shape = (pool, kv_heads, 16, 128)
        self.ck, self.cv = (torch.full(shape, math.nan, dtype=BF, device=dev) for _ in range(2))
        self.q_out = torch.full((self.rows, self.Hq, 128), math.nan, dtype=BF, device=dev)
        self.lens_t = torch.tensor(lens, dtype=torch.int32, device=dev)
        self.row_start = torch.tensor(self.starts, dtype=torch.int32, device=dev)

    def view(self, **kw):
        return P.make_view(self.ck, self.cv, self.lens_t, page_table=self.table, **kw)

    def ctx(self, **kw):
        return P.Context(num_layers=1, max_batch=self.B, num_q_heads=self.Hq, num_kv_heads=self.H, max_context=self.cap, max_k=16, max_window=16,
                         max_sinks=4, page_size=16 if self.paged else 0, **kw)

    def slot(self, b, pos):
        """Index of a position in ck / cv, but for the head."""
        return (int(self.table[b, pos // 16]), slice(None), pos % 16) if self.paged else (b, slice(None), pos)

    def tokens(self):
        for b in range(self.B):
            for j in range(self.new[b]):
                yield b, self.starts[b] + j, self.lens[b] - self.new[b] + j


def freqs(rot, base=10000.0):
    return (base ** (-2 * torch.arange(rot // 2, dtype=torch.float64) / max(rot, 1))).float()


def prepared(x, weight, norm, eps, angle, adjacent, scale=1.0):
    """[heads][128] -> (value, bound) in 64 bits; angle [rot / 2] in extended precision."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, np.float64))
    n = len(angle)
    turn = np.remainder(angle, np.longdouble(8) * np.arctan(np.longdouble(1)))
    c, s = (f(turn).astype(np.float64) * scale for f in (np.cos, np.sin))
    y, near = x.copy(), np.abs(x) * 2.0 ** -17
    if n:
        i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
        a, b = x[..., i], x[..., j]
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
        off = (2.0 ** -17 + 2.0 ** -51 * np.abs(angle).astype(np.float64)) * (np.abs(a) + np.abs(b)) * abs(scale)
        near[..., i] = near[..., j] = off
    return y, 2.0 ** -8 * np.abs(y) + 1.01 * near + 2.0 ** -134


def check(got, want, bound):
    got = np64(got)
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / bound).max()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("rot,adjacent,axes,norm", [(128, False, 0, "weights"), (128, False, 3, "ones"), (128, True, 0, None), (64, False, 2, "weights"),
                                                    (2, False, 0, "weights"), (126, False, 4, None), (90, True, 3, "weights"), (0, False, 0, "weights"),
                                                    (0, False, 0, None)])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kv_heads,group", [(2, 4), (1, 7), (3, 1)])
def test_append_against_the_formula(cuda_device, rot, adjacent, axes, norm, paged, kv_heads, group):
    t = Batch(cuda_device, [37, 5, 1, 16, 40], [20, 0, 1, 16, 3], kv_heads, group, paged, seed=rot + axes)
    g = torch.Generator().manual_seed(1)
    qw, kw = ((1 + 0.3 * torch.randn(128, generator=g)).to(cuda_device) for _ in range(2)) if norm == "weights" else (None, None)
    inv = freqs(rot)
    axis_of = torch.randint(0, axes, (rot // 2,), generator=g).tolist() if axes else None
    if axis_of:
        axis_of[0] = axes - 1
    positions = torch.randint(-50, 5000, (axes, t.rows), generator=g, dtype=torch.int32).to(cuda_device) if axes else None
    prep = P.make_qk_prep(qw, kw, eps=1e-5, norm=norm is not None, inv_freq=inv.to(cuda_device) if rot else None, adjacent=adjacent, axis_of=axis_of)
    ctx = t.ctx()
    ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, t.B, t.q_out, row_start=t.row_start, positions=positions)
    assert ctx.check() == 0
    q_out, ck, cv, x = t.q_out.cpu(), t.ck.cpu(), t.cv.cpu(), t.x.cpu()
    touched = torch.zeros(ck.shape[0], ck.shape[2], dtype=torch.bool)
    for b, r, pos in t.tokens():
        at = [int(positions[a, r]) if axes else pos for a in (axis_of or [0] * (rot // 2))]
        angle = np.array(at, np.longdouble) * inv.numpy().astype(np.longdouble)
        w = [None if v is None else np64(v) for v in (qw, kw)]
        check(q_out[r], *prepared(np64(x[r, :t.Hq]), w[0], norm, 1e-5, angle, adjacent))
        where = t.slot(b, pos)
        check(ck[where], *prepared(np64(x[r, t.Hq:t.Hq + t.H]), w[1], norm, 1e-5, angle, adjacent))
        assert torch.equal(cv[where], x[r, t.Hq + t.H:])
        touched[where[0], where[2]] = True
    assert torch.isnan(q_out[t.starts[-1]:]).all()
    for c in (ck, cv):
        assert torch.isnan(c.transpose(1, 2)[~touched]).all()


def test_far_positions_and_rotation_scale(cuda_device):
    """Angles up to 2^31 radians."""
    t = Batch(cuda_device, [9], [9], 1, 2, False)
    pos = torch.tensor([[2**31 - 1, -2**31, 2**30 + 12345, 1048575, 999999, 16777217, -1, 0, 123456789] + [0] * 3], dtype=torch.int32)
    inv = freqs(128, 500000.0)
    prep = P.make_qk_prep(inv_freq=inv.to(cuda_device), axis_of=[0] * 64, rot_scale=1.25)
    t.ctx().qkv_append(t.q, t.k, t.v, t.view(), prep, 1, t.q_out, row_start=t.row_start, positions=pos.to(cuda_device))
    for r in range(9):
        angle = np.array([int(pos[0, r])], np.longdouble) * inv.numpy().astype(np.longdouble)
        check(t.q_out[r], *prepared(np64(t.q[r]), None, False, 0.0, angle, False, 1.25))
        check(t.ck[0, :, r], *prepared(np64(t.k[r]), None, False, 0.0, angle, False, 1.25))


def test_one_row_each_without_row_start_equals_the_packed_call(cuda_device):
    lens = [33, 1, 16, 250]
    prep = None
    out = []
    for row_start in (True, False):
        t = Batch(cuda_device, lens, [1] * 4, 4, 8, True, pad_rows=0, seed=5)
        prep = P.make_qk_prep(norm=True, inv_freq=freqs(128).to(cuda_device))
        t.ctx().qkv_append(t.q, t.k, t.v, t.view(), prep, 4, t.q_out, row_start=t.row_start if row_start else None)
        out.append((t.q_out, t.ck, t.cv))
    for a, b in zip(*out):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_many_sequences_and_a_long_one(cuda_device):
    """Rows find their sequence among 1100, most of them without new tokens; heads in chunks and whole rows agree."""
    B = 1100
    new = [0] * B
    for b in (0, 31, 32, 33, 700, 1023, 1024, 1099):
        new[b] = 1 + b % 3
    new[500] = 700
    lens = [n + 2 for n in new]
    t = Batch(cuda_device, lens, new, 1, 1, False, seed=3)
    prep = P.make_qk_prep(inv_freq=freqs(128).to(cuda_device))
    ctx = t.ctx()
    ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, B, t.q_out, row_start=t.row_start)
    assert ctx.check() == 0
    x, q_out, ck, cv = t.x.cpu(), t.q_out.cpu(), t.ck.cpu(), t.cv.cpu()
    n = 0
    for b, r, pos in t.tokens():
        assert torch.equal(cv[b, :, pos], x[r, 2:])
        if pos % 50 < 4:
            angle = np.array([pos], np.longdouble) * freqs(128).numpy().astype(np.longdouble)
            check(ck[b, :, pos], *prepared(np64(x[r, 1:2]), None, False, 0.0, angle, False))
            check(q_out[r], *prepared(np64(x[r, :1]), None, False, 0.0, angle, False))
        n += 1
    assert int((~torch.isnan(cv[..., 0])).sum()) == n


def bytes_of(c):
    return [c.k.view(torch.uint8), c.v.view(torch.uint8), c.ks.view(torch.int32), c.vs.view(torch.int32), c.kt.view(torch.int16), c.vt.view(torch.int16)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("rot,adjacent", [(128, False), (40, False), (128, True)])
@pytest.mark.parametrize("chunks", [[1] * 35, [70], [5, 30, 0, 12, 1, 16, 17], [16, 15, 2, 31]])
def test_8_bit_append_is_the_bf16_append_quantised(cuda_device, fmt, paged, rot, adjacent, chunks):
    """The bf16 call's rows through bytekv_append, and the one call: the same to the bit, queries included."""
    H, G, B = 3, 5, 4
    total = sum(chunks)
    share = lambda c, b: c if b == 0 else c // 2 if b == 1 else max(0, c - 3) if b == 2 else 0  # noqa: E731
    g = torch.Generator().manual_seed(2)
    one, two = (Cache(fmt, B, H, total + 16, paged, cuda_device, seed=4) for _ in range(2))
    prep = P.make_qk_prep((1 + 0.2 * torch.randn(128, generator=g)).to(cuda_device), None, inv_freq=freqs(rot).to(cuda_device), adjacent=adjacent)
    have = [0] * B
    for i, c in enumerate(chunks):
        new = [share(c, b) for b in range(B)]
        have = [h + n for h, n in zip(have, new)]
        t = Batch(cuda_device, have, new, H, G, False, seed=10 + i, amp=2.0 ** (i - 2))
        ctx = P.Context(num_layers=1, max_batch=B, num_q_heads=H * G, num_kv_heads=H, max_context=one.cap, max_k=16, max_window=16, max_sinks=4,
                        page_size=16 if paged else 0)
        for cache in (one, two):
            cache.set_lens(have)
        t.ctx().qkv_append(t.q, t.k, t.v, t.view(), prep, B, t.q_out, row_start=t.row_start)
        most = max(max(new), 1)
        rows = torch.full((2, B, H, most, 128), math.nan, dtype=BF, device=cuda_device)
        for b in range(B):
            rows[0, b, :, :new[b]] = t.ck[b, :, have[b] - new[b]:have[b]]
            rows[1, b, :, :new[b]] = t.cv[b, :, have[b] - new[b]:have[b]]
        ctx.bytekv_append(rows[0], rows[1], torch.tensor(new, dtype=torch.int32, device=cuda_device), one.view(), B)
        q_out = torch.full_like(t.q_out, math.nan)
        ctx.bytekv_qkv_append(t.q, t.k, t.v, two.view(), prep, B, q_out, row_start=t.row_start)
        assert ctx.check() == 0
        assert torch.equal(q_out.view(torch.int16), t.q_out.view(torch.int16))
        for a, b in zip(bytes_of(one), bytes_of(two)):
            assert torch.equal(a, b)


def test_8_bit_append_records_what_is_not_finite(cuda_device):
    cache = Cache("e4m3", 1, 2, 32, False, cuda_device)
    t = Batch(cuda_device, [16], [16], 2, 1, False)
    ctx = t.ctx()
    cache.set_lens([16])
    t.v[3, 1, 7] = math.inf
    ctx.bytekv_qkv_append(t.q, t.k, t.v, cache.view(max_seq_len=16), P.make_qk_prep(), 1, t.q_out, row_start=t.row_start)
    with pytest.raises(P.PrhsError) as e:
        ctx.check()
    assert e.value.status == 7
    assert float(cache.v[0, 1, 3, 7].float()) == 448.0 and float(cache.vs[0, 1, 0]) == 2.0 ** 120


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
def test_read_back(cuda_device, fmt, paged):
    lens, first = [70, 16, 5, 0, 33, 64, 48], [0, 16, 0, 0, 30, 17, 47]
    cache = Cache(fmt, len(lens), 2, 80, paged, cuda_device, seed=1)
    t = Batch(cuda_device, lens, lens, 2, 1, paged, amp=30.0)
    t.cap = 80
    ctx = t.ctx()
    cache.set_lens(lens)
    ctx.bytekv_qkv_append(t.q, t.k, t.v, cache.view(), P.make_qk_prep(), t.B, t.q_out, row_start=t.row_start)
    for start in (None, first):
        out = Batch(cuda_device, [80] * len(lens), lens, 2, 1, paged, seed=9)
        ctx.bytekv_read(cache.view(), out.view(), t.B, first=None if start is None else torch.tensor(start, dtype=torch.int32, device=cuda_device))
        assert ctx.check() == 0
        touched = torch.zeros(out.ck.shape[0], out.ck.shape[2], dtype=torch.bool)
        for b, n in enumerate(lens):
            for which, c in (("k", out.ck), ("v", out.cv)):
                for h in range(2):
                    want = cache.rows(which, b, h, n)
                    for pos in range(start[b] if start else 0, n):
                        where = out.slot(b, pos)
                        assert np.array_equal(np64(c[where])[h], want[pos])
                        touched[where[0], where[2]] = True
        for c in (out.ck, out.cv):
            assert torch.isnan(c.cpu().transpose(1, 2)[~touched]).all()


def test_read_back_keeps_codes_that_are_not_finite_and_rounds_small_ones_once(cuda_device):
    cache = Cache("e5m2", 1, 1, 16, False, cuda_device)
    codes = torch.arange(256, dtype=torch.uint8).repeat(8).view(1, 1, 16, 128).to(cuda_device)
    for c, z in ((cache.k, 2.0 ** -126), (cache.v, 2.0 ** 100)):
        c.copy_(codes.view(DTYPE["e5m2"]))
        (cache.ks if c is cache.k else cache.vs).fill_(z)
    cache.set_lens([16])
    t = Batch(cuda_device, [16], [0], 1, 1, False)
    t.ctx().bytekv_read(cache.view(), t.view(), 1)
    x = codes.view(DTYPE["e5m2"]).double()
    for got, z in ((t.ck, 2.0 ** -126), (t.cv, 2.0 ** 100)):
        want = (x * z).float().to(BF)                      # products of a few bits: exact in fp32 down to its subnormals, as here
        assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(want, 7.0)) and torch.equal(got.isnan(), want.isnan())


# ------------------------------------------------------------------- what does not fit, streams, graphs
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("paged", [False, True])
def test_sequences_that_do_not_fit_are_left_out_and_recorded(cuda_device, eight, paged):
    lens, new = [20, 4, 33, 18], [20, 6, 1, 17]             # the second has fewer positions than rows
    t = Batch(cuda_device, [64] * 4, new, 2, 2, paged)
    t.lens_t.copy_(torch.tensor(lens, dtype=torch.int32))
    cache = Cache("e4m3", 4, 2, 64, paged, cuda_device)
    cache.set_lens(lens)
    ctx, prep = t.ctx(), P.make_qk_prep(norm=True)
    call = ctx.bytekv_qkv_append if eight else ctx.qkv_append
    view = (lambda **kw: cache.view(**kw)) if eight else (lambda **kw: t.view(**kw))
    call(t.q, t.k, t.v, view(max_seq_len=32), prep, 4, t.q_out, row_start=t.row_start)     # and the third more than allowed
    with pytest.raises(P.PrhsError):
        ctx.check()
    done = ~torch.isnan(t.q_out[:, 0, 0]).cpu()
    want = torch.zeros(t.rows, dtype=torch.bool)
    want[:20] = want[27:44] = True
    assert torch.equal(done, want)
    # row_start that runs backwards or past the rows
    for starts in ([0, 20, 10, 12, 20], [0, 20, 26, 27, t.rows + 5], [-3, 2, 5, 6, 9]):
        t.q_out.fill_(math.nan)
        call(t.q, t.k, t.v, view(), prep, 4, t.q_out, row_start=torch.tensor(starts, dtype=torch.int32, device=cuda_device))
        with pytest.raises(P.PrhsError):
            ctx.check()
    # a page that is not in the pool
    if paged:
        table = cache.table if eight else t.table
        keep = int(table[0, 0])
        table[0, 0] = 10**6
        cache.set_lens([20, 6, 1, 17])
        t.lens_t.copy_(cache.lens)
        t.ck.fill_(math.nan)
        cache.ks.fill_(math.nan)
        t.q_out.fill_(math.nan)
        call(t.q, t.k, t.v, view(), prep, 4, t.q_out, row_start=t.row_start)
        with pytest.raises(P.PrhsError):
            ctx.check()
        assert not torch.isnan(t.q_out[:44]).any()
        # the first sixteen rows of the first sequence are not written anywhere: 28 of 44 rows, one of two whole blocks
        assert int((~torch.isnan(cache.ks)).sum()) == 2 if eight else int((~torch.isnan(t.ck[..., 0])).sum()) == 28 * 2
        table[0, 0] = keep
    assert ctx.check() == 0


def test_read_leaves_out_what_does_not_fit(cuda_device):
    cache = Cache("e4m3", 3, 1, 64, False, cuda_device)
    t = Batch(cuda_device, [64] * 3, [64] * 3, 1, 1, False)
    ctx = t.ctx()
    cache.set_lens([64] * 3)
    ctx.bytekv_qkv_append(t.q, t.k, t.v, cache.view(), P.make_qk_prep(), 3, t.q_out, row_start=t.row_start)
    assert ctx.check() == 0
    for first, lens, kw, good in (([0, 65, -1], [64, 64, 64], {}, [64, 0, 0]), ([0, 60, 59], [64] * 3, dict(max_new=4), [0, 4, 0]),
                                  ([0, 0, 0], [64, 70, 48], {}, [64, 0, 48])):      # 48: whole blocks, an open one would have no rows in the tail
        cache.set_lens(lens)
        t.ck.fill_(math.nan)
        ctx.bytekv_read(cache.view(), t.view(), 3, first=torch.tensor(first, dtype=torch.int32, device=cuda_device), **kw)
        with pytest.raises(P.PrhsError):
            ctx.check()
        assert (~torch.isnan(t.ck[:, 0, :, 0])).sum(-1).tolist() == good


def test_another_stream_and_a_captured_graph(cuda_device):
    prep = P.make_qk_prep(norm=True, inv_freq=freqs(128).to(cuda_device))
    t = Batch(cuda_device, [40, 17], [1, 1], 2, 4, True, pad_rows=0)
    cache = Cache("e4m3", 2, 2, 48, True, cuda_device)
    back = Batch(cuda_device, [40, 17], [1, 1], 2, 4, True, pad_rows=0)
    ctx = t.ctx()
    cache.set_lens([40, 17])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step():
        ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, 2, t.q_out)
        ctx.bytekv_qkv_append(t.q, t.k, t.v, cache.view(), prep, 2, t.q_out)
        ctx.bytekv_read(cache.view(), back.view(), 2, first=cache.lens - 1, max_new=1)
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        first = cache.lens - 1
        with torch.cuda.graph(graph, stream=s):
            ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, 2, t.q_out)
            ctx.bytekv_qkv_append(t.q, t.k, t.v, cache.view(), prep, 2, t.q_out)
            ctx.bytekv_read(cache.view(), back.view(), 2, first=first, max_new=1)
    torch.cuda.synchronize()
    for seed in (1, 2):
        g = torch.Generator().manual_seed(seed)
        t.x.copy_(torch.randn(t.x.shape, generator=g).to(BF))
        for c in (t.ck, back.ck, t.q_out):
            c.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for b, pos in ((0, 39), (1, 16)):
            assert torch.equal(back.ck[back.slot(b, pos)], t.ck[t.slot(b, pos)])        # open blocks are bf16
            assert torch.equal(back.cv[back.slot(b, pos)], t.v[b])
        assert not torch.isnan(t.q_out).any()
    assert ctx.check() == 0


def test_refusals(cuda_device):
    t = Batch(cuda_device, [16, 16], [16, 16], 2, 2, False, pad_rows=0)
    cache = Cache("e4m3", 2, 2, 16, False, cuda_device)
    ctx, prep = t.ctx(), P.make_qk_prep()
    ok = dict(row_start=t.row_start)
    for call, view in ((ctx.qkv_append, t.view()), (ctx.bytekv_qkv_append, cache.view())):
        bad = [
            (t.q.float(), t.k, t.v, t.q_out, ok), (t.q[:, :3], t.k, t.v, t.q_out, ok), (t.q, t.k[:-1], t.v, t.q_out, ok), (t.q, t.k, t.v[..., :64], t.q_out, ok),
            (t.q.cpu(), t.k, t.v, t.q_out, ok), (t.q, t.k, t.v, t.q_out.transpose(0, 1), ok), (t.q, t.k, t.v, t.q_out, {}),
            (t.q, t.k, t.v, t.q_out, dict(row_start=t.row_start[:2])), (t.q, t.k, t.v, t.q_out, dict(row_start=t.row_start.long())),
            (t.q, t.k, t.v, t.q_out, dict(positions=torch.zeros(1, t.rows - 1, dtype=torch.int32, device=cuda_device), **ok)),
            (t.q, t.k, t.v, t.q_out, dict(positions=torch.zeros(1, t.rows, device=cuda_device), **ok)),
        ]
        for q, k, v, out, kw in bad:
            with pytest.raises(AssertionError):
                call(q, k, v, view, prep, 2, out, **kw)
        with pytest.raises(P.PrhsError):                     # an output over its input
            x = torch.zeros(32, 4, 128, dtype=BF, device=cuda_device)
            call(x, t.k, t.v, view, prep, 2, x, **ok)
        with pytest.raises(P.PrhsError):                     # rows that are not 16-byte aligned
            x = torch.zeros(32, 4, 132, dtype=BF, device=cuda_device)
            call(x[..., 2:130], t.k, t.v, view, prep, 2, t.q_out, **ok)
        with pytest.raises(AssertionError):                  # two axes are named, one is given
            call(t.q, t.k, t.v, view, P.make_qk_prep(inv_freq=freqs(4).to(cuda_device), axis_of=[0, 1]), 2, t.q_out,
                 positions=torch.zeros(1, t.rows, dtype=torch.int32, device=cuda_device), **ok)
        for change in (dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=2), dict(num_axes=0), dict(num_axes=5), dict(flags=4), dict(eps=-1.0, flags=1),
                       dict(eps=math.nan, flags=1), dict(q_weight=t.lens_t.data_ptr())):
            p = P.make_qk_prep()
            for n, val in change.items():
                setattr(p, n, val)
            with pytest.raises(P.PrhsError):
                call(t.q, t.k, t.v, view, p, 2, t.q_out, **ok)
        p = P.make_qk_prep(inv_freq=freqs(4).to(cuda_device))
        p.axis_of[1] = 1
        with pytest.raises(P.PrhsError):
            call(t.q, t.k, t.v, view, p, 2, t.q_out, **ok)
    for call, view in ((ctx.qkv_append, t.view()), (ctx.bytekv_qkv_append, cache.view())):       # no rows at all: nothing to do
        call(t.q[:0], t.k[:0], t.v[:0], view, prep, 2, t.q_out[:0], row_start=torch.zeros(3, dtype=torch.int32, device=cuda_device))
    with pytest.raises(AssertionError):
        ctx.bytekv_read(cache.view(), t.view(), 2, first=t.lens_t.long())
    with pytest.raises(P.PrhsError):
        ctx.bytekv_read(cache.view(), t.view(max_seq_len=8), 2)
    with pytest.raises(P.PrhsError):
        ctx.bytekv_read(cache.view(), t.view(), 2, max_new=17)
    with pytest.raises(P.PrhsError):
        ctx.bytekv_read(cache.view(), t.view(), 2, max_new=-1)
    assert ctx.check() == 0


@pytest.mark.parametrize("rot,adjacent", [(128, False), (128, True), (90, False), (0, False)])
def test_as_many_heads_as_there_is_room_for(cuda_device, rot, adjacent):
    """512 heads of queries, keys and values beside the rotation's tables; more are refused."""
    t = Batch(cuda_device, [5, 40], [2, 1], 32, 14, False)
    inv = freqs(rot)
    prep = P.make_qk_prep(norm=True, eps=1e-5, inv_freq=inv.to(cuda_device) if rot else None, adjacent=adjacent)
    ctx = t.ctx()
    ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, 2, t.q_out, row_start=t.row_start)
    assert ctx.check() == 0
    for b, r, pos in t.tokens():
        angle = np.array([pos], np.longdouble) * inv.numpy().astype(np.longdouble)
        check(t.q_out[r], *prepared(np64(t.q[r]), None, True, 1e-5, angle, adjacent))
        check(t.ck[b, :, pos], *prepared(np64(t.k[r]), None, True, 1e-5, angle, adjacent))
        assert torch.equal(t.cv[b, :, pos], t.v[r])
    t = Batch(cuda_device, [5], [2], 33, 14, False)
    with pytest.raises(P.PrhsError) as e:
        t.ctx().qkv_append(t.q, t.k, t.v, t.view(), prep, 1, t.q_out, row_start=t.row_start)
    assert e.value.status == 2


def bits(t):
    return t.view(torch.int16)


@pytest.mark.parametrize("rows", [470, 900, 3605, 7100])
@pytest.mark.parametrize("rot,adjacent,axes", [(128, False, 3), (128, True, 0), (90, False, 0), (64, False, 2)])
@pytest.mark.parametrize("kv_heads,group,paged", [(1, 3, False), (3, 5, True)])
def test_append_of_many_rows(cuda_device, rows, rot, adjacent, axes, kv_heads, group, paged):
    """Several rows per CTA (from six rows an SM on, up to eight), a last CTA that is not full, heads that are no multiple of four: the same to the
    bit as calls of few rows, in which a CTA has one, and a sample against the formula."""
    new = [rows // 2 - 3, 0, 1, rows // 5, 40]
    new.append(rows - sum(new))
    lens = [n + 17 * (i % 3) for i, n in enumerate(new)]
    t = Batch(cuda_device, lens, new, kv_heads, group, paged, seed=rows)
    g = torch.Generator().manual_seed(6)
    inv = freqs(rot)
    axis_of = [int(a) for a in torch.randint(0, axes, (rot // 2,), generator=g)] if axes else None
    positions = torch.randint(-50, 5000, (axes, t.rows), generator=g, dtype=torch.int32).to(cuda_device) if axes else None
    weights = [(1 + 0.3 * torch.randn(128, generator=g)).to(cuda_device) for _ in range(2)]
    prep = P.make_qk_prep(*weights, eps=1e-5, inv_freq=inv.to(cuda_device), adjacent=adjacent, axis_of=axis_of)
    if axis_of and max(axis_of) + 1 < axes:
        positions = positions[:max(axis_of) + 1].contiguous()
    ctx = t.ctx()
    ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, t.B, t.q_out, row_start=t.row_start, positions=positions)
    # the same in calls of at most 97 rows, sequences cut wherever that falls
    q2, k2, v2 = torch.full_like(t.q_out, math.nan), torch.full_like(t.ck, math.nan), torch.full_like(t.cv, math.nan)
    for a in range(0, t.starts[-1], 97):
        b = min(a + 97, t.starts[-1])
        cut = [min(max(s, a), b) for s in t.starts]
        have = [min(max(n - (t.starts[i + 1] - cut[i + 1]), 0), n) for i, n in enumerate(lens)]
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device=cuda_device)  # noqa: E731
        view = P.make_view(k2, v2, dev(have), page_table=t.table)
        ctx.qkv_append(t.q[a:b], t.k[a:b], t.v[a:b], view, prep, t.B, q2[a:b], row_start=dev([c - a for c in cut]),
                       positions=None if positions is None else positions[:, a:b])
    assert ctx.check() == 0
    for x, y in ((t.q_out, q2), (t.ck, k2), (t.cv, v2)):
        assert torch.equal(bits(x), bits(y))
    x, q_out, ck, cv = t.x.cpu(), t.q_out.cpu(), t.ck.cpu(), t.cv.cpu()
    table = None if t.table is None else t.table.cpu()
    pos_cpu = None if positions is None else positions.cpu().numpy()
    w = [np64(v) for v in weights]
    n = 0
    for b, r, pos in t.tokens():
        where = (int(table[b, pos // 16]), slice(None), pos % 16) if paged else (b, slice(None), pos)
        assert torch.equal(cv[where], x[r, t.Hq + t.H:])
        n += 1
        if r % 23 and r < t.starts[-1] - 9:
            continue
        at = [int(pos_cpu[a, r]) if axes else pos for a in (axis_of or [0] * (rot // 2))]
        angle = np.array(at, np.longdouble) * inv.numpy().astype(np.longdouble)
        check(q_out[r], *prepared(np64(x[r, :t.Hq]), w[0], True, 1e-5, angle, adjacent))
        check(ck[where], *prepared(np64(x[r, t.Hq:t.Hq + t.H]), w[1], True, 1e-5, angle, adjacent))
    assert torch.isnan(q_out[t.starts[-1]:]).all() and int((~torch.isnan(cv[..., 0])).sum()) == n * t.H


@pytest.mark.parametrize("fmt,paged", [("e4m3", False), ("e5m2", True)])
@pytest.mark.parametrize("rot,adjacent,axes", [(128, False, 3), (40, False, 0), (128, True, 2)])
@pytest.mark.parametrize("kv_heads,group", [(32, 1), (8, 7)])
@pytest.mark.parametrize("chunks", [[1] * 18, [5, 37, 1, 10, 16, 3], [9, 4900, 30]])
def test_8_bit_append_of_many_heads_and_blocks(cuda_device, fmt, paged, rot, adjacent, axes, kv_heads, group, chunks):
    """A block's heads over several CTAs (few blocks) and several heads to a warp (many blocks), tails that are closed and opened again, several
    axes of positions: the bf16 call's rows through bytekv_append, and the one call, the same to the bit."""
    H, G, B = kv_heads, group, 2
    total = sum(chunks)
    share = lambda c, b: c if b == 0 else c // 3  # noqa: E731
    g = torch.Generator().manual_seed(2)
    one, two = (Cache(fmt, B, H, total + 16, paged, cuda_device, seed=4) for _ in range(2))
    axis_of = [i % axes for i in range(rot // 2)] if axes else None
    prep = P.make_qk_prep((1 + 0.2 * torch.randn(128, generator=g)).to(cuda_device), None, inv_freq=freqs(rot).to(cuda_device), adjacent=adjacent,
                          axis_of=axis_of)
    ctx = P.Context(num_layers=1, max_batch=B, num_q_heads=H * G, num_kv_heads=H, max_context=one.cap, max_k=16, max_window=16, max_sinks=4,
                    page_size=16 if paged else 0)
    have = [0] * B
    for i, c in enumerate(chunks):
        new = [share(c, b) for b in range(B)]
        have = [h + n for h, n in zip(have, new)]
        t = Batch(cuda_device, have, new, H, G, False, seed=10 + i)
        positions = torch.randint(0, 9000, (axes, t.rows), generator=g, dtype=torch.int32).to(cuda_device) if axes else None
        for cache in (one, two):
            cache.set_lens(have)
        t.ctx().qkv_append(t.q, t.k, t.v, t.view(), prep, B, t.q_out, row_start=t.row_start, positions=positions)
        most = max(max(new), 1)
        rows = torch.full((2, B, H, most, 128), math.nan, dtype=BF, device=cuda_device)
        for b in range(B):
            rows[0, b, :, :new[b]] = t.ck[b, :, have[b] - new[b]:have[b]]
            rows[1, b, :, :new[b]] = t.cv[b, :, have[b] - new[b]:have[b]]
        ctx.bytekv_append(rows[0], rows[1], torch.tensor(new, dtype=torch.int32, device=cuda_device), one.view(), B)
        q_out = torch.full_like(t.q_out, math.nan)
        ctx.bytekv_qkv_append(t.q, t.k, t.v, two.view(), prep, B, q_out, row_start=t.row_start, positions=positions)
        assert ctx.check() == 0
        assert torch.equal(bits(q_out), bits(t.q_out))
        for a, b in zip(bytes_of(one), bytes_of(two)):
            assert torch.equal(a, b)
