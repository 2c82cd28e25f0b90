"""The 8-bit cache: append, attention over all positions, attention over lists, against the 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2602_08329_b200 import binding as P
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
DTYPE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
NAN_CODE = {"e4m3": 0x7F, "e5m2": 0x7E}


def np64(t):
    return t.detach().double().cpu().numpy()


def values_of(codes):
    """Code values as float64 (numpy) of a float8 tensor."""
    return codes.cpu().double().numpy()


class Cache:
    """An 8-bit cache with its reference content.  Everything that holds nothing is NaN."""

    def __init__(self, fmt, batch, kv_heads, cap, paged, dev, seed=0, pad=0):
        self.fmt, self.B, self.H, self.paged, self.dev = fmt, batch, kv_heads, paged, dev
        self.cap = -(-cap // 16) * 16
        nb = self.cap // 16
        g = torch.Generator().manual_seed(seed)
        if paged:
            self.pool = batch * nb + 3
            self.table_cpu = torch.randperm(self.pool, generator=g)[: batch * nb].view(batch, nb).to(torch.int32)
            self.table = self.table_cpu.to(dev)
            shape, sshape = (self.pool, kv_heads, 16, 128), (self.pool, kv_heads)
        else:
            self.table = None
            shape, sshape = (batch, kv_heads, self.cap + pad * 16, 128), (batch, kv_heads, nb + pad)
        raw = lambda: torch.full(shape, NAN_CODE[fmt], dtype=torch.uint8, device=dev).view(DTYPE[fmt])  # noqa: E731
        self.k, self.v = raw(), raw()
        self.ks, self.vs = (torch.full(sshape, math.nan, device=dev) for _ in range(2))
        self.kt, self.vt = (torch.full((batch, kv_heads, 16, 128), math.nan, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)

    def view(self, **kw):
        return P.make_bytekv_view(self.k, self.v, self.ks, self.vs, self.kt, self.vt, self.lens, page_table=self.table, **kw)

    def set_lens(self, lens):
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))

    def block(self, which, b, h, j):
        codes, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        if self.paged:
            page = int(self.table_cpu[b, j])
            return values_of(codes[page, h]), float(scale[page, h])
        return values_of(codes[b, h, 16 * j: 16 * j + 16]), float(scale[b, h, j])

    def rows(self, which, b, h, t):
        """The rows as the attention sees them, float64 [t][128]."""
        out = [c * s for c, s in (self.block(which, b, h, j) for j in range(t // 16))]
        tail = np64((self.kt if which == "k" else self.vt)[b, h, : t % 16])
        return np.concatenate(out + [tail]) if out else tail


def make_ctx(cache, group, cap=None, **kw):
    return P.Context(num_layers=1, max_batch=cache.B, num_q_heads=cache.H * group, num_kv_heads=cache.H,
                     max_context=cap or cache.cap, max_k=16, max_window=16, max_sinks=4, page_size=16 if cache.paged else 0, **kw)


def fill(ctx, cache, lens, seed=1, amp=None):
    """Appends random rows up to `lens` in one call; returns them [2][B][H][max][128] (bf16, on the device)."""
    g = torch.Generator().manual_seed(seed)
    n = max(max(lens), 1)
    new = torch.randn(2, cache.B, cache.H, n, 128, generator=g)
    if amp is not None:
        new = new * amp(torch.arange(n))[None, None, None, :, None]
    new = new.to(torch.bfloat16).to(cache.dev)
    cache.set_lens(lens)
    ctx.bytekv_append(new[0], new[1], cache.lens.clone(), cache.view(), cache.B)
    return new


# ---------------------------------------------------------------------------------- append
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("chunks", [[70], [1] * 37, [5, 30, 0, 12, 1, 16, 16], [16, 15, 2, 31], [33, 64, 47]])
def test_append_is_exact_and_touches_nothing_else(cuda_device, fmt, paged, chunks):
    B, H = 3, 2
    total = sum(chunks)
    # every sequence takes its own share of each chunk: all of it, half of it, none before the last
    share = lambda c, b, last: c if b == 0 else c // 2 if b == 1 else (c if last else 0)  # noqa: E731
    cache = Cache(fmt, B, H, total + 20, paged, cuda_device)
    ctx = make_ctx(cache, 1)
    g = torch.Generator().manual_seed(7)
    amp = torch.exp2(torch.randint(-40, 30, (2, B, H, total, 1), generator=g).float())
    rows = (torch.randn(2, B, H, total, 128, generator=g) * amp).to(torch.bfloat16)
    rows[:, :, :, 3] = 0.0
    rows[0, 0, 0, : min(16, total)] = 0.0                      # a block of zeros
    have = [0] * B
    for i, c in enumerate(chunks):
        n = [share(c, b, i == len(chunks) - 1) for b in range(B)]
        m = max(max(n), 1)
        # token-major input with padding between the rows: strides of every axis differ
        buf = torch.full((B, m, H, 136), math.nan, dtype=torch.bfloat16, device=cuda_device)
        new = []
        for w in range(2):
            x = buf.clone()
            for b in range(B):
                x[b, : n[b], :, :128] = rows[w, b, :, have[b]: have[b] + n[b]].transpose(0, 1).to(cuda_device)
            new.append(x[..., :128].transpose(1, 2))
        have = [h + k for h, k in zip(have, n)]
        cache.set_lens(have)
        ctx.bytekv_append(new[0], new[1], torch.tensor(n, dtype=torch.int32, device=cuda_device), cache.view(), B)
    assert ctx.check() == 0
    used = set()
    for b in range(B):
        for h in range(H):
            for w, name in enumerate("kv"):
                x = rows[w, b, h, : have[b]].double().numpy()
                for j in range(have[b] // 16):
                    want, s = R.quantise(x[16 * j: 16 * j + 16], fmt)
                    got, gs = cache.block(name, b, h, j)
                    assert gs == s and np.array_equal(got, want), (b, h, name, j)
                    used.add((int(cache.table_cpu[b, j]) if paged else (b, j), h))
                tail = np64((cache.kt if name == "k" else cache.vt)[b, h])
                assert np.array_equal(tail[: have[b] % 16], x[have[b] // 16 * 16:])
    # blocks that never became whole still hold what was there
    for x, s in ((cache.k, cache.ks), (cache.v, cache.vs)):
        raw, sc = x.view(torch.uint8).cpu(), s.cpu()
        for o in range(raw.shape[0]):
            for h in range(H):
                if paged:
                    if (o, h) not in used:
                        assert bool((raw[o, h] == NAN_CODE[fmt]).all()) and math.isnan(sc[o, h])
                else:
                    for j in range(sc.shape[2]):
                        if ((o, j), h) not in used:
                            assert bool((raw[o, h, 16 * j: 16 * j + 16] == NAN_CODE[fmt]).all()) and math.isnan(sc[o, h, j])
    ctx.close()


def test_append_refuses_contradictory_lengths_and_records_nonfinite(cuda_device):
    cache = Cache("e4m3", 4, 1, 64, False, cuda_device)
    ctx = make_ctx(cache, 1)
    new = torch.ones(4, 1, 20, 128, dtype=torch.bfloat16, device=cuda_device)
    cache.set_lens([10, 32, 65, 16])                     # more new rows than positions; above max_new; beyond the cache; fine
    n = torch.tensor([11, 21, 1, 16], dtype=torch.int32, device=cuda_device)
    ctx.bytekv_append(new, new, n, cache.view(), 4)
    with pytest.raises(P.PrhsError) as e:
        ctx.check()
    assert e.value.status == 7
    raw = cache.k.view(torch.uint8)
    assert bool((raw[:3] == NAN_CODE["e4m3"]).all()) and bool((cache.k[3, 0, :16].float() * cache.ks[3, 0, 0] == 1.0).all())
    new[3, 0, 2, 5], new[3, 0, 3, 6] = math.inf, math.nan
    cache.set_lens([0, 0, 0, 16])
    ctx.bytekv_append(new, new, torch.tensor([0, 0, 0, 16], dtype=torch.int32, device=cuda_device), cache.view(), 4)
    with pytest.raises(P.PrhsError):
        ctx.check()
    assert float(cache.k[3, 0, 2, 5].float()) == 448.0 and math.isnan(float(cache.k[3, 0, 3, 6].float()))
    assert ctx.check() == 0
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_a_nan_leaves_the_rest_of_its_block_as_it_is(cuda_device, fmt):
    """The scale is that of the numbers; a block of NaNs has the smallest; infinities keep the one that their exponent gives."""
    cache = Cache(fmt, 1, 2, 64, False, cuda_device)
    ctx = make_ctx(cache, 1)
    rows = torch.randn(2, 1, 2, 64, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    rows[0, 0, 0, 3, 7], rows[1, 0, 1, 17] = math.nan, math.nan
    rows[0, 0, 1, 32:48], rows[1, 0, 0, 50, 9], rows[1, 0, 0, 51, 10] = math.nan, -math.inf, math.nan
    cache.set_lens([64])
    ctx.bytekv_append(rows[0].to(cuda_device), rows[1].to(cuda_device), cache.lens.clone(), cache.view(), 1)
    with pytest.raises(P.PrhsError):
        ctx.check()
    for w, name in enumerate("kv"):
        for h in range(2):
            for j in range(4):
                x = rows[w, 0, h, 16 * j: 16 * j + 16].double().numpy()
                codes, s = cache.block(name, 0, h, j)
                if np.isinf(x).any():
                    top = R.TOP[fmt][0]
                    assert s == (2.0 ** 120 if fmt == "e4m3" else 2.0 ** 113) and codes[2, 9] == -top
                    assert np.all(codes[~np.isinf(x) & ~np.isnan(x)] == 0)
                else:
                    want, ws = R.quantise(np.where(np.isnan(x), 0.0, x), fmt)
                    assert s == ws and np.array_equal(codes[~np.isnan(x)], want[~np.isnan(x)]), (name, h, j)
                assert np.array_equal(np.isnan(codes), np.isnan(x))
    ctx.close()


def test_bad_pages_are_skipped_and_recorded(cuda_device):
    cache = Cache("e4m3", 2, 2, 64, True, cuda_device)
    ctx = make_ctx(cache, 2)
    bad = cache.table_cpu.clone()
    bad[0, 1], bad[1, 0] = -1, cache.pool
    good, cache.table = cache.table, bad.to(cuda_device)
    new = fill(ctx, cache, [50, 20])
    with pytest.raises(P.PrhsError):
        ctx.check()
    q = torch.randn(2, 4, 128, device=cuda_device).to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device=cuda_device)
    ctx.bytekv_decode_attn(q, cache.view(), 2, out, lse)
    with pytest.raises(P.PrhsError):
        ctx.check()
    cache.table_cpu = bad
    keep = {0: [0, 2], 1: []}                             # whole blocks that were found
    for b, t in ((0, 50), (1, 20)):
        for h in range(4):
            kv = []
            for w in "kv":
                parts = [c * s for c, s in (cache.block(w, b, h // 2, j) for j in keep[b])]
                kv.append(np.concatenate(parts + [np64((cache.kt if w == "k" else cache.vt)[b, h // 2, : t % 16])]))
            y, l, tol, ltol = R.attend(np64(q[b, h]), kv[0], kv[1], True)
            assert np.all(np.abs(np64(out[b, h]) - y) <= tol) and abs(float(lse[b, h]) - l) <= ltol
    assert good is not None and new is not None
    ctx.close()


# ------------------------------------------------------------------------------- attention
def check_dense(ctx, cache, lens, group, q, out, lse):
    y_all, l_all, qh = np64(out), np64(lse), np64(q)
    for b, t in enumerate(lens):
        for h in range(cache.H):
            k, v = cache.rows("k", b, h, t), cache.rows("v", b, h, t)
            for j in range(group):
                u = h * group + j
                y, l, tol, ltol = R.attend(qh[b, u], k, v, t % 16 > 0)
                assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u, np.max(np.abs(y_all[b, u] - y) / np.maximum(tol, 1e-30)))
                assert l_all[b, u] == l if math.isinf(l) else abs(l_all[b, u] - l) <= ltol, (b, u, l_all[b, u], l, ltol)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,group", [(2, 1), (1, 3), (2, 4), (1, 8), (1, 9), (1, 16)])
def test_attention_over_all_positions(cuda_device, fmt, paged, heads, group):
    lens = [0, 1, 15, 16, 17, 96, 527, 2050]
    cache = Cache(fmt, len(lens), heads, 2050, paged, cuda_device, pad=0 if paged else 2)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    q = (torch.randn(len(lens), heads * group, 128, generator=torch.Generator().manual_seed(3)) * 2).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_decode_attn(q, cache.view(), len(lens), out, lse)
    assert ctx.check() == 0
    check_dense(ctx, cache, lens, group, q, out, lse)
    again = torch.empty_like(out)
    ctx.bytekv_decode_attn(q, cache.view(), len(lens), again)            # tickets are clean, no log-sum-exp wanted
    assert torch.equal(again, out)
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("shape", ["rising", "falling", "zero blocks", "peaks", "tiny"])
def test_attention_with_scales_far_apart(cuda_device, fmt, shape):
    # magnitudes of neighbouring blocks differ by up to 2^40: the reference of the weighted values has to follow
    step = {"rising": lambda i: torch.exp2((i // 16).float() - 20), "falling": lambda i: torch.exp2(20 - (i // 16).float()),
            "zero blocks": lambda i: ((i // 16) % 3 > 0).float(), "peaks": lambda i: torch.where(i % 100 == 37, 60.0, 0.05),
            "tiny": lambda i: torch.full(i.shape, 2.0 ** -124)}[shape]
    lens = [640, 333]
    cache = Cache(fmt, 2, 1, 640, False, cuda_device)
    ctx = make_ctx(cache, 4)
    g = torch.Generator().manual_seed(5)
    k = torch.randn(2, 1, 640, 128, generator=g) * (1.0 if shape != "peaks" else 3.0)
    v = torch.randn(2, 1, 640, 128, generator=g) * step(torch.arange(640))[None, None, :, None]
    if shape == "falling":
        k *= torch.linspace(0.1, 3.0, 640)[None, None, :, None]          # small weights on large values first
    cache.set_lens(lens)
    ctx.bytekv_append(k.to(torch.bfloat16).to(cuda_device), v.to(torch.bfloat16).to(cuda_device), cache.lens.clone(), cache.view(), 2)
    q = (torch.randn(2, 4, 128, generator=g) * torch.tensor([0.0, 0.01, 1.0, 40.0])[None, :, None]).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device=cuda_device)
    ctx.bytekv_decode_attn(q, cache.view(), 2, out, lse)
    assert ctx.check() == 0
    check_dense(ctx, cache, lens, 4, q, out, lse)
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,group", [(2, 1), (1, 4), (1, 16)])
def test_attention_over_lists(cuda_device, fmt, paged, heads, group):
    lens = [5, 16, 300, 1205]
    cache = Cache(fmt, len(lens), heads, 1300, paged, cuda_device)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    U, stride = heads * group, 777
    rng = np.random.default_rng(4)
    idx = np.full((len(lens), U, stride), 1 << 30, np.int32)
    cnt = np.zeros((len(lens), U), np.int32)
    sizes = [0, 1, 2, 15, 16, 17, 33, 300, 777]
    lists = {}
    for b, t in enumerate(lens):
        for u in range(U):
            n = sizes[(b * U + u) % len(sizes)]
            c = rng.integers(0, t, n)                       # any order, repeats
            if n > 3:
                c[:3] = t - 1                               # the newest position three times
            lists[(b, u)] = c
            idx[b, u, :n], cnt[b, u] = c, n
    idx_d, cnt_d = torch.from_numpy(idx).to(cuda_device), torch.from_numpy(cnt).to(cuda_device)
    q = torch.randn(len(lens), U, 128, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_sparse_decode_attn(q, cache.view(), idx_d, cnt_d, len(lens), out, lse)
    assert ctx.check() == 0
    y_all, l_all, qh = np64(out), np64(lse), np64(q)
    rows = {(b, h): (cache.rows("k", b, h, t), cache.rows("v", b, h, t)) for b, t in enumerate(lens) for h in range(heads)}
    for (b, u), c in lists.items():
        k, v = rows[(b, u // group)]
        y, l, tol, ltol = R.attend(qh[b, u], k[c], v[c], True)
        assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u)
        assert l_all[b, u] == l if math.isinf(l) else abs(l_all[b, u] - l) <= ltol
    # an entry outside the sequence is left out and recorded
    b, u = next(k for k, c in lists.items() if len(c) >= 15 and lens[k[0]] > 16)
    idx_d[b, u, 4], idx_d[b, u, 9] = lens[b], -1
    ctx.bytekv_sparse_decode_attn(q, cache.view(), idx_d, cnt_d, len(lens), out, lse)
    with pytest.raises(P.PrhsError):
        ctx.check()
    c = np.delete(lists[(b, u)], [4, 9])
    k, v = rows[(b, u // group)]
    y, l, tol, ltol = R.attend(qh[b, u], k[c], v[c], True)
    assert np.all(np.abs(np64(out[b, u]) - y) <= tol) and abs(float(lse[b, u]) - l) <= ltol
    ctx.close()


@pytest.mark.parametrize("heads,group", [(2, 1), (1, 4), (1, 5), (1, 8), (1, 9), (1, 16)])
def test_weights_of_the_open_block_keep_their_low_bits(cuda_device, heads, group):
    """Over fewer than sixteen positions everything is in the open block; over all of them and over lists with repeats."""
    lens = list(range(1, 16))
    cache = Cache("e4m3", 15, heads, 16, False, cuda_device)
    ctx = make_ctx(cache, group)
    new = torch.randn(2, 15, heads, 16, 128, generator=torch.Generator().manual_seed(23))
    new[1] = torch.where(new[1] > 0, 1.0, -1.0)
    new = new.to(torch.bfloat16)
    cache.set_lens(lens)
    ctx.bytekv_append(new[0].to(cuda_device), new[1].to(cuda_device), cache.lens.clone(), cache.view(), 15)
    U = heads * group
    q = torch.randn(15, U, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    lists = {b: np.arange(40) * 7 % t for b, t in enumerate(lens)}
    idx = torch.from_numpy(np.stack([lists[b] for b in range(15)])).to(torch.int32)[:, None].expand(15, U, 40).contiguous().to(cuda_device)
    cnt = torch.full((15, U), 40, dtype=torch.int32, device=cuda_device)
    for listed in (False, True):
        out, lse = torch.full_like(q, math.nan), torch.full((15, U), math.nan, device=cuda_device)
        if listed:
            ctx.bytekv_sparse_decode_attn(q, cache.view(), idx, cnt, 15, out, lse)
        else:
            ctx.bytekv_decode_attn(q, cache.view(), 15, out, lse)
        assert ctx.check() == 0
        y_all, l_all, qh = np64(out), np64(lse), np64(q)
        for b, t in enumerate(lens):
            at = lists[b] if listed else np.arange(t)
            for u in range(U):
                y, l, tol, ltol = R.attend_few(qh[b, u], *(new[w, b, u // group].double().numpy()[at] for w in range(2)), 2.0 ** -16)
                assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u, np.max(np.abs(y_all[b, u] - y) / tol))
                assert abs(l_all[b, u] - l) <= ltol, (b, u)
    ctx.close()


def test_offsets_beyond_32_bits(cuda_device):
    # a pool whose last pages lie more than 2^32 bytes behind the base
    H, pool = 8, (1 << 32) // (8 * 16 * 128) + 40
    codes = torch.empty(2, pool, H, 16, 128, dtype=torch.uint8, device=cuda_device)
    scale = torch.empty(2, pool, H, device=cuda_device)
    table = (torch.arange(40, dtype=torch.int32, device=cuda_device) + (pool - 40)).flip(0).view(1, 40)
    lens = torch.tensor([633], dtype=torch.int32, device=cuda_device)
    tails = torch.empty(2, 1, H, 16, 128, dtype=torch.bfloat16, device=cuda_device)
    view = P.make_bytekv_view(codes[0].view(DTYPE["e4m3"]), codes[1].view(DTYPE["e4m3"]), scale[0], scale[1], tails[0], tails[1],
                              lens, page_table=table)
    ctx = P.Context(1, 1, H, H, 640, 16, 16, 4, page_size=16)
    new = torch.randn(2, 1, H, 633, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(cuda_device)
    ctx.bytekv_append(new[0], new[1], lens.clone(), view, 1)
    q = torch.randn(1, H, 128, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(cuda_device)
    idx = torch.arange(633, dtype=torch.int32, device=cuda_device).expand(1, H, 633).contiguous()
    cnt = torch.full((1, H), 633, dtype=torch.int32, device=cuda_device)
    out, lse = torch.empty(2, 1, H, 128, dtype=torch.bfloat16, device=cuda_device), torch.empty(2, 1, H, device=cuda_device)
    ctx.bytekv_decode_attn(q, view, 1, out[0], lse[0])
    ctx.bytekv_sparse_decode_attn(q, view, idx, cnt, 1, out[1], lse[1])
    assert ctx.check() == 0
    for h in range(H):
        kv = []
        for w in range(2):
            x = np64(new[w, 0, h])
            blocks = [c * s for c, s in (R.quantise(x[16 * j: 16 * j + 16], "e4m3") for j in range(39))]
            kv.append(np.concatenate(blocks + [x[624:]]))
        y, l, tol, ltol = R.attend(np64(q[0, h]), kv[0], kv[1], True)
        for i in range(2):
            assert np.all(np.abs(np64(out[i, 0, h]) - y) <= tol) and abs(float(lse[i, 0, h]) - l) <= ltol
    ctx.close()


def test_decode_run_in_a_graph(cuda_device):
    # a prompt, then tokens one by one: append and attention captured once and replayed, lengths advance on the device
    cache = Cache("e4m3", 3, 2, 128, True, cuda_device)
    ctx = make_ctx(cache, 4)
    lens = [37, 16, 60]
    prompt = fill(ctx, cache, lens)
    new = torch.zeros(2, 3, 2, 1, 128, dtype=torch.bfloat16, device=cuda_device)
    one = torch.ones(3, dtype=torch.int32, device=cuda_device)
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device=cuda_device)
    out, lse = torch.empty_like(q), torch.empty(3, 8, device=cuda_device)
    view = cache.view()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        cache.lens.add_(one)
        ctx.bytekv_append(new[0], new[1], one, view, 3)
        ctx.bytekv_decode_attn(q, view, 3, out, lse)
    g = torch.Generator().manual_seed(9)
    rows = {(w, b, h): np64(prompt[w, b, h, : lens[b]]) for w in range(2) for b in range(3) for h in range(2)}
    for step in range(20):
        x = torch.randn(2, 3, 2, 1, 128, generator=g).to(torch.bfloat16)
        new.copy_(x)
        q.copy_(torch.randn(3, 8, 128, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        lens = [t + 1 for t in lens]
        assert cache.lens.tolist() == lens
        for key in rows:
            rows[key] = np.concatenate([rows[key], np64(x[key[0], key[1], key[2]])])
        for b, t in enumerate(lens):
            for h in range(8):
                kv = []
                for w in range(2):
                    r = rows[(w, b, h // 4)]
                    kv.append(np.concatenate([c * s for c, s in (R.quantise(r[16 * j: 16 * j + 16], "e4m3") for j in range(t // 16))] + [r[t // 16 * 16:]]))
                y, l, tol, ltol = R.attend(np64(q[b, h]), kv[0], kv[1], True)
                assert np.all(np.abs(np64(out[b, h]) - y) <= tol) and abs(float(lse[b, h]) - l) <= ltol
    assert ctx.check() == 0
    ctx.close()


@pytest.mark.parametrize("heads,group,batch", [(2, 2, 70), (4, 8, 40), (8, 1, 100), (3, 16, 33)])
def test_many_ragged_sequences(cuda_device, heads, group, batch):
    # more units than parts: equal runs that cross units, sequences without whole blocks or without anything
    g = torch.Generator().manual_seed(8)
    lens = torch.randint(0, 420, (batch,), generator=g).tolist()
    for b in range(0, batch, 9):
        lens[b] = [0, 3, 16, 417, 15][b // 9 % 5]
    cache = Cache("e4m3", batch, heads, 420, True, cuda_device)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    q = torch.randn(batch, heads * group, 128, generator=g).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_decode_attn(q, cache.view(), batch, out, lse)
    assert ctx.check() == 0
    check_dense(ctx, cache, lens, group, q, out, lse)
    ctx.close()


@pytest.mark.parametrize("heads,group,batch,paged", [(8, 2, 50, True), (8, 1, 60, False), (8, 16, 50, False), (4, 16, 10, True)])
def test_short_sequences_beside_long_ones(cuda_device, heads, group, batch, paged):
    # runs that cross units with the units below and above the number of CTAs; few short units, a CTA each
    lens = torch.randint(0, 100, (batch,), generator=torch.Generator().manual_seed(4)).tolist()
    cap = 100 if batch == 10 else 713
    if cap > 100:
        lens[3], lens[-1], lens[-2] = 713, 704, 0
    cache = Cache("e5m2", batch, heads, cap, paged, cuda_device)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    q = torch.randn(batch, heads * group, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    for _ in range(2):
        ctx.bytekv_decode_attn(q, cache.view(), batch, out, lse)
    assert ctx.check() == 0
    check_dense(ctx, cache, lens, group, q, out, lse)
    ctx.close()


@pytest.mark.parametrize("heads,group,batch,stride", [(4, 4, 16, 70), (2, 1, 3, 1500), (4, 8, 2, 900)])
def test_lists_in_one_cta_and_in_parts(cuda_device, heads, group, batch, stride):
    # 256 units: one CTA each; few units: even parts, with counts from nothing to the whole stride
    U = heads * group
    lens = [600 + 37 * b for b in range(batch)]
    cache = Cache("e4m3", batch, heads, max(lens), False, cuda_device)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    rng = np.random.default_rng(6)
    cnt = rng.integers(0, stride + 1, (batch, U)).astype(np.int32)
    cnt[0, 0], cnt[-1, -1] = 0, stride
    idx = np.stack([rng.integers(0, lens[b], (U, stride)) for b in range(batch)]).astype(np.int32)
    q = torch.randn(batch, U, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_sparse_decode_attn(q, cache.view(), torch.from_numpy(idx).to(cuda_device), torch.from_numpy(cnt).to(cuda_device), batch, out, lse)
    assert ctx.check() == 0
    y_all, l_all = np64(out), np64(lse)
    for b in range(batch):
        kv = {h: (cache.rows("k", b, h, lens[b]), cache.rows("v", b, h, lens[b])) for h in range(heads)}
        for u in range(U):
            c = idx[b, u, : cnt[b, u]]
            y, l, tol, ltol = R.attend(np64(q[b, u]), kv[u // group][0][c], kv[u // group][1][c], True)
            assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u)
            assert l_all[b, u] == l if math.isinf(l) else abs(l_all[b, u] - l) <= ltol
    ctx.close()


def test_lengths_out_of_range_are_cut_and_recorded(cuda_device):
    cache = Cache("e4m3", 3, 1, 64, False, cuda_device)
    ctx = make_ctx(cache, 2)
    fill(ctx, cache, [64, 64, 64])
    cache.set_lens([-3, 1 << 30, 20])
    q = torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.empty_like(q), torch.empty(3, 2, device=cuda_device)
    idx = torch.arange(64, dtype=torch.int32, device=cuda_device).expand(3, 2, 64).contiguous()
    cnt = torch.full((3, 2), 20, dtype=torch.int32, device=cuda_device)
    for call in (lambda: ctx.bytekv_decode_attn(q, cache.view(), 3, out, lse),
                 lambda: ctx.bytekv_sparse_decode_attn(q, cache.view(), idx, cnt, 3, out, lse)):
        call()
        with pytest.raises(P.PrhsError):
            ctx.check()
        assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())
    ctx.close()


def test_a_list_stride_near_the_end_of_int32_is_refused(cuda_device):
    """(Rounded up to sixteen it would leave int32.)  A stride is only a distance: with one unit the buffer need not be that long."""
    cache = Cache("e4m3", 1, 1, 64, False, cuda_device)
    ctx = make_ctx(cache, 1)
    fill(ctx, cache, [64])
    q = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device=cuda_device)
    out, lse = torch.full_like(q, 7.0), torch.full((1, 1), 7.0, device=cuda_device)
    idx, cnt = torch.arange(64, dtype=torch.int32, device=cuda_device), torch.full((1,), 40, dtype=torch.int32, device=cuda_device)
    view = cache.view()
    for stride in ((1 << 30) + 1, (1 << 31) - 16, (1 << 31) - 1):
        rc = ctx.lib.prhs_bytekv_sparse_decode_attn(ctx.h, q.data_ptr(), P.C.byref(view), idx.data_ptr(), cnt.data_ptr(), stride, 1, out.data_ptr(),
                                                    lse.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert rc == 2, stride
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    rc = ctx.lib.prhs_bytekv_sparse_decode_attn(ctx.h, q.data_ptr(), P.C.byref(view), idx.data_ptr(), cnt.data_ptr(), 1 << 20, 1, out.data_ptr(),
                                                lse.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and ctx.check() == 0 and abs(float(lse[0, 0]) - math.log(40)) <= 2.0 ** -18
    ctx.close()


# What the tests above grant the weights, two bf16 roundings for every row, would hide a block of values that is left out or
# counted twice.  Here each row can be seen on its own.
def visible_values(t, seed, by_row):
    """Values [t][128], a power of two per row: block j at coordinate 5 j mod 128, blocks 128 apart with opposite signs; by_row:
    the block's rows eight coordinates apart.  Codes, weights and products are exact."""
    i = torch.arange(t)
    j = i // 16
    v = torch.zeros(t, 128)
    v[i, (5 * j + (8 * (i % 16) if by_row else 0)) % 128] = torch.exp2(((j + seed) % 3 - i % 4).float()) * (1.0 - 2.0 * (j // 128 % 2).float())
    return v


def check_visible(out, lse, v, at, where):
    """q = 0: every row in `at` has the weight 1 / n; one block, or one listed row, is a good part of its coordinate's sum."""
    n = len(at)
    want = v[at].sum(0) / n
    size = np.abs(v[at]).sum(0) / n
    assert np.all(np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * size), where
    assert abs(lse - math.log(n)) <= 2.0 ** -18, where


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("heads,group,lens", [
    (1, 2, [2050]), (2, 4, [9001, 37]), (1, 16, [4708]), (1, 1, [70000]),                                         # even parts
    (8, 2, [500] * 12 + [17, 0, 16, 499]), (8, 4, [1500, 20, 800, 333, 2500, 1] * 6),                             # one part each; runs
    (8, 9, [2047, 100, 1000, 3] * 8), (8, 4, [160 + 16 * (b % 19) for b in range(70)])])                          # wide; whole units
def test_every_block_counts_once(cuda_device, fmt, heads, group, lens):
    B = len(lens)
    cache = Cache(fmt, B, heads, max(lens), B > 1, cuda_device)
    ctx = make_ctx(cache, group)
    v = torch.stack([torch.stack([visible_values(max(lens), 2 * b + h, False) for h in range(heads)]) for b in range(min(B, 6))])
    cache.set_lens(lens)
    new_v = v.to(torch.bfloat16).to(cuda_device)[torch.arange(B, device=cuda_device) % len(v)]
    ctx.bytekv_append(torch.ones_like(new_v), new_v, cache.lens.clone(), cache.view(), B)
    q = torch.zeros(B, heads * group, 128, dtype=torch.bfloat16, device=cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_decode_attn(q, cache.view(), B, out, lse)
    assert ctx.check() == 0
    y, l, v64 = np64(out), np64(lse), v.double().numpy()
    for b, t in enumerate(lens):
        for u in range(heads * group):
            if t == 0:
                assert not y[b, u].any() and l[b, u] == -math.inf
            else:
                check_visible(y[b, u], l[b, u], v64[b % len(v), u // group], np.arange(t), (b, u))
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,group,B,t,stride", [(2, 1, 1, 2050, 1500), (1, 4, 3, 700, 300), (8, 4, 10, 1003, 130), (8, 2, 16, 400, 33)])
def test_every_entry_counts_once(cuda_device, fmt, paged, heads, group, B, t, stride):
    """Lists in parts and in whole: each entry as often as it is listed."""
    U = heads * group
    cache = Cache(fmt, B, heads, t, paged, cuda_device)
    ctx = make_ctx(cache, group)
    v = torch.stack([torch.stack([visible_values(t, 2 * b + h, True) for h in range(heads)]) for b in range(B)])
    cache.set_lens([t] * B)
    new_v = v.to(torch.bfloat16).to(cuda_device)
    ctx.bytekv_append(torch.ones_like(new_v), new_v, cache.lens.clone(), cache.view(), B)
    rng = np.random.default_rng(3)
    idx = rng.integers(0, t, (B, U, stride)).astype(np.int32)
    idx[:, :, ::3] = np.sort(idx[:, :, ::3], -1)
    cnt = rng.integers(1, stride + 1, (B, U)).astype(np.int32)
    cnt[0, 0] = stride
    q = torch.zeros(B, U, 128, dtype=torch.bfloat16, device=cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full((B, U), math.nan, device=cuda_device)
    ctx.bytekv_sparse_decode_attn(q, cache.view(), torch.from_numpy(idx).to(cuda_device), torch.from_numpy(cnt).to(cuda_device), B, out, lse)
    assert ctx.check() == 0
    y, l, v64 = np64(out), np64(lse), v.double().numpy()
    for b in range(B):
        for u in range(U):
            check_visible(y[b, u], l[b, u], v64[b, u // group], idx[b, u, : cnt[b, u]], (b, u))
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("size", [2.0 ** 4, 2.0 ** 9, 2.0 ** 12, 2.0 ** 20])
@pytest.mark.parametrize("v_size", [2.0 ** -40, 1.0, 2.0 ** 20])
def test_large_logits_leave_the_scales_of_the_values_alone(cuda_device, fmt, size, v_size):
    """Equal keys, so every row has the same weight whatever the logits' size (up to 2^44, where a step of fp32 is 2^20)."""
    lens, heads, group = [1610, 331, 96], 2, 3
    cache = Cache(fmt, 3, heads, 1610, False, cuda_device)
    ctx = make_ctx(cache, group)
    v = torch.stack([torch.stack([visible_values(1610, 2 * b + h, False) for h in range(heads)]) for b in range(3)]) * v_size
    k = torch.full((3, heads, 1610, 128), size, dtype=torch.bfloat16, device=cuda_device)
    cache.set_lens(lens)
    ctx.bytekv_append(k, v.to(torch.bfloat16).to(cuda_device), cache.lens.clone(), cache.view(), 3)
    U = heads * group
    q = torch.full((3, U, 128), size, dtype=torch.bfloat16, device=cuda_device)
    idx = torch.arange(1610, dtype=torch.int32, device=cuda_device).expand(3, U, 1610).contiguous()
    cnt = torch.tensor(lens, dtype=torch.int32, device=cuda_device)[:, None].expand(3, U).contiguous()
    for listed in (False, True):
        out = torch.full_like(q, math.nan)
        if listed:
            ctx.bytekv_sparse_decode_attn(q, cache.view(), idx, cnt, 3, out)
        else:
            ctx.bytekv_decode_attn(q, cache.view(), 3, out)
        assert ctx.check() == 0
        y, v64 = np64(out), v.double().numpy()
        for b, t in enumerate(lens):
            for u in range(U):
                check_visible(y[b, u], math.log(t), v64[b, u // group], np.arange(t), (b, u, listed))
    ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("heads,group,lens", [(2, 1, [2050, 16, 37]), (1, 4, [333, 640, 5]), (1, 12, [1000, 77, 2048])])
def test_weights_of_whole_blocks_keep_the_bits_of_fp16(cuda_device, fmt, heads, group, lens):
    """Rows of the 8-bit cache are granted 2^-11 a weight, those of the open block 2^-16."""
    B, t_max = len(lens), max(lens)
    cache = Cache(fmt, B, heads, t_max, True, cuda_device)
    ctx = make_ctx(cache, group)
    fill(ctx, cache, lens)
    q = (torch.randn(B, heads * group, 128, generator=torch.Generator().manual_seed(3)) * 2).to(torch.bfloat16).to(cuda_device)
    idx = torch.stack([torch.arange(t_max) * 11 % t for t in lens]).to(torch.int32)[:, None].expand(B, heads * group, t_max).contiguous().to(cuda_device)
    cnt = torch.tensor(lens, dtype=torch.int32, device=cuda_device)[:, None].expand(B, heads * group).contiguous()
    qh = np64(q)
    for listed in (False, True):
        out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
        if listed:
            ctx.bytekv_sparse_decode_attn(q, cache.view(), idx, cnt, B, out, lse)
        else:
            ctx.bytekv_decode_attn(q, cache.view(), B, out, lse)
        assert ctx.check() == 0
        y_all = np64(out)
        for b, t in enumerate(lens):
            at = np64(idx[b, 0, :t]).astype(int) if listed else np.arange(t)
            for u in range(heads * group):
                k, v = cache.rows("k", b, u // group, t)[at], cache.rows("v", b, u // group, t)[at]
                y, _, tol, _ = R.attend_few(qh[b, u], k, v, np.where(at < t // 16 * 16, 2.0 ** -11, 2.0 ** -16))
                p = np.exp(k @ qh[b, u] * R.S)
                small = 2.0 ** -31 * (p / p.sum()).max() * np.abs(v).max() * t          # fp16's smallest step
                assert np.all(np.abs(y_all[b, u] - y) <= tol + small), (b, u, np.max(np.abs(y_all[b, u] - y) / (tol + small)))
    ctx.close()


def test_split_counts_agree(cuda_device):
    # one long sequence runs split over many CTAs, a batch of copies with fewer splits: both near the 64-bit value
    for batch in (1, 48):
        lens = [9000] * batch
        cache = Cache("e4m3", batch, 1, 9000, False, cuda_device)
        ctx = make_ctx(cache, 2)
        fill(ctx, cache, lens)
        q = torch.randn(batch, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
        out, lse = torch.empty_like(q), torch.empty(batch, 2, device=cuda_device)
        ctx.bytekv_decode_attn(q, cache.view(), batch, out, lse)
        assert ctx.check() == 0
        for b in {0, batch - 1}:
            k, v = cache.rows("k", b, 0, 9000), cache.rows("v", b, 0, 9000)
            for u in range(2):
                y, l, tol, ltol = R.attend(np64(q[b, u]), k, v, True)
                assert np.all(np.abs(np64(out[b, u]) - y) <= tol) and abs(float(lse[b, u]) - l) <= ltol
        ctx.close()


# ------------------------------------------------------------------------------ not finite
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("heads,group,batch,t", [(2, 2, 3, 2055), (1, 12, 2, 535), (8, 2, 50, 90), (4, 4, 70, 400)])
def test_numbers_that_are_not_finite_show(cuda_device, fmt, heads, group, batch, t):
    """A NaN key, or an infinite one in the open block, makes the softmax NaN for the heads that read it and for no other; a NaN
    value its coordinate.  Over all positions (runs, parts, whole units) and over lists."""
    cache = Cache(fmt, batch, heads, t, False, cuda_device)
    ctx = make_ctx(cache, group)
    lens = [t - 2 * b % t for b in range(batch)]
    g = torch.Generator().manual_seed(41)
    rows = (torch.randn(2, batch, heads, t, 128, generator=g) * torch.tensor([0.25, 1.0])[:, None, None, None, None]).to(torch.bfloat16)
    rows[0, 0, 0, 33, 5] = math.nan                                       # a key in the 8-bit cache
    rows[0, 1, heads - 1, lens[1] - 1, 6] = math.inf                      # a key of the open block: +inf for every head (q > 0)
    rows[1, 1, 0, 35, 8] = math.nan                                       # a value
    if batch > 2:
        rows[1, 2, 0, lens[2] - 1, 9] = math.inf                          # a value of the open block
    cache.set_lens(lens)
    ctx.bytekv_append(rows[0].to(cuda_device), rows[1].to(cuda_device), cache.lens.clone(), cache.view(), batch)
    with pytest.raises(P.PrhsError):
        ctx.check()
    U = heads * group
    q = torch.randn(batch, U, 128, generator=g).abs().to(torch.bfloat16)
    if batch > 2:
        q[2, U - 1, 3] = math.nan
    q = q.to(cuda_device)
    idx = torch.arange(t, dtype=torch.int32, device=cuda_device).expand(batch, U, t).contiguous()
    cnt = torch.tensor(lens, dtype=torch.int32, device=cuda_device)[:, None].expand(batch, U).contiguous()
    for call in (lambda o, s: ctx.bytekv_decode_attn(q, cache.view(), batch, o, s),
                 lambda o, s: ctx.bytekv_sparse_decode_attn(q, cache.view(), idx, cnt, batch, o, s)):
        out, lse = torch.full_like(q, 7.0), torch.full((batch, U), 7.0, device=cuda_device)
        call(out, lse)
        assert ctx.check() == 0
        y_all, l_all = np64(out), np64(lse)
        for b in [0, 1, 2, batch // 2, batch - 1]:
            for u in range(U if b < batch else 0):
                h = u // group
                if (b, h) in ((0, 0), (1, heads - 1)) or (b == 2 and u == U - 1):
                    assert np.isnan(y_all[b, u]).all() and np.isnan(l_all[b, u]), (b, u)
                    continue
                d = {(1, 0): 8, (2, 0): 9}.get((b, h), -1)
                k, v = cache.rows("k", b, h, lens[b]), cache.rows("v", b, h, lens[b])
                v = np.where(np.isfinite(v), v, 0.0)
                y, l, tol, ltol = R.attend(np64(q[b, u]), k, v, True)
                rest = np.arange(128) != d
                assert np.all(np.abs(y_all[b, u] - y)[rest] <= tol[rest]) and abs(l_all[b, u] - l) <= ltol, (b, u)
                assert d < 0 or not np.isfinite(y_all[b, u, d]), (b, u)
    ctx.close()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("units,stride", [(2, 900), (80, 60)])
def test_rows_of_the_open_block_that_a_list_leaves_out_do_not_matter(cuda_device, paged, units, stride):
    """Infinities and NaNs in keys and values of open rows that no entry names; rows named once and several times beside them."""
    t, batch = 1003, 3
    cache = Cache("e4m3", batch, units, t, paged, cuda_device)
    ctx = make_ctx(cache, 1)
    new = fill(ctx, cache, [t] * batch)
    assert ctx.check() == 0 and new is not None
    for x, bad in ((cache.kt, math.nan), (cache.vt, math.inf)):          # open rows 992 .. 1002 are tail rows 0 .. 10
        x[:, :, 1], x[:, :, 4], x[:, :, 10] = bad, -bad, math.nan
    rng = np.random.default_rng(7)
    idx = rng.integers(0, 992, (batch, units, stride)).astype(np.int32)
    named = [992, 994, 994, 994, 999, 995, 999]
    idx[:, :, 3:10] = named                                              # in one part of a list that is dealt in parts
    idx[0, 0, -1] = 994                                                  # and in another
    cnt = np.full((batch, units), stride, np.int32)
    cnt[1, 1] = 12
    idx[2, 0, 3:10] = 5                                                  # no open row at all
    q = torch.randn(batch, units, 128, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.bytekv_sparse_decode_attn(q, cache.view(), torch.from_numpy(idx).to(cuda_device), torch.from_numpy(cnt).to(cuda_device), batch, out, lse)
    assert ctx.check() == 0
    y_all, l_all, qh = np64(out), np64(lse), np64(q)
    for b in range(batch):
        for u in sorted({0, 1, units // 2, units - 1}):
            c = idx[b, u, : cnt[b, u]]
            y, l, tol, ltol = R.attend(qh[b, u], cache.rows("k", b, u, t)[c], cache.rows("v", b, u, t)[c], True)
            assert np.all(np.abs(y_all[b, u] - y) <= tol) and abs(l_all[b, u] - l) <= ltol, (b, u)
    ctx.close()


# -------------------------------------------------------------------------------- refusals
def test_refusals(cuda_device):
    cache = Cache("e4m3", 2, 2, 64, False, cuda_device)
    ctx = make_ctx(cache, 2)
    lib, C = ctx.lib, P.C
    new = torch.zeros(2, 2, 4, 128, dtype=torch.bfloat16, device=cuda_device)
    n = torch.zeros(2, dtype=torch.int32, device=cuda_device)
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=cuda_device)
    out = torch.full_like(q, 7.0)
    idx, cnt = torch.zeros(2, 4, 8, dtype=torch.int32, device=cuda_device), torch.zeros(2, 4, dtype=torch.int32, device=cuda_device)
    st = torch.cuda.current_stream().cuda_stream

    def append(view, **kw):
        a = dict(k=new.data_ptr(), v=new.data_ptr(), s=1024, h=512, r=128, n=n.data_ptr(), m=4, b=2)
        a.update(kw)
        return lib.prhs_bytekv_append(ctx.h, C.byref(view), a["k"], a["v"], a["s"], a["h"], a["r"], a["n"], a["m"], a["b"], st)

    def attn(view, b=2, o=None):
        return lib.prhs_bytekv_decode_attn(ctx.h, q.data_ptr(), C.byref(view), b, out.data_ptr() if o is None else o, None, st)

    def rows(view, stride=8, i=None):
        return lib.prhs_bytekv_sparse_decode_attn(ctx.h, q.data_ptr(), C.byref(view), idx.data_ptr() if i is None else i,
                                                  cnt.data_ptr(), stride, 2, out.data_ptr(), None, st)

    assert append(cache.view()) == 0 and attn(cache.view()) == 0 and rows(cache.view()) == 0
    torch.cuda.synchronize()
    out.fill_(7.0)
    INVALID, UNSUPPORTED, CAPACITY = 1, 2, 6
    for field, value, status in [("k", None, INVALID), ("v_scale", None, INVALID), ("k_tail", None, INVALID), ("seq_lens", None, INVALID),
                                 ("k", cache.k.data_ptr() + 8, INVALID), ("v_tail", cache.vt.data_ptr() + 2, INVALID),
                                 ("stride_outer", 100, INVALID), ("stride_head", -128, INVALID), ("scale_stride_outer", 0, INVALID),
                                 ("max_seq_len", 65, CAPACITY), ("max_seq_len", -1, INVALID), ("format", 2, UNSUPPORTED),
                                 ("page_table", idx.data_ptr(), INVALID)]:
        view = cache.view()
        setattr(view, field, value)
        assert append(view) == status and attn(view) == status and rows(view) == status, (field, value)
    view = cache.view()
    assert append(view, m=0) == INVALID and append(view, m=65) == CAPACITY and append(view, r=4) == INVALID
    assert append(view, k=None) == INVALID and append(view, n=None) == INVALID and append(view, v=new.data_ptr() + 2) == INVALID
    assert append(view, b=3) == CAPACITY and attn(view, b=0) == INVALID and attn(view, o=out.data_ptr() + 4) == INVALID
    assert attn(view, o=q.data_ptr()) == INVALID and attn(view, o=q.data_ptr() + 256) == INVALID     # q and out overlap
    assert rows(view, stride=0) == INVALID
    assert lib.prhs_bytekv_decode_attn(None, q.data_ptr(), C.byref(view), 2, out.data_ptr(), None, st) == INVALID
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    with pytest.raises(AssertionError):
        ctx.bytekv_decode_attn(q.float(), cache.view(), 2, out)
    with pytest.raises(AssertionError):
        ctx.bytekv_decode_attn(q[:1], cache.view(), 2, out)
    with pytest.raises(AssertionError):
        P.make_bytekv_view(cache.k, cache.v, cache.ks[:, :, :-1], cache.vs, cache.kt, cache.vt, cache.lens)
    with pytest.raises(AssertionError):
        P.make_bytekv_view(cache.k.cpu(), cache.v.cpu(), cache.ks.cpu(), cache.vs.cpu(), cache.kt.cpu(), cache.vt.cpu(), cache.lens.cpu())
    paged = Cache("e4m3", 1, 1, 64, True, cuda_device)
    pctx = make_ctx(paged, 1)
    view = paged.view()
    view.page_table_stride = 3
    assert lib.prhs_bytekv_decode_attn(pctx.h, q.data_ptr(), C.byref(view), 1, out.data_ptr(), None, st) == INVALID
    pctx.close()
    ctx.close()
