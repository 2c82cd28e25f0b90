"""Block bounds, block scores and selection, attention over blocks, and whole steps, against the 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2602_08329_b200 import binding as P
from tests import cache_ref as R

pytestmark = pytest.mark.gpu


def np64(t):
    return t.detach().double().cpu().numpy()


class Cache:
    """A bf16 cache, contiguous or paged, with its bounds.  What holds nothing is NaN (rows) or 99 (bounds)."""

    def __init__(self, batch, kv_heads, cap, paged, dev, seed=0):
        self.B, self.H, self.paged, self.dev = batch, kv_heads, paged, dev
        self.nb = -(-cap // 16)
        g = torch.Generator().manual_seed(seed)
        if paged:
            self.pool = batch * self.nb + 2
            self.table_cpu = torch.randperm(self.pool, generator=g)[: batch * self.nb].view(batch, self.nb).to(torch.int32)
            self.table = self.table_cpu.to(dev)
            shape, bshape = (self.pool, kv_heads, 16, 128), (self.pool, kv_heads)
        else:
            self.table = None
            shape, bshape = (batch, kv_heads, self.nb * 16, 128), (batch, kv_heads, self.nb)
        self.k, self.v = (torch.full(shape, math.nan, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.codes = torch.full(bshape + (2, 128), 99, dtype=torch.int8, device=dev)
        self.scale = torch.full(bshape, 99.0, device=dev)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.rows = torch.zeros(2, batch, kv_heads, 0, 128, dtype=torch.bfloat16)

    def view(self, **kw):
        return P.make_view(self.k, self.v, self.lens, page_table=self.table, **kw)

    def bounds(self):
        return P.make_block_bounds(self.codes, self.scale)

    def place(self, rows, lens):
        """rows [2][B][H][n][128]: the first lens[b] positions of every sequence."""
        self.rows = rows
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for w, x in enumerate((self.k, self.v)):
            for b, t in enumerate(lens):
                if not self.paged:
                    x[b, :, :t] = rows[w, b, :, :t].to(self.dev)
                else:
                    for j in range(-(-t // 16)):
                        part = rows[w, b, :, 16 * j: min(16 * j + 16, t)]
                        x[int(self.table_cpu[b, j]), :, : part.shape[1]] = part.to(self.dev)

    def bound_of(self, b, h, j):
        o = (int(self.table_cpu[b, j]), h) if self.paged else (b, h, j)
        return self.codes[o].cpu().numpy(), float(self.scale[o])

    def ref_bounds(self, b, h, t):
        x = self.rows[0, b, h, :t].double().numpy()
        got = [R.block_bounds(x[16 * j: 16 * j + 16]) for j in range(-(-t // 16))]
        return np.stack([c for c, _ in got]) if got else np.zeros((0, 2, 128), np.int8), np.array([s for _, s in got])


def make_ctx(cache, group, cap=None):
    return P.Context(num_layers=1, max_batch=cache.B, num_q_heads=cache.H * group, num_kv_heads=cache.H,
                     max_context=cap or cache.nb * 16, max_k=16, max_window=16, max_sinks=4, page_size=16 if cache.paged else 0)


def random_rows(B, H, n, seed, drift=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, B, H, n, 128, generator=g)
    if drift:
        x[0] += torch.randn(B, H, -(-n // 16), 1, 128, generator=g).expand(-1, -1, -1, 16, -1).reshape(B, H, -1, 128)[:, :, :n]
    return x.to(torch.bfloat16)


def ref_sets(cache, q, lens, group, top, sink, recent, shared):
    """{(b, unit): blocks}, from the reference bounds."""
    sets = {}
    for b, t in enumerate(lens):
        nb = -(-t // 16)
        for h in range(cache.H):
            codes, scales = cache.ref_bounds(b, h, t)
            sc = [R.block_scores(q[b, h * group + j], codes, scales) for j in range(group)]
            if shared and group > 1:
                sets[(b, h)] = R.select_blocks(np.max(sc, 0), nb, top, sink, recent)
            else:
                for j in range(group):
                    sets[(b, h * group + j)] = R.select_blocks(sc[j], nb, top, sink, recent)
    return sets


def check_attention(cache, q, lens, group, sets, shared, out, lse):
    y_all, l_all = np64(out), np64(lse)
    for b, t in enumerate(lens):
        for u in range(cache.H * group):
            blocks = sets[(b, u // group if shared and group > 1 else u)]
            pos = np.array([i for j in blocks for i in range(16 * j, min(16 * j + 16, t))], np.int64)
            k, v = (cache.rows[w, b, u // group].double().numpy()[pos] for w in range(2))
            y, l, tol, ltol = R.attend(q[b, u], k, v, True)
            assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u)
            assert l_all[b, u] == l if math.isinf(l) else abs(l_all[b, u] - l) <= ltol, (b, u)


# ---------------------------------------------------------------------------------- bounds
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("first", ["all", "some", "last"])
def test_bounds_are_exact_and_touch_nothing_else(cuda_device, paged, first):
    lens = [0, 1, 16, 17, 150, 333]
    cache = Cache(len(lens), 2, 340, paged, cuda_device)
    ctx = make_ctx(cache, 1)
    rows = random_rows(len(lens), 2, 340, 1)
    rows[0, 4, 0, 32:48] = 0.0                                           # a block of zeros
    rows[0, 5, 1] *= torch.exp2(torch.arange(340).float() / 4 - 60)[:, None].to(torch.bfloat16)
    rows[0, 5, 0, 48:64, 7] = 127.0                                      # amax / 127 is a power of two
    cache.place(rows, lens)
    frm = {"all": [0] * 6, "some": [0, 0, 15, 17, 100, 16], "last": [t - 1 if t else 0 for t in lens]}[first]
    kw = {} if first == "all" else dict(first=torch.tensor(frm, dtype=torch.int32, device=cuda_device),
                                        max_new=1 if first == "last" else 0)
    ctx.block_bounds(cache.view(), cache.bounds(), len(lens), **kw)
    assert ctx.check() == 0
    touched = set()
    for b, t in enumerate(lens):
        for h in range(2):
            codes, scales = cache.ref_bounds(b, h, t)
            for j in range(frm[b] // 16, -(-t // 16) if frm[b] < t else 0):
                c, s = cache.bound_of(b, h, j)
                assert s == scales[j] and np.array_equal(c, codes[j]), (b, h, j)
                touched.add((int(cache.table_cpu[b, j]), h) if paged else (b, h, j))
    sc = cache.scale.cpu()
    for o in np.ndindex(*sc.shape):
        if o not in touched:
            assert sc[o] == 99.0 and bool((cache.codes[o] == 99).all()), o
    ctx.close()


def test_bounds_refuse_contradictory_lengths(cuda_device):
    cache = Cache(3, 1, 64, False, cuda_device)
    ctx = make_ctx(cache, 1)
    cache.place(random_rows(3, 1, 64, 1), [40, 40, 40])
    ctx.block_bounds(cache.view(), cache.bounds(), 3, first=torch.tensor([-1, 41, 39], dtype=torch.int32, device=cuda_device))
    with pytest.raises(P.PrhsError):
        ctx.check()
    assert bool((cache.scale[:2] == 99.0).all()) and cache.scale[2, 0].tolist()[:2] == [99.0, 99.0] and float(cache.scale[2, 0, 2]) != 99.0
    cache.scale.fill_(99.0)
    ctx.block_bounds(cache.view(), cache.bounds(), 3, first=torch.tensor([8, 37, 38], dtype=torch.int32, device=cuda_device), max_new=2)
    with pytest.raises(P.PrhsError):           # 32 and 3 new positions where two were announced
        ctx.check()
    assert bool((cache.scale[:2] == 99.0).all()) and float(cache.scale[2, 0, 2]) != 99.0
    ctx.close()


# ------------------------------------------------------------------------------- selection
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,group,shared", [(2, 1, False), (2, 4, False), (2, 4, True), (1, 16, False), (1, 16, True), (1, 11, True)])
@pytest.mark.parametrize("budget", [(5, 1, 2), (0, 0, 0), (1, 0, 0), (200, 3, 0), (7, 500, 1), (30, 0, 8)])
def test_selection_is_exact(cuda_device, paged, heads, group, shared, budget):
    top, sink, recent = budget
    lens = [0, 1, 16, 33, 700, 2047]
    cache = Cache(len(lens), heads, 2047, paged, cuda_device)
    ctx = make_ctx(cache, group)
    cache.place(random_rows(len(lens), heads, 2047, 3), lens)
    ctx.block_bounds(cache.view(), cache.bounds(), len(lens))
    q = torch.randn(len(lens), heads * group, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    q[:, 0] = 0.0                                                        # every score zero: ties everywhere
    q = q.to(cuda_device)
    units = heads if shared else heads * group
    blocks = torch.full((len(lens), units, max(1, min(top + sink + recent, 128)) + 3), 7, dtype=torch.int32, device=cuda_device)
    count = torch.full((len(lens), units), -5, dtype=torch.int32, device=cuda_device)
    sched = P.make_block_schedule(top, sink, recent, P.PRHS_GROUP_SETS if shared else 0)
    ctx.block_topk(q, cache.view(), cache.bounds(), sched, len(lens), blocks, count)
    assert ctx.check() == 0
    for (b, u), want in ref_sets(cache, np64(q), lens, group, top, sink, recent, shared).items():
        got = blocks[b, u].tolist()
        assert int(count[b, u]) == len(want) and got[: len(want)] == want and all(x == -1 for x in got[len(want):]), (b, u)
    ctx.close()


def test_ties_go_to_the_lower_block(cuda_device):
    # keys repeat with a period of five blocks: every score occurs many times
    cache = Cache(1, 2, 5000, False, cuda_device)
    ctx = make_ctx(cache, 2)
    rows = random_rows(1, 2, 80, 6)
    rows = rows.repeat(1, 1, 1, 63, 1)[:, :, :, :5000].contiguous()
    cache.place(rows, [5000])
    ctx.block_bounds(cache.view(), cache.bounds(), 1)
    q = torch.randn(1, 4, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(cuda_device)
    for top in (1, 62, 63, 64, 130, 300):
        blocks, count = torch.empty(1, 4, top + 1, dtype=torch.int32, device=cuda_device), torch.empty(1, 4, dtype=torch.int32, device=cuda_device)
        ctx.block_topk(q, cache.view(), cache.bounds(), P.make_block_schedule(top, 0, 1), 1, blocks, count)
        for (b, u), want in ref_sets(cache, np64(q), [5000], 2, top, 0, 1, False).items():
            assert blocks[b, u].tolist()[: int(count[b, u])] == want, (top, u)
    ctx.close()


# ------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads,group,shared", [(2, 1, False), (2, 4, False), (2, 4, True), (1, 16, True), (1, 11, False)])
def test_attention_over_blocks(cuda_device, paged, heads, group, shared):
    lens = [0, 3, 16, 250, 1599]
    cache = Cache(len(lens), heads, 1600, paged, cuda_device)
    ctx = make_ctx(cache, group)
    cache.place(random_rows(len(lens), heads, 1600, 8), lens)
    units = heads if shared else heads * group
    rng = np.random.default_rng(2)
    sets, stride = {}, 131
    blocks, count = np.full((len(lens), units, stride), 1 << 28, np.int32), np.zeros((len(lens), units), np.int32)
    for b, t in enumerate(lens):
        nb = -(-t // 16)
        for u in range(units):
            n = 0 if nb == 0 else [131, 0, 1, 2, 3, 17, 64][(u + b) % 7]
            sets[(b, u)] = rng.integers(0, nb, n).tolist() if n else []      # any order, repeats
            blocks[b, u, :n], count[b, u] = sets[(b, u)], n
    bd, cd = torch.from_numpy(blocks).to(cuda_device), torch.from_numpy(count).to(cuda_device)
    q = torch.randn(len(lens), heads * group, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    flags = P.PRHS_GROUP_SETS if shared else 0
    ctx.block_decode_attn(q, cache.view(), bd, cd, len(lens), out, lse, flags)
    assert ctx.check() == 0
    check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    # a block outside the sequence is left out and recorded
    b, u = next(k for k, s in sets.items() if len(s) >= 3 and k[0] >= 3)
    bd[b, u, 1], bd[b, u, 2] = -(-lens[b] // 16), -3
    sets[(b, u)] = sets[(b, u)][:1] + sets[(b, u)][3:]
    ctx.block_decode_attn(q, cache.view(), bd, cd, len(lens), out, lse, flags)
    with pytest.raises(P.PrhsError):
        ctx.check()
    check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    ctx.close()


@pytest.mark.parametrize("heads,group,shared", [(2, 1, False), (2, 4, True), (1, 4, False), (1, 5, True), (2, 8, True), (1, 9, True), (1, 16, True)])
def test_weights_keep_their_low_bits(cuda_device, heads, group, shared):
    """Values of one size and either sign nearly cancel: what is left shows the weights' own rounding, 2^-16 for two bf16."""
    lens = list(range(1, 41, 3)) + [96, 200]
    cache = Cache(len(lens), heads, 200, False, cuda_device)
    ctx = make_ctx(cache, group)
    rows = random_rows(len(lens), heads, 200, 19, drift=False)
    rows[1] = torch.where(rows[1] > 0, 1.0, -1.0).to(torch.bfloat16)
    cache.place(rows, lens)
    units = heads if shared else heads * group
    nb = [-(-t // 16) for t in lens]
    blocks = torch.arange(13, dtype=torch.int32, device=cuda_device).expand(len(lens), units, 13).contiguous()
    count = torch.tensor(nb, dtype=torch.int32, device=cuda_device)[:, None].expand(len(lens), units).contiguous()
    q = torch.randn(len(lens), heads * group, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.block_decode_attn(q, cache.view(), blocks, count, len(lens), out, lse, P.PRHS_GROUP_SETS if shared else 0)
    assert ctx.check() == 0
    y_all, l_all, qh = np64(out), np64(lse), np64(q)
    for b, t in enumerate(lens):
        for u in range(heads * group):
            y, l, tol, ltol = R.attend_few(qh[b, u], *(rows[w, b, u // group, :t].double().numpy() for w in range(2)), 2.0 ** -16)
            assert np.all(np.abs(y_all[b, u] - y) <= tol), (b, u, np.max(np.abs(y_all[b, u] - y) / tol))
            assert abs(l_all[b, u] - l) <= ltol, (b, u)
    ctx.close()


def test_bad_pages_are_skipped_and_recorded(cuda_device):
    cache = Cache(1, 1, 160, True, cuda_device)
    ctx = make_ctx(cache, 1)
    cache.place(random_rows(1, 1, 160, 8), [160])
    ctx.block_bounds(cache.view(), cache.bounds(), 1)
    cache.table[0, 3], cache.table[0, 5] = -1, cache.pool
    q = torch.randn(1, 1, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(cuda_device)
    blocks, count = torch.empty(1, 1, 10, dtype=torch.int32, device=cuda_device), torch.empty(1, 1, dtype=torch.int32, device=cuda_device)
    out, lse = torch.empty_like(q), torch.empty(1, 1, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(9, 0, 1), 1, out, lse, blocks, count)
    with pytest.raises(P.PrhsError):
        ctx.check()
    assert blocks[0, 0].tolist() == list(range(10))
    check_attention(cache, np64(q), [160], 1, {(0, 0): [0, 1, 2, 4, 6, 7, 8, 9]}, False, out, lse)
    ctx.block_bounds(cache.view(), cache.bounds(), 1)
    with pytest.raises(P.PrhsError):
        ctx.check()
    assert ctx.check() == 0
    ctx.close()


# ------------------------------------------------------------------------------------ steps
@pytest.mark.parametrize("paged,group,shared", [(False, 1, False), (True, 4, True), (True, 4, False), (False, 16, True)])
def test_decode_run(cuda_device, paged, group, shared):
    # a prompt's bounds, then tokens one by one through whole steps captured in a graph
    lens, H, cap = [30, 239, 16], 2, 300
    cache = Cache(3, H, cap, paged, cuda_device)
    ctx = make_ctx(cache, group)
    rows = random_rows(3, H, cap, 12)
    cache.place(rows, lens)
    ctx.block_bounds(cache.view(), cache.bounds(), 3)
    units = H if shared else H * group
    q = torch.zeros(3, H * group, 128, dtype=torch.bfloat16, device=cuda_device)
    blocks, count = torch.empty(3, units, 8, dtype=torch.int32, device=cuda_device), torch.empty(3, units, dtype=torch.int32, device=cuda_device)
    out, lse = torch.empty_like(q), torch.empty(3, H * group, device=cuda_device)
    sched = P.make_block_schedule(4, 1, 2, P.PRHS_GROUP_SETS if shared else 0)
    view, bounds = cache.view(), cache.bounds()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        ctx.block_decode_step(q, view, bounds, sched, 3, out, lse, blocks, count)
    g = torch.Generator().manual_seed(13)
    for step in range(20):
        lens = [t + 1 for t in lens]
        cache.place(rows, lens)
        q.copy_(torch.randn(3, H * group, 128, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        sets = ref_sets(cache, np64(q), lens, group, 4, 1, 2, shared)
        for (b, u), want in sets.items():
            assert blocks[b, u].tolist()[: int(count[b, u])] == want, (step, b, u)
        check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    for b, t in enumerate(lens):                                           # the bounds kept up with the tokens
        for h in range(H):
            codes, scales = cache.ref_bounds(b, h, t)
            for j in range(-(-t // 16)):
                c, s = cache.bound_of(b, h, j)
                assert s == scales[j] and np.array_equal(c, codes[j])
    assert ctx.check() == 0
    ctx.close()


@pytest.mark.parametrize("heads,group,shared,batch", [(2, 2, False, 70), (8, 8, True, 40), (1, 12, True, 65)])
def test_steps_of_many_ragged_sequences(cuda_device, heads, group, shared, batch):
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 700, (batch,), generator=g).tolist()
    for b in range(0, batch, 7):
        lens[b] = [0, 1, 16, 690, 17][b // 7 % 5]
    cache = Cache(batch, heads, 700, True, cuda_device)
    ctx = make_ctx(cache, group)
    cache.place(random_rows(batch, heads, 700, 5), [max(t - 1, 0) for t in lens])
    ctx.block_bounds(cache.view(), cache.bounds(), batch)
    cache.place(cache.rows, lens)
    units = heads if shared else heads * group
    q = torch.randn(batch, heads * group, 128, generator=g).to(torch.bfloat16).to(cuda_device)
    blocks, count = torch.empty(batch, units, 12, dtype=torch.int32, device=cuda_device), torch.empty(batch, units, dtype=torch.int32, device=cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    sched = P.make_block_schedule(8, 2, 2, P.PRHS_GROUP_SETS if shared else 0)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, batch, out, lse, blocks, count)
    assert ctx.check() == 0
    sets = ref_sets(cache, np64(q), lens, group, 8, 2, 2, shared)
    for (b, u), want in sets.items():
        assert blocks[b, u].tolist() == want + [-1] * (12 - len(want)), (b, u)
    check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    for b, t in enumerate(lens):
        for h in range(heads):
            codes, scales = cache.ref_bounds(b, h, t)
            for j in range(-(-t // 16)):
                c, s = cache.bound_of(b, h, j)
                assert s == scales[j] and np.array_equal(c, codes[j])
    ctx.close()


def test_empty_batch_and_lengths_out_of_range(cuda_device):
    cache = Cache(3, 1, 64, False, cuda_device)
    ctx = make_ctx(cache, 2)
    cache.place(random_rows(3, 1, 64, 1), [64, 64, 64])
    ctx.block_bounds(cache.view(), cache.bounds(), 3)
    q = torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.empty_like(q), torch.empty(3, 2, device=cuda_device)
    blocks, count = torch.empty(3, 2, 4, dtype=torch.int32, device=cuda_device), torch.empty(3, 2, dtype=torch.int32, device=cuda_device)
    step = lambda: ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(2, 1, 1), 3, out, lse, blocks, count)  # noqa: E731
    cache.lens.zero_()
    step()
    assert ctx.check() == 0 and bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert bool((count == 0).all()) and bool((blocks == -1).all())
    cache.lens.copy_(torch.tensor([64, -1, 65], dtype=torch.int32))
    step()
    with pytest.raises(P.PrhsError):
        ctx.check()
    sets = ref_sets(cache, np64(q)[:1], [64], 2, 2, 1, 1, False)
    check_attention(cache, np64(q), [64], 2, sets, False, out, lse)
    assert bool((out[1] == 0).all()) and count[1].tolist() == [0, 0]
    ctx.close()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("cap,top", [(8192, 1), (8192, 255), (8192, 256), (8192, 257), (8192, 600), (8208, 16), (48, 2)])
def test_a_step_selects_as_block_topk_does(cuda_device, cap, top, shared):
    """On both sides of the sizes up to which the attention kernel selects for itself; a zero query ties all blocks."""
    group, lens = 2, [cap, cap - 7, 33, 0]
    cache = Cache(4, 2, cap, True, cuda_device, seed=cap + top)
    ctx = make_ctx(cache, group)
    cache.place(random_rows(4, 2, cap, cap + top), lens)
    ctx.block_bounds(cache.view(), cache.bounds(), 4)
    q = torch.randn(4, 4, 128, generator=torch.Generator().manual_seed(top)).to(torch.bfloat16)
    q[1, 1], q[1, 2:] = 0, 0
    q = q.to(cuda_device)
    sched = P.make_block_schedule(top, 1, 2, P.PRHS_GROUP_SETS if shared else 0)
    units = 2 if shared else 4
    got, want = ((torch.full((4, units, top + 3), 7, dtype=torch.int32, device=cuda_device),
                  torch.full((4, units), 7, dtype=torch.int32, device=cuda_device)) for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty(4, 4, device=cuda_device)
    for _ in range(2):
        ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, 4, out, lse, *got)
    ctx.block_topk(q, cache.view(), cache.bounds(), sched, 4, *want)
    assert ctx.check() == 0
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    sets = ref_sets(cache, np64(q), lens, group, top, 1, 2, shared)
    for (b, u), blocks in sets.items():
        assert got[0][b, u, : int(got[1][b, u])].tolist() == list(blocks)
    check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    ctx.close()


@pytest.mark.parametrize("heads,group,shared", [(8, 2, False), (16, 2, True), (10, 16, True)])
def test_many_short_lists(cuda_device, heads, group, shared):
    """So many units that a warp takes one alone; empty sequences and lists among them, the last CTA not full."""
    batch = 61
    lens = torch.randint(1, 150, (batch,), generator=torch.Generator().manual_seed(3)).tolist()
    lens[0], lens[7], lens[60] = 0, 1, 150
    cache = Cache(batch, heads, 150, True, cuda_device, seed=9)
    ctx = make_ctx(cache, group)
    cache.place(random_rows(batch, heads, 150, 9), lens)
    ctx.block_bounds(cache.view(), cache.bounds(), batch)
    q = torch.randn(batch, heads * group, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda_device)
    flags, units = (P.PRHS_GROUP_SETS, heads) if shared else (0, heads * group)
    blocks, count = (torch.empty(batch, units, 6, dtype=torch.int32, device=cuda_device), torch.empty(batch, units, dtype=torch.int32, device=cuda_device))
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(3, 1, 2, flags), batch, out, lse, blocks, count)
    assert ctx.check() == 0
    sets = ref_sets(cache, np64(q), lens, group, 3, 1, 2, shared)
    check_attention(cache, np64(q), lens, group, sets, shared, out, lse)
    again, lse2 = torch.full_like(q, math.nan), torch.full_like(lse, math.nan)
    ctx.block_decode_attn(q, cache.view(), blocks, count, batch, again, lse2, flags)
    check_attention(cache, np64(q), lens, group, sets, shared, again, lse2)
    count[7], count[-1, -1] = 0, 0
    ctx.block_decode_attn(q, cache.view(), blocks, count, batch, again, lse2, flags)
    assert ctx.check() == 0 and bool((again[7] == 0).all()) and bool((lse2[7] == -math.inf).all())
    assert bool((again[-1, -1] == 0).all())
    ctx.close()


def test_a_step_leaves_the_bounds_of_an_impossible_length(cuda_device):
    """A step writes bounds of last blocks only, and none for a length that is cut."""
    cache = Cache(3, 2, 64, True, cuda_device, seed=5)
    ctx = make_ctx(cache, 1)
    cache.place(random_rows(3, 2, 64, 5), [50, 64, 64])
    ctx.block_bounds(cache.view(), cache.bounds(), 3)
    before = cache.codes.clone(), cache.scale.clone()
    for b, j in ((0, 3), (1, 3), (2, 3)):
        page = int(cache.table_cpu[b, j])
        cache.codes[page], cache.scale[page] = 77, 77.0
    cache.lens.copy_(torch.tensor([50, 65, -3], dtype=torch.int32))
    q = torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.empty_like(q), torch.empty(3, 2, device=cuda_device)
    blocks, count = torch.empty(3, 2, 3, dtype=torch.int32, device=cuda_device), torch.empty(3, 2, dtype=torch.int32, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(1, 1, 1), 3, out, lse, blocks, count)
    with pytest.raises(P.PrhsError):
        ctx.check()
    for b in (1, 2):
        page = int(cache.table_cpu[b, 3])
        before[0][page], before[1][page] = 77, 77.0
    assert torch.equal(cache.codes, before[0]) and torch.equal(cache.scale, before[1])
    ctx.close()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("cap", [640, 8208])
def test_a_length_beyond_the_maximum_selects_as_the_maximum(cuda_device, paged, cap):
    """A length that is cut has scores like any other: nothing of an earlier call's is ranked.  (8208: a kernel of its own selects.)"""
    cache = Cache(3, 2, cap, paged, cuda_device, seed=cap)
    ctx = make_ctx(cache, 2)
    cache.place(random_rows(3, 2, cap, 11), [cap] * 3)
    ctx.block_bounds(cache.view(), cache.bounds(), 3)
    new = lambda: (torch.full((3, 4, 9), 7, dtype=torch.int32, device=cuda_device), torch.full((3, 4), 7, dtype=torch.int32, device=cuda_device))  # noqa: E731
    out, lse = torch.empty(3, 4, 128, dtype=torch.bfloat16, device=cuda_device), torch.empty(3, 4, device=cuda_device)
    sched = P.make_block_schedule(6, 1, 2)
    before, q = (torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(cuda_device) for i in range(2))
    calls = (lambda q, lists: ctx.block_topk(q, cache.view(), cache.bounds(), sched, 3, *lists),
             lambda q, lists: ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, 3, out, lse, *lists))
    want = ref_sets(cache, np64(q), [cap] * 3, 2, 6, 1, 2, False)
    for call in calls:
        cache.lens.fill_(cap)
        call(before, new())                                              # other scores in the workspace
        cache.lens.copy_(torch.tensor([cap, cap + 1, 1 << 30], dtype=torch.int32))
        blocks, count = new()
        call(q, (blocks, count))
        with pytest.raises(P.PrhsError):
            ctx.check()
        for (b, u), w in want.items():
            assert blocks[b, u].tolist() == w and int(count[b, u]) == len(w), (b, u)
    check_attention(cache, np64(q), [cap] * 3, 2, want, False, out, lse)
    ctx.close()


def test_all_blocks_are_the_dense_attention(cuda_device):
    cache = Cache(2, 2, 700, False, cuda_device)
    ctx = make_ctx(cache, 2)
    cache.place(random_rows(2, 2, 700, 8), [700, 77])
    ctx.block_bounds(cache.view(), cache.bounds(), 2)
    q = torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(cuda_device)
    blocks, count = torch.empty(2, 4, 44, dtype=torch.int32, device=cuda_device), torch.empty(2, 4, dtype=torch.int32, device=cuda_device)
    out, lse, want, wl = torch.empty_like(q), torch.empty(2, 4, device=cuda_device), torch.empty_like(q), torch.empty(2, 4, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(1000, 1, 1), 2, out, lse, blocks, count)
    ctx.dense_decode_attn(q, cache.view(), 2, want, wl)
    assert count.tolist() == [[44] * 4, [5] * 4]
    assert float((out.float() - want.float()).abs().max()) <= 2.0 ** -6 and float((lse - wl).abs().max()) <= 2.0 ** -16
    ctx.close()


@pytest.mark.parametrize("t,top", [(40000, 300), (100001, 1000), (1 << 18, 1900), ((1 << 18) + 4003, 1900)])
def test_long_context_selection(cuda_device, t, top):
    # 2500, 6251 and 16384 blocks are selected from registers, 16635 from memory
    cache = Cache(1, 1, t, False, cuda_device)
    ctx = make_ctx(cache, 2)
    g = torch.Generator(device=cuda_device).manual_seed(3)
    cache.k.copy_(torch.randn(cache.k.shape, generator=g, device=cuda_device))
    cache.v.copy_(torch.randn(cache.v.shape, generator=g, device=cuda_device))
    cache.lens.fill_(t)
    ctx.block_bounds(cache.view(), cache.bounds(), 1)
    q = torch.randn(1, 2, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    q[0, 1] = 0.0                                                        # the whole middle ties
    q = q.to(cuda_device)
    blocks, count = torch.empty(1, 2, 2000, dtype=torch.int32, device=cuda_device), torch.empty(1, 2, dtype=torch.int32, device=cuda_device)
    out, lse = torch.empty_like(q), torch.empty(1, 2, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(top, 1, 1), 1, out, lse, blocks, count)
    assert ctx.check() == 0
    codes, scale = cache.codes[0, 0].cpu().numpy(), np64(cache.scale[0, 0])
    for u in range(2):
        want = R.select_blocks(R.block_scores(np64(q[0, u]), codes, scale), -(-t // 16), top, 1, 1)
        assert blocks[0, u].tolist()[: int(count[0, u])] == want
        pos = torch.tensor([i for j in want for i in range(16 * j, min(16 * j + 16, t))], device=cuda_device)
        y, l, tol, ltol = R.attend(np64(q[0, u]), np64(cache.k[0, 0, pos]), np64(cache.v[0, 0, pos]), True)
        assert np.all(np.abs(np64(out[0, u]) - y) <= tol) and abs(float(lse[0, u]) - l) <= ltol
    ctx.close()


def test_more_sequences_than_a_grid_axis_holds(cuda_device):
    """65600 sequences over the same pages, 73 blocks each: the result of sequence b is that of b mod 64."""
    batch, t, nb = 65600, 1165, 73
    g = torch.Generator().manual_seed(5)
    rows = torch.randn(2, nb * 16, 128, generator=g).to(torch.bfloat16)
    pool = rows.view(2, nb, 1, 16, 128).to(cuda_device)
    lens = torch.full((batch,), t, dtype=torch.int32, device=cuda_device)
    table = torch.arange(nb, dtype=torch.int32, device=cuda_device).expand(batch, nb).contiguous()
    view = P.make_view(pool[0], pool[1], lens, page_table=table)
    q64 = torch.randn(64, 1, 128, generator=g).to(torch.bfloat16)
    q = q64.repeat(batch // 64, 1, 1).to(cuda_device)
    blocks = torch.arange(nb, dtype=torch.int32, device=cuda_device).expand(batch, 1, nb).contiguous()
    count = torch.full((batch, 1), nb, dtype=torch.int32, device=cuda_device)
    out, lse = torch.full_like(q, math.nan), torch.full((batch, 1), math.nan, device=cuda_device)
    ctx = P.Context(1, batch, 1, 1, nb * 16, 16, 16, 4, page_size=16)
    ctx.block_decode_attn(q, view, blocks, count, batch, out, lse)
    assert ctx.check() == 0
    assert torch.equal(out, out[:64].repeat(batch // 64, 1, 1)) and torch.equal(lse, lse[:64].repeat(batch // 64, 1))
    for b in (0, 5, 63):
        y, l, tol, ltol = R.attend(np64(q64[b, 0]), rows[0, :t].double().numpy(), rows[1, :t].double().numpy(), True)
        assert np.all(np.abs(np64(out[b, 0]) - y) <= tol) and abs(float(lse[b, 0]) - l) <= ltol
    ctx.close()


def test_offsets_beyond_32_bits(cuda_device):
    # pages whose rows lie more than 2^32 elements behind the base
    H, pool = 8, (1 << 32) // (8 * 16 * 128) + 40
    k, v = (torch.empty(pool, H, 16, 128, dtype=torch.bfloat16, device=cuda_device) for _ in range(2))
    codes, scale = torch.empty(pool, H, 2, 128, dtype=torch.int8, device=cuda_device), torch.empty(pool, H, device=cuda_device)
    table_cpu = (torch.arange(40, dtype=torch.int32) + (pool - 40)).flip(0).view(1, 40)
    t = 633
    rows = random_rows(1, H, t, 21)
    for w, x in enumerate((k, v)):
        for j in range(40):
            part = rows[w, 0, :, 16 * j: min(16 * j + 16, t)]
            x[int(table_cpu[0, j]), :, : part.shape[1]] = part.to(cuda_device)
    lens = torch.tensor([t], dtype=torch.int32, device=cuda_device)
    view = P.make_view(k, v, lens, page_table=table_cpu.to(cuda_device))
    bounds = P.make_block_bounds(codes, scale)
    ctx = P.Context(1, 1, H, H, 640, 16, 16, 4, page_size=16)
    ctx.block_bounds(view, bounds, 1)
    q = torch.randn(1, H, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(cuda_device)
    blocks, count = torch.empty(1, H, 12, dtype=torch.int32, device=cuda_device), torch.empty(1, H, dtype=torch.int32, device=cuda_device)
    out, lse = torch.empty_like(q), torch.empty(1, H, device=cuda_device)
    ctx.block_decode_step(q, view, bounds, P.make_block_schedule(10, 1, 1), 1, out, lse, blocks, count)
    assert ctx.check() == 0
    for h in range(H):
        x = rows[0, 0, h].double().numpy()
        ref = [R.block_bounds(x[16 * j: 16 * j + 16]) for j in range(40)]
        want = R.select_blocks(R.block_scores(np64(q[0, h]), np.stack([c for c, _ in ref]), np.array([s for _, s in ref])), 40, 10, 1, 1)
        assert blocks[0, h].tolist() == want
        pos = [i for j in want for i in range(16 * j, min(16 * j + 16, t))]
        y, l, tol, ltol = R.attend(np64(q[0, h]), x[pos], rows[1, 0, h].double().numpy()[pos], True)
        assert np.all(np.abs(np64(out[0, h]) - y) <= tol) and abs(float(lse[0, h]) - l) <= ltol
    ctx.close()


def test_steps_on_another_stream_and_two_graphs_of_one_context(cuda_device):
    cache = Cache(2, 2, 500, True, cuda_device)
    ctx = make_ctx(cache, 2)
    cache.place(random_rows(2, 2, 500, 8), [500, 77])
    ctx.block_bounds(cache.view(), cache.bounds(), 2)
    sched = P.make_block_schedule(6, 1, 2)
    qs = [torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(cuda_device) for i in range(2)]
    new = lambda: (torch.empty_like(qs[0]), torch.empty(2, 4, device=cuda_device), torch.empty(2, 4, 9, dtype=torch.int32, device=cuda_device),  # noqa: E731
                   torch.empty(2, 4, dtype=torch.int32, device=cuda_device))
    want = [new(), new()]
    for q, w in zip(qs, want):
        ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, 2, *w)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), [new(), new()]
    with torch.cuda.stream(side):
        for q, w in zip(qs, got):
            ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, 2, *w)
    side.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    graphs, got = [], [new(), new()]
    for q, w in zip(qs, got):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            ctx.block_decode_step(q, cache.view(), cache.bounds(), sched, 2, *w)
    for _ in range(3):
        for w in got:
            for x in w:
                x.fill_(9)
        for g in graphs:                                                   # one after the other on one stream
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    assert ctx.check() == 0
    ctx.close()


# ------------------------------------------------------------------------------ not finite
def mild(rows):
    """Keys small enough that no weight vanishes."""
    rows[0] *= 0.25
    return rows


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("heads,group,shared,batch", [(2, 2, False, 2), (1, 12, True, 2), (8, 4, True, 60), (16, 2, False, 60)])
def test_a_key_that_is_not_finite_shows(cuda_device, bad, heads, group, shared, batch):
    """The softmax over a NaN, or over an infinite logit, is NaN: for the heads that meet it and for no other, however the
    list is dealt (parts, whole units, a warp per unit)."""
    lens = [400 - 3 * b for b in range(batch)]
    cache = Cache(batch, heads, 400, True, cuda_device, seed=2)
    ctx = make_ctx(cache, group)
    rows = mild(random_rows(batch, heads, 400, 31))
    q = torch.randn(batch, heads * group, 128, generator=torch.Generator().manual_seed(1)).abs().to(torch.bfloat16)
    hit = [(0, 0, 37), (1, heads - 1, lens[1] - 1)]                       # an ordinary block, the open one
    for b, h, i in hit:
        rows[0, b, h, i, 5] = bad                                        # q > 0: the logit is +inf or NaN
    cache.place(rows, lens)
    units = heads if shared else heads * group
    nb = [-(-t // 16) for t in lens]
    blocks = torch.zeros(batch, units, 25, dtype=torch.int32)
    count = torch.zeros(batch, units, dtype=torch.int32)
    for b in range(batch):
        blocks[b, :, : nb[b]], count[b] = torch.arange(nb[b]), nb[b]
    skip = units - 1                                                     # the last unit of sequence 0 leaves block 2 out
    blocks[0, skip, : nb[0] - 1], count[0, skip] = torch.tensor([j for j in range(nb[0]) if j != 2]), nb[0] - 1
    q = q.to(cuda_device)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=cuda_device)
    ctx.block_decode_attn(q, cache.view(), blocks.to(cuda_device), count.to(cuda_device), batch, out, lse, P.PRHS_GROUP_SETS if shared else 0)
    y, l, per = np64(out), np64(lse), group if shared else 1
    for b in range(batch):
        for u in range(heads * group):
            listed = blocks[b, u // per, : count[b, u // per]].tolist()
            met = any((b, u // group) == x[:2] and x[2] // 16 in listed for x in hit)
            if met:
                assert np.isnan(y[b, u]).all() and np.isnan(l[b, u]), (b, u)
            else:
                pos = [i for j in listed for i in range(16 * j, min(16 * j + 16, lens[b]))]
                k, v = (rows[w, b, u // group].double().numpy()[pos] for w in range(2))
                want, wl, tol, ltol = R.attend(np64(q[b, u]), k, v, True)
                assert np.all(np.abs(y[b, u] - want) <= tol) and abs(l[b, u] - wl) <= ltol, (b, u)
    ctx.close()


def test_values_and_queries_that_are_not_finite_show_in_a_step(cuda_device):
    cache = Cache(3, 2, 700, False, cuda_device)
    ctx = make_ctx(cache, 2)
    rows, lens = mild(random_rows(3, 2, 700, 5)), [700, 650, 333]
    rows[1, 0, 0, 3, 9], rows[1, 1, 1, 649, 11], rows[0, 2, 1, 332, 7] = math.nan, math.inf, -math.inf
    cache.place(rows, lens)
    ctx.block_bounds(cache.view(), cache.bounds(), 3)
    try:                                                                 # the infinite key may be recorded
        ctx.check()
    except P.PrhsError:
        pass
    q = torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    q[0, 3, 77] = math.nan
    q[2, 2:, 7] = 1.0                                                    # the key's logit is -inf: no weight, its value counts nothing
    q = q.to(cuda_device)
    blocks, count = torch.empty(3, 4, 44, dtype=torch.int32, device=cuda_device), torch.empty(3, 4, dtype=torch.int32, device=cuda_device)
    out, lse = torch.full_like(q, 7.0), torch.full((3, 4), 7.0, device=cuda_device)
    ctx.block_decode_step(q, cache.view(), cache.bounds(), P.make_block_schedule(50, 1, 1), 3, out, lse, blocks, count)
    y, l = np64(out), np64(lse)
    assert np.isnan(y[0, 3]).all() and np.isnan(l[0, 3])
    rows[1, 0, 0, 3, 9], rows[1, 1, 1, 649, 11] = 0, 0
    for b, u, d in [(0, 0, 9), (0, 1, 9), (0, 2, None), (1, 0, None), (1, 1, None), (1, 2, 11), (1, 3, 11), (2, 0, None), (2, 2, None), (2, 3, None)]:
        k, v = (rows[w, b, u // 2, : lens[b]].double().numpy() for w in range(2))
        keep = np.arange(lens[b]) != (332 if (b, u // 2) == (2, 1) else -1)
        want, wl, tol, ltol = R.attend(np64(q[b, u]), k[keep], v[keep], True)
        rest = np.arange(128) != (-1 if d is None else d)
        assert np.all(np.abs(y[b, u] - want)[rest] <= tol[rest]) and abs(l[b, u] - wl) <= ltol, (b, u)
        assert d is None or not np.isfinite(y[b, u, d]), (b, u)
    ctx.close()


def coded(x):
    """int8 codes and scale of numbers among which are infinities (the largest code; the scale follows their exponent) and NaNs
    (left out)."""
    finite = np.where(np.isnan(x), 0.0, x)
    s = 2.0 ** 122 if np.isinf(finite).any() else float(R.scale_of(np.abs(finite).max(), 127.0))
    return np.clip(np.where(np.isinf(finite), np.sign(finite) * 127, np.rint(np.where(np.isinf(finite), 0, finite) / s)), -127, 127), s


@pytest.mark.parametrize("paged", [False, True])
def test_bounds_and_scores_of_numbers_that_are_not_finite(cuda_device, paged):
    cache = Cache(1, 2, 320, paged, cuda_device)
    ctx = make_ctx(cache, 2)
    rows = random_rows(1, 2, 320, 17)
    rows[0, 0, 0, 20, 3], rows[0, 0, 0, 40, 4], rows[0, 0, 0, 41, 4] = math.inf, math.inf, -math.inf
    rows[0, 0, 1, 50, 5], rows[0, 0, 1, 64:80, 6], rows[0, 0, 1, 81] = math.nan, math.nan, math.nan
    rows[0, 0, 1, 100, 7], rows[0, 0, 1, 101, 7] = math.nan, -math.inf
    cache.place(rows, [320])
    ctx.block_bounds(cache.view(), cache.bounds(), 1)
    with pytest.raises(P.PrhsError) as e:                                 # recorded
        ctx.check()
    assert e.value.status == 7
    bounds = {}
    for h in range(2):
        for j in range(20):
            x = rows[0, 0, h, 16 * j: 16 * j + 16].double().numpy()
            lo, hi = np.where(np.isnan(x), math.inf, x).min(0), np.where(np.isnan(x), -math.inf, x).max(0)
            empty = np.isnan(x).all(0)
            want, s = coded(np.stack([np.where(empty, 0, lo), np.where(empty, 0, hi)]))
            got, gs = cache.bound_of(0, h, j)
            assert gs == s and np.array_equal(got, want), (h, j)
            bounds[h, j] = want, s
    q = torch.randn(1, 4, 128, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    q[0, 0, 3], q[0, 1, 9], q[0, 3, 5] = 2.0, math.inf, -math.inf
    q[0, 1, 8], q[0, 3, 4], q[0, 3, 6] = 1.0, -1.0, 1.0                   # neighbours of the infinite element keep their codes
    blocks, count = torch.empty(1, 4, 5, dtype=torch.int32, device=cuda_device), torch.empty(1, 4, dtype=torch.int32, device=cuda_device)
    ctx.block_topk(q.to(cuda_device), cache.view(), cache.bounds(), P.make_block_schedule(5, 0, 0), 1, blocks, count)
    for u in range(4):
        q8, qs = coded(np64(q[0, u]))
        score = [np.maximum(q8 * bounds[u // 2, j][0][0], q8 * bounds[u // 2, j][0][1]).sum() * bounds[u // 2, j][1] * qs for j in range(20)]
        with np.errstate(over="ignore"):
            score = [float(np.float32(x)) for x in score]
        assert blocks[0, u].tolist() == R.select_blocks(score, 20, 5, 0, 0), u
    assert 1 in blocks[0, 0].tolist()                                     # q . k is +inf in block 1: it is attended over
    ctx.close()


# -------------------------------------------------------------------------------- refusals
def test_tensors_of_a_view_elsewhere_are_refused(cuda_device):
    """Host lengths or page tables, fewer rows than the batch, values of another size: refused before any kernel."""
    for paged in (False, True):
        cache = Cache(2, 2, 64, paged, cuda_device)
        ctx = make_ctx(cache, 2)
        cache.place(random_rows(2, 2, 64, 1), [64, 64])
        q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=cuda_device)
        out = torch.full_like(q, 7.0)
        blocks, count = torch.zeros(2, 4, 4, dtype=torch.int32, device=cuda_device), torch.zeros(2, 4, dtype=torch.int32, device=cuda_device)
        sched = P.make_block_schedule(1, 1, 1)
        wrong = [dict(lens=cache.lens.cpu()), dict(v=cache.v.cpu()), dict(v=cache.v[:1]), dict(lens=cache.lens[None]),
                 dict(lens=torch.zeros(3, dtype=torch.int32, device=cuda_device)[::2]), dict(lens=cache.lens[:1])]
        wrong += [dict(table=cache.table.cpu()), dict(table=cache.table[:1]), dict(table=cache.table[0])] if paged else [dict(k=cache.k[:1], v=cache.v[:1])]
        for w in wrong:
            a = {**dict(k=cache.k, v=cache.v, lens=cache.lens, table=cache.table), **w}
            view = P.make_view(a["k"], a["v"], a["lens"], page_table=a["table"])
            for call in (lambda: ctx.block_bounds(view, cache.bounds(), 2),
                         lambda: ctx.block_topk(q, view, cache.bounds(), sched, 2, blocks, count),
                         lambda: ctx.block_decode_attn(q, view, blocks, count, 2, out),
                         lambda: ctx.block_decode_step(q, view, cache.bounds(), sched, 2, out, None, blocks, count)):
                with pytest.raises(AssertionError):
                    call()
        torch.cuda.synchronize()
        assert bool((out == 7.0).all()) and bool((cache.scale == 99.0).all())
        ctx.close()


def test_a_slice_of_a_page_table_bounds_the_lengths(cuda_device):
    """Columns beyond the slice are another's: a length that would need them is cut and recorded."""
    cache = Cache(2, 2, 160, True, cuda_device)
    ctx = make_ctx(cache, 2)
    rows = random_rows(2, 2, 160, 3)
    cache.place(rows, [160, 160])
    ctx.block_bounds(cache.view(), cache.bounds(), 2)
    assert ctx.check() == 0
    view = P.make_view(cache.k, cache.v, cache.lens, page_table=cache.table[:, :5])
    q = torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(cuda_device)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device=cuda_device)
    blocks, count = torch.empty(2, 4, 5, dtype=torch.int32, device=cuda_device), torch.empty(2, 4, dtype=torch.int32, device=cuda_device)
    for lens, cut in (([80, 33], 0), ([81, 160], 1)):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ctx.block_decode_step(q, view, cache.bounds(), P.make_block_schedule(3, 1, 1), 2, out, lse, blocks, count)
        if cut:
            with pytest.raises(P.PrhsError):
                ctx.check()
        assert ctx.check() == 0
        lens = [min(t, 80) for t in lens]
        sets = {(b, u): list(range(-(-t // 16))) for b, t in enumerate(lens) for u in range(4)}
        for (b, u), w in sets.items():
            assert blocks[b, u].tolist()[: len(w)] == w
        check_attention(cache, np64(q), lens, 2, sets, False, out, lse)
    ctx.close()


def test_refusals(cuda_device):
    cache = Cache(2, 2, 64, False, cuda_device)
    ctx = make_ctx(cache, 2)
    cache.place(random_rows(2, 2, 64, 1), [64, 64])
    lib, C = ctx.lib, P.C
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=cuda_device)
    out = torch.full_like(q, 7.0)
    blocks, count = torch.zeros(2, 4, 4, dtype=torch.int32, device=cuda_device), torch.zeros(2, 4, dtype=torch.int32, device=cuda_device)
    st = torch.cuda.current_stream().cuda_stream
    INVALID, CAPACITY = 1, 6

    def bounds(bd=None, view=None, new=0, b=2):
        bd, view = bd or cache.bounds(), view or cache.view()
        return lib.prhs_block_bounds(ctx.h, C.byref(view), C.byref(bd), None, new, b, st)

    def step(sched=None, bd=None, view=None, stride=4, o=None, cnt=None):
        bd, view, sched = bd or cache.bounds(), view or cache.view(), sched or P.make_block_schedule(1, 1, 1)
        return lib.prhs_block_decode_step(ctx.h, q.data_ptr(), C.byref(view), C.byref(bd), C.byref(sched), 2,
                                          out.data_ptr() if o is None else o, None, blocks.data_ptr(), stride,
                                          count.data_ptr() if cnt is None else cnt, st)

    def attn(stride=4, flags=0):
        view = cache.view()
        return lib.prhs_block_decode_attn(ctx.h, q.data_ptr(), C.byref(view), blocks.data_ptr(), count.data_ptr(), stride, flags, 2,
                                          out.data_ptr(), None, st)

    assert bounds() == 0 and step() == 0 and attn() == 0
    torch.cuda.synchronize()
    out.fill_(7.0)
    for field, value in [("codes", None), ("scale", None), ("codes", cache.codes.data_ptr() + 8), ("stride_outer", 0), ("stride_head", -1)]:
        bd = cache.bounds()
        setattr(bd, field, value)
        assert bounds(bd) == INVALID and step(bd=bd) == INVALID, field
    assert bounds(new=-1) == INVALID and bounds(b=3) == CAPACITY
    for sched, status in [(P.make_block_schedule(-1, 1, 1), INVALID), (P.make_block_schedule(1, -1, 1), INVALID),
                          (P.make_block_schedule(1, 1, 0), INVALID), (P.make_block_schedule(1, 1, 1, 1), INVALID),
                          (P.make_block_schedule(1 << 20, 1, 1), CAPACITY), (P.make_block_schedule(9, 1, 1), None)]:
        assert step(sched) == (0 if status is None else status)           # nine middle blocks: the context has four in all
    torch.cuda.synchronize()
    out.fill_(7.0)
    assert step(P.make_block_schedule(9, 1, 1), stride=3) == CAPACITY
    assert step(o=out.data_ptr() + 2) == INVALID and step(o=q.data_ptr() + 1024) == INVALID
    view = cache.view()
    view.max_seq_len = 65
    assert step(view=view) == CAPACITY and bounds(view=view) == CAPACITY
    assert attn(stride=0) == INVALID and attn(flags=1) == INVALID
    assert lib.prhs_block_topk(None, q.data_ptr(), C.byref(view), None, None, 2, blocks.data_ptr(), 4, count.data_ptr(), st) == INVALID
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    with pytest.raises(AssertionError):
        ctx.block_decode_attn(q, cache.view(), blocks[:, :2].contiguous(), count[:, :2].contiguous(), 2, out)
    with pytest.raises(AssertionError):
        P.make_block_bounds(cache.codes.float(), cache.scale)
    pc = Cache(1, 1, 64, True, cuda_device)
    pctx = make_ctx(pc, 1)
    pview, pb = pc.view(), pc.bounds()
    pview.page_table_stride = 3
    assert lib.prhs_block_bounds(pctx.h, C.byref(pview), C.byref(pb), None, 0, 1, st) == INVALID
    pctx.close()
    ctx.close()
