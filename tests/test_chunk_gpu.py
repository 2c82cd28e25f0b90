"""Attention of many new tokens against its 64-bit form.

Error bound, with A = sum_i p_i |v_i| (p normalised) over the n positions that a token sees: logits, 131 fp32 operations of at most 2^-23
each, e = s 131 * 2^-23 sum|q k|, s = 128^-1/2; exponentials to 2^-20; weights rounded to bf16, half a step, 2^-8; n additions in
numerator and divisor, 2^-23 each; the result's rounding 2^-8 |y| and 2^-134.  That is the bound of one value.  Over many values the
roundings are independent: two of 2^-8 at most, uniform within it, are sqrt(2 / 3) 2^-8 = 0.0032 of the norm.
"""
import math

import pytest
import torch

from paper_2602_08329_b200 import binding as P
from tests.test_tokens_gpu import BF, Batch, bits, freqs

pytestmark = pytest.mark.gpu
S = 128 ** -0.5


def fill(t, seed=0, k_amp=1.0):
    """Random rows of every position that a sequence has; q packed, contiguous.  Everything else stays NaN."""
    g = torch.Generator().manual_seed(seed)
    t.full_k, t.full_v = [], []
    for b, n in enumerate(t.lens):
        k, v = (torch.randn(t.H, n, 128, generator=g) * k_amp).to(BF), torch.randn(t.H, n, 128, generator=g).to(BF)
        t.full_k.append(k.to(t.dev))
        t.full_v.append(v.to(t.dev))
    store(t)
    t.qc = t.q.contiguous()
    t.out = torch.full_like(t.qc, math.nan)
    t.lse = torch.full(t.qc.shape[:2], math.nan, device=t.dev)
    return t


def store(t):
    for b, n in enumerate(t.lens):
        for c, x in ((t.ck, t.full_k[b]), (t.cv, t.full_v[b])):
            if t.paged:
                for j in range(0, n, 16):
                    m = min(16, n - j)
                    c[int(t.table[b, j // 16]), :, :m] = x[:, j:j + m]
            else:
                c[b, :, :n] = x


def first_visible(u, window, share):
    lo = max(0, min(math.floor(share * u), u))
    return max(lo, u - window) if window else lo


def reference(t, sinks=0, window=0, share=0.0):
    """out, lse, bound on out, bound on lse over the packed rows (float64); rows of no sequence NaN."""
    rows, Hq = t.qc.shape[:2]
    out, lse, tol, ltol = (torch.full((rows, Hq, 128)[:n], math.nan, dtype=torch.float64, device=t.dev) for n in (3, 2, 3, 2))
    for b, n in enumerate(t.new):
        if not n:
            continue
        T, r0 = t.lens[b], t.starts[b]
        u = torch.arange(T - n + 1, T + 1, device=t.dev)
        lo = torch.tensor([first_visible(int(x), window, share) for x in u], device=t.dev)
        i = torch.arange(T, device=t.dev)
        see = (i < u[:, None]) & ((i < sinks) | (i >= lo[:, None]))
        for h in range(Hq):
            k, v, q = t.full_k[b][h // t.G].double(), t.full_v[b][h // t.G].double(), t.qc[r0:r0 + n, h].double()
            a = (q @ k.T * S).masked_fill(~see, -math.inf)
            z = torch.logsumexp(a, -1)
            p = torch.exp(a - z.masked_fill(z == -math.inf, 0.0)[:, None])
            y = p @ torch.where(torch.isfinite(v), v, 0.0)
            e = (S * 131 * 2.0 ** -23 * (q.abs() @ k.abs().T)).masked_fill(~see, 0.0).amax(-1)
            e = torch.nan_to_num(e, nan=0.0, posinf=0.0)
            big = p @ torch.nan_to_num(v.abs(), nan=0.0, posinf=0.0)
            out[r0:r0 + n, h], lse[r0:r0 + n, h] = y, z
            tol[r0:r0 + n, h] = 2.0 ** -8 * y.abs() + (2 * e + 2.0 ** -20 + T * 2.0 ** -22 + 2.0 ** -8)[:, None] * big + 2.0 ** -134
            ltol[r0:r0 + n, h] = e + 2.0 ** -20 + T * 2.0 ** -23 + 2.0 ** -22 * torch.nan_to_num(z.abs(), posinf=0.0)
    return out, lse, tol, ltol


def compare(t, **kw):
    out, lse, tol, ltol = reference(t, **kw)
    live = t.starts[-1]
    got, gl = t.out.double(), t.lse.double()
    assert torch.isnan(got[live:]).all() and torch.isnan(gl[live:]).all()
    got, gl, out, lse, tol, ltol = (x[:live] for x in (got, gl, out, lse, tol, ltol))
    assert torch.isfinite(got).all()
    worst = ((got - out).abs() / tol).max() if live else torch.zeros(())
    assert worst <= 1.0, worst
    empty = lse == -math.inf
    assert torch.equal(empty, gl == -math.inf) and not got[empty].any()
    assert (((gl - lse).abs() / ltol)[~empty] <= 1.0).all()
    if live * t.Hq >= 64 and not empty.any():
        assert torch.linalg.norm(got - out) <= 0.0033 * torch.linalg.norm(out)


def call(t, ctx=None, mask=None, row_start=True, **kw):
    ctx = ctx or t.ctx()
    ctx.chunk_attn(t.qc, t.view(**kw), t.B, t.out, t.lse, row_start=t.row_start if row_start else None, mask=mask)
    assert ctx.check() == 0
    return ctx


# the new tokens of a sequence fill one row, part of a subtile, exactly one, several items; lengths around tiles and pages
SHAPES = [([1], [1]), ([5, 1, 128, 129], [5, 1, 128, 129]), ([300, 17, 40, 256], [3, 0, 40, 1]), ([700], [700]), ([1000, 33, 512], [130, 33, 1]),
          ([2500, 3], [5, 2]), ([384, 640], [256, 257])]


@pytest.mark.parametrize("lens,new", SHAPES)
@pytest.mark.parametrize("kv_heads,group", [(2, 4), (1, 7), (3, 1), (1, 16), (2, 3)])
@pytest.mark.parametrize("paged", [False, True])
def test_causal(cuda_device, lens, new, kv_heads, group, paged):
    t = fill(Batch(cuda_device, lens, new, kv_heads, group, paged, seed=len(lens)), seed=group)
    call(t)
    compare(t)


@pytest.mark.parametrize("sinks,window,layer", [(4, 100, -1), (0, 1, -1), (130, 64, -1), (0, 128, -1), (200, 0, 30), (4, 700, 31), (5000, 3, 31), (0, 0, 28)])
@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("paged", [False, True])
def test_masks(cuda_device, sinks, window, layer, group, paged):
    """First positions, a window, the window that slides with depth, and together."""
    t = fill(Batch(cuda_device, [900, 129, 1400], [700, 129, 6], 2, group, paged, seed=1))
    ctx = P.Context(num_layers=32, max_batch=3, num_q_heads=2 * group, num_kv_heads=2, max_context=t.cap, max_k=1, max_window=1, max_sinks=4,
                    page_size=16 if paged else 0, min_layer_group=32)
    mask = P.make_chunk_mask(sinks=sinks, window=window, layer=max(layer, 0), psaw_layer_start=24 if layer >= 0 else 0)
    call(t, ctx, mask)
    share = 1.0 - float(torch.tensor(0.7)) ** ((layer + 1 - 24) / 8) if layer + 1 >= 24 else 0.0
    compare(t, sinks=sinks, window=window, share=share)


def test_a_mask_that_leaves_rows_empty(cuda_device):
    """phi^alpha rounds to nothing: every position before the token's own end is masked."""
    t = fill(Batch(cuda_device, [300, 128], [200, 128], 1, 2, False))
    ctx = P.Context(num_layers=2, max_batch=2, num_q_heads=2, num_kv_heads=1, max_context=t.cap, max_k=1, max_window=1, max_sinks=4)
    for sinks in (0, 3):
        t.out.fill_(math.nan)
        call(t, ctx, P.make_chunk_mask(sinks=sinks, layer=1, psaw_layer_start=1, psaw_phi=1e-30, psaw_alpha=100.0))
        compare(t, sinks=sinks, share=1.0)


@pytest.mark.parametrize("batch,new,length", [(1, 3, 20000), (1, 300, 9000), (3, 1, 30001), (40, 2, 700)])
@pytest.mark.parametrize("paged", [False, True])
def test_items_in_many_pieces_and_few(cuda_device, batch, new, length, paged):
    lens = [max(new, length - 37 * b) for b in range(batch)]
    t = fill(Batch(cuda_device, lens, [new] * batch, 1 if batch < 3 else 2, 4, paged), k_amp=0.5)
    ctx = call(t)
    compare(t)
    first = (t.out.clone(), t.lse.clone())
    for _ in range(3):                          # the order of arrival does not show
        call(t, ctx)
        assert torch.equal(first[0].view(torch.int16), t.out.view(torch.int16)) and torch.equal(first[1].view(torch.int32), t.lse.view(torch.int32))


@pytest.mark.parametrize("lens,new,group", [([3000, 50], [5, 1], 4), ([300, 300, 1000, 65], [0, 60, 1, 0], 4), ([700], [9], 7), ([20000], [8], 8), ([513], [64], 1), ([900], [4], 16)])
def test_few_tokens_have_weights_of_two_parts(cuda_device, lens, new, group):
    """Up to 64 / group rows per sequence on average: the error is that of the result's own rounding, at most 2^-8 and so 2^-8 / sqrt(3) = 0.00226 of
    the norm, where a weight of one part brings as much again (0.0032)."""
    t = fill(Batch(cuda_device, lens, new, 4, group, False, pad_rows=0), k_amp=0.3)
    call(t)
    compare(t)
    out = reference(t)[0][:t.starts[-1]]
    assert torch.linalg.norm(t.out[:t.starts[-1]].double() - out) <= 0.00226 * torch.linalg.norm(out)


def test_one_token_is_what_dense_decode_gives(cuda_device):
    t = fill(Batch(cuda_device, [2047, 1, 16, 400], [1] * 4, 4, 8, True, pad_rows=0))
    ctx = call(t, row_start=False)
    compare(t)
    out, lse = torch.empty_like(t.out), torch.empty_like(t.lse)
    ctx.dense_decode_attn(t.qc, t.view(), 4, out, lse)
    assert torch.allclose(lse, t.lse, rtol=2.0 ** -20, atol=2.0 ** -18)
    assert (out.float() - t.out.float()).abs().max() <= 2.0 ** -6 * out.float().abs().max()      # two roundings of each


def test_references_that_keep_rising(cuda_device):
    """Every tile's logits exceed those before by more than 2^8: the accumulators are rescaled each time."""
    t = fill(Batch(cuda_device, [1100], [400], 1, 2, False))
    scale = torch.exp2((torch.arange(1100, device=cuda_device) // 128).float() * 0.75)
    t.full_k[0] = (t.full_k[0].float() * scale[:, None]).to(BF)
    t.qc[:, :] = (t.qc.float() * 4).to(BF)
    store(t)
    call(t)
    compare(t)


def test_extreme_logits(cuda_device):
    """One key far above the others; all logits equal; logits of zero."""
    t = fill(Batch(cuda_device, [260, 260, 260], [130, 130, 130], 1, 1, False))
    t.full_k[0][:, 7] *= 100
    t.full_k[1][:] = t.full_k[1][:, :1]
    t.full_k[2][:] = 0
    store(t)
    call(t)
    compare(t)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("lens,new,group", [([300], [200], 1), ([300], [200], 4), ([129], [3], 4), ([5000], [2], 7)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(cuda_device, paged, lens, new, group):
    t = fill(Batch(cuda_device, lens, new, 2, group, paged))
    T, n = lens[0], new[0]
    odd = [(0, T - 1, 3, math.inf), (0, T - 2, 70, -math.inf), (1, T - n, 5, math.nan), (1, T - 1, 127, math.inf), (1, T - 1, 126, -math.inf),
           (0, T // 2, 9, math.nan)]
    for h, pos, d, x in odd:
        t.full_v[0][h, pos, d] = x
    store(t)
    call(t)
    out, lse, tol, _ = reference(t)
    u = torch.arange(T - n + 1, T + 1, device=t.dev)
    want = out[:n].clone()
    for h, pos, d, x in odd:
        sel = torch.zeros(n, t.Hq, 128, dtype=torch.bool, device=t.dev)
        sel[u > pos, h * group:(h + 1) * group, d] = True
        want[sel] = want[sel] + x
    got = t.out[:n].double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(want), torch.isnan(got)) and torch.equal(torch.isfinite(got), fine)
    assert torch.equal(want[~fine & ~torch.isnan(want)], got[~fine & ~torch.isnan(want)])
    assert (((got - want).abs() / tol[:n])[fine] <= 1.0).all()


def test_keys_that_are_not_finite(cuda_device):
    """A NaN or +inf logit makes the rows that see it NaN, and no others; one of -inf has no weight."""
    t = fill(Batch(cuda_device, [200], [150], 1, 2, False))
    t.qc[:, :, 0] = 1.0
    for pos, x in ((190, math.nan), (180, math.inf), (60, -math.inf)):
        t.full_k[0][0, pos] = 0.0
        t.full_k[0][0, pos, 0] = x
    store(t)
    ctx = t.ctx()
    ctx.chunk_attn(t.qc, t.view(), 1, t.out, t.lse, row_start=t.row_start)
    t.full_k[0][0, 190], t.full_k[0][0, 180] = 0.0, 0.0
    out, lse, tol, _ = reference(t)
    sees = torch.arange(51, 201, device=t.dev) > 180
    assert torch.isnan(t.out[:150][sees]).all() and torch.isnan(t.lse[:150][sees]).all()
    got = t.out[:150][~sees].double()
    want = out[:150][~sees]
    assert torch.isfinite(got).all() and ((got - want).abs() <= tol[:150][~sees].nan_to_num(nan=math.inf)).all()


@pytest.mark.parametrize("paged", [False, True])
def test_sequences_that_do_not_fit_are_left_out_and_recorded(cuda_device, paged):
    t = fill(Batch(cuda_device, [200, 64, 30, 90], [150, 6, 7, 20], 1, 2, paged))
    t.lens_t.copy_(torch.tensor([200, 5, 30, 90], dtype=torch.int32))            # the second: six rows, five positions
    ctx = t.ctx()
    ctx.chunk_attn(t.qc, t.view(max_seq_len=128), 4, t.out, t.lse, row_start=t.row_start)       # and the first too long
    with pytest.raises(P.PrhsError):
        ctx.check()
    done = torch.zeros(t.rows, dtype=torch.bool)
    done[156:183] = True
    assert torch.equal(~torch.isnan(t.lse[:, 0]).cpu(), done)
    t.lens[1], keep = 64, (t.out.clone(), t.lse.clone())
    out, lse, tol, _ = reference(t)
    assert ((keep[0].double() - out).abs()[156:183] <= tol[156:183]).all()
    for starts in ([0, 150, 100, 120, 183], [0, 150, 156, 163, t.rows + 1], [-1, 150, 156, 163, 183]):
        ctx.chunk_attn(t.qc, t.view(), 4, t.out, t.lse, row_start=torch.tensor(starts, dtype=torch.int32, device=cuda_device))
        with pytest.raises(P.PrhsError):
            ctx.check()
    assert ctx.check() == 0


def test_a_page_outside_the_pool_counts_as_zeros(cuda_device):
    t = fill(Batch(cuda_device, [100], [40], 1, 2, True))
    t.table[0, 2] = 12345
    ctx = t.ctx()
    ctx.chunk_attn(t.qc, t.view(), 1, t.out, t.lse, row_start=t.row_start)
    with pytest.raises(P.PrhsError):
        ctx.check()
    t.full_k[0][:, 32:48] = 0
    t.full_v[0][:, 32:48] = 0
    compare(t)


def test_strides_of_the_cache_and_a_wider_table(cuda_device):
    """Heads of a larger allocation, sequences further apart than their capacity, page tables wider than needed."""
    t = fill(Batch(cuda_device, [150, 77], [60, 77], 2, 4, False))
    big = [torch.full((2, 5, t.cap + 32, 128), math.nan, dtype=BF, device=cuda_device) for _ in range(2)]
    for b, c in zip(big, (t.ck, t.cv)):
        b[:, 1:3, :t.cap] = c
    ctx = P.Context(num_layers=1, max_batch=4, num_q_heads=8, num_kv_heads=2, max_context=4096, max_k=1, max_window=1, max_sinks=4)
    ctx.chunk_attn(t.qc, P.make_view(big[0][:, 1:3, :], big[1][:, 1:3, :], t.lens_t), 2, t.out, t.lse, row_start=t.row_start)
    assert ctx.check() == 0
    compare(t)


def test_another_stream_and_captured_graphs_of_one_context(cuda_device):
    """Lengths and queries change between replays; two graphs of a context, replayed in turn on one stream."""
    t = fill(Batch(cuda_device, [3000, 700], [8, 8], 2, 4, True, pad_rows=0))
    t2 = fill(Batch(cuda_device, [400], [300], 2, 4, True, pad_rows=0), seed=3)
    ctx = P.Context(num_layers=1, max_batch=2, num_q_heads=8, num_kv_heads=2, max_context=3008, max_k=1, max_window=1, max_sinks=4, page_size=16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        for x in (t, t2):
            ctx.chunk_attn(x.qc, x.view(), x.B, x.out, x.lse, row_start=x.row_start)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                ctx.chunk_attn(x.qc, x.view(), x.B, x.out, x.lse, row_start=x.row_start)
            graphs.append(g)
    torch.cuda.synchronize()
    for lens in ([3000, 700], [2111, 9], [130, 650]):
        t.lens_t.copy_(torch.tensor(lens, dtype=torch.int32))
        for x in (t, t2):
            x.out.fill_(math.nan)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for g in graphs * 2:
                g.replay()
        torch.cuda.synchronize()
        keep = t.lens, t.full_k, t.full_v
        t.full_k, t.full_v = ([x[:, :n] for x, n in zip(c, lens)] for c in (t.full_k, t.full_v))
        t.lens = lens
        compare(t)
        compare(t2)
        t.lens, t.full_k, t.full_v = keep
    assert ctx.check() == 0


def test_prompt_then_tokens_as_a_program_would(cuda_device):
    """A prompt in two parts, then tokens: append, chunk attention, append, decode; the 8-bit cache read back for its prompt."""
    dev, H, G, n = cuda_device, 2, 4, 300
    g = torch.Generator().manual_seed(11)
    x = torch.randn(n + 4, H * G + 2 * H, 128, generator=g).to(BF).to(dev)
    prep = P.make_qk_prep((1 + 0.1 * torch.randn(128, generator=g)).to(dev), None, inv_freq=freqs(128).to(dev))
    ctx = P.Context(num_layers=1, max_batch=1, num_q_heads=H * G, num_kv_heads=H, max_context=320, max_k=300, max_window=16, max_sinks=4)
    ck, cv, rk, rv = (torch.full((1, H, 320, 128), math.nan, dtype=BF, device=dev) for _ in range(4))
    lens = torch.zeros(1, dtype=torch.int32, device=dev)
    kv = P.make_view(ck, cv, lens)
    c8 = [torch.zeros(1, H, 320, 128, dtype=torch.float8_e4m3fn, device=dev) for _ in range(2)]
    s8 = [torch.ones(1, H, 20, device=dev) for _ in range(2)]
    t8 = [torch.zeros(1, H, 16, 128, dtype=BF, device=dev) for _ in range(2)]
    kv8 = P.make_bytekv_view(*c8, *s8, *t8, lens)
    back = P.make_view(rk, rv, lens)
    sched = P.make_schedule(top_k=300, window=16, sinks=4)
    q_out = torch.empty(n + 4, H * G, 128, dtype=BF, device=dev)
    q8 = torch.empty_like(q_out)
    out, out8, step_out = torch.empty_like(q_out), torch.empty_like(q_out), torch.empty(4, 1, H * G, 128, dtype=BF, device=dev)
    for a, b in [(0, 170), (170, n)] + [(i, i + 1) for i in range(n, n + 4)]:
        lens.fill_(b)
        start = torch.tensor([0, b - a], dtype=torch.int32, device=dev)
        q, k, v = x[a:b, :H * G], x[a:b, H * G:-H], x[a:b, -H:]
        ctx.qkv_append(q, k, v, kv, prep, 1, q_out[a:b], row_start=start)
        ctx.bytekv_qkv_append(q, k, v, kv8, prep, 1, q8[a:b], row_start=start)
        ctx.chunk_attn(q_out[a:b], kv, 1, out[a:b], row_start=start)
        ctx.bytekv_read(kv8, back, 1)
        ctx.chunk_attn(q8[a:b], back, 1, out8[a:b], row_start=start)
        if b - a == 1:
            ctx.decode_step(0, a - n, sched, q_out[a:b], kv, 1, step_out[a - n])
    assert ctx.check() == 0 and torch.equal(q_out, q8)

    def attend(k, v):
        a = torch.einsum("nhgd,hid->nhgi", q_out.double().unflatten(1, (H, G)), k[0, :, :n + 4].double()) * S
        i = torch.arange(n + 4, device=dev)
        a.masked_fill_((i > i[:, None])[:, None, None], -math.inf)
        return torch.einsum("nhgi,hid->nhgd", a.softmax(-1), v[0, :, :n + 4].double()).flatten(1, 2)
    want = attend(ck, cv)
    assert torch.linalg.norm(out.double() - want) <= 0.0033 * torch.linalg.norm(want)
    for i in range(4):           # everything is selected: the decode step is dense attention, with weights in bf16 as well
        assert torch.linalg.norm(step_out[i, 0].double() - want[n + i]) <= 0.0046 * torch.linalg.norm(want[n + i])
    rk[:, :, n + 4:] = rv[:, :, n + 4:] = 0
    got8 = out8[n:].double()
    # (earlier rows were attended over while their block was still open: the last ones see the blocks as they are now)
    want8 = attend(rk, rv)[n + 3:]
    assert torch.linalg.norm(got8[3:] - want8) <= 0.0033 * torch.linalg.norm(want8)


def test_refusals(cuda_device):
    t = fill(Batch(cuda_device, [40, 40], [20, 3], 2, 2, False))
    ctx = t.ctx()
    ok = dict(row_start=t.row_start)
    for q, out, lse, kw in [(t.qc.float(), t.out, t.lse, ok), (t.qc, t.out[:-1], t.lse, ok), (t.qc, t.out, t.lse.double(), ok), (t.qc[:, :3], t.out, t.lse, ok),
                            (t.q, t.out, t.lse, ok), (t.qc, t.out, t.lse, {}), (t.qc, t.out, t.lse, dict(row_start=t.row_start[:2])), (t.qc, None, t.lse, ok),
                            (t.qc.cpu(), t.out, t.lse, ok), (t.qc, t.out, t.lse, dict(row_start=t.row_start.float()))]:
        with pytest.raises(AssertionError):
            ctx.chunk_attn(q, t.view(), 2, out, lse, **kw)
    with pytest.raises(P.PrhsError):
        ctx.chunk_attn(t.qc, t.view(), 2, t.qc, t.lse, **ok)
    for mask in (dict(sinks=-1), dict(window=-1), dict(psaw_layer_start=-1), dict(psaw_layer_start=1, psaw_phi=1.0), dict(psaw_layer_start=1, psaw_alpha=-1.0),
                 dict(psaw_layer_start=1, layer=1), dict(psaw_layer_start=1, layer=-1), dict(psaw_layer_start=1, psaw_phi=math.nan)):
        with pytest.raises(P.PrhsError):
            ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse, mask=P.make_chunk_mask(**mask), **ok)
    with pytest.raises(AssertionError):
        ctx.chunk_attn(t.qc, t.view(), 3, t.out, t.lse, **ok)
    ctx.chunk_attn(t.qc[:0], t.view(), 2, t.out[:0], t.lse[:0], row_start=torch.zeros(3, dtype=torch.int32, device=cuda_device))
    assert ctx.check() == 0 and torch.isnan(t.out).all()


@pytest.mark.parametrize("paged", [False, True])
def test_many_sequences_some_without_tokens(cuda_device, paged):
    g = torch.Generator().manual_seed(8)
    lens = torch.randint(0, 150, (300,), generator=g).tolist()
    new = [min(n, int(m)) for n, m in zip(lens, torch.randint(0, 4, (300,), generator=g))]
    new[37] = lens[37] = 140
    t = fill(Batch(cuda_device, lens, new, 1, 2, paged))
    call(t)
    compare(t)


def test_rows_of_no_sequence_alone(cuda_device):
    """Padding only: nothing is computed, nothing written, and the next call is as ever."""
    t = fill(Batch(cuda_device, [40, 200], [0, 0], 2, 4, False, pad_rows=300))
    ctx = call(t)
    assert torch.isnan(t.out).all() and torch.isnan(t.lse).all()
    t.row_start[2] = 5
    ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse, row_start=t.row_start)
    assert ctx.check() == 0 and int((~torch.isnan(t.lse[:, 0])).sum()) == 0      # (padding rows hold NaN queries: their rows are NaN)
    prep = P.make_qk_prep()
    t.row_start.zero_()
    t.ck.fill_(math.nan)
    ctx.qkv_append(t.q, t.k, t.v, t.view(), prep, 2, t.q_out, row_start=t.row_start)
    assert ctx.check() == 0 and torch.isnan(t.ck).all() and torch.isnan(t.q_out).all()


@pytest.mark.parametrize("paged", [False, True])
def test_short_pieces_without_mending_after_launches_with_notes(cuda_device, paged):
    """Pieces of a few tiles that every row sees whole, on SMs whose shared memory still holds the notes of a launch that mended many: the first
    tiles of a short cache are a piece of their own (four draft tokens over 2047 positions: two tiles), and nothing orders it but its notes' barrier."""
    odd = fill(Batch(cuda_device, [500] * 16, [200] * 16, 2, 4, paged, pad_rows=0))
    for b in range(16):
        odd.full_v[b][:, 300::7, 3] = math.inf
    store(odd)
    ctx = P.Context(num_layers=1, max_batch=16, num_q_heads=8, num_kv_heads=2, max_context=2048, max_k=1, max_window=1, max_sinks=4,
                    page_size=16 if paged else 0)
    for lens, new in (([2047], [4]), ([2047, 300, 900], [4, 1, 2]), ([2047] * 12, [60] * 12)):
        t = fill(Batch(cuda_device, lens, new, 2, 4, paged, pad_rows=0), seed=len(lens))
        for _ in range(20):
            ctx.chunk_attn(odd.qc, odd.view(), 16, odd.out, odd.lse, row_start=odd.row_start)
            ctx.chunk_attn(t.qc, t.view(), t.B, t.out, t.lse, row_start=t.row_start)
            t.out.clone()
        assert ctx.check() == 0
        compare(t)


def test_calls_are_sound_again_after_lengths_changed_under_way(cuda_device):
    """Another stream sets lengths while calls of several rounds are under way; after a check the next call is as ever."""
    lens, new = [40000, 20000], [4096, 2500]             # four rounds
    t = fill(Batch(cuda_device, lens, new, 8, 4, False, pad_rows=0))
    ctx = t.ctx()
    call(t, ctx)
    want = t.out.clone(), t.lse.clone()
    other = torch.cuda.Stream()
    for i, wrong in enumerate(([5000, 3000], [40000, 40000], [4096, 2500], [20000, 40000]) * 3):
        n = torch.tensor(wrong, dtype=torch.int32, device=cuda_device)
        torch.cuda.synchronize()
        for _ in range(3):
            ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse, row_start=t.row_start)
        with torch.cuda.stream(other):
            torch.cuda._sleep(200000 + 150000 * i)
            t.lens_t.copy_(n)
        torch.cuda.synchronize()
        try:
            ctx.check()
        except P.PrhsError as e:
            assert e.status == 7
        t.lens_t.copy_(torch.tensor(lens, dtype=torch.int32))
        call(t, ctx)
        for a, b in zip(want, (t.out, t.lse)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_lanes_of_a_warp_with_notes_of_their_own(cuda_device):
    """Rows of a warp that differ in how many noted positions they see (loops of their own length between loads of tensor memory), in a group that
    leaves rows of the warp unused."""
    for group, paged in ((7, False), (3, True), (1, False)):
        t = fill(Batch(cuda_device, [400, 65], [390, 65], 1, group, paged))
        for b in range(2):
            t.full_v[b][0, 1::2, 5] = math.nan
            t.full_v[b][0, 64, 99] = math.inf
        store(t)
        call(t)
        out, lse, tol, ltol = reference(t)
        for b, (r0, n, T) in enumerate(((0, 390, 400), (390, 65, 65))):
            u = torch.arange(T - n + 1, T + 1, device=t.dev)
            got, want, near = (x[r0:r0 + n].double().clone() for x in (t.out, out, tol))
            assert torch.isnan(got[u > 1][..., 5]).all() and torch.isfinite(got[u == 1]).all()
            assert (got[u > 64][..., 99] == math.inf).all()
            got[u > 1, :, 5] = want[u > 1, :, 5]
            got[u > 64, :, 99] = want[u > 64, :, 99]
            assert ((got - want).abs() <= near).all()
            assert ((t.lse[r0:r0 + n].double() - lse[r0:r0 + n]).abs() <= ltol[r0:r0 + n]).all()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("length,new,group", [(20000, 2, 4), (700, 3, 7), (300, 300, 2), (9000, 200, 4), (40, 40, 1)])
def test_values_that_are_not_finite_where_all_logits_are_minus_infinity(cuda_device, length, new, group, paged):
    """Zero times an infinity or a NaN is NaN, in whichever piece of the work it lies: the coordinate is not finite for all that see it, the others
    are as without it.  A token that sees such logits alone has lse = -inf and zeros elsewhere."""
    gone = length // 2
    t = fill(Batch(cuda_device, [length], [new], 2, group, paged, pad_rows=0), k_amp=0.5)
    t.qc[:, :, 0] = 1.0
    t.full_k[0][:, :gone, 0] = -math.inf
    odd = [(0, 0, 3, math.inf), (0, gone - 1, 70, math.nan), (1, gone // 2, 127, -math.inf), (1, gone - 1, 9, math.inf)]
    for h, pos, d, x in odd:
        t.full_v[0][h, pos, d] = x
    store(t)
    call(t)
    out, lse, tol, ltol = reference(t)
    got, gl = t.out.double(), t.lse.double()
    u = torch.arange(length - new + 1, length + 1, device=t.dev)
    where = torch.zeros_like(got, dtype=torch.bool)
    for h, pos, d, x in odd:
        where[u > pos, h * group:(h + 1) * group, d] = True
    assert torch.isfinite(got[~where]).all() and not torch.isfinite(got[where]).any()
    tol = torch.nan_to_num(tol, nan=math.inf)
    empty = u <= gone
    assert not got[empty][~where[empty]].any() and (gl[empty] == -math.inf).all()
    assert ((got - out).abs()[~empty] <= tol[~empty])[~where[~empty]].all()
    assert ((gl - lse).abs()[~empty] <= ltol[~empty]).all()


def test_a_context_without_the_workspace(cuda_device):
    """PRHS_CFG_NO_CHUNK_ATTN: attention of many tokens is refused, its memory is not taken, and everything else runs."""
    t = fill(Batch(cuda_device, [300, 40], [1, 1], 2, 4, False, pad_rows=0))
    make = lambda flags: P.Context(num_layers=1, max_batch=2, num_q_heads=8, num_kv_heads=2, max_context=304, max_k=1, max_window=1, max_sinks=4, flags=flags)  # noqa: E731
    make(0).close()
    taken = []
    for flags in (0, P.PRHS_CFG_NO_CHUNK_ATTN):
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info()[0]
        ctx = make(flags)
        taken.append(free - torch.cuda.mem_get_info()[0])
        if not flags:
            ctx.close()
    assert taken[0] - taken[1] >= 32 << 20
    with pytest.raises(P.PrhsError) as e:
        ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse)
    assert e.value.status == 2
    ctx.dense_decode_attn(t.qc, t.view(), 2, t.out, t.lse)
    assert ctx.check() == 0
    compare(t)


def test_a_context_in_tight_memory(cuda_device):
    """A context that finds no memory for the chunk attention's workspace, or for less of it than it would take, serves the rest."""
    t = fill(Batch(cuda_device, [300, 40], [1, 1], 1, 4, False, pad_rows=0))
    make = lambda: P.Context(num_layers=1, max_batch=2, num_q_heads=4, num_kv_heads=1, max_context=1 << 19, max_k=1, max_window=1, max_sinks=4)  # noqa: E731
    ctx = make()                                    # 158 MB of workspace, and every kernel loaded
    for f in (ctx.dense_decode_attn, ctx.chunk_attn):
        f(t.qc, t.view(), 2, t.out, t.lse)
    assert ctx.check() == 0
    ctx.close()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held, MB = [], 1 << 20
    try:
        for left in (130 * MB, 36 * MB):            # room for two rounds or one; for none
            while True:
                free = torch.cuda.mem_get_info()[0] - left
                if free < 2 * MB:
                    break
                try:
                    held.append(torch.empty(min(free, 4096 * MB) // (2 * MB) * (2 * MB), dtype=torch.uint8, device=cuda_device))
                except torch.cuda.OutOfMemoryError:
                    break
            ctx = make()
            t.out.fill_(math.nan)
            ctx.dense_decode_attn(t.qc, t.view(), 2, t.out, t.lse)
            assert ctx.check() == 0
            compare(t)
            t.out.fill_(math.nan)
            if left > 39 * MB:
                ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse)
                assert ctx.check() == 0
                compare(t)
            else:
                with pytest.raises(P.PrhsError) as e:
                    ctx.chunk_attn(t.qc, t.view(), 2, t.out, t.lse)
                assert e.value.status == 3 and ctx.check() == 0
            ctx.close()
    finally:
        del held
        torch.cuda.empty_cache()


def rows_of(t, b, rows, heads, sinks=0, window=0):
    """out, lse and their bounds (float64) for some new tokens of sequence b and some heads, as reference()."""
    T, n, out = t.lens[b], t.new[b], []
    u = torch.tensor([T - n + 1 + r for r in rows], device=t.dev)
    lo = torch.tensor([first_visible(int(x), window, 0.0) for x in u], device=t.dev)
    i = torch.arange(T, device=t.dev)
    see = (i < u[:, None]) & ((i < sinks) | (i >= lo[:, None]))
    for h in heads:
        k, v, q = t.full_k[b][h // t.G].double(), t.full_v[b][h // t.G].double(), t.qc[[t.starts[b] + r for r in rows], h].double()
        a = (q @ k.T * S).masked_fill(~see, -math.inf)
        z = torch.logsumexp(a, -1)
        p = torch.exp(a - z[:, None])
        y = p @ v
        e = (S * 131 * 2.0 ** -23 * (q.abs() @ k.abs().T)).masked_fill(~see, 0.0).amax(-1)
        out.append((y, z, 2.0 ** -8 * y.abs() + (2 * e + 2.0 ** -20 + T * 2.0 ** -22 + 2.0 ** -8)[:, None] * (p @ v.abs()) + 2.0 ** -134,
                    e + 2.0 ** -20 + T * 2.0 ** -23 + 2.0 ** -22 * z.abs()))
    return [torch.stack(x, 1) for x in zip(*out)]


@pytest.mark.parametrize("lens,new,kv_heads,group,sinks,window", [([40000, 3000], [2300, 1500], 8, 4, 0, 0), ([60000, 130], [4200, 130], 8, 4, 0, 0),
                                                                  ([24000, 9000, 24001], [2048, 0, 1999], 32, 1, 130, 17000)])
def test_several_rounds(cuda_device, lens, new, kv_heads, group, sinks, window):
    """From 56832 units of work (148 SMs, runs of 192) over more than 1024 tiles: three rounds, four, and two under a window with ungrouped heads.  Paged and
    contiguous give the same bits, as a second call does, and a sample is right."""
    got = []
    mask = P.make_chunk_mask(sinks=sinks, window=window) if window else None
    for paged in (False, True):
        t = fill(Batch(cuda_device, lens, new, kv_heads, group, paged), k_amp=0.7)
        ctx = P.Context(num_layers=1, max_batch=len(lens), num_q_heads=kv_heads * group, num_kv_heads=kv_heads, max_context=t.cap, max_k=1, max_window=1,
                        max_sinks=4, page_size=16 if paged else 0)
        for _ in range(2):
            t.out.fill_(math.nan)
            call(t, ctx, mask)
            got.append((t.out.clone(), t.lse.clone()))
    for out, lse in got[1:]:
        assert torch.equal(bits(out), bits(got[0][0])) and torch.equal(lse.view(torch.int32), got[0][1].view(torch.int32))
    live = t.starts[-1]
    assert torch.isnan(t.out[live:]).all() and torch.isfinite(t.out[:live]).all() and torch.isfinite(t.lse[:live]).all()
    heads = sorted({0, 1, t.Hq // 2, t.Hq - 1})
    for b, n in enumerate(new):
        if not n:
            continue
        rows = sorted({0, n - 1, n // 2} | set(range(5, n, max(1, n // 60))))
        out, lse, tol, ltol = rows_of(t, b, rows, heads, sinks, window)
        at = [t.starts[b] + r for r in rows]
        assert ((t.out[at][:, heads].double() - out).abs() <= tol).all()
        assert ((t.lse[at][:, heads].double() - lse).abs() <= ltol).all()


@pytest.mark.parametrize("lens,new,group", [([20000], [2], 4), ([3000, 300], [700, 300], 4), ([9000], [200], 1)])
def test_large_values_under_logits_that_jump(cuda_device, lens, new, group):
    """Values of 2^50, and logits that rise by 58 binary orders from one stretch of tiles to the next: weights up to 2^58 against the reference that
    stands, nothing overflows."""
    t = fill(Batch(cuda_device, lens, new, 1, group, False, pad_rows=0))
    t.qc.fill_(4.0)
    high = 58 * math.log(2.0) / (4 * 128 * S)
    for b, n in enumerate(lens):
        stretch = torch.arange(n, device=cuda_device) // 128 % 5
        t.full_k[b][:] = torch.where(stretch == 2, high, 0.0).to(BF)[None, :, None]
        t.full_v[b] = (t.full_v[b].sign() * 2.0 ** 50).to(BF)
        t.full_v[b][..., :64] = 2.0 ** 50
    store(t)
    call(t)
    compare(t)
