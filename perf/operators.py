"""Measured cases of the decode operators over an 8-bit cache and over selected blocks.

Three groups, all of one decode layer with rows of 128 values, caches contiguous or in pages of 16 positions:

  append8        rows of keys and values come in as bf16 and go into an 8-bit cache (e4m3 or e5m2) with one
                 power-of-two scale per block of 16 positions and KV head; the open block stays in bf16
  attend8        decode attention over every position of that cache
  attend8_rows   the same restricted to an explicit list of positions per query head
  bounds         per block of 16 keys the coordinate-wise minimum and maximum, in 8 bits with one scale
  block_step     one token: the last block's bounds, a score of every block against the query, the blocks
                 that are attended over (first, best scoring, last), and the attention over them

`run` is the plain form, or with `own` the library's calls.  Sequence lengths and index lists' sizes follow
from the case alone, values from the seed.
"""
import math
import random

import torch

own = False

D = 128                 # values per row
BLOCK = 16              # positions per block and per page
FORMATS = {"e4m3": (torch.float8_e4m3fn, 9), "e5m2": (torch.float8_e5m2, 16)}   # largest finite value: 0.875 * 2^n
INT8_TOP = (127 / 128, 7)                                                         # 127 = (127 / 128) * 2^7
SCALE = D ** -0.5


# ------------------------------------------------------------------------------------------ cases
def listed():
    base = dict(kv_heads=8, group=4, ragged=0, paged=False, format="e4m3")
    c = lambda name, kind, **kw: {"name": name, "kind": kind, **base, **kw}  # noqa: E731
    return [
        # a prompt of 32K tokens for four sequences goes into the cache after prefill
        c("append8_prompt", "append8", batch=4, context=32768, new=32768),
        # one token of each sequence of a serving batch, ragged, some of them close a block
        c("append8_token", "append8", batch=64, context=4099, new=1, ragged=3, paged=True),
        # a single user with a short grouped-query context: latency
        c("attend8_single", "attend8", batch=1, context=2047),
        # the 7B layer without grouped queries at 32K: the largest stream
        c("attend8_mha_32k", "attend8", batch=8, context=32768, kv_heads=32, group=1),
        # a ragged paged serving batch, the wider exponent format
        c("attend8_paged_ragged", "attend8", batch=32, context=16384, ragged=5, paged=True, format="e5m2"),
        # the index sets of a sharing step of the 7B layer (sinks, dilated middle, window)
        c("attend8_rows_mha_32k", "attend8_rows", batch=8, context=32768, kv_heads=32, group=1, rows=1838),
        # a small set for one user over pages
        c("attend8_rows_single", "attend8_rows", batch=1, context=8190, rows=333, paged=True),
        # the bounds of a prompt's blocks
        c("bounds_prompt", "bounds", batch=4, context=32768, new=32768),
        # the bounds after a few more tokens of every sequence of a paged batch
        c("bounds_chunk", "bounds", batch=16, context=9001, new=40, ragged=7, paged=True),
        # one user, 8K: latency of a whole step
        c("block_step_single", "block_step", batch=1, context=8191, top=16, first=1, last=2, shared=False),
        # the 7B layer at 32K with a budget of 1024 positions per head
        c("block_step_mha_32k", "block_step", batch=8, context=32768, kv_heads=32, group=1, top=64, first=1, last=8,
          shared=False),
        # long ragged contexts in pages, one set per KV head
        c("block_step_shared_paged", "block_step", batch=16, context=65536, ragged=9, paged=True, top=128, first=1,
          last=8, shared=True),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["append8", "attend8", "attend8", "attend8_rows", "bounds", "block_step", "block_step"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    c = dict(kind=kind, kv_heads=kv_heads, group=rng.choice([1, 2, 3, 4, 4, 7, 8, 16]) if kv_heads < 32 else 1,
             batch=_log_uniform(rng, 1, 64), ragged=rng.choice([0, 1]) * rng.randint(1, 1000),
             paged=rng.random() < 0.5, format=rng.choice(["e4m3", "e5m2"]))
    most = 131072 * 16 if kind in ("append8", "bounds") else 131072 * 64      # rows over all KV heads
    c["context"] = _log_uniform(rng, 1, max(1, min(131072, most // (c["batch"] * kv_heads))))
    if kind in ("append8", "bounds"):
        c["new"] = rng.choice([1, c["context"], _log_uniform(rng, 1, c["context"])])
    if kind == "attend8_rows":
        most = min(c["context"], 4096, max(1, 800000 // (c["batch"] * kv_heads * c["group"])))
        c["rows"] = _log_uniform(rng, 1, most)
    if kind == "block_step":
        c["shared"] = rng.random() < 0.5
        most = max(1, min(256, 60000 // (c["batch"] * kv_heads * (1 if c["shared"] else c["group"]))))
        c["top"], c["first"], c["last"] = _log_uniform(rng, 1, most), rng.choice([0, 1, 2]), rng.choice([1, 2, 8])
    return c


def _lengths(case):
    """(positions after the call, of those new) per sequence, from the case alone."""
    B, n = case["batch"], case["context"]
    new = case.get("new", 1)
    if not case["ragged"]:
        return [n] * B, [min(new, n)] * B
    r = random.Random(case["ragged"])
    lens = [r.randint(max(1, n // 8), n) for _ in range(B)]
    lens[r.randrange(B)] = n
    return lens, [min(t, new if new == 1 else r.randint(0, new) if i else new) for i, t in enumerate(lens)]


def _units(case):
    return case["kv_heads"] * (1 if case.get("shared") else case["group"])


def _selected(case, t):
    """How many blocks a head attends over at length t."""
    nb = -(-t // BLOCK)
    lo = min(case["first"], nb)
    hi = max(lo, nb - case["last"])
    return lo, hi, nb, lo + min(case["top"], hi - lo) + nb - hi


def work(case):
    lens, new = _lengths(case)
    H, G, kind = case["kv_heads"], case["group"], case["kind"]
    io = case["batch"] * H * G * (2 * 2 * D + 4)            # q in, out and lse
    if kind == "append8":
        return {"bytes": sum(new) * H * 2 * D * 3, "flops": sum(new) * H * 2 * D * 2}
    if kind == "attend8":
        blocks = sum(-(-t // BLOCK) for t in lens)
        return {"bytes": sum(lens) * H * 2 * D + blocks * H * 8 + io, "flops": 4 * D * G * H * sum(lens)}
    if kind == "attend8_rows":
        rows = sum(min(case["rows"], t) for t in lens) * H * G
        return {"bytes": rows * (2 * D + 4) + io, "flops": 4 * D * rows}
    if kind == "bounds":
        read = sum(t - (t - n) // BLOCK * BLOCK for t, n in zip(lens, new)) * H
        return {"bytes": read * 2 * D + read // BLOCK * (2 * D + 4), "flops": 2 * D * read}
    blocks = sum(-(-t // BLOCK) for t in lens) * H
    att = sum(min(_selected(case, t)[3] * BLOCK, t) for t in lens) * _units(case)
    return {"bytes": blocks * (2 * D + 4) + att * 4 * D + io,
            "flops": blocks * G * 4 * D + att * 4 * D * (G if case["shared"] else 1)}


# ------------------------------------------------------------------------------------------ inputs
def _exponent(amax, top):
    """The smallest e >= -126 with amax <= top[0] * 2^(top[1] + e)."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, (e - top[1] + (m > top[0]).to(e.dtype)).clamp_min(-126), -126)


def _pow2(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, fmt):
    """[..., 16, 128] fp32 -> 8-bit values and the blocks' scales [...]."""
    dtype, n = FORMATS[fmt]
    scale = _pow2(_exponent(x.abs().amax((-2, -1)), (0.875, n)))
    return (x / scale[..., None, None]).to(dtype), scale


def _bounds_of(x, valid):
    """[..., 16, 128] fp32 and [..., 16] -> int8 [..., 2, 128] (minimum, maximum) and scales [...]."""
    lo = x.masked_fill(~valid[..., None], math.inf).amin(-2)
    hi = x.masked_fill(~valid[..., None], -math.inf).amax(-2)
    both = torch.stack([lo, hi], -2)
    both = torch.where(both.isfinite(), both, 0.0)          # a block without positions
    scale = _pow2(_exponent(both.abs().amax((-2, -1)), INT8_TOP))
    return (both / scale[..., None, None]).round().to(torch.int8), scale


def _keys(case, g, dev):
    """bf16 [B][H][cap][128]: keys drift along the sequence (neighbours are alike), a few channels are large."""
    B, H = case["batch"], case["kv_heads"]
    cap = -(-case["context"] // BLOCK) * BLOCK
    out = torch.empty(B, H, cap, D, dtype=torch.bfloat16, device=dev)
    channel = torch.where(torch.rand(H, 1, D, generator=g, device=dev) < 0.05, 3.0, 1.0)
    for b in range(B):
        centre = torch.randn(H, cap // BLOCK, 1, D, generator=g, device=dev)
        x = torch.randn(H, cap, D, generator=g, device=dev) * 0.8
        x = (x.view(H, cap // BLOCK, BLOCK, D) + 0.6 * centre).view(H, cap, D)
        out[b] = (x * channel).to(torch.bfloat16)
    return out


def _values(case, g, dev):
    B, H = case["batch"], case["kv_heads"]
    cap = -(-case["context"] // BLOCK) * BLOCK
    out = torch.empty(B, H, cap, D, dtype=torch.bfloat16, device=dev)
    for b in range(B):
        out[b] = torch.randn(H, cap, D, generator=g, device=dev).to(torch.bfloat16)
    return out


def _pages(case, lens, g, dev):
    need = [-(-t // BLOCK) for t in lens]
    order = torch.randperm(sum(need), generator=g, device=dev).to(torch.int32)
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need)


def _to_pages(x, table, lens, pool):
    """[B][H][blocks][...] -> [pool][H][...]."""
    out = torch.zeros(pool, x.shape[1], *x.shape[3:], dtype=x.dtype, device=x.device)
    raw_out = out.view(torch.uint8) if out.dtype.itemsize == 1 else out
    raw = x.view(torch.uint8) if x.dtype.itemsize == 1 else x
    for b, t in enumerate(lens):
        n = -(-t // BLOCK)
        raw_out[table[b, :n].long()] = raw[b, :, :n].transpose(0, 1)
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    lens, new = _lengths(case)
    B, H, G, kind = case["batch"], case["kv_heads"], case["group"], case["kind"]
    k, v = _keys(case, g, dev), _values(case, g, dev)
    cap = k.shape[2]
    s = {"case": case, "max_len": max(lens), "max_new": max(new),
         "lens": torch.tensor(lens, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev)}
    s["table"], pool = _pages(case, lens, g, dev) if case["paged"] else (None, 0)
    if kind in ("attend8", "attend8_rows", "block_step"):
        s["q"] = torch.randn(B, H * G, D, generator=g, device=dev).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(B, H * G, device=dev)
    start = s["lens"] - s["new"]
    if kind == "append8":
        # the new rows of every sequence, and the cache and open block as they were before them
        at = (start[:, None] + torch.arange(s["max_new"], device=dev)).clamp(0, cap - 1).long()
        at = at[:, None, :, None].expand(B, H, -1, D)
        s["new_k"], s["new_v"] = k.gather(2, at), v.gather(2, at)
        held = start
    else:
        held = s["lens"]
    if kind in ("append8", "attend8", "attend8_rows"):
        first = (held // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device=dev)
        at = first.clamp(0, cap - 1).long()[:, None, :, None].expand(B, H, -1, D)
        s["k_tail"], s["v_tail"] = k.gather(2, at), v.gather(2, at)
        again = kind == "append8" and s["max_new"] > 1 and any((t - n) % BLOCK for t, n in zip(lens, new))
        s["tails"] = (s["k_tail"].clone(), s["v_tail"].clone()) if again else None
        for n, x in (("k", k), ("v", v)):
            codes = torch.empty(B, H, cap, D, dtype=FORMATS[case["format"]][0], device=dev)
            scale = torch.empty(B, H, cap // BLOCK, device=dev)
            for b in range(B):
                y, scale[b] = _quantise(x[b].float().view(H, -1, BLOCK, D), case["format"])
                codes[b] = y.view(H, cap, D)
            if kind == "append8":      # what was there before is older content, not the rows to come
                codes, scale = codes.view(torch.uint8).roll(1, 1).view(codes.dtype), scale.roll(1, 1)
            if case["paged"]:
                codes = _to_pages(codes.view(B, H, -1, BLOCK, D), s["table"], lens, pool)
                scale = _to_pages(scale, s["table"], lens, pool)
            s[n + "8"], s[n + "_scale"] = codes, scale
    if kind == "attend8_rows":
        # positions in ascending order, no duplicates: the shape of the library's index sets
        n = min(case["rows"], max(lens))
        s["count"] = torch.tensor([min(n, t) for t in lens], dtype=torch.int32, device=dev)[:, None].expand(B, H * G).contiguous()
        r = torch.rand(B, H * G, max(lens), generator=g, device=dev)
        r.masked_fill_(torch.arange(max(lens), device=dev) >= s["lens"][:, None, None], 2.0)
        idx = r.topk(n, -1, largest=False).indices
        idx.masked_fill_(torch.arange(n, device=dev) >= s["count"][..., None], 1 << 30)
        s["idx"] = idx.sort(-1).values.to(torch.int32)
    if kind in ("bounds", "block_step"):
        nb = cap // BLOCK
        seen = s["lens"] - 1 if kind == "block_step" else start
        codes = torch.zeros(B, H, nb, 2, D, dtype=torch.int8, device=dev)
        scale = torch.zeros(B, H, nb, device=dev)
        for b in range(B):
            ok = torch.arange(cap, device=dev).view(nb, BLOCK) < seen[b]
            y, z = _bounds_of(k[b].float().view(H, nb, BLOCK, D), ok.expand(H, nb, BLOCK))
            have = ok[:, 0]
            codes[b], scale[b] = y * have[:, None, None], z * have
        s["start"] = start
        if case["paged"]:
            codes, scale = _to_pages(codes, s["table"], lens, pool), _to_pages(scale, s["table"], lens, pool)
            k = _to_pages(k.view(B, H, nb, BLOCK, D), s["table"], lens, pool)
            v = _to_pages(v.view(B, H, nb, BLOCK, D), s["table"], lens, pool) if kind == "block_step" else k
        s["bounds"], s["bounds_scale"], s["k"] = codes, scale, k
        if kind == "block_step":
            s["v"] = v
            room = case["first"] + case["top"] + case["last"]
            s["blocks"] = torch.empty(B, _units(case), room, dtype=torch.int32, device=dev)
            s["count"] = torch.empty(B, _units(case), dtype=torch.int32, device=dev)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _at(x, s, blocks):
    """Blocks [B][H][n] (numbers within the sequence) of x, contiguous [B][H][blocks][...] or pages [pool][H][...]."""
    B, H, n = blocks.shape
    b = torch.arange(B, device=blocks.device)[:, None, None]
    h = torch.arange(H, device=blocks.device)[None, :, None]
    raw = x.view(torch.uint8) if x.dtype.itemsize == 1 else x
    got = raw[s["table"][b, blocks].long(), h] if s["table"] is not None else raw[b, h, blocks]
    return got.view(x.dtype) if x.dtype.itemsize == 1 else got


def _put(x, s, blocks, keep, values):
    """Writes values [B][H][n][...] into those blocks of x where keep [B][n]."""
    b, i = keep.nonzero(as_tuple=True)
    raw = x.view(torch.uint8) if x.dtype.itemsize == 1 else x
    val = values.view(torch.uint8) if values.dtype.itemsize == 1 else values
    where = blocks[b, i].long()
    if s["table"] is not None:
        raw[s["table"][b, where].long()] = val[b, :, i]
    else:
        raw[b, :, where] = val[b, :, i]


def _by_block(x, s):
    """[B][H][cap][...] seen as [B][H][blocks][16][...]; pages are blocks already."""
    return x if s["table"] is not None else x.view(x.shape[0], x.shape[1], -1, BLOCK, *x.shape[3:])


def _attend(q, k, v, valid):
    """q [B][U][g][128], k and v [B][U][n][128], valid [B][1 or U][n] -> out [B][U][g][128], lse [B][U][g], fp32."""
    k, v = torch.where(valid[..., None], k, 0.0), torch.where(valid[..., None], v, 0.0)
    a = (q @ k.transpose(-1, -2) * SCALE).masked_fill(~valid[:, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(top.isfinite(), top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    return out, (torch.where(top.isfinite(), top, 0.0) + total.log()).squeeze(-1)


def _plain_append(s):
    case, t, n = s["case"], s["lens"], s["new"]
    B, H = case["batch"], case["kv_heads"]
    dev = t.device
    start = t - n
    fb = start // BLOCK
    nblk = -(-(s["max_new"] + BLOCK - 1) // BLOCK) + (1 if s["max_new"] > 1 else 0)
    pos = fb[:, None] * BLOCK + torch.arange(nblk * BLOCK, device=dev)          # [B][rows]
    from_new = (pos - start[:, None]).clamp(0, s["max_new"] - 1).long()[:, None, :, None].expand(B, H, -1, D)
    from_tail = (pos % BLOCK).long()[:, None, :, None].expand(B, H, -1, D)
    old, live = (pos < start[:, None])[:, None, :, None], (pos < t[:, None])[:, None, :, None]
    blocks = fb[:, None] + torch.arange(nblk, device=dev)
    whole = ((blocks + 1) * BLOCK <= t[:, None]) & (n[:, None] > 0)
    opens = (blocks == (t // BLOCK)[:, None]) & (n[:, None] > 0)
    for new, tail, codes, scale in ((s["new_k"], s["k_tail"], s["k8"], s["k_scale"]), (s["new_v"], s["v_tail"], s["v8"], s["v_scale"])):
        x = torch.where(old, tail.gather(2, from_tail), torch.where(live, new.gather(2, from_new), tail.gather(2, from_tail)))
        x = x.view(B, H, nblk, BLOCK, D)
        y, z = _quantise(x.float(), case["format"])
        _put(_by_block(codes, s), s, blocks, whole, y)
        _put(scale, s, blocks, whole, z)
        b, i = opens.nonzero(as_tuple=True)
        tail[b] = x[b, :, i]
    return [s["k8"], s["k_scale"], s["v8"], s["v_scale"], s["k_tail"], s["v_tail"]]


def _plain_attend8(s):
    case, t = s["case"], s["lens"]
    B, H, G = case["batch"], case["kv_heads"], case["group"]
    nb = -(-s["max_len"] // BLOCK)
    blocks = torch.arange(nb, device=t.device).expand(B, H, nb)
    pos = torch.arange(nb * BLOCK, device=t.device)
    tail_at = (pos >= (t // BLOCK * BLOCK)[:, None])[:, None, :, None]
    kv = []
    for codes, scale, tail in ((s["k8"], s["k_scale"], s["k_tail"]), (s["v8"], s["v_scale"], s["v_tail"])):
        x = _at(_by_block(codes, s), s, blocks).float() * _at(scale, s, blocks)[..., None, None]
        x = x.view(B, H, nb * BLOCK, D)
        kv.append(torch.where(tail_at, tail.float()[:, :, pos % BLOCK], x))
    out, lse = _attend(s["q"].float().view(B, H, G, D), kv[0], kv[1], (pos < t[:, None])[:, None])
    return [out.view(B, H * G, D).to(torch.bfloat16), lse.view(B, H * G)]


def _plain_attend8_rows(s):
    case, t, idx = s["case"], s["lens"].long(), s["idx"].long()
    B, H, G = case["batch"], case["kv_heads"], case["group"]
    U, n = H * G, idx.shape[-1]
    valid = torch.arange(n, device=idx.device) < s["count"][..., None]
    idx = torch.where(valid, idx, 0)
    b = torch.arange(B, device=idx.device)[:, None, None]
    h = (torch.arange(U, device=idx.device) // G)[None, :, None]
    blk, row = idx // BLOCK, idx % BLOCK
    in_tail = (idx >= (t // BLOCK * BLOCK)[:, None, None])[..., None]
    kv = []
    for codes, scale, tail in ((s["k8"], s["k_scale"], s["k_tail"]), (s["v8"], s["v_scale"], s["v_tail"])):
        raw = _by_block(codes, s).view(torch.uint8)
        if s["table"] is not None:
            page = s["table"][b, blk].long()
            x, z = raw[page, h, row], scale[page, h]
        else:
            x, z = raw[b, h, blk, row], scale[b, h, blk]
        kv.append(torch.where(in_tail, tail[b, h, row].float(), x.view(codes.dtype).float() * z[..., None]))
    out, lse = _attend(s["q"].float().view(B, U, 1, D), kv[0], kv[1], valid)
    return [out.view(B, U, D).to(torch.bfloat16), lse.view(B, U)]


def _update_bounds(s, first, most):
    """Bounds of the blocks that hold positions [first, t); `most` = the largest t - first."""
    case, t = s["case"], s["lens"]
    B, H = case["batch"], case["kv_heads"]
    fb = first.clamp_min(0) // BLOCK
    nblk = -(-(most + BLOCK - 1) // BLOCK) + (1 if most > 1 else 0)
    blocks = fb[:, None] + torch.arange(nblk, device=t.device)
    live = (blocks * BLOCK < t[:, None]) & (first < t)[:, None]
    room = s["table"].shape[1] if s["table"] is not None else s["bounds"].shape[2]
    x = _at(_by_block(s["k"], s), s, blocks.clamp_max(room - 1).long()[:, None].expand(B, H, nblk)).float()
    ok = (blocks[..., None] * BLOCK + torch.arange(BLOCK, device=t.device) < t[:, None, None])[:, None].expand(B, H, nblk, BLOCK)
    y, z = _bounds_of(x, ok)
    _put(s["bounds"], s, blocks, live, y)
    _put(s["bounds_scale"], s, blocks, live, z)


def _plain_block_step(s):
    case, t = s["case"], s["lens"]
    B, H, G = case["batch"], case["kv_heads"], case["group"]
    _update_bounds(s, t - 1, 1)
    nb = -(-s["max_len"] // BLOCK)
    every = torch.arange(nb, device=t.device)
    q = s["q"].float().view(B, H, G, D)
    q_scale = _pow2(_exponent(q.abs().amax(-1), INT8_TOP))
    q8 = (q / q_scale[..., None]).round()
    bounds = _at(s["bounds"], s, every.expand(B, H, nb)).float()
    scale = _at(s["bounds_scale"], s, every.expand(B, H, nb))
    # whole numbers below 2^24 and powers of two: exact in 32 bits in any order
    dot = q8.clamp_min(0) @ bounds[..., 1, :].transpose(-1, -2) + q8.clamp_max(0) @ bounds[..., 0, :].transpose(-1, -2)
    score = dot * scale[:, :, None] * q_scale[..., None]                        # [B][H][G][blocks]
    score = score.amax(2) if case["shared"] else score.reshape(B, H * G, nb)
    U = score.shape[1]
    n = -(-t // BLOCK)
    lo = n.clamp_max(case["first"])
    hi = torch.maximum(lo, n - case["last"])
    middle = ((every >= lo[:, None]) & (every < hi[:, None]))[:, None]
    order = score.masked_fill(~middle, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, every.expand(B, U, nb).contiguous())
    taken = torch.where(middle, rank < case["top"], (every < n[:, None])[:, None])
    room = s["blocks"].shape[-1]
    count = taken.sum(-1)
    blocks = torch.where(taken, every, nb).sort(-1).values[..., :room]
    if nb < room:
        blocks = torch.nn.functional.pad(blocks, (0, room - nb), value=nb)
    valid = blocks < nb
    at = torch.where(valid, blocks, 0)
    per = 1 if case["shared"] else G
    b = torch.arange(B, device=t.device)[:, None, None]
    h = (torch.arange(U, device=t.device) // per)[None, :, None]
    kv = []
    for x in (s["k"], s["v"]):
        x = _by_block(x, s)
        x = x[s["table"][b, at].long(), h] if s["table"] is not None else x[b, h, at]
        kv.append(x.float().view(B, U, room * BLOCK, D))
    pos = at[..., None] * BLOCK + torch.arange(BLOCK, device=t.device)
    ok = (valid[..., None] & (pos < t[:, None, None, None])).view(B, U, room * BLOCK)
    out, lse = _attend(q.view(B, U, G if case["shared"] else 1, D), kv[0], kv[1], ok)
    return [out.view(B, H * G, D).to(torch.bfloat16), lse.view(B, H * G), torch.where(valid, blocks, -1).to(torch.int32),
            count.to(torch.int32), s["bounds"], s["bounds_scale"]]


# ------------------------------------------------------------------------------------------ the library
_contexts = {}


def _context(s):
    """A program keeps one context for its model: heads, page size and the largest batch and context."""
    from paper_2602_08329_b200 import binding as P
    case = s["case"]
    key = (case["batch"], case["kv_heads"], case["group"], s["max_len"], case["paged"])
    if key not in _contexts:
        while len(_contexts) >= 4:
            _contexts.pop(next(iter(_contexts))).close()
        _contexts[key] = P.Context(num_layers=1, max_batch=case["batch"], num_q_heads=case["kv_heads"] * case["group"],
                                   num_kv_heads=case["kv_heads"], max_context=s["max_len"], max_k=16, max_window=16,
                                   max_sinks=4, page_size=BLOCK if case["paged"] else 0)
    return _contexts[key]


def _own(s):
    from paper_2602_08329_b200 import binding as P
    case = s["case"]
    ctx, B, kind = _context(s), case["batch"], case["kind"]
    if kind in ("append8", "attend8", "attend8_rows"):
        kv = P.make_bytekv_view(s["k8"], s["v8"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"], s["lens"],
                             page_table=s["table"], max_seq_len=s["max_len"])
        if kind == "append8":
            ctx.bytekv_append(s["new_k"], s["new_v"], s["new"], kv, B)
            return [s["k8"], s["k_scale"], s["v8"], s["v_scale"], s["k_tail"], s["v_tail"]]
        if kind == "attend8":
            ctx.bytekv_decode_attn(s["q"], kv, B, s["out"], s["lse"])
        else:
            ctx.bytekv_sparse_decode_attn(s["q"], kv, s["idx"], s["count"], B, s["out"], s["lse"])
        return [s["out"], s["lse"]]
    kv = P.make_view(s["k"], s["v"] if kind == "block_step" else s["k"], s["lens"], page_table=s["table"],
                     max_seq_len=s["max_len"])
    bounds = P.make_block_bounds(s["bounds"], s["bounds_scale"])
    if kind == "bounds":
        ctx.block_bounds(kv, bounds, B, first=s["start"], max_new=s["max_new"])
        return [s["bounds"], s["bounds_scale"]]
    sched = P.make_block_schedule(top_blocks=case["top"], sink_blocks=case["first"], recent_blocks=case["last"],
                                  flags=P.PRHS_GROUP_SETS if case["shared"] else 0)
    ctx.block_decode_step(s["q"], kv, bounds, sched, B, s["out"], s["lse"], s["blocks"], s["count"])
    return [s["out"], s["lse"], s["blocks"], s["count"], s["bounds"], s["bounds_scale"]]


def run(state):
    if state.get("tails") is not None:      # the open blocks as they were before these rows came in
        state["k_tail"].copy_(state["tails"][0])
        state["v_tail"].copy_(state["tails"][1])
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "append8":
        return _plain_append(state)
    if kind == "attend8":
        return _plain_attend8(state)
    if kind == "attend8_rows":
        return _plain_attend8_rows(state)
    if kind == "bounds":
        _update_bounds(state, state["start"], state["max_new"])
        return [state["bounds"], state["bounds_scale"]]
    return _plain_block_step(state)


# ------------------------------------------------------------------------------------------ 64 bits
def _round8(v, fmt):
    """Nearest representable value (ties to even) of |v| within the format's range, in 64 bits."""
    bits, lowest = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(v).exponent.double().sub(1).clamp_min(lowest)
    step = _two_to(e - bits)
    return torch.round(v / step) * step


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _scale64(amax, top):
    e = torch.ceil(torch.log2(amax / top)).clamp_min(-126.0)
    e = e + (amax > top * _two_to(e)).double()              # log2 may be off by a rounding at a power of two
    e = torch.where((e > -126) & (amax <= top * _two_to(e - 1)), e - 1, e)
    return _two_to(e)


def _soft64(q, k, v):
    a = (k @ q) * SCALE
    m = a.max()
    p = torch.exp(a - m)
    return (p @ v) / p.sum(), m + torch.log(p.sum())


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    B, H, G, kind = case["batch"], case["kv_heads"], case["group"], case["kind"]

    def rows_of(x, b, n):
        """Blocks 0..n-1 of sequence b, [H][n][...]."""
        return x[s["table"][b, :n].long()].transpose(0, 1) if case["paged"] else _by_block(x, s)[b, :, :n]

    if kind == "append8":
        top = 448.0 if case["format"] == "e4m3" else 57344.0
        res = []
        for n, tail in (("k", s["k_tail"]), ("v", s["v_tail"])):
            codes, scale = s[n + "8"].to(torch.float64), s[n + "_scale"].double()
            end = tail.double()
            for b in range(B):
                t0, t1 = lens[b] - new[b], lens[b]
                f = t0 // BLOCK
                rows = torch.cat([tail[b, :, :t0 - f * BLOCK].double(), s["new_" + n][b, :, :new[b]].double()], 1)
                whole = rows.shape[1] // BLOCK
                if whole and new[b]:
                    x = rows[:, :whole * BLOCK].reshape(H, whole, BLOCK, D)
                    z = _scale64(x.abs().amax((-2, -1)), top)
                    y = _round8(x / z[..., None, None], case["format"])
                    if case["paged"]:
                        ids = s["table"][b, f:f + whole].long()
                        codes[ids], scale[ids] = y.transpose(0, 1), z.transpose(0, 1)
                    else:
                        codes[b, :, f * BLOCK:(f + whole) * BLOCK] = y.reshape(H, whole * BLOCK, D)
                        scale[b, :, f:f + whole] = z
                left = rows.shape[1] - whole * BLOCK
                if left and new[b]:
                    end[b, :, :left] = rows[:, whole * BLOCK:]
            res.append((codes, scale, end))
        return [res[0][0], res[0][1], res[1][0], res[1][1], res[0][2], res[1][2]]
    if kind == "attend8":
        out = torch.zeros(B, H * G, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(B, H * G, dtype=torch.float64, device="cuda")
        for b, t in enumerate(lens):
            w = t // BLOCK
            kv = []
            for n in "kv":
                codes = s[n + "8"].view(torch.uint8)
                x = rows_of(codes, b, w).contiguous().view(s[n + "8"].dtype).double()
                z = (s[n + "_scale"][s["table"][b, :w].long()].transpose(0, 1) if case["paged"] else s[n + "_scale"][b, :, :w]).double()
                kv.append(torch.cat([(x * z[..., None, None]).reshape(H, w * BLOCK, D), s[n + "_tail"][b, :, :t - w * BLOCK].double()], 1))
            q = s["q"][b].double().view(H, G, D)
            a = torch.einsum("hgd,hnd->hgn", q, kv[0]) * SCALE
            lse[b] = torch.logsumexp(a, -1).view(-1)
            out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(a, -1), kv[1]).reshape(H * G, D)
        return [out, lse]
    if kind == "attend8_rows":
        if B * H * G > 1500:
            return None
        out = torch.zeros(B, H * G, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(B, H * G, dtype=torch.float64, device="cuda")
        for b, t in enumerate(lens):
            w = t // BLOCK * BLOCK
            for u in range(H * G):
                i = s["idx"][b, u, :min(case["rows"], t)].long()
                h = u // G
                kv = []
                for n in "kv":
                    codes, z = s[n + "8"].view(torch.uint8), s[n + "_scale"]
                    if case["paged"]:
                        ids = s["table"][b, i // BLOCK].long()
                        x, z = codes[ids, h, i % BLOCK], z[ids, h]
                    else:
                        x, z = codes[b, h, i], z[b, h, i // BLOCK]
                    x = x.view(s[n + "8"].dtype).double() * z.double()[:, None]
                    kv.append(torch.where((i >= w)[:, None], s[n + "_tail"][b, h, i % BLOCK].double(), x))
                out[b, u], lse[b, u] = _soft64(s["q"][b, u].double(), kv[0], kv[1])
        return [out, lse]

    def bounds64(x):
        """[H][n][16 or fewer][128] in 64 bits."""
        both = torch.stack([x.amin(-2), x.amax(-2)], -2)
        z = _scale64(both.abs().amax((-2, -1)), 127.0)
        return torch.round(both / z[..., None, None]), z

    codes, scale = s["bounds"].clone(), s["bounds_scale"].double()
    for b, t in enumerate(lens):
        f = (t - 1 if kind == "block_step" else t - new[b]) // BLOCK
        if kind == "bounds" and not new[b]:
            continue
        n = -(-t // BLOCK)
        x = rows_of(s["k"], b, n)[:, f:].double()
        parts = ([(x[:, :-1], range(f, n - 1))] if n - 1 > f else []) + [(x[:, -1:, :t - (n - 1) * BLOCK], range(n - 1, n))]
        for part, where in parts:
            y, z = bounds64(part)
            if case["paged"]:
                ids = s["table"][b, where.start:where.stop].long()
                codes[ids], scale[ids] = y.transpose(0, 1).to(torch.int8), z.transpose(0, 1)
            else:
                codes[b, :, where.start:where.stop], scale[b, :, where.start:where.stop] = y.to(torch.int8), z
    if kind == "bounds":
        return [codes, scale]
    if B * _units(case) > 1500:
        return None
    out = torch.zeros(B, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, H * G, dtype=torch.float64, device="cuda")
    blocks, count = torch.full_like(s["blocks"], -1), torch.zeros_like(s["count"])
    per = G if case["shared"] else 1
    for b, t in enumerate(lens):
        lo, hi, n, _ = _selected(case, t)
        q = s["q"][b].double()
        qz = _scale64(q.abs().amax(-1).clamp_min(2.0 ** -140), 127.0)
        q8 = torch.round(q / qz[:, None])
        ids = s["table"][b, :n].long() if case["paged"] else None
        cb = (codes[ids].transpose(0, 1) if case["paged"] else codes[b, :, :n]).double()
        sb = scale[ids].transpose(0, 1) if case["paged"] else scale[b, :, :n]
        kk, vv = rows_of(s["k"], b, n), rows_of(s["v"], b, n)
        for u in range(_units(case)):
            h = u * per // G
            sc = torch.stack([torch.maximum(q8[u * per + j] * cb[h, :, 0], q8[u * per + j] * cb[h, :, 1]).sum(-1) * sb[h] * qz[u * per + j]
                              for j in range(per)]).amax(0)
            best = sc[lo:hi].sort(dim=0, descending=True, stable=True).indices[:case["top"]].sort().values + lo
            dev = best.device
            pick = torch.cat([torch.arange(lo, device=dev), best, torch.arange(hi, n, device=dev)])
            blocks[b, u, :len(pick)], count[b, u] = pick.to(torch.int32), len(pick)
            at = (pick[:, None] * BLOCK + torch.arange(BLOCK, device=dev)).view(-1)
            at = at[at < t]
            k64, v64 = (x[h].reshape(-1, D)[at].double() for x in (kk, vv))
            for j in range(per):
                out[b, u * per + j], lse[b, u * per + j] = _soft64(q[u * per + j], k64, v64)
    return [out, lse, blocks, count, codes, scale]
