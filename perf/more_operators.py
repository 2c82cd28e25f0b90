"""Measured cases of the operators around the decode step: new tokens into the cache, and attention of many new tokens.

All of one layer with rows of 128 values, caches contiguous or in pages of 16 positions, new tokens of several sequences
packed one after another (sequence b has rows row_start[b] to row_start[b + 1]; rows behind the last one are padding):

  qkv     queries, keys and values of new tokens, as the projection leaves them: queries and keys are normalised per head
          and rotated by their positions (one axis, or time, height and width), keys and values go into the bf16 cache
  qkv8    the same into the 8-bit cache (e4m3 or e5m2, a power-of-two scale per block of 16 positions and KV head,
          the open block in bf16)
  read8   rows of the 8-bit cache read back as bf16
  chunk   causal attention of the new tokens (a prompt, a part of one, draft tokens) over everything cached, optionally
          over the first positions and a window only

`run` is the plain form, or with `own` the library's calls.  Sequence lengths follow from the case alone, values from
the seed.
"""
import math
import random

import torch

own = False

D = 128                 # values per row
BLOCK = 16              # positions per block and per page
FORMATS = {"e4m3": (torch.float8_e4m3fn, 9), "e5m2": (torch.float8_e5m2, 16)}   # largest finite value: 0.875 * 2^n
SCALE = D ** -0.5
EPS = 1e-6
LAYERS, PHI, ALPHA, FROM_LAYER = 32, 0.7, 1.0, 24      # the window that slides with depth: layer l masks a share of the past


# ------------------------------------------------------------------------------------------ cases
def listed():
    base = dict(kv_heads=8, group=4, ragged=0, paged=False)
    prep = dict(norm=True, pairs="half", rot=128, sections="", spread=False)
    qkv = lambda name, **kw: {"name": name, "kind": "qkv", **base, **prep, **kw}                        # noqa: E731
    qkv8 = lambda name, **kw: {"name": name, "kind": "qkv8", "format": "e4m3", **base, **prep, **kw}    # noqa: E731
    read8 = lambda name, **kw: {"name": name, "kind": "read8", "format": "e4m3", **base, **kw}          # noqa: E731
    chunk = lambda name, **kw: {"name": name, "kind": "chunk", "sinks": 0, "window": 0, "layer": 0, **base, **kw}  # noqa: E731
    return [
        # one user, the next token: latency
        qkv("qkv_token_single", batch=1, context=8191, new=1),
        # prompts with images of a ragged paged batch: three axes, dealt out over the frequencies
        qkv("qkv_image_prompts", batch=12, context=5000, new=4096, kv_heads=4, group=7, ragged=3, paged=True,
            sections="24 20 20", spread=True),
        # one token of each sequence of a serving batch, some of them close a block
        qkv8("qkv8_token", batch=64, context=4099, new=1, ragged=3, paged=True),
        # two long prompts go into the 8-bit cache
        qkv8("qkv8_prompt", batch=2, context=16384, new=16384, norm=False),
        # the rows of two long contexts are read back for a prompt's attention
        read8("read8_prompt", batch=2, context=32768, new=32768),
        # the newest rows of a ragged paged batch, the wider exponent format
        read8("read8_chunk", batch=16, context=9001, new=200, ragged=7, paged=True, format="e5m2"),
        # one user's four draft tokens are checked: latency
        chunk("chunk_single", batch=1, context=2047, new=4),
        # five draft tokens of every sequence of a serving batch: the stream of the cache
        chunk("chunk_draft", batch=16, context=16384, new=5, ragged=5, paged=True),
        # a prompt
        chunk("chunk_prompt", batch=1, context=8192, new=8192),
        # prompts and parts of prompts of a ragged paged batch, grouped by seven
        chunk("chunk_ragged", batch=8, context=8192, new=4096, kv_heads=4, group=7, ragged=9, paged=True),
        # the 7B layer without grouped queries: first positions and the newest ones, in a deep layer
        chunk("chunk_window", batch=2, context=16384, new=4096, kv_heads=32, group=1, sinks=4, window=4096, layer=30),
        # a part of a very long prompt: the largest
        chunk("chunk_long", batch=1, context=131072, new=2048),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["qkv", "qkv", "qkv8", "read8", "chunk", "chunk", "chunk", "chunk"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    c = dict(kind=kind, kv_heads=kv_heads, group=rng.choice([1, 2, 3, 4, 4, 7, 8, 16]) if kv_heads < 32 else 1,
             batch=_log_uniform(rng, 1, 64), ragged=rng.choice([0, 1]) * rng.randint(1, 1000), paged=rng.random() < 0.5)
    most = 131072 * 8                                                   # rows over all KV heads
    c["context"] = _log_uniform(rng, 1, max(1, min(131072, most // (c["batch"] * kv_heads))))
    c["new"] = rng.choice([1, c["context"], _log_uniform(rng, 1, c["context"]), _log_uniform(rng, 1, min(16, c["context"]))])
    if kind in ("qkv", "qkv8"):
        c["new"] = max(1, min(c["new"], 1500000 // (c["batch"] * kv_heads * (c["group"] + 2))))
        c["norm"], c["pairs"] = rng.random() < 0.7, rng.choice(["half", "half", "adjacent"])
        c["rot"] = rng.choice([128, 128, 64, 2 * rng.randint(1, 64)])
        c["sections"], c["spread"] = "", False
        if rng.random() < 0.4:
            n, parts = c["rot"] // 2, rng.choice([2, 3, 4])
            cuts = sorted(rng.randint(0, n) for _ in range(parts - 1))
            c["sections"] = " ".join(str(b - a) for a, b in zip([0] + cuts, cuts + [n]))
            c["spread"] = rng.random() < 0.5
    if kind in ("qkv8", "read8"):
        c["format"] = rng.choice(["e4m3", "e5m2"])
    if kind == "chunk":
        # logits of one KV head over the padded batch, and of all heads
        c["new"] = max(1, min(c["new"], 1 << 14, (1 << 30) // (c["batch"] * c["group"] * c["context"]),
                              8 * (1 << 30) // (c["batch"] * kv_heads * c["group"] * c["context"])))
        c["sinks"], c["window"], c["layer"] = 0, 0, 0
        if rng.random() < 0.4:
            c["sinks"], c["window"] = rng.choice([0, 4, 130]), rng.choice([0, _log_uniform(rng, 1, c["context"])])
            c["layer"] = rng.choice([0, 27, 31])
    return c


def _lengths(case):
    """(positions after the call, of those new) per sequence, from the case alone."""
    B, n, new = case["batch"], case["context"], case["new"]
    if not case["ragged"]:
        return [n] * B, [min(new, n)] * B
    r = random.Random(case["ragged"])
    lens = [r.randint(max(1, n // 8), n) for _ in range(B)]
    lens[r.randrange(B)] = n
    return lens, [min(t, new if new == 1 else r.randint(0, new) if i else new) for i, t in enumerate(lens)]


def _sections(case):
    """How many of the frequencies each axis of the positions has (none given: one axis)."""
    return [int(n) for n in case["sections"].split()]


def _rows(new):
    """Rows of the packed tensors: the new tokens, padded to a multiple of eight where there are several."""
    n = sum(new)
    return n if n < 8 else -(-n // 8) * 8


def _share(case):
    """The share of the past that the layer's sliding window masks (0: none)."""
    if case["layer"] + 1 < FROM_LAYER:
        return 0.0
    return 1.0 - float(torch.tensor(PHI)) ** (ALPHA * (case["layer"] + 1 - FROM_LAYER) / (LAYERS - FROM_LAYER))


def _visible(case, u):
    """How many positions the token at position u - 1 attends over."""
    lo = max(u - case["window"] if case["window"] else 0, math.floor(_share(case) * u), 0)
    return u - max(0, lo - case["sinks"])


def work(case):
    lens, new = _lengths(case)
    H, G, kind = case["kv_heads"], case["group"], case["kind"]
    n = sum(new)
    if kind in ("qkv", "qkv8"):
        out = 2 * D * (G + 2) if kind == "qkv" else 2 * D * G + 2 * D + 2 * 4 / BLOCK
        pos = 4 * max(1, len(_sections(case)))
        return {"bytes": n * (H * (2 * D * (G + 2) + out) + pos), "flops": n * H * (G + 1) * 8 * D}
    if kind == "read8":
        return {"bytes": n * H * 2 * (D + 4 / BLOCK + 2 * D), "flops": n * H * 2 * D}
    pairs = sum(_visible(case, u) for t, m in zip(lens, new) for u in (range(t - m + 1, t + 1) if m < 64 else ()))
    for t, m in zip(lens, new):
        if m >= 64:                              # by sixteenths of a long chunk
            at = [t - m + 1 + round((m - 1) * i / 16) for i in range(17)]
            v = [_visible(case, u) for u in at]
            pairs += sum((b - a) * (x + y) / 2 for a, b, x, y in zip(at, at[1:], v, v[1:])) + v[-1]
    seen = sum(t - (max(0, (t - _visible(case, t - m + 1)) - m + 1) if case["window"] or _share(case) else 0)
               for t, m in zip(lens, new) if m)
    return {"bytes": seen * H * 4 * D + n * H * G * (4 * D + 4), "flops": int(4 * D * G * H * pairs)}


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


def _draw_rows(g, dev, *shape):
    return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)


def _positions(case, start, new, rows, dev):
    """int32 [axes][rows]: text counts on, every other stretch of 400 tokens is an image of 20 x 20."""
    axes = len(_sections(case))
    p = torch.cat([torch.arange(s, s + n) for s, n in zip(start, new)] + [torch.zeros(rows - sum(new), dtype=torch.int64)])
    at, image = p % 400, p // 400 % 2 == 1
    per_axis = [p - torch.where(image, at, 0), p - torch.where(image, at - at // 20, 0), p - torch.where(image, at - at % 20, 0), p]
    return torch.stack(per_axis[:axes]).to(torch.int32).to(dev)


def _pages(lens, g, dev):
    need = [-(-t // BLOCK) for t in lens]
    order = torch.randperm(sum(need), generator=g, device=dev).to(torch.int32)
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    lens, new = _lengths(case)
    start = [t - n for t, n in zip(lens, new)]
    B, H, G, kind = case["batch"], case["kv_heads"], case["group"], case["kind"]
    cap = -(-max(lens) // BLOCK) * BLOCK
    rows = _rows(new)
    s = {"case": case, "max_len": max(lens), "max_new": max(new), "rows": rows,
         "lens": torch.tensor(lens, dtype=torch.int32, device=dev),
         "row_start": torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)}
    s["table"], pool = _pages(lens, g, dev) if case["paged"] else (None, 0)
    shape = (pool, H, BLOCK, D) if case["paged"] else (B, H, cap, D)
    channel = torch.where(torch.rand(H, 1, D, generator=g, device=dev) < 0.05, 3.0, 1.0)
    if kind in ("qkv", "qkv8"):
        s["qkv"] = _draw_rows(g, dev, rows, (H * G + 2 * H) * D)
        s["q_out"] = torch.zeros(rows, H * G, D, dtype=torch.bfloat16, device=dev)
        s["q_weight"], s["k_weight"] = ((1 + 0.2 * torch.randn(D, generator=g, device=dev)) for _ in range(2))
        s["inv_freq"] = (500000.0 ** (-2 * torch.arange(case["rot"] // 2, dtype=torch.float64) / case["rot"])).float().to(dev)
        s["positions"] = _positions(case, start, new, rows, dev) if case["sections"] else None
    if kind in ("qkv", "chunk"):
        s["k"] = (_draw_rows(g, dev, *shape).float() * channel).to(torch.bfloat16) if kind == "chunk" else _draw_rows(g, dev, *shape)
        s["v"] = _draw_rows(g, dev, *shape)
    if kind == "chunk":
        s["q"] = _draw_rows(g, dev, rows, H * G, D)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(rows, H * G, device=dev)
    if kind in ("qkv8", "read8"):
        for n in "kv":
            codes = torch.empty(shape, dtype=FORMATS[case["format"]][0], device=dev)
            scale = torch.empty(shape[:2] if case["paged"] else (B, H, cap // BLOCK), device=dev)
            for i in range(0, shape[0], 1 if not case["paged"] else 4096):
                part = slice(i, i + (1 if not case["paged"] else 4096))
                x = torch.randn(codes[part].shape, generator=g, device=dev) * channel * 2.0 ** (torch.arange(H, device=dev) % 3 - 1)[:, None, None]
                y, z = _quantise(x.view(x.shape[0], H, -1, BLOCK, D), case["format"])
                codes[part], scale[part] = y.view(x.shape), z.view(scale[part].shape)
            s[n + "8"], s[n + "_scale"] = codes, scale
            s[n + "_tail"] = _draw_rows(g, dev, B, H, BLOCK, D)
    if kind == "qkv8":
        again = any(n > 1 and t // BLOCK > a // BLOCK and a % BLOCK for t, n, a in zip(lens, new, start))
        s["tails"] = (s["k_tail"].clone(), s["v_tail"].clone()) if again else None
    if kind == "read8":
        s["first"] = torch.tensor(start, dtype=torch.int32, device=dev)
        s["k"], s["v"] = (torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(2))
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _tokens(s):
    """Sequence and position of every row that belongs to a sequence."""
    row = torch.arange(s["rows"], device=s["lens"].device)
    b = torch.searchsorted(s["row_start"][1:].contiguous(), row.to(torch.int32), right=True)
    live = b < s["lens"].shape[0]
    row, b = row[live], b[live]
    return row, b, (s["lens"][b] - s["row_start"][b + 1]).long() + row


def _axis_of(case):
    """The axis that each frequency takes its position from."""
    n, axes = case["rot"] // 2, _sections(case) or [case["rot"] // 2]
    if not case["spread"]:
        return [a for a, k in enumerate(axes) for _ in range(k)]
    left, out = list(axes), []
    while len(out) < n:                          # in turn, as long as an axis has frequencies left
        for a in range(len(axes)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return out


def _prepared(x, weight, cos, sin, case):
    """Heads [rows][heads][128] in fp32: normalised, then the first `rot` values rotated."""
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    r = case["rot"]
    if case["pairs"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)
    a, b = x[..., :r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)


def _split(s):
    case = s["case"]
    H, G = case["kv_heads"], case["group"]
    x = s["qkv"].view(s["rows"], H * G + 2 * H, D)
    return x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]


def _plain_heads(s):
    case = s["case"]
    row, b, pos = _tokens(s)
    at = s["positions"][:, row].long() if s["positions"] is not None else pos[None]
    axis = torch.tensor(_axis_of(case), device=row.device)
    angle = at[axis].T.double() * s["inv_freq"].double()               # far positions need more than 32 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q, k, v = _split(s)
    q = _prepared(q[row].float(), s["q_weight"], cos, sin, case).to(torch.bfloat16)
    k = _prepared(k[row].float(), s["k_weight"], cos, sin, case).to(torch.bfloat16)
    s["q_out"][row] = q
    return row, b, pos, k, v[row]


def _plain_qkv(s):
    row, b, pos, k, v = _plain_heads(s)
    if s["table"] is not None:
        page = s["table"][b, pos // BLOCK].long()
        s["k"][page, :, pos % BLOCK], s["v"][page, :, pos % BLOCK] = k, v
    else:
        s["k"][b, :, pos], s["v"][b, :, pos] = k, v
    return [s["q_out"], s["k"], s["v"]]


def _plain_qkv8(s):
    case, t = s["case"], s["lens"].long()
    row, b, pos, k, v = _plain_heads(s)
    H = case["kv_heads"]
    new = (s["row_start"][1:] - s["row_start"][:-1]).long()
    first = (t - new) // BLOCK
    span = -(-(s["max_new"] + BLOCK - 1) // BLOCK) + 1                  # blocks that a sequence may touch
    blk = first[:, None] + torch.arange(span, device=t.device)
    whole = ((blk + 1) * BLOCK <= t[:, None]) & (new[:, None] > 0)
    opens = (blk == (t // BLOCK)[:, None]) & (new[:, None] > 0)
    wb, wi = whole.nonzero(as_tuple=True)
    ob, oi = opens.nonzero(as_tuple=True)
    for x, tail, codes, scale in ((k, s["k_tail"], s["k8"], s["k_scale"]), (v, s["v_tail"], s["v8"], s["v_scale"])):
        full = torch.zeros(t.shape[0], H, span * BLOCK, D, dtype=torch.bfloat16, device=t.device)
        full[:, :, :BLOCK] = tail                                       # rows of the first block that were there
        full[b, :, pos - first[b] * BLOCK] = x
        full = full.view(t.shape[0], H, span, BLOCK, D)
        y, z = _quantise(full[wb, :, wi].float(), case["format"])
        where = blk[wb, wi]
        raw, y = codes.view(torch.uint8), y.view(torch.uint8)
        if s["table"] is not None:
            page = s["table"][wb, where].long()
            raw[page], scale[page] = y, z
        else:
            raw.view(*raw.shape[:2], -1, BLOCK, D)[wb, :, where], scale[wb, :, where] = y, z
        fresh = (blk[ob, oi] * BLOCK)[:, None] + torch.arange(BLOCK, device=t.device)
        fresh = (fresh >= (t - new)[ob][:, None]) & (fresh < t[ob][:, None])
        tail[ob] = torch.where(fresh[:, None, :, None], full[ob, :, oi], tail[ob])
    return [s["q_out"], s["k8"], s["k_scale"], s["v8"], s["v_scale"], s["k_tail"], s["v_tail"]]


def _plain_read8(s):
    t, first = s["lens"].long(), s["first"].long()
    pos = first[:, None] + torch.arange(s["max_new"], device=t.device)
    b, i = (pos < t[:, None]).nonzero(as_tuple=True)
    pos = pos[b, i]
    blk, row = pos // BLOCK, pos % BLOCK
    opened = (pos >= (t // BLOCK * BLOCK)[b])[:, None, None]
    for out, codes, scale, tail in ((s["k"], s["k8"], s["k_scale"], s["k_tail"]), (s["v"], s["v8"], s["v_scale"], s["v_tail"])):
        raw = codes.view(torch.uint8)
        if s["table"] is not None:
            page = s["table"][b, blk].long()
            x, z = raw[page, :, row], scale[page]
        else:
            x, z = raw[b, :, pos], scale[b, :, blk]
        x = torch.where(opened, tail[b, :, row].float(), x.view(codes.dtype).float() * z[..., None]).to(torch.bfloat16)
        if s["table"] is not None:
            out[page, :, row] = x
        else:
            out[b, :, pos] = x
    return [s["k"], s["v"]]


def _plain_chunk(s):
    case, t = s["case"], s["lens"].long()
    B, H, G, n = case["batch"], case["kv_heads"], case["group"], s["max_new"]
    dev = t.device
    row, b, pos = _tokens(s)
    at = (pos - (t - (s["row_start"][1:] - s["row_start"][:-1]).long())[b])       # which of its sequence's new tokens
    u = torch.zeros(B, n, dtype=torch.int64, device=dev)                       # visible length of each token, 0: none
    u[b, at] = pos + 1
    i = torch.arange(s["max_len"], device=dev)
    lo = (u.double() * _share(case)).floor().long()
    if case["window"]:
        lo = torch.maximum(lo, u - case["window"])
    see = (i < u[..., None]) & ((i < case["sinks"]) | (i >= lo[..., None]))    # [B][n][len]
    blocks = torch.arange(-(-s["max_len"] // BLOCK), device=dev)
    for h in range(H):
        q = torch.zeros(B, n, G, D, device=dev)
        q[b, at] = s["q"][row, h * G:h * G + G].float()
        k, v = ((x[s["table"][:, blocks].long(), h].flatten(1, 2) if s["table"] is not None else x[:, h])[:, :s["max_len"]].float()
                for x in (s["k"], s["v"]))
        held = (i < t[:, None])[..., None]
        k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)
        a = (q.view(B, n * G, D) @ k.transpose(-1, -2)).view(B, n, G, -1)
        a.mul_(SCALE).masked_fill_(~see[:, :, None], -math.inf)
        top = a.amax(-1, keepdim=True)
        p = a.sub_(torch.where(top.isfinite(), top, 0.0)).exp_()
        total = p.sum(-1, keepdim=True)
        out = (p.view(B, n * G, -1) @ v).view(B, n, G, D) / torch.where(total > 0, total, 1.0)
        s["out"][row, h * G:h * G + G] = out[b, at].to(torch.bfloat16)
        s["lse"][row, h * G:h * G + G] = (top + total.log())[b, at, :, 0]
    return [s["out"], s["lse"]]


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
        _contexts[key] = P.Context(num_layers=LAYERS, max_batch=case["batch"], num_q_heads=case["kv_heads"] * case["group"],
                                   num_kv_heads=case["kv_heads"], max_context=s["max_len"], max_k=1, max_window=1,
                                   max_sinks=4, page_size=BLOCK if case["paged"] else 0, min_layer_group=LAYERS)
    return _contexts[key]


def _own(s):
    from paper_2602_08329_b200 import binding as P
    case = s["case"]
    ctx, B, kind = _context(s), case["batch"], case["kind"]
    if kind in ("qkv", "qkv8"):
        if "prep" not in s:                      # kept with the layer's weights
            s["prep"] = P.make_qk_prep(s["q_weight"] if case["norm"] else None, s["k_weight"] if case["norm"] else None, eps=EPS,
                                       norm=case["norm"], inv_freq=s["inv_freq"], adjacent=case["pairs"] == "adjacent",
                                       axis_of=_axis_of(case) if case["sections"] else None)
        q, k, v = _split(s)
    if kind in ("qkv8", "read8"):
        kv8 = P.make_bytekv_view(s["k8"], s["v8"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"], s["lens"],
                                 page_table=s["table"], max_seq_len=s["max_len"])
        if kind == "qkv8":
            ctx.bytekv_qkv_append(q, k, v, kv8, s["prep"], B, s["q_out"], row_start=s["row_start"], positions=s["positions"])
            return [s["q_out"], s["k8"], s["k_scale"], s["v8"], s["v_scale"], s["k_tail"], s["v_tail"]]
    kv = P.make_view(s["k"], s["v"], s["lens"], page_table=s["table"], max_seq_len=s["max_len"])
    if kind == "qkv":
        ctx.qkv_append(q, k, v, kv, s["prep"], B, s["q_out"], row_start=s["row_start"], positions=s["positions"])
        return [s["q_out"], s["k"], s["v"]]
    if kind == "read8":
        ctx.bytekv_read(kv8, kv, B, first=s["first"], max_new=s["max_new"])
        return [s["k"], s["v"]]
    mask = P.make_chunk_mask(sinks=case["sinks"], window=case["window"], layer=case["layer"], psaw_phi=PHI, psaw_alpha=ALPHA,
                             psaw_layer_start=FROM_LAYER)
    ctx.chunk_attn(s["q"], kv, B, s["out"], s["lse"], row_start=s["row_start"], mask=mask)
    return [s["out"], s["lse"]]


def run(state):
    if state.get("tails") is not None:      # the open blocks as they were before these rows came in
        state["k_tail"].copy_(state["tails"][0])
        state["v_tail"].copy_(state["tails"][1])
    if own:
        return _own(state)
    return {"qkv": _plain_qkv, "qkv8": _plain_qkv8, "read8": _plain_read8, "chunk": _plain_chunk}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------ 64 bits
def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round8(v, fmt):
    """Nearest representable value (ties to even) of |v| within the format's range, in 64 bits."""
    bits, lowest = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(v).exponent.double().sub(1).clamp_min(lowest)
    step = _two_to(e - bits)
    return torch.round(v / step) * step


def _scale64(amax, top):
    e = torch.ceil(torch.log2(amax / top)).clamp_min(-126.0)
    e = e + (amax > top * _two_to(e)).double()              # log2 may be off by a rounding at a power of two
    e = torch.where((e > -126) & (amax <= top * _two_to(e - 1)), e - 1, e)
    return _two_to(e)


def _heads64(s, b, n, start):
    """Prepared queries and keys and the values of sequence b's new tokens, [n][heads][128] in 64 bits."""
    case = s["case"]
    H, G, r0, r = case["kv_heads"], case["group"], int(s["row_start"][b]), case["rot"]
    x = s["qkv"][r0:r0 + n].double().view(n, H * G + 2 * H, D)
    q, k, v = x[:, :H * G], x[:, H * G:-H], x[:, -H:]
    res = []
    where = torch.arange(start, start + n, dtype=torch.float64, device=x.device)[:, None].expand(n, r // 2)
    if s["positions"] is not None:
        where = torch.stack([s["positions"][a, r0:r0 + n].double() for a in _axis_of(case)], -1)
    turn = torch.polar(torch.ones_like(where), where * s["inv_freq"].double())[:, None]
    for y, w in ((q, s["q_weight"]), (k, s["k_weight"])):
        if case["norm"]:
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
        first, rest = y[..., :r], y[..., r:]
        z = first.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["pairs"] == "half" else first.unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = (z.transpose(-1, -2) if case["pairs"] == "half" else z).flatten(-2)
        res.append(torch.cat([z, rest], -1))
    return res[0], res[1], v


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    H, G, kind = case["kv_heads"], case["group"], case["kind"]
    dev = s["lens"].device

    def ids(b, n0, n1):
        return s["table"][b, n0:n1].long()

    if kind in ("qkv", "qkv8"):
        q_out = s["q_out"].double()
        if kind == "qkv":
            cache = {n: s[n].double() for n in "kv"}
        else:
            cache = {n: s[n + "8"].to(torch.float64) for n in "kv"}
            scales, tails = ({n: s[n + e].double() for n in "kv"} for e in ("_scale", "_tail"))
        for b, (t, n) in enumerate(zip(lens, new)):
            if not n:
                continue
            q, k, v = _heads64(s, b, n, t - n)
            r0 = int(s["row_start"][b])
            q_out[r0:r0 + n] = q
            for name, x in (("k", k), ("v", v)):
                c = cache[name]
                if kind == "qkv":
                    p = torch.arange(t - n, t, device=dev)
                    if case["paged"]:
                        c[s["table"][b, p // BLOCK].long(), :, p % BLOCK] = x
                    else:
                        c[b, :, t - n:t] = x.transpose(0, 1)
                    continue
                f = (t - n) // BLOCK
                # the cache's rows are bf16 before they are quantised
                x = torch.cat([s[name + "_tail"][b, :, :t - n - f * BLOCK], x.to(torch.bfloat16).transpose(0, 1)], 1).double()
                w = x.shape[1] // BLOCK
                if w:
                    y = x[:, :w * BLOCK].reshape(H, w, BLOCK, D)
                    z = _scale64(y.abs().amax((-2, -1)), 448.0 if case["format"] == "e4m3" else 57344.0)
                    y = _round8(y / z[..., None, None], case["format"])
                    if case["paged"]:
                        c[ids(b, f, f + w)], scales[name][ids(b, f, f + w)] = y.transpose(0, 1), z.transpose(0, 1)
                    else:
                        c[b, :, f * BLOCK:(f + w) * BLOCK], scales[name][b, :, f:f + w] = y.reshape(H, w * BLOCK, D), z
                left = x.shape[1] - w * BLOCK
                if left:
                    tails[name][b, :, :left] = x[:, w * BLOCK:]
        if kind == "qkv":
            return [q_out, cache["k"], cache["v"]]
        return [q_out, cache["k"], scales["k"], cache["v"], scales["v"], tails["k"], tails["v"]]
    if kind == "read8":
        res = []
        for name in "kv":
            out, codes, scale = s[name].double(), s[name + "8"].view(torch.uint8), s[name + "_scale"].double()
            for b, (t, n) in enumerate(zip(lens, new)):
                for blk in [slice(i, min(i + 512, t // BLOCK)) for i in range((t - n) // BLOCK, t // BLOCK, 512)]:
                    p = torch.arange(max(blk.start * BLOCK, t - n), blk.stop * BLOCK, device=dev)
                    if case["paged"]:
                        page = s["table"][b, p // BLOCK].long()
                        out[page, :, p % BLOCK] = codes[page, :, p % BLOCK].view(s[name + "8"].dtype).double() * scale[page][..., None]
                    else:
                        y = codes[b, :, p].view(s[name + "8"].dtype).double() * scale[b][:, p // BLOCK][..., None]
                        out[b, :, p] = y
                p = torch.arange(max(t // BLOCK * BLOCK, t - n), t, device=dev)
                if len(p):
                    y = s[name + "_tail"][b, :, p % BLOCK].double()
                    if case["paged"]:
                        out[s["table"][b, t // BLOCK].long(), :, p % BLOCK] = y
                    else:
                        out[b, :, p] = y
            res.append(out)
        return res
    out, lse = s["out"].double(), s["lse"].double()
    share = _share(case)
    for b, (t, n) in enumerate(zip(lens, new)):
        if not n:
            continue
        r0, blocks = int(s["row_start"][b]), -(-t // BLOCK)
        for h in range(H):
            k, v = ((s[x][ids(b, 0, blocks), h].reshape(-1, D) if case["paged"] else s[x][b, h])[:t].double() for x in "kv")
            step = max(1, (1 << 27) // (t * G))
            for j in range(0, n, step):
                m = min(step, n - j)
                u = torch.arange(t - n + j + 1, t - n + j + m + 1, device=dev)
                a = torch.einsum("ngd,id->ngi", s["q"][r0 + j:r0 + j + m, h * G:h * G + G].double(), k) / math.sqrt(D)
                lo = torch.floor(share * u.double()).long()
                if case["window"]:
                    lo = torch.maximum(lo, u - case["window"])
                i = torch.arange(t, device=dev)
                hidden = (i >= u[:, None]) | ((i >= case["sinks"]) & (i < lo[:, None]))
                a.masked_fill_(hidden[:, None], -math.inf)
                z = torch.logsumexp(a, -1)
                lse[r0 + j:r0 + j + m, h * G:h * G + G] = z
                out[r0 + j:r0 + j + m, h * G:h * G + G] = a.sub_(z[..., None]).exp_() @ v
    return [out, lse]
