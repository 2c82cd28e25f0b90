"""The calls of the 8-bit cache and of block selection without a GPU: layouts, refusals, and the 64-bit forms' own pins."""
import ctypes as C
import os
import re
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

from paper_2602_08329_b200 import binding as P
from paper_2602_08329_b200 import build as B
from tests import cache_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load()


# ------------------------------------------------------------------------------- layouts
def struct_fields(name):
    """Field names of a struct of the header, in order."""
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "prhs.h")).read(), flags=re.S)
    body = next(b for b, n in re.findall(r"typedef struct \{([^}]*)\}\s*(\w+);", text) if n == name)
    names = []
    for decl in body.split(";"):
        names += [re.sub(r".*[\s*]", "", part.strip()) for part in decl.split(",") if part.strip()]
    return names


@pytest.mark.parametrize("name,mirror,size", [("prhs_bytekv_view", P.ByteKvView, 112), ("prhs_block_bounds_view", P.BlockBoundsView, 32),
                                              ("prhs_block_schedule", P.BlockSchedule, 16)])
def test_structs_mirror_the_header(name, mirror, size):
    assert [f for f, _ in mirror._fields_] == struct_fields(name) and C.sizeof(mirror) == size


def test_packed_views_have_the_struct_layout():
    view = P.ByteKvView.from_buffer_copy(P._BYTEKV_PACK(*range(1, 17)))
    assert [getattr(view, f) for f, _ in P.ByteKvView._fields_] == list(range(1, 17))
    view = P.KvView.from_buffer_copy(P._KV_PACK(*range(1, 10)))
    assert [getattr(view, f) for f, _ in P.KvView._fields_] == list(range(1, 10))


def test_header_formats_match():
    text = open(os.path.join(ROOT, "include", "prhs.h")).read()
    for name in ("PRHS_BYTEKV_E4M3", "PRHS_BYTEKV_E5M2"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(P, name)


# ------------------------------------------------------------------------------- build
def test_the_compiled_binding_is_built_again_for_another_torch(lib, monkeypatch):
    assert P._load_marshal().built_for == B._built_for() and not B.stale()
    commands = []
    monkeypatch.setattr(B, "_run", lambda cmd, what: commands.append((what, cmd)) or "")
    B.build()
    assert commands == []
    for version, made in (("99.1.0", ["g++"]), (None, [])):
        monkeypatch.setattr(B.importlib.metadata, "version", lambda name, version=version: version)
        monkeypatch.setattr(B.importlib.util, "find_spec", lambda name, version=version: version)
        commands.clear()
        assert B.stale() == bool(made)
        B.build()
        assert [what for what, _ in commands] == made
    B.build(force=True)                          # no torch: the C library alone
    assert [what for what, _ in commands] == ["nvcc"]


def test_a_torch_without_metadata_is_known_by_its_version(monkeypatch):
    def unknown(name):
        raise B.importlib.metadata.PackageNotFoundError(name)
    monkeypatch.setattr(B.importlib.metadata, "version", unknown)
    assert torch.__version__ in B._built_for()


# ------------------------------------------------------------------------------- refusals
def test_null_context_is_refused(lib):
    kv, bounds, view = P.ByteKvView(), P.BlockBoundsView(), P.KvView()
    sched = P.make_block_schedule(1)
    assert lib.prhs_bytekv_append(None, C.byref(kv), None, None, 0, 0, 0, None, 1, 1, None) == 1
    assert lib.prhs_bytekv_decode_attn(None, None, C.byref(kv), 1, None, None, None) == 1
    assert lib.prhs_bytekv_sparse_decode_attn(None, None, C.byref(kv), None, None, 1, 1, None, None, None) == 1
    assert lib.prhs_block_bounds(None, C.byref(view), C.byref(bounds), None, 0, 1, None) == 1
    assert lib.prhs_block_topk(None, None, C.byref(view), C.byref(bounds), C.byref(sched), 1, None, 1, None, None) == 1
    assert lib.prhs_block_decode_attn(None, None, C.byref(view), None, None, 1, 0, 1, None, None, None) == 1
    assert lib.prhs_block_decode_step(None, None, C.byref(view), C.byref(bounds), C.byref(sched), 1, None, None, None, 1, None, None) == 1


def test_host_tensors_and_wrong_types_are_refused(lib):
    k = torch.zeros(2, 3, 32, 128, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 3, 2)
    t = torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError, match="CUDA"):
        P.make_bytekv_view(k, k, s, s, t, t, lens)
    with pytest.raises(AssertionError, match="float8"):
        P.make_bytekv_view(t, t, s, s, t, t, lens)
    with pytest.raises(AssertionError):
        P.make_bytekv_view(k, None, s, s, t, t, lens)
    with pytest.raises(AssertionError, match="CUDA"):
        P.make_block_bounds(torch.zeros(2, 3, 4, 2, 128, dtype=torch.int8), torch.zeros(2, 3, 4))
    with pytest.raises(AssertionError):
        P.make_view(t.float(), t.float(), lens)
    m, N = P._load_marshal(), None
    calls = ((m.kv_view, (N, N, N, N)), (m.bytekv_view, (N,) * 8 + (0,)), (m.bounds_view, (N, N)),
             (m.bytekv_append, (0, 0, t, t, lens, 2, 3, 0, 0, 0)), (m.bytekv_append, (0, 0, N, N, N, 2, 3, 0, 0, 0)),
             (m.bytekv_decode_attn, (0, 0, t, t, N, 2, 3, 0, 0)), (m.bytekv_decode_attn, (0, 0, N, N, N, 2, 3, 0, 0)),
             (m.bytekv_sparse_decode_attn, (0, 0, t, t, N, 2, 3, 0, 0, lens, lens)), (m.block_bounds, (0, 0, 0, lens, 0, 2, 0, 0)),
             (m.block_topk, (0, 0, 0, 0, t, 2, 3, 3, 0, 0, lens, lens)), (m.block_decode_attn, (0, 0, t, t, N, 2, 3, 3, 0, 0, lens, lens, 0)),
             (m.block_decode_step, (0, 0, 0, 0, t, t, N, 2, 3, 3, 0, 0, lens, lens)))
    for f, args in calls:
        with pytest.raises(AssertionError):
            f(*args)                            # nothing there, or host tensors where device 0 is asked for
        with pytest.raises(TypeError):
            f(*args[:-1])
        with pytest.raises(TypeError):
            f(*args, N)
    with pytest.raises(TypeError):
        m.bytekv_decode_attn("ctx", 0, t, t, N, 2, 3, 0, 0)


def test_tensors_without_storage_raise(lib):
    """torch's C++ exception has to arrive as Python's; out of a C function it would end the process."""
    sparse = torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16).to_sparse()
    dense, lens = torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises((RuntimeError, AssertionError)):
        P.make_view(sparse, sparse, lens)
    with pytest.raises(RuntimeError, match="storage"):
        P.make_view(dense, dense, lens.to_sparse())


NO_DATA = """
import torch
from paper_2602_08329_b200 import binding as P
m = P._load_marshal()
t, lens, n = torch.zeros(5, 2, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), None
lists = torch.zeros(2, 3, 4, dtype=torch.int32)
calls = {
    "append": lambda x: m.bytekv_append(0, 0, x, x, lens, 2, 3, -1, 0, 0),
    "append, lengths": lambda x: m.bytekv_append(0, 0, t[0], t[0], x[:, 0, 0, 0].to(torch.int32), 2, 3, -1, 0, 0),
    "attend": lambda x: m.bytekv_decode_attn(0, 0, x[:, :, 0].contiguous(), None, n, 2, 3, -1, 0),
    "lists": lambda x: m.bytekv_sparse_decode_attn(0, 0, x[:, :, 0].contiguous(), None, n, 2, 3, -1, 0, lists, lists[:, :, 0].contiguous()),
    "bounds": lambda x: m.block_bounds(0, 0, 0, x[:, 0, 0, 0].to(torch.int32), 0, 2, -1, 0),
    "blocks": lambda x: m.block_decode_attn(0, 0, t[0, :, :, 0].contiguous(), None, n, 2, 3, 3, -1, 0, x[..., 0].to(torch.int32), lists[:, :, 0].contiguous(), 0),
}
for name, call in calls.items():
    try:
        torch.vmap(lambda x: call(x) and x)(t)
    except RuntimeError as e:
        assert "storage" in str(e) or "data" in str(e), (name, e)
        print(name)
"""


def test_calls_with_tensors_that_have_no_data_raise(lib):
    """A batched tensor has sizes, strides and a type, but no address.  (In a process of its own: without the interpreter's
    lock an exception ends it.)"""
    res = subprocess.run([sys.executable, "-X", "faulthandler", "-c", NO_DATA], cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    assert res.stdout.split("\n")[:-1] == ["append", "append, lengths", "attend", "lists", "bounds", "blocks"]


def test_views_take_rows_of_a_wider_page_table(lib):
    pool, lens = torch.zeros(9, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 8, dtype=torch.int32)
    for t in (table, table[:, :4], table[:, 2:]):
        view = P.make_view(pool, pool, lens, page_table=t)
        assert (view.page_table_stride, view.page_table, view.num_pages) == (8, t.data_ptr(), 9)
    for t in (table[:, ::2], table.long()):
        with pytest.raises(AssertionError):
            P.make_view(pool, pool, lens, page_table=t)


def stand_in(**kw):
    """What Context._fit reads of a context (none can be made without a GPU); its device is that of host tensors."""
    return types.SimpleNamespace(**{**dict(_hkv=2, _max_context=64, _dev=-1), **kw})


def test_the_block_calls_refuse_views_that_do_not_fit(lib):
    k, lens = torch.zeros(3, 2, 64, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    pool, table = torch.zeros(9, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32)
    fit = lambda view, batch=3, **kw: P.Context._fit(stand_in(**kw), view, batch)  # noqa: E731
    for view, why in ((P.make_view(k, k, lens), "one CUDA device"), (P.make_view(pool, pool, lens, page_table=table), "one CUDA device"),
                      (P.make_view(k, k[:2], lens), "alike"), (P.make_view(k, k, torch.zeros(6, dtype=torch.int32)[::2]), "contiguous"),
                      (P.make_view(k, k, lens[None]), "contiguous"), (P.make_view(k[:, 0], k[:, 0], lens), "four axes"),
                      (P.make_view(pool, pool, lens[:1], page_table=table[0]), "pages of 16"),
                      (P.make_view(k, k, lens, page_table=table), "pages of 16"),
                      (P.make_view(k.to("meta"), k.to("meta"), lens), "one CUDA device")):
        assert view._dev == -1
        for dev in (0, 1):
            with pytest.raises(AssertionError, match=why):
                fit(view, 1, _dev=dev)
    # a view of one device against a context of another, and batches beyond the cache's or the table's rows
    for view in (P.make_view(k, k, lens), P.make_view(pool, pool, lens, page_table=table)):
        view._why, view._dev = None, 1
        fit(view, _dev=1)
        for wrong in (dict(_dev=0), dict(_dev=1, _hkv=4), dict(_dev=1, batch=4)):
            with pytest.raises(AssertionError, match="those of the context"):
                fit(view, wrong.pop("batch", 3), **wrong)
    assert P.make_view(k[:2], k[:2], lens)._batch == 2 and P.make_view(pool, pool, lens, page_table=table[:1])._batch == 1


def test_lengths_end_with_the_cache_or_a_row_of_the_page_table(lib):
    k, lens = torch.zeros(3, 2, 48, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    pool, table = torch.zeros(9, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.int32)
    for make in (lambda **kw: P.make_view(k, k, lens, **kw), lambda **kw: P.make_view(pool, pool, lens, page_table=table[:, 2:5], **kw)):
        view = make()
        for context, bound in ((640, 48), (48, 0), (32, 0), (64, 48)):      # 0: the context's maximum
            P.Context._fit(stand_in(_max_context=context), view, 3)         # one view, several contexts
            assert view.max_seq_len == bound
        P.Context._fit(stand_in(), make(max_seq_len=48), 3)
        with pytest.raises(AssertionError, match="at most"):
            P.Context._fit(stand_in(), make(max_seq_len=49), 3)


# --------------------------------------------------------------------- the 64-bit forms' pins
@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_codes_are_torchs_rounding(fmt, dtype):
    g = torch.Generator().manual_seed(1)
    top = R.TOP[fmt][0]
    x = (torch.rand(20000, generator=g) * 2 - 1) * top * torch.exp2(-torch.randint(0, 24, (20000,), generator=g).float())
    x = torch.cat([x, torch.tensor([0.0, top, -top])])
    assert np.array_equal(R.round_code(x.double().numpy(), fmt), x.to(dtype).double().numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_scales(fmt):
    top = R.TOP[fmt][0]
    assert float(R.scale_of(top, top)) == 1.0 and float(R.scale_of(np.nextafter(top, 1e9), top)) == 2.0
    assert float(R.scale_of(top / 2, top)) == 0.5 and float(R.scale_of(0.0, top)) == 2.0 ** -126
    assert float(R.scale_of(1e-40, top)) == 2.0 ** -126
    rng = np.random.default_rng(0)
    rows = rng.standard_normal((16, 128)) * np.exp2(rng.integers(-6, 6, (16, 1)))
    codes, s = R.quantise(rows, fmt)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(rows / s), 2.0 ** R.TOP[fmt][2]))) - R.TOP[fmt][1])
    assert np.all(np.abs(codes * s - rows) <= s * step / 2) and np.abs(codes).max() <= top


def test_scores_bound_every_key_inside_the_coded_box():
    rng = np.random.default_rng(3)
    for _ in range(20):
        rows = rng.standard_normal((rng.integers(1, 17), 128)) * 2
        codes, s = R.block_bounds(rows)
        q = rng.standard_normal(128)
        q8, qs = R.query_codes(q)
        score = R.block_scores(q, codes[None], np.array([s]))[0]
        inside = codes[0] + (codes[1].astype(int) - codes[0]) * rng.random((50, 128))
        assert np.all(inside * s @ (q8 * qs) <= score * (1 + 1e-12) + 1e-9)
        # a key is at most half a code outside its box, a query at most half a code off
        off = 0.5 * s * np.abs(q8 * qs).sum() + 0.5 * qs * np.abs(rows).sum(-1).max()
        assert (rows @ q).max() <= score + off


def test_selection_takes_the_best_and_the_lowest_of_equals():
    score = np.array([5.0, 1.0, 3.0, 3.0, 3.0, 9.0, 0.0, 3.0])
    assert R.select_blocks(score, 8, 2, 1, 1) == [0, 2, 5, 7]
    assert R.select_blocks(score, 8, 3, 0, 0) == [0, 2, 5]
    assert R.select_blocks(score, 8, 100, 2, 2) == list(range(8))
    assert R.select_blocks(score[:1], 1, 5, 3, 3) == [0] and R.select_blocks(score[:0], 0, 5, 3, 3) == []


def test_attention_bounds_cover_a_bf16_emulation():
    # weights rounded to bf16, result rounded to bf16: the error stays inside the stated bound
    g = torch.Generator().manual_seed(2)
    q, k, v = torch.randn(128, generator=g), torch.randn(300, 128, generator=g), torch.randn(300, 128, generator=g)
    y, lse, tol, ltol = R.attend(q.numpy(), k.numpy(), v.numpy(), True)
    a = (k @ q) * R.S
    p = torch.exp(a - a.max()).to(torch.bfloat16).float()
    got = ((p @ v) / p.sum()).to(torch.bfloat16).double().numpy()
    assert np.all(np.abs(got - y) <= tol) and abs(float(torch.logsumexp(a, 0)) - lse) <= ltol
