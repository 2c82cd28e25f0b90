"""New tokens, the read-back and the attention of many tokens without a GPU: layouts, refusals, and the helpers."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2602_08329_b200 import binding as P
from paper_2602_08329_b200 import build as B
from tests.test_byte_blocks_host import struct_fields

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load()


@pytest.mark.parametrize("name,mirror,size", [("prhs_token_rows", P.TokenRows, 104), ("prhs_qk_prep", P.QkPrep, 112), ("prhs_chunk_mask", P.ChunkMask, 24)])
def test_structs_mirror_the_header(name, mirror, size):
    assert [f for f, _ in mirror._fields_] == [f.split("[")[0] for f in struct_fields(name)] and C.sizeof(mirror) == size


def test_header_constants_match():
    text = open(os.path.join(ROOT, "include", "prhs.h")).read()
    for name in ("PRHS_PREP_NORM", "PRHS_PREP_ADJACENT", "PRHS_MAX_AXES"):
        assert int(re.search(rf"#define {name}\s+(\d+)", text).group(1)) == getattr(P, name)


def test_null_context_is_refused(lib):
    rows, prep, kv8, kv, mask = P.TokenRows(), P.make_qk_prep(), P.ByteKvView(), P.KvView(), P.make_chunk_mask()
    assert lib.prhs_qkv_append(None, C.byref(rows), C.byref(prep), C.byref(kv), 1, None, None) == 1
    assert lib.prhs_bytekv_qkv_append(None, C.byref(rows), C.byref(prep), C.byref(kv8), 1, None, None) == 1
    assert lib.prhs_bytekv_read(None, C.byref(kv8), C.byref(kv), None, 0, 1, None) == 1
    assert lib.prhs_chunk_attn(None, None, None, 1, C.byref(kv), C.byref(mask), 1, None, None, None) == 1


def test_prep_arguments():
    p = P.make_qk_prep()
    assert (p.flags, p.rot_dim, p.num_axes, p.inv_freq, p.rot_scale) == (0, 0, 1, None, 1.0)
    assert P.make_qk_prep(norm=True, adjacent=True).flags == P.PRHS_PREP_NORM | P.PRHS_PREP_ADJACENT
    for kw in (dict(q_weight=torch.ones(128)), dict(inv_freq=torch.ones(64)), dict(axis_of=[0])):
        with pytest.raises(AssertionError):
            P.make_qk_prep(**kw)


def test_rotation_axes():
    assert P.rotation_axes([2, 0, 1]) == [0, 0, 2]
    assert P.rotation_axes([3, 1, 2], interleaved=True) == [0, 1, 2, 0, 2, 0]
    assert P.rotation_axes([]) == P.rotation_axes([], interleaved=True) == []
    for sections in ([24, 20, 20], [1, 30, 5, 28]):
        for interleaved in (False, True):
            axes = P.rotation_axes(sections, interleaved)
            assert [axes.count(a) for a in range(len(sections))] == sections


def test_chunk_mask_arguments():
    m = P.make_chunk_mask(sinks=4, window=100, layer=3, psaw_layer_start=2, psaw_phi=0.5, psaw_alpha=2.0)
    assert [getattr(m, f) for f, _ in P.ChunkMask._fields_] == [4, 100, 3, 2, 0.5, 2.0]


def test_host_tensors_and_wrong_counts_are_refused(lib):
    m, n = P._load_marshal(), None
    q, k, lens = torch.zeros(5, 6, 128, dtype=torch.bfloat16), torch.zeros(5, 2, 128, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int32)
    lse = torch.zeros(5, 6)
    calls = ((m.qkv_append, (0, 0, 0, q, k, k, q, n, n, 5, 6, 2, 1, 0, 0)), (m.bytekv_qkv_append, (0, 0, 0, q, k, k, q, lens, n, 5, 6, 2, 1, 0, 0)),
             (m.qkv_append, (0, 0, 0, n, n, n, n, n, n, 5, 6, 2, 1, 0, 0)), (m.bytekv_read, (0, 0, 0, lens, 0, 5, 0, 0)),
             (m.chunk_attn, (0, 0, 0, q, q, lse, n, 5, 6, 0, 0)), (m.chunk_attn, (0, 0, 0, n, n, n, n, 5, 6, 0, 0)))
    for f, args in calls:
        with pytest.raises(AssertionError):
            f(*args)                            # nothing there, or host tensors where device 0 is asked for
        with pytest.raises(TypeError):
            f(*args[:-1])
        with pytest.raises(TypeError):
            f(*args, n)
    with pytest.raises(TypeError):
        m.chunk_attn("ctx", 0, 0, q, q, lse, n, 5, 6, 0, 0)


def test_shapes_are_refused_before_the_call(lib):
    """On the host's 'device' (-1) the checks behind the types are reached; the context is NULL, so that a call that passes them all
    returns PRHS_ERR_INVALID_ARG (1)."""
    m, n = P._load_marshal(), None
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)   # noqa: E731
    q, k = z(5, 6, 128), z(5, 2, 128)
    append = lambda q=q, k=k, v=k, out=q, start=i32(4), pos=n, batch=3, axes=1: m.qkv_append(  # noqa: E731
        0, 0, 0, q, k, v, out, start, pos, batch, 6, 2, axes, -1, 0)
    assert append() == 1 and append(start=n, batch=5) == 1 and append(pos=i32(5)) == 1 and append(pos=i32(3, 9)[:, 2:7], axes=3) == 1
    for kw in (dict(q=z(5, 5, 128)), dict(k=z(4, 2, 128)), dict(v=z(5, 2, 64)), dict(out=z(6, 5, 128).transpose(0, 1)), dict(start=i32(3)), dict(start=n),
               dict(start=i32(8)[::2]), dict(pos=i32(4)), dict(pos=i32(1, 5), axes=2), dict(pos=i32(1, 10)[:, ::2]), dict(q=q.float()), dict(pos=torch.zeros(5))):
        with pytest.raises(AssertionError):
            append(**kw)
    lse = torch.zeros(5, 6)
    chunk = lambda q=q, out=q, lse=lse, start=i32(4), batch=3: m.chunk_attn(0, 0, 0, q, out, lse, start, batch, 6, -1, 0)  # noqa: E731
    assert chunk() == 1 and chunk(lse=n) == 1 and chunk(start=n, batch=5) == 1
    for kw in (dict(q=z(5, 6, 64)), dict(out=z(4, 6, 128)), dict(out=n), dict(lse=lse.double()), dict(lse=torch.zeros(6, 5).T), dict(start=i32(3)), dict(start=n)):
        with pytest.raises(AssertionError):
            chunk(**kw)
    assert m.bytekv_read(0, 0, 0, n, 0, 3, -1, 0) == 1 and m.bytekv_read(0, 0, 0, i32(3), 0, 3, -1, 0) == 1
    with pytest.raises(AssertionError):
        m.bytekv_read(0, 0, 0, i32(2), 0, 3, -1, 0)


NO_DATA = """
import torch
from paper_2602_08329_b200 import binding as P
m = P._load_marshal()
t, start, n = torch.zeros(4, 5, 6, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), None
k = torch.zeros(5, 2, 128, dtype=torch.bfloat16)
calls = {
    "append": lambda x: m.qkv_append(0, 0, 0, x, k, k, t[0], start, n, 3, 6, 2, 1, -1, 0),
    "append, starts": lambda x: m.bytekv_qkv_append(0, 0, 0, t[0], k, k, t[0], x[:4, 0, 0].to(torch.int32), n, 3, 6, 2, 1, -1, 0),
    "append, positions": lambda x: m.qkv_append(0, 0, 0, t[0], k, k, t[0], start, x[:, 0, 0].to(torch.int32), 3, 6, 2, 1, -1, 0),
    "read": lambda x: m.bytekv_read(0, 0, 0, x[:, 0, 0].to(torch.int32), 0, 3, -1, 0),
    "attend": lambda x: m.chunk_attn(0, 0, 0, x, t[0], n, start, 3, 6, -1, 0),
}
for name, call in calls.items():
    try:
        torch.vmap(lambda x: call(x) and x)(t)
    except RuntimeError as e:
        assert "storage" in str(e) or "data" in str(e), (name, e)
        print(name)
"""


def test_calls_with_tensors_that_have_no_data_raise(lib):
    res = subprocess.run([sys.executable, "-X", "faulthandler", "-c", NO_DATA], cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    assert res.stdout.split("\n")[:-1] == ["append", "append, starts", "append, positions", "read", "attend"]
