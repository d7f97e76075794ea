"""Host side of the attention calls (include/spconv_attention.h): the boundary, the
refusals (nothing is queued: every call here has a wrong argument), the rotary
frequencies and the rows of a batch. No GPU."""
import ctypes
import math
import re
from pathlib import Path

import numpy as np
import pytest
import torch

from paper_2005_04091_amd import attention as A

ROOT = Path(__file__).resolve().parent.parent
P = 4096  # an aligned address; nothing is read there


def test_header_binding_and_library_agree():
    text = (ROOT / "include" / "spconv_attention.h").read_text()
    declared = re.findall(r"^int\s+(spconv_\w+)\(", text, flags=re.M)
    assert sorted(declared) == sorted(A.EXPORTED)
    lib = ctypes.CDLL(str(A.spconv.LIB_PATH))
    for name in declared:
        assert hasattr(lib, name)
    assert ctypes.sizeof(A.spconv_batch) == 64 and ctypes.sizeof(A.spconv_rope_scaling) == 40


def batch(**kw):
    f = dict(sequences=2, block=64, max_blocks=8, q_block=1, tokens=10, pages=20, table_stride=8, table=P, kv_len=P, q_start=P)
    f.update(kw)
    return A.spconv_batch(*(f[n] for n, _ in A.spconv_batch._fields_))


BAD_BATCH = [dict(sequences=0), dict(block=0), dict(block=24), dict(block=272), dict(max_blocks=0), dict(max_blocks=1 << 25, table_stride=1 << 25),
             dict(q_block=0), dict(q_block=129), dict(tokens=0), dict(tokens=1 << 31), dict(pages=0), dict(pages=1 << 31),
             dict(table_stride=7), dict(q_start=None)]


def append(b, dtype=2, k=P, kt=1024, kh=128, v=P, vt=1024, vh=128, heads=8, dim=128, positions=None, freq=P, rot=128, flags=0,
           amplitude=1.0, kc=P, vc=P, sums=P):
    return A._lib.spconv_cache_append(dtype, b, k, kt, kh, v, vt, vh, heads, dim, positions, freq, rot, flags, amplitude, kc, vc,
                                      sums, None)


def scores(b, dtype=2, q=P, qt=4096, qh=128, q_heads=32, heads=8, dim=128, sums=P, out=P):
    return A._lib.spconv_block_scores(dtype, b, q, qt, qh, q_heads, heads, dim, sums, out, None)


def select(b, heads=8, s=P, keep=4, sink=1, local=1, blocks=P, counts=P):
    return A._lib.spconv_select_blocks(b, heads, s, keep, sink, local, blocks, counts, None)


def attend(b, dtype=2, q=P, qt=4096, qh=128, q_heads=32, heads=8, dim=128, kc=P, vc=P, scale=0.1, blocks=P, counts=P, keep=4, out=P,
           ot=4096, oh=128, lse=None, ws=P, size=1 << 40):
    return A._lib.spconv_block_attention(dtype, b, q, qt, qh, q_heads, heads, dim, kc, vc, scale, blocks, counts, keep, out, ot, oh,
                                         lse, ws, size, None)


@pytest.mark.parametrize("call", [append, scores, select, attend])
@pytest.mark.parametrize("bad", BAD_BATCH + [dict(table=None), dict(kv_len=None)], ids=str)
def test_bad_batches(call, bad):
    assert call(batch(**bad)) == A.SPCONV_EINVAL
    if "table" not in bad and "kv_len" not in bad:
        assert A._lib.spconv_batch_rows(batch(**bad), ctypes.c_int64()) == A.SPCONV_EINVAL


@pytest.mark.parametrize("call", [append, scores, select, attend])
def test_no_batch(call):
    assert call(None) == A.SPCONV_EINVAL
    assert A._lib.spconv_batch_rows(batch(), None) == A.SPCONV_EINVAL


def test_append_refusals():
    for bad in [dict(dtype=3), dict(dtype=-1), dict(k=None), dict(v=None), dict(kc=None), dict(vc=None), dict(heads=0),
                dict(heads=65536), dict(dim=0), dict(dim=12), dict(dim=264), dict(rot=-2), dict(rot=3), dict(rot=130), dict(freq=None),
                dict(rot=0), dict(flags=2), dict(flags=4), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(kt=-1),
                dict(kh=-1), dict(vt=-1), dict(vh=-1), dict(kc=P + 8), dict(vc=P + 4), dict(sums=P + 4)]:
        assert append(batch(), **bad) == A.SPCONV_EINVAL, bad


def test_scores_refusals():
    for bad in [dict(dtype=3), dict(q=None), dict(sums=None), dict(out=None), dict(q_heads=12), dict(q_heads=0), dict(heads=0),
                dict(q_heads=65536), dict(dim=100), dict(dim=264), dict(qt=-1), dict(qh=-1), dict(sums=P + 4)]:
        assert scores(batch(), **bad) == A.SPCONV_EINVAL, bad
    assert scores(batch(tokens=(1 << 31) - 1)) == A.SPCONV_EINVAL  # rows * heads


def test_select_refusals():
    for bad in [dict(heads=0), dict(heads=65536), dict(s=None), dict(blocks=None), dict(counts=None), dict(keep=0), dict(keep=1),
                dict(sink=-1), dict(local=-1), dict(sink=4)]:
        assert select(batch(), **bad) == A.SPCONV_EINVAL, bad
    # What is always listed: sink, local and the row's own blocks.
    assert select(batch(q_block=128, block=32), keep=5, sink=1, local=1) == A.SPCONV_EINVAL
    assert select(batch(tokens=(1 << 31) - 1)) == A.SPCONV_EINVAL


def test_attention_refusals():
    for bad in [dict(dtype=3), dict(q=None), dict(kc=None), dict(vc=None), dict(out=None), dict(q_heads=12), dict(heads=0), dict(dim=4),
                dict(dim=20), dict(dim=264), dict(qt=-1), dict(qh=-1), dict(ot=64), dict(oh=64), dict(ot=-4096), dict(kc=P + 8),
                dict(vc=P + 8), dict(scale=math.nan), dict(scale=math.inf), dict(keep=-1), dict(keep=0), dict(blocks=None),
                dict(blocks=None, keep=0), dict(ws=None, keep=64), dict(ws=P + 4, keep=64), dict(size=100, keep=64)]:
        assert attend(batch(), **bad) == A.SPCONV_EINVAL, bad
    assert attend(batch(tokens=(1 << 31) - 1)) == A.SPCONV_EINVAL


def test_workspace():
    n = ctypes.c_int64(-1)
    ask = lambda b, q_heads=32, heads=8, dim=128, keep=64, dtype=2: A._lib.spconv_attention_workspace(dtype, b, q_heads, heads, dim,
                                                                                                     keep, n)
    assert ask(batch()) == A.SPCONV_OK and n.value > 0  # ten rows: shares
    assert ask(batch(tokens=100000)) == A.SPCONV_OK and n.value == 0
    assert ask(batch(), keep=-1) == ask(batch(), q_heads=3) == ask(batch(), dtype=7) == ask(batch(block=8)) == A.SPCONV_EINVAL
    assert A._lib.spconv_attention_workspace(2, batch(), 32, 8, 128, 0, None) == A.SPCONV_EINVAL


def rope(dtype=2, x=P, xt=1024, xh=128, tokens=4, heads=8, dim=128, positions=P, freq=P, rot=128, flags=0, amplitude=1.0, out=2 * P,
         ot=1024, oh=128):
    return A._lib.spconv_rope(dtype, x, xt, xh, tokens, heads, dim, positions, freq, rot, flags, amplitude, out, ot, oh, None)


def test_rope_refusals():
    for bad in [dict(dtype=3), dict(x=None), dict(out=None), dict(positions=None), dict(freq=None), dict(tokens=0), dict(tokens=1 << 31),
                dict(heads=0), dict(heads=65536), dict(dim=0), dict(dim=1025), dict(rot=-2), dict(rot=7), dict(rot=130), dict(flags=4),
                dict(amplitude=math.inf), dict(xt=-1), dict(xh=-1), dict(ot=64), dict(oh=64), dict(out=P, ot=2048)]:
        assert rope(**bad) == A.SPCONV_EINVAL, bad


def test_frequencies():
    f = A.spconv_rope_frequencies(64, 10000.0)
    want = 10000.0 ** (-np.arange(0, 64, 2) / 64)
    assert np.allclose(f, want, rtol=1e-14, atol=0)
    assert np.allclose(A.spconv_rope_frequencies(64, 10000.0, dict(kind="linear", factor=4.0)), want / 4, rtol=1e-14, atol=0)
    g = A.spconv_rope_frequencies(64, 10000.0, dict(kind="base", factor=4.0))
    assert np.isclose(g[0], 1.0, rtol=1e-14) and np.isclose(g[-1], want[-1] / 4, rtol=1e-13)
    s = dict(kind="by_parts", factor=8.0, low=1.0, high=4.0, original=8192.0)
    h = A.spconv_rope_frequencies(64, 10000.0, s)
    for fi, w in zip(h, want):
        length = 2 * math.pi / w
        if length < 8192 / 4:
            v = w
        elif length > 8192:
            v = w / 8
        else:
            t = (8192 / length - 1.0) / 3.0
            v = (1 - t) * w / 8 + t * w
        assert math.isclose(fi, v, rel_tol=1e-13)
    assert np.allclose(h[:5], want[:5], rtol=1e-14) and np.allclose(h[-5:], want[-5:] / 8, rtol=1e-14)


@pytest.mark.parametrize("args", [
    (63, 10000.0, None), (0, 10000.0, None), (64, 0.0, None), (64, -1.0, None), (64, math.nan, None), (64, math.inf, None),
    (64, 10000.0, A.spconv_rope_scaling(9, 1.0)), (64, 10000.0, A.spconv_rope_scaling(-1, 1.0)),
    (64, 10000.0, dict(kind="linear", factor=0.5)), (64, 10000.0, dict(kind="linear", factor=math.nan)),
    (2, 10000.0, dict(kind="base", factor=2.0)), (64, 1e308, dict(kind="base", factor=1e300)),
    (64, 10000.0, dict(kind="by_parts", factor=2.0, low=0.0, high=4.0, original=8192)),
    (64, 10000.0, dict(kind="by_parts", factor=2.0, low=4.0, high=4.0, original=8192)),
    (64, 10000.0, dict(kind="by_parts", factor=2.0, low=1.0, high=math.inf, original=8192)),
    (64, 10000.0, dict(kind="by_parts", factor=2.0, low=1.0, high=4.0, original=0.0)),
], ids=str)
def test_frequency_refusals(args):
    with pytest.raises(A.SpconvError):
        A.spconv_rope_frequencies(*args)


def test_scaling_fields_are_known():
    with pytest.raises(ValueError):
        A.spconv_rope_frequencies(64, 1e4, dict(kind="other"))
    with pytest.raises(ValueError):
        A.spconv_rope_frequencies(64, 1e4, dict(kind="linear", factr=2.0))


def test_rows():
    n = ctypes.c_int64()
    for kw, want in [(dict(), 10), (dict(q_block=4), 10 // 4 + 2), (dict(q_block=128), 2), (dict(q_start=None, tokens=2), 2),
                     (dict(q_block=2, tokens=1, sequences=1), 1)]:
        assert A._lib.spconv_batch_rows(batch(**kw), n) == A.SPCONV_OK and n.value == want


def test_rows_hold_every_token():
    """The row formula: rows of different sequences never meet, and all lie below R."""
    from attention_oracle import Rows
    rng = np.random.default_rng(0)
    for _ in range(300):
        B, qb = int(rng.integers(1, 6)), int(rng.integers(1, 9))
        n = rng.integers(0, 20, B)
        start = np.concatenate([[0], np.cumsum(n)])
        tokens = max(int(start[-1]), 1) + int(rng.integers(0, 3))
        r = Rows(start, n + 1, tokens, qb)
        assert sum(len(t) for _, t, _ in r.of.values()) == start[-1]


def test_binding_refuses_host_tensors_and_wrong_types():
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(TypeError):
        A.CacheBatch(t, torch.ones(2, dtype=torch.int32), 16)
    x = torch.zeros(2, 4, 64)
    with pytest.raises(TypeError):
        A.spconv_rope(x, torch.zeros(2, dtype=torch.int32), torch.ones(32, dtype=torch.float64))
