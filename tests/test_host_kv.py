"""Refusals of the rotary, cache and attention calls, and the frequencies: all on
the host, before any launch (stand-in device pointers are never dereferenced)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_02652_amd as P  # noqa: E402
from paper_2609_02652_amd import _lib  # noqa: E402

FAKE = 256
ARG, SHAPE = -1, -3


def cache(**kw):
    d = dict(type=_lib.INT8, heads=2, dim=64, page_size=32, pages=4, k=FAKE, v=FAKE, k_scale=FAKE,
             v_scale=FAKE)
    d.update(kw)
    return _lib.KVCacheDesc(*(d[n] for n, _ in _lib.KVCacheDesc._fields_))


def rows(data=FAKE, type=_lib.F16, token=128, head=64):
    return _lib.Rows(data, type, token, head)


def rotary(freq=FAKE, magnitude=1.0, width=64, interleaved=0):
    return _lib.RotaryDesc(freq, magnitude, width, interleaved)


def refused(code, fn, *args):
    with pytest.raises(P.LeechError) as e:
        fn(*args)
    assert e.value.code == code, _lib.lib.leech_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(type=_lib.F32), ARG), (dict(type=7), ARG), (dict(k=0), ARG), (dict(v=0), ARG),
    (dict(k_scale=0), ARG), (dict(v_scale=0), ARG), (dict(k=FAKE + 8), ARG),
    (dict(v_scale=FAKE + 2), ARG), (dict(heads=0), SHAPE), (dict(dim=0), SHAPE),
    (dict(dim=72), SHAPE), (dict(dim=272), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=48), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(pages=0), SHAPE),
    (dict(pages=1 << 31), SHAPE)])
def test_a_cache_that_is_not_one(kw, code):
    refused(code, _lib.check_cache, cache(**kw))


def test_no_cache_and_no_token():
    refused(ARG, _lib.check_cache, None)
    _lib.check_cache(cache())
    _lib.check_cache(cache(type=_lib.BF16, k_scale=0, v_scale=0))
    _lib.rope(0, 2, 64, rows(), FAKE, rotary(), False, rows())
    _lib.cache_write(cache(), 0, rows(), rows(), FAKE, None, None, 0, None, None)


@pytest.mark.parametrize("args,code", [
    ((-1, 2, 64, rows(), FAKE, rotary(), 0, rows()), SHAPE),
    ((4, 0, 64, rows(), FAKE, rotary(), 0, rows()), SHAPE),
    ((4, 2, 60, rows(), FAKE, rotary(), 0, rows()), SHAPE),
    ((4, 2, 264, rows(), FAKE, rotary(), 0, rows()), SHAPE),
    ((4, 2, 64, None, FAKE, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(0), FAKE, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(), None, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE + 4, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, None, 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(0), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(FAKE + 4), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(width=72), 0, rows()), SHAPE),
    ((4, 2, 64, rows(), FAKE, rotary(width=12), 0, rows()), SHAPE),
    ((4, 2, 64, rows(), FAKE, rotary(width=0), 0, rows()), SHAPE),
    ((4, 2, 64, rows(), FAKE, rotary(magnitude=0.0), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(magnitude=math.nan), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(interleaved=2), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(), 2, rows()), ARG),
    ((4, 2, 64, rows(FAKE + 1), FAKE, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(type=_lib.INT8), FAKE, rotary(), 0, rows()), ARG),
    ((4, 2, 64, rows(), FAKE, rotary(), 0, rows(token=64)), SHAPE),      # tokens share heads
    ((4, 2, 64, rows(), FAKE, rotary(), 0, rows(head=32)), SHAPE),
    ((4, 2, 64, rows(), FAKE, rotary(), 0, rows(token=0)), SHAPE),
    ((1 << 33, 16, 64, rows(), FAKE, rotary(), 0, rows(token=1024)), SHAPE)])   # a launch's threads
def test_rope_refuses(args, code):
    refused(code, _lib.rope, *args)


@pytest.mark.parametrize("args,code", [
    ((None, 4, rows(), rows(), FAKE, None, None, 0, None, None), ARG),
    ((cache(), -1, rows(), rows(), FAKE, None, None, 0, None, None), SHAPE),
    ((cache(), 4, None, rows(), FAKE, None, None, 0, None, None), ARG),
    ((cache(), 4, rows(), rows(0), FAKE, None, None, 0, None, None), ARG),
    ((cache(), 4, rows(), rows(type=_lib.F32), FAKE, None, None, 0, None, None), ARG),
    ((cache(), 4, rows(), rows(), FAKE, FAKE, rotary(), 2, rows(type=_lib.BF16), rows()), ARG),
    ((cache(), 4, rows(), rows(), None, None, None, 0, None, None), ARG),
    ((cache(), 4, rows(), rows(), FAKE, None, rotary(), 0, None, None), ARG),   # no positions
    ((cache(), 4, rows(), rows(), FAKE, None, None, 2, rows(), rows()), ARG),   # q without rotary
    ((cache(), 4, rows(), rows(), FAKE, FAKE, rotary(), -1, None, None), SHAPE),
    ((cache(), 4, rows(), rows(), FAKE, FAKE, rotary(), 2, rows(), None), ARG),
    ((cache(), 4, rows(), rows(), FAKE, FAKE, rotary(), 4, rows(), rows()), SHAPE),
    ((cache(), 4, rows(), rows(), FAKE, FAKE, rotary(width=128), 0, None, None), SHAPE)])
def test_cache_write_refuses(args, code):
    refused(code, _lib.cache_write, *args)


@pytest.mark.parametrize("args,code", [
    ((cache(), -1, FAKE, rows(), rows()), SHAPE), ((cache(), 4, None, rows(), rows()), ARG),
    ((cache(), 4, FAKE, rows(0), rows()), ARG), ((cache(), 4, FAKE, rows(), None), ARG),
    ((cache(), 4, FAKE, rows(), rows(token=64)), SHAPE),
    ((cache(), 4, FAKE, rows(type=_lib.E4M3), rows()), ARG),
    ((cache(), 4, FAKE, rows(type=_lib.BF16), rows()), ARG)])
def test_cache_read_refuses(args, code):
    refused(code, _lib.cache_read, *args)


def attend_args(**kw):
    d = dict(type=_lib.F16, q_heads=4, T=8, q=FAKE, q_token_stride=256, q_head_stride=64,
             out=FAKE, out_token_stride=256, out_head_stride=64, lse=None, B=2, q_start=FAKE,
             kv_len=FAKE, page_table=FAKE, table_stride=4, table_pages=4, max_new=8, causal=1,
             window=0, scale=0.125, workspace=None, workspace_bytes=0)
    d.update(kw)
    return _lib.AttendArgs(*(d[n] for n, _ in _lib.AttendArgs._fields_))


@pytest.mark.parametrize("kw,code", [
    (dict(type=_lib.F32), ARG), (dict(type=_lib.INT8), ARG), (dict(q_heads=3), SHAPE),
    (dict(q_heads=0), SHAPE), (dict(T=-1), SHAPE), (dict(T=1 << 31), SHAPE), (dict(B=-1), SHAPE),
    (dict(max_new=-1), SHAPE), (dict(table_pages=-1), SHAPE), (dict(table_pages=1 << 26), SHAPE),
    (dict(q_start=None), SHAPE), (dict(causal=2), ARG), (dict(window=-1), ARG),
    (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG), (dict(q=None), ARG),
    (dict(out=None), ARG), (dict(q=FAKE + 8), ARG), (dict(q_head_stride=60), ARG),
    (dict(out_token_stride=252), ARG), (dict(out_token_stride=128), SHAPE),
    (dict(out_head_stride=56), SHAPE), (dict(kv_len=None), ARG), (dict(page_table=None), ARG),
    (dict(kv_len=FAKE + 2), ARG), (dict(lse=FAKE + 1), ARG)])
def test_attend_refuses(kw, code):
    refused(code, _lib.attend, cache(), attend_args(**kw))


def test_attend_refuses_mixed_16_bit_types_and_no_arguments():
    refused(ARG, _lib.attend, cache(type=_lib.BF16), attend_args())
    refused(ARG, _lib.attend, cache(), None)
    refused(ARG, _lib.attend, None, attend_args())
    for kw in (dict(T=0), dict(B=0), dict(max_new=0)):      # nothing to do
        _lib.attend(cache(), attend_args(**kw))


def test_attend_refuses_a_workspace_that_is_too_small():
    args = attend_args(T=2, q_start=None, max_new=1, table_pages=1 << 16)
    need = _lib.attend_workspace(cache(), args)
    assert need > 0
    for p, n in ((None, need), (FAKE, need - 1), (FAKE + 4, need)):
        args.workspace, args.workspace_bytes = p, n
        refused(ARG, _lib.attend, cache(), args)


def test_the_python_calls_refuse_host_tensors_and_wrong_shapes():
    x = torch.zeros(2, 3, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        P.KVCache.empty(2, 32, 2, 64, torch.float16, "cpu")
    with pytest.raises(ValueError):
        P.KVCache.empty(2, 32, 2, 64, torch.float32, "cpu")
    with pytest.raises(ValueError):
        P.KVCache.empty(2, 12, 2, 64, torch.float16, "cpu")
    with pytest.raises(ValueError):
        P.Rotary(torch.zeros(32))
    r = P.Rotary(torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        P.rope(x, torch.zeros(2, dtype=torch.int64), r)


def test_frequencies():
    f, a = P.rotary_frequencies(8)
    assert a == 1.0 and np.allclose(f, [1, 0.1, 0.01, 0.001], rtol=1e-15)
    g, _ = P.rotary_frequencies(8, scaling="linear", factor=4.0)
    assert np.allclose(g * 4, f, rtol=1e-15)
    g, _ = P.rotary_frequencies(8, scaling="ntk", factor=4.0)
    assert g[0] == 1.0 and np.isclose(g[-1] * 4, f[-1]) and (np.diff(g * 4 / f) < 0).all()
    g, a = P.rotary_frequencies(8, scaling="parts", factor=4.0, original=2000, low=1, high=32)
    turns = 2000 * f / (2 * math.pi)
    assert turns[0] > 32 and g[0] == f[0] and turns[-1] < 1 and np.isclose(g[-1] * 4, f[-1])
    keep = (turns[1] - 1) / 31
    assert np.isclose(g[1], f[1] * (keep + (1 - keep) / 4)) and np.isclose(a, 1 + 0.1 * math.log(4))
    for bad in (dict(width=7), dict(width=0), dict(width=8, base=0.0), dict(width=8, factor=0.5),
                dict(width=8, scaling="x"), dict(width=8, scaling="parts", factor=2.0),
                dict(width=2, scaling="ntk", factor=2.0)):
        with pytest.raises(ValueError):
            P.rotary_frequencies(**bad)
