"""The cache's and attention's oracle against things other than itself."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv as O  # noqa: E402


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(1)
    x, pos, freq = rng.normal(size=(5, 2, 12)), [0, 1, 7, -3, 40], rng.uniform(0, 2, 4)
    y = O.rotate64(x, pos, freq, interleaved)
    a, b = (x[..., 0:8:2], x[..., 1:8:2]) if interleaved else (x[..., :4], x[..., 4:8])
    z = (a + 1j * b) * np.exp(1j * np.outer(pos, freq))[:, None]
    ya, yb = (y[..., 0:8:2], y[..., 1:8:2]) if interleaved else (y[..., :4], y[..., 4:8])
    assert np.allclose(ya, z.real) and np.allclose(yb, z.imag)
    assert (y[..., 8:] == x[..., 8:]).all() and (y[0] == x[0]).all()
    back = O.rotate64(y, pos, freq, interleaved, transpose=True)
    assert np.allclose(back, x)
    # what a swapped sign would give is something else
    assert not np.allclose(O.rotate64(x, pos, -freq, interleaved), y)


def test_scores_of_turned_rows_depend_on_their_distance():
    rng = np.random.default_rng(2)
    q, k, freq = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8)), [1.0, 0.3, 0.1, 0.01]
    dots = [float((O.rotate64(q, [p + 5], freq) * O.rotate64(k, [p], freq)).sum())
            for p in (0, 3, 1000)]
    assert np.allclose(dots, dots[0])


def test_e4m3_codes_are_those_of_torch():
    x = np.concatenate([np.linspace(-448, 448, 5001), np.linspace(-0.04, 0.04, 5001),
                        O.e4m3_values(), -O.e4m3_values()])
    mid = (O.e4m3_values()[1:] + O.e4m3_values()[:-1]) / 2          # ties
    x = np.concatenate([x, mid, -mid]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert (O.nearest_code(x.astype(np.float64), "e4m3") == want).all()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_codes_are_within_half_a_step_and_reach_the_largest(kind):
    x = np.random.default_rng(3).normal(size=(50, 16)).astype(np.float32)
    x[7], x[8, 3], x[9, 0] = 0, np.nan, np.inf
    codes, scale = O.quantise(x, kind)
    ok = np.isfinite(scale)
    assert list(np.flatnonzero(~ok)) == [8, 9] and scale[7] == 0 and (codes[7] == 0).all()
    err = np.abs(codes * scale[:, None] - x)[ok]
    step = scale[ok, None] * (0.5 if kind == "int8" else 1) * np.ones_like(err)
    if kind == "e4m3":          # half a step: 2^-4 of the value, or of the smallest normal
        step = np.maximum(np.abs(x[ok]) * 2.0 ** -4, scale[ok, None] * 2.0 ** -10)
    assert (err <= step * (1 + 1e-5)).all()
    full = ok.copy()
    full[7] = False
    assert (np.abs(codes[full]).max(1) == O.LARGEST[kind]).all()


def test_indices_enumerate_the_cache():
    heads, page, dim = 3, 32, 16
    for run in (8, 16):
        at = {O.value_index(s, h, d, heads, page, dim, run)
              for s in range(64) for h in range(heads) for d in range(dim)}
        assert at == set(range(64 * heads * dim))
        v = np.arange(2 * heads * page * dim).reshape(2, heads, page // run, dim, run)
        assert v[1, 2, 17 // run, 5, 17 % run] == O.value_index(32 + 17, 2, 5, heads, page, dim, run)
    k = np.arange(2 * heads * page * dim).reshape(2, heads, page, dim)
    assert k[1, 2, 17, 5] == O.key_index(32 + 17, 2, 5, heads, page, dim)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 2)])
def test_attention_equals_a_masked_softmax(causal, window):
    rng = np.random.default_rng(4)
    new, length, group = 5, 9, 2
    q, k, v = (rng.normal(size=(n, h, 8)) for n, h in ((new, 4), (length, 2), (length, 2)))
    out, lse, _ = O.attend64(q, k, v, new, length, causal, window)
    s = torch.einsum("ihd,jhd->hij", torch.from_numpy(q),
                     torch.from_numpy(k).repeat_interleave(group, 1)) / math.sqrt(8)
    p = torch.arange(length - new, length)[:, None]
    j = torch.arange(length)
    sees = ((j <= p) | (not causal)) & ((j > p - window) | (window == 0))
    s = s.masked_fill(~sees, -math.inf)
    want = torch.einsum("hij,jhd->ihd", s.softmax(-1),
                        torch.from_numpy(v).repeat_interleave(group, 1))
    assert np.allclose(out, want.numpy()) and np.allclose(lse.T, s.logsumexp(-1).numpy())


def test_rows_that_see_nothing():
    q = np.ones((3, 1, 8))
    kv = np.ones((2, 1, 8))
    out, lse, _ = O.attend64(q, kv, kv, 3, 2)       # more new tokens than cached ones
    assert (out[0] == 0).all() and lse[0, 0] == -np.inf and (out[1:] == 1).all()
