"""GPU parity of rotary positions, the paged cache and the attention over it
against the f64 oracle, through the public Python API.

Tolerances, with u a type's half step (f16 2^-11, bf16 2^-8 ... 2^-9 of the value
rounded to nearest; f32 2^-24):
  rotation   f32 arithmetic: the reduced angle is off by less than 2^-22, the
             sine, cosine and the four products and sums by a few 2^-24: below
             2^-21 (|a| + |b|), then one rounding, u |y|.  The angle itself is an
             f64 product: the oracle's p·f is off by 2^-53 of it, the kernel's
             p·f·(1/2π) by 2^-53 for each product and for the constant, together
             2^-51 |p f| (which is 2^-11 at position 2^40, and nothing at 2^20)
  codes      half a step of the row's scale (e4m3: 2^-4 of the value or 2^-10 of
             the scale), and what the rotation was off by
  attention  the weights are rounded to q's type, u each: u Σ p |v| (a weight
             under f16's normal range is off by 2^-25 of the largest: with it
             2^-25 Σ over the tokens of the largest |v|; so too for bf16 queries over
             8-bit codes, whose weights, times the value's scale over the largest
             scale seen, are f16); a score's f32 error e_s
             = (dim + 8) 2^-24 Σ |q k| scale + 2^-21 moves out by 2 e_s Σ p |v|
             and lse by e_s; then one rounding of out.  A weight under f32's normal
             range (or out, 8 bits of exponent too) may be lost whole: 2^-126 for
             each token, times the largest |v|
"""
import math
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_02652_amd as P  # noqa: E402
from oracle import kv as O  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16,
         "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
PAIRS = [("f16", "f16"), ("bf16", "bf16"), ("f16", "int8"), ("bf16", "int8"), ("f16", "e4m3"),
         ("bf16", "e4m3")]


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    return torch.device("cuda:0")


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bits(t):
    """A tensor's bit patterns (copyable, comparable for every type and NaN)."""
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def numbers(rng, shape, name):
    return torch.from_numpy(rng.normal(size=shape).astype(np.float32)).to(TYPES[name])


# ------------------------------------------------------------------- rotation
def check_turned(y, x, pos, freq, out, magnitude=1.0, **how):
    """y against the oracle's rotation of x (f64 arrays)."""
    want = O.rotate64(x, pos, freq, magnitude=magnitude, **how)
    n = len(freq)
    bound = U[out] * np.abs(want) + (2.0 ** -25 if out == "f16" else 0)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if how.get("interleaved") else (i, i + n)
        near = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
        angle = np.abs(np.asarray(pos, np.float64) * freq[i])[:, None]
        bound[..., a] += near * (2.0 ** -21 + 2.0 ** -51 * angle)
        bound[..., b] += near * (2.0 ** -21 + 2.0 ** -51 * angle)
    far = float((np.abs(y - want) - bound).max())
    assert far <= 0, far
    return want


@pytest.mark.parametrize("T,heads,dim,rot,src,dst,inter,first", [
    (1, 1, 8, 8, "f32", "f32", False, 0), (1, 40, 128, 128, "f32", "f16", False, 8191),
    (3, 5, 64, 40, "f16", "bf16", True, -7), (7, 17, 256, 256, "bf16", "f32", True, 1 << 40),
    (255, 3, 72, 64, "f32", "bf16", False, 1_000_000), (256, 9, 128, 64, "bf16", "bf16", True, 5),
    (300, 2, 136, 136, "f16", "f16", False, 99), (513, 16, 64, 64, "f16", "f32", False, 0)])
def test_rope(dev, T, heads, dim, rot, src, dst, inter, first):
    say(f"[rope] T={T} heads={heads} dim={dim} rot={rot} {src}->{dst} interleaved={inter}")
    rng = np.random.default_rng(T + dim)
    x = numbers(rng, (T, heads, dim), src).to(dev)
    freq, _ = P.rotary_frequencies(rot)
    pos = first + torch.arange(T)
    r = P.Rotary(torch.from_numpy(freq).to(dev), inter, 1.25)
    y = P.rope(x, pos.to(dev), r, dtype=TYPES[dst])
    back = P.rope(x, pos.to(dev), r, dtype=TYPES[dst], transpose=True)
    torch.cuda.synchronize()
    how = dict(interleaved=inter)
    check_turned(f64(y), f64(x), pos.tolist(), freq, dst, 1.25, **how)
    check_turned(f64(back), f64(x), pos.tolist(), freq, dst, 1.25, transpose=True, **how)


def test_rope_strides_alignment_and_in_place(dev):
    rng = np.random.default_rng(5)
    freq, _ = P.rotary_frequencies(48)
    r = P.Rotary(torch.from_numpy(freq).to(dev))
    pos = torch.arange(9).to(dev) * 11
    for src in ("f32", "f16"):
        for offset, pitch in ((0, 200), (1, 203), (2, 202)):
            buf = numbers(rng, (9 * pitch + offset,), src).to(dev)
            x = buf.as_strided((9, 2, 64), (pitch, 80, 1), offset)
            before = buf.clone()
            want = check_turned(f64(P.rope(x, pos, r)), f64(x), pos.tolist(), freq, src)
            P.rope(x, pos, r, out=x)
            torch.cuda.synchronize()
            assert np.allclose(f64(x), want, atol=2e-2)
            outside = torch.ones(buf.shape, dtype=torch.bool)
            outside.as_strided((9, 2, 64), (pitch, 80, 1), offset)[:] = False
            assert (bits(buf.cpu())[outside] == bits(before.cpu())[outside]).all()
    # heads ahead of tokens: a transposed view
    x = numbers(rng, (3, 9, 64), "f32").to(dev).transpose(0, 1)
    check_turned(f64(P.rope(x, pos, r)), f64(x), pos.tolist(), freq, "f32")


def test_rope_gradient_is_the_transposed_turn(dev):
    """<g, R x> = <Rᵀ g, x>, and a difference quotient agrees (R is linear: its
    step is exact up to rounding)."""
    rng = np.random.default_rng(6)
    x, g, e = (numbers(rng, (4, 3, 64), "f32").to(dev) for _ in range(3))
    pos = torch.tensor([0, 3, 1000, 123_456]).to(dev)
    r = P.Rotary.of(64, device=dev, scaling="parts", factor=8.0, original=4096)
    grad = P.rope(g, pos, r, transpose=True)
    moved = (f64(P.rope(x + e, pos, r)) - f64(P.rope(x, pos, r)))
    lhs, rhs = (f64(g) * moved).sum(), (f64(grad) * f64(e)).sum()
    # 768 products of numbers of size ~1, each off by a few 2^-22
    assert abs(lhs - rhs) <= 768 * 2.0 ** -19
    back = P.rope(P.rope(x, pos, r), pos, r, transpose=True)
    assert np.abs(f64(back) - r.magnitude ** 2 * f64(x)).max() <= 2.0 ** -18


# ---------------------------------------------------------------------- cache
def sentinel(cache):
    """Patterns that a call must leave where it does not write: NaN numbers, odd
    codes, NaN scales."""
    for t in (cache.k, cache.v):
        bits(t).fill_(0x7F if t.element_size() == 1 else 0x7FC1)
    for t in (cache.k_scale, cache.v_scale):
        if t is not None:
            t.fill_(math.nan)
    return [bits(t).clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)
            if t is not None]


def rows_in_cache(cache, slots):
    """k and v element values and scales of slots, by the oracle's indices."""
    h, page, dim, run = cache.heads, cache.page_size, cache.dim, cache.v.shape[-1]
    s, hh, d = np.meshgrid(slots, np.arange(h), np.arange(dim), indexing="ij")
    ki = O.key_index(s, hh, d, h, page, dim)
    vi = O.value_index(s, hh, d, h, page, dim, run)
    si = (s[..., 0] // page * h + hh[..., 0]) * page + s[..., 0] % page
    k, v = (bits(t).reshape(-1)[torch.from_numpy(i).to(t.device)].view(t.dtype)
            for t, i in ((cache.k, ki), (cache.v, vi)))
    scales = [None if t is None else t.reshape(-1).cpu().numpy()[si]
              for t in (cache.k_scale, cache.v_scale)]
    return f64(k), f64(v), scales, (ki, vi, si)


def slots_of(kind, T, page, pages, rng):
    if kind == "run":                       # consecutive places from inside a page
        start = page // 2 + 3
        order = rng.permutation(pages)
        at = start + np.arange(T)
        return order[at // page] * page + at % page
    s = rng.permutation(pages * page)[:T].astype(np.int64)
    if kind == "holes" and T > 2:           # rows of a padded batch, and out of range
        s[1::3] = -1
        s[2::7] = pages * page + 5
    return s


@pytest.mark.parametrize("cache_type", ["f16", "bf16", "int8", "e4m3"])
@pytest.mark.parametrize("T,q_heads,heads,dim,page,src,kind", [
    (1, 5, 1, 128, 16, "f32", "any"), (7, 8, 2, 64, 32, "f16", "holes"),
    (50, 3, 3, 16, 64, "bf16", "run"), (64, 4, 2, 256, 16, "f32", "holes"),
    (300, 6, 2, 80, 32, "f32", "run"), (271, 2, 1, 128, 128, "bf16", "holes"),
    (259, 2, 2, 192, 16, "f16", "run")])
def test_cache_write_and_read(dev, cache_type, T, q_heads, heads, dim, page, src, kind):
    say(f"[cache] {cache_type} T={T} {q_heads}/{heads}x{dim} page={page} {src} {kind}")
    rng = np.random.default_rng(T + dim)
    pages = -(-T // page) + 3
    slots = slots_of(kind, T, page, pages, rng)
    live = np.flatnonzero((slots >= 0) & (slots < pages * page))
    x = numbers(rng, (T, (q_heads + 2 * heads), dim), src)
    x[live[-1], -1] = 0                     # a row of zeros (the last value head)
    xd = x.to(dev)
    q, k, v = xd[:, :q_heads], xd[:, q_heads:q_heads + heads], xd[:, q_heads + heads:]
    freq, _ = P.rotary_frequencies(dim // 2 // 8 * 8)
    pos = torch.from_numpy(rng.integers(0, 100_000, T))
    r = P.Rotary(torch.from_numpy(freq).to(dev), interleaved=page > 16)
    cache = P.KVCache.empty(pages, page, heads, dim, TYPES[cache_type], dev)
    at = torch.from_numpy(slots).to(dev)

    # without a rotary the format is defined to the bit
    before = sentinel(cache)
    assert cache.write(k, v, at) is None
    torch.cuda.synchronize()
    gk, gv, scales, index = rows_in_cache(cache, slots[live])
    for got, want, scale in ((gk, k, scales[0]), (gv, v, scales[1])):
        want = want.cpu()[torch.from_numpy(live)].float().numpy()
        if scale is None:
            assert (got == f64(torch.from_numpy(want).to(TYPES[cache_type]))).all()
        else:
            codes, s = O.quantise(want, cache_type)
            assert (s == scale).all() and (got == codes).all()
    # everything else stays
    after = [bits(t) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    for a, b, i in zip(after, before, index[:2] + (index[2],) * 2):
        same = (a == b).reshape(-1).cpu()
        same[torch.from_numpy(i.reshape(-1))] = True
        assert same.all()

    # read back, and with a rotary
    for dst in ("f32", "f16", "bf16"):
        rk, rv = cache.read(at, dtype=TYPES[dst])
        torch.cuda.synchronize()
        for got, code, scale in ((rk, gk, scales[0]), (rv, gv, scales[1])):
            want = code if scale is None else code * scale.astype(np.float64)[..., None]
            want = torch.from_numpy(want).to(torch.float32)     # (code · scale rounded once is
            assert (f64(got)[live] == f64(want.to(TYPES[dst]))).all() or dst != "f32" and \
                (np.abs(f64(got)[live] - want.double().numpy()) <= U[dst] * np.abs(want.double().numpy())
                 + 2.0 ** -25).all()                              # within half a step of it)
            gone = np.setdiff1d(np.arange(T), live)
            assert (f64(got)[gone] == 0).all()

    out = cache.write(k, v, at, r, pos.to(dev), q, dtype=torch.float16)
    torch.cuda.synchronize()
    how = dict(interleaved=r.interleaved)
    check_turned(f64(out), f64(q), pos.tolist(), freq, "f16", **how)
    tk, tv, tscales, _ = rows_in_cache(cache, slots[live])
    assert (tv == gv).all()
    xk = f64(k)[live]
    if tscales[0] is None:
        check_turned(tk, xk, pos.numpy()[live].tolist(), freq, cache_type, **how)
        return
    want = O.rotate64(xk, pos.numpy()[live].tolist(), freq, **how)
    scale = tscales[0].astype(np.float64)[..., None]
    off = 2.0 ** -20 * np.abs(xk).max(-1, keepdims=True)
    half = 0.5 * scale if cache_type == "int8" else np.maximum(np.abs(want) * 2.0 ** -4,
                                                              scale * 2.0 ** -10)
    assert (np.abs(tk * scale - want) <= half * (1 + 2.0 ** -20) + off).all()


@pytest.mark.parametrize("cache_type", ["f16", "int8", "e4m3"])
def test_numbers_that_are_not_finite_stay_in_their_rows(dev, cache_type):
    x = numbers(np.random.default_rng(8), (40, 2, 32), "f32")
    x[3, 0, 5], x[20, 1, 0], x[21, 0, 31] = math.nan, math.inf, -math.inf
    cache = P.KVCache.empty(3, 16, 2, 32, TYPES[cache_type], dev)
    at = torch.arange(40).to(dev) + 1
    cache.write(x.to(dev), x.to(dev), at)
    for got in cache.read(at, dtype=torch.float32):
        bad = ~torch.isfinite(got.cpu())
        rows = bad.any(-1).nonzero().tolist()
        assert rows == [[3, 0], [20, 1], [21, 0]]
        if cache_type == "f16":
            assert bad.sum() == 3
        else:
            assert torch.isnan(got[3, 0]).all() and torch.isnan(got[20, 1]).all()


def test_tiny_rows_keep_their_size(dev):
    """Scales below f32's normal range, and rows that vanish in the scale."""
    x = torch.zeros(4, 1, 16)
    x[0, 0, :3] = torch.tensor([1e-38, -5e-39, 1e-40])
    x[1, 0, :2] = torch.tensor([3e-43, -1e-43])
    x[2, 0, 0] = 1e-45
    x[3, 0, :2] = torch.tensor([3e38, -1e38])
    for kind in ("int8", "e4m3"):
        cache = P.KVCache.empty(1, 16, 1, 16, TYPES[kind], dev)
        at = torch.arange(4).to(dev)
        cache.write(x.to(dev), x.to(dev), at)
        codes, scale = O.quantise(x.numpy(), kind)
        k, v, scales, _ = rows_in_cache(cache, np.arange(4))
        assert (k == codes).all() and (v == codes).all()
        assert (scales[0] == scale).all() and (scales[1] == scale).all()


# ------------------------------------------------------------------ attention
class Batch:
    """Sequences over a cache of random pages; every place that no token fills
    holds NaN (or a NaN scale and NaN codes)."""

    def __init__(self, dev, seed, lens, q_heads, heads, dim, page, q_type, cache_type, spare=0,
                 sharp=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.dim = lens, dim
        used = [-(-length // page) for _, length in lens]
        self.cache = P.KVCache.empty(sum(used) + 2, page, heads, dim, TYPES[cache_type], dev)
        sentinel(self.cache)
        order = rng.permutation(sum(used) + 2)
        width = max(used) + spare
        table = np.full((len(lens), max(width, 1)), -1, np.int32)
        at, self.kv, slots = 0, [], []
        for b, (_, length) in enumerate(lens):
            table[b, :used[b]] = order[at:at + used[b]]
            at += used[b]
            j = np.arange(length)
            slots.append(table[b][j // page].astype(np.int64) * page + j % page)
            self.kv.append([numbers(rng, (length, heads, dim), "f32") for _ in range(2)])
        self.slots = slots
        self.put(range(len(lens)))
        self.table = torch.from_numpy(table).to(dev)
        self.kv_len = torch.tensor([n for _, n in lens], dtype=torch.int32, device=dev)
        starts = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
        self.starts, self.q_start = starts, torch.from_numpy(starts.astype(np.int32)).to(dev)
        self.max_new = max(n for n, _ in lens)
        self.q = (sharp * numbers(rng, (int(starts[-1]), q_heads, dim), "f32")).to(
            TYPES[q_type]).to(dev)

    def put(self, which):
        for b in which:
            if len(self.slots[b]):
                k, v = (t.to(self.cache.device) for t in self.kv[b])
                self.cache.write(k, v, torch.from_numpy(self.slots[b]).to(self.cache.device))

    def attend(self, **kw):
        a = dict(q_start=self.q_start, max_new=self.max_new)
        a.update(kw)
        return self.cache.attend(self.q, self.table, self.kv_len, **a)

    def values(self, b):
        """What the cache stands for: k, v in f64."""
        k, v, scales, _ = rows_in_cache(self.cache, self.slots[b])
        if scales[0] is not None:
            k, v = (x * s.astype(np.float64)[..., None] for x, s in zip((k, v), scales))
        return k, v

    def check(self, out, lse=None, causal=True, window=0, scale=None):
        kind = "f16" if self.q.dtype == torch.float16 else "bf16"
        out, worst = f64(out), 0.0
        lse = None if lse is None else f64(lse)
        factor = self.dim ** -0.5 if scale is None else scale
        for b, (new, length) in enumerate(self.lens):
            if new == 0:
                continue
            rows = slice(self.starts[b], self.starts[b + 1])
            q = f64(self.q[rows])
            if length == 0:
                assert (out[rows] == 0).all()
                assert lse is None or (lse[rows] == -np.inf).all()
                continue
            k, v = self.values(b)
            want, want_lse, w = O.attend64(q, k, v, new, length, causal, window, scale)
            group = q.shape[1] // k.shape[1]
            for h in range(q.shape[1]):
                kh = k[:, h // group]
                av = w[:, h] @ np.abs(v[:, h // group])
                es = (self.dim + 8) * 2.0 ** -24 * abs(factor) * (
                    np.abs(q[:, h]) @ np.abs(kh).T).max(1) + 2.0 ** -21
                bound = (U[kind] + 2 * es)[:, None] * av + U[kind] * np.abs(want[:, h])
                bound += (length + 1) * 2.0 ** -126 * (1 + np.abs(v[:, h // group]).max())
                if kind == "f16" or self.cache.k_scale is not None:
                    bound += 2.0 ** -25 * ((w[:, h] > 0).sum(1) / np.maximum(
                        (w[:, h] / w[:, h].max(1, keepdims=True).clip(1e-300)).sum(1), 1.0)
                        * np.abs(v[:, h // group]).max())[:, None] + 2.0 ** -25
                err = np.abs(out[rows, h] - want[:, h])
                assert (err <= bound).all(), (b, h, float((err - bound).max()))
                worst = max(worst, float((err / np.maximum(bound, 1e-30)).max()))
                if lse is not None:
                    got, ref = lse[rows, h], want_lse[:, h]
                    gone = ref == -np.inf
                    assert (got[gone] == -np.inf).all()
                    got, ref, es = got[~gone], ref[~gone], es[~gone]
                    assert (np.abs(got - ref) <= es + 2.0 ** -21 * (1 + np.abs(ref))).all()
        say(f"    largest error / bound {worst:.2f}")


MIXES = {
    "decode": [(1, n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 700, 0, 1500)],
    "few": [(5, 5), (3, 200), (1, 64), (0, 50), (4, 2), (2, 0), (7, 129), (1, 1)],
    "chunks": [(100, 100), (37, 300), (1, 1), (130, 131), (2, 900), (64, 64), (0, 0)],
    "long": [(1, 9000), (2, 4111), (1, 17)],
}


@pytest.mark.parametrize("q_type,cache_type", PAIRS)
@pytest.mark.parametrize("mix,q_heads,heads,dim,page", [
    ("decode", 8, 2, 128, 64), ("few", 10, 2, 128, 16), ("chunks", 8, 2, 128, 32),
    ("long", 4, 1, 64, 128)])
def test_attend(dev, mix, q_heads, heads, dim, page, q_type, cache_type):
    say(f"[attend] {mix} {q_heads}/{heads}x{dim} page={page} {q_type} over {cache_type}")
    b = Batch(dev, 11, MIXES[mix], q_heads, heads, dim, page, q_type, cache_type, sharp=2.0)
    out, lse = b.attend(with_lse=True)
    torch.cuda.synchronize()
    b.check(out, lse)


@pytest.mark.parametrize("cache_type", ["f16", "int8"])
@pytest.mark.parametrize("q_heads,heads,dim", [(1, 1, 16), (3, 3, 48), (40, 1, 64), (12, 4, 80),
                                               (7, 1, 96), (16, 2, 112), (6, 2, 192), (8, 1, 256)])
def test_attend_head_layouts(dev, q_heads, heads, dim, cache_type):
    say(f"[attend] heads {q_heads}/{heads}x{dim} over {cache_type}")
    for lens in ([(1, 77), (3, 40), (1, 333)], [(90, 200), (20, 20)]):
        b = Batch(dev, 12, lens, q_heads, heads, dim, 16, "f16", cache_type)
        out, lse = b.attend(with_lse=True)
        torch.cuda.synchronize()
        b.check(out, lse)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 33), (False, 50),
                                           (True, 100_000)])
@pytest.mark.parametrize("mix", ["few", "chunks", "long"])
def test_attend_masks(dev, mix, causal, window):
    say(f"[attend] {mix} causal={causal} window={window}")
    b = Batch(dev, 13, MIXES[mix], 6, 2, 64, 32, "bf16", "e4m3", spare=3)
    out, lse = b.attend(causal=causal, window=window, with_lse=True, scale=0.3)
    torch.cuda.synchronize()
    b.check(out, lse, causal, window, 0.3)


def test_attend_scores_far_apart(dev):
    """Maxima that grow along the keys by more than a type's range, both ways, a
    negative scale, and one that makes all scores equal."""
    for q_type, cache_type in (("f16", "f16"), ("bf16", "int8")):
        for lens in ([(1, 700), (2, 65)], [(80, 300)]):
            b = Batch(dev, 14, lens, 4, 2, 64, 16, q_type, cache_type)
            for k, _ in b.kv:
                n = k.shape[0]
                k *= torch.linspace(0.01, 20, n)[:, None, None]
            b.put(range(len(lens)))
            for scale in (1.0, -1.0, 0.0, 1e-30):
                out, lse = b.attend(with_lse=True, scale=scale)
                torch.cuda.synchronize()
                b.check(out, lse, scale=scale)


@pytest.mark.parametrize("new", [1, 70])
def test_value_scales_far_apart(dev, new):
    """Value rows whose 8-bit scales differ by many powers of two, zero rows too."""
    b = Batch(dev, 15, [(new, 400)], 4, 2, 64, 16, "f16", "int8")
    _, v = b.kv[0]
    v *= torch.logspace(-6, 4, 400)[torch.randperm(400, generator=torch.Generator().manual_seed(1))][
        :, None, None]
    v[::9] = 0
    b.put([0])
    out = b.attend()
    torch.cuda.synchronize()
    b.check(out)


@pytest.mark.parametrize("cache_type", ["f16", "int8"])
@pytest.mark.parametrize("q_heads,lens", [(2, [(6, 50), (1, 40)]), (8, [(90, 150), (1, 40)])])
def test_numbers_that_are_not_finite_reach_only_rows_that_see_them(dev, cache_type, q_heads, lens):
    """A NaN or infinity in a key or value behind a row's mask does not reach it."""
    new, length = lens[0]
    b = Batch(dev, 16, lens, q_heads, 2, 64, 16, "f16", cache_type)
    clean = f64(b.attend())
    for part, bad in ((0, math.nan), (1, math.nan), (1, math.inf), (0, -math.inf)):
        token = length - 3                       # seen by the last three queries only
        saved = b.kv[0][part][token].clone()
        b.kv[0][part][token, 0, 5] = bad
        b.put([0])
        out = f64(b.attend())
        group = q_heads // 2
        assert (out[:new - 3] == clean[:new - 3]).all()
        assert (out[:, group:] == clean[:, group:]).all()           # the other head
        assert (out[new:] == clean[new:]).all()                     # the other sequence
        seen = out[new - 3:new, :group]
        if not (part == 0 and math.isinf(bad)):
            assert (~np.isfinite(seen)).any(-1).all()
        b.kv[0][part][token] = saved
        b.put([0])
        # a window that ends before a token hides it as well
        early = length - new
        b.kv[0][part][early] = bad
        b.put([0])
        w = f64(b.attend(window=2))
        assert np.isfinite(w[2:new]).all()
        b.kv[0][part][early] = b.kv[1][part][0]
        b.put([0])
        clean = f64(b.attend())


def test_bad_pages_lengths_and_starts_stay_in_bounds(dev):
    b = Batch(dev, 17, [(1, 100), (2, 90), (1, 30)], 4, 2, 64, 16, "bf16", "bf16")
    good = f64(b.attend())
    b.table[1, 3] = 1 << 30                      # places 48..63 of the second sequence
    b.table[0, 2] = -5
    out = f64(b.attend())
    assert np.isnan(out[0]).all() and np.isnan(out[1:3]).all() and (out[3] == good[3]).all()
    out = f64(b.attend(window=20))               # neither page is seen now
    assert np.isfinite(out).all()
    b = Batch(dev, 17, [(1, 100), (2, 90), (1, 30)], 4, 2, 64, 16, "bf16", "bf16")
    b.kv_len[0] = 1 << 30                        # longer than the table: all of the table's places
    b.kv_len[2] = -4
    out, lse = b.attend(with_lse=True)
    assert (f64(out)[1:3] == good[1:3]).all() and (f64(out)[3] == 0).all()
    assert (f64(lse)[3] == -np.inf).all()
    keep = torch.full_like(b.q, 7.0)
    b.q_start[:] = torch.tensor([-3, 1, 1 << 30, 2], dtype=torch.int32)
    b.attend(out=keep)
    torch.cuda.synchronize()


@pytest.mark.parametrize("cache_type", ["bf16", "e4m3"])
def test_bad_pages_of_a_chunk(dev, cache_type):
    """Many rows: only those that see a place of the missing page become NaN."""
    b = Batch(dev, 30, [(80, 200), (70, 180)], 4, 2, 64, 16, "bf16", cache_type)
    good = f64(b.attend())
    b.table[0, 9] = b.cache.pages                # places 144..159: position 144 is row 24
    out = f64(b.attend())
    assert (out[:24] == good[:24]).all() and (out[80:] == good[80:]).all()
    assert np.isnan(out[24:80]).all()
    out = f64(b.attend(window=30))               # rows from position 189 on do not see 159
    assert np.isnan(out[24:69]).all() and np.isfinite(out[69:]).all()


@pytest.mark.parametrize("new", [2, 60])
def test_scales_and_codes_that_are_no_numbers(dev, new):
    """In the cache itself: a NaN code, an infinite or NaN scale of a key or a value."""
    length = 100
    for kind in ("int8", "e4m3"):
        b = Batch(dev, 31, [(new, length), (1, 30)], 4, 2, 64, 16, "f16", kind)
        clean = f64(b.attend())
        slot = int(b.slots[0][length - 1])       # the last token: seen by the last row
        page, place = slot // 16, slot % 16
        for part, bad in (("k_scale", math.nan), ("v_scale", math.nan), ("v_scale", math.inf),
                          ("k", None), ("v", None)):
            if bad is None and kind == "int8":
                continue
            t = getattr(b.cache, part)
            saved = t.clone() if bad is not None else bits(t).clone()
            if bad is not None:
                t[page, 0, place] = bad
            elif part == "k":
                bits(t)[page, 0, place, 7] = 0x7F
            else:
                bits(t)[page, 0, 0, 7, place] = 0xFF
            out = f64(b.attend())
            assert (out[:new - 1] == clean[:new - 1]).all(), (kind, part, bad)
            assert (out[new:] == clean[new:]).all() and (out[:, 2:] == clean[:, 2:]).all()
            assert (~np.isfinite(out[new - 1, :2])).any(-1).all(), (kind, part, bad)
            if bad is not None:
                t.copy_(saved)
            else:
                bits(t).copy_(saved)


@pytest.mark.parametrize("q_type,cache_type", [("f16", "f16"), ("bf16", "int8"), ("f16", "e4m3")])
@pytest.mark.parametrize("dim,window", [(64, 0), (128, 700), (192, 0)])
def test_chunks_over_long_contexts_split(dev, dim, window, q_type, cache_type):
    """Many rows whose keys are split over workgroups and joined."""
    b = Batch(dev, 32, [(41, 2500), (9, 1300), (33, 3001)], 4, 1, dim, 32, q_type, cache_type)
    out, lse = b.attend(window=window, with_lse=True)
    torch.cuda.synchronize()
    b.check(out, lse, window=window)


def test_rows_of_no_sequence_are_left_alone(dev):
    for lens, q_heads in (([(2, 40), (1, 9)], 4), ([(60, 80), (30, 30)], 8)):
        b = Batch(dev, 18, lens, q_heads, 2, 64, 16, "f16", "f16")
        n = b.q.shape[0]
        want = b.attend()
        q = torch.cat([torch.ones_like(b.q[:1].expand(3, -1, -1)), b.q,
                       torch.ones_like(b.q[:1].expand(5, -1, -1))])
        out = torch.full((n + 8, q_heads, 72), 3.0, dtype=torch.float16, device=dev)[..., :64]
        b.cache.attend(q, b.table, b.kv_len, q_start=b.q_start + 3, max_new=b.max_new, out=out)
        assert (out[3:3 + n] == want).all()
        assert (out[:3] == 3).all() and (out[3 + n:] == 3).all()
        # rows past max_new too
        out = torch.full_like(b.q, 3.0)
        b.attend(max_new=1, out=out)
        for s, e in zip(b.starts[:-1], b.starts[1:]):
            assert (out[s] == want[s]).all() or e == s
            assert (out[s + 1:e] == 3).all()


def test_strided_queries_and_outputs(dev):
    b = Batch(dev, 19, MIXES["few"], 6, 2, 64, 16, "bf16", "bf16")
    want = b.attend()
    T = b.q.shape[0]
    wide = torch.full((T, 6 * 64 + 128), 9.0, dtype=torch.bfloat16, device=dev)
    q = torch.empty((6, T, 64), dtype=torch.bfloat16, device=dev).transpose(0, 1)
    q.copy_(b.q)
    out = wide[:, 8:8 + 384].view(T, 6, 64)
    b.cache.attend(q, b.table, b.kv_len, q_start=b.q_start, max_new=b.max_new, out=out)
    live = torch.ones(T, dtype=torch.bool)
    assert (out[live] == want[live]).all()
    assert (wide[:, :8] == 9).all() and (wide[:, 392:] == 9).all()


def test_one_new_token_a_sequence_needs_no_starts(dev):
    b = Batch(dev, 20, MIXES["decode"], 8, 2, 128, 64, "f16", "e4m3")
    want = b.attend()
    got = b.cache.attend(b.q, b.table, b.kv_len)
    assert (got == want).all()
    b.check(b.cache.attend(b.q, b.table, b.kv_len, q_start=b.q_start))


def test_empty_batches(dev):
    b = Batch(dev, 21, [(1, 20)], 4, 2, 64, 16, "f16", "f16")
    none = torch.zeros((0, 3), dtype=torch.int32, device=dev)
    out = b.cache.attend(b.q[:0], none, b.kv_len[:0])
    assert out.shape == (0, 4, 64)
    zero = torch.zeros(2, dtype=torch.int32, device=dev)
    b.cache.attend(b.q[:0], b.table, b.kv_len, q_start=zero)
    k, v = b.cache.read(torch.zeros(0, dtype=torch.int64, device=dev))
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)


def test_a_captured_step_replays_with_new_lengths(dev):
    """write (turning q) and attend captured once; positions, slots, lengths and
    numbers change between replays, with eager work beside."""
    lens = [(1, 100), (1, 600), (1, 31)]
    b = Batch(dev, 22, [(1, 730)] * 3, 4, 2, 64, 16, "f16", "int8")
    r = P.Rotary.of(64, device=dev)
    x = torch.zeros(3, 8, 64, device=dev)
    pos = torch.zeros(3, dtype=torch.int64, device=dev)
    slots = torch.full((3,), -1, dtype=torch.int64, device=dev)
    out = torch.zeros(3, 4, 64, dtype=torch.float16, device=dev)

    def step(o):
        q = b.cache.write(x[:, 4:6], x[:, 6:], slots, r, pos, x[:, :4], dtype=torch.float16)
        b.cache.attend(q, b.table, b.kv_len, out=o)
        return q

    step(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out)
    rng = np.random.default_rng(3)
    for turn in range(4):
        x.copy_(torch.from_numpy(rng.normal(size=(3, 8, 64)).astype(np.float32)))
        now = [n + 40 * turn for _, n in lens]
        pos.copy_(torch.tensor([n - 1 for n in now]))
        slots.copy_(torch.tensor([int(b.slots[i][n - 1]) for i, n in enumerate(now)]))
        b.kv_len.copy_(torch.tensor(now, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        eager = torch.zeros_like(out)
        b.q = step(eager)
        torch.cuda.synchronize()
        assert (out == eager).all()
        b.lens = [(1, n) for n in now]
        saved = b.slots
        b.slots = [s[:n] for s, n in zip(b.slots, now)]
        b.check(out)
        b.slots = saved


@pytest.mark.parametrize("cache_type", ["bf16", "e4m3"])
def test_a_captured_prompt_replays(dev, cache_type):
    """Chunks of many rows (LDS above 64 KiB) and of few in one captured call, with
    other lengths and starts on replay."""
    b = Batch(dev, 26, [(150, 400), (2, 300), (1, 90)], 8, 2, 128, 32, "bf16", cache_type)
    out = torch.zeros_like(b.q)
    b.attend(out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.attend(out=out)
    for lens in ([(150, 400), (2, 300), (1, 90)], [(1, 399), (100, 200), (52, 90)],
                 [(0, 17), (0, 0), (153, 90)]):
        starts = np.concatenate([[0], np.cumsum([n for n, _ in lens])])
        b.q_start.copy_(torch.from_numpy(starts.astype(np.int32)))
        b.kv_len.copy_(torch.tensor([n for _, n in lens], dtype=torch.int32))
        out.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(out, 5.0)
        b.attend(out=eager)
        torch.cuda.synchronize()
        assert (out == eager).all()
        # max_new (150) leaves the rows past it alone
        b.lens, b.starts = [(min(n, 150), length) for n, length in lens], starts
        if max(n for n, _ in lens) <= 150:
            saved = b.slots
            b.slots = [s[:length] for s, (_, length) in zip(b.slots, lens)]
            b.check(out)
            b.slots = saved
        else:
            assert (out[150:] == 5).all() and torch.isfinite(out[:150].float()).all()


@pytest.mark.parametrize("B,q_heads,heads", [(70, 2, 1), (130, 3, 3), (300, 8, 4)])
def test_many_sequences(dev, B, q_heads, heads):
    """More sequences than a wave has lanes: split (few workgroups) and not."""
    rng = np.random.default_rng(B)
    long = 3000 if heads == 1 else 500
    lens = [(int(rng.integers(0, 3)), int(rng.integers(0, 60))) for _ in range(B)]
    lens[3], lens[B - 2] = (1, long), (2, long - 7)
    b = Batch(dev, 27, lens, q_heads, heads, 64, 16, "f16", "f16")
    out, lse = b.attend(with_lse=True)
    torch.cuda.synchronize()
    b.check(out, lse)
    ones = [i for i, (n, _) in enumerate(lens) if n == 1]
    q = b.q[torch.from_numpy(b.starts[ones]).to(dev)]
    at = torch.tensor(ones).to(dev)
    got = b.cache.attend(q, b.table[at], b.kv_len[at])
    want = f64(out)[b.starts[ones]]
    # (another split: both are within the tolerance of the oracle)
    assert np.abs(f64(got) - want).max() <= 2.0 ** -8


def test_out_may_be_the_queries(dev):
    for lens, heads in (([(1, 3000), (3, 70)], 4), ([(90, 200), (40, 40)], 8)):
        b = Batch(dev, 28, lens, heads, 2, 64, 16, "f16", "int8")
        want = b.attend()
        assert b.attend(out=b.q) is b.q
        assert (b.q == want).all()


def test_two_streams_at_once(dev):
    """Calls on two streams share nothing: each allocates its own workspace."""
    one = Batch(dev, 23, [(1, 9000), (1, 3000)], 8, 1, 128, 64, "f16", "f16")
    two = Batch(dev, 24, [(1, 8000), (1, 5000)], 8, 1, 128, 64, "f16", "f16")
    want = [b.attend().clone() for b in (one, two)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, b in enumerate((one, two)):
            got[i].append(b.attend(stream=streams[i]))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all((x == w).all() for x in g)
    got = one.attend(stream=streams[0].cuda_stream)
    streams[0].synchronize()
    assert (got == want[0]).all()


def test_the_same_call_gives_the_same_bits(dev):
    for lens, heads in ((MIXES["long"], 4), (MIXES["chunks"], 8)):
        b = Batch(dev, 25, lens, heads, 1, 64, 32, "bf16", "int8")
        want = b.attend()
        for _ in range(5):
            assert (bits(b.attend()) == bits(want)).all()


def test_a_cache_past_32_bit_offsets(dev):
    """Keys and values of more than 2^32 elements; tokens at both ends."""
    page, heads, dim = 256, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 8
    cache = P.KVCache(torch.empty((pages, heads, page, dim), dtype=torch.int8, device=dev),
                      torch.empty((pages, heads, page // 16, dim, 16), dtype=torch.int8, device=dev),
                      torch.empty((pages, heads, page), device=dev),
                      torch.empty((pages, heads, page), device=dev))
    rng = np.random.default_rng(9)
    n = 600
    table = torch.tensor([[pages - 1, 0, pages - 3]], dtype=torch.int32, device=dev)
    j = np.arange(n)
    slots = torch.from_numpy(table.cpu().numpy()[0][j // page].astype(np.int64) * page + j % page)
    kv = [numbers(rng, (n, heads, dim), "f32") for _ in range(2)]
    cache.write(kv[0].to(dev), kv[1].to(dev), slots.to(dev))
    back = cache.read(slots.to(dev), dtype=torch.float32)
    torch.cuda.synchronize()
    want = []
    for x, got in zip(kv, back):
        codes, scale = O.quantise(x.numpy(), "int8")
        want.append(codes * scale.astype(np.float64)[..., None])
        assert (np.abs(f64(got) - want[-1]) <= 2.0 ** -23 * np.abs(want[-1])).all()
    for new in (1, 40):
        q = numbers(rng, (new, 16, dim), "f16").to(dev)
        starts = torch.tensor([0, new], dtype=torch.int32, device=dev)
        out = cache.attend(q, table, torch.tensor([n], dtype=torch.int32, device=dev), starts)
        ref, _, _ = O.attend64(f64(q), want[0], want[1], new, n)
        assert np.abs(f64(out) - ref).max() <= 2.0 ** -9


# --------------------------------------------------------------- all together
def test_a_layer_from_its_codes_to_its_output(dev):
    """q/k/v product, rotary and cache write, attention, rotation, o product: the
    Leech-coded matrices around the operators, tokens one after the other, against
    the same chain in f64."""
    from oracle import decode as D
    from oracle import rotation as R
    from paper_2609_02652_amd import synth
    hidden, heads, kv, dim = 768, 6, 2, 128
    cb = P.Codebook(12)
    dcb = P.DeviceCodebook(cb, dev)

    def matrix(M, K, name):
        inp = synth.make_gemv_inputs(M, K, seed=31, name=name)
        cls, sm, lv = cb.fields_from_points(inp.z)
        mat = P.LeechMatrix.from_fields(dcb, P.PLANES14, cls, inp.gain, sm, lv, inp.scale, dev)
        return inp, mat, D.weights64_from_points(inp.z, inp.gain, inp.scale, (1.0, 1.0))

    qkv, wqkv, w64 = matrix((heads + 2 * kv) * dim, hidden, "kv-qkv")
    o, wo, o64 = matrix(hidden, heads * dim, "kv-o")
    signs = synth.make_signs(heads * dim, seed=31, name="kv-o")
    cache = P.KVCache.empty(3, 16, kv, dim, torch.float16, dev)
    freq, _ = P.rotary_frequencies(dim)
    r = P.Rotary(torch.from_numpy(freq).to(dev))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=dev)
    ks, vs = [], []
    rng = np.random.default_rng(31)
    for t in range(20):
        x = np.zeros(qkv.Kpad, np.float16)
        x[:hidden] = (8 * rng.normal(size=hidden)).astype(np.float16)
        y = wqkv.gemv(torch.from_numpy(x).to(dev)).view(1, heads + 2 * kv, dim)
        pos = torch.tensor([t], device=dev)
        slot = torch.tensor([[2, 0, 1][t // 16] * 16 + t % 16], device=dev)
        q = cache.write(y[:, heads:heads + kv], y[:, heads + kv:], slot, r, pos, y[:, :heads],
                        dtype=torch.float16)
        a = cache.attend(q, table, torch.tensor([t + 1], dtype=torch.int32, device=dev))
        out = wo.gemv(P.rotate_x(a.view(-1), torch.from_numpy(signs).to(dev), wo.Kpad))
        y64 = (w64 @ x.astype(np.float64)).reshape(1, heads + 2 * kv, dim)
        turned = O.rotate64(y64[:, :heads + kv], [t], freq)
        ks.append(turned[0, heads:])
        vs.append(y64[0, heads + kv:])
        a64, _, _ = O.attend64(turned[:, :heads], np.stack(ks), np.stack(vs), 1, t + 1)
        want = o64 @ R.rotate_padded64(a64.reshape(-1), signs, wo.Kpad)
        err = np.abs(out.cpu().numpy() - want).max()
        size = np.linalg.norm(o64, axis=1).max() * np.linalg.norm(a64)
        # q, k, v, the weights, out and the rotation's output are each rounded to
        # f16 (2^-11): a score moves by up to 2·2^-11·|q||k|/√dim, the rest adds up
        sc = 2 * 2.0 ** -11 * max(np.linalg.norm(turned[0, :heads], axis=1)) * \
            max(np.linalg.norm(k, axis=1).max() for k in ks) / math.sqrt(dim)
        big = max(np.linalg.norm(v, axis=1).max() for v in vs) * math.sqrt(heads)
        assert err <= np.linalg.norm(o64, axis=1).max() * big * (2 * sc + 5 * 2.0 ** -11), (t, err, size)
