"""The attention's numbers where they are hardest, against f64 from the oracle.

u is a type's half step (f16 2^-11, bf16 2^-8); tolerances are derived at each test.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_02652_amd as P  # noqa: E402
from oracle import kv as O  # noqa: E402
from test_gpu_kv import Batch, TYPES, U, f64, numbers, say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    return torch.device("cuda:0")


def light_keys_beside_a_heavy_one(dev, B, new, spread, q_type, cache_type):
    """32845 keys that share a thousandth of a row's mass, beside one that has the
    rest and a value of 0: out is the light ones' alone.  Neither call's keys are
    split over workgroups (512 of them either way): one base and sum for a tile of
    rows, one for each wave of a single token.  Yields for three rows (of a
    group's heads each) out, lse, the oracle's out, lse and weights, a bound of a
    score's error, and the values."""
    n, heads, group, dim, page = 32845, 8, 8, 64, 64
    say(f"[attend] heavy key: B={B} new={new} spread={spread} {q_type} over {cache_type}")
    rng = np.random.default_rng(3)
    pages = -(-n // page)
    cache = P.KVCache.empty(pages, page, heads, dim, TYPES[cache_type], dev)
    heavy, mass = 12_345, 0.999
    k = spread * numbers(rng, (n, heads, dim), "f32")
    k[..., 0] = 0
    k[heavy] = 0
    k[heavy, :, 0] = math.log(mass / (1 - mass) * n) + 0.5 * spread ** 2
    v = 1 + 0.2 * numbers(rng, (n, heads, dim), "f32").clamp(-4.5, 4.5)
    v[heavy] = 0
    slots = torch.from_numpy(rng.permutation(pages)[np.arange(n) // page] * page
                             + np.arange(n) % page).to(dev)
    cache.write(k.to(dev), v.to(dev), slots)
    table = (slots[::page] // page).int().expand(B, -1).contiguous()
    q = numbers(rng, (B * new, heads * group, dim), "f32")
    q[..., 0] = 8.0                              # scale · 8 · k[0] = k[0]
    q = q.to(TYPES[q_type]).to(dev)
    starts = torch.arange(B + 1, dtype=torch.int32, device=dev) * new
    out, lse = cache.attend(q, table, torch.full((B,), n, dtype=torch.int32, device=dev), starts,
                            max_new=new, causal=False, with_lse=True)
    k64, v64 = (f64(t) for t in cache.read(slots, dtype=torch.float32))
    for row, head in ((0, 0), (B * new // 2 + 5, 3), (B * new - 1, heads - 1)):
        own = slice(head * group, (head + 1) * group)
        q64, kh, vh = f64(q[row:row + 1, own]), k64[:, head:head + 1], v64[:, head:head + 1]
        want, want_lse, w = O.attend64(q64, kh, vh, 1, n, causal=False)
        es = (dim + 8) * 2.0 ** -24 / 8 * (np.abs(q64[0]) @ np.abs(kh[:, 0]).T).max(1) + 2.0 ** -21
        yield f64(out[row, own]), f64(lse[row, own]), want[0], want_lse[0], w[0], es, vh[:, 0]


HEAVY = [(B, new, spread) + pair for B, new in ((64, 1), (1, 1024)) for spread in (0.0, 1.0)
         for pair in (("f16", "f16"), ("f16", "int8"), ("bf16", "e4m3"), ("bf16", "bf16"))]


@pytest.mark.parametrize("case", HEAVY)
def test_the_sum_of_light_weights_beside_a_heavy_one(dev, case):
    """The sum of the weights takes a step's (of 32 tokens at least) as one f32
    addition, and a step's are 64 at most: a relative error of (n / 32 + 64) 2^-24."""
    for _, lse, _, want, w, es, _ in light_keys_beside_a_heavy_one(dev, *case):
        bound = es + (w.shape[1] / 32 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + want)
        far = np.abs(lse - want) / bound
        say(f"    lse {want[0]:.3f}, error {np.abs(lse - want).max():.2e}, of the bound {far.max():.2f}")
        assert (far <= 1).all()


@pytest.mark.parametrize("case", HEAVY)
def test_light_keys_beside_a_heavy_one(dev, case):
    """A weight times its value's scale, over the largest weight and the largest scale
    (equal to a few bits here: values are 0, or between 0.1 and 1.9), is off by u of
    itself or 2^-36.  The sum's error as above, a score's e_s twice (above and below
    the fraction), out's own rounding; what f16 holds under 2^-14 is off by 2^-25."""
    q_type, cache_type = case[-2:]
    for out, _, want, _, w, es, v in light_keys_beside_a_heavy_one(dev, *case):
        n, av = w.shape[1], w @ np.abs(v)
        u = U["bf16" if cache_type == "bf16" else "f16"]       # the second product's type
        bound = ((u + 2 * es + (n / 32 + 64) * 2.0 ** -24)[:, None] * av + U[q_type] * np.abs(want)
                 + 2.0 ** -25)
        if cache_type != "bf16":
            bound += n * 2.0 ** -36 * w.max(1)[:, None] * np.abs(v).max()
        far = np.abs(out - want) / bound
        say(f"    out {np.abs(want).mean():.2e}, error {np.abs(out - want).max():.2e}, "
            f"of the bound {far.max():.2f}")
        assert (far <= 1).all()


@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 25])
@pytest.mark.parametrize("q_type,cache_type", [("f16", "f16"), ("bf16", "int8"), ("bf16", "bf16")])
@pytest.mark.parametrize("new", [1, 70])
def test_scores_of_any_size(dev, new, size, q_type, cache_type):
    """Scores that grow along the keys up to `size` (512 steps; in bf16 and int8 some
    neighbours are equal).  Equal scores weigh alike, whatever their size; a distance
    between others is off by twice e_s = 2^-22 size (the product, its scale, the base)."""
    n, dim = 512, 64
    k = torch.zeros(n, 1, dim)
    k[:, 0, 0] = torch.arange(n) / n                          # exact in f16, a code's multiple
    k[:, 0, 1] = 1.0                                          # int8: a scale of 1 / 127
    v = numbers(np.random.default_rng(4), (n, 1, dim), "f32")
    cache = P.KVCache.empty(n // 16, 16, 1, dim, TYPES[cache_type], dev)
    slots = torch.arange(n).to(dev)
    cache.write(k.to(dev), v.to(dev), slots)
    table = torch.arange(n // 16, dtype=torch.int32, device=dev).view(1, -1)
    q = torch.zeros(new, 1, dim)
    q[:, 0, 0] = 128.0
    q = q.to(TYPES[q_type]).to(dev)
    starts = torch.tensor([0, new], dtype=torch.int32, device=dev)
    out, lse = cache.attend(q, table, torch.tensor([n], dtype=torch.int32, device=dev), starts,
                            scale=size / 128, with_lse=True)
    k64, v64 = (f64(t) for t in cache.read(slots, dtype=torch.float32))
    want, want_lse, w = O.attend64(f64(q), k64, v64, new, n, scale=size / 128)
    es = 2.0 ** -22 * size
    av = w[:, 0] @ np.abs(v64[:, 0])
    bound = (U[q_type] + U["bf16" if cache_type == "bf16" else "f16"]) * av + 2.0 ** -20
    top = w[:, 0] == w[:, 0].max(-1, keepdims=True)
    mixed = (w[:, 0] * ~top).sum(-1)[:, None]              # mass of scores under the largest
    bound += np.where(mixed > 2.0 ** -30, 2 * math.expm1(min(2 * es, 1.0)), 0.0) * av
    err = np.abs(f64(out)[:, 0] - want[:, 0])
    assert (err <= bound).all(), float((err - bound).max())
    assert (np.abs(f64(lse) - want_lse) <= 2 * es + 2.0 ** -20).all()


@pytest.mark.parametrize("cache_type", ["f16", "int8", "e4m3"])
@pytest.mark.parametrize("new", [1, 40])
def test_a_value_that_is_no_number_in_a_part_of_no_weight(dev, new, cache_type):
    """Keys split over workgroups; the part with the NaN has weights of e^-400 beside
    the others': 0 in f32, and still its rows are not finite."""
    n, dim = 9000, 64
    rng = np.random.default_rng(5)
    k = numbers(rng, (n, 1, dim), "f32")
    k[..., 0] = 0
    k[:4000, :, 0] = -400.0
    v = numbers(rng, (n, 1, dim), "f32")
    q = numbers(rng, (2 * new, 1, dim), "f16").to(dev)
    q[..., 0] = 8.0
    cache = P.KVCache.empty(2 * (n // 16 + 1), 16, 1, dim, TYPES[cache_type], dev)
    table = torch.arange(cache.pages, dtype=torch.int32, device=dev).view(2, -1)
    lens = torch.tensor([n, n], dtype=torch.int32, device=dev)
    starts = torch.tensor([0, new, 2 * new], dtype=torch.int32, device=dev)
    at = torch.arange(n).to(dev)
    for first in (0, cache.pages // 2 * 16):
        cache.write(k.to(dev), v.to(dev), at + first)
    clean = cache.attend(q, table, lens, starts, max_new=new)
    assert torch.isfinite(clean).all()
    v[1000, 0, 7] = math.nan
    cache.write(k[1000:1001].to(dev), v[1000:1001].to(dev), at[1000:1001])
    out = cache.attend(q, table, lens, starts, max_new=new)
    assert torch.isnan(out[:new, 0, 7]).all()
    assert (out[new:] == clean[new:]).all()


@pytest.mark.parametrize("q_type,cache_type,size,scale", [("f16", "f16", 1.0, 3e38),
                                                          ("bf16", "bf16", 1.0, -3e38),
                                                          ("bf16", "int8", 2.0 ** 100, 2.0 ** 60)])
@pytest.mark.parametrize("new", [1, 40])
def test_scales_at_the_end_of_their_range(dev, new, q_type, cache_type, size, scale):
    """Keys of zeros: every score is 0 whatever the scale (times log2 e, or times the
    power of two taken out of a bf16 query, it would pass f32's range)."""
    n, dim = 100, 64
    v = numbers(np.random.default_rng(6), (n, 1, dim), "f32").to(dev)
    cache = P.KVCache.empty(7, 16, 1, dim, TYPES[cache_type], dev)
    slots = torch.arange(n).to(dev)
    cache.write(torch.zeros_like(v), v, slots)
    table = torch.arange(7, dtype=torch.int32, device=dev).view(1, -1)
    q = torch.full((new, 1, dim), size, dtype=TYPES[q_type], device=dev)
    out, lse = cache.attend(q, table, torch.tensor([n], dtype=torch.int32, device=dev),
                            torch.tensor([0, new], dtype=torch.int32, device=dev), causal=False,
                            scale=scale, with_lse=True)
    v64 = f64(cache.read(slots, dtype=torch.float32)[1])[:, 0]
    # weights are equal (over int8 rounded with their values' scales: u each)
    bound = 2 * U[q_type] * np.abs(v64).mean(0) + 2.0 ** -20
    assert (np.abs(f64(out)[:, 0] - v64.mean(0)) <= bound).all()
    assert (np.abs(f64(lse) - math.log(n)) <= 2.0 ** -18).all()


@pytest.mark.parametrize("kind,part", [("f16", "key"), ("bf16", "key"), ("int8", "scale"),
                                       ("e4m3", "scale")])
@pytest.mark.parametrize("scale", [0.125, -0.125])
@pytest.mark.parametrize("new", [2, 60])
def test_infinite_scores(dev, new, scale, kind, part):
    """An infinite key, or key scale, on the token that only the last row sees: a score
    of +inf makes that row NaN, one of -inf leaves it as it is without the token.  A row
    that sees only such a token is as one that sees nothing."""
    n, dim = 100, 64
    rng = np.random.default_rng(7)
    q_type = "bf16" if kind == "bf16" else "f16"
    k, v = (numbers(rng, (n, 1, dim), "f32") for _ in range(2))
    q = numbers(rng, (new, 1, dim), q_type)
    k[-1] = 2 * q[-1:].float()                                  # a positive product
    q = q.to(dev)
    slots, table = torch.arange(n).to(dev), torch.arange(7, dtype=torch.int32, device=dev).view(1, -1)
    starts = torch.tensor([0, new], dtype=torch.int32, device=dev)
    lens = torch.tensor([n], dtype=torch.int32, device=dev)
    cache = P.KVCache.empty(7, 16, 1, dim, TYPES[kind], dev)
    cache.write(k.to(dev), v.to(dev), slots)
    clean, clean_lse = cache.attend(q, table, lens, starts, scale=scale, with_lse=True)
    k64, v64 = (f64(t) for t in cache.read(slots, dtype=torch.float32))
    want, want_lse, w = O.attend64(f64(q[-1:]), k64[:-1], v64[:-1], 1, n - 1, scale=scale)
    place = (6, 0, (n - 1) % 16)
    for sign in (1.0, -1.0):
        if part == "key":
            d = int(q[-1, 0].abs().argmax())
            saved = cache.k[place][d].clone()
            cache.k[place][d] = math.copysign(math.inf, sign * float(q[-1, 0, d]))
        else:
            saved = cache.k_scale[place].clone()
            cache.k_scale[place] = sign * math.inf
        out, lse = cache.attend(q, table, lens, starts, scale=scale, with_lse=True)
        assert (out[:-1] == clean[:-1]).all() and (lse[:-1] == clean_lse[:-1]).all()
        one, one_lse = cache.attend(q, table, lens, starts, scale=scale, window=1, with_lse=True)
        if sign * scale > 0:
            assert torch.isnan(out[-1]).all() and torch.isnan(lse[-1]).all()
            assert torch.isnan(one[-1]).all() and torch.isnan(one_lse[-1]).all()
        else:
            av = w[0] @ np.abs(v64[:-1, 0])
            es = (dim + 8) * 2.0 ** -24 * 0.125 * (np.abs(f64(q[-1, 0])) @ np.abs(k64[:-1, 0]).T).max() + 2.0 ** -21
            bound = (U[q_type] + 2 * es) * av + U[q_type] * np.abs(want[0]) + 2.0 ** -25
            assert (np.abs(f64(out[-1]) - want[0]) <= bound).all()
            assert (np.abs(f64(lse[-1]) - want_lse[0]) <= es + 2.0 ** -21 * (1 + np.abs(want_lse[0]))).all()
            assert (one[-1] == 0).all() and (one_lse[-1] == -math.inf).all()
        if part == "key":
            cache.k[place][d] = saved
        else:
            cache.k_scale[place] = saved


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_codes_read_as_the_rounded_f32_product(dev, kind):
    """To the bit, for every code, in each type."""
    rng = np.random.default_rng(8)
    n, heads, dim = 64, 2, 256
    cache = P.KVCache.empty(4, 16, heads, dim, TYPES[kind], dev)
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(TYPES[kind])
    cache.k.copy_(codes.to(dev).expand_as(cache.k))
    cache.v.copy_(codes.to(dev)[:, None].expand_as(cache.v))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.from_numpy(np.exp2(rng.uniform(-12, 2, t.shape)).astype(np.float32)))
    slots = torch.from_numpy(rng.permutation(n)).to(dev)
    for dst in ("f32", "f16", "bf16"):
        for got, scale in zip(cache.read(slots, dtype=TYPES[dst]), (cache.k_scale, cache.v_scale)):
            s = scale.transpose(1, 2).reshape(n, heads)[slots]          # [pages, heads, page]
            want = (codes.float().to(dev) * s[..., None]).to(TYPES[dst])
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
            assert torch.equal(got.isnan(), want.isnan())


@pytest.mark.parametrize("cache_type", ["f16", "e4m3"])
def test_more_single_tokens_than_the_card_takes_at_once(dev, cache_type):
    """1100 sequences of 4 heads stay whole, however long the table; empty ones too."""
    rng = np.random.default_rng(9)
    lens = [(1, int(n)) for n in rng.integers(0, 40, 1100)]
    lens[7], lens[1000] = (1, 2000), (1, 1)
    b = Batch(dev, 33, lens, 4, 4, 32, 16, "f16", cache_type)
    for starts in (None, b.q_start):
        out, lse = b.attend(q_start=starts, max_new=None if starts is None else 1, with_lse=True)
        torch.cuda.synchronize()
        b.check(out, lse)
