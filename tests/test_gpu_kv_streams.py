"""Tensors that a call on another stream uses and that its caller drops at once."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_02652_amd as P  # noqa: E402

pytestmark = pytest.mark.gpu
T, HEADS, DIM, PAGE = 48, 2, 64, 16


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    return torch.device("cuda:0")


def inputs(dev):
    """A call's tensors, the same numbers each time, in memory of their own."""
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    x = [torch.randn(T, h, DIM, generator=gen, device=dev) for h in (HEADS, HEADS, 4)]
    return dict(k=x[0], v=x[1], q=x[2].half(), positions=torch.arange(T, device=dev) + 5,
                slots=torch.arange(T, device=dev), starts=torch.tensor([0, T], dtype=torch.int32,
                                                                       device=dev),
                lens=torch.tensor([T], dtype=torch.int32, device=dev),
                table=torch.arange(3, dtype=torch.int32, device=dev).view(1, 3))


def run(what, cache, turn, i, stream=None):
    if what == "rope":
        return P.rope(i["k"], i["positions"], turn, stream=stream)
    if what == "write":
        return cache.write(i["k"], i["v"], i["slots"], turn, i["positions"], i["k"][:, :1],
                           stream=stream)
    if what == "read":
        return cache.read(i["slots"], stream=stream)[0]
    return cache.attend(i["q"], i["table"], i["lens"], i["starts"], stream=stream)


@pytest.mark.parametrize("kind", [torch.float16, torch.int8])
@pytest.mark.parametrize("what", ["rope", "write", "read", "attend"])
def test_dropped_tensors_last_until_the_stream_has_read_them(dev, what, kind):
    """The stream waits behind other work while the caller drops what it passed and
    fills as many tensors of the same sizes."""
    turn = P.Rotary.of(DIM, device=dev)
    cache = P.KVCache.empty(3, PAGE, HEADS, DIM, kind, dev)
    run("write", cache, turn, inputs(dev))
    want = run(what, cache, turn, inputs(dev)).clone()
    kept = cache.k.clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        i = inputs(dev)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
        got = run(what, cache, turn, i, side)
        sizes = [t.shape for t in i.values()], [t.dtype for t in i.values()]
        del i
        others = [torch.full(s, 3, dtype=d, device=dev) for s, d in zip(*sizes) for _ in range(2)]
        torch.cuda.synchronize()
        assert (got == want).all() and (cache.k.view(torch.uint8) == kept.view(torch.uint8)).all()
        del others, got


def test_a_cache_dropped_while_it_is_read(dev):
    turn = P.Rotary.of(DIM, device=dev)
    side = torch.cuda.Stream()
    cache = P.KVCache.empty(3, PAGE, HEADS, DIM, torch.int8, dev)
    i = inputs(dev)
    run("write", cache, turn, i)
    want = run("attend", cache, turn, i)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
    got = run("attend", cache, turn, i, side)
    parts = [(t.shape, t.dtype) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    del cache
    others = [torch.ones(s, dtype=d, device=dev) for s, d in parts for _ in range(2)]
    torch.cuda.synchronize()
    assert (got == want).all() and len(others) == 8


@pytest.mark.parametrize("how", ["handle", "external", "default"])
def test_streams_named_by_their_handle(dev, how):
    """Run where they say; nothing is noted on a stream that may end before the tensors."""
    turn, i = P.Rotary.of(DIM, device=dev), inputs(dev)
    cache = P.KVCache.empty(3, PAGE, HEADS, DIM, torch.float16, dev)
    run("write", cache, turn, i)
    want = run("attend", cache, turn, i)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = {"handle": side.cuda_stream, "default": 0,
              "external": torch.cuda.ExternalStream(side.cuda_stream, device=dev)}[how]
    got = run("attend", cache, turn, i, stream)
    torch.cuda.synchronize()
    assert (got == want).all()


def test_a_call_captured_on_a_given_stream(dev):
    """The capture's own stream is named, its tensors are from outside; replays beside
    eager work, and calls after their memory is given back."""
    turn, i = P.Rotary.of(DIM, device=dev), inputs(dev)
    cache = P.KVCache.empty(3, PAGE, HEADS, DIM, torch.int8, dev)
    run("write", cache, turn, i)
    want = run("attend", cache, turn, i)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        stream = torch.cuda.current_stream()
        run("write", cache, turn, i, stream)
        got = run("attend", cache, turn, i, stream)
    for turn_no in range(3):
        i["v"].mul_(-1)                                 # v is linear in the output
        run("read", cache, turn, i)
        got.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        assert (got == (want if turn_no % 2 else -want)).all()
    del i, cache, got, g
    i, cache = inputs(dev), P.KVCache.empty(3, PAGE, HEADS, DIM, torch.int8, dev)
    again = run("attend", cache, turn, i)
    torch.cuda.synchronize()
    assert (again == 0).all()                           # an empty cache's values
