"""Memory that calls on node rows make for another stream than the current one."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ff import pipad, weights  # noqa: E402,F401

N, F, HIDDEN, FO = 6000, 64, 320, 48  # (results and workspaces of more than a megabyte: pieces of their own in the allocator)


def calls(pipad, W, b, X, dY, v, **kw):  # noqa: F811
    """Every function once; what it returns."""
    y = pipad.gated_ff(X, *W, *b, **kw)
    d = pipad.gated_ff_backward(X, dY, *W, *b[:2], **kw)
    r, z = pipad.residual_norm(X, X, X, post="layer", pre="rms", w_post=v, **kw)
    e = pipad.residual_norm_backward(X, X, X, X, X, post="layer", pre="rms", w_post=v, **kw)
    return [t for x in (y, *d, r, z, *e) if x is not None for t in (x if isinstance(x, list) else [x])]


def operands(listed):
    gen = torch.Generator(device="cuda").manual_seed(21)
    W, b = weights(gen, F, HIDDEN, FO, True)
    X, dY = torch.randn((N, 2, F), device="cuda", generator=gen), torch.randn((N, 2, FO), device="cuda", generator=gen)
    if listed:
        X, dY = list(X.transpose(0, 1).contiguous().unbind(0)), list(dY.transpose(0, 1).contiguous().unbind(0))
    return W, b, X, dY, torch.randn(F, device="cuda", generator=gen)


@pytest.mark.parametrize("wrapped", [False, True])
@pytest.mark.parametrize("listed", [False, True])
def test_memory_for_another_stream_is_not_the_current_ones(pipad, monkeypatch, listed, wrapped):  # noqa: F811
    """Pieces that the current stream has just given back are still read by what is queued there: a call on another stream has to leave
    them alone, for results, gradients and workspaces."""
    from paper_2301_00391_amd import rows
    W, b, X, dY, v = operands(listed)
    want = calls(pipad, W, b, X, dY, v)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    spare = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in (256, 4096, 1 << 17, 1 << 21, 1 << 22, 1 << 23, 1 << 24, 1 << 25, 1 << 26) for _ in range(12)]
    spans = [(s.data_ptr(), s.data_ptr() + s.numel()) for s in spare]
    del spare
    made, empty = [], torch.empty

    def seen(*args, **kw):
        made.append(empty(*args, **kw))
        return made[-1]

    monkeypatch.setattr(rows.torch, "empty", seen)

    class Other:  # (anything that names a stream)
        cuda_stream = side.cuda_stream

    got = calls(pipad, W, b, X, dY, v, stream=Other() if wrapped else side)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert len(made) >= 20
    for t in made:
        at = t.data_ptr()
        assert not any(low <= at < high for low, high in spans)
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_results_dropped_early_wait_for_the_current_stream(pipad):  # noqa: F811
    """A result made on another stream and dropped while the current one is still busy with it is not given out again before."""
    W, b, X, dY, v = operands(False)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    got = calls(pipad, W, b, X, dY, v, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(400_000_000)  # (a fifth of a second, in place of what reads the results)
    large = [t for t in got if t.numel() * 4 > 1 << 20]
    sizes, at = [t.numel() * 4 for t in large], {t.data_ptr() for t in large}
    assert len(large) == 7
    del got, large
    with torch.cuda.stream(side):
        again = [torch.empty(size, dtype=torch.uint8, device="cuda") for size in sizes]
    busy = not torch.cuda.current_stream().query()
    assert not busy or not any(t.data_ptr() in at for t in again)
    torch.cuda.synchronize()
    assert busy


@pytest.mark.parametrize("wrapped", [False, True])
def test_the_default_stream_from_another_one(pipad, wrapped):  # noqa: F811
    W, b, X, dY, v = operands(True)
    want = calls(pipad, W, b, X, dY, v)
    torch.cuda.synchronize()

    class Other:
        cuda_stream = 0

    with torch.cuda.stream(torch.cuda.Stream()):
        got = calls(pipad, W, b, X, dY, v, stream=Other() if wrapped else torch.cuda.default_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_another_stream_within_a_graph(pipad):  # noqa: F811
    """Calls that a captured stream hands to a second one, which is captured with it, and their memory: replayed beside eager work."""
    W, b, X, dY, v = operands(False)
    calls(pipad, W, b, X, dY, v)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        first = calls(pipad, W, b, X, dY, v, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for t in calls(pipad, W, b, X, dY, v, stream=side)[::2]:  # (and some that are dropped at once)
            del t
        torch.cuda.current_stream().wait_stream(side)
        second = calls(pipad, W, b, X, dY, v)
    for replay in range(3):
        X.normal_(generator=torch.Generator(device="cuda").manual_seed(replay))
        want = calls(pipad, W, b, X, dY, v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got in (first, second):
            assert all(torch.equal(x, y) for x, y in zip(want, got)), replay
