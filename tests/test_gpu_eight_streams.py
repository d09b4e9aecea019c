"""The 8-bit path's calls run on the stream that they are given and keep nothing that
two of them share.

Behind a delay on another stream the inputs are renewed, then the call follows: one that
ran on the default stream would read the old inputs (the delay has to be still running
when the call returns, or the test shows nothing).  Results are compared on that stream,
one whose hardware queue is not the default stream's: streams share a few of those, and
in one queue the order of the launches would hold by itself."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu
NAMES = ["norm", "norm_8bit", "norm_backward", "norm_backward_one", "quantise", "few", "few_odd", "tiles", "parts", "parts_odd", "many",
         "weights_grad", "layer_2", "layer_40", "layer_40_8bit"]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.fixture(scope="module")
def side():
    """A stream that does not hold up the default one."""
    import torch
    one = torch.zeros(1, device="cuda")
    for _ in range(16):
        stream, done = torch.cuda.Stream(), torch.cuda.Event()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(100_000_000)
        done.record(stream)
        one.add_(1)
        torch.cuda.current_stream().synchronize()
        apart = not done.query()
        torch.cuda.synchronize()
        if apart:
            return stream
    pytest.skip("every stream shares the default one's queue")


def make(name, seed, room):
    """Inputs and a call that takes the stream; room: with a workspace of its own."""
    import torch
    import eight_util as u

    def space(size):
        return torch.empty((size,), dtype=torch.uint8, device="cuda") if room and size else None

    half = torch.bfloat16
    if name.startswith("norm"):
        rows = 1 if name.endswith("one") else 300
        X, R, w, D = (u.normal(s, half, seed + i) for i, s in enumerate(((rows, 1000), (rows, 1000), (1000,), (rows, 1000))))
        if name.startswith("norm_backward"):
            work = space(oz.ozaki25_rms_norm_backward_workspace_size(rows, 1000))
            return [X, R, w, D], lambda **kw: oz.ozaki25_rms_norm_backward(X, R, w, dH=D, workspace=work, **kw)
        return [X, R, w], lambda **kw: oz.ozaki25_rms_norm(X, w, residual=R, quantised=name.endswith("8bit"), **kw)
    if name == "quantise":
        X = u.normal((3, 150, 140), torch.float32, seed)
        return [X], lambda **kw: oz.ozaki25_quantise(X, layout="both", **kw)
    if name.startswith("layer"):
        tokens, eight = int(name.split("_")[1]), name.endswith("8bit")
        X = u.normal((tokens, 256), half, seed)
        up, down = u.normal((6, 100, 256), half, seed + 1, 1 / 16), u.normal((6, 256, 100), half, seed + 2, 0.1)
        us = ds = None
        if eight:
            (up, us), (down, ds) = oz.ozaki25_quantise(up, squares=True), oz.ozaki25_quantise(down, squares=True)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        which = torch.randint(-1, 6, (tokens, 3), device="cuda", dtype=torch.int32, generator=gen)
        gates = torch.rand((tokens, 3), device="cuda", generator=gen)
        work = space(oz.ozaki25_expert_layer_workspace_size(tokens, 3, 256, 100, 256))
        inputs = [X, which, gates, *([up.view(torch.uint8), us, down.view(torch.uint8), ds] if eight else [up, down])]
        return inputs, lambda **kw: oz.ozaki25_expert_layer(X, which, gates, up, down, gate=up, up_scales=us, down_scales=ds, gate_scales=us,
                                                            workspace=work, **kw)
    rows, n, k = {"few": (5, 200, 600), "few_odd": (5, 200, 601), "tiles": (300, 200, 600), "parts": (100, 70, 6200),
                  "parts_odd": (30, 70, 4001), "many": (2100, 2050, 300), "weights_grad": (500, 300, 3200)}[name]
    squares, odd = name != "weights_grad", name.endswith("odd")
    A, a = u.quantised(u.normal((rows, k), torch.float32, seed))
    B, b = u.quantised(u.normal((n, k), torch.float32, seed + 1), squares)
    A, B = u.e4m3_rows(A, 0 if odd else -k % 16), u.e4m3_rows(B, 0 if odd else -k % 16)
    work = space(oz.ozaki25_scaled_matmul_workspace_size(rows, n, k))
    out = half if squares else torch.float32
    return [A.view(torch.uint8), a, B.view(torch.uint8), b], lambda **kw: oz.ozaki25_scaled_matmul(
        A, a, B, b, squares=squares, out_dtype=out, workspace=work, **kw)


def bits(out):
    import torch
    return [t.contiguous().view(torch.uint8).clone() for t in (out if isinstance(out, tuple) else (out,))]


def equal(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("way", ["current", "argument", "handle"])
@pytest.mark.parametrize("name", NAMES)
def test_the_call_is_behind_what_its_stream_holds(name, way, room, side):
    import torch
    inputs, call = make(name, 10, room)
    renewed, call_renewed = make(name, 20, room)
    old, want = bits(call()), bits(call_renewed())
    assert not equal(old, want)
    done = torch.cuda.Event()
    call(**({} if way == "current" else {"stream": side}))  # whatever a first call loads
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        for t, v in zip(inputs, renewed):
            t.copy_(v)
        if way == "current":
            got = call()
    if way != "current":
        got = call(stream=side if way == "argument" else side.cuda_stream)
    done.record(side)
    assert not done.query(), "the delay was over before the call was made"
    with torch.cuda.stream(side):
        assert equal(bits(got), want)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["norm_8bit", "quantise", "tiles", "layer_40"])
def test_elsewhere_it_would_read_what_was_there(name, side):
    """The same with the call on the default stream: the old inputs' result, so that the
    test above would see one that ran there."""
    import torch
    inputs, call = make(name, 10, True)
    renewed, _ = make(name, 20, True)
    old, done = bits(call()), torch.cuda.Event()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        for t, v in zip(inputs, renewed):
            t.copy_(v)
    done.record(side)
    got = bits(call())
    torch.cuda.current_stream().synchronize()
    assert not done.query(), "the delay was over before the call was made"
    assert equal(got, old)
    torch.cuda.synchronize()


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_two_streams_at_once(name, room):
    """Different inputs on two streams that were let go together, several calls each."""
    import torch
    sides = [torch.cuda.Stream() for _ in range(2)]
    made = [make(name, seed, room) for seed in (30, 40)]
    want = [bits(call()) for _, call in made]
    assert not equal(*want)
    torch.cuda.synchronize()
    outs = [[], []]
    for side in sides:
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
    for _ in range(8):
        for i, side in enumerate(sides):
            with torch.cuda.stream(side):
                outs[i].append(made[i][1]())
    for i, side in enumerate(sides):
        with torch.cuda.stream(side):
            assert all(equal(bits(out), want[i]) for out in outs[i])
    torch.cuda.synchronize()
