"""The 8-bit path at the ends of what it takes: every quotient of 16-bit numbers, the
smallest numbers, workspaces that hold anything, offsets beyond 2^32, the most experts
and choices."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def of_bits(bits, dtype):
    import torch
    return bits.to(torch.int16).view(dtype)


@pytest.mark.parametrize("dtype,mantissa", [("bf16", 7), ("f16", 10)])
def test_quotients_are_those_of_one_division(dtype, mantissa):
    """Every number from 2^-10 to 1 (bfloat16) or 2^-7 to 1 (half) beside every number of
    [1, 2) as a block's largest: scales and bytes are those of one correctly rounded
    division each, computed on the CPU.  Many of these quotients are next to a tie."""
    import torch
    import eight_util as u
    t = u.TYPES[dtype]
    one = {"bf16": 0x3f80, "f16": 0x3c00}[dtype]
    step = 1 << mantissa
    tops = of_bits(torch.arange(one, one + step), t)
    down = {"bf16": 10, "f16": 7}[dtype]
    below = of_bits(torch.arange(one - down * step, one), t)
    blocks = -(-len(below) // 127)
    below = torch.cat([below, below.new_zeros(blocks * 127 - len(below))]).reshape(blocks, 127)
    below[:, 1::2] = -below[:, 1::2]
    for part in tops.split(256):
        X = torch.cat([part[:, None, None].expand(-1, blocks, 1), below[None].expand(len(part), -1, -1)], 2).reshape(len(part), -1)
        Q, s = oz.ozaki25_quantise(X.cuda())
        true = part.float() / torch.tensor(448.0)
        assert torch.equal(s.cpu(), true[None].expand(blocks, -1))
        q = (X.float() / true[:, None]).to(u.E4M3)
        assert torch.equal(Q.cpu().float(), q.float())


@pytest.mark.parametrize("rows", [3, 40, 300, 4096])
def test_the_smallest_numbers_of_e4m3(rows):
    """Sums of products of subnormal numbers, 2^-9 and below 2^-6: exact."""
    import torch
    import eight_util as u
    n, k = 3600 if rows == 4096 else 70, 256
    gen = torch.Generator(device="cuda").manual_seed(rows)
    A, B = (torch.randint(0, 8, (v, k), device="cuda", generator=gen) + 128 * torch.randint(0, 2, (v, k), device="cuda", generator=gen)
            for v in (rows, n))
    A, B = A.to(torch.uint8).view(u.E4M3), B.to(torch.uint8).view(u.E4M3)
    assert float(A.float().abs().max()) == 7 * 2.0 ** -9
    want = A.double() @ B.double().t() * 2.0 ** 14
    for squares in (True, False):
        a, b = torch.full((2, rows), 2.0 ** 14, device="cuda"), torch.ones((-(-n // 128), 2) if squares else (2, n), device="cuda")
        for dtype in u.TYPES.values():
            Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares, out_dtype=dtype)
            assert torch.equal(Y, want.to(dtype))


@pytest.mark.parametrize("tokens", [2, 30])
@pytest.mark.parametrize("small", ["x", "up", "down"])
def test_subnormal_halves_in_a_layer(small, tokens):
    """Numbers of half below 2^-14 in X and in the weights count."""
    import torch
    import eight_util as u
    import test_gpu_layer as layer
    H = torch.float16
    X, up, gate, down = (u.normal(s, H, i) for i, s in enumerate(((tokens, 200), (5, 100, 200), (5, 100, 200), (5, 150, 100))))
    low = 2.0 ** -17
    if small == "x":
        X, up, gate = X * low, up * 32, gate * 32
    elif small == "up":
        X, up, gate = X * 32, up * low, gate * low
    else:
        X, up, gate, down = X * 8, up * 8, gate * 8, down * low
    which, gates = layer.routes(tokens, 2, 5, 7)
    gates = gates * (2.0 ** 10 if small != "down" else 1.0)
    Y = oz.ozaki25_expert_layer(X, which, gates, up, down, gate=gate)
    want, off = layer.expected(X, which, gates, up.double(), gate.double(), down.double())
    bad = (Y.double() - want).abs() - off - (want.abs() + off) * 2.0 ** -11 - 2.0 ** -25
    assert bool((bad <= 0).all()) and float(want.abs().max()) > 2.0 ** -8


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens,top,inner", [(2, 3, 101), (40, 4, 101), (200, 2, 37)])
def test_workspaces_that_hold_anything(tokens, top, inner, eight):
    """Workspaces full of NaN: results as without one, bit for bit."""
    import torch
    import eight_util as u
    import test_gpu_layer as layer
    width, out, experts = 130, 99, 6
    X = u.normal((tokens, width), torch.bfloat16, 1)
    (up, us, _), (gate, gs, _), (down, ds, _) = (layer.weights(experts, *s, "bf16", eight, i)
                                                 for i, s in ((2, (inner, width)), (3, (inner, width)), (4, (out, inner))))
    which, gates = layer.routes(tokens, top, experts, 5)
    call = lambda **kw: oz.ozaki25_expert_layer(X, which, gates, up, down, gate=gate, up_scales=us, down_scales=ds, gate_scales=gs, **kw)  # noqa: E731
    size = oz.ozaki25_expert_layer_workspace_size(tokens, top, width, inner, out)
    assert torch.equal(call(), call(workspace=torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")))
    H, dY = u.normal((tokens, 1031), torch.bfloat16, 6), u.normal((tokens, 1031), torch.bfloat16, 7)
    room = torch.full((oz.ozaki25_rms_norm_backward_workspace_size(tokens, 1031),), 0xff, dtype=torch.uint8, device="cuda")
    for a, b in zip(oz.ozaki25_rms_norm_backward(dY, H), oz.ozaki25_rms_norm_backward(dY, H, workspace=room)):
        assert torch.equal(a, b)


def test_norms_beyond_32_bit_offsets():
    """Rows whose elements and bytes lie past 2^32: the last ones as alone."""
    import torch
    import eight_util as u
    rows, width = (1 << 20) + 5, 4104
    X = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    X[-9:] = u.normal((9, width), torch.bfloat16, 1)
    w, few = u.normal((width,), torch.bfloat16, 2), X[-9:].clone()
    Q, s, H = oz.ozaki25_rms_norm(X, w, residual=X, quantised=True)
    q, t, h = oz.ozaki25_rms_norm(few, w, residual=few, quantised=True)
    assert torch.equal(Q[-9:].view(torch.uint8), q.view(torch.uint8)) and torch.equal(s[:, -9:], t) and torch.equal(H[-9:], h)
    assert bool((Q[:100].view(torch.uint8) == 0).all())
    del Q, s, H
    torch.cuda.empty_cache()
    dX, dw = oz.ozaki25_rms_norm_backward(X, X, w, dH=X)
    dx, dv = oz.ozaki25_rms_norm_backward(few, few, w, dH=few)
    # rows of zeros add nothing to the weights' gradient: the nine rows' sums, grouped otherwise
    terms = few.double().square() / (few.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    assert torch.equal(dX[-9:], dx) and bool(((dw.double() - dv.double()).abs() <= terms.sum(0) * 2 * (9 + 37) * u.U).all())


@pytest.mark.parametrize("eight", [False, True])
def test_the_most_choices_and_experts(eight):
    import torch
    import test_gpu_layer as layer
    layer.run(256, 32, 4096, 24, 16, 24, "bf16", eight, True, seed=3)
    which = torch.full((256, 32), 7, dtype=torch.int32, device="cuda")
    layer.run(256, 32, 9, 40, 24, 16, "f16", eight, False, which=which)
