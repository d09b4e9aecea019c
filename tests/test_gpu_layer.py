"""The layer of experts for few tokens against the formula in 64 bits.

With U = 2^-24: a hidden sum over `width` terms is off by at most width U of the sum
of its magnitudes (products of 16-bit numbers are exact; e4m3 weights add a rounding
by their scale and one per block), silu by 8 U of its value and its slope times that,
the gate's product by a rounding.  The second product's operands carry 16 bits of the
hidden value (2^-17), half's weights all of theirs less 2^-16 of a product (the two
rests).  Everything is propagated by magnitudes below, beside the output's rounding."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def weights(experts, n, k, dtype, eight, seed, layout=0):
    """A stack as the call takes it, its scales, and its values in 64 bits."""
    import torch
    import eight_util as u
    W = u.normal((experts, n, k), u.TYPES[dtype], seed, k ** -0.5)
    if not eight:
        return u.padded(W, layout, float("nan")) if layout else W, None, W.double()
    Q, s = zip(*(u.quantised(w, True) for w in W))
    V = torch.stack([q.double() * u.spread(c, n, k, True).double() for q, c in zip(Q, s)])
    return u.e4m3_rows(torch.stack(Q), layout), torch.stack(s), V


def routes(tokens, top, experts, seed, dropped=True):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = torch.rand((tokens, experts), device="cuda", generator=gen)
    which = r.argsort(1)[:, :top].to(torch.int32).contiguous()
    if dropped and tokens > 2:
        which[1] = -1                       # a token without any expert
        which[2, 0] = experts + 3
    gates = torch.rand((tokens, top), device="cuda", generator=gen) + 0.1
    return which, gates


def expected(X, which, gates, U_, G, D):
    """The result and a bound of what the stated roundings may add up to."""
    import torch
    import eight_util as u
    tokens, width = X.shape
    inner, x = U_.shape[1], X.double()
    Y = torch.zeros((tokens, D.shape[1]), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(Y)
    for t in range(tokens):
        for e, g in zip(which[t].tolist(), gates[t].double().tolist()):
            if not 0 <= e < U_.shape[0]:
                continue
            up, eu = U_[e] @ x[t], (U_[e].abs() @ x[t].abs()) * (width + 130) * u.U
            a, ea = (up, eu) if G is None else (G[e] @ x[t], (G[e].abs() @ x[t].abs()) * (width + 130) * u.U)
            act = a * torch.sigmoid(a)
            eact = 1.1 * ea + 8 * u.U * act.abs()
            h = act if G is None else act * up
            eh = eact if G is None else eact * up.abs() + act.abs() * eu + eact * eu
            eh = eh + h.abs() * (4 * u.U + 2.0 ** -17 + 2.0 ** -16)
            Y[t] += g * (D[e] @ h)
            off[t] += abs(g) * (D[e].abs() @ (eh + h.abs() * (2 * inner + 300) * u.U))
    return Y, off


def run(tokens, top, experts, width, inner, out, dtype, eight, gated, seed=0, layout=0, which=None):
    import eight_util as u
    X = u.normal((tokens, width), u.TYPES[dtype], seed + 1, pad=layout)
    up, us, U_ = weights(experts, inner, width, dtype, eight, seed + 2, layout)
    gate, gs, G = weights(experts, inner, width, dtype, eight, seed + 3, layout) if gated else (None, None, None)
    down, ds, D = weights(experts, out, inner, dtype, eight, seed + 4, layout)
    w, gates = routes(tokens, top, experts, seed + 5)
    which = w if which is None else which
    Y = oz.ozaki25_expert_layer(X, which, gates, up, down, gate=gate, up_scales=us, down_scales=ds, gate_scales=gs)
    want, off = expected(X, which, gates, U_, G, D)
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    bad = (Y.double() - want).abs() - off - (want.abs() + off) * u.half_step(Y.dtype) - tiny
    assert Y.shape == (tokens, out) and bool((bad <= 0).all()), (float(bad.max()), int((bad > 0).sum()))
    return Y


CASES = [
    # tokens, top, experts, width, inner, out
    (1, 1, 1, 1, 1, 1), (1, 2, 8, 128, 64, 128), (1, 2, 8, 200, 100, 150), (2, 3, 5, 1000, 333, 777), (3, 1, 4, 129, 8, 9),
    (16, 4, 16, 256, 130, 264), (16, 32, 40, 64, 40, 48), (9, 2, 3, 7, 5, 3), (5, 2, 300, 130, 257, 100),
    (17, 2, 8, 128, 64, 128), (40, 4, 6, 300, 129, 200), (64, 8, 64, 256, 128, 256), (100, 1, 2, 65, 31, 33),
    (256, 2, 5, 136, 72, 88), (200, 32, 33, 40, 24, 16),
]


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,top,experts,width,inner,out", CASES)
def test_layer(tokens, top, experts, width, inner, out, dtype, eight, gated):
    run(tokens, top, experts, width, inner, out, dtype, eight, gated, seed=tokens + width, layout=(0, 3, 16)[(width + tokens) % 3])


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens,experts,inner", [(20, 20, 500), (64, 64, 900), (130, 20, 500), (200, 16, 520)])
def test_forms(tokens, experts, inner, eight, gated):
    """Enough blocks for the narrower, the wider and the many-row form of the hidden
    values."""
    run(tokens, 2, experts, 70, inner, 40, "bf16" if inner == 500 else "f16", eight, gated, seed=inner, layout=(0, 16)[eight])


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,experts,width,inner,out", [(100, 64, 130, 270, 250), (60, 16, 72, 1030, 1030), (50, 16, 40, 2050, 1030)])
def test_many_choices_of_an_expert(tokens, experts, width, inner, out, dtype, eight, gated):
    """The blocks of 64 rows of weights and 32 choices, some of them in part."""
    run(tokens, 8, experts, width, inner, out, dtype, eight, gated, seed=inner, layout=(3, 16)[eight])


def test_wide_outputs_of_few_choices():
    for eight in (False, True):
        run(2, 3, 5, 130, 70, 4100, "bf16", eight, True)


@pytest.mark.parametrize("eight", [False, True])
def test_larger(eight):
    run(1, 2, 4, 2048, 1024, 2048, "bf16", eight, True)
    run(24, 2, 4, 1024, 1536, 1024, "f16", eight, True)


@pytest.mark.parametrize("tokens", [4, 30])
def test_choices(tokens):
    """Nobody's, everybody's, one expert twice, the highest of many."""
    import torch
    for ids in ([-1, -1], [3, 3], [0, 4999], [4095, 7], [-(2 ** 31), 2 ** 31 - 1]):
        which = torch.tensor([ids] * tokens, dtype=torch.int32, device="cuda")
        Y = run(tokens, 2, 4096, 24, 16, 24, "bf16", False, True, which=which)
        assert ids != [-1, -1] or bool((Y == 0).all())


@pytest.mark.parametrize("tokens", [6, 50])
def test_what_a_token_does_not_reach_it_does_not_see(tokens):
    """A NaN expert, a NaN token: only those that meet are NaN.  The same rows as
    alone otherwise."""
    import torch
    import eight_util as u
    experts, width, inner = 6, 200, 100
    X = u.normal((tokens, width), torch.bfloat16, 1)
    up, gate, down = (u.normal((experts, *s), torch.bfloat16, i, 0.1) for i, s in
                      ((2, (inner, width)), (3, (inner, width)), (4, (width, inner))))
    which, gates = routes(tokens, 2, experts, 5, dropped=False)
    clean = oz.ozaki25_expert_layer(X, which, gates, up, down, gate=gate)
    for W in (up, gate, down):
        spoilt = W.clone()
        spoilt[2] = float("nan")
        Y = oz.ozaki25_expert_layer(X, which, gates, *(spoilt if W is v else v for v in (up, down)),
                                    gate=spoilt if W is gate else gate)
        meets = (which == 2).any(1)
        assert bool(torch.isnan(Y[meets]).all()) and torch.equal(Y[~meets], clean[~meets])
    x = X.clone()
    x[3] = float("inf")
    Y = oz.ozaki25_expert_layer(x, which, gates, up, down, gate=gate)
    assert not bool(torch.isfinite(Y[3]).any())
    rest = torch.arange(tokens, device="cuda") != 3
    assert torch.equal(Y[rest], clean[rest])


@pytest.mark.parametrize("tokens", [2, 40])
def test_slices_and_an_expert_slice(tokens):
    """gate and up as halves of one stack, Y as a slice, X from a wider matrix; also
    as e4m3 with the scales' halves."""
    import torch
    import eight_util as u
    experts, width, inner = 5, 256, 128
    both = u.normal((experts, 2 * inner, width), torch.bfloat16, 1, 0.06)
    down = u.normal((experts, width, inner), torch.bfloat16, 2, 0.1)
    X = u.normal((tokens, width), torch.bfloat16, 3, pad=9)
    which, gates = routes(tokens, 2, experts, 4)
    gate, up = both[:, :inner], both[:, inner:]
    whole = oz.ozaki25_expert_layer(X.contiguous(), which, gates, up.contiguous(), down, gate=gate.contiguous())
    wide = torch.full((tokens, width + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    oz.ozaki25_expert_layer(X, which, gates, up, down, gate=gate, Y=wide[:, 3:3 + width])
    assert torch.equal(wide[:, 3:3 + width], whole) and bool((wide[:, :3] == 5).all()) and bool((wide[:, 3 + width:] == 5).all())
    Q, s = oz.ozaki25_quantise(both, squares=True)
    D, d = oz.ozaki25_quantise(down, squares=True)
    a = oz.ozaki25_expert_layer(X, which, gates, Q[:, inner:], D, gate=Q[:, :inner], up_scales=s[:, 1:], gate_scales=s[:, :1],
                                down_scales=d)
    b = oz.ozaki25_expert_layer(X, which, gates, Q[:, inner:].clone(), D, gate=Q[:, :inner].clone(), up_scales=s[:, 1:].clone(),
                                gate_scales=s[:, :1].clone(), down_scales=d)
    assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [3, 20])
def test_nothing_between(tokens):
    import torch
    for experts, width, inner, top in ((0, 8, 8, 2), (3, 0, 8, 2), (3, 8, 0, 2), (3, 8, 8, 0)):
        X = torch.ones((tokens, width), dtype=torch.bfloat16, device="cuda")
        up = torch.ones((experts, inner, width), dtype=torch.bfloat16, device="cuda")
        down = torch.ones((experts, 16, inner), dtype=torch.bfloat16, device="cuda")
        Y = torch.full((tokens, 16), 3.0, dtype=torch.bfloat16, device="cuda")
        oz.ozaki25_expert_layer(X, torch.zeros((tokens, top), dtype=torch.int32, device="cuda"),
                                torch.ones((tokens, top), device="cuda"), up, down, gate=up, Y=Y)
        assert bool((Y == 0).all())
    X = torch.ones((0, 8), dtype=torch.bfloat16, device="cuda")
    up = torch.ones((3, 8, 8), dtype=torch.bfloat16, device="cuda")
    assert oz.ozaki25_expert_layer(X, torch.zeros((0, 2), dtype=torch.int32, device="cuda"), torch.ones((0, 2), device="cuda"),
                                   up, up).shape == (0, 8)


@pytest.mark.parametrize("tokens", [1, 33])
def test_hidden_values_beyond_half(tokens):
    """Hidden values past 65504 whose outputs half holds."""
    import torch
    X = torch.full((tokens, 64), 100.0, dtype=torch.float16, device="cuda")
    up = torch.full((2, 32, 64), 1.0, dtype=torch.float16, device="cuda")
    down = torch.full((2, 16, 32), 2.0 ** -18, dtype=torch.float16, device="cuda")
    Y = oz.ozaki25_expert_layer(X, torch.zeros((tokens, 1), dtype=torch.int32, device="cuda"), torch.ones((tokens, 1), device="cuda"),
                                up, down, gate=up)
    want = 6400.0 * 6400 * 32 * 2.0 ** -18
    assert float((Y.double() - want).abs().max()) <= want * (2.0 ** -11 + 2.0 ** -15)


def test_large_offsets():
    """A stack beyond 2^32 bytes."""
    import torch
    import eight_util as u
    experts, width, inner = 70, 4096, 8192
    up = torch.zeros((experts, inner, width), dtype=torch.bfloat16, device="cuda")
    down = torch.zeros((experts, width, inner), dtype=torch.bfloat16, device="cuda")
    up[69] = u.normal((inner, width), torch.bfloat16, 1, 1 / 64)
    down[69] = u.normal((width, inner), torch.bfloat16, 2, 1 / 90)
    for tokens in (1, 18):
        X = u.normal((tokens, width), torch.bfloat16, 3)
        which = torch.full((tokens, 1), 69, dtype=torch.int32, device="cuda")
        Y = oz.ozaki25_expert_layer(X, which, torch.ones((tokens, 1), device="cuda"), up, down)
        h = X.double() @ up[69].double().t()
        want = (h * torch.sigmoid(h)) @ down[69].double().t()
        assert float((Y.double() - want).norm() / want.norm()) < 2.0 ** -8
