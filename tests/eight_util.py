"""Plain forms, in 64 bits, of the operators with 8-bit operands, and the
tolerances that follow from their stated roundings."""
import torch

BLOCK, TOP, LEAST = 128, 448.0, 2.0 ** -126
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24  # half a step of FP32


def half_step(dtype):
    """What one rounding is off by at most, relative to the value."""
    return torch.finfo(dtype).eps / 2


def padded(t, pad, fill=None):
    """t as a slice of a matrix with `pad` more columns, which hold `fill`."""
    full = torch.empty((*t.shape[:-1], t.shape[-1] + pad), dtype=t.dtype, device=t.device)
    if fill is not None:
        full.fill_(fill)
    full[..., :t.shape[-1]] = t
    return full[..., :t.shape[-1]]


def e4m3_rows(Q, pad, fill=0x7f):
    """An e4m3 matrix in rows with `pad` more bytes, NaN by default."""
    full = torch.full((*Q.shape[:-1], Q.shape[-1] + pad), fill, dtype=torch.uint8, device=Q.device)
    full[..., :Q.shape[-1]] = Q.view(torch.uint8)
    return full.view(E4M3)[..., :Q.shape[-1]]


def normal(shape, dtype, seed, scale=1.0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(shape, device="cuda", generator=gen) * scale
    return padded(t.to(dtype), pad) if pad else t.to(dtype)


def block_scales(X, squares=False):
    """Scales of X (rows x cols) with blocks along the rows, in FP32 as stated:
    [col blocks][rows], or of squares [row blocks][col blocks]."""
    rows, cols = X.shape
    rb, cb = -(-rows // BLOCK), -(-cols // BLOCK)
    full = torch.zeros((rb * BLOCK, cb * BLOCK), dtype=torch.float32, device=X.device)
    full[:rows, :cols] = X.float().abs()
    if squares:
        most = full.reshape(rb, BLOCK, cb, BLOCK).amax((1, 3))
    else:
        most = full[:rows].reshape(rows, cb, BLOCK).amax(2).t()
    s = (most.cpu() / TOP).clamp_min(LEAST)
    s[~torch.isfinite(most.cpu())] = float("nan")
    return s.to(X.device).contiguous()


def spread(s, rows, cols, squares=False):
    """The scales by element, rows x cols."""
    if squares:
        return s.repeat_interleave(BLOCK, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
    return s.t().repeat_interleave(BLOCK, 1)[:, :cols]


def assert_e4m3(Q, V, slack=2 * U):
    """Q is V rounded to e4m3: within half a step (2^-4 of the value, 2^-10 among
    the subnormal numbers) of a value that is off by `slack` at most."""
    q, v = Q.double(), V.double()
    assert torch.equal(torch.isnan(q), torch.isnan(v))
    off = torch.nan_to_num((q - v).abs())
    allowed = torch.nan_to_num(torch.clamp(2.0 ** -4 * v.abs() * (1 + slack), min=2.0 ** -10) + v.abs() * slack)
    worst = off - allowed
    assert bool((worst <= 0).all()), (float(worst.max()), int((worst > 0).sum()))


def quantised(X, squares=False):
    """X (rows x cols) in e4m3 by the stated rule, and its scales."""
    s = block_scales(X, squares)
    return (X.float() / spread(s, *X.shape, squares)).to(E4M3), s
