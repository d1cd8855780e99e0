"""The operators of the 8-bit Dense Part and of gradient clipping from their definitions, in 64 bits, and what the kernels may be
off by: every bound counts roundings (u = 2^-24 for fp32, 2^-8 for bf16, half a step for e4m3)."""
import torch

U32, UBF = 2.0 ** -24, 2.0 ** -8
BLOCK, TINY = 128, 2.0 ** -100


def u_of(dtype):
    return {torch.float32: U32, torch.bfloat16: UBF}[dtype]


def blocks(K):
    return (K + BLOCK - 1) // BLOCK


def e4m3_rows(n, K, device="cuda", fill=None):
    """n rows of K e4m3 values whose starts are multiples of 16 bytes; what lies between K and the next row is `fill`."""
    ld = (K + 15) // 16 * 16
    t = torch.zeros((n, ld), dtype=torch.uint8, device=device)
    if fill is not None:
        t.fill_(fill)
    return t.view(torch.float8_e4m3fn)[:, :K]


def block_amax(h):
    n, K = h.shape
    pad = torch.zeros((n, blocks(K) * BLOCK), dtype=h.dtype, device=h.device)
    pad[:, :K] = h
    return pad.view(n, blocks(K), BLOCK).abs().amax(2)


def scales(h):
    return block_amax(h).clamp_min(TINY) / 448


def spread(s, K):
    return s.repeat_interleave(BLOCK, 1)[:, :K]


def check_q8(q, scale, h, rel):
    """q, scale against the 64-bit rows h, of which the kernel's own fp32 ones are within rel: the scale is that of a value within rel,
    divided with one rounding; a value is off by half an e4m3 step of the quotient (2^-4 relative, 2^-10 at least), which itself is
    within rel and three roundings (the scale, its reciprocal, the product)."""
    q, scale, s = q.double(), scale.double(), scales(h)
    assert ((scale - s).abs() <= s * (rel + 2 * U32) * 1.01).all()
    off = (q * spread(scale, h.shape[1]) - h).abs()
    half = torch.maximum(h.abs() * 2.0 ** -4, spread(s, h.shape[1]) * 2.0 ** -10)
    allowed = half * (1 + 2.0 ** -10) + h.abs() * (rel + 4 * U32) * 1.1
    assert (off <= allowed).all(), float((off / allowed).max())


def rms(y, eps):
    return 1.0 / torch.sqrt((y * y).mean(1, keepdim=True) + eps)


def rms_rel(cols):
    """h = y r w in fp32: the sum of squares adds at most cols / 32 + 16 terms one after the other (a lane's, then trees), each with a
    rounding, relative to a sum without cancellation; half of that goes into r, with four roundings for mean, eps, root and quotient; two
    products more."""
    return ((cols / 32 + 16) / 2 + 6) * U32
