"""The forms of the norm and of its gradients that only many rows reach, and what is not finite or very small in every form."""
import pytest
import torch

from operator_reference import BLOCK, U32, block_amax, blocks, check_q8, e4m3_rows, rms, rms_rel, scales, spread
from test_gpu_operators import BF16, E4M3, F32, back_case, back_exact, gb, norm_case, randn, rng, status, strided  # noqa: F401  (gb: the fixture)

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


# ------------------------------------------------------------------------------------------------ many rows
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [520, 768, 777, 1000, 1300, 1536, 2001, 2048])
def test_norm_of_many_wide_rows(gb, dtype, cols):
    """A row to a warp, five to sixteen pieces of columns: from 24576 rows on; one row fewer goes to the block's form."""
    for n, out_dtype, kw in ((24_575, E4M3, dict(res=True)), (24_576, E4M3, dict(res=True)), (24_576, F32, {}), (25_001, BF16, dict(res=True, weight=False)),
                             (24_577, E4M3, dict(ids=True, live=24_000, res=True)), (25_000, E4M3, dict(view=1))):
        norm_case(gb, n, cols, dtype, out_dtype, seed=n, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [8, 64, 128, 248, 256, 504, 512, 768, 1000, 1024, 1536])
def test_norm_backward_of_many_rows(gb, dtype, cols):
    """Streams of rows to warps: from some thousand rows of whole 16-byte vectors on, one to six pieces a warp (four with the residual's gradient)."""
    for n, res, kw in ((4735, False, {}), (4736, False, {}), (4736, True, {}), (6001, False, dict(weight=False)), (6001, True, dict(ids=True, live=5000)),
                       (6001, False, dict(ids=True)), (9001, True, dict(want=("dx",))), (9001, False, dict(want=("dw",))), (9001, True, dict(live=1)),
                       (9001, False, dict(live=0)), (20_011, True, {})):
        back_case(gb, n, cols, dtype, res, seed=n, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [128, 500, 512, 1000])
def test_norm_backward_of_many_rows_in_place_and_twice(gb, dtype, cols):
    """dx may be dout or dres where rows are on their way ahead of the results, too; the same call gives the same bits."""
    n, cols = 6001, cols if dtype == F32 else cols // 8 * 8
    x, g, s, w = randn((n, cols), 1, dtype), randn((n, cols), 2, dtype), randn((n, cols), 3, dtype), randn((cols,), 4)
    ws = torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda")
    for res in (True, False):
        got = []
        for into in ("apart", "dout", "dres" if res else "apart", "apart"):
            a, b, dw = g.clone(), s.clone(), torch.empty(cols, device="cuda")
            dx = {"apart": torch.empty_like(x), "dout": a, "dres": b}[into]
            gb.gear_rms_norm_backward(x, w, a, dx, dw, ws, dres=b if res else None)
            got.append((dx, dw))
        for dx, dw in got[1:]:
            assert torch.equal(dx, got[0][0]) and torch.equal(dw, got[0][1])


# ------------------------------------------------------------------------------------------------ not finite, very small
# rows, columns: a warp to a row of one piece, a block to a few rows, a block of two pieces a warp, a warp to a row of several pieces, the wide form;
# with rows of whole vectors and without
FORMS = [(40, 128), (40, 90), (40, 1000), (40, 1001), (3000, 1536), (2000, 512), (2000, 513), (25_000, 1000), (25_000, 1001), (6, 9000), (6, 33_000)]


def odd_rows(n, cols, dtype, seed):
    """Rows with a NaN, an infinity, both, a block that is very small, one that is smaller still, a block of zeros; the last rows are usual."""
    x = randn((n, cols), seed, dtype)
    last = (cols - 1) // BLOCK * BLOCK
    x[0, cols - 1], x[1, 5], x[2, 3] = NAN, INF, -INF
    x[2, cols - 2] = NAN
    x[3, last:] = x[3, last:] * 1e-29             # above 2^-100, below 2^-90
    x[4, last:] = x[4, last:] * 1e-35             # below 2^-100
    if n > 6:
        x[5, last:] = 0
    return x


def check_odd(got, scale, h, rel, out_dtype):
    """Values against the 64-bit h, whose NaN are as the definition has them."""
    nan = h.isnan()
    if out_dtype != E4M3:
        assert torch.equal(got.isnan(), nan)
        h0 = torch.where(nan, torch.zeros_like(h), h)
        off = (torch.where(nan, torch.zeros_like(got), got).double() - h0).abs()
        u = 0 if out_dtype == F32 else 2.0 ** -8
        # (bf16: below 2^-126 half of the smallest number)
        assert (off <= h0.abs() * ((1 + rel * 1.01) * (1 + u) - 1) + (2.0 ** -134 if u else 1e-44)).all()
        return
    bad = block_amax(nan.double()) > 0            # a block with a NaN: a NaN for its scale and in all its values
    where = spread(bad, h.shape[1])
    assert torch.equal(scale.isnan(), bad)
    assert torch.equal(got.float().isnan(), where)
    z = torch.where(where, torch.zeros_like(h), h)
    check_q8(torch.where(where, torch.zeros((), device="cuda"), got.float()), torch.where(bad, scales(z).float(), scale), z, rel)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,cols", FORMS)
def test_norm_of_what_is_not_finite(gb, n, cols, dtype):
    """With and without a residual, its sum kept or not (in place too), rows by ID: every way the out-of-line form makes a value again."""
    w = 1 + 0.3 * randn((cols,), 2)
    x, r = odd_rows(n, cols, dtype, 1), randn((n, cols), 3, dtype)
    r[3, (cols - 1) // BLOCK * BLOCK:] = 0
    r[4, (cols - 1) // BLOCK * BLOCK:] = 0
    if n > 6:
        r[5, (cols - 1) // BLOCK * BLOCK:] = 0
    eps, rel = 1e-5, rms_rel(cols)
    total = (x.float() + r.float()).to(dtype)     # (rounded once: the sum of two bf16 values is rounded to fp32 only below what bf16 keeps)
    back = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    for out_dtype in (E4M3, F32, BF16):
        for res, kept, ids in ((False, "no", False), (True, "no", False), (True, "apart", False), (True, "res", False), (True, "x", False), (False, "apart", True),
                               (True, "no", True)):
            a, b = x.clone(), r.clone()
            t = {"no": None, "apart": torch.empty_like(x), "res": b, "x": a}[kept]
            out = e4m3_rows(n, cols) if out_dtype == E4M3 else torch.empty((n, cols), dtype=out_dtype, device="cuda")
            scale = torch.empty((n, blocks(cols)), device="cuda") if out_dtype == E4M3 else None
            st = status()
            rows = x.flip(0) if ids else x
            gb.gear_rms_norm(rows.contiguous() if ids else a, w, out, scale, eps, res=b if res else None, res_out=t, ids=back if ids else None, status=st)
            y = total if res else x
            if t is not None:
                assert torch.equal(t.nan_to_num(7.0), y.nan_to_num(7.0)) and torch.equal(t.isnan(), y.isnan())
            h = y.double() * rms(y.double(), eps) * w.double()
            check_odd(out, scale, h, rel, out_dtype)
            assert st.tolist() == [0, 0]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,cols", [(40, 128), (40, 90), (40, 1000), (40, 1001), (6000, 128), (6000, 1000), (5000, 1001), (6, 9000), (6, 33_000)])
@pytest.mark.parametrize("res", [False, True])
def test_gradients_of_what_is_not_finite(gb, n, cols, dtype, res):
    """A NaN or an infinity in a row, in its gradient, in the residual's: NaN and infinities where the formula has them, the other rows as they are."""
    x, g, s = randn((n, cols), 1, dtype), randn((n, cols), 2, dtype), randn((n, cols), 3, dtype) if res else None
    w = 1 + 0.3 * randn((cols,), 4)
    x[0, 3], x[1, cols - 1], g[2, 5], g[3, 0] = NAN, INF, NAN, -INF
    if res:
        s[4, 7], s[4, 8] = NAN, INF
    eps, dx, dw = 1e-4, torch.empty_like(x), torch.empty(cols, device="cuda")
    gb.gear_rms_norm_backward(x, w, g, dx, dw, torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda"), eps, dres=s)
    want, dw64 = back_exact(x, w, g, eps, s)
    assert torch.equal(dx.isnan(), want.isnan()) and torch.equal(dx.isinf(), want.isinf())
    assert torch.equal(torch.sign(dx[dx.isinf()]).double(), torch.sign(want[want.isinf()]))
    k = cols / 32 + 16
    xd, gd = x[5:].double(), (g[5:].double() * w.double())
    r = rms(xd, eps)
    size = gd.abs() * r + xd.abs() * r ** 3 * (gd * xd).abs().mean(1, keepdim=True) + (0 if s is None else s[5:].double().abs())
    allowed = size * (3 * rms_rel(cols) + (k + 8) * U32) + (0 if dtype == F32 else want[5:].abs() * 2.0 ** -8 * 1.01) + 1e-44
    assert ((dx[5:].double() - want[5:]).abs() <= allowed).all()
    assert torch.equal(dw.isnan(), dw64.isnan()) and dw.isnan().all()      # (the row with a NaN has a factor of NaN)
    x[0, 3] = 1.0                                  # without it: the columns' own
    gb.gear_rms_norm_backward(x, w, g, None, dw, torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda"), eps)
    dw64 = back_exact(x, w, g, eps, None)[1]
    assert torch.equal(dw.isnan(), dw64.isnan()) and torch.equal(dw.isinf(), dw64.isinf())
    assert dw.isnan().sum() == 2 and dw.isinf().sum() == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,cols", [(3, 64), (40, 1000), (40, 1001), (6000, 128), (6000, 1000), (6, 33_000)])
def test_gradients_of_very_small_rows(gb, n, cols, dtype):
    """Rows of zeros and of 1e-20 with an eps below what fp32 squares keep: r is 2e19 and more, its square beyond fp32, the gradients are not."""
    g, w, ws = randn((n, cols), 1, dtype), 1 + 0.3 * randn((cols,), 2), torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda")
    for x, eps in ((torch.zeros((n, cols), dtype=dtype, device="cuda"), 1e-40), (randn((n, cols), 3, dtype) * 4e-20, 0.0), (randn((n, cols), 3, dtype) * 4e-20, 1e-39)):
        eps = float(torch.tensor(eps, dtype=F32))
        dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
        gb.gear_rms_norm_backward(x, w, g, dx, dw, ws, eps)
        want, dw64 = back_exact(x, w, g, eps, None)
        xd, gd = x.double(), g.double() * w.double()
        r = rms(xd, eps)
        # beside the roundings of rows of usual size: what lies below 2^-126 is a multiple of 2^-149, off by 2^-150.  A sum of cols squares and of
        # the lanes' and warps' sums (64 and fewer) has that for each, so their mean is off by (1 + 64 / cols) 2^-150, and by 2^-150 each for the product with 1 / cols and
        # for eps, relative to mean + eps = 1 / r^2; half of it goes into r, which dx has to the third power.
        k = cols / 32 + 16
        small = (3 + 64 / cols) * 2.0 ** -150 * r ** 2
        size = gd.abs() * r + xd.abs() * r ** 3 * (gd * xd).abs().mean(1, keepdim=True)
        allowed = size * (3 * rms_rel(cols) + (k + 8) * U32 + 1.6 * small) + (0 if dtype == F32 else want.abs() * 2.0 ** -8 * 1.01)
        assert ((dx.double() - want).abs() <= allowed).all()
        size = (g.double() * xd).abs() * r
        assert ((dw.double() - dw64).abs() <= (size * (rms_rel(cols) + (n / 592 + 110) * U32 + 0.6 * small)).sum(0) + 1e-44).all()


# ------------------------------------------------------------------------------------------------ the 8-bit quotient
def to_e4m3(x):
    """64-bit values of at most 448 rounded once to e4m3 (nearest, ties to even): steps of 2^(exponent - 3), 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


@pytest.mark.parametrize("dtype,cols", [(F32, 1536), (F32, 1001), (BF16, 1536)])
def test_quotients_are_rounded_as_divisions_are(gb, dtype, cols):
    """The quotient v / (largest / 448) is rounded to fp32 once, half a step or 2^-24 of it, and then to e4m3: a value differs from the quotient
    rounded to e4m3 at once only where the quotient lies that near to the middle between two e4m3 values.  What the quotient's correction itself
    leaves: its remainder, 2^-22 of the value, comes with roundings of 2^-24 and a reciprocal off by 2^-23, so 2^-44; the factor 1 + 2^-8 is more."""
    off = 0
    for seed in range(8):
        n = 1000
        x = (randn((n, cols), seed) * torch.logspace(-12, 12, n, device="cuda")[:, None]).to(dtype)
        q, s = e4m3_rows(n, cols), torch.empty((n, blocks(cols)), device="cuda")
        gb.gear_q8_rows(x, q, s)
        exact = x.double() * 448 / spread(block_amax(x.double()), cols)
        want, got = to_e4m3(exact), q.double()
        differs = want != got
        middle = (want + got) / 2
        assert ((exact - middle).abs()[differs] <= exact.abs()[differs] * U32 * (1 + 2.0 ** -8)).all()
        off += int(differs.sum())
    assert off < 1e-4 * 8 * 1000 * cols           # (the share of values so near to a middle: 2^-24 against a spacing of 2^-3 to 2^-4)
