"""Gradient clipping, RMS norm and its gradients, 8-bit rows, weights and products on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

from operator_reference import (BLOCK, U32, blocks, block_amax, check_q8, e4m3_rows, rms, rms_rel, scales, spread, u_of)

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def gb():
    from paper_1806_03925_b200 import build
    build.build()
    from paper_1806_03925_b200 import binding
    binding.load()
    return binding


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=rng(seed), device="cuda").to(dtype)


def status():
    return torch.zeros(2, dtype=torch.int32, device="cuda")


def strided(t, gap=8, start=0):
    """The same rows inside wider ones, `start` values behind a 16-byte boundary."""
    n, c = t.shape
    wide = torch.full((n, c + gap + start), float("nan"), dtype=t.dtype, device=t.device)
    v = wide[:, start:start + c]
    v.copy_(t)
    return v


# ------------------------------------------------------------------------------------------------ norm
def norm_case(gb, n, cols, dtype, out_dtype, res=False, ids=False, weight=True, live=None, view=0, seed=0, eps=1e-5):
    V = n + 7 if ids else n
    x = randn((V, cols), seed, dtype) * 3
    if n > 2 and not ids:
        x[1] = 0                                    # a row of zeros
    r = randn((n, cols), seed + 1, dtype) if res else None
    w = 1 + 0.3 * randn((cols,), seed + 2) if weight else None
    idx = None
    if ids:
        idx = torch.randint(0, V, (n,), generator=rng(seed + 3), device="cuda", dtype=torch.int32)
        idx[0] = V                                  # one behind the table: a row of zeros
        if n > 3:
            idx[3] = idx[2]
    if view:
        x, r = strided(x, 8, view), None if r is None else strided(r, 8, view)
    st, d_n = status(), None if live is None else torch.tensor([live], dtype=torch.int64, device="cuda")
    out = e4m3_rows(n, cols, fill=0x31) if out_dtype == E4M3 else torch.full((n, cols), 77.0, dtype=out_dtype, device="cuda")
    scale = torch.full((n, blocks(cols)), 55.0, device="cuda") if out_dtype == E4M3 else None
    total = torch.full((n, cols), 33.0, dtype=dtype, device="cuda") if res else None
    gb.gear_rms_norm(x, w, out, scale, eps, res=r, res_out=total, ids=idx, d_n=d_n, status=st)
    m = n if live is None else max(0, min(n, live))
    xs = x.double()
    if ids:
        ok = (idx >= 0) & (idx < V)
        xs = torch.where(ok[:, None], xs[idx.long().clamp(0, V - 1)], torch.zeros((), dtype=torch.float64, device="cuda"))
        assert st.tolist() == [gb.GEAR_DEV_BAD_ID if m > 0 else 0, 0]
    else:
        assert st.tolist() == [0, 0]
    if res:
        # the sum, rounded once: within half a step, u relative (the sum of two values of a type is exact in 64 bits but for terms 2^29 and
        # more below the larger one); the norm is that of the kept sum
        exact = xs + r.double()
        assert ((total[:m].double() - exact[:m]).abs() <= exact[:m].abs() * u_of(dtype) * (1 + 2.0 ** -20)).all() and (total[m:] == 33.0).all()
        xs = torch.cat([total[:m].double(), exact[m:]])
    h = xs * rms(xs, eps) * (1 if w is None else w.double())
    rel = rms_rel(cols)
    if out_dtype == E4M3:
        check_q8(out[:m], scale[:m], h[:m], rel)
        assert (scale[m:] == 55.0).all() and (out.view(torch.uint8)[m:] == 0x31).all()
    else:
        u = 0 if out_dtype == F32 else u_of(BF16)
        assert ((out[:m].double() - h[:m]).abs() <= h[:m].abs() * ((1 + rel * 1.01) * (1 + u) - 1) + 1e-44).all()
        assert (out[m:] == 77.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("out_dtype", [E4M3, BF16, F32])
@pytest.mark.parametrize("n,cols", [(1, 1), (1, 1536), (3, 8), (5, 127), (33, 128), (7, 129), (64, 512), (9, 520), (2, 2048), (11, 2056), (3, 8192), (2, 8200), (2, 20001),
                                    (1500, 200), (1300, 1001), (1301, 2048)])
def test_norm(gb, n, cols, dtype, out_dtype):
    norm_case(gb, n, cols, dtype, out_dtype, res=cols % 2 == 0, weight=cols != 512)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [64, 200, 1536, 2100, 9001])
def test_norm_by_id_with_live_count(gb, dtype, cols):
    for n, live in ((40, 23), (40, 0), (40, 100), (40, -3), (1400, 1399)):
        norm_case(gb, n, cols, dtype, E4M3, res=True, ids=True, live=live, seed=n + live)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("view", [1, 4, 8])
def test_norm_of_views(gb, dtype, view):
    for n, cols in ((6, 136), (1400, 264), (6, 9000)):
        norm_case(gb, n, cols, dtype, E4M3, res=True, view=view, seed=view)
        norm_case(gb, n, cols, dtype, BF16, view=view, seed=view + 1)


@pytest.mark.parametrize("cols", [96, 1024, 4096, 12000])
def test_norm_keeps_the_residual_stream_in_place(gb, cols):
    """res_out may be res, or x itself."""
    x, r = randn((50, cols), 1, BF16), randn((50, cols), 2, BF16)
    total = (x.float() + r.float()).to(BF16)
    outs = []
    for into in ("apart", "res", "x"):
        a, b = x.clone(), r.clone()
        o, t = torch.empty((50, cols), device="cuda"), {"apart": torch.empty_like(x), "res": b, "x": a}[into]
        gb.gear_rms_norm(a, None, o, eps=1e-5, res=b, res_out=t)
        assert torch.equal(t, total)
        outs.append(o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    copy = torch.empty_like(x)                      # a copy of the rows without a residual
    gb.gear_rms_norm(x, None, outs[0], res_out=copy)
    assert torch.equal(copy, x)


@pytest.mark.parametrize("cols", [130, 1024, 9000])
def test_q8_rows_and_what_is_not_finite(gb, cols):
    """Rows of all magnitudes; a block with an infinity or a NaN, alone or together; the others keep their values."""
    n = 12
    x = randn((n, cols), 5) * torch.logspace(-30, 30, n, device="cuda")[:, None]
    x[2] = 0
    x[3] = 1e-42                                    # below 2^-100: a scale of its own
    q, s = e4m3_rows(n, cols), torch.empty((n, blocks(cols)), device="cuda")
    gb.gear_q8_rows(x, q, s)
    check_q8(q, s, x.double(), 0.0)
    assert (q[2].float() == 0).all() and (s[2] == torch.tensor(2.0 ** -100 / 448, device="cuda")).all()
    inf, nan = float("inf"), float("nan")
    y = randn((4, cols), 6)
    y[0, 5], y[1, 7], y[2, 3], y[2, 9], y[3, cols - 1] = inf, nan, -inf, nan, nan
    q, s = e4m3_rows(4, cols), torch.empty((4, blocks(cols)), device="cuda")
    gb.gear_q8_rows(y, q, s)
    last = blocks(cols) - 1
    assert s[0, 0] == inf and s[1, 0].isnan() and s[2, 0].isnan() and s[3, last].isnan()
    v = q.float()
    assert v[0, 5].isnan() and (v[0, :5] == 0).all() and (v[0, 6:BLOCK] == 0).all()
    assert v[1, :BLOCK].isnan().all() and v[2, :BLOCK].isnan().all() and v[3, last * BLOCK:].isnan().all()
    fine = torch.ones((4, blocks(cols)), dtype=torch.bool, device="cuda")
    fine[:3, 0] = False
    fine[3, last] = False
    keep = spread(fine, cols)
    z = torch.where(keep, y, torch.zeros((), device="cuda"))
    check_q8(torch.where(keep, v, torch.zeros((), device="cuda")), torch.where(fine, s, scales(z.double()).float()), z.double(), 0.0)


# ------------------------------------------------------------------------------------------------ its gradients
def back_exact(x, w, g, eps, dres):
    x, g = x.double(), g.double()
    r, wg = rms(x, eps), g * (1 if w is None else w.double())
    dx = r * wg - x * r ** 3 * (wg * x).mean(1, keepdim=True)
    return dx if dres is None else dx + dres.double(), (g * x * r).sum(0)


def back_case(gb, n, cols, dtype, res, weight=True, ids=False, live=None, view=0, want=("dx", "dw"), eps=1e-4, seed=0):
    V = n + 5 if ids else n
    x, g = randn((V, cols), seed, dtype) * 2, randn((n, cols), seed + 1, dtype)
    if n > 2 and not ids:
        x[1] = 0
    w = 1 + 0.3 * randn((cols,), seed + 2) if weight else None
    dres = randn((n, cols), seed + 3, dtype) if res else None
    idx = None
    if ids:
        idx = torch.randint(0, V, (n,), generator=rng(seed + 4), device="cuda", dtype=torch.int32)
        idx[n - 1] = -1
    if view:
        x, g, dres = strided(x, 8, view), strided(g, 8, view), None if dres is None else strided(dres, 8, view)
    dx = torch.full((n, cols), 7.0, dtype=dtype, device="cuda") if "dx" in want else None
    dw = torch.full((cols,), 9.0, device="cuda") if "dw" in want else None
    ws = torch.full((gb.GEAR_NORM_WORKSPACE_ROWS, cols), float("nan"), device="cuda") if "dw" in want else None
    d_n, st = None if live is None else torch.tensor([live], dtype=torch.int64, device="cuda"), status()
    gb.gear_rms_norm_backward(x, w, g, dx, dw, ws, eps, dres=dres, ids=idx, d_n=d_n, status=st)
    m = n if live is None else max(0, min(n, live))
    xs = x
    if ids:
        ok = (idx >= 0) & (idx < V)
        xs = torch.where(ok[:, None], x[idx.long().clamp(0, V - 1)], torch.zeros((), dtype=dtype, device="cuda"))
    dx64, dw64 = back_exact(xs[:m], w, g[:m], eps, None if dres is None else dres[:m])
    xd, gd = xs[:m].double(), g[:m].double()
    r, wd = rms(xd, eps), 1 if w is None else w.double()
    if dx is not None:
        # the two terms of dx with their own roundings: r as in the norm; the sum of g y is off by (its terms one after the other) times the sum of
        # magnitudes; then the output's rounding
        k = cols / 32 + 16
        size = (gd * wd).abs() * r + xd.abs() * r ** 3 * (gd * wd * xd).abs().mean(1, keepdim=True) + (0 if dres is None else dres[:m].double().abs())
        allowed = size * (3 * rms_rel(cols) + (k + 8) * U32) + (0 if dtype == F32 else dx64.abs() * u_of(BF16) * 1.01) + 1e-44
        assert ((dx[:m].double() - dx64).abs() <= allowed).all()
        assert (dx[m:] == 7.0).all()
    if dw is not None:
        size = (gd * xd).abs() * r
        # a lane's rows one after the other, then warps and blocks: fewer than the rows / 592 + 592 / 8 + 32 terms
        allowed = size.sum(0) * (rms_rel(cols) + (m / 592 + 74 + 32 + 4) * U32) + 1e-44
        assert ((dw.double() - dw64).abs() <= allowed).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,cols", [(1, 1), (1, 1536), (5, 127), (33, 128), (7, 129), (2500, 512), (9, 520), (3, 2048), (11, 2056), (3, 8192), (4, 8200), (700, 9001),
                                    (2600, 200), (1300, 1001), (2601, 2048), (3000, 101)])
def test_norm_backward(gb, n, cols, dtype):
    back_case(gb, n, cols, dtype, res=cols % 2 == 0, weight=cols != 512)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [64, 203, 1536, 9001])
def test_norm_backward_by_id_views_and_parts(gb, dtype, cols):
    for live in (0, 17, 100):
        back_case(gb, 40, cols, dtype, True, ids=True, live=live, seed=live)
    back_case(gb, 40, cols, dtype, True, view=1)
    back_case(gb, 1400, cols, dtype, False, view=8)
    back_case(gb, 40, cols, dtype, True, want=("dx",))
    back_case(gb, 40, cols, dtype, False, want=("dw",))
    dw, ws = torch.full((cols,), 9.0, device="cuda"), torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda")
    x = randn((4, cols), 1, dtype)
    gb.gear_rms_norm_backward(x, None, x, None, dw, ws, n=0)
    assert (dw == 0).all()                           # no rows: a sum of nothing


def test_norm_backward_in_place_and_twice(gb):
    """dx may be dout or dres; the same call gives the same bits."""
    n, cols = 3001, 1000
    x, g, s, w = randn((n, cols), 1), randn((n, cols), 2), randn((n, cols), 3), randn((cols,), 4)
    ws = torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda")
    got = []
    for into in ("apart", "dout", "dres", "apart"):
        a, b, dw = g.clone(), s.clone(), torch.empty(cols, device="cuda")
        dx = {"apart": torch.empty_like(x), "dout": a, "dres": b}[into]
        gb.gear_rms_norm_backward(x, w, a, dx, dw, ws, dres=b)
        got.append((dx, dw))
    for dx, dw in got[1:]:
        assert torch.equal(dx, got[0][0]) and torch.equal(dw, got[0][1])


def test_norm_gradient_against_differences(gb):
    """d loss / d x and d loss / d weight of loss = sum(c h), by central differences of the 64-bit definition."""
    n, cols, eps = 3, 40, 1e-3
    x, c, w = randn((n, cols), 1), randn((n, cols), 2), 1 + 0.2 * randn((cols,), 3)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    gb.gear_rms_norm_backward(x, w, c, dx, dw, torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, cols), device="cuda"), eps)

    def loss(x, w):
        return float((c.double() * x * rms(x, eps) * w).sum())
    step = 1e-5                                      # error step^2 times third derivatives (below 100 here) and rounding 2^-53 / step * loss
    for i, j in ((0, 0), (1, 17), (2, 39)):
        e = torch.zeros((n, cols), dtype=torch.float64, device="cuda")
        e[i, j] = step
        assert abs((loss(x.double() + e, w.double()) - loss(x.double() - e, w.double())) / (2 * step) - float(dx[i, j])) < 2e-5
        f = torch.zeros(cols, dtype=torch.float64, device="cuda")
        f[j] = step
        assert abs((loss(x.double(), w.double() + f) - loss(x.double(), w.double() - f)) / (2 * step) - float(dw[j])) < 2e-5


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("K,N", [(1, 1), (16, 8), (128, 128), (129, 127), (200, 300), (1536, 64), (37, 1024)])
def test_weights(gb, K, N):
    W = strided(randn((K, N), 1) * torch.logspace(-3, 3, N, device="cuda"), 5)
    q, s, qt, st = e4m3_rows(N, K), torch.empty((blocks(N), blocks(K)), device="cuda"), e4m3_rows(K, N), torch.empty((blocks(K), blocks(N)), device="cuda")
    gb.gear_q8_weights(W, q, s, qt, st)
    assert torch.equal(s, st.t()) and torch.equal(q.float(), qt.float().t())
    # rows of a block of 128 share the largest of their scales
    row = block_amax(W.t().double().contiguous())
    pad = torch.zeros((blocks(N) * BLOCK, blocks(K)), dtype=torch.float64, device="cuda")
    pad[:N] = row
    want = pad.view(blocks(N), BLOCK, blocks(K)).amax(1).clamp_min(2.0 ** -100) / 448
    assert ((s.double() - want).abs() <= want * 2 * U32).all()
    wide, h = spread(s.double().repeat_interleave(BLOCK, 0)[:N], K), W.t().double()
    assert ((q.double() * wide - h).abs() <= torch.maximum(h.abs() * 2.0 ** -4, wide * 2.0 ** -10) * (1 + 2.0 ** -10) + h.abs() * 5 * U32).all()
    only, only_s = e4m3_rows(N, K), torch.empty_like(s)
    gb.gear_q8_weights(W, only, only_s)
    assert torch.equal(only.float(), q.float()) and torch.equal(only_s, s)
    only_t, only_st = e4m3_rows(K, N), torch.empty_like(st)
    gb.gear_q8_weights(W, q_t=only_t, scale_t=only_st)
    assert torch.equal(only_t.float(), qt.float()) and torch.equal(only_st, st)


@pytest.mark.parametrize("K,N", [(1, 8_400_001), (130, 8_388_500), (8_400_001, 1)])
def test_weights_with_one_side_very_long(gb, K, N):
    """More than 65535 blocks of 128 along a side."""
    W = randn((K, N), 1)
    q, s, qt, st = e4m3_rows(N, K), torch.empty((blocks(N), blocks(K)), device="cuda"), e4m3_rows(K, N), torch.empty((blocks(K), blocks(N)), device="cuda")
    gb.gear_q8_weights(W, q, s, qt, st)
    assert torch.equal(s, st.t())
    for k0, n0 in ((0, 0), (0, max(0, (N - 1) // BLOCK * BLOCK)), (max(0, (K - 1) // BLOCK * BLOCK), 0), (K // 2 // BLOCK * BLOCK, N // 2 // BLOCK * BLOCK)):
        w, b, t = W[k0:k0 + BLOCK, n0:n0 + BLOCK].double(), q[n0:n0 + BLOCK, k0:k0 + BLOCK].double(), qt[k0:k0 + BLOCK, n0:n0 + BLOCK].double()
        scale, want = float(s[n0 // BLOCK, k0 // BLOCK]), float(w.abs().max()) / 448
        assert abs(scale - want) <= want * 2 * U32 and torch.equal(b, t.t())
        assert ((t * scale - w).abs() <= torch.maximum(w.abs() * 2.0 ** -4, torch.tensor(scale * 2.0 ** -10, device="cuda")) * (1 + 2.0 ** -10) + w.abs() * 5 * U32).all()


# ------------------------------------------------------------------------------------------------ products
def q8_data(n, K, N, seed, fill=0x7f):
    """Random operands; what lies behind K in a row is NaN, which no result may see."""
    a, b = e4m3_rows(n, K, fill=fill), e4m3_rows(N, K, fill=fill)
    a.copy_((randn((n, K), seed) * 60).clamp(-448, 448).to(E4M3))
    b.copy_((randn((N, K), seed + 1) * 60).clamp(-448, 448).to(E4M3))
    sa = torch.exp(randn((n, blocks(K)), seed + 2)) * 1e-2
    sb = torch.exp(randn((blocks(N), blocks(K)), seed + 3)) * 1e-2
    return a, sa, b, sb


def product_exact(a, sa, b, sb):
    N, K = b.shape
    A = a.double() * spread(sa.double(), K)
    B = b.double() * spread(sb.double().repeat_interleave(BLOCK, 0)[:N], K)
    return A @ B.t(), A.abs() @ B.abs().t()


def check_product(out, a, sa, b, sb):
    want, size = product_exact(a, sa, b, sb)
    K = b.shape[1]
    # a block's 128 products are exact and added one after the other in fp32 (each addition at most one unit in the last place of what has
    # been added up in magnitude: 2^-23), then one product of scales, one multiply-add per block
    allowed = size * (min(K, 128) + blocks(K) + 4) * 2.0 ** -23 + want.abs() * (0 if out.dtype == F32 else u_of(BF16) * 1.01) + 1e-44
    off = (out.double() - want).abs()
    assert (off <= allowed).all(), float((off / allowed).max())


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,N", [(1, 1, 1), (1, 1536, 64), (2, 16, 8), (3, 100, 33), (4, 2048, 130), (7, 513, 65), (8, 128, 256), (9, 128, 64), (9, 1, 1), (100, 1000, 200),
                                   (128, 256, 64), (129, 129, 129), (130, 17, 300), (300, 640, 72), (1000, 48, 1000), (3001, 200, 1000), (5000, 384, 257),
                                   (20000, 144, 520), (40000, 1040, 256), (8, 300, 2000), (1, 200, 10000), (70, 77, 16), (1100, 500, 5)])
def test_product(gb, n, K, N, out_dtype):
    a, sa, b, sb = q8_data(n, K, N, n + K + N)
    st, out = status(), torch.full((n, N), 5.0, dtype=out_dtype, device="cuda")
    gb.gear_q8_matmul(a, sa, b, sb, out, st)
    assert st.tolist() == [0, 0]
    check_product(out, a, sa, b, sb)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,N", [(131_072, 16, 64), (131_072, 64, 64), (131_072, 128, 64), (100_003, 130, 36), (90_001, 256, 20), (200_000, 128, 52), (60_000, 16, 128),
                                   (150_000, 40, 100), (80_000, 128, 256)])
def test_product_many_tiles_a_block(gb, n, K, N, out_dtype):
    """Several row tiles to every CTA at one or two blocks of K: a tile's results are put together while those of the one before it are
    still leaving.  All rows, three times the same bits."""
    a, sa, b, sb = q8_data(n, K, N, n + K + N)
    st, outs = status(), [torch.full((n, N), 5.0, dtype=out_dtype, device="cuda") for _ in range(3)]
    for o in outs:
        gb.gear_q8_matmul(a, sa, b, sb, o, st)
    assert st.tolist() == [0, 0]
    check_product(outs[0], a, sa, b, sb)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("n,N", [(6, 72), (500, 64), (500, 1000), (30000, 256)])
def test_product_rows_behind_the_live_ones(gb, n, N):
    """d_n on the device; rows behind it, columns beside the output and a row's misaligned start."""
    K = 272
    a, sa, b, sb = q8_data(n, K, N, 3)
    for out_dtype in (F32, BF16):
        for live in (0, 1, n // 2 + 1, n, n + 9, -1):
            d_n, st = torch.tensor([live], dtype=torch.int64, device="cuda"), status()
            wide = torch.full((n, N + 7), 5.0, dtype=out_dtype, device="cuda")
            gb.gear_q8_matmul(a, sa, b, sb, wide[:, 3:3 + N], st, d_n=d_n)
            m = max(0, min(n, live))
            assert (wide[m:] == 5.0).all() and (wide[:, :3] == 5.0).all() and (wide[:, 3 + N:] == 5.0).all()
            if m:
                check_product(wide[:m, 3:3 + N], a[:m], sa[:m], b, sb)


def test_product_of_what_is_not_finite(gb):
    """A row with a NaN or an infinite scale is its own loss; a weight's NaN is its column's."""
    for n in (5, 200):
        a, sa, b, sb = q8_data(n, 300, 70, 9)
        a.view(torch.uint8)[2, 7] = 0x7f
        sa[3, 1] = float("inf")
        b.view(torch.uint8)[11, 4] = 0xff
        out = torch.empty((n, 70), device="cuda")
        gb.gear_q8_matmul(a, sa, b, sb, out, status())
        bad = torch.zeros((n, 70), dtype=torch.bool, device="cuda")
        bad[2:4], bad[:, 11] = True, True
        assert out[2].isnan().all() and out[:, 11].isnan().all() and (~out[3].isfinite()).all()
        keep = [i for i in range(70) if i != 11]
        rows = [i for i in range(n) if i not in (2, 3)]
        assert out[~bad].isfinite().all()
        b2 = b.view(torch.uint8).clone()
        b2[11] = 0
        want, size = product_exact(a[rows], sa[rows], b2.view(E4M3), sb)
        off = (out[rows][:, keep].double() - want[:, keep]).abs()
        assert (off <= size[:, keep] * 135 * 2.0 ** -23).all()


@pytest.mark.parametrize("n", [1, 3, 8])
def test_product_of_rows_that_end_with_their_memory(gb, n):
    """Every remainder of K by 16, in tensors that end with the last row's last value, and with NaN behind every row."""
    for K in list(range(1, 18)) + [100, 127, 499, 1535]:
        N, ld = 40, (K + 15) // 16 * 16
        a, sa, b, sb = q8_data(n, K, N, K)
        ends = [torch.full(((t.shape[0] - 1) * ld + K,), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3).as_strided(t.shape, (ld, 1)) for t in (a, b)]
        ends[0].copy_(a)
        ends[1].copy_(b)
        out, same = torch.full((n, N), 5.0, device="cuda"), torch.full((n, N), 6.0, device="cuda")
        gb.gear_q8_matmul(ends[0], sa, ends[1], sb, out, status())
        gb.gear_q8_matmul(a, sa, b, sb, same, status())
        check_product(out, a, sa, b, sb)
        assert torch.equal(out, same)


def test_product_repeats(gb):
    a, sa, b, sb = q8_data(7000, 1536, 256, 21)
    outs = [torch.empty((7000, 256), device="cuda") for _ in range(3)]
    for o in outs:
        gb.gear_q8_matmul(a, sa, b, sb, o, status())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_product_one_row_does_not_depend_on_its_neighbours(gb):
    """The paths for few and for many rows agree to their roundings."""
    a, sa, b, sb = q8_data(300, 1000, 200, 31)
    many = torch.empty((300, 200), device="cuda")
    gb.gear_q8_matmul(a, sa, b, sb, many, status())
    for n in (1, 2, 4, 8):
        few = torch.empty((n, 200), device="cuda")
        gb.gear_q8_matmul(a, sa, b, sb, few, status())
        check_product(few, a[:n], sa[:n], b, sb)
        check_product(many[:n], a[:n], sa[:n], b, sb)


def test_products_side_by_side(gb):
    """Products of several widths on two streams at once, each with a status of its own: the same bits as one after the other."""
    data = [q8_data(n, K, N, n) for n, K, N in ((3000, 520, 64), (9000, 1040, 256), (700, 128, 1000), (20000, 260, 128))]
    want = []
    for a, sa, b, sb in data:
        want.append(torch.empty((a.shape[0], b.shape[0]), device="cuda"))
        gb.gear_q8_matmul(a, sa, b, sb, want[-1], status())
    torch.cuda.synchronize()
    streams, sts, outs = [torch.cuda.Stream() for _ in range(2)], [status(), status()], [[], []]
    torch.cuda.synchronize()
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            for r in range(5):
                for i, (a, sa, b, sb) in enumerate(data if k == 0 else data[::-1]):
                    o = torch.empty((a.shape[0], b.shape[0]), device="cuda")
                    gb.gear_q8_matmul(a, sa, b, sb, o, sts[k])
                    outs[k].append((i if k == 0 else len(data) - 1 - i, o))
    torch.cuda.synchronize()
    assert sts[0].tolist() == sts[1].tolist() == [0, 0]
    for i, o in outs[0] + outs[1]:
        assert torch.equal(o, want[i])


def test_product_says_that_a_wait_gave_up(gb):
    """A status whose second word is not zero marks results as void until it is cleared; the call ends, and the next one is whole again."""
    a, sa, b, sb = q8_data(5000, 520, 200, 5)
    st, out = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.empty((5000, 200), device="cuda")
    gb.gear_q8_matmul(a, sa, b, sb, out, st)
    torch.cuda.synchronize()
    assert st[0].item() & gb_timeout == gb_timeout and st[1].item() == 3
    st.zero_()
    gb.gear_q8_matmul(a, sa, b, sb, out, st)
    assert st.tolist() == [0, 0]
    check_product(out, a, sa, b, sb)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,N", [(40_000, 1040, 256), (20_000, 144, 520), (131_072, 64, 64), (50_000, 300, 100), (20_000, 2048, 1024), (200, 16, 300)])
def test_product_ends_whole_after_an_early_exit(gb, n, K, N, out_dtype):
    """The epilogue leaves at once, with the operands' copies and the first products under way; the waits of the others give up.  The call
    says so, writes nothing, and the calls behind it, with a clear status, are whole."""
    a, sa, b, sb = q8_data(n, K, N, n + K + N)
    want, out = torch.empty((n, N), dtype=out_dtype, device="cuda"), torch.full((n, N), 5.0, dtype=out_dtype, device="cuda")
    gb.gear_q8_matmul(a, sa, b, sb, want, status())
    check_product(want, a, sa, b, sb)
    for _ in range(3):
        st = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
        for _ in range(2):
            gb.gear_q8_matmul(a, sa, b, sb, out, st)
        assert st.tolist() == [gb_timeout, 3]
        assert (out == 5.0).all()
        st.zero_()
        got = torch.empty_like(out)
        gb.gear_q8_matmul(a, sa, b, sb, got, st)
        assert st.tolist() == [0, 0] and torch.equal(got, want)


def test_product_results_beyond_32_bits(gb):
    n, K, N = (1 << 31) // 1024 + 300, 48, 1024
    a, b = torch.zeros((n, K), dtype=torch.uint8, device="cuda").view(E4M3), e4m3_rows(N, K)
    small, sa_small, b2, sb = q8_data(300, K, N, 7)
    b.copy_(b2)
    a[-300:] = small
    sa = torch.ones((n, 1), device="cuda")
    sa[-300:] = sa_small
    st, out = status(), torch.full((n, N), 5.0, dtype=BF16, device="cuda")
    gb.gear_q8_matmul(a, sa, b, sb, out, st)
    assert st.tolist() == [0, 0]
    check_product(out[-300:], a[-300:], sa[-300:], b, sb)
    assert (out[:1000] == 0).all() and (out[n // 2:n // 2 + 1000] == 0).all()


# ------------------------------------------------------------------------------------------------ clipping
gb_timeout = 16                                     # GEAR_DEV_TIMEOUT


def workspace(gb):
    return torch.full((gb.GEAR_CLIP_WORKSPACE_BYTES // 8,), float("nan"), dtype=torch.float64, device="cuda")


def clip_check(grads, outs, norm, max_norm):
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads)) if grads else 0.0
    c = min(1.0, float(torch.tensor(max_norm, dtype=F32)) / (total + 1e-6))      # (max_norm is an fp32 argument)
    # 64-bit sums of exact squares; norm and c are rounded to fp32 once
    assert abs(float(norm[0]) - total) <= total * (U32 + 1e-12)
    assert abs(float(norm[1]) - c) <= c * (U32 + 1e-12)
    for g, o in zip(grads, outs):
        want = g.double() * c
        # c's rounding, the product's and (bf16) the output's; below the normal range half of the smallest number
        allowed = want.abs() * (2 * U32 + (u_of(BF16) if g.dtype == BF16 else 0)) * 1.01 + (2.0 ** -149 if g.dtype == F32 else 2.0 ** -133)
        assert ((o.double() - want).abs() <= allowed).all()


@pytest.mark.parametrize("sizes", [[], [0], [1], [3], [4], [5, 0, 1], [1023], [1 << 20], [17] * 33, [100_003, 1, 7, 2048, 30_000], [5] * 1024, [4099] * 1025, [64] * 2100,
                                   [3_000_001, 8191]])
@pytest.mark.parametrize("mixed", [False, True])
def test_clip(gb, sizes, mixed):
    dtypes = [BF16 if mixed and i % 2 else F32 for i in range(len(sizes))]
    grads = [randn((s,), i, d) for i, (s, d) in enumerate(zip(sizes, dtypes))]
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    norm, ws = torch.full((2,), 3.0, device="cuda"), workspace(gb)
    gb.gear_grad_norm(grads, norm, ws)
    assert abs(float(norm[0]) - total) <= total * (U32 + 1e-12) and float(norm[1]) == 3.0
    for ratio in (0.3, 3.0):
        outs = [torch.full_like(g, 9.0) for g in grads]
        gb.gear_clip_grads(grads, ratio * total, norm, ws, outs=outs)
        clip_check(grads, outs, norm, ratio * total)
        place = [g.clone() for g in grads]
        gb.gear_clip_grads(place, ratio * total, norm, ws)
        assert all(torch.equal(p, o) for p, o in zip(place, outs))


def test_clip_any_alignment(gb):
    """Slices of packed buffers, as a head's parameters are, and outputs aligned in another way than their gradients."""
    ws, norm = workspace(gb), torch.empty(2, device="cuda")
    for dtype in (F32, BF16):
        flat = randn((50_000,), 1, dtype)
        cuts = [1, 2, 3, 5, 4097, 12_345, 30_000]
        grads = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
        for shift in (0, 1, 3):
            back = torch.full((50_100,), 9.0, dtype=dtype, device="cuda")
            outs = [back[a + shift:b + shift] for a, b in zip(cuts, cuts[1:])]
            gb.gear_clip_grads(grads, 1.5, norm, ws, outs=outs)
            clip_check(grads, outs, norm, 1.5)
            assert (back[:1 + shift] == 9.0).all() and (back[30_000 + shift:] == 9.0).all()


def test_clip_extremes(gb):
    ws, norm = workspace(gb), torch.empty(2, device="cuda")
    for scale in (1e-38, 1e-25, 1e25, 1e34):
        g = [randn((5000,), 1) * scale, (randn((333,), 2) * scale).to(BF16)]
        outs = [torch.empty_like(t) for t in g]
        gb.gear_clip_grads(g, 0.5 * scale, norm, ws, outs=outs)
        clip_check(g, outs, norm, 0.5 * scale)
    zeros = [torch.zeros(100, device="cuda")]
    gb.gear_clip_grads(zeros, 1.0, norm, ws)
    assert norm.tolist() == [0.0, 1.0] and (zeros[0] == 0).all()
    gb.gear_clip_grads([torch.ones(4, device="cuda")], 0.0, norm, ws)
    assert norm.tolist() == [2.0, 0.0]
    g = torch.ones(1000, device="cuda")
    g[7] = float("inf")
    gb.gear_clip_grads([g], 1.0, norm, ws)
    assert float(norm[0]) == float("inf") and float(norm[1]) == 0.0 and g[7].isnan() and (g[8:] == 0).all()
    g = torch.ones(1000, device="cuda")
    g[7] = float("nan")
    gb.gear_clip_grads([g], 1.0, norm, ws)
    assert norm.isnan().all() and g.isnan().all()


def test_clip_to_an_infinite_norm(gb):
    ws, norm = workspace(gb), torch.empty(2, device="cuda")
    g = [randn((5000,), 1) * 1e30, randn((333,), 2).to(BF16)]
    outs = [torch.empty_like(t) for t in g]
    gb.gear_clip_grads(g, float("inf"), norm, ws, outs=outs)
    assert norm[0].isfinite() and float(norm[1]) == 1.0 and all(torch.equal(a, b) for a, b in zip(g, outs))
    g[0][7] = float("inf")
    gb.gear_clip_grads(g, float("inf"), norm, ws, outs=outs)
    assert float(norm[0]) == float("inf") and norm[1].isnan() and outs[0].isnan().all() and outs[1].isnan().all()


def test_clip_beyond_32_bits(gb):
    n = (1 << 31) + 77
    g = torch.full((n,), 0.5, dtype=BF16, device="cuda")
    g[-1] = 3.0
    norm, ws = torch.empty(2, device="cuda"), workspace(gb)
    total = math.sqrt((n - 1) * 0.25 + 9.0)
    gb.gear_clip_grads([g], total / 4, norm, ws)     # c = 1/4 but for roundings: 0.125 and 0.75 are bf16 values
    assert abs(float(norm[0]) - total) <= total * (U32 + 1e-12)
    assert (g[:1000] == 0.125).all() and (g[n // 2:n // 2 + 1000] == 0.125).all() and g[-1] == 0.75 and (g[-1000:-1] == 0.125).all()


def test_clip_repeats(gb):
    g = [randn((1_000_003,), 1), randn((77_777,), 2, BF16)]
    got = []
    for _ in range(3):
        norm, ws = torch.empty(2, device="cuda"), workspace(gb)
        gb.gear_grad_norm(g, norm, ws)
        got.append(float(norm[0]))
    assert got[0] == got[1] == got[2]


# ------------------------------------------------------------------------------------------------ how they are called
def test_python_refusals(gb):
    x, w = randn((4, 64), 1), randn((64,), 2)
    q, s = e4m3_rows(4, 64), torch.empty((4, 1), device="cuda")
    ws = torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, 64), device="cuda")
    st, norm, cws = status(), torch.empty(2, device="cuda"), workspace(gb)
    for call in (lambda: gb.gear_rms_norm(x.cpu(), w, q, s), lambda: gb.gear_rms_norm(x, w.cpu(), q, s), lambda: gb.gear_rms_norm(x, w[:32], q, s),
                 lambda: gb.gear_rms_norm(x, w, q[:, :32], s), lambda: gb.gear_rms_norm(x[:2], w, q, s), lambda: gb.gear_rms_norm(x, w, q, s[:2]),
                 lambda: gb.gear_rms_norm(x.half(), w, q, s), lambda: gb.gear_rms_norm(x.t(), w, q, s), lambda: gb.gear_rms_norm(x, w, q, s, res=x.to(BF16)),
                 lambda: gb.gear_rms_norm(x, w, q, s, ids=torch.zeros(4, dtype=torch.int64, device="cuda")),
                 lambda: gb.gear_rms_norm(x, w, q, s, d_n=torch.zeros(1, dtype=torch.int32, device="cuda")), lambda: gb.gear_rms_norm(x, w, q, s, n=5),
                 lambda: gb.gear_rms_norm_backward(x, w, x, x.clone(), w.clone(), None), lambda: gb.gear_rms_norm_backward(x, w, x, x.clone(), w.clone(), ws[:10]),
                 lambda: gb.gear_rms_norm_backward(x, w, x.to(BF16), x.clone(), None, None),
                 lambda: gb.gear_q8_rows(x, q, None), lambda: gb.gear_q8_rows(x, x.clone(), s), lambda: gb.gear_q8_weights(x.to(BF16), q, s),
                 lambda: gb.gear_q8_weights(x, e4m3_rows(64, 8), s), lambda: gb.gear_q8_matmul(q, s, e4m3_rows(8, 32), s, x, st),
                 lambda: gb.gear_q8_matmul(q, None, q, s, torch.empty((4, 4), device="cuda"), st),
                 lambda: gb.gear_q8_matmul(q, s, q, s, torch.empty((4, 5), device="cuda"), st),
                 lambda: gb.gear_clip_grads([x.double()], 1.0, norm, cws), lambda: gb.gear_clip_grads([x.t()], 1.0, norm, cws),
                 lambda: gb.gear_clip_grads([x], 1.0, norm[:1], cws), lambda: gb.gear_clip_grads([x], 1.0, norm, cws[:9]),
                 lambda: gb.gear_clip_grads([x, x], 1.0, norm, cws), lambda: gb.gear_clip_grads([x], 1.0, norm, cws, outs=[x[:2]]),
                 lambda: gb.gear_clip_grads([x], 1.0, norm, cws, outs=[]), lambda: gb.gear_clip_grads(gb.make_grads([x]), 1.0, norm, cws, outs=[x])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: gb.gear_q8_matmul(q, s, q, s, torch.empty((4, 4), device="cuda"), None), lambda: gb.gear_rms_norm(x, w, x.clone(), s),
                 lambda: gb.gear_rms_norm(x, w, q), lambda: gb.gear_rms_norm(x, w, q, s, eps=-1.0), lambda: gb.gear_q8_weights(x),
                 lambda: gb.gear_q8_matmul(q[:, :40], s, torch.empty((4, 40), dtype=torch.uint8, device="cuda"), s, torch.empty((4, 4), device="cuda"), st),
                 lambda: gb.gear_clip_grads([x], -1.0, norm, cws)):
        with pytest.raises(gb.GearError) as e:
            call()
        assert e.value.code == gb.GEAR_ERR_ARG


def layer(gb, x, w, W8, s8, bufs, stream=None):
    q, s, out, st = bufs
    gb.gear_rms_norm(x, w, q, s, stream=stream)
    gb.gear_q8_matmul(q, s, W8, s8, out, st, stream=stream)
    return out


def test_streams_and_capture(gb):
    """The calls on a stream of the caller's, and captured and replayed on new inputs; two captured programs side by side."""
    n, K, N = 700, 520, 200
    W8, s8 = e4m3_rows(N, K), torch.empty((blocks(N), blocks(K)), device="cuda")
    gb.gear_q8_weights(randn((K, N), 1), W8, s8)
    w = randn((K,), 2)
    bufs = lambda: (e4m3_rows(n, K), torch.empty((n, blocks(K)), device="cuda"), torch.empty((n, N), device="cuda"), status())
    xs = [randn((n, K), 10 + i) for i in range(4)]
    want = [layer(gb, x, w, W8, s8, bufs()).clone() for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = bufs()
    torch.cuda.synchronize()
    layer(gb, xs[0], w, W8, s8, b, stream=side)
    side.synchronize()
    assert torch.equal(b[2], want[0])
    graphs = []
    for _ in range(2):
        x, b = torch.empty((n, K), device="cuda"), bufs()
        grads = [torch.empty((n, K), device="cuda")]
        norm, cws = torch.empty(2, device="cuda"), workspace(gb)
        dw, ws = torch.empty(K, device="cuda"), torch.empty((gb.GEAR_NORM_WORKSPACE_ROWS, K), device="cuda")
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            layer(gb, x, w, W8, s8, b)
            gb.gear_rms_norm_backward(x, w, x, grads[0], dw, ws)
            gb.gear_clip_grads(grads, 1.0, norm, cws)
        graphs.append((g, x, b, grads, norm, dw))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for round_ in range(2):
        for k, (g, x, *_rest) in enumerate(graphs):
            with torch.cuda.stream(streams[k]):
                x.copy_(xs[2 * round_ + k])
                g.replay()
        torch.cuda.synchronize()
        for k, (g, x, b, grads, norm, dw) in enumerate(graphs):
            assert torch.equal(b[2], want[2 * round_ + k])
            dx, dw2 = back_exact(xs[2 * round_ + k], w, xs[2 * round_ + k], 1e-6, None)
            assert abs(float(norm[0]) / float(dx.norm()) - 1) < 1e-5 and abs(float(grads[0].norm()) - 1) < 1e-5
            assert torch.allclose(dw.double(), dw2, rtol=1e-4, atol=1e-3)


def test_offsets_beyond_32_bits(gb):
    """Rows behind the 2^31st value of a table, and results behind it."""
    cols = 4096
    rows = (1 << 31) // cols + 40
    table = torch.empty((rows, cols), dtype=BF16, device="cuda")
    table[-3:] = randn((3, cols), 1, BF16)
    ids = torch.tensor([rows - 1, rows - 2, rows - 3], dtype=torch.int32, device="cuda")
    out = torch.empty((3, cols), device="cuda")
    gb.gear_rms_norm(table, None, out, ids=ids)
    h = table[ids.long()].double()
    assert ((out.double() - h * rms(h, 1e-6)).abs() <= h.abs() * rms(h, 1e-6) * rms_rel(cols) * 1.01).all()
    q = torch.empty((rows, cols), dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.empty((rows, blocks(cols)), device="cuda")
    table[:-3] = 1.0
    gb.gear_q8_rows(table, q, s)
    check_q8(q[-3:], s[-3:], table[-3:].double(), 0.0)
    assert (q.view(torch.uint8)[1000:1003] == 0x7e).all()
