"""Performance cases of the operators around an 8-bit Dense Part and its training: what a user of the package calls, over the
range of sizes.

Kinds of case (the "kind" key):

  clip     the global norm of a list of gradients and their clipping to a largest norm, into a second list: the head's
           parameters, the Dense Part's weights and gradient tables of the embeddings, fp32 and bf16 side by side.
  norm     rows of the Dense Part's input (optionally picked by Image ID, optionally with a residual added): root-mean-square
           norm, then e4m3 with one scale for every 128 columns, or fp32 / bf16.  "normed" false: the 8-bit form alone.
  back     the norm's gradients: of its input (with the residual path's gradient added) and of its weights.
  product  rows in e4m3 times weights in e4m3, a scale for every 128 columns of a row and for every 128 x 128 weights;
           fp32 or bf16 results.  "grad": the direction back through the layer: rows are put into 8 bits first, the weights are
           the transposed copy.
  weights  fp32 weights into both 8-bit copies (after every optimiser step of a training program).

own = False: elementary torch operations in 32 bits (sums of squares over all gradients in 64); own = True: the package's calls.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

BLOCK = 128                    # columns (and rows of a weight matrix) that share a scale
E4M3_MAX = 448.0
TINY = 2.0 ** -100             # a block's largest magnitude counts as at least this
EPS = 1e-6
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


# ------------------------------------------------------------------------------------------------ the cases
def _clip(name, tensors, f32, bf16, clips):
    return dict(name=name, kind="clip", tensors=tensors, f32=f32, bf16=bf16, clips=clips)


def _norm(name, n, cols, dtype, out, res=False, vocab=0, normed=True):
    return dict(name=name, kind="norm", n=n, cols=cols, dtype=dtype, out=out, res=res, vocab=vocab, normed=normed)


def _back(name, n, cols, dtype, res):
    return dict(name=name, kind="back", n=n, cols=cols, dtype=dtype, res=res)


def _product(name, n, K, N, out, grad=False):
    return dict(name=name, kind="product", n=n, K=K, N=N, out=out, grad=grad)


def _weights(name, K, N):
    return dict(name=name, kind="weights", K=K, N=N)


def listed():
    return [
        # a training step's dense gradients on preset "medium" with a linear Dense Part of 1536 raw values: a few small tensors
        _clip("clip_dense_f32", 7, 180_737, 0, True),
        # the same job with gradient tables of two embedding tables of a million rows, and a deep Dense Part in bf16
        _clip("clip_tables_mixed", 150, 64_082_433, 30_000_019, True),
        # one image's features on their way through the Dense Part while it is being served
        _norm("norm_one_row_bf16", 1, 1536, "bf16", "e4m3", res=True),
        # the refresh of expired images on preset "split_image": their raw rows, picked by ID
        _norm("norm_by_id_f32", 2500, 1536, "f32", "e4m3", vocab=50_000),
        # a layer inside the Dense Part over a whole refresh of a large table, residual stream in bf16
        _norm("norm_large_bf16", 262_144, 1536, "bf16", "e4m3", res=True),
        # gradients of the norm for the emissions of one step, odd width
        _back("back_ragged_f32", 3001, 1001, "f32", False),
        # ... and for a large batch of averages, residual stream in bf16
        _back("back_large_bf16", 131_072, 1536, "bf16", True),
        # one image through the output layer of preset "split_image"
        _product("product_one_row_f32", 1, 1536, 64, "f32"),
        # the gradient of a batch's averages back through a layer whose widths fit no tile
        _product("product_grad_ragged", 3001, 1000, 200, "bf16", grad=True),
        # an inner layer of the Dense Part over the refresh of a large table
        _product("product_large_bf16", 131_072, 2048, 1024, "bf16"),
        # the linear Dense Part's weights on preset "split_image", after every optimiser step
        _weights("weights_small", 1536, 64),
        # an inner layer's
        _weights("weights_large", 2048, 1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["clip", "norm", "norm", "norm", "back", "back", "product", "product", "product", "weights"])
    if kind == "clip":
        f32 = _log_int(rng, 1000, 64_000_000)
        c = _clip("", _log_int(rng, 1, 200), f32, rng.choice([0, _log_int(rng, 1000, 30_000_000)]), rng.random() < 0.8)
    elif kind == "norm":
        cols = rng.choice([_log_int(rng, 64, 2048), 8 * _log_int(rng, 8, 256), 128 * rng.randint(1, 16)])
        n = _log_int(rng, 1, 262_144 * 1536 // max(cols, 1536))
        vocab = rng.choice([0, 0, n + _log_int(rng, 1, 50_000)])
        dtype = rng.choice(["bf16", "f32"])
        if dtype == "f32":
            n = max(1, n // 2)
        c = _norm("", n, cols, dtype, rng.choice(["e4m3", "e4m3", "bf16", "f32"]), rng.random() < 0.5, vocab, True)
        if rng.random() < 0.2:
            c.update(normed=False, res=False, vocab=0, out="e4m3")
    elif kind == "back":
        cols = rng.choice([_log_int(rng, 64, 2048), 8 * _log_int(rng, 8, 256)])
        c = _back("", _log_int(rng, 1, 131_072 * 1536 // max(cols, 1536) // 2), cols, rng.choice(["bf16", "f32"]), rng.random() < 0.5)
    elif kind == "product":
        c = _product("", _log_int(rng, 1, 131_072), rng.choice([_log_int(rng, 16, 2048), 16 * _log_int(rng, 4, 128)]),
                     rng.choice([_log_int(rng, 8, 1024), 8 * _log_int(rng, 4, 128)]), rng.choice(["bf16", "f32"]), rng.random() < 0.3)
    else:
        c = _weights("", _log_int(rng, 16, 2048), _log_int(rng, 8, 1024))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
@functools.lru_cache(maxsize=1)
def _package():
    from paper_1806_03925_b200 import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed & (2**63 - 1))
    return g


def _split(total, parts):
    """Sizes of `parts` tensors (one at least) of `total` values in all: their logarithms spread, odd ones among them."""
    if total == 0:
        return []
    r = random.Random(total * 1009 + parts)
    w = [math.exp(r.uniform(0.0, 7.0)) for _ in range(min(parts, total))]
    scale, sizes = (total - len(w)) / sum(w), []
    for x in w[:-1]:
        sizes.append(1 + int(x * scale))
    return sizes + [total - sum(sizes)]


def _rows(gen, n, cols, dtype, per_column=True):
    """Features: normal, columns of different spread."""
    x = torch.randn((n, cols), generator=gen, device="cuda", dtype=dtype)
    if per_column:
        x *= torch.exp(torch.randn(cols, generator=gen, device="cuda")).to(dtype)
    return x


def _ld(K):
    return -(-K // 16) * 16                   # rows of 8-bit values start at multiples of 16 bytes


def _e4m3(n, K):
    return torch.empty((n, _ld(K)), dtype=torch.float8_e4m3fn, device="cuda")[:, :K]


def _blocks(K):
    return -(-K // BLOCK)


def _padded(x, rows=1):
    """x with zeros up to whole blocks."""
    n, K = x.shape
    return torch.nn.functional.pad(x, (0, _blocks(K) * BLOCK - K, 0, -(-n // rows) * rows - n))


def _q8_rows(x):
    """fp32 rows in e4m3: (values, scales [n][blocks])."""
    n, K = x.shape
    b = _padded(x).view(n, -1, BLOCK)
    scale = b.abs().amax(2).clamp_min(TINY) / E4M3_MAX
    return (b / scale[:, :, None]).view(n, -1)[:, :K].to(torch.float8_e4m3fn), scale


def _q8_weights(W):
    """W [K][N] fp32 as the product reads it: (values [N][K], scales [blocks of N][blocks of K])."""
    K, N = W.shape
    b = _padded(W.t(), BLOCK).view(_blocks(N), BLOCK, _blocks(K), BLOCK)
    scale = b.abs().amax((1, 3)).clamp_min(TINY) / E4M3_MAX
    return (b / scale[:, None, :, None]).view(_blocks(N) * BLOCK, -1)[:N, :K].to(torch.float8_e4m3fn), scale


def _spread(scale, rows, K, per_row):
    """Scales, one for every value."""
    s = scale.repeat_interleave(BLOCK, 1)[:, :K]
    return s if per_row else s.repeat_interleave(BLOCK, 0)[:rows]


def _kept(q):
    """8-bit values in rows whose starts are multiples of 16 bytes."""
    out = _e4m3(*q.shape)
    out.copy_(q)
    return out


def prepare(case, seed):
    c, gen, dev = case, _gen(seed), "cuda"
    s = {"case": c}
    if c["kind"] == "clip":
        sigma = 1e-3
        for name, dtype in (("f32", torch.float32), ("bf16", torch.bfloat16)):
            sizes = _split(c[name], max(1, c["tensors"] if c["bf16"] == 0 else c["tensors"] // 2))
            flat = torch.randn(c[name], generator=gen, device=dev, dtype=dtype) * sigma
            s[name], s[name + "_out"] = flat, torch.empty_like(flat)
            s[name + "_list"], s[name + "_outs"] = list(flat.split(sizes)), list(s[name + "_out"].split(sizes))
        s["max_norm"] = sigma * math.sqrt(c["f32"] + c["bf16"]) * (0.5 if c["clips"] else 2.0)
        s["norm"] = torch.zeros(2, device=dev)
        s["workspace"] = torch.zeros(4096, dtype=torch.float64, device=dev)
        if own:                                   # the list as the call takes it: a training program's buffers stay where they are
            s["grads"] = _package().make_grads(s["f32_list"] + s["bf16_list"], s["f32_outs"] + s["bf16_outs"])
        return s
    if c["kind"] in ("norm", "back"):
        n, cols, dtype = c["n"], c["cols"], _DTYPES[c["dtype"]]
        s["weight"] = 1.0 + 0.1 * torch.randn(cols, generator=gen, device=dev)
        s["x"] = _rows(gen, c.get("vocab") or n, cols, dtype)
        s["res"] = _rows(gen, n, cols, dtype) if c["res"] else None
        if c["kind"] == "back":
            s["dout"] = _rows(gen, n, cols, dtype, False) * 1e-3
            s["dx"], s["dweight"] = torch.empty_like(s["x"]), torch.empty(cols, device=dev)
            s["workspace"] = torch.empty((592, cols), device=dev)
            return s
        s["ids"] = None
        if c["vocab"]:
            s["ids"] = torch.randperm(c["vocab"], generator=gen, device=dev)[:n].sort().values.to(torch.int32)
        s["sum"] = torch.empty((n, cols), dtype=dtype, device=dev) if c["res"] else None
        s["out"] = _e4m3(n, cols) if c["out"] == "e4m3" else torch.empty((n, cols), dtype=_DTYPES[c["out"]], device=dev)
        s["scale"] = torch.empty((n, _blocks(cols)), device=dev) if c["out"] == "e4m3" else None
        return s
    K, N = c["K"], c["N"]
    W = torch.randn((K, N), generator=gen, device=dev) * (1.0 / math.sqrt(K))
    if c["kind"] == "weights":
        s["W"] = W
        s["q"], s["scale"] = _e4m3(N, K), torch.empty((_blocks(N), _blocks(K)), device=dev)
        s["q_t"], s["scale_t"] = _e4m3(K, N), torch.empty((_blocks(K), _blocks(N)), device=dev)
        return s
    b, s["b_scale"] = _q8_weights(W.t() if c["grad"] else W)
    s["b"] = _kept(b)
    inner, width = (N, K) if c["grad"] else (K, N)
    if c["grad"]:
        s["rows"] = _rows(gen, c["n"], inner, torch.float32, False) * 1e-3
        s["a"], s["a_scale"] = _e4m3(c["n"], inner), torch.empty((c["n"], _blocks(inner)), device=dev)
    else:
        a, s["a_scale"] = _q8_rows(_rows(gen, c["n"], inner, torch.float32))
        s["a"] = _kept(a)
    s["out"] = torch.empty((c["n"], width), dtype=_DTYPES[c["out"]], device=dev)
    s["status"] = torch.zeros(2, dtype=torch.int32, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    _gb, c, kind = _package(), s["case"], s["case"]["kind"]
    if kind == "clip":
        _gb.gear_clip_grads(s["grads"], s["max_norm"], s["norm"], s["workspace"])
        return {"norm": s["norm"], "f32": s["f32_out"], "bf16": s["bf16_out"]}
    if kind == "norm":
        if c["normed"]:
            _gb.gear_rms_norm(s["x"], s["weight"], s["out"], s["scale"], EPS, res=s["res"], res_out=s["sum"], ids=s["ids"])
        else:
            _gb.gear_q8_rows(s["x"], s["out"], s["scale"])
        return {"out": s["out"], "scale": s["scale"], "sum": s["sum"]}
    if kind == "back":
        _gb.gear_rms_norm_backward(s["x"], s["weight"], s["dout"], s["dx"], s["dweight"], s["workspace"], EPS, dres=s["res"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if kind == "weights":
        _gb.gear_q8_weights(s["W"], s["q"], s["scale"], s["q_t"], s["scale_t"])
        return {"q": s["q"], "scale": s["scale"], "q_t": s["q_t"], "scale_t": s["scale_t"]}
    if c["grad"]:
        _gb.gear_q8_rows(s["rows"], s["a"], s["a_scale"])
    _gb.gear_q8_matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], s["out"], s["status"])
    return s["out"]


def _run_plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "clip":
        norm = (s["f32"].double().square().sum() + s["bf16"].double().square().sum()).sqrt()
        coef = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
        return {"norm": torch.stack([norm.float(), coef]), "f32": s["f32"] * coef, "bf16": (s["bf16"].float() * coef).bfloat16()}
    if kind == "norm":
        x = s["x"] if s["ids"] is None else s["x"][s["ids"].long()]
        total = None
        if s["res"] is not None:
            total = (x.float() + s["res"].float()).to(x.dtype)
            x = total
        h = x.float()
        if c["normed"]:
            h = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["weight"]
        q, scale = _q8_rows(h) if c["out"] == "e4m3" else (h.to(_DTYPES[c["out"]]), None)
        return {"out": q, "scale": scale, "sum": total}
    if kind == "back":
        x, g = s["x"].float(), s["dout"].float()
        r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
        xn, wg = x * r, g * s["weight"]
        dx = r * (wg - xn * (wg * xn).mean(1, keepdim=True))
        if s["res"] is not None:
            dx = dx + s["res"].float()
        return {"dx": dx.to(s["x"].dtype), "dweight": (g * xn).sum(0)}
    if kind == "weights":
        q, scale = _q8_weights(s["W"])
        return {"q": q, "scale": scale, "q_t": q.float().t().to(torch.float8_e4m3fn), "scale_t": scale.t()}
    a, a_scale = _q8_rows(s["rows"]) if c["grad"] else (s["a"], s["a_scale"])
    K, N = a.shape[1], s["b"].shape[0]
    A = a.float() * _spread(a_scale, c["n"], K, True)
    B = s["b"].float() * _spread(s["b_scale"], N, K, False)
    return (A @ B.t()).to(s["out"].dtype)


# ------------------------------------------------------------------------------------------------ work, values in 64 bits
def work(case):
    """Each input once and each output once; two operations for every multiply-add of a product, a few for every value elsewhere."""
    c = case
    if c["kind"] == "clip":
        return {"bytes": 2.0 * (4 * c["f32"] + 2 * c["bf16"]), "flops": 3.0 * (c["f32"] + c["bf16"])}
    if c["kind"] in ("norm", "back"):
        size = {"f32": 4, "bf16": 2, "e4m3": 1 + 4 / BLOCK}
        n, cols, b = c["n"], c["cols"], size[c["dtype"]]
        if c["kind"] == "back":
            return {"bytes": n * cols * b * (4 if c["res"] else 3) + 8.0 * cols, "flops": 12.0 * n * cols}
        return {"bytes": n * cols * (b * (3 if c["res"] else 1) + size[c["out"]]) + (4.0 * n if c["vocab"] else 0.0) + 4.0 * cols,
                "flops": 8.0 * n * cols}
    K, N = c["K"], c["N"]
    if c["kind"] == "weights":
        return {"bytes": 6.0 * K * N, "flops": 4.0 * K * N}
    n, inner, width = c["n"], N if c["grad"] else K, K if c["grad"] else N
    rows = n * inner * (4 if c["grad"] else 1 + 4 / BLOCK)
    return {"bytes": rows + K * N + n * width * (2.0 if c["out"] == "bf16" else 4.0), "flops": 2.0 * n * K * N}


def _round_e4m3(v):
    """The e4m3 value nearest to v (64 bits; ties to even), for |v| up to the largest: three bits behind the leading one, steps of
    2^-9 below 2^-6."""
    mantissa, exponent = torch.frexp(v)
    step = torch.exp2((exponent.double() - 4).clamp_min(-9.0))
    del mantissa
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_rows(h):
    n, K = h.shape
    pad = torch.zeros((n, _blocks(K) * BLOCK), dtype=torch.float64, device=h.device)
    pad[:, :K] = h
    pad = pad.view(n, _blocks(K), BLOCK)
    largest = torch.maximum(pad.max(2).values, -pad.min(2).values)
    scale = torch.maximum(largest, torch.full_like(largest, TINY)) / E4M3_MAX
    return _round_e4m3(pad / scale.unsqueeze(2)).reshape(n, -1)[:, :K], scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "clip":
        a, b = s["f32"].double(), s["bf16"].double()
        norm = math.sqrt(float(torch.dot(a, a)) + (float(torch.dot(b, b)) if c["bf16"] else 0.0))
        coef = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor([norm, coef], dtype=torch.float64), "f32": a * coef, "bf16": b * coef}
    if c["kind"] == "norm":
        x = s["x"].double()
        if s["ids"] is not None:
            x = x.index_select(0, s["ids"].long())
        total = None
        if c["res"]:
            total = x + s["res"].double()
            x = total.to(s["x"].dtype).double()             # the sum is kept, and normed, in the stream's type
        if c["normed"]:
            x = x / torch.sqrt((x * x).sum(1, keepdim=True) / c["cols"] + EPS) * s["weight"].double()
        if c["out"] != "e4m3":
            return {"out": x, "scale": None, "sum": total}
        q, scale = _exact_rows(x)
        return {"out": q, "scale": scale, "sum": total}
    if c["kind"] == "back":
        x, g, w = s["x"].double(), s["dout"].double(), s["weight"].double()
        inv = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) / c["cols"] + EPS)
        dot = (g * w * x).sum(1, keepdim=True)
        dx = inv * w * g - x * (inv ** 3 * dot / c["cols"])
        if c["res"]:
            dx = dx + s["res"].double()
        return {"dx": dx, "dweight": (g * x * inv).sum(0)}
    if c["kind"] == "weights":
        K, N = c["K"], c["N"]
        W, q = s["W"].double(), torch.empty((N, K), dtype=torch.float64, device="cuda")
        scale = torch.empty((_blocks(N), _blocks(K)), dtype=torch.float64, device="cuda")
        for i in range(_blocks(N)):
            for j in range(_blocks(K)):
                part = W[j * BLOCK:(j + 1) * BLOCK, i * BLOCK:(i + 1) * BLOCK]
                scale[i, j] = part.abs().max().clamp_min(TINY) / E4M3_MAX
                q[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK] = _round_e4m3(part / scale[i, j]).t()
        return {"q": q, "scale": scale, "q_t": q.t().contiguous(), "scale_t": scale.t().contiguous()}
    a, a_scale = _exact_rows(s["rows"].double()) if c["grad"] else (s["a"].double(), s["a_scale"].double())
    b, out = s["b"].double(), torch.zeros((c["n"], s["b"].shape[0]), dtype=torch.float64, device="cuda")
    for k in range(a_scale.shape[1]):
        part = slice(k * BLOCK, (k + 1) * BLOCK)
        wide = s["b_scale"].double()[:, k].repeat_interleave(BLOCK)[:out.shape[1]]
        out += (a[:, part] @ b[:, part].t()) * a_scale[:, k:k + 1] * wide
    return out
