"""The calls of the 8-bit Dense Part together, as a training program uses them: images expire, are recomputed in 8 bits and
refreshed; a step hands averages over; they go back through the Dense Part; gradients are clipped, Adam takes a step."""
import numpy as np
import pytest
import torch

from operator_reference import U32, block_amax, blocks, check_q8, rms, rms_rel, spread

pytestmark = pytest.mark.gpu


def make(raw_dtype=torch.float32, raw_dim=200, seed=0, max_rows=None):
    from paper_1806_03925_b200 import binding as gb
    from paper_1806_03925_b200 import build, workloads
    from paper_1806_03925_b200.dense_part import NormedDensePart
    from paper_1806_03925_b200.session import DeviceBatch, GearSession
    build.build()
    p = workloads.PRESETS["tiny"].scaled(user_vocab=500, url_vocab=400, img_vocab=1200, M=2, expire=5)
    src = workloads.BatchSource(p, seed)
    s = GearSession(p, workloads.head_params(p, seed), max_batch=256, max_nnz=1024, seed=seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    raw = (torch.randn((p.img_vocab, raw_dim), generator=g, device="cuda") * 3).to(raw_dtype)
    Wd = torch.randn((raw_dim, p.dfv_dim), generator=g, device="cuda") / raw_dim ** 0.5
    part = NormedDensePart(s, raw, Wd, adam=gb.make_adam(lr=1e-2), max_norm=0.05, max_rows=max_rows)
    return gb, p, s, part, [DeviceBatch.from_host(src.batch(k)) for k in range(3)]


@pytest.mark.parametrize("raw_dtype,raw_dim", [(torch.float32, 200), (torch.bfloat16, 200), (torch.float32, 129)])
def test_the_whole_way(raw_dtype, raw_dim):
    gb, p, s, part, batches = make(raw_dtype, raw_dim)
    V, D, R = p.img_vocab, p.dfv_dim, raw_dim
    rows = torch.full((V, D), 7.0, device="cuda")
    try:
        for now, b in enumerate(batches, 1):
            # ---- events 2 and 3: what has expired is computed again, by a count the host does not know
            s.collect_expired(now, restamp=True, sync=False)
            part.forward(s.expired_ids, rows, n=V, d_n=s.d_counts[1:2])
            s.refresh_dfv(s.expired_ids, rows, now, n=V, d_n=s.d_counts[1:2])
            n = int(s.d_counts[1])
            assert 0 < n < V
            ids = s.expired_ids[:n].long()
            x = part.raw[ids].double()
            h = x * rms(x, part.eps) * part.weight.double()
            check_q8(part.q[:n], part.q_scale[:n], h, rms_rel(R))
            W8 = part.W8.double() * spread(part.W8_scale.double().repeat_interleave(128, 0)[:D], R)
            A = part.q[:n].double() * spread(part.q_scale[:n].double(), R)
            want, size = A @ W8.t(), A.abs() @ W8.abs().t()
            assert ((rows[:n].double() - want).abs() <= size * (128 + blocks(R) + 4) * 2.0 ** -23).all()
            # ... and what that is against the Dense Part without any rounding: each of the R products is off by two roundings to e4m3, 2^-4 of
            # the value, or 2^-10 of a scale (which is the block's largest / 448) below the normal range
            half = lambda v, largest: torch.maximum(v.abs() * 2.0 ** -4, largest * (2.0 ** -10 / 448)) * (1 + 2.0 ** -9)
            W = part.Wd.double()
            dh = half(h, spread(block_amax(h), R))
            dW = half(W, W.abs().amax())
            assert ((rows[:n].double() - h @ W).abs() <= dh @ W.abs() + h.abs() @ dW + dh @ dW + 1e-6).all()
            assert (rows[n:] == 7.0).all() or now > 1
            dfv = s.dfv[ids].float()
            assert torch.equal(dfv, rows[:n].to(s.dfv.dtype).float())
            # ---- events 1, 4, 5, 6
            s.forward_backward(b)
            s.accumulate_collect_from_step(b, sync=False)
            part.backward(b.nnz, d_n=s.d_counts[0:1])
            e = int(s.d_counts[0])
            assert e > 0
            ids, avg = s.ready_ids[:e].long(), s.ready_avg[:e].double()
            x = part.raw[ids].double()
            xr = x * rms(x, part.eps)
            h = xr * part.weight.double()
            size = h.abs().t() @ avg.abs()
            assert ((part.Wd_grad.double() - h.t() @ avg).abs() <= size * (rms_rel(R) + (e + 8) * U32) + 1e-30).all()
            check_q8(part.g[:e], part.g_scale[:e], avg, 0.0)
            G = part.g[:e].double() * spread(part.g_scale[:e].double(), D)
            dh, size = G @ W8, G.abs() @ W8.abs()
            assert ((part.dh[:e].double() - dh).abs() <= size * (128 + blocks(D) + 4) * 2.0 ** -23).all()
            used = part.dh[:e].to(raw_dtype).double()
            got, size = part.weight_grad.double(), (used * xr).abs().sum(0)
            assert ((got - (used * xr).sum(0)).abs() <= size * (rms_rel(R) + (e + 110) * U32) + 1e-30).all()
            # ---- clipping with the head's gradient beside, Adam, 8-bit copies
            before = [t.double().clone() for t in (part.Wd_grad, part.weight_grad, s.head_grad)]
            Wd0 = part.Wd.clone()
            part.step(more=[s.head_grad])
            total = float(torch.sqrt(sum((t * t).sum() for t in before)))
            c = min(1.0, float(np.float32(part.max_norm)) / (total + 1e-6))      # (an fp32 argument)
            assert abs(float(part.norm[0]) - total) <= total * (U32 + 1e-12) and abs(float(part.norm[1]) - c) <= c * (U32 + 1e-12)
            assert c < 1.0
            for t, o in zip(before, (part.Wd_grad, part.weight_grad, s.head_grad)):
                assert ((o.double() - c * t).abs() <= (c * t).abs() * 2.01 * U32 + 2.0 ** -149).all()
            assert not torch.equal(part.Wd, Wd0)
            scale = part.Wd.abs().double().amax() / 448
            back = part.W8.double() * spread(part.W8_scale.double().repeat_interleave(128, 0)[:D], R)
            assert ((back - part.Wd.t().double()).abs() <= torch.maximum(part.Wd.t().abs().double() * 2.0 ** -4, scale * 2.0 ** -10) * (1 + 2.0 ** -9)).all()
            part.check()
        assert s.status()[1] == 0
    finally:
        s.close()


def test_gradient_against_differences():
    """d loss / d Wd and d loss / d weight of loss = sum(avg . DFV), by differences of the 64-bit Dense Part without 8-bit rounding: exact
    for Wd (the loss is linear in it); for weight the gradient goes back through e4m3 weights and e4m3 averages, 2^-4 each."""
    gb, p, s, part, batches = make(raw_dim=64)
    try:
        s.forward_backward(batches[0])
        s.accumulate_collect_from_step(batches[0], sync=False)
        part.backward(batches[0].nnz, d_n=s.d_counts[0:1])
        e = int(s.d_counts[0])
        x, avg = part.raw[s.ready_ids[:e].long()].double(), s.ready_avg[:e].double()

        def loss(W, w):
            return float((((x * rms(x, part.eps) * w) @ W) * avg).sum())
        W, w = part.Wd.double(), part.weight.double()
        size = float(((x * rms(x, part.eps)).abs() @ W.abs() * avg.abs()).sum())
        for i, j in ((0, 0), (13, 40), (63, 63)):
            d = torch.zeros_like(W)
            d[i, j] = 1.0
            diff = (loss(W + d, w) - loss(W - d, w)) / 2
            assert abs(diff - float(part.Wd_grad[i, j])) <= 1e-5 * float((x * rms(x, part.eps))[:, i].abs() @ avg[:, j].abs()) + 1e-12 * size
            d = torch.zeros_like(w)
            d[i] = 1.0
            diff = (loss(W, w + d) - loss(W, w - d)) / 2
            terms = float(((x * rms(x, part.eps))[:, i:i + 1].abs() * avg.abs() * W[i].abs()).sum())
            # two roundings to e4m3 of 2^-4 each; below the normal range 2^-10 of the scale of a block of 64 values: a few percent more
            floor = float(((x * rms(x, part.eps))[:, i:i + 1].abs() * (avg.abs() * W.abs().amax() + avg.abs().amax(1, keepdim=True) * W[i].abs())).sum()) * 2.0 ** -10 / 448 * 1.1
            assert abs(diff - float(part.weight_grad[i])) <= terms * (2.0 ** -3 + 2.0 ** -8) + floor + 1e-9 * size
    finally:
        s.close()


def test_backward_of_few_averages_touches_few_rows():
    """bf16 raw rows: what backward takes from the allocator, and converts, goes by its n."""
    gb, p, s, part, batches = make(torch.bfloat16, 2000)
    try:
        s.forward_backward(batches[0])
        s.accumulate_collect_from_step(batches[0], sync=False)
        n = 16
        part.backward(n, d_n=s.d_counts[0:1])
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        held = torch.cuda.memory_allocated()
        part.backward(n, d_n=s.d_counts[0:1])
        torch.cuda.synchronize()
        assert torch.cuda.max_memory_allocated() - held <= n * 2000 * 2 + 512
        e = min(n, int(s.d_counts[0]))
        x = part.raw[s.ready_ids[:e].long()].double()
        xr, used = x * rms(x, part.eps), part.dh[:e].to(torch.bfloat16).double()
        assert e > 0 and ((part.weight_grad.double() - (used * xr).sum(0)).abs() <= (used * xr).abs().sum(0) * (rms_rel(2000) + (e + 110) * U32) + 1e-30).all()
        part.check()
    finally:
        s.close()


def test_a_wait_that_gave_up_on_one_way_leaves_the_other():
    """Serving and training may run beside each other: what voids forward's results does not void backward's, and check tells."""
    gb, p, s, part, batches = make(torch.float32, 2000)
    try:
        s.forward_backward(batches[0])
        s.accumulate_collect_from_step(batches[0], sync=False)
        part.backward(batches[0].nnz, d_n=s.d_counts[0:1])
        e, want = int(s.d_counts[0]), part.weight_grad.clone()
        part.check()
        part.status[1] = 3
        part.dh.fill_(7.0)
        part.backward(batches[0].nnz, d_n=s.d_counts[0:1])
        assert torch.equal(part.weight_grad, want) and not (part.dh[:e] == 7.0).all(1).any()
        rows = torch.full((p.img_vocab, p.dfv_dim), 7.0, device="cuda")
        part.forward(torch.arange(p.img_vocab, dtype=torch.int32, device="cuda"), rows)
        assert (rows == 7.0).all()
        with pytest.raises(gb.GearError) as err:
            part.check()
        assert err.value.code == gb.GEAR_ERR_CUDA
        part.check()
        part.forward(torch.arange(p.img_vocab, dtype=torch.int32, device="cuda"), rows)
        assert not (rows == 7.0).any()
        part.check()
    finally:
        s.close()


@pytest.mark.parametrize("raw_dtype", [torch.float32, torch.bfloat16])
def test_both_ways_beside_each_other(raw_dtype):
    """forward on one stream, backward on another, over and over: what either gives alone."""
    gb, p, s, part, batches = make(raw_dtype, 1000)
    try:
        s.forward_backward(batches[0])
        s.accumulate_collect_from_step(batches[0], sync=False)
        ids = torch.arange(p.img_vocab, dtype=torch.int32, device="cuda")
        want, rows = torch.empty((p.img_vocab, p.dfv_dim), device="cuda"), [torch.full((p.img_vocab, p.dfv_dim), 7.0, device="cuda") for _ in range(20)]
        part.forward(ids, want)
        part.backward(batches[0].nnz, d_n=s.d_counts[0:1])
        e, grad = int(s.d_counts[0]), part.weight_grad.clone()
        dh, Wd_grad = part.dh[:e].clone(), part.Wd_grad.clone()
        one, two = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        grads = []
        for r in rows:
            with torch.cuda.stream(one):
                part.forward(ids, r)
            with torch.cuda.stream(two):
                part.backward(batches[0].nnz, d_n=s.d_counts[0:1])
                grads.append((part.weight_grad.clone(), part.dh[:e].clone()))
        torch.cuda.synchronize()
        part.check()
        assert all(torch.equal(r, want) for r in rows)
        assert all(torch.equal(a, grad) and torch.equal(b, dh) for a, b in grads)
        # (its sums are in an order the hardware picks)
        assert ((part.Wd_grad - Wd_grad).abs() <= part.h[:e].abs().t() @ s.ready_avg[:e].abs() * (2 * (e + 8) * U32) + 1e-30).all()
    finally:
        s.close()


def test_more_averages_than_images():
    """A step may complete several groups of one image: its averages are bounded by its occurrences, not by the table."""
    from paper_1806_03925_b200 import binding as gb
    from paper_1806_03925_b200 import build, workloads
    from paper_1806_03925_b200.dense_part import NormedDensePart
    from paper_1806_03925_b200.session import DeviceBatch, GearSession
    build.build()
    p = workloads.PRESETS["tiny"].scaled(user_vocab=500, url_vocab=400, img_vocab=30, M=1, expire=5)
    s = GearSession(p, workloads.head_params(p, 0), max_batch=256, max_nnz=1024, seed=0)
    raw, R, D = torch.randn((p.img_vocab, 200), device="cuda"), 200, p.dfv_dim
    part = NormedDensePart(s, raw, torch.randn((R, D), device="cuda") / 14)
    b = DeviceBatch.from_host(workloads.BatchSource(p, 0).batch(0))
    try:
        s.forward_backward(b)
        s.accumulate_collect_from_step(b, sync=False)
        e = int(s.d_counts[0])
        assert p.img_vocab < e <= b.nnz
        part.backward(b.nnz, d_n=s.d_counts[0:1])
        x, avg = raw[s.ready_ids[:e].long()].double(), s.ready_avg[:e].double()
        xr = x * rms(x, part.eps)
        h = xr * part.weight.double()
        assert ((part.Wd_grad.double() - h.t() @ avg).abs() <= h.abs().t() @ avg.abs() * (rms_rel(R) + (e + 8) * U32) + 1e-30).all()
        used = part.dh[:e].double()
        assert ((part.weight_grad.double() - (used * xr).sum(0)).abs() <= (used * xr).abs().sum(0) * (rms_rel(R) + (e + 110) * U32) + 1e-30).all()
        part.check()
        with pytest.raises(ValueError):
            part.backward(s.ready_cap + 1)
        with pytest.raises(ValueError):
            NormedDensePart(s, raw, part.Wd, max_rows=max(s.ready_cap, p.img_vocab) + 1)
        assert NormedDensePart(s, raw, part.Wd, max_rows=s.ready_cap).max_rows == s.ready_cap
    finally:
        s.close()


def test_bad_ids_and_refusals():
    gb, p, s, part, batches = make(max_rows=50)
    from paper_1806_03925_b200.dense_part import NormedDensePart
    try:
        rows = torch.zeros((60, p.dfv_dim), device="cuda")
        ids = torch.tensor([3, p.img_vocab, -1, 7], dtype=torch.int32, device="cuda")
        part.forward(ids, rows)
        assert (rows[1:3] == 0).all() and (rows[0] != 0).any()
        with pytest.raises(gb.GearError):
            part.check()
        part.check()
        with pytest.raises(ValueError):
            part.forward(torch.zeros(60, dtype=torch.int32, device="cuda"), rows)
        with pytest.raises(ValueError):
            part.backward(51)
        with pytest.raises(ValueError):
            NormedDensePart(s, part.raw[:10], part.Wd)
        with pytest.raises(ValueError):
            NormedDensePart(s, part.raw, part.Wd[:, :8])
        with pytest.raises(ValueError):
            NormedDensePart(s, part.raw, part.Wd, max_rows=0)
    finally:
        s.close()
