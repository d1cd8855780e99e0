"""A linear Dense Part behind a root-mean-square norm, served in 8 bits and trained in fp32:

    DFV[id] = (raw[id] / rms(raw[id]) * weight) . Wd

The way of a training program around GearSession: the images an expiry scan lists go through forward (events 2 and 3: their rows are
normed, put into e4m3 and multiplied with the weights' 8-bit copy) to refresh_dfv; the averages a step hands over go through
backward (event 6); step clips the gradients by their global norm, takes an Adam step and makes the 8-bit copies anew.
No arithmetic happens here: every step is a call of the binding, but for one conversion: the norm's gradients take x and dout of one type, so
where raw is bf16 the gradient of the normed rows is rounded to bf16 (2^-8 of each value at most) on its way to weight's.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as gb
from .session import GearSession


def e4m3_rows(n: int, cols: int, device="cuda") -> torch.Tensor:
    """n rows of e4m3 values as gear_q8_matmul takes them: rows start at multiples of 16 bytes."""
    return torch.empty((n, (cols + 15) // 16 * 16), dtype=torch.float8_e4m3fn, device=device)[:, :cols]


class NormedDensePart:
    """raw: [img_vocab][raw_dim] fp32 or bf16; Wd: [raw_dim][dfv_dim] fp32 and weight: [raw_dim] fp32, both updated in place by step.
    forward and backward share no buffer that either writes and have a status each, so they may run on two streams; step (and requantise) writes what
    both read, and belongs behind them and ahead of the next ones.  Calls of one way belong to one stream, or are ordered by the caller.
    max_rows: most rows of one forward or backward call (default: all images; all averages the session can hand over, ready_cap)."""

    def __init__(self, session: GearSession, raw: torch.Tensor, Wd: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 adam: Optional["gb.gear_adam"] = None, max_norm: float = 1.0, max_rows: Optional[int] = None):
        V, R = raw.shape
        D = session.p.dfv_dim
        if V != session.p.img_vocab or Wd.shape != (R, D) or (weight is not None and weight.shape != (R,)):
            raise ValueError("raw: [img_vocab][raw_dim], Wd: [raw_dim][dfv_dim], weight: [raw_dim]")
        n, back = (V, session.ready_cap) if max_rows is None else (int(max_rows), int(max_rows))
        if not 1 <= n <= max(V, session.ready_cap):
            raise ValueError("max_rows in [1, the larger of img_vocab and ready_cap]")
        dev = raw.device
        f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)
        self.session, self.raw, self.Wd, self.eps, self.max_rows, self.max_norm = session, raw, Wd, eps, n, max_norm
        self.max_averages = back
        self.weight = torch.ones(R, dtype=torch.float32, device=dev) if weight is None else weight
        self.adam, self.t = adam or gb.make_adam(), 0
        blocks = lambda k: (k + gb.GEAR_Q8_BLOCK - 1) // gb.GEAR_Q8_BLOCK
        self.W8, self.W8_scale = e4m3_rows(D, R, dev), f(blocks(D), blocks(R))
        self.W8_t, self.W8_t_scale = e4m3_rows(R, D, dev), f(blocks(R), blocks(D))
        self.q, self.q_scale = e4m3_rows(n, R, dev), f(n, blocks(R))
        # a status for each way, in one place
        self._statuses = torch.zeros((2, 2), dtype=torch.int32, device=dev)
        self.status, self.status_back = self._statuses[0], self._statuses[1]
        # the way back
        self.h, self.dh = f(min(back, V), R), f(back, R)         # normed rows; their gradient
        self.g, self.g_scale = e4m3_rows(back, D, dev), f(back, blocks(D))
        self.iota = torch.arange(min(back, V), dtype=torch.int32, device=dev)
        self.Wd_grad, self.weight_grad = torch.zeros_like(Wd), torch.zeros_like(self.weight)
        self.norm_workspace = f(gb.GEAR_NORM_WORKSPACE_ROWS, R)
        self.clip_workspace = torch.empty(gb.GEAR_CLIP_WORKSPACE_BYTES, dtype=torch.uint8, device=dev)
        self.norm = torch.zeros(2, dtype=torch.float32, device=dev)
        self.moments = [(torch.zeros_like(p), torch.zeros_like(p)) for p in (self.Wd, self.weight)]
        self.grads = gb.make_grads([self.Wd_grad, self.weight_grad])
        self.requantise()

    def requantise(self):
        """The weights' 8-bit copies (after any change of Wd)."""
        gb.gear_q8_weights(self.Wd, self.W8, self.W8_scale, self.W8_t, self.W8_t_scale)

    def forward(self, ids: torch.Tensor, rows: torch.Tensor, n: Optional[int] = None, d_n=None):
        """rows[k] (fp32) = the Dense Feature Vector of ids[k], k < n and k < *d_n: what GearSession.refresh_dfv takes."""
        n = int(ids.shape[0]) if n is None else n
        if n > self.max_rows:
            raise ValueError("more rows than max_rows")
        gb.gear_rms_norm(self.raw, self.weight, self.q, self.q_scale, self.eps, ids=ids, n=n, d_n=d_n, status=self.status)
        gb.gear_q8_matmul(self.q, self.q_scale, self.W8, self.W8_scale, rows, self.status, n=n, d_n=d_n)

    def backward(self, n: int, d_n=None):
        """Wd_grad and weight_grad from the averages the session handed over last (ready_ids, ready_avg).  The 8-bit rounding counts as
        none, except that the gradient goes back through the weights as they were used; with bf16 raw rows it is rounded to bf16 behind them."""
        if n > self.max_averages:
            raise ValueError("more averages than max_rows, or than the session hands over")
        s = self.session
        ids = s.ready_ids
        self.Wd_grad.zero_()
        if n <= self.raw.shape[0]:                   # the images' normed rows, one for each average
            gb.gear_rms_norm(self.raw, self.weight, self.h, None, self.eps, ids=ids, n=n, d_n=d_n, status=self.status_back)
            gb.gear_dense_backward(s.ctx, self.h, self.iota, s.ready_avg, n, self.Wd_grad, d_n=d_n)
        else:                                        # more averages than images (M completed groups are an average each): every image's once
            gb.gear_rms_norm(self.raw, self.weight, self.h, None, self.eps, status=self.status_back)
            gb.gear_dense_backward(s.ctx, self.h, ids, s.ready_avg, n, self.Wd_grad, d_n=d_n)
        gb.gear_q8_rows(s.ready_avg, self.g, self.g_scale, n=n, d_n=d_n)
        gb.gear_q8_matmul(self.g, self.g_scale, self.W8_t, self.W8_t_scale, self.dh, self.status_back, n=n, d_n=d_n)
        raw_grad = self.dh if self.raw.dtype == torch.float32 else self.dh[:n].to(self.raw.dtype)
        gb.gear_rms_norm_backward(self.raw, self.weight, raw_grad, None, self.weight_grad, self.norm_workspace, self.eps, ids=ids, n=n, d_n=d_n,
                                  status=self.status_back)

    def step(self, more: Sequence[torch.Tensor] = ()):
        """Clips the gradients of Wd and weight, and those in `more` (the head's), by their norm together; an Adam step on Wd and weight;
        their 8-bit copies.  norm holds the norm and the factor.  (t counts on the host: a step that is captured and replayed repeats one t.  With `more`
        the list of gradients is made anew each time.)"""
        grads = self.grads if not more else [self.Wd_grad, self.weight_grad, *more]
        gb.gear_clip_grads(grads, self.max_norm, self.norm, self.clip_workspace)
        self.t += 1
        for p, g, (m, v) in zip((self.Wd, self.weight), (self.Wd_grad, self.weight_grad), self.moments):
            gb.gear_adam_dense(p, g, m, v, self.t, self.adam)
        self.requantise()

    def check(self):
        """Raises if an ID was outside the table or a wait gave up since the last check; synchronises the current stream."""
        (bits, code), (back_bits, back_code) = self._statuses.tolist()
        if bits or code or back_bits or back_code:
            self._statuses.zero_()
            raise gb.GearError(gb.GEAR_ERR_CUDA if (bits | back_bits) & gb.GEAR_DEV_TIMEOUT else gb.GEAR_ERR_BAD_ID, "NormedDensePart",
                               "forward: status bits %d, code %d; backward: %d, %d" % (bits, code, back_bits, back_code))
