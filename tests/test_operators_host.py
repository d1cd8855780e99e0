"""What the calls of the 8-bit Dense Part and of gradient clipping refuse, before anything reaches a GPU: the C entry points on
numbers that only look like pointers, and the Python layer on tensors of the wrong kind."""
import ctypes as C

import pytest
import torch

P = 1 << 20                      # a 16-byte aligned "address"; a call that is refused does not look at it


@pytest.fixture(scope="module")
def gb():
    from paper_1806_03925_b200 import build
    build.build()
    from paper_1806_03925_b200 import binding
    binding.load()
    return binding


NORM = dict(x=P, ldx=64, dtype=0, ids=None, vocab=0, res=None, ld_res=0, res_out=None, ld_res_out=0, weight=P, n=4, d_n=None, cols=64,
            eps=1e-6, out=P, ld_out=64, out_dtype=2, scale=P, status=None, stream=None)
BACK = dict(x=P, ldx=64, dtype=0, ids=None, vocab=0, weight=P, dout=P, ld_dout=64, dres=None, ld_dres=0, n=4, d_n=None, cols=64, eps=1e-6,
            dx=P, ld_dx=64, dweight=P, workspace=P, status=None, stream=None)
ROWS = dict(x=P, ldx=64, dtype=0, n=4, d_n=None, cols=64, q=P, ldq=64, scale=P, stream=None)
WEIGHTS = dict(W=P, ldw=32, K=64, N=32, q=P, ldq=64, scale=P, q_t=P, ldq_t=32, scale_t=P, stream=None)
MATMUL = dict(a=P, lda=64, a_scale=P, b=P, ldb=64, b_scale=P, n=4, d_n=None, N=32, K=64, out=P, ld_out=32, out_dtype=0, status=P, stream=None)


@pytest.mark.parametrize("name,base,wrong", [
    ("gear_rms_norm", NORM, [dict(dtype=2), dict(dtype=7), dict(n=-1), dict(n=1 << 31), dict(cols=0), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None),
                             dict(x=P + 2), dict(ldx=63), dict(out=None), dict(out=P + 2, out_dtype=0, scale=None), dict(ld_out=63), dict(out_dtype=3),
                             dict(scale=None), dict(out_dtype=0), dict(out_dtype=1), dict(scale=P + 1), dict(weight=P + 1), dict(res=P, ld_res=63),
                             dict(res=P + 1, ld_res=64), dict(res_out=P, ld_res_out=10), dict(ids=P, vocab=0), dict(ids=P, vocab=1 << 31)]),
    ("gear_rms_norm_backward", BACK, [dict(dtype=2), dict(n=-1), dict(cols=0), dict(eps=-1.0), dict(x=None), dict(ldx=63), dict(dout=None), dict(ld_dout=63),
                                      dict(dx=None, dweight=None), dict(workspace=None), dict(workspace=P + 4), dict(ld_dx=63), dict(dres=P, ld_dres=63),
                                      dict(dres=P + 1, ld_dres=64), dict(dweight=P + 2), dict(ids=P, vocab=-1)]),
    ("gear_q8_rows", ROWS, [dict(dtype=2), dict(n=-1), dict(cols=0), dict(x=None), dict(ldx=63), dict(q=None), dict(scale=None), dict(ldq=63), dict(scale=P + 2)]),
    ("gear_q8_weights", WEIGHTS, [dict(K=0), dict(N=0), dict(W=None), dict(W=P + 2), dict(ldw=31), dict(q=None, q_t=None), dict(scale=None), dict(scale_t=None),
                                  dict(ldq=63), dict(ldq_t=31)]),
    ("gear_q8_matmul", MATMUL, [dict(n=-1), dict(n=(1 << 31) - 1), dict(N=0), dict(K=0), dict(out_dtype=2), dict(status=None), dict(a=None), dict(b=None),
                                dict(a_scale=None), dict(b_scale=None), dict(out=None), dict(a=P + 8), dict(b=P + 8), dict(lda=72), dict(ldb=72), dict(lda=48),
                                dict(ldb=48), dict(K=65), dict(ld_out=31), dict(out=P + 2), dict(a_scale=P + 2)]),
])
def test_refusals(gb, name, base, wrong):
    fn = getattr(gb.load(), name)
    for change in wrong:
        assert fn(*dict(base, **change).values()) == gb.GEAR_ERR_ARG, change
        assert b"bad argument" in gb.load().gear_last_error()
    for b in (base, ) if "n" in base else ():
        if name != "gear_rms_norm_backward":            # (it clears dweight)
            assert fn(*dict(b, n=0).values()) == gb.GEAR_OK         # nothing to do, nothing looked at


def test_rows_too_long_to_step_over_are_refused(gb):
    """Columns are counted in 32 bits, in steps of up to 1024: the numbers of longer rows would wrap around."""
    L, far = gb.load(), 1 << 32
    for cols in ((1 << 31) - 1023, (1 << 31) - 512, (1 << 31) - 1):
        for name, base, long in (("gear_rms_norm", NORM, dict(cols=cols, ldx=far, ld_out=far)),
                                 ("gear_rms_norm_backward", BACK, dict(cols=cols, ldx=far, ld_dout=far, ld_dx=far)),
                                 ("gear_q8_rows", ROWS, dict(cols=cols, ldx=far, ldq=far)),
                                 ("gear_q8_weights", WEIGHTS, dict(K=cols, ldq=far)), ("gear_q8_weights", WEIGHTS, dict(N=cols, ldw=far, ldq_t=far)),
                                 ("gear_q8_matmul", MATMUL, dict(K=cols, lda=far, ldb=far)), ("gear_q8_matmul", MATMUL, dict(N=cols, ld_out=far))):
            assert getattr(L, name)(*dict(base, **long).values()) == gb.GEAR_ERR_ARG, (name, long)
            assert b"bad argument" in L.gear_last_error()


def test_no_rows_by_id_of_an_empty_table(gb):
    """Nothing to do: as with no rows of any other table.  (A row needs a table.)"""
    L = gb.load()
    assert L.gear_rms_norm(*dict(NORM, x=None, ids=P, vocab=0, n=0).values()) == gb.GEAR_OK
    assert L.gear_rms_norm_backward(*dict(BACK, x=None, ids=P, vocab=0, n=0, dweight=None, workspace=None).values()) == gb.GEAR_OK
    assert L.gear_rms_norm(*dict(NORM, ids=P, vocab=0, n=1).values()) == L.gear_rms_norm(*dict(NORM, ids=P, vocab=-1, n=0).values()) == gb.GEAR_ERR_ARG


def test_misaligned_scales_of_weights_are_refused(gb):
    for wrong in (dict(scale=P + 2), dict(scale_t=P + 1), dict(q=None, scale_t=P + 2), dict(q_t=None, scale=P + 3)):
        assert gb.load().gear_q8_weights(*dict(WEIGHTS, **wrong).values()) == gb.GEAR_ERR_ARG, wrong
        assert b"scale" in gb.load().gear_last_error()


def test_refusals_of_gradient_lists(gb):
    L = gb.load()

    def call(items, norm=P, workspace=P, max_norm=1.0, count=None, clip=True):
        a = (gb.gear_grad * max(1, len(items)))(*items)
        n = len(items) if count is None else count
        return L.gear_clip_grads(a, n, max_norm, norm, workspace, None) if clip else L.gear_grad_norm(a, n, norm, workspace, None)

    good = (P, P, 8, 0)
    for kw in (dict(norm=None), dict(workspace=None), dict(workspace=P + 4), dict(norm=P + 1), dict(count=-1), dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        assert call([good], **kw) == gb.GEAR_ERR_ARG, kw
    for item in ((None, P, 8, 0), (P, None, 8, 0), (P + 2, P, 8, 0), (P, P + 2, 8, 0), (P + 1, P, 8, 1), (P, P, -1, 0), (P, P, 8, 2)):
        assert call([good, item]) == gb.GEAR_ERR_ARG, item
    assert call([(None, None, 8, 0)], clip=False) == gb.GEAR_ERR_ARG
    assert L.gear_clip_grads(None, 1, 1.0, P, P, None) == gb.GEAR_ERR_ARG


def test_a_norm_of_the_same_gradient_twice(gb, monkeypatch):
    """Nothing is written, so nothing is written twice: the sum has the gradient's squares twice."""
    class Library:
        def gear_grad_norm(self, items, count, norm, workspace, stream):
            self.seen = [(items[i].grad, items[i].n) for i in range(count)]
            return gb.GEAR_OK
    lib = Library()
    monkeypatch.setattr(gb, "_lib", lib)
    monkeypatch.setattr(gb, "_device", lambda: -1)
    monkeypatch.setattr(gb, "_current_stream", lambda dev: 0)
    g = torch.ones(10)
    gb.gear_grad_norm([g, g, g[2:5]], torch.zeros(2), torch.empty(gb.GEAR_CLIP_WORKSPACE_BYTES, dtype=torch.uint8))
    assert lib.seen == [(g.data_ptr(), 10), (g.data_ptr(), 10), (g.data_ptr() + 8, 3)]


def test_overlapping_gradients_are_refused(gb, monkeypatch):
    """What is written may be its own gradient, whole, and nothing else of the call."""
    monkeypatch.setattr(gb, "_device", lambda: -1)
    flat, back = torch.zeros(100), torch.zeros(100)
    for grads, outs in (([flat[:10], flat[9:20]], None), ([flat[9:20], flat[:10]], None), ([flat, flat[50:60]], None), ([flat[:50], flat[3:4], flat[60:]], None),
                        ([flat[:10], flat[10:20]], [back[:10], back[9:19]]), ([flat[:10]], [flat[1:11]]), ([flat[:10], flat[10:20]], [flat[10:20], flat[:10]]),
                        ([flat[:10], flat[20:30]], [flat[20:30], back[:10]]), ([flat[:10], flat[:10]], [back[:10], back[:10]]),
                        ([flat[:10], flat[2:4]], [flat[:10], back[:2]])):
        with pytest.raises(TypeError, match="overlap|written twice"):
            gb.make_grads(grads, outs)
    half = flat.view(torch.bfloat16)
    with pytest.raises(TypeError, match="overlap|written twice"):
        gb.make_grads([flat[:10], half[19:30]])
    for grads, outs in (([flat[:10], flat[10:20], flat[20:]], None), ([flat[10:20], flat[:10], flat[:0], flat[5:5]], None), ([flat[:10], flat[5:15]], [back[:10], back[10:20]]),
                        ([flat[:10], half[20:30]], None), ([flat[:10], flat[20:30]], [flat[:10], flat[40:50]]), ([], None), ([flat[:0], flat[:0]], None)):
        l = gb.make_grads(grads, outs)
        assert l.count == len(grads)
        for i, (g, o) in enumerate(zip(grads, outs or grads)):
            assert (l.items[i].grad or 0, l.items[i].out or 0, l.items[i].n) == (g.data_ptr(), o.data_ptr(), g.numel())


def test_struct_layout_of_gradient_lists(gb, tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = [f for f, _ in gb.gear_grad._fields_]
    src = tmp_path / "l.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gear.h"\nint main(void){printf("%zu", sizeof(gear_grad));' +
                   "".join('printf(" %%zu", offsetof(gear_grad, %s));' % f for f in fields) +
                   'printf(" %d %d %d %d\\n", GEAR_E4M3, GEAR_Q8_BLOCK, GEAR_NORM_WORKSPACE_ROWS, GEAR_CLIP_WORKSPACE_BYTES);return 0;}\n')
    subprocess.check_call([cc, "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "l")])
    seen = [int(v) for v in subprocess.check_output([str(tmp_path / "l")], text=True).split()]
    assert seen == [C.sizeof(gb.gear_grad)] + [getattr(gb.gear_grad, f).offset for f in fields] + \
        [gb.GEAR_E4M3, gb.GEAR_Q8_BLOCK, gb.GEAR_NORM_WORKSPACE_ROWS, gb.GEAR_CLIP_WORKSPACE_BYTES]


def test_row_checks_of_the_binding(gb):
    """The shape checks of the Python layer, on host tensors taken for those of "device" -1."""
    x = torch.zeros((6, 40))
    assert gb._rows(x, gb._FLOATS, -1) == (x.data_ptr(), 40, gb.GEAR_F32)
    assert gb._rows(x[:, 8:24], gb._FLOATS, -1, 6, 16)[1] == 40
    assert gb._rows(x[1:2, :8], gb._FLOATS, -1)[1] >= 8
    for bad in (lambda: gb._rows(x.t(), gb._FLOATS, -1), lambda: gb._rows(x[:, ::2], gb._FLOATS, -1), lambda: gb._rows(x, gb._FLOATS, -1, 7),
                lambda: gb._rows(x, gb._FLOATS, -1, 6, 41), lambda: gb._rows(x.double(), gb._FLOATS, -1), lambda: gb._rows(x[0], gb._FLOATS, -1),
                lambda: gb._rows(x, gb._FLOATS, 0), lambda: gb._vec(x.t(), torch.float32, -1), lambda: gb._vec(x, torch.float32, -1, 241),
                lambda: gb._vec(x, torch.int32, -1), lambda: gb._vec(x, torch.float32, 0), lambda: gb._row_count(7, x), lambda: gb._row_count(-1, x)):
        with pytest.raises(TypeError):
            bad()
    assert gb._vec(None, torch.float32, 0) is None and gb._row_count(None, x) == (6, 40) and gb._row_count(2, x) == (2, 40)
