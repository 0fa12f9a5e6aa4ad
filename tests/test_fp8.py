"""What the operators on 8-bit floats refuse (no GPU: everything is refused on the host, before a launch), and the plain forms
that the GPU tests compare with, against each other."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import fp8_util as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2111_09547_amd", "lib", "libqgtc.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libqgtc.so not built (run __graft_entry__.build())")

OK, NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 4, 6, 7


@pytest.fixture(scope="module")
def b():
    import paper_2111_09547_amd.binding as b
    return b


def form(b, rows, cols, **more):
    d = b._Fp8C()
    assert b.lib().qgtc_fp8_describe(C.byref(d), rows, cols) == OK
    d.codes, d.scales = 0x10000, 0x20000            # never dereferenced: nothing is launched
    for k, v in more.items():
        setattr(d, k, v)
    return d


@needs_lib
def test_describe(b):
    for rows, cols, ld, lds in ((3, 1, 128, 4), (3, 128, 128, 4), (5, 513, 640, 8), (5, 512, 512, 4), (0, 0, 0, 0), (7, 4096, 4096, 32)):
        d = form(b, rows, cols)
        assert (d.rows, d.cols, d.ld, d.ld_scales) == (rows, cols, ld, lds)
    d = b._Fp8C()
    assert b.lib().qgtc_fp8_describe(C.byref(d), -1, 4) == SHAPE and b.lib().qgtc_fp8_describe(None, 1, 1) == NULL


@needs_lib
@pytest.mark.parametrize("columns", [0, 1])
def test_quantize_refuses(b, columns):
    f = b.lib().qgtc_fp8_quantize

    def call(rows=8, cols=300, ld=300, type=0, src=0x30000, dst=None, **more):
        d = form(b, *((cols, rows) if columns else (rows, cols)), **more) if dst is None else dst
        return f(src, type, rows, cols, ld, columns, C.byref(d), None)
    assert call(src=None) == NULL and f(0x30000, 0, 8, 300, 300, columns, None, None) == NULL
    assert call(codes=None) == NULL and call(scales=None) == NULL
    assert call(type=3) == UNSUPPORTED and call(type=-1) == UNSUPPORTED
    assert call(rows=-1, dst=form(b, 8, 300)) == SHAPE and call(ld=299) == SHAPE
    assert call(dst=form(b, 9, 300)) == SHAPE
    assert call(codes=0x10008) == ALIGN and call(scales=0x20002) == ALIGN and call(ld=300, src=0x30001) == ALIGN
    assert call(src=0x30002) == ALIGN                # fp32 at half an entry
    bad = form(b, *((300, 8) if columns else (8, 300)))
    bad.ld += 64
    assert call(dst=bad) == ALIGN
    bad.ld -= 64 + 128
    assert call(dst=bad) == SHAPE
    bad = form(b, *((300, 8) if columns else (8, 300)))
    bad.ld_scales = 5
    assert call(dst=bad) == ALIGN
    bad.ld_scales = 0
    assert call(dst=bad) == SHAPE
    big = form(b, 1, 1)
    big.rows, big.cols, big.ld = (1, (1 << 29) + 1, 1 << 30)
    assert f(0x30000, 0, 1, (1 << 29) + 1, 1 << 30, 0, C.byref(big), None) == SHAPE
    assert call(rows=0, src=None) == OK


@needs_lib
def test_norm_refuses(b):
    f = b.lib().qgtc_rms_norm

    def call(out=None, **more):
        n = b._NormC(0, 0, 8, 300, 1e-6, 0, 0x10000, 300, None, 0, 0x20000, 0x30000, 300, 0x40000, 300, 0x50000)
        if out is not None:
            n.out = C.addressof(out)
        for k, v in more.items():
            setattr(n, k, v)
        return f(C.byref(n), None)
    assert f(None, None) == NULL and call(x=None) == NULL and call(weight=None) == NULL
    assert call(type=3) == UNSUPPORTED and call(weight_type=-1) == UNSUPPORTED
    assert call(cols=32769, ld_x=32769, ld_sum=32769, ld_y=32769) == UNSUPPORTED
    assert call(rows=-1) == SHAPE and call(cols=-1) == SHAPE
    assert call(ld_x=299) == SHAPE and call(ld_sum=299) == SHAPE and call(ld_y=299) == SHAPE and call(residual=0x60000, ld_residual=1) == SHAPE
    assert call(x=0x10002) == ALIGN and call(sum=0x30001) == ALIGN and call(rstd=0x50002) == ALIGN and call(type=1, x=0x10001) == ALIGN
    assert call(sum=0x10000, ld_sum=301) == SHAPE
    assert call(out=form(b, 8, 301)) == SHAPE and call(out=form(b, 7, 300)) == SHAPE and call(out=form(b, 8, 300, codes=None)) == NULL
    assert call(rows=0, x=None) == OK and call(cols=0, x=None) == OK
    assert call(sum=None, y=None, rstd=None) == OK   # nothing is asked for


@needs_lib
def test_norm_backward_refuses(b):
    f, size = b.lib().qgtc_rms_norm_backward, b.lib().qgtc_rms_norm_backward_workspace_bytes
    need = size(8, 300)
    assert need >= 300 * 4 and size(0, 300) == 0 and size(8, 0) == 0 and size(8, 32769) == 0 and size(-1, 5) == 0

    def call(ws=0x90000, nbytes=need, **more):
        n = b._NormGradC(0, 0, 8, 300, 0x10000, 300, 0x20000, 300, 0x30000, 0x40000, None, 0, 0x50000, 300, 0x60000)
        for k, v in more.items():
            setattr(n, k, v)
        return f(C.byref(n), ws, nbytes, None)
    assert f(None, None, 0, None) == NULL
    for k in ("dy", "sum", "weight", "rstd", "dx"):
        assert call(**{k: None}) == NULL, k
    assert call(ws=None) == NULL and call(ws=0x90008) == ALIGN and call(nbytes=need - 1) == WORKSPACE
    assert call(type=7) == UNSUPPORTED and call(weight_type=7) == UNSUPPORTED and call(cols=32769) == UNSUPPORTED
    assert call(dx=0x20000) == UNSUPPORTED           # the sum is read again by nobody, but its row is shared
    assert call(ld_dy=299) == SHAPE and call(ld_sum=1) == SHAPE and call(ld_dx=2) == SHAPE and call(dsum=0x70000, ld_dsum=2) == SHAPE
    assert call(dx=0x10000, ld_dx=304) == SHAPE and call(rows=-1) == SHAPE
    assert call(dy=0x10002) == ALIGN and call(rstd=0x40002) == ALIGN and call(dweight=0x60001) == ALIGN
    assert call(rows=0, dweight=None, dy=None) == OK and call(cols=0) == OK


@needs_lib
def test_product_refuses(b):
    f = b.lib().qgtc_fp8_product
    X, W = form(b, 8, 300), form(b, 20, 300)

    def call(x=X, w=W, type=0, out=0x30000, ld=20):
        return f(C.byref(x) if x else None, C.byref(w) if w else None, type, out, ld, None)
    assert call(x=None) == NULL and call(w=None) == NULL and call(out=None) == NULL
    assert call(x=form(b, 8, 300, codes=None)) == NULL
    assert call(w=form(b, 20, 301)) == SHAPE and call(ld=19) == SHAPE and call(x=form(b, 8, 300, ld=256)) == SHAPE
    assert call(type=3) == UNSUPPORTED
    assert call(out=0x30002) == ALIGN and call(type=2, out=0x30001) == ALIGN
    assert call(x=form(b, 8, 300, ld=448)) == ALIGN and call(w=form(b, 20, 300, codes=0x10004)) == ALIGN
    for more in ({"ld": (1 << 24) + 128}, {"ld_scales": (1 << 24) + 4}):
        assert call(x=form(b, 8, 300, **more)) == UNSUPPORTED and call(w=form(b, 20, 300, **more)) == UNSUPPORTED
    assert call(x=form(b, 8, 1 << 24), w=form(b, 20, 1 << 24)) == UNSUPPORTED
    assert call(x=form(b, 0, 300), out=None) == OK and call(w=form(b, 0, 300), out=None) == OK


@needs_lib
def test_gated_refuses(b):
    f, size = b.lib().qgtc_fp8_gated, b.lib().qgtc_fp8_gated_workspace_bytes
    X, G, P = form(b, 8, 300), form(b, 20, 300), form(b, 20, 300)
    ref = lambda m: C.byref(m) if m is not None else None          # noqa: E731

    def call(x=X, g=G, u=P, act=0, out=None, type=0, h=0x30000, ld=20, ws=0x40000, nbytes=1 << 20):
        return f(ref(x), ref(g), ref(u), act, ref(out), type, h, ld, ws, nbytes, None)
    assert call(x=None) == NULL and call(g=None) == NULL and call(u=None) == NULL and call(h=None) == NULL
    assert call(act=2) == UNSUPPORTED and call(act=-1) == UNSUPPORTED and call(type=3) == UNSUPPORTED
    assert call(u=form(b, 21, 300)) == SHAPE and call(u=form(b, 20, 299)) == SHAPE and call(g=form(b, 20, 299)) == SHAPE and call(ld=19) == SHAPE
    assert call(out=form(b, 8, 21)) == SHAPE and call(out=form(b, 7, 20)) == SHAPE and call(out=form(b, 8, 20, scales=None)) == NULL
    need = size(8, 20, 300)
    if need:
        assert call(out=form(b, 8, 20), ws=None, type=2) == NULL and call(out=form(b, 8, 20), ws=0x40008, type=2) == ALIGN
        assert call(out=form(b, 8, 20), nbytes=need - 1, type=2) == WORKSPACE and call(out=form(b, 8, 20), h=None, ws=None) == NULL
    assert size(0, 20, 300) == 0 and size(8, 0, 300) == 0
    assert call(x=form(b, 0, 300), h=None, out=form(b, 0, 20)) == OK

    f2 = b.lib().qgtc_fp8_gated_backward

    def back(x=X, g=G, u=P, act=0, type=0, dh=0x30000, ld_dh=20, dg=0x50000, ld_dg=40, du=0x60000, ld_du=40):
        return f2(ref(x), ref(g), ref(u), act, type, dh, ld_dh, dg, ld_dg, du, ld_du, None)
    for k in ("x", "g", "u", "dh", "dg", "du"):
        assert back(**{k: None}) == NULL, k
    assert back(act=5) == UNSUPPORTED and back(type=5) == UNSUPPORTED
    assert back(ld_dh=19) == SHAPE and back(ld_dg=19) == SHAPE and back(ld_du=19) == SHAPE and back(u=form(b, 21, 300)) == SHAPE
    assert back(dh=0x30002) == ALIGN and back(type=1, du=0x60001) == ALIGN
    assert back(x=form(b, 0, 300), dh=None) == OK


@needs_lib
def test_python_refuses_what_is_not_on_the_device():
    import paper_2111_09547_amd as q
    x = torch.zeros((4, 256))
    for call in (lambda: q.qgtc_fp8_quantize(x), lambda: q.qgtc_rms_norm(x, torch.ones(256)),
                 lambda: q.qgtc_rms_norm_backward(x, x, torch.ones(256), torch.ones(4)),
                 lambda: q.Fp8(torch.zeros((4, 256), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: q.qgtc_fp8_quantize(x.double()), lambda: q.qgtc_fp8_quantize(x[0]),
                 lambda: q.Fp8(x, torch.zeros((4, 4), dtype=torch.uint8))):
        with pytest.raises(TypeError):
            call()


# ---- the plain forms --------------------------------------------------------------------------------------------
def test_plain_quantizer():
    x = U.activations(30, 500, 1).numpy()
    x[3, 200], x[4] = 1e30, 0.0
    x[5, :128] = 448.0
    x[6, :128] = np.nextafter(np.float32(448.0), np.float32(1e9))
    codes, scales = U.quantized(x)
    v = U.values(codes, scales, 500)
    top = np.abs(np.pad(x, ((0, 0), (0, 12))).reshape(30, 4, 128)).max(2)
    two = np.ldexp(1.0, scales.astype(int) - 127)
    assert (448 * two >= top).all() and ((224 * two < top) | (scales == 0)).all()
    assert scales[5, 0] == 127 and scales[6, 0] == 128 and (v[4] == 0).all()
    half = np.maximum(np.abs(x) / 16, np.repeat(two, 128, 1)[:, :500] * 2.0 ** -10)
    assert (np.abs(v - x) <= half).all()


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_plain_gate_slopes_are_differences(name):
    g = np.linspace(-9, 9, 400)
    a, s, curve = U.act(name, g)
    step = 1e-5
    assert np.abs((U.act(name, g + step)[0] - U.act(name, g - step)[0]) / (2 * step) - s).max() < 1e-9
    assert np.abs((U.act(name, g + step)[1] - U.act(name, g - step)[1]) / (2 * step)).max() <= curve
    assert np.abs(s).max() <= 1.13


@needs_lib
def test_python_refuses_to_lose_gradients():
    """Where torch would record: every operand that requires a gradient.  (Refused before a tensor's device is looked at.)"""
    import paper_2111_09547_amd as q
    x, g = torch.zeros((4, 256)), torch.zeros((4, 256), requires_grad=True)
    for call in (lambda: q.qgtc_fp8_quantize(g), lambda: q.qgtc_fp8_quantize(g, columns=True), lambda: q.qgtc_rms_norm(g, torch.ones(256)),
                 lambda: q.qgtc_rms_norm_backward(x, g, torch.ones(256), torch.ones(4))):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="device"):
            call()
