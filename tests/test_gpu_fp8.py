"""Operators on 8-bit floats on an MI355X, against plain forms in 64 bits (fp8_util.py)."""
import numpy as np
import pytest
import torch

import fp8_util as U

pytestmark = pytest.mark.gpu

q = pytest.importorskip("paper_2111_09547_amd")

ROWS = [1, 2, 15, 17, 33, 64, 100, 129, 260]


def fp8_of(x, ld=None, cols=None):
    """A CPU matrix in 8-bit floats on the device, made by the definition."""
    codes, scales = U.quantized(x.float().numpy())
    rows, blocks = codes.shape[0], scales.shape[1]
    wide = torch.zeros((rows, ld or codes.shape[1]), dtype=torch.uint8)
    wide[:, :codes.shape[1]] = torch.from_numpy(codes)
    s = torch.full((rows, -(-blocks // 4) * 4), 255, dtype=torch.uint8)     # (past the last block: never used)
    s[:, :blocks] = torch.from_numpy(scales)
    return q.Fp8(wide.cuda(), s.cuda(), x.shape[1] if cols is None else cols), U.values(codes, scales, x.shape[1])


def odd(t, dtype):
    """t on the device as a view that starts at an odd entry and whose rows lie apart."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + 5) + 8,), 7.0, dtype=dtype, device="cuda")
    v = buf[3:3 + rows * (cols + 5)].view(rows, cols + 5)[:, :cols]
    v.copy_(t.to(dtype))
    return v


# ---- quantizing ---------------------------------------------------------------------------------------------------
def special(rows, cols, dtype, seed):
    x = U.activations(rows, cols, seed).to(dtype)
    top = torch.finfo(dtype).max
    put = [0.0, -0.0, torch.finfo(dtype).tiny, torch.finfo(dtype).smallest_normal / 4, top, -top]
    flat = x.view(-1)
    for i, v in enumerate(put):
        flat[(i * 7919) % flat.numel()] = v
    return x


@pytest.mark.parametrize("dtype", U.TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 127), (2, 128), (3, 129), (5, 1000), (130, 512), (257, 513), (4, 4100), (64, 64)])
@pytest.mark.parametrize("columns", [False, True])
def test_quantize_is_the_definition(dtype, rows, cols, columns):
    x = special(rows, cols, dtype, rows + cols)
    for src in (x.cuda(), odd(x, dtype)):
        m = q.qgtc_fp8_quantize(src, columns=columns)
        codes, scales = U.quantized((x.t() if columns else x).float().numpy())
        assert (m.rows, m.cols) == ((cols, rows) if columns else (rows, cols))
        assert (U.raw(m.scales)[:, :m.blocks] == scales).all()
        assert (U.raw(m.codes) == codes).all()


@pytest.mark.parametrize("columns", [False, True])
def test_quantize_borders_and_non_finite_blocks(columns):
    rows = 40
    x = torch.zeros((rows, 300))
    for i in range(rows - 4):                          # largest entries at and one step above 448 * 2^k
        top = np.float32(np.ldexp(448.0, i * 7 - 130))
        x[i, 5] = float(top)
        x[i, 140] = float(np.nextafter(top, np.float32(np.inf)))
        x[i, 280] = -float(np.nextafter(top, np.float32(0)))
        x[i, 6] = float(top) / 1000
    x[-1, 7], x[-2, 130], x[-3, 299] = float("inf"), float("nan"), float("-inf")
    x[-1, 3], x[-2, 131], x[-3, 298] = 1.0, 2.0, 3.0
    src = x.t().contiguous() if columns else x
    m = q.qgtc_fp8_quantize(src.cuda(), columns=columns)
    codes, scales = U.quantized(x.numpy())
    assert (U.raw(m.scales)[:, :m.blocks] == scales).all()
    assert (U.raw(m.codes) == codes).all()
    assert (scales == 255).sum() == 3


def test_quantize_leaves_what_is_behind():
    x = U.activations(9, 200, 3)
    codes = torch.full((12, 512), 99, dtype=torch.uint8, device="cuda")
    scales = torch.full((12, 8), 98, dtype=torch.uint8, device="cuda")
    m = q.qgtc_fp8_quantize(x.cuda(), out=q.Fp8(codes[:9], scales[:9], 200))
    want, s = U.quantized(x.numpy())
    assert (U.raw(codes)[:9, :256] == want).all() and (U.raw(codes)[:9, 256:] == 99).all() and (U.raw(codes)[9:] == 99).all()
    assert (U.raw(scales)[:9, :2] == s).all() and (U.raw(scales)[:, 2:] == 98).all() and (U.raw(scales)[9:] == 98).all()
    assert m.codes is codes[:9] or m.codes.data_ptr() == codes.data_ptr()


# ---- norm -----------------------------------------------------------------------------------------------------------
COLS = [1, 8, 127, 128, 500, 512, 513, 1000, 1024, 1030, 2048, 4096, 5000, 8192, 8193, 16384, 20000, 32768]


@pytest.mark.parametrize("dtype", U.TYPES)
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(dtype, cols, residual):
    rows, eps = (7 if cols < 4096 else 3), 1e-5
    x, res = (U.activations(rows, cols, k).to(dtype) for k in (1, 2))
    w = (1 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(3))).to(torch.float32 if cols % 2 else dtype)
    for at in (lambda t: t.cuda(), lambda t: odd(t, dtype)):
        n = q.qgtc_rms_norm(at(x), w.cuda(), eps, residual=at(res) if residual else None, y=True, rstd=True)
        s = (x.float() + res.float()).to(dtype) if residual else x
        assert torch.equal(n.sum.cpu(), s)
        s = U.f64(s)
        root = 1 / np.sqrt((s * s).mean(1) + np.float64(np.float32(eps)))
        # a lane adds up to 32 squares, 64 lanes and 16 waves follow: at most 56 roundings of the sum, half of that in its root,
        # and four more for the division, the addition, the root and its reciprocal
        off = (28 + 4) * 2.0 ** -24
        U.close(n.rstd, root, off * root, "rstd")
        y = s * root[:, None] * U.f64(w)
        tol = np.abs(y) * (off + 2 * 2.0 ** -24)
        U.close(n.y, y, tol * 1.01 + U.rounded_tol(y, dtype), "y")
        U.check_codes(n.fp8, y, tol + 2.0 ** -149, "codes")


@pytest.mark.parametrize("cols", [128, 513, 4096])
def test_norm_in_place_and_single_outputs(cols):
    x, res = (U.activations(5, cols, k).bfloat16().cuda() for k in (4, 5))
    w = torch.ones(cols, device="cuda")
    want = q.qgtc_rms_norm(x, w, residual=res, y=True, rstd=True)
    for other in ("x", "residual"):
        a, b = x.clone(), res.clone()
        n = q.qgtc_rms_norm(a, w, residual=b, sum_out=a if other == "x" else b)
        assert n.sum is (a if other == "x" else b) and torch.equal(n.sum, want.sum)
        assert torch.equal(n.fp8.codes.view(torch.uint8), want.fp8.codes.view(torch.uint8)) and n.y is None and n.rstd is None
    n = q.qgtc_rms_norm(x, w, residual=res, fp8=False, y=True)
    assert n.fp8 is None and torch.equal(n.y, want.y)


def test_norm_keeps_bad_rows_to_themselves():
    x = U.activations(6, 700, 6)
    want = q.qgtc_rms_norm(x.cuda(), torch.ones(700, device="cuda"), y=True)
    x[1, 3], x[4, 699] = float("nan"), float("inf")
    x[2] = 0.0
    n = q.qgtc_rms_norm(x.cuda(), torch.ones(700, device="cuda"), y=True)
    for r in (0, 3, 5):
        assert torch.equal(n.y[r], want.y[r]) and (U.raw(n.fp8.codes)[r] == U.raw(want.fp8.codes)[r]).all()
    assert torch.isnan(n.y[1]).all() and np.isnan(U.fp8_values(n.fp8)[1]).all()
    assert torch.isnan(n.y[4, 699]) and (n.y[4, :699] == 0).all()          # x / inf
    assert (n.y[2] == 0).all() and (U.raw(n.fp8.codes)[2] == 0).all()
    assert (U.raw(n.fp8.codes)[:, 700:] == 0).all()


@pytest.mark.parametrize("dtype", U.TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 128), (5, 500), (7, 512), (600, 300), (9, 513), (530, 1030), (700, 4096), (3, 5000), (4, 8192), (5, 9000), (3, 20000), (2, 32768)])
@pytest.mark.parametrize("dsum", [False, True])
def test_norm_gradients(dtype, rows, cols, dsum):
    s, ds = (U.activations(rows, cols, k).to(dtype) for k in (7, 8))
    dy = (torch.randn((rows, cols), generator=torch.Generator().manual_seed(9)) * 0.1).to(dtype)
    w = (1 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(3))).to(dtype)
    root = (1 / torch.sqrt(s.double().square().mean(1) + 1e-5)).float()
    hat, g, r = U.f64(s) * U.f64(root)[:, None], U.f64(dy) * U.f64(w), U.f64(root)[:, None]
    want = r * (g - hat * (g * hat).mean(1, keepdims=True))
    # the mean: at most 56 roundings of the sum as above, and of its terms; a few more for the rest
    tol = 2.0 ** -24 * r * (4 * np.abs(g) + np.abs(hat) * 64 * np.abs(g * hat).mean(1, keepdims=True))
    if dsum:
        want = want + U.f64(ds)
        tol = tol + 2.0 ** -24 * np.abs(want)
    tol = tol * 1.01 + U.rounded_tol(want, dtype)
    dw = (U.f64(dy) * hat).sum(0)
    dw_tol = (rows + 8) * 2.0 ** -24 * np.abs(U.f64(dy) * hat).sum(0) + 1e-38
    for at in (lambda t: t.cuda(), lambda t: odd(t, dtype)):
        dx, dweight = q.qgtc_rms_norm_backward(at(dy), at(s), w.cuda(), root.cuda(), dsum=at(ds) if dsum else None)
        U.close(dx, want, tol, "dx")
        U.close(dweight, dw, dw_tol, "dweight")
        only, none = q.qgtc_rms_norm_backward(at(dy), at(s), w.cuda(), root.cuda(), dsum=at(ds) if dsum else None, dweight=False)
        assert none is None and torch.equal(only, dx)


def test_norm_gradients_in_place_and_of_no_rows():
    s, dy, ds = (U.activations(40, 700, k).cuda() for k in (1, 2, 3))
    w = torch.ones(700, device="cuda")
    root = torch.rsqrt(s.square().mean(1) + 1e-6)
    dx, dw = q.qgtc_rms_norm_backward(dy, s, w, root, dsum=ds)
    for k in (0, 1):
        a, b = dy.clone(), ds.clone()
        got, gw = q.qgtc_rms_norm_backward(a, s, w, root, dsum=b, out=(a, b)[k])
        assert torch.equal(got, dx) and torch.equal(gw, dw)
    empty = torch.empty((0, 700), device="cuda")
    got, gw = q.qgtc_rms_norm_backward(empty, empty, w, torch.empty(0, device="cuda"))
    assert got.shape == (0, 700) and (gw == 0).all()


def test_norm_gradients_are_differences():
    """dx against central differences of the norm itself, in 64 bits."""
    rows, cols, eps = 2, 40, 1e-5
    s = torch.randn((rows, cols), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    w = 1 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    dy = torch.randn((rows, cols), generator=torch.Generator().manual_seed(3), dtype=torch.float64)

    def loss(t):
        return (t / torch.sqrt(t.square().mean(1, keepdim=True) + eps) * w * dy).sum()
    root = 1 / torch.sqrt(s.square().mean(1) + eps)
    dx, dw = q.qgtc_rms_norm_backward(dy.float().cuda(), s.float().cuda(), w.float().cuda(), root.float().cuda())
    step = 1e-5
    for i in range(rows):
        for j in range(0, cols, 7):
            d = torch.zeros_like(s)
            d[i, j] = step
            want = float(loss(s + d) - loss(s - d)) / (2 * step)
            # differences: step^2 times third derivatives (below 100 here), roundings 1e-16 * 40 / step; the kernel's fp32 and
            # its fp32 inputs: some 2^-24 of sums of at most 40 terms of size 3
            assert abs(float(dx[i, j]) - want) < 1e-8 + 1e-9 + 100 * 2.0 ** -24 * 3


# ---- products -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("cols,inner", [(1, 1), (16, 128), (17, 129), (100, 500), (256, 512), (129, 640), (300, 1030), (31, 4200)])
def test_product(rows, cols, inner):
    X, x = fp8_of(U.activations(rows, inner, 1))
    W, w = fp8_of(U.weights(cols, inner, 2))
    want = x @ w.T
    for dtype in U.TYPES:
        tol = U.product_tol(x, w, dtype == torch.float32)
        U.close(q.qgtc_fp8_product(X, W, dtype), want, tol * 1.01 + U.rounded_tol(want, dtype), (rows, cols, inner, dtype))


@pytest.mark.parametrize("rows,cols,inner", [(3, 40, 300), (70, 200, 300), (300, 300, 900), (513, 1030, 260)])
def test_product_between_other_data(rows, cols, inner):
    """Leading dimensions of operands and result, an output at an odd address, and nothing written around it."""
    X, x = fp8_of(U.activations(rows, inner, 1), ld=1280)
    W, w = fp8_of(U.weights(cols, inner, 2), ld=1152)
    want = x @ w.T
    for dtype in U.TYPES:
        tol = U.product_tol(x, w, dtype == torch.float32)
        buf = torch.full((rows + 2, cols + 7), 5.0, dtype=dtype, device="cuda")
        out = buf[1:rows + 1, 3:cols + 3]
        assert q.qgtc_fp8_product(X, W, out=out) is out
        U.close(out, want, tol * 1.01 + U.rounded_tol(want, dtype))
        buf[1:rows + 1, 3:cols + 3] = 5.0
        assert (buf == 5.0).all()


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_product_of_bad_blocks(rows):
    """An infinity in a row of X or W reaches that row's and that column's results and no others."""
    xs, ws = U.activations(rows, 700, 1), U.weights(300, 700, 2)
    xs[rows // 2, 699], ws[77, 130] = float("inf"), float("nan")
    xs[0] = 0.0
    (X, x), (W, w) = fp8_of(xs), fp8_of(ws)
    x[rows // 2], w[77] = 0.0, 0.0
    want = x @ w.T
    for dtype in U.TYPES:
        got = U.f64(q.qgtc_fp8_product(X, W, dtype))
        bad = np.zeros(got.shape, bool)
        bad[rows // 2], bad[:, 77] = True, True
        assert np.isnan(got[bad]).all()
        ok = np.abs(got - want) <= U.product_tol(x, w, dtype == torch.float32) * 1.01 + U.rounded_tol(want, dtype)
        assert (ok | bad).all() and (got[0][~bad[0]] == 0).all()


def test_product_of_extreme_scales():
    """Products of scales far apart: the instruction's exponents add up, in the range of fp32."""
    xs, ws = U.activations(20, 512, 1), U.weights(64, 512, 2)
    for b, (p, r) in enumerate([(60, -60), (-100, 90), (0, 0), (100, -110)]):
        xs[:, b * 128:b * 128 + 128] *= 2.0 ** p
        ws[:, b * 128:b * 128 + 128] *= 2.0 ** r
    (X, x), (W, w) = fp8_of(xs), fp8_of(ws)
    want = x @ w.T
    for dtype in (torch.float32, torch.bfloat16):
        U.close(q.qgtc_fp8_product(X, W, dtype), want, U.product_tol(x, w, dtype == torch.float32) * 1.01 + U.rounded_tol(want, dtype))


@pytest.mark.parametrize("rows", [5, 300])
def test_product_of_the_smallest_scales(rows):
    """Blocks whose scale is 2^-127 and a little more."""
    xs, ws = U.activations(rows, 384, 1), U.weights(300, 384, 2) * 2.0 ** 100
    xs[:, :128] *= 2.0 ** -126
    xs[:, 128:256] *= 2.0 ** -122
    xs[:, 256:] *= 2.0 ** -118
    (X, x), (W, w) = fp8_of(xs), fp8_of(ws)
    assert (U.raw(X.scales)[:, 0] == 0).all() and (U.raw(X.scales)[:, 2] > 0).any()
    want = x @ w.T
    for dtype in (torch.bfloat16, torch.float32):
        tol = U.product_tol(x, w, dtype == torch.float32) * 1.01 + U.rounded_tol(want, dtype)
        if dtype == torch.float32:                      # values below 2^-126 go as subnormal bf16, with steps of 2^-133
            tol = tol + 2.0 ** -134 * np.abs(w).sum(1)[None, :]
        U.close(q.qgtc_fp8_product(X, W, dtype), want, tol, dtype)


def test_product_of_nothing():
    X, W = q.Fp8(torch.empty((5, 0), dtype=torch.uint8, device="cuda"), torch.empty((5, 0), dtype=torch.uint8, device="cuda")), \
        q.Fp8(torch.empty((300, 0), dtype=torch.uint8, device="cuda"), torch.empty((300, 0), dtype=torch.uint8, device="cuda"))
    assert (q.qgtc_fp8_product(X, W, torch.float32) == 0).all()
    X, W = q.alloc_fp8(0, 128, "cuda"), q.alloc_fp8(7, 128, "cuda")
    assert q.qgtc_fp8_product(X, W).shape == (0, 7) and q.qgtc_fp8_product(W, X).shape == (7, 0)
    assert q.qgtc_fp8_gated(X, W, W).codes.shape == (0, 128)
    assert q.qgtc_fp8_quantize(torch.empty((0, 5), device="cuda")).rows == 0
    assert q.qgtc_rms_norm(torch.empty((0, 5), device="cuda"), torch.ones(5, device="cuda")).fp8.rows == 0


@pytest.mark.parametrize("rows", [2, 300])
def test_offsets_past_32_bits(rows):
    """Rows that lie further apart than 2^32 bytes from first to last."""
    ld, n, inner = 1 << 24, 300, 300
    W, w = fp8_of(U.weights(n, inner, 2))
    buf = torch.empty((n, ld), dtype=torch.uint8, device="cuda")                # 5 GB
    buf[:, :384] = W.codes[:, :384]
    X, x = fp8_of(U.activations(rows, inner, 1))
    want = x @ w.T
    far = q.Fp8(buf, W.scales, inner)
    for dtype in (torch.float32, torch.bfloat16):
        tol = U.product_tol(x, w, dtype == torch.float32) * 1.01 + U.rounded_tol(want, dtype)
        U.close(q.qgtc_fp8_product(X, far, dtype), want, tol)
        U.close(q.qgtc_fp8_product(far, X, dtype), want.T, tol.T)
    wide = buf.view(torch.bfloat16)                                            # [n, 2^23]
    wide[:, :inner] = torch.from_numpy(w).bfloat16().cuda()
    m = q.qgtc_fp8_quantize(wide[:, :inner])
    codes, scales = U.quantized(torch.from_numpy(w).bfloat16().float().numpy())
    assert (U.raw(m.codes) == codes).all() and (U.raw(m.scales)[:, :3] == scales).all()


def test_norm_offsets_past_32_bits():
    rows, cols, ld = 300, 200, 1 << 23
    buf = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")          # 5 GB: everything in columns of it
    x, res, total, dy, dx = (buf[:, 1000 * k:1000 * k + cols] for k in range(5))
    a, b, c = (U.activations(rows, cols, k).bfloat16().cuda() for k in (1, 2, 3))
    x.copy_(a), res.copy_(b), dy.copy_(c)
    w = torch.ones(cols, device="cuda")
    n, want = q.qgtc_rms_norm(x, w, residual=res, sum_out=total, rstd=True), q.qgtc_rms_norm(a, w, residual=b, rstd=True)
    assert torch.equal(total, want.sum) and (U.raw(n.fp8.codes) == U.raw(want.fp8.codes)).all()
    got, dw = q.qgtc_rms_norm_backward(dy, total, w, n.rstd, out=dx)
    dx2, dw2 = q.qgtc_rms_norm_backward(c, want.sum, w, want.rstd)
    assert torch.equal(got, dx2) and torch.equal(dw, dw2)


def test_more_rows_than_a_launch_takes():
    rows = (1 << 25) + 70                                  # 64 lanes a row: 2^31 and some
    x = torch.ones((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[-1], x[1 << 25], x[(1 << 25) - 1] = 3.0, 5.0, 7.0
    n = q.qgtc_rms_norm(x, torch.full((1,), 2.0, device="cuda"), eps=0.0, fp8=False, y=True, rstd=True)
    assert bool((n.y == 2.0).all()) and n.rstd[-1].item() == pytest.approx(1 / 3) and n.rstd[1 << 25].item() == pytest.approx(0.2)
    m = q.qgtc_fp8_quantize(x)                             # four rows a wave: one launch, of 4 GB of codes
    tail = m.codes[-80:, :1].float() * m.scales[-80:, :1].float()
    assert torch.equal(tail, x[-80:].float()) and bool((m.codes[:, 1:].view(torch.uint8) == 0).all())


# ---- the gated block ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("cols,inner", [(1, 1), (16, 128), (100, 130), (128, 512), (300, 260), (257, 1030)])
def test_gated_and_its_gradients(act, rows, cols, inner):
    X, x = fp8_of(U.activations(rows, inner, 1) * 2)
    G, wg = fp8_of(U.weights(cols, inner, 2))
    P, wu = fp8_of(U.weights(cols, inner, 3))
    h, th, fg, tfg, a, ta = U.gated(x, wg, wu, act)
    th = th * 1.01 + 2.0 ** -149
    U.check_codes(q.qgtc_fp8_gated(X, G, P, act), h, th)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        if dtype == torch.float32:
            h, th, fg, tfg, a, ta = U.gated(x, wg, wu, act, True)
            th = th * 1.01 + 2.0 ** -149
        buf = torch.full((rows, cols + 3), 5.0, dtype=dtype, device="cuda")
        both = q.qgtc_fp8_gated(X, G, P, act, h=buf[:, 1:cols + 1])
        U.check_codes(both, h, th)
        U.close(buf[:, 1:cols + 1], h, th + U.rounded_tol(h, dtype))
        assert (buf[:, 0] == 5.0).all() and (buf[:, cols + 1:] == 5.0).all()
        alone = torch.empty((rows, cols), dtype=dtype, device="cuda")
        assert q.qgtc_fp8_gated(X, G, P, act, fp8=False, h=alone) is None
        U.close(alone, h, th + U.rounded_tol(h, dtype))
        dh = torch.randn((rows, cols), generator=torch.Generator().manual_seed(4)).to(dtype)
        d = f64 = U.f64(dh)
        got = q.qgtc_fp8_gated_backward(X, G, P, odd(dh, dtype), act)
        assert got.dtype == dtype
        for at, f, tf in ((0, fg, tfg), (cols, a, ta)):
            want = f64 * f
            U.close(got[:, at:at + cols], want, np.abs(d) * tf * 1.01 + 2.0 ** -23 * np.abs(want) + U.rounded_tol(want, dtype), (at, dtype))


# ---- the same at sizes that larger tiles are taken for: 128 x 128 and 256 x 256 by their number (a round of tiles per 256 compute
# units), ragged at every edge, of one, two, odd and many blocks.  In 64 bits on the device.
LARGE = [(300, 4100, 2050), (1000, 2056, 4100), (700, 8190, 100), (513, 4099, 260),              # 128 x 128
         (8190, 4090, 1100), (8100, 8200, 520), (4090, 8190, 2048), (8192, 8192, 640), (3333, 8190, 3000)]   # 256 x 256
GATED = [(300, 2050, 2050), (1000, 1030, 1030), (130, 4090, 260),
         (4090, 4090, 1100), (4090, 8190, 100), (4090, 8190, 200), (2048, 8192, 1152), (2500, 5000, 2100)]


def on_device(rows, cols, inner, seeds):
    made = []
    for (n, seed) in ((rows, seeds[0]),) + tuple((cols, s) for s in seeds[1:]):
        t = U.activations(n, inner, seed) if seed == seeds[0] else U.weights(n, inner, seed)
        m = q.qgtc_fp8_quantize(t.cuda())
        wide = m.codes.double() * m.scales[:, :m.blocks].double().repeat_interleave(128, 1)
        made.append((m, wide[:, :inner].contiguous()))
    return made


def device_tol(x, w, exact_products):
    """U.product_tol of device matrices."""
    blocks = -(-x.shape[1] // 128)
    tol = (blocks + 128) * 2.0 ** -23 * (x.abs() @ w.abs().t().contiguous())
    if not exact_products:
        def tops(v):
            return torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 8)).view(v.shape[0], -1, 8).amax(2)
        tol = tol + 7 * 2.0 ** -13 * (tops(x) @ tops(w).t().contiguous())
    return tol * 1.01


def device_close(got, want, tol):
    bad = (got.double() - want).abs() > tol + want.abs() * U.HALF[got.dtype] + U.TINY[got.dtype]
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("rows,cols,inner", LARGE)
def test_large_product(rows, cols, inner):
    (X, x), (W, w) = on_device(rows, cols, inner, (1, 2))
    want = x @ w.t().contiguous()
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        buf = torch.full((rows + 1, cols + 5), 9.0, dtype=dtype, device="cuda")
        out = buf[:rows, 3:cols + 3]
        q.qgtc_fp8_product(X, W, out=out)
        device_close(out, want, device_tol(x, w, dtype == torch.float32))
        buf[:rows, 3:cols + 3] = 9.0
        assert bool((buf == 9.0).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,cols,inner", GATED)
def test_large_gated_and_its_gradients(rows, cols, inner, act):
    (X, x), (G, wg), (P, wu) = on_device(rows, cols, inner, (1, 2, 3))
    g, u = x @ wg.t().contiguous(), x @ wu.t().contiguous()
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        tg, tu = device_tol(x, wg, dtype == torch.float32), device_tol(x, wu, dtype == torch.float32)
        if act == "silu":
            s, curve = torch.sigmoid(g), 0.5
            a, slope = g * s, s * (1 + g * (1 - s))
        else:
            k = (2 / np.pi) ** 0.5
            s, curve = torch.sigmoid(2 * k * (g + 0.044715 * g ** 3)), 1.2
            a, slope = g * s, s + g * s * (1 - s) * 2 * k * (1 + 3 * 0.044715 * g * g)
        own = 16 * 2.0 ** -24
        # (the short form of the sigmoid, for results of 16 and 8 bits, is off by |z| 2^-24 of it, z the sigmoid's argument; s |z| is
        # below |g| + 1 for both, and so is its effect on the slope)
        ta = 1.13 * tg + own * (a.abs() + 1)
        ts = curve * tg + own * (1 + slope.abs()) + own * g.abs()
        h, th = a * u, 1.01 * (ta * u.abs() + a.abs() * tu + ta * tu + 2.0 ** -23 * (a * u).abs())
        room = torch.full((rows, cols + 3), 9.0, dtype=dtype, device="cuda")
        m = q.qgtc_fp8_gated(X, G, P, act, h=room[:, 1:cols + 1])
        device_close(room[:, 1:cols + 1], h, th)
        assert bool((room[:, 0] == 9.0).all()) and bool((room[:, cols + 1:] == 9.0).all())
        both = [m]
        if dtype == torch.bfloat16:
            both.append(q.qgtc_fp8_gated(X, G, P, act))
        for m in both:
            e = m.scales[:, :m.blocks].double()
            got = m.codes.double() * e.repeat_interleave(128, 1)
            assert bool((m.codes[:, cols:].view(torch.uint8) == 0).all())
            half = torch.maximum(h.abs() * 2.0 ** -4, 2.0 ** -10 * e.repeat_interleave(128, 1)[:, :cols])
            bad = (got[:, :cols] - h).abs() > half + th * 1.0625
            assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())
            top = torch.nn.functional.pad(h.abs(), (0, -cols % 128)).view(rows, -1, 128).amax(2)
            slack = torch.nn.functional.pad(th, (0, -cols % 128)).view(rows, -1, 128).amax(2)
            assert bool((448 * e >= top - slack).all()) and bool((224 * e < top + slack).all())
        dh = torch.randn((rows, cols), device="cuda").to(dtype)
        d = q.qgtc_fp8_gated_backward(X, G, P, dh, act)
        f = dh.double()
        device_close(d[:, :cols], f * slope * u, f.abs() * (ts * u.abs() + slope.abs() * tu + ts * tu) * 1.01 + 2.0 ** -22 * (f * slope * u).abs())
        device_close(d[:, cols:], f * a, f.abs() * ta * 1.01 + 2.0 ** -22 * (f * a).abs())


def test_large_rows_keep_to_themselves():
    """A row of X with an infinity, in the first and in the last tile: no other row changes, by tiles of either size."""
    for rows, cols, inner in ((300, 4100, 2050), (4090, 4090, 1100)):
        xs = U.activations(rows, inner, 1)
        (G, _), (P, _) = on_device(cols, cols, inner, (2, 3))
        want, wp = q.qgtc_fp8_gated(q.qgtc_fp8_quantize(xs.cuda()), G, P), q.qgtc_fp8_product(q.qgtc_fp8_quantize(xs.cuda()), G)
        bad = [0, 17, rows - 1]
        for r in bad:
            xs[r, inner - 1] = float("inf")
        X = q.qgtc_fp8_quantize(xs.cuda())
        got, gp = q.qgtc_fp8_gated(X, G, P), q.qgtc_fp8_product(X, G)
        ok = torch.ones(rows, dtype=torch.bool)
        ok[bad] = False
        assert (U.raw(got.codes)[ok] == U.raw(want.codes)[ok]).all() and (U.raw(got.scales)[ok][:, :got.blocks] == U.raw(want.scales)[ok][:, :got.blocks]).all()
        assert torch.equal(gp[ok], wp[ok]) and bool(torch.isnan(gp[bad]).all())
        assert (U.raw(got.scales)[bad][:, :got.blocks] == 255).all() and (U.raw(got.codes)[bad][:, cols:] == 0).all()
        assert (U.raw(got.codes)[bad][:, :cols] == 0x7f).all()


@pytest.mark.parametrize("rows,cols,inner", [(8, 8192, 512), (512, 8192, 520), (4096, 8192, 512)])
def test_gated_scales_are_those_of_fp32_sums(rows, cols, inner):
    """Every block's scale, but where the largest entry lies within 2^-18 of a border between two (sums of 512 products in fp32 are off
    by 512 * 2^-24 of the sum of their sizes at the very worst, by some 2^-22 of the largest entries in fact; the 8-bit instruction by
    2^-16 and more, which would miss several of 262144 blocks)."""
    ops = [q.qgtc_fp8_quantize(t.cuda()) for t in (U.activations(rows, inner, 1), U.weights(cols, inner, 2), U.weights(cols, inner, 3))]

    def whole(m):
        return m.codes.double()[:, :inner] * m.scales.double().repeat_interleave(128, 1)[:, :inner]
    x, wg, wu = (whole(m) for m in ops)
    g, u = x @ wg.t(), x @ wu.t()
    top = (g * torch.sigmoid(g) * u).abs().view(rows, -1, 128).amax(2)
    m, p = torch.frexp(top)
    e = p + 118 + (m > 0.875).int()
    got = q.qgtc_fp8_gated(*ops).scales.view(torch.uint8)[:, :cols // 128].int()
    unsure = ((m - 0.875).abs() < 0.875 * 2.0 ** -18)
    assert ((got == e) | unsure).all(), int(((got != e) & ~unsure).sum())
    print(int((got != e).sum()), "of", got.numel(), "beside the border")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gate_far_out(act):
    """Gates of a size where the exponential leaves fp32's range: the activation is the identity or nothing."""
    vals = torch.tensor([0.0, 1e-3, -1e-3, 1.0, -1.0, 30.0, -30.0, 86.0, -86.0, 88.0, -88.0, 200.0, -200.0, 448.0, -448.0, 1e4, -1e4])
    g = torch.zeros((17, 128))
    g[:, 0] = vals
    one = torch.zeros((16, 128))
    one[:, 0] = 1.0
    (X, x), (G, wg) = fp8_of(g), fp8_of(one)
    up = torch.zeros((16, 128))
    up[:, 0] = 1.0
    P, wu = fp8_of(up)
    h = torch.empty((17, 16), device="cuda")
    q.qgtc_fp8_gated(X, G, P, act, fp8=False, h=h)
    gg = (x @ wg.T)
    a, s, _ = U.act(act, gg)
    # (the kernel's sigmoid does not fall below that of -87, e^-87 < 1.7e-38: that times what it is multiplied with)
    least, dz = 1.7e-38 * np.abs(gg), 1.6 * (1 + 0.135 * gg * gg)
    U.close(h, a * gg, np.abs(a * gg) * 2.0 ** -20 + least * np.abs(gg))
    d = q.qgtc_fp8_gated_backward(X, G, P, torch.ones((17, 16), device="cuda"), act)
    U.close(d[:, :16], s * gg, 2.0 ** -20 * (1 + np.abs(s)) * np.abs(gg) + least * (1 + np.abs(gg) * dz))
    U.close(d[:, 16:], a, np.abs(a) * 2.0 ** -20 + least)


def test_gated_gradients_are_differences():
    """dg and du against differences of act(g) u in 64 bits."""
    X, x = fp8_of(U.activations(5, 256, 1))
    G, wg = fp8_of(U.weights(20, 256, 2))
    P, wu = fp8_of(U.weights(20, 256, 3))
    g, u, step = x @ wg.T, x @ wu.T, 1e-5
    for act in ("silu", "gelu"):
        d = U.f64(q.qgtc_fp8_gated_backward(X, G, P, torch.ones((5, 20), device="cuda"), act))
        want = (U.act(act, g + step)[0] - U.act(act, g - step)[0]) / (2 * step) * u
        tol = 1e-9 * (1 + np.abs(u)) + 1e-10 + U.gated(x, wg, wu, act, True)[3]
        assert (np.abs(d[:, :20] - want) <= tol).all()
