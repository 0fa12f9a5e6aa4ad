"""Operators on 8-bit floats on an MI355X where their numbers are far from ordinary: sums that cancel, gates and scales at the ends of
their range, sizes that take several launches."""
import numpy as np
import pytest
import torch

import fp8_util as U

pytestmark = pytest.mark.gpu

q = pytest.importorskip("paper_2111_09547_amd")

# one size for each kernel of the products: few rows, tiles of 128 x 128, tiles of 256 x 256
SIZES = [(3, 128, 128), (300, 2050, 2050), (4090, 4090, 1100)]


def on_device(m):
    """What a matrix in 8-bit floats holds, fp32."""
    return (m.codes.float() * m.scales[:, :m.blocks].float().repeat_interleave(128, 1))[:, :m.cols]


@pytest.mark.parametrize("rows,cols,inner", SIZES)
@pytest.mark.parametrize("groups,small", [(1, -5), (2, -6), (4, -7), (1, -1), (1, 7), (4, 7)])
def test_gated_scale_where_sums_cancel(rows, cols, inner, groups, small):
    """Column 0's gate is 448^2 - 448^2 + 6 small in each of some groups of 8 products, and 56: the 8-bit instruction cuts the small ones
    off, and h = 56 * 8 lies on a border between two scales.  Computed again it is anything up to 98 * 8.  Whatever column 0 becomes
    between the two (silu is monotonous from -1 on and within 0.3 of 0 below), the other columns' sums are exact: 52 * 8."""
    x, g, u = torch.zeros((rows, inner)), torch.zeros((cols, inner)), torch.zeros((cols, inner))
    for k in range(0, 8 * groups, 8):
        x[:, k:k + 2], x[:, k + 2:k + 8] = 448.0, 1.0
        g[0, k], g[0, k + 1], g[0, k + 2:k + 8] = 448.0, -448.0, float(small)
    x[:, 120:122] = 1.0
    g[0, 120], g[1:, 120], g[1:, 100] = 56.0, 52.0, 448.0        # (scales are 1: no code is rounded)
    u[:, 121], u[:, 101] = 8.0, 448.0
    X, G, P = (q.qgtc_fp8_quantize(t.cuda()) for t in (x, g, u))
    got = on_device(q.qgtc_fp8_gated(X, G, P))
    exact = 56.0 + 6 * small * groups
    lo, hi = 8 * min(56.0, max(exact, -0.3)), 8 * max(56.0, exact)
    assert bool((got[:, 1:] == 416.0).all())                     # (13 * 32: an e4m3)
    assert bool((got[:, 0] >= lo * (1 + 2.0 ** -4 * np.sign(-lo))).all() and (got[:, 0] <= hi * (1 + 2.0 ** -4)).all()), got[:2, 0].tolist()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,cols,inner", [(40, 128, 256)] + SIZES[1:])
def test_gates_to_the_end_of_their_range(rows, cols, inner, act):
    """Every gate is one product, which is exact, and u is 1: h, dg and du are the activation, its slope and itself.

    Bounds: the sigmoid is 88 * 2^-24 < 2^-17 of itself off at most (the instruction's argument is rounded) and 0 below 2^-126; a few
    roundings come to less than as much again.  In the slope it is s and g z' s (1 - s) that are off by so much, and where 1 - s is a
    difference of fp32 (z > 0, to z = 17.4, g z' < 53) that by 2^-24: 53 * 2^-24 < 2^-18."""
    vals = [s * v for v in (0.25, 1.0, 3.0, 16.0, 80.0, 96.0, 1e3, 1e4, 1e8, 1e12, 5e12, 1e13, 2e13, 1e18, 3e19, 1e25, 1e37, 1.5e38) for s in (1, -1)]
    x = torch.zeros((rows, inner))
    x[:len(vals), 0], x[:, 128] = torch.tensor(vals), 1.0
    one = torch.zeros((2, cols, inner))
    one[0, :, 0], one[1, :, 128] = 1.0, 1.0
    X, G, P = (q.qgtc_fp8_quantize(t.cuda()) for t in (x, *one))
    g = on_device(X)[:, 0].double()
    if act == "silu":
        z, gdz = g, g.clone()
    else:
        k = 2 * (2 / np.pi) ** 0.5
        z, gdz = k * (g + 0.044715 * g ** 3), k * (g + 3 * 0.044715 * g ** 3)
    s = torch.sigmoid(z)
    bend = torch.where(z.abs() < 700, gdz * s * torch.sigmoid(-z), torch.zeros_like(z))
    value, slope = (g * s)[:, None], (s + bend)[:, None]
    off = (g.abs() * (s * 2.0 ** -16 + 2.0 ** -126))[:, None]
    off_slope = ((s + bend.abs()) * 2.0 ** -16 + (z > 0) * 2.0 ** -18 + 513 * 2.0 ** -126)[:, None]

    def check(got, want, tol):
        bad = ~((got.double() - want).abs() <= tol + want.abs() * U.HALF[got.dtype] + U.TINY[got.dtype])
        assert not bool(bad.any()), (got.dtype, [(g[i].item(), got[i, j].item(), want[i, 0].item()) for i, j in bad.nonzero()[:4].tolist()])
    for dtype in (torch.float32, torch.bfloat16):
        h = torch.empty((rows, cols), dtype=dtype, device="cuda")
        m = q.qgtc_fp8_gated(X, G, P, act, h=h)
        check(h, value, off)
        assert not bool((m.scales.view(torch.uint8)[:, :m.blocks] == 255).any())
        d = q.qgtc_fp8_gated_backward(X, G, P, torch.ones((rows, cols), dtype=dtype, device="cuda"), act)
        check(d[:, :cols], slope, off_slope)
        check(d[:, cols:], value, off)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,cols,inner", [(40, 128, 256)] + SIZES[1:])
def test_gates_of_nan(rows, cols, inner, act):
    """A NaN in a gate is one in the value and in the slope."""
    x = torch.zeros((rows, inner))
    x[3, 0], x[:, 128] = float("nan"), 1.0
    one = torch.zeros((2, cols, inner))
    one[0, :, 0], one[1, :, 128] = 1.0, 1.0
    X, G, P = (q.qgtc_fp8_quantize(t.cuda()) for t in (x, *one))
    for dtype in (torch.float32, torch.bfloat16):
        d = q.qgtc_fp8_gated_backward(X, G, P, torch.ones((rows, cols), dtype=dtype, device="cuda"), act)
        assert bool(d[3].isnan().all()) and not bool(d[:3].isnan().any()) and not bool(d[4:].isnan().any())


# sizes for each kernel of fp32 results (few rows, tiles of 128 x 128) and, the last, of 16 bits
SCALED = [(5, 40), (50, 40), (1000, 2056), (4090, 4090)]


def scaled(rows, cols, blocks, sx, sw, seed):
    """Operands with given scales (bytes [rows, blocks]) and codes of normal data, and their values in 64 bits."""
    made = []
    for n, s, k in ((rows, sx, 1), (cols, sw, 2)):
        c = torch.randn((n, blocks * 128), generator=torch.Generator().manual_seed(seed + k)) * 8
        c[:, 1::9] *= 20.0
        codes = c.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).cuda()        # (what is larger becomes NaN)
        wide = torch.zeros((n, -(-blocks // 4) * 4), dtype=torch.uint8)
        wide[:, :blocks] = s
        two = torch.ldexp(torch.ones((n, blocks), dtype=torch.float64), s.int() - 127).cuda()
        made.append((q.Fp8(codes, wide.cuda(), blocks * 128), codes.double() * two.repeat_interleave(128, 1)))
    return made


def product_close(got, x, w):
    want = x @ w.t().contiguous()
    blocks = x.shape[1] // 128
    tol = (blocks + 128) * 2.0 ** -23 * (x.abs() @ w.abs().t().contiguous())          # (U.product_tol)
    if got.dtype != torch.float32:
        tops = [v.abs().view(v.shape[0], -1, 8).amax(2) for v in (x, w)]
        tol = tol + 7 * 2.0 ** -13 * (tops[0] @ tops[1].t().contiguous())
    bad = ~((got.double() - want).abs() <= tol * 1.01 + want.abs() * U.HALF[got.dtype] + U.TINY[got.dtype])
    assert not bool(bad.any()), (got.dtype, int(bad.sum()), [(got[i, j].item(), want[i, j].item()) for i, j in bad.nonzero()[:3].tolist()])


@pytest.mark.parametrize("rows,cols", SCALED)
def test_product_of_scales_from_end_to_end(rows, cols):
    """Blocks of every scale there is, 0 to 254, against blocks of the opposite scale: every product is of one size, and no partial sum
    leaves fp32's range."""
    blocks = 17
    base = torch.tensor([0, 254, 1, 9, 10, 11, 235, 236, 237, 245, 246, 247, 253, 64, 127, 190, 128])
    near = [torch.randint(-3, 4, (n, blocks), generator=torch.Generator().manual_seed(n)) for n in (rows, cols + 7)]
    sx, sw = (base + near[0]).clamp(0, 254).byte(), (254 - base + near[1][:cols]).clamp(0, 254).byte()
    (X, x), (W, w) = scaled(rows, cols, blocks, sx, sw, 3)
    for dtype in (torch.float32, torch.bfloat16):
        product_close(q.qgtc_fp8_product(X, W, dtype), x, w)


@pytest.mark.parametrize("rows,cols", SCALED)
@pytest.mark.parametrize("up", [105, 90, -105, -125])
def test_product_results_from_end_to_end(rows, cols, up):
    """Results of about 2^(up + 16), those near fp32's ends among them.  Below 2^-126 a rounding is by half of 2^-149, of each of the two
    blocks' sums and of the result."""
    sx, sw = torch.full((rows, 2), 127 + up // 2, dtype=torch.uint8), torch.full((cols, 2), 127 + (up - up // 2), dtype=torch.uint8)
    (X, x), (W, w) = scaled(rows, cols, 2, sx, sw, 5)
    assert bool((x @ w.t().contiguous()).abs().max() < 2.0 ** 127)
    for dtype in (torch.float32, torch.bfloat16):
        product_close(q.qgtc_fp8_product(X, W, dtype), x, w)


@pytest.mark.parametrize("rows,cols", SCALED)
def test_product_of_the_largest_number(rows, cols):
    """fp32's largest number becomes 256 * 2^120; multiplied with 2^-100 that is 2^28, and 0 times it is 0."""
    x, w = torch.zeros((rows, 300)), torch.zeros((cols, 300))
    x[:, 3], x[:, 200], w[:, 3], w[0, 3], w[:, 200] = torch.finfo(torch.float32).max, 1.0, 2.0 ** -100, 0.0, 3.0
    X, W = q.qgtc_fp8_quantize(x.cuda()), q.qgtc_fp8_quantize(w.cuda())
    for dtype in (torch.float32, torch.bfloat16):
        y = q.qgtc_fp8_product(X, W, dtype)
        want = torch.tensor(2.0 ** 28 + 3).to(dtype).cuda()
        assert bool((y[:, 1:] == want).all()) and bool((y[:, 0] == 3.0).all())


@pytest.mark.parametrize("rows,cols", SCALED)
@pytest.mark.parametrize("code", [0x38, 0x00])
def test_product_of_blocks_without_a_scale(rows, cols, code):
    """A scale of 255 is NaN and so is its block, whatever the codes: 1 or 0."""
    ones = torch.ones((rows, 400)), torch.ones((cols, 400))
    for side in (0, 1):
        ops = [q.qgtc_fp8_quantize(t.cuda()) for t in ones]
        ops[side].codes.view(torch.uint8)[2, 128:256], ops[side].scales.view(torch.uint8)[2, 1] = code, 255
        for dtype in (torch.float32, torch.bfloat16):
            y = q.qgtc_fp8_product(*ops, dtype)
            y = y if side == 0 else y.t()
            assert bool(y[2].isnan().all()) and bool((y[:2] == 400).all()) and bool((y[3:] == 400).all())


@pytest.mark.parametrize("width,words", [(256, 4), (300, 4), (1000, 7), (513, 6)])
def test_one_row_of_any_width(width, words):
    """A matrix of one row in tensors that are wider than its blocks, by any number of bytes."""
    x = U.activations(1, 200, 1)
    codes, scales = U.quantized(x.numpy())
    c, s = torch.full((1, width), 99, dtype=torch.uint8, device="cuda"), torch.full((1, words), 98, dtype=torch.uint8, device="cuda")
    m = q.qgtc_fp8_quantize(x.cuda(), out=q.Fp8(c, s, 200))
    assert (U.raw(c)[:, :256] == codes).all() and (U.raw(s)[:, :2] == scales).all()
    assert (U.raw(c)[:, 256:] == 99).all() and (U.raw(s)[:, 2:] == 98).all()
    W = q.qgtc_fp8_quantize(U.weights(40, 200, 2).cuda())
    assert torch.equal(q.qgtc_fp8_product(m, W), q.qgtc_fp8_product(q.qgtc_fp8_quantize(x.cuda()), W))


def test_norm_without_columns():
    """There is nothing in any output, and no mean for rstd to be made from."""
    x, w = torch.empty((5, 0), device="cuda"), torch.empty(0, device="cuda")
    n = q.qgtc_rms_norm(x, w, residual=x, y=True)
    assert n.sum.shape == n.y.shape == (5, 0) and (n.fp8.rows, n.fp8.cols) == (5, 0)
    with pytest.raises(ValueError, match="columns"):
        q.qgtc_rms_norm(x, w, rstd=True)


def test_sizes_beyond_32_bits():
    """2^32 and some rows or columns are refused, and not taken for the few that 32 bits make of them."""
    n = (1 << 32) + 5
    tall = torch.empty((n, 1), dtype=torch.bfloat16, device="cuda")                # 8 GB
    one = torch.ones(1, device="cuda")
    for call in (lambda: q.qgtc_rms_norm(tall, one, fp8=False, y=True), lambda: q.qgtc_fp8_quantize(tall, columns=True),
                 lambda: q.qgtc_fp8_quantize(tall.t()), lambda: q.alloc_fp8(1, n, "cuda"),
                 lambda: q.Fp8(tall.view(torch.uint8).view(1, 2 * n), torch.empty((1, 4), dtype=torch.uint8, device="cuda"), n)):
        with pytest.raises(ValueError, match="2\\^29"):
            call()


# ---- more than one launch takes: what is written at the border between two launches and at the end ------------------------------------
def test_quantize_rows_in_two_launches():
    """2^25 waves of four rows a launch."""
    first, rows = 1 << 27, (1 << 27) + 70
    x = torch.ones((rows, 1), dtype=torch.bfloat16, device="cuda")
    for i, r in enumerate((0, first - 1, first, first + 1, rows - 1)):
        x[r] = 3.0 * 2.0 ** i
    m = q.qgtc_fp8_quantize(x)                               # 17 GB of codes
    for part in (slice(0, 40), slice(first - 40, first + 40), slice(rows - 40, rows)):
        assert torch.equal(m.codes[part, :1].float() * m.scales[part, :1].float(), x[part].float())
        assert bool((m.codes[part, 1:].view(torch.uint8) == 0).all())


def test_quantize_columns_in_two_launches():
    """65535 blocks of rows a launch."""
    first, rows = 65535 * 128, 65535 * 128 + 333
    x = torch.randn((rows, 3), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    m, a, b = (q.qgtc_fp8_quantize(t, columns=True) for t in (x, x[:first], x[first:]))
    for name, cut in (("codes", first), ("scales", first // 128)):
        whole, head, tail = (getattr(t, name).view(torch.uint8) for t in (m, a, b))
        n = b.blocks * 128 if name == "codes" else b.blocks
        assert torch.equal(whole[:, :cut], head[:, :cut]) and torch.equal(whole[:, cut:cut + n], tail[:, :n])


def counted(rows, at):
    """rows x 128 in 8-bit floats with scale 1: 64 at column 0, and 1 + row % 13 at column `at`."""
    codes = torch.zeros((rows, 128), dtype=torch.uint8, device="cuda")
    n = (1 + torch.arange(rows, device="cuda") % 13).float()
    codes[:, 0] = 0x68                                       # 2^6
    codes[:, at] = n.to(torch.float8_e4m3fn).view(torch.uint8)
    return q.Fp8(codes, torch.full((rows, 4), 127, dtype=torch.uint8, device="cuda"), 128), n


def test_product_of_few_in_two_launches_of_rows():
    """65535 times 64 rows of X a launch, results in fp32."""
    (X, n), (W, k) = counted(65535 * 64 + 70, 1), counted(5, 1)
    assert torch.equal(q.qgtc_fp8_product(X, W, torch.float32), 4096 + n[:, None] * k[None, :])


def test_product_of_few_in_two_launches_of_columns():
    """2^26 rows of W a launch, results in fp32."""
    (X, n), (W, k) = counted(3, 1), counted((1 << 26) + 40, 1)
    y = q.qgtc_fp8_product(X, W, torch.float32)
    for i in range(3):
        assert torch.equal(y[i], 4096 + n[i] * k)


def test_gated_rows_in_two_launches():
    """2^25 waves, each with up to 512 columns of a row, a launch of what makes 8-bit floats of the gated results."""
    rows = (1 << 25) + 70
    X, n = counted(rows, 1)
    one = torch.zeros((2, 1, 128), device="cuda")
    one[0, 0, 0], one[1, 0, 1] = 1.0, 1.0
    m = q.qgtc_fp8_gated(X, *(q.qgtc_fp8_quantize(t) for t in one))          # silu(64) = 64, times n
    assert torch.equal(m.codes[:, 0].float() * m.scales[:, 0].float(), 64 * n)
    for part in (slice(0, 40), slice((1 << 25) - 40, (1 << 25) + 40), slice(rows - 40, rows)):
        assert bool((m.codes[part, 1:].view(torch.uint8) == 0).all())


# ---- operands and results in wider memory: the same bits -----------------------------------------------------------------------------
def apart(m, codes_by, scales_by):
    """m in memory whose rows lie further apart, with other bytes between them."""
    c = torch.full((m.rows, m.blocks * 128 + 128 * codes_by), 0x7f, dtype=torch.uint8, device="cuda")
    s = torch.full((m.rows, m.scales.shape[1] + 4 * scales_by), 255, dtype=torch.uint8, device="cuda")
    c[:, :m.blocks * 128] = m.codes.view(torch.uint8)[:, :m.blocks * 128]
    s[:, :m.blocks] = m.scales.view(torch.uint8)[:, :m.blocks]
    return q.Fp8(c, s, m.cols)


def within(t, left, right):
    buf = torch.full((t.shape[0], t.shape[1] + left + right), 7.0, dtype=t.dtype, device="cuda")
    v = buf[:, left:left + t.shape[1]]
    v.copy_(t)
    return v


@pytest.mark.parametrize("rows,cols,inner", SIZES + [(40, 300, 1100), (700, 1030, 260), (4090, 4090, 200)])
def test_gated_of_matrices_within_others(rows, cols, inner):
    """X, G, U, h, the gradient and the results each with a pitch of its own."""
    X, G, P = (q.qgtc_fp8_quantize(t.cuda()) for t in (U.activations(rows, inner, 1), U.weights(cols, inner, 2), U.weights(cols, inner, 3)))
    x, g, p = apart(X, 1, 3), apart(G, 2, 1), apart(P, 5, 2)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        h, h2 = (torch.zeros((rows, cols), dtype=dtype, device="cuda") for _ in range(2))
        h2 = within(h2, 3, 2)
        want = q.qgtc_fp8_gated(X, G, P, h=h)
        out = apart(want, 3, 2)
        before = out.codes.clone(), out.scales.clone()
        out.codes[:, :want.blocks * 128], out.scales[:, :want.blocks] = 99, 99
        q.qgtc_fp8_gated(x, g, p, out=out, h=h2)
        assert torch.equal(h2, h) and torch.equal(out.codes, before[0]) and torch.equal(out.scales, before[1])
        dh = torch.randn((rows, cols), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(dtype)
        d = q.qgtc_fp8_gated_backward(X, G, P, dh, "gelu")
        d2 = within(torch.zeros_like(d), 1, 4)
        q.qgtc_fp8_gated_backward(x, g, p, within(dh, 5, 3), "gelu", out=d2)
        assert torch.equal(d2, d)
        y = q.qgtc_fp8_product(X, G, dtype)
        assert torch.equal(q.qgtc_fp8_product(x, g, out=within(torch.zeros_like(y), 3, 4)), y)


@pytest.mark.parametrize("rows,cols", SCALED[:3])
def test_rows_in_fp32_keep_to_themselves(rows, cols):
    """A row that has a NaN, or numbers whose sums leave fp32's range on the way: no bit of the other rows' results changes."""
    x, w = U.activations(rows, 900, 1), U.weights(cols, 900, 2)
    W = q.qgtc_fp8_quantize(w.cuda())
    want = q.qgtc_fp8_product(q.qgtc_fp8_quantize(x.cuda()), W, torch.float32)
    for r, v in ((0, float("nan")), (rows - 1, 3e38), (rows // 2, float("inf"))):
        bad = x.clone()
        bad[r, 77] = v
        got = q.qgtc_fp8_product(q.qgtc_fp8_quantize(bad.cuda()), W, torch.float32)
        keep = torch.arange(rows) != r
        assert torch.equal(got[keep], want[keep]) and not torch.equal(got[r], want[r])
