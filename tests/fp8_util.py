"""Plain forms in 64 bits of the operators on 8-bit floats, on the CPU, and the bounds their kernels are held to.

Half a step of a type, relative: fp32 2^-24, fp16 2^-11, bf16 2^-8, e4m3 2^-4 (below 2^-6 an e4m3's step is 2^-9: half of it 2^-10)."""
import numpy as np
import torch

BLOCK = 128
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the smallest step
TYPES = [torch.float32, torch.float16, torch.bfloat16]
E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def padded(n, to):
    return -(-n // to) * to


def f64(t):
    return t.detach().cpu().double().numpy()


def scale_exponents(amax):
    """The byte of each block's scale, for fp32 maxima (exact: comparisons with 448 times powers of two)."""
    amax = np.asarray(amax, dtype=np.float64)
    m, p = np.frexp(np.where(np.isfinite(amax), amax, 1.0))
    e = np.where(amax > 0, p + 118 + (m > 0.875), 0)
    return np.where(np.isfinite(amax), np.clip(e, 0, 254), 255).astype(np.uint8)


def quantized(x):
    """fp32 matrix (numpy) -> codes [rows, whole blocks] uint8, scales [rows, blocks] uint8, by the definition."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    wide = np.zeros((rows, padded(cols, BLOCK)), dtype=np.float32)
    wide[:, :cols] = x
    b = wide.reshape(rows, -1, BLOCK)
    with np.errstate(invalid="ignore"):
        amax = np.abs(b).max(2) if b.size else np.zeros((rows, 0), np.float32)
    e = scale_exponents(amax)
    q = torch.from_numpy(np.ldexp(np.where(np.isfinite(b), b, 0.0).astype(np.float64), (127 - e.astype(np.int64))[:, :, None]))
    codes = q.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
    codes[e == 255] = 0x7f
    codes = codes.reshape(rows, -1)
    codes[:, cols:] = 0
    return codes, e


def values(codes, scales, cols):
    """What uint8 codes and scales stand for."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    blocks = codes.shape[1] // BLOCK
    two = np.where(scales[:, :blocks] == 255, np.nan, np.ldexp(1.0, scales[:, :blocks].astype(np.int64) - 127))
    with np.errstate(invalid="ignore"):
        v = E4M3[codes].reshape(codes.shape[0], blocks, BLOCK) * two[:, :, None]
    return v.reshape(codes.shape)[:, :cols]


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


def fp8_values(m):
    return values(raw(m.codes)[:, :m.blocks * BLOCK], raw(m.scales), m.cols)


def check_codes(m, y, tol, what=""):
    """m holds y (fp64) in 8-bit floats, where y itself may be off by tol before it is rounded."""
    codes, scales = raw(m.codes), raw(m.scales)[:, :m.blocks]
    assert (codes[:, m.cols:m.blocks * BLOCK] == 0).all(), what
    wide, off = (np.zeros((m.rows, m.blocks * BLOCK)) for _ in range(2))
    wide[:, :m.cols], off[:, :m.cols] = np.abs(y), tol
    b, o = wide.reshape(m.rows, -1, BLOCK), off.reshape(m.rows, -1, BLOCK)
    with np.errstate(invalid="ignore"):
        top, lo, hi = b.max(2), (b - o).max(2), (b + o).max(2)
    bad = ~np.isfinite(top)
    assert (scales[bad] == 255).all(), what
    e = scales.astype(np.int64)
    fits = np.ldexp(448.0, e - 127) >= lo
    least = (e == 0) | (np.ldexp(224.0, e - 127) < hi)
    assert (fits | bad).all() and (least | bad).all(), what
    got = fp8_values(m)
    half = np.maximum(np.abs(y) * 2.0 ** -4, np.repeat(np.ldexp(2.0 ** -10, e - 127), BLOCK, 1)[:, :m.cols])
    ok = np.abs(got - y) <= half + tol * (1 + 2.0 ** -4)
    ok |= np.repeat(bad, BLOCK, 1)[:, :m.cols] & np.isnan(got)
    assert ok.all(), (what, np.argwhere(~ok)[:4], got[~ok][:4], y[~ok][:4])


def close(got, want, tol, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    ok = (np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (what, int((~ok).sum()), np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4], np.broadcast_to(tol, want.shape)[~ok][:4])


def product_tol(x, w, exact_products=False):
    """Bound of a sum of the products of x and w (fp64 values).  In fp32 an instruction adds 128 exact products to a sum: each may
    be cut at 2^-23 of the largest (128 of them), and each of the blocks' sums once more.  The 8-bit instruction (results of 16
    and 8 bits) adds groups of 8 consecutive products, of which it cuts all but the largest at 2^-13 of that one, itself no larger
    than the product of the groups' largest entries: 7 * 2^-13 of that, summed over the groups."""
    blocks = -(-x.shape[1] // BLOCK)
    tol = (blocks + 128) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)
    if not exact_products:
        def tops(v):
            wide = np.zeros((v.shape[0], padded(v.shape[1], 8)))
            wide[:, :v.shape[1]] = np.abs(v)
            return wide.reshape(v.shape[0], -1, 8).max(2)
        tol = tol + 7 * 2.0 ** -13 * (tops(x) @ tops(w).T)
    return tol


def rounded_tol(want, dtype):
    return np.abs(want) * HALF[dtype] + TINY[dtype]


def sigmoid(z):
    """1 / (1 + exp(-z)), exact in relative terms for negative z as well ((1 + tanh(z/2)) / 2 is not: it subtracts)."""
    e = np.exp(-np.abs(z))
    return np.where(z < 0, e, 1.0) / (1 + e)


def act(name, g):
    """The activation, its slope, and a bound of the slope's own slope."""
    if name == "silu":
        s = sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), 0.5
    k = np.sqrt(2 / np.pi)
    z, dz = k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g)
    s = sigmoid(2 * z)
    return g * s, s + g * s * (1 - s) * 2 * dz, 1.2


def gated(x, wg, wu, name, exact_products=False):
    """h, its bound in fp32, and both gradients' factors (h = a u: dg = dh * s u, du = dh * a) with theirs."""
    g, u = x @ wg.T, x @ wu.T
    tg, tu = product_tol(x, wg, exact_products), product_tol(x, wu, exact_products)
    a, s, curve = act(name, g)
    # the gate itself: the exponential, the reciprocal and a few products, 16 roundings of fp32 at most, each of them
    # relative to a term that is no larger than 1 + |g| in the slope (g s' grows as |g| e^-|g|)
    own = 16 * 2.0 ** -24
    ta = 1.13 * tg + own * np.abs(a) + 2.0 ** -120
    ts = curve * tg + own * (1 + np.abs(s))
    h = a * u
    th = ta * np.abs(u) + np.abs(a) * tu + ta * tu + 2.0 ** -23 * np.abs(h)
    fg = s * u
    tfg = ts * np.abs(u) + np.abs(s) * tu + ts * tu + 2.0 ** -23 * np.abs(fg)
    return h, th, fg, tfg, a, ta


def activations(rows, cols, seed):
    """A residual stream: normal, some loud columns, rows of differing size."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp(0.5 * torch.randn((rows, 1), generator=g))
    return x * torch.where(torch.rand(cols, generator=g) < 0.02, 12.0, 1.0)


def weights(rows, cols, seed):
    return torch.randn((rows, cols), generator=torch.Generator().manual_seed(seed)) * max(cols, 1) ** -0.5
