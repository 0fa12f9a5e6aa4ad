"""The operators on 8-bit floats whose speed this framework is judged by, each as a user's program calls it.

A matrix in 8-bit floats has e4m3 codes, row by row, and for every 128 consecutive entries of a row one scale,
a power of two (e8m0): the smallest with which the largest entry stays within 448.  Rows of codes are padded with
zeros to whole blocks; scales lie row by row, padded to four.  Kinds of work:

  norm            s = x + residual, root-mean-square norm of s times a weight, into 8-bit floats for the product behind it
  norm_backward   gradients of s and of the weight
  quantize        a matrix into 8-bit floats along its rows, or along its columns (transposed, as the products of a
                  backward pass contract over them)
  product         X.W' of two matrices in 8-bit floats
  gated           act(X.G') * (X.U') into 8-bit floats: the first half of a gated feed-forward block
  gated_backward  gradients of both projections' outputs, side by side, from X, G, U and the gradient of their gated product
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # one token of a serving loop: latency
        {"name": "norm 1x4096", "do": "norm", "rows": 1, "cols": 4096, "type": "bf16", "residual": True},
        # a training or prefill batch
        {"name": "norm 8192x4096", "do": "norm", "rows": 8192, "cols": 4096, "type": "bf16", "residual": True},
        # single precision, rows of no whole block, the first norm of a network (nothing to add)
        {"name": "norm 2049x1000 f32", "do": "norm", "rows": 2049, "cols": 1000, "type": "f32", "residual": False},
        # the norm's gradients on a ragged batch
        {"name": "norm_backward 4095x5120", "do": "norm_backward", "rows": 4095, "cols": 5120, "type": "f16", "residual": True},
        # gradients into 8 bits for the product that contracts over the tokens
        {"name": "quantize columns 8192x4096", "do": "quantize", "rows": 8192, "cols": 4096, "type": "bf16", "columns": True},
        # a few rows of odd length
        {"name": "quantize rows 333x1000", "do": "quantize", "rows": 333, "cols": 1000, "type": "f32", "columns": False},
        # one token through a square projection: the weights' bytes
        {"name": "product 1x4096x4096", "do": "product", "rows": 1, "inner": 4096, "cols": 4096, "type": "bf16"},
        # a small ragged batch
        {"name": "product 300x2000x1001", "do": "product", "rows": 300, "inner": 2000, "cols": 1001, "type": "f32"},
        # a large batch through a wide projection: the matrix cores
        {"name": "product 8192x8192x8192", "do": "product", "rows": 8192, "inner": 8192, "cols": 8192, "type": "bf16"},
        # a few sequences decoding together
        {"name": "gated 8x4096x8192", "do": "gated", "rows": 8, "inner": 4096, "cols": 8192, "act": "silu"},
        # a prefill batch
        {"name": "gated 4096x4096x8192", "do": "gated", "rows": 4096, "inner": 4096, "cols": 8192, "act": "silu"},
        # a training step's backward pass
        {"name": "gated_backward 2048x4096x8192", "do": "gated_backward", "rows": 2048, "inner": 4096, "cols": 8192,
         "type": "bf16", "act": "gelu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["norm", "norm_backward", "quantize", "product", "product", "gated", "gated", "gated_backward"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if do in ("norm", "norm_backward", "quantize"):
        rows, cols = _log(rng, 1, 8192), _log(rng, 64, 8192)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        rows = min(rows, 8192 * 4096 // cols)
        case = {"do": do, "rows": rows, "cols": cols, "type": kind}
        if do == "quantize":
            return dict(case, columns=rng.random() < 0.5)
        return dict(case, residual=rng.random() < 0.7)
    rows, inner, cols = _log(rng, 1, 8192), _log(rng, 256, 8192), _log(rng, 256, 8192)
    if rng.random() < 0.6:
        inner, cols = inner // 128 * 128, cols // 128 * 128
    case = {"do": do, "rows": rows, "inner": inner, "cols": cols}
    if do != "product":
        case["rows"] = min(rows, 4096)
        case["act"] = rng.choice(["silu", "gelu"])
    if do != "gated":
        case["type"] = kind
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------
def _padded(n, to):
    return -(-n // to) * to


def _codes(x):
    """fp32 [rows, cols] -> e4m3 codes [rows, cols padded to whole blocks], e8m0 scales [rows, blocks padded to four]."""
    rows, cols = x.shape
    wide = torch.zeros((rows, _padded(cols, BLOCK)), dtype=torch.float32, device=x.device)
    wide[:, :cols] = x
    blocks = wide.view(rows, -1, BLOCK)
    amax = blocks.abs().amax(2)
    m, p = torch.frexp(amax)
    e = torch.where(amax > 0, p + 118 + (m > 0.875).int(), torch.zeros_like(p)).clamp(0, 254)
    e = torch.where(torch.isfinite(amax), e, torch.full_like(e, 255))
    codes = torch.ldexp(blocks, (127 - e).unsqueeze(2)).to(torch.float8_e4m3fn).view(rows, -1)
    scales = torch.zeros((rows, _padded(blocks.shape[1], 4)), dtype=torch.uint8, device=x.device)
    scales[:, :blocks.shape[1]] = e.to(torch.uint8)
    return codes, scales.view(torch.float8_e8m0fnu)


def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed(1000003 * salt + seed)


def _activations(rows, cols, gen):
    """What a residual stream looks like: normal, some columns much larger than the others, rows of differing size."""
    x = torch.randn((rows, cols), device="cuda", generator=gen)
    loud = torch.rand(cols, device="cuda", generator=gen) < 0.01
    return x * torch.where(loud, 12.0, 1.0) * torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=gen))


def _weights(rows, cols, gen):
    return torch.randn((rows, cols), device="cuda", generator=gen) * cols ** -0.5


def prepare(case, seed):
    do, rows, cols = case["do"], case["rows"], case["cols"]
    g = _generator(seed, 1 + rows % 97)
    state = {"case": case}
    if do in ("norm", "norm_backward", "quantize"):
        t = TYPES[case["type"]]
        state["x"] = _activations(rows, cols, g).to(t)
        if do != "quantize":
            state["weight"] = (1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(t)
            if case["residual"]:
                state["residual"] = _activations(rows, cols, g).to(t)
        if do == "norm_backward":
            # (the forward pass has left its sum, here x, and the inverse root of its mean square)
            state["rstd"] = torch.rsqrt(state["x"].float().square().mean(1) + EPS)
            state["dy"] = (torch.randn((rows, cols), device="cuda", generator=g) * 1e-2).to(t)
        return state
    inner = case["inner"]
    state["x"] = _codes(_activations(rows, inner, g))
    state["w"] = _codes(_weights(cols, inner, g))
    if do != "product":
        state["u"] = _codes(_weights(cols, inner, g))
    if do == "gated_backward":
        state["dh"] = (torch.randn((rows, cols), device="cuda", generator=g) * 1e-2).to(TYPES[case["type"]])
    return state


# ---- plain forms ------------------------------------------------------------------------------------------------
def _values(form, cols, to=torch.float32):
    """The numbers that codes and scales stand for."""
    codes, scales = form
    c = codes.to(to).view(codes.shape[0], -1, BLOCK)
    return (c * scales.to(to)[:, :c.shape[1]].unsqueeze(2)).view(codes.shape)[:, :cols]


def _act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _eight_bits(x):
    codes, scales = _codes(x)
    return {"codes": codes[:, :x.shape[1]], "scales": scales[:, :codes.shape[1] // BLOCK]}


def _plain(state):
    case = state["case"]
    do, rows, cols = case["do"], case["rows"], case["cols"]
    if do == "quantize":
        x = state["x"].float()
        return _eight_bits(x.t() if case["columns"] else x)
    if do == "norm":
        t, s = state["x"].dtype, state["x"]
        if case["residual"]:
            s = (s.float() + state["residual"].float()).to(t)
        f = s.float()
        r = torch.rsqrt(f.square().mean(1, keepdim=True) + EPS)
        out = _eight_bits(f * r * state["weight"].float())
        return dict(out, sum=s) if case["residual"] else out
    if do == "norm_backward":
        f, r, dy = state["x"].float(), state["rstd"].unsqueeze(1), state["dy"].float()
        hat, gw = f * r, dy * state["weight"].float()
        dx = r * (gw - hat * (gw * hat).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + state["residual"].float()
        return {"dx": dx.to(state["x"].dtype), "dweight": (dy * hat).sum(0)}
    inner = case["inner"]
    x = _values(state["x"], inner)
    w = _values(state["w"], inner)
    if do == "product":
        return (x @ w.t()).to(TYPES[case["type"]])
    a, da = _act(case["act"], x @ w.t())
    u = x @ _values(state["u"], inner).t()
    if do == "gated":
        return _eight_bits(a * u)
    dh = state["dh"].float()
    return torch.cat([dh * u * da, dh * a], 1).to(state["dh"].dtype)


# ---- the framework's --------------------------------------------------------------------------------------------
def _shown(m):
    return {"codes": m.codes[:, :m.cols], "scales": m.scales[:, :m.blocks]}


def _own(state):
    import paper_2111_09547_amd as q
    case = state["case"]
    do = case["do"]
    if do == "quantize":
        return _shown(q.qgtc_fp8_quantize(state["x"], columns=case["columns"]))
    if do == "norm":
        n = q.qgtc_rms_norm(state["x"], state["weight"], EPS, residual=state.get("residual"))
        return dict(_shown(n.fp8), sum=n.sum) if case["residual"] else _shown(n.fp8)
    if do == "norm_backward":
        dx, dw = q.qgtc_rms_norm_backward(state["dy"], state["x"], state["weight"], state["rstd"], dsum=state.get("residual"))
        return {"dx": dx, "dweight": dw}
    x = q.Fp8(*state["x"], cols=case["inner"])
    w = q.Fp8(*state["w"], cols=case["inner"])
    if do == "product":
        return q.qgtc_fp8_product(x, w, TYPES[case["type"]])
    u = q.Fp8(*state["u"], cols=case["inner"])
    if do == "gated":
        return _shown(q.qgtc_fp8_gated(x, w, u, case["act"]))
    return q.qgtc_fp8_gated_backward(x, w, u, state["dh"], case["act"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    do, n, c = case["do"], case["rows"], case["cols"]
    eight = 1 + 1 / BLOCK
    if do in ("norm", "norm_backward", "quantize"):
        b = BYTES[case["type"]]
        if do == "quantize":
            return {"bytes": n * c * (b + eight), "flops": 2 * n * c}
        if do == "norm":
            return {"bytes": n * c * ((3 if case["residual"] else 1) * b + eight) + b * c, "flops": 6 * n * c}
        return {"bytes": n * c * b * (4 if case["residual"] else 3) + (b + 4) * c + 4 * n, "flops": 12 * n * c}
    k = case["inner"]
    if do == "product":
        return {"bytes": (n + c) * k * eight + n * c * BYTES[case["type"]], "flops": 2 * n * c * k}
    read = (n + 2 * c) * k * eight
    if do == "gated":
        return {"bytes": read + n * c * eight, "flops": 4 * n * c * k}
    return {"bytes": read + 3 * n * c * BYTES[case["type"]], "flops": 4 * n * c * k}


# ---- in 64 bits -------------------------------------------------------------------------------------------------
def _quotients(y):
    """What the codes of y round, and the scales: y over the power of two that brings each block's largest entry under 448."""
    rows, cols = y.shape
    codes, scales = [], []
    for at in range(0, cols, BLOCK):
        part = y[:, at:at + BLOCK]
        top = part.abs().amax(1)
        two = torch.exp2(torch.ceil(torch.log2(top.clamp_min(2.0 ** -300) / 448)).clamp_min(-127.0))
        two = torch.where(two * 448 < top, two * 2, torch.where((two / 2 * 448 >= top) & (two > 2.0 ** -127), two / 2, two))
        codes.append(part / two.unsqueeze(1))
        scales.append(two)
    return {"codes": torch.cat(codes, 1), "scales": torch.stack(scales, 1)}


def exact(case, seed):
    state = prepare(case, seed)
    do, rows, cols = case["do"], case["rows"], case["cols"]
    if do == "quantize":
        x = state["x"].double()
        return _quotients(x.t().contiguous() if case["columns"] else x)
    if do == "norm":
        s = state["x"].double()
        if case["residual"]:
            s = s + state["residual"].double()
        # (the norm is of the sum as it is kept, in the inputs' type)
        kept = s.to(state["x"].dtype).double()
        out = _quotients(kept / torch.sqrt((kept * kept).sum(1, keepdim=True) / cols + EPS) * state["weight"].double())
        return dict(out, sum=s) if case["residual"] else out
    if do == "norm_backward":
        s, dy, w, r = state["x"].double(), state["dy"].double(), state["weight"].double(), state["rstd"].double()
        along = torch.einsum("ij,j,ij->i", dy, w, s)
        dx = r[:, None] * dy * w - (r ** 3 * along / cols)[:, None] * s
        if case["residual"]:
            dx = dx + state["residual"].double()
        return {"dx": dx, "dweight": torch.einsum("ij,ij,i->j", dy, s, r)}
    inner = case["inner"]

    def whole(form):
        codes, scales = form
        return codes.double()[:, :inner] * scales.double().repeat_interleave(BLOCK, 1)[:, :inner]

    x = whole(state["x"])
    g = x @ whole(state["w"]).t()
    if do == "product":
        return g
    u = x @ whole(state["u"]).t()
    if case["act"] == "silu":
        half = torch.tanh(g / 2)
        a, da = g * (1 + half) / 2, (1 + half) / 2 + g * (1 - half * half) / 4
    else:
        z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        dz = math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)
        a, da = g / (1 + torch.exp(-2 * z)), 1 / (1 + torch.exp(-2 * z)) + g * dz / (2 * torch.cosh(z.clamp(-300, 300)) ** 2)
    if do == "gated":
        return _quotients(a * u)
    dh = state["dh"].double()
    return torch.cat([dh * u * da, dh * a], 1)
