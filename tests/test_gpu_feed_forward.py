"""Norm, gate and product together, as a feed-forward block runs them: every step against its formula in 64 bits on what the
step before has left, eagerly, recorded, on another stream, and backwards."""
import numpy as np
import pytest
import torch

import fp8_util as U

pytestmark = pytest.mark.gpu

q = pytest.importorskip("paper_2111_09547_amd")
from paper_2111_09547_amd.feed_forward import GatedFeedForward  # noqa: E402


def block(d, h, dtype, act, training=False):
    t = lambda v: v.to(dtype).cuda()                      # noqa: E731
    w = 1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(9))
    return GatedFeedForward(t(w), t(U.weights(h, d, 1)), t(U.weights(h, d, 2)), t(U.weights(d, h, 3)), act=act, training=training)


def values(m):
    return U.fp8_values(m)


def product_close(got, x, w):
    want = values(x) @ values(w).T
    tol = U.product_tol(values(x), values(w), got.dtype == torch.float32)
    U.close(got, want, tol * 1.01 + U.rounded_tol(want, got.dtype))


@pytest.mark.parametrize("dtype", U.TYPES)
@pytest.mark.parametrize("rows,d,h", [(1, 256, 512), (33, 200, 300), (300, 384, 640)])
def test_forward_is_its_steps(dtype, rows, d, h):
    b = block(d, h, dtype, "silu")
    x, res = (U.activations(rows, d, k).to(dtype).cuda() for k in (4, 5))
    y, s = b.forward(x, res)
    n = q.qgtc_rms_norm(x, b.norm_weight, b.eps, residual=res)
    hq = q.qgtc_fp8_gated(n.fp8, b.gate_q, b.up_q)
    assert torch.equal(s, n.sum) and torch.equal(y, q.qgtc_fp8_product(hq, b.down_q, dtype))
    g = U.gated(values(n.fp8), values(b.gate_q), values(b.up_q), "silu")
    U.check_codes(hq, g[0], g[1] * 1.01 + 2.0 ** -149)
    product_close(y, hq, b.down_q)
    # and the whole of it near the block without 8 bits: four roundings to e4m3 of 2^-5 of an entry on average and less
    f = [t.double().cpu() for t in (s, b.norm_weight, b.gate, b.up, b.down)]
    m = f[0] / torch.sqrt(f[0].square().mean(1, keepdim=True) + b.eps) * f[1]
    want = (torch.nn.functional.silu(m @ f[2].T) * (m @ f[3].T)) @ f[4].T
    assert float((y.double().cpu() - want).norm() / want.norm()) < 4 * 2.0 ** -4


@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.float32, "gelu"), (torch.float16, "gelu")])
@pytest.mark.parametrize("rows,d,h", [(1, 130, 256), (150, 256, 300), (513, 384, 512)])
def test_gradients(dtype, act, rows, d, h):
    b = block(d, h, dtype, act, training=True)
    x, res, ds = (U.activations(rows, d, k).to(dtype).cuda() for k in (4, 5, 6))
    dy = (0.1 * torch.randn((rows, d), generator=torch.Generator().manual_seed(7))).to(dtype).cuda()
    y, s = b.forward(x, res)
    (n, kept), f32 = b._kept, torch.float32
    grads = b.backward(dy, ds)
    with pytest.raises(RuntimeError):
        b.backward(dy, ds)
    # each step from what the kernels in front of it have left
    quant = q.qgtc_fp8_quantize
    product_close(grads["down"], quant(dy, columns=True), quant(kept, columns=True))
    dh = q.qgtc_fp8_product(quant(dy), b.down_t, dtype)
    product_close(dh, quant(dy), b.down_t)
    h64, th, fg, tfg, a, ta = U.gated(values(n.fp8), values(b.gate_q), values(b.up_q), act, dtype == f32)
    d2 = q.qgtc_fp8_gated_backward(n.fp8, b.gate_q, b.up_q, dh, act)
    for at, f, tf in ((0, fg, tfg), (h, a, ta)):
        want = U.f64(dh) * f
        U.close(d2[:, at:at + h], want, np.abs(U.f64(dh)) * tf * 1.01 + 2.0 ** -23 * np.abs(want) + U.rounded_tol(want, dtype))
    whole = torch.cat([grads["gate"], grads["up"]])
    product_close(whole, quant(d2, columns=True), quant(n.y, columns=True))
    dn = q.qgtc_fp8_product(quant(d2), b.gate_up_t, dtype)
    product_close(dn, quant(d2), b.gate_up_t)
    dx, dw = q.qgtc_rms_norm_backward(dn, s, b.norm_weight, n.rstd, dsum=ds)
    assert torch.equal(dx, grads["x"]) and torch.equal(dw, grads["norm_weight"])
    # and the whole of them near the gradients without 8 bits (a chain of at most ten roundings to e4m3, each 2^-5 on average)
    p = [t.double().cpu().requires_grad_() for t in (s, b.norm_weight, b.gate, b.up, b.down)]
    m = p[0] / torch.sqrt(p[0].square().mean(1, keepdim=True) + b.eps) * p[1]
    fn = torch.nn.functional.silu if act == "silu" else lambda v: torch.nn.functional.gelu(v, approximate="tanh")
    ((fn(m @ p[2].T) * (m @ p[3].T)) @ p[4].T).backward(dy.double().cpu())
    for name, v in zip(("x", "norm_weight", "gate", "up", "down"), p):
        got, want = grads[name].double().cpu(), v.grad + (ds.double().cpu() if name == "x" else 0)
        assert float((got - want).norm() / want.norm()) < 10 * 2.0 ** -5, name


@pytest.mark.parametrize("rows", [1, 40, 600])
def test_recorded_passes(rows):
    """Two recorded blocks of one size, replayed in turn with eager work between: every replay is the eager pass on what its inputs
    hold then."""
    b, c = block(384, 640, torch.bfloat16, "silu"), block(384, 640, torch.bfloat16, "gelu")
    make = lambda k: U.activations(rows, 384, k).bfloat16().cuda()      # noqa: E731
    x1, r1, x2 = make(1), make(2), make(3)
    g1, y1, s1 = b.capture(x1, r1)
    g2, y2, s2 = c.capture(x2)
    assert s2 is x2
    for k in range(4):
        x1.copy_(make(10 + k))
        r1.copy_(make(20 + k))
        x2.copy_(make(30 + k))
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        want1, want2 = b.forward(x1.clone(), r1.clone()), c.forward(x2.clone())
        assert torch.equal(y1, want1[0]) and torch.equal(s1, want1[1]) and torch.equal(y2, want2[0])


def test_recorded_gradients():
    """Each operator's gradients in one graph, replayed several times."""
    rows, d, h = 200, 256, 384
    b = block(d, h, torch.bfloat16, "silu", training=True)
    n = q.qgtc_rms_norm(U.activations(rows, d, 1).bfloat16().cuda(), b.norm_weight, rstd=True, y=True)
    dh, dn = (torch.randn((rows, k), device="cuda").bfloat16() for k in (h, d))

    def step():
        d2 = q.qgtc_fp8_gated_backward(n.fp8, b.gate_q, b.up_q, dh)
        w = q.qgtc_fp8_product(q.qgtc_fp8_quantize(d2, columns=True), q.qgtc_fp8_quantize(n.y, columns=True), torch.float32)
        return (d2, w) + tuple(q.qgtc_rms_norm_backward(dn, n.sum, b.norm_weight, n.rstd))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for k in range(4):
        dh.copy_(torch.randn((rows, h), device="cuda"))
        dn.copy_(torch.randn((rows, d), device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        for a, w in zip(got, step()):
            assert torch.equal(a, w)


def test_another_stream():
    """Work goes to the stream that is current, behind what is in front of it there."""
    b = block(512, 1024, torch.bfloat16, "silu")
    x = U.activations(300, 512, 1).bfloat16().cuda()
    want, _ = b.forward(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = torch.zeros_like(x)
        for _ in range(20):
            late = late + 1
        late.copy_(x)
        y, _ = b.forward(late)
        z = y.clone()
    side.synchronize()
    assert torch.equal(z, want)


def test_the_same_bits_every_time():
    b = block(640, 900, torch.bfloat16, "silu", training=True)
    x, dy = (U.activations(700, 640, k).bfloat16().cuda() for k in (1, 2))
    runs = []
    for _ in range(3):
        y, _ = b.forward(x)
        runs.append((y, b.backward(dy)))
    for y, g in runs[1:]:
        assert torch.equal(y, runs[0][0]) and all(torch.equal(g[k], runs[0][1][k]) for k in g)


def test_refuses():
    b = block(256, 300, torch.float32, "silu")
    with pytest.raises(ValueError):
        b.forward(torch.zeros((4, 255), device="cuda"))
    with pytest.raises(TypeError):
        b.forward(torch.zeros((4, 256), device="cuda"), torch.zeros((4, 256), device="cuda", dtype=torch.bfloat16))
    with pytest.raises(RuntimeError):
        b.backward(torch.zeros((4, 256), device="cuda"))
    with pytest.raises(ValueError):
        GatedFeedForward(b.norm_weight, b.gate, b.up, b.gate)
    with pytest.raises(q.QgtcError):
        q.qgtc_fp8_product(q.alloc_fp8(4, 256, "cuda"), q.alloc_fp8(4, 300, "cuda"))
    with pytest.raises(KeyError):
        q.qgtc_fp8_gated(q.alloc_fp8(4, 256, "cuda"), b.gate_q, b.up_q, "tanh")


def test_recorded_pass_takes_weights_packed_again():
    """pack() leaves the weights where a recorded pass reads them; those of other sizes go elsewhere."""
    b = block(256, 300, torch.bfloat16, "silu", training=True)
    b.training = False
    x = U.activations(20, 256, 1).bfloat16().cuda()
    graph, y, _ = b.capture(x)
    before = [m.codes.data_ptr() for m in (b.gate_q, b.up_q, b.down_q)]
    for k in range(3):
        b.gate.copy_(U.weights(300, 256, 20 + k))
        b.down = U.weights(256, 300, 30 + k).bfloat16().cuda()
        b.pack()
        assert [m.codes.data_ptr() for m in (b.gate_q, b.up_q, b.down_q)] == before
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, b.forward(x)[0])
    held = b.gate_q
    b.gate, b.up = (U.weights(100, 256, k).bfloat16().cuda() for k in (40, 41))
    b.down = U.weights(256, 100, 42).bfloat16().cuda()
    b.pack()
    assert (b.gate_q.rows, b.down_q.cols) == (100, 100) and held.codes.data_ptr() == before[0]
    fresh = GatedFeedForward(b.norm_weight, b.gate, b.up, b.down)
    assert torch.equal(b.forward(x)[0], fresh.forward(x)[0])


def test_recorded_pass_keeps_what_it_reads():
    """The block and its inputs are let go, and the memory that this frees is written."""
    b = block(384, 500, torch.bfloat16, "gelu")
    x, res = (U.activations(40, 384, k).bfloat16().cuda() for k in (1, 2))
    graph, y, s = b.capture(x, res)
    want = [t.clone() for t in b.forward(x, res)]
    sizes = [t.numel() * t.element_size() for t in (x, res, b.norm_weight, b.gate_q.codes, b.gate_q.scales, b.down_q.codes, b.down_q.scales)]
    del b, x, res
    for _ in range(3):
        taken = [torch.full((n,), 0x55, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(s, want[1])
        del taken


def test_recorded_on_the_device_of_its_inputs(monkeypatch):
    """On a stream of that device, whichever is current."""
    index = torch.cuda.device_count() - 1
    b = block(256, 300, torch.bfloat16, "silu")
    for name in ("norm_weight", "gate", "up", "down"):
        setattr(b, name, getattr(b, name).to(f"cuda:{index}"))
    b.pack()
    x = U.activations(20, 256, 1).bfloat16().to(f"cuda:{index}")
    streams, graph_of = [], torch.cuda.graph
    monkeypatch.setattr(torch.cuda, "graph", lambda graph, stream=None: (streams.append(stream), graph_of(graph, stream=stream))[1])
    with torch.cuda.device(0):
        graph, y, _ = b.capture(x)
        assert torch.cuda.current_device() == 0
        graph.replay()
    assert streams[0] is not None and streams[0].device.index == index == y.get_device()
    torch.cuda.synchronize(index)
    assert torch.equal(y, b.forward(x)[0])


def test_gradients_are_of_the_weights_packed_last():
    """Weights that were packed while the block was not training."""
    b = block(256, 300, torch.bfloat16, "silu", training=True)
    x, dy = (U.activations(20, 256, k).bfloat16().cuda() for k in (1, 2))
    b.forward(x)
    b.backward(dy)
    b.training = False
    b.gate, b.up = (U.weights(300, 256, k).bfloat16().cuda() for k in (20, 21))
    b.down = U.weights(256, 300, 22).bfloat16().cuda()
    b.pack()
    b.training = True
    fresh = GatedFeedForward(b.norm_weight, b.gate, b.up, b.down, training=True)
    assert torch.equal(b.forward(x)[0], fresh.forward(x)[0])
    got, want = b.backward(dy), fresh.backward(dy)
    assert set(got) == set(want) and all(torch.equal(got[k], want[k]) for k in got)


def test_training_set_later():
    """A block made without: backward() wants its weights packed for it, and then it is as one made with."""
    b, want = (block(256, 300, torch.bfloat16, "gelu", training=t) for t in (False, True))
    x, dy = (U.activations(20, 256, k).bfloat16().cuda() for k in (1, 2))
    b.training = True
    b.forward(x)
    with pytest.raises(RuntimeError, match="pack"):
        b.backward(dy)
    b.pack()
    b.forward(x)
    want.forward(x)
    got, want = b.backward(dy), want.backward(dy)
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_packing_lets_go_of_a_forward_pass():
    """Between a forward pass and its gradients weights are not exchanged, and there is no other forward pass."""
    b = block(256, 300, torch.bfloat16, "silu", training=True)
    x, dy = (U.activations(20, 256, k).bfloat16().cuda() for k in (1, 2))
    b.forward(x)
    b.gate.copy_(U.weights(300, 256, 20))
    b.pack()
    with pytest.raises(RuntimeError, match="forward"):
        b.backward(dy)
    b.forward(x)
    b.training = False
    b.forward(2 * x)
    b.training = True
    with pytest.raises(RuntimeError, match="forward"):
        b.backward(dy)


def test_gradients_are_not_lost_silently():
    """The operators refuse a tensor that requires a gradient; a block takes parameters, whose gradients backward() returns."""
    b = block(256, 300, torch.float32, "silu", training=True)
    x, dy = (U.activations(20, 256, k).cuda() for k in (1, 2))
    xg, w, wg = x.clone().requires_grad_(), b.norm_weight, b.norm_weight.clone().requires_grad_()
    n = q.qgtc_rms_norm(x, w, rstd=True)
    h, hg = torch.empty((20, 300), device="cuda"), torch.empty((20, 300), device="cuda", requires_grad=True)
    for call in (lambda: q.qgtc_rms_norm(xg, w), lambda: q.qgtc_rms_norm(x, wg), lambda: q.qgtc_rms_norm(x, w, residual=xg),
                 lambda: q.qgtc_rms_norm_backward(xg, x, w, n.rstd), lambda: q.qgtc_rms_norm_backward(dy, x, wg, n.rstd),
                 lambda: q.qgtc_rms_norm_backward(dy, x, w, n.rstd, dsum=xg), lambda: q.qgtc_fp8_product(n.fp8, b.gate_q, out=hg),
                 lambda: q.qgtc_fp8_gated(n.fp8, b.gate_q, b.up_q, h=hg), lambda: q.qgtc_fp8_gated_backward(n.fp8, b.gate_q, b.up_q, hg),
                 lambda: b.forward(xg), lambda: b.forward(x, xg)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    y, _ = b.forward(x)
    want = b.backward(dy)
    p = [torch.nn.Parameter(t) for t in (b.norm_weight, b.gate, b.up, b.down)]
    c = GatedFeedForward(*p, training=True)
    assert torch.equal(c.forward(x)[0], y)
    got = c.backward(dy)
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_a_refused_gradient_can_be_given_again():
    b = block(256, 300, torch.bfloat16, "silu", training=True)
    x, dy = (U.activations(20, 256, k).bfloat16().cuda() for k in (1, 2))
    b.forward(x)
    want = b.backward(dy)
    b.forward(x)
    for bad, error in ((dy.float(), TypeError), (dy[:19], q.QgtcError), (dy[:, :128], q.QgtcError)):
        with pytest.raises(error):
            b.backward(bad)
    with pytest.raises(ValueError):
        b.backward(dy, dy[:19])
    got = b.backward(dy)
    assert all(torch.equal(got[k], want[k]) for k in want)
