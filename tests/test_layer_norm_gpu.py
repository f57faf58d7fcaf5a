"""Layer norm and its gradient against the formulas in 64 bits on the same inputs.

Bounds, u = half a step of the type: x^ = (x - m) r carries some 8 roundings of fp32 and what cancels in x - m, 2^-22 (|x| + |m|) r; y one rounding more.
dx: 2^-20 of r (|g| + mean |g| + |x^| mean |g x^|), the errors of x^, one rounding.  dw, db: 2^-21 of the summands' magnitudes (sums of runs).
"""
import ctypes

import pytest
import torch

from paper_2312_08874_b200 import AgentAttention, AgentAttnError

pytestmark = pytest.mark.gpu
BF, FH, F32 = torch.bfloat16, torch.float16, torch.float32


def handle(dt):
    return AgentAttention(1, 1, 64, 1, 1, dt)


def check(x, w, b, dy, eps=1e-5, mod=None):
    dt, C = x.dtype, x.shape[-1]
    u = torch.finfo(dt).eps / 2
    low = torch.finfo(dt).smallest_normal * torch.finfo(dt).eps if dt is FH else 0.0
    mod = mod or handle(dt)
    y = mod.layer_norm(x, w, b, eps=eps)
    g = mod.layer_norm_backward(x, dy, w, b, eps=eps)
    again = mod.layer_norm_backward(x, dy, w, b, eps=eps)
    assert all(torch.equal(g[n], again[n]) for n in g)
    X, D = x.double().reshape(-1, C), dy.double().reshape(-1, C)
    W, Bi = (torch.ones(C, device="cuda").double() if w is None else w.double()), (torch.zeros(C, device="cuda").double() if b is None else b.double())
    m = X.mean(1, keepdim=True)
    r = 1 / ((X - m).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (X - m) * r
    exh = 2.0 ** -21 * xh.abs() + 2.0 ** -22 * (X.abs() + X.abs().mean(1, keepdim=True)) * r * (1 + xh.abs() / 4)       # (of r, too: its sum is made of such differences)
    want = xh * W + Bi
    assert ((y.double().reshape(-1, C) - want).abs() <= u * want.abs() + exh * W.abs() + 2.0 ** -23 * want.abs() + low).all()
    G = D * W
    a, c = G.abs().mean(1, keepdim=True), (G * xh).abs().mean(1, keepdim=True)
    dx = r * (G - G.mean(1, keepdim=True) - xh * (G * xh).mean(1, keepdim=True))
    bound = 2.0 ** -20 * r * (G.abs() + a + xh.abs() * c) + r * (exh * c + xh.abs() * (G.abs() * exh).mean(1, keepdim=True)) + (exh.amax(1, keepdim=True) * dx.abs())
    assert ((g["dx"].double().reshape(-1, C) - dx).abs() <= u * dx.abs() + bound + low).all()
    assert ("dw" in g) == (w is not None) and ("db" in g) == (b is not None)
    if w is not None:
        assert g["dw"].dtype is F32
        assert ((g["dw"].double() - (D * xh).sum(0)).abs() <= (2.0 ** -21 * (D * xh).abs() + D.abs() * exh).sum(0) + 1e-30).all()
    if b is not None:
        assert ((g["db"].double() - D.sum(0)).abs() <= 2.0 ** -21 * D.abs().sum(0) + 1e-30).all()
    return y, g


def make(rows, C, dt, seed=0, mean=0.5, std=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return (r(rows, C) * std + mean * r(C)).to(dt), (1 + 0.1 * r(C)).to(dt), (0.1 * r(C)).to(dt), r(rows, C).to(dt)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("C", [1, 2, 7, 8, 20, 24, 32, 64, 96, 100, 127, 192, 320, 384, 513, 640, 768, 1000, 1023, 1024, 1280, 1536, 2047, 2048, 2056, 4096, 5000, 8191, 8192, 9000,
                               16384, 16392, 20001, 65536])
def test_channels(dt, C):
    for rows in (1, 67):
        check(*make(rows, C, dt))


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("rows,C", [(1, 64), (2, 64), (31, 192), (33, 192), (5000, 64), (4099, 320), (20011, 96), (3000, 1280), (300000, 8), (1203, 5001)])
def test_rows(dt, rows, C):
    check(*make(rows, C, dt))


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("C", [192, 100, 3000, 20001])
def test_without_weight_or_bias_and_in_place(dt, C):
    x, w, b, dy = make(50, C, dt)
    check(x.view(5, 10, C), None, None, dy.view(5, 10, C))
    check(x, w, None, dy)
    check(x, None, b, dy)
    y, g = check(x, w, b, dy)
    mod = handle(dt)
    only = mod.layer_norm_backward(x, dy, w, b, need_weight_grads=False)
    assert list(only) == ["dx"] and torch.equal(only["dx"], g["dx"])
    rest = mod.layer_norm_backward(x, dy, w, b, need_input_grad=False)
    assert torch.equal(rest["dw"], g["dw"]) and torch.equal(rest["db"], g["db"])
    x2, dy2 = x.clone(), dy.clone()
    assert mod.layer_norm(x2, w, b, out=x2) is x2 and torch.equal(x2, y)
    got = mod.layer_norm_backward(x, dy2, w, b, out=dy2)
    assert got["dx"] is dy2 and all(torch.equal(got[n], g[n]) for n in g)


@pytest.mark.parametrize("dt", [F32, BF, FH])
def test_addresses_off_a_vector(dt):
    """Slices that begin inside a vector of 16 bytes: the same numbers."""
    C = 320
    x, w, b, dy = make(40, C, dt)
    y, g = check(x, w, b, dy)
    flat = torch.empty(40 * C + 1, dtype=dt, device="cuda")
    flat[1:].copy_(x.flatten())
    mod = handle(dt)
    y2, g2 = mod.layer_norm(flat[1:].view(40, C), w, b), mod.layer_norm_backward(flat[1:].view(40, C), dy, w, b)
    check(flat[1:].view(40, C), w, b, dy)
    assert (y2.double() - y.double()).abs().max() <= torch.finfo(dt).eps * 8 and set(g2) == set(g)


@pytest.mark.parametrize("dt", [F32, BF])
def test_rows_far_from_zero_constant_rows_and_non_finite_ones(dt):
    x, w, b, dy = make(64, 192, dt, mean=0.0, std=1.0)
    check((x.float() + 300.0).to(dt), w, b, dy)
    x2 = x.clone()
    x2[3] = 2.5                                                          # no variance: the bias, and a gradient of 1 / sqrt(eps)
    check(x2, w, b, dy)
    mod = handle(dt)
    y = mod.layer_norm(x, w, b)
    g = mod.layer_norm_backward(x, dy, w, b)
    x2 = x.clone()
    x2[5, 7], x2[9, 0] = float("nan"), float("inf")
    y2, g2 = mod.layer_norm(x2, w, b), mod.layer_norm_backward(x2, dy, w, b)
    keep = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(y2[keep], y[keep]) and torch.equal(g2["dx"][keep], g["dx"][keep])
    assert y2[[5, 9]].isnan().all() and g2["dw"].isnan().all() and torch.equal(g2["db"], g["db"])
    zero = mod.layer_norm(torch.zeros_like(x), None, None, eps=0.0)
    assert zero.isnan().all()                                            # 0 / 0, as in the formula


def test_gradient_against_differences():
    x, w, b, dy = make(40, 96, F32)
    g = handle(F32).layer_norm_backward(x, dy, w, b)
    f = lambda x, w, b: (torch.nn.functional.layer_norm(x, (96,), w, b) * dy.double()).sum()  # noqa: E731
    for i, n in enumerate(("dx", "dw", "db")):
        args = [t.double() for t in (x, w, b)]
        step = torch.randn(args[i].shape, device="cuda").double()
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * step, args[i] - 1e-5 * step
        got = (g[n].double() * step).sum()
        assert abs((f(*up) - f(*down)) / 2e-5 - got) <= 1e-5 * (g[n].double() * step).norm() + 1e-5


def test_streams_and_graphs():
    x, w, b, dy = make(5000, 192, BF)
    mod = handle(BF)
    y, g = check(x, w, b, dy, mod=mod)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [(mod.layer_norm(x, w, b, stream=side), mod.layer_norm_backward(x, dy, w, b, stream=side), mod.layer_norm_backward(x, dy, w, b)) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, y) and all(torch.equal(t[n], g[n]) for t in (c, d) for n in g) for a, c, d in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, g2 = mod.layer_norm(x, w, b), mod.layer_norm_backward(x, dy, w, b)
    x.copy_(x.flip(0))
    dy.copy_(dy.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y2, y.flip(0)) and torch.equal(g2["dx"], g["dx"].flip(0))


def test_offsets_past_32_bits():
    rows, C = (1 << 22) + 3, 1024
    x = torch.zeros((rows, C), dtype=BF, device="cuda")
    x[-1] = torch.randn(C, device="cuda").to(BF)
    mod = handle(BF)
    y = mod.layer_norm(x)
    assert torch.equal(y[-1:], mod.layer_norm(x[-1:].clone())) and (y[-2] == 0).all()


def test_refusals():
    x, w, b, dy = make(8, 64, BF)
    mod = handle(BF)
    for change in (dict(x=x.float()), dict(x=x.t()), dict(x=x.cpu()), dict(weight=w[:32]), dict(bias=b.float()), dict(out=x[:4]), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            mod.layer_norm(**{**dict(x=x, weight=w, bias=b), **change})
    for change, code in ((dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(x=x[:0]), 1), (dict(out=w.view(1, 64), x=x[:1]), 1),
                         (dict(x=torch.zeros((1, 65544), dtype=BF, device="cuda"), weight=None, bias=None), 2)):
        with pytest.raises(AgentAttnError) as e:
            mod.layer_norm(**{**dict(x=x, weight=w, bias=b), **change})
        assert e.value.status == code, change.keys()
    for change in (dict(d_out=dy[:4]), dict(d_out=dy.float()), dict(out=x), dict(need_input_grad=False, need_weight_grads=False), dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, AgentAttnError)):
            mod.layer_norm_backward(**{**dict(x=x, d_out=dy, weight=w, bias=b), **change})


def test_gradient_buffers_that_alias_are_refused():
    x, w, b, dy = make(8, 64, BF)
    mod = handle(BF)
    a, g = mod._layer_norm(x, w, b, 1e-5), torch.zeros(64, device="cuda")
    ws = torch.empty(mod.lib.agent_attn_layer_norm_workspace_bytes(mod._h, 8, 64), dtype=torch.uint8, device="cuda")
    args = (mod._h, ctypes.byref(a), dy.data_ptr())
    assert mod.lib.agent_attn_layer_norm_backward(*args, None, g.data_ptr(), g.data_ptr(), ws.data_ptr(), ws.numel(), None) == 1
    assert mod.lib.agent_attn_layer_norm_backward(*args, x.data_ptr(), g.data_ptr(), None, ws.data_ptr(), ws.numel(), None) == 1
    torch.cuda.synchronize()
    assert (g == 0).all()


@pytest.mark.parametrize("dt,rows,C", [(BF, 1 << 21, 2048), (F32, 1 << 17, 8192), (FH, 1 << 18, 1023), (BF, 1 << 16, 20001), (FH, (1 << 22) + 3, 8), (F32, 200704, 64)])
def test_gain_gradients_of_equal_rows(dt, rows, C):
    """Equal summands, which are rounded the same way at every step.  A sum of n of them is off by n 2^-25 at most: 256 rows of a thread, up to 256 shares of a warp in the join and
    the warps' 32; x^ itself, the same in every row, by 2^-21."""
    x = make(1, C, dt)[0].expand(rows, C).contiguous()
    dy = torch.full((rows, C), 0.7, dtype=dt, device="cuda")
    w, b = torch.ones(C, dtype=dt, device="cuda"), torch.zeros(C, dtype=dt, device="cuda")
    g = handle(dt).layer_norm_backward(x, dy, w, b, need_input_grad=False)
    X, d = x[0].double(), dy[0, 0].double()
    m = X.mean()
    r = 1 / ((X - m).square().mean() + 1e-5).sqrt()
    xh, few = (X - m) * r, 2.0 ** -25 * (256 + min(256, rows / 256) + 64)
    assert (g["db"].double() / (d * rows) - 1).abs().max() <= few
    exh = 2.0 ** -21 * xh.abs() + 2.0 ** -22 * (X.abs() + X.abs().mean()) * r * (1 + xh.abs() / 4)
    assert ((g["dw"].double() - d * rows * xh).abs() <= d * rows * (few * xh.abs() + exh)).all()
