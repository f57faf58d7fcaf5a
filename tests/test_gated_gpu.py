"""The gated feed-forward product (`gated`, `gated_backward`) against the formulas in 64 bits.

Tolerances.  16-bit types, forward: products of 16-bit numbers are exact in fp32, their sum over up to 600 channels loses at most 40 steps of 2^-23
of its size in tensor memory, activation and product some 2^-21; then one rounding, at most 2^-8 or 2^-11 of the result: 2e-5 of the largest result beside
it.  Backward: the gradients of both projections are rounded to the element type (2^-9 / sqrt(3) = 1.1e-3 for bf16, 2.8e-4 for f16,
of the power of two above), and
the result again: 1.6e-3 and 4e-4, and twice that for what the few numbers of a small case leave to chance; a bias of few rows sums unrounded
numbers and is inside that.  fp32: three bf16 terms hold 24 bits; sums lose up to a step of 2^-23 each 16 summands: 2e-6 forward (600 channels),
4e-6 for sums of up to 2500 numbers and more, which are cut into shares.
"""
import math

import pytest
import torch

from paper_2312_08874_b200 import AgentAttention, AgentAttnError

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = {n: torch.finfo(DT[n]).eps / 2 for n in ("bf16", "f16")}
REL_FWD, REL_BWD = 2e-6, {"f32": 4e-6, "bf16": 3.2e-3, "f16": 8e-4}


def act(name, g):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * (1 + torch.erf(g / math.sqrt(2)))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def inputs(M, C, F, dtype, biases, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def draw(shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(DT[dtype])
    return (draw((M, C)), draw((F, C), C ** -0.5), draw((F, C), C ** -0.5), draw((M, F)),
            draw((F,), 0.5) if "g" in biases else None, draw((F,), 0.5) if "u" in biases else None)


def reference(x, wg, wu, dh, bg, bu, name):
    leaves = [t.double().requires_grad_() if t is not None else None for t in (x, wg, wu, bg, bu)]
    g, u = leaves[0] @ leaves[1].T, leaves[0] @ leaves[2].T
    g = g if bg is None else g + leaves[3]
    u = u if bu is None else u + leaves[4]
    h = act(name, g) * u
    h.backward(dh.double())
    return h.detach(), {n: t.grad for n, t in zip(("dx", "dw_gate", "dw_up", "db_gate", "db_up"), leaves) if t is not None}


def rel(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


def check_forward(got, ref, dtype):
    assert torch.isfinite(got).all()
    if dtype == "f32":
        assert rel(got, ref) <= REL_FWD
    else:
        err = (got.double() - ref).abs()
        assert (err <= STEP[dtype] * ref.abs() + 2e-5 * ref.abs().max()).all()


SIZES = [(1, 8, 8), (1, 320, 1280), (2, 40, 136), (63, 72, 200), (128, 64, 128), (129, 136, 264), (300, 600, 72), (257, 192, 520), (1000, 320, 128), (2500, 24, 1368)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("name,biases", [("silu", ""), ("gelu", "gu"), ("gelu_tanh", "g"), ("silu", "u")])
def test_both_directions_match_the_formulas(size, dtype, name, biases):
    M, C, F = size
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, biases, seed=M)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    h, grads = reference(x, wg, wu, dh, bg, bu, name)
    out = torch.full((M, F), float("nan"), device="cuda", dtype=DT[dtype])
    args = dict(b_gate=bg, b_up=bu, activation=name)
    got = mod.gated(x, wg, wu, out=out, **args)
    check_forward(got, h, dtype)
    need = int(mod.lib.agent_attn_gated_workspace_bytes(mod._h, M, C, F, 1))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")               # NaN wherever it is read before it is written
    back = mod.gated_backward(x, wg, wu, dh, workspace=ws, **args)
    assert mod.query_status() == 0
    for n, t in back.items():
        assert torch.isfinite(t).all() and rel(t, grads[n]) <= REL_BWD[dtype], (n, rel(t, grads[n]))
    assert ("db_gate" in back) == (biases == "gu")
    again = mod.gated_backward(x, wg, wu, dh, **args)
    assert all(torch.equal(again[n], back[n]) for n in back)                       # sums in a fixed order


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [(1, 1024, 4096), (3, 24, 72), (4, 264, 136), (5, 512, 88), (8, 640, 1704), (9, 640, 1704), (64, 256, 1032), (33, 520, 40)])
def test_few_rows_and_small_problems(size, dtype):
    """Single tokens, a few of them, and what lies just past the lines of the kernels for few rows and small fp32 problems."""
    M, C, F = size
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=C)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    for name in ("silu", "gelu", "gelu_tanh"):
        for g, u in ((bg, bu), (None, bu), (None, None)):
            h, _ = reference(x, wg, wu, dh, g, u, name)
            out = torch.full((M, F), float("nan"), device="cuda", dtype=DT[dtype])
            check_forward(mod.gated(x, wg, wu, b_gate=g, b_up=u, activation=name, out=out), h, dtype)
    assert mod.query_status() == 0


@pytest.mark.parametrize("dtype,M,C,F", [("bf16", 20000, 192, 512), ("f16", 8192, 320, 1280), ("f32", 6000, 64, 256), ("bf16", 3000, 1032, 2728), ("f32", 200, 1024, 4096)])
def test_long_sums_and_large_sizes(dtype, M, C, F):
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=5)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    h, grads = reference(x, wg, wu, dh, bg, bu, "gelu")
    args = dict(b_gate=bg, b_up=bu, activation="gelu")
    check_forward(mod.gated(x, wg, wu, **args), h, dtype)
    back = mod.gated_backward(x, wg, wu, dh, **args)
    assert mod.query_status() == 0
    for n, t in back.items():
        assert rel(t, grads[n]) <= REL_BWD[dtype], (n, rel(t, grads[n]))


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_activations_over_their_range(name, dtype):
    """One channel, weights of one: G is the input itself, U a bias of one.  Saturated ends and extreme inputs give neither NaN nor wrong signs."""
    big = 6e4 if dtype == "f16" else 1e30
    x = torch.cat([torch.linspace(-12, 12, 2001), torch.tensor([-big, -300.0, -40.0, 40.0, 300.0, big])]).to(DT[dtype]).cuda()[:, None]
    x = torch.cat([x, torch.zeros((x.shape[0], 7), device="cuda", dtype=x.dtype)], 1)
    wg = torch.zeros((8, 8), device="cuda", dtype=x.dtype)
    wg[:, 0] = 1
    wu, one = torch.zeros_like(wg), torch.ones(8, device="cuda", dtype=x.dtype)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    got = mod.gated(x, wg, wu, b_up=one, activation=name)
    g = x[:, :1].double()
    want = torch.where(g < -100, 0.0, torch.where(g > 100, g, act(name, g.clamp(-100, 100))))
    tol = 2.4e-7 * g.abs().clamp(max=100) + (STEP.get(dtype, 2.0 ** -23)) * want.abs() + (6e-8 if dtype == "f16" else 1e-12)
    tol = tol + 1e-6 * g.abs().clamp(max=6)                  # absolute error of the sigmoid and of the normal distribution
    assert torch.isfinite(got).all() and ((got.double() - want).abs() <= tol).all()
    # derivative: d(act)/dg is the gradient of the gate's bias, row by row
    for i in (0, 700, 1000, 1200, 2000, 2001, 2006):
        leaf = g[i:i + 1].clamp(-100, 100).requires_grad_()
        act(name, leaf).sum().backward()
        back = mod.gated_backward(x[i:i + 1].contiguous(), wg, wu, torch.ones((1, 8), device="cuda", dtype=x.dtype), b_gate=torch.zeros_like(one), b_up=one, activation=name)
        assert abs(float(back["db_gate"][0]) - float(leaf.grad)) <= 2 * STEP.get(dtype, 2.0 ** -22) * abs(float(leaf.grad)) + 3e-6


def test_gradient_against_differences():
    """Central differences of the forward call in fp32 with steps of 1e-2."""
    M, C, F = 40, 24, 64
    x, wg, wu, dh, bg, bu = inputs(M, C, F, "f32", "gu", seed=9)
    t = inputs(M, C, F, "f32", "gu", seed=10)
    mod = AgentAttention(1, 1, 64, 1, 1, torch.float32)

    def loss(s):
        h = mod.gated(x + s * t[0], wg + s * t[1], wu + s * t[2], b_gate=bg + s * t[4], b_up=bu + s * t[5], activation="gelu")
        return float((h.double() * dh).sum())
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation="gelu")
    parts = [back[n].double() * d for n, d in (("dx", t[0]), ("dw_gate", t[1]), ("dw_up", t[2]), ("db_gate", t[4]), ("db_up", t[5]))]
    slope, size = float(sum(p.sum() for p in parts)), float(sum(p.abs().sum() for p in parts))
    assert abs((loss(1e-2) - loss(-1e-2)) / 2e-2 - slope) <= 1e-3 * size


def test_non_finite_rows_stay_alone():
    """A NaN or an infinity in a row of X reaches that row only; in a row of a weight, that hidden unit only."""
    for dtype in ("bf16", "f32"):
        x, wg, wu, dh, bg, bu = inputs(200, 64, 136, dtype, "", seed=2)
        mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
        clean = mod.gated(x, wg, wu)
        x[77, 3], x[130, 0], wu[9, 9] = float("nan"), float("inf"), float("nan")
        got = mod.gated(x, wg, wu)
        rows, cols = torch.ones(200, dtype=torch.bool, device="cuda"), torch.ones(136, dtype=torch.bool, device="cuda")
        rows[[77, 130]], cols[9] = False, False
        assert torch.equal(got[rows][:, cols], clean[rows][:, cols])
        assert torch.isnan(got[77]).all() and torch.isnan(got[:, 9]).all()


def test_streams_batched_shapes_fused_weights_and_parts():
    x, wg, wu, dh, bg, bu = inputs(6 * 50, 64, 128, "bf16", "gu", seed=4)
    mod = AgentAttention(1, 1, 64, 1, 1, torch.bfloat16)
    want = mod.gated(x, wg, wu, b_gate=bg, b_up=bu, activation="gelu")
    fused = torch.cat([wg, wu])
    a, b = fused.chunk(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mod.gated(x.view(6, 50, 64), a, b, b_gate=bg, b_up=bu, activation="gelu", stream=side)
    back = mod.gated_backward(x, a, b, dh, b_gate=bg, b_up=bu, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert got.shape == (6, 50, 128) and torch.equal(got.view(300, 128), want)
    only_x = mod.gated_backward(x, a, b, dh, b_gate=bg, b_up=bu, need_weight_grads=False)
    only_w = mod.gated_backward(x, a, b, dh, b_gate=bg, b_up=bu, need_input_grad=False)
    assert list(only_x) == ["dx"] and "dx" not in only_w
    assert all(torch.equal(back[n], t) for part in (only_x, only_w) for n, t in part.items())


def test_refusals():
    x, wg, wu, dh, bg, bu = inputs(16, 64, 128, "bf16", "gu")
    mod = AgentAttention(1, 1, 64, 1, 1, torch.bfloat16)
    for bad in (lambda: mod.gated(x, wg, wu, activation="relu"), lambda: mod.gated(x.float(), wg, wu), lambda: mod.gated(x, wg, wu[:-1]),
                lambda: mod.gated(x, wg, wu, b_gate=bg[:-1]), lambda: mod.gated(x[:, ::2], wg[:, ::2], wu), lambda: mod.gated(x.cpu(), wg, wu),
                lambda: mod.gated_backward(x, wg, wu, dh[:-1])):
        with pytest.raises(ValueError):
            bad()

    def status(call):
        with pytest.raises(AgentAttnError) as e:
            call()
        return e.value.status
    assert status(lambda: mod.gated(x[:, :60].contiguous(), wg[:, :60].contiguous(), wu[:, :60].contiguous())) == 2      # rows of no 16 bytes
    assert status(lambda: mod.gated(x, wg[:100].contiguous(), wu[:100].contiguous())) == 2
    assert status(lambda: mod.gated(x[:0], wg, wu)) == 1                                                                  # no rows
    assert status(lambda: mod.gated_backward(x, wg, wu, dh, need_input_grad=False, need_weight_grads=False)) == 1
    assert status(lambda: mod.gated_backward(x, wg, wu, dh, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))) == 3
    wide = torch.empty(16 * 64 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(16, 64)                                 # off by an element
    assert status(lambda: mod.gated(wide, wg, wu)) == 1
    assert status(lambda: mod.gated(x, wg[:64].contiguous(), wu[:64].contiguous(), out=x)) == 1
    lib = mod.lib
    assert lib.agent_attn_gated(mod._h, None, x.data_ptr(), None, 0, None) == 1
    assert lib.agent_attn_gated_workspace_bytes(mod._h, 16, 60, 128, 0) == 0 and lib.agent_attn_gated_workspace_bytes(mod._h, 16, 64, 128, 0) == 0
    assert lib.agent_attn_gated_workspace_bytes(mod._h, 16, 64, 128, 1) > 0


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("dtype,M,C,F", [("f32", 12000, 64, 264), ("f16", 9000, 72, 648), ("bf16", 5200, 520, 1032), ("bf16", 9473, 136, 320)])
def test_tiles_that_pairs_of_blocks_share(dtype, M, C, F, name):
    """More tiles than pairs of blocks and no multiple of them: runs that begin or end with half of a tile, with a tile whose second half lies past the
    hidden units, and gradients whose shares come from many pairs."""
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=M)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    h, grads = reference(x, wg, wu, dh, bg, bu, name)
    args = dict(b_gate=bg, b_up=bu, activation=name)
    check_forward(mod.gated(x, wg, wu, **args), h, dtype)
    back = mod.gated_backward(x, wg, wu, dh, **args)
    assert mod.query_status() == 0
    for n, t in back.items():
        assert torch.isfinite(t).all() and rel(t, grads[n]) <= REL_BWD[dtype], (n, rel(t, grads[n]))
    again = mod.gated_backward(x, wg, wu, dh, need_input_grad=False, **args)
    assert all(torch.equal(again[n], back[n]) for n in again)


def hidden_errors(x, wg, wu, dh, bg, bu, name, step, tiny):
    """What an element of dG and dU may be off by: `step` of itself (how it is held, the order of the sum), 4e-6 of dH U for the derivative and its
    argument and of dH act' for U (sums of fp32 numbers around 1), 2e-6 of dH (1 + |G|) for the activation."""
    g, u = x.double() @ wg.double().T + bg.double(), x.double() @ wu.double().T + bu.double()
    g.requires_grad_()
    a = act(name, g)
    da, = torch.autograd.grad(a.sum(), g)
    d, a = dh.double(), a.detach()
    return (step * (d * u * da).abs() + 4e-6 * ((d * u).abs() + (d * da).abs()) + tiny, step * (d * a).abs() + 2e-6 * (d * (1 + g.detach().abs())).abs() + tiny)


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(1, 32, 64), (1, 320, 1280), (7, 64, 176), (33, 96, 256), (128, 40, 72)])
def test_gradients_of_few_rows_are_rounded_once(size, dtype, name):
    """Element by element: one rounding of the result, and what the two terms of each summand leave (`hidden_errors`); in f16 half a step of its
    smallest numbers for each second term."""
    M, C, F = size
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=M + F)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    _, grads = reference(x, wg, wu, dh, bg, bu, name)
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation=name)
    eg, eu = hidden_errors(x, wg, wu, dh, bg, bu, name, 2.0 ** -16 + 1e-5, 6e-8 if dtype == "f16" else 0.0)
    xa = x.double().abs()
    left = dict(dx=eg @ wg.double().abs() + eu @ wu.double().abs(), dw_gate=eg.T @ xa, dw_up=eu.T @ xa, db_gate=eg.sum(0), db_up=eu.sum(0))
    for n, t in back.items():
        bound = STEP[dtype] * grads[n].abs() + left[n] + (6e-8 if dtype == "f16" else 0.0)
        assert ((t.double() - grads[n]).abs() <= bound).all(), (n, float(((t.double() - grads[n]).abs() / bound).max()))


@pytest.mark.parametrize("dtype,M,C,F", [("bf16", 9473, 136, 320), ("f16", 700, 64, 256), ("f16", 8192, 64, 2560), ("bf16", 300, 64, 136)])
def test_biases_are_summed_before_they_are_rounded(dtype, M, C, F):
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=F)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    _, grads = reference(x, wg, wu, dh, bg, bu, "gelu")
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation="gelu")
    for n, e in zip(("db_gate", "db_up"), hidden_errors(x, wg, wu, dh, bg, bu, "gelu", 1e-5, 0.0)):
        bound = STEP[dtype] * grads[n].abs() + e.sum(0) + (6e-8 if dtype == "f16" else 0.0)
        assert ((back[n].double() - grads[n]).abs() <= bound).all()


def test_offsets_past_32_bits():
    """More than 2^31 hidden values.  Only some rows have a gradient, among them the last: what the others add is zero."""
    M, C, F, dtype = 2100000, 8, 1032, "bf16"
    gen = torch.Generator(device="cuda").manual_seed(9)
    x, wg, wu = ((torch.randn(s, generator=gen, device="cuda") * f).to(DT[dtype]) for s, f in (((M, C), 1.0), ((F, C), C ** -0.5), ((F, C), C ** -0.5)))
    some = torch.tensor([0, 1, 127, 255, 256, M // 2, M // 2 + 77, M - 300, M - 2, M - 1], device="cuda")
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    out = mod.gated(x, wg, wu, activation="gelu")
    dh = torch.randn((len(some), F), generator=gen, device="cuda").to(DT[dtype])
    h, grads = reference(x[some], wg, wu, dh, None, None, "gelu")
    check_forward(out[some], h, dtype)
    out.zero_()
    out[some] = dh
    back = mod.gated_backward(x, wg, wu, out, activation="gelu")
    assert mod.query_status() == 0
    assert rel(back["dx"][some], grads["dx"]) <= REL_BWD[dtype] and int(back["dx"].abs().sum(1).count_nonzero()) <= len(some)
    for n in ("dw_gate", "dw_up"):
        assert rel(back[n], grads[n]) <= REL_BWD[dtype]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinite_gradients_of_few_rows_stay_infinite(dtype):
    """What rounding an infinity to the element type leaves is nothing: the second term does not make NaN of it."""
    x, wg, wu, dh, bg, bu = inputs(3, 16, 24, dtype, "gu", seed=2)
    dh[1, 5] = math.inf
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    g, u = x.double() @ wg.double().T + bg.double(), x.double() @ wu.double().T + bu.double()
    s = torch.sigmoid(g)
    dg, du = dh.double() * u * (s + g * s * (1 - s)), dh.double() * g * s
    want = dict(dw_gate=dg.T @ x.double(), dw_up=du.T @ x.double(), db_gate=dg.sum(0), db_up=du.sum(0))
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation="silu")
    rest = torch.arange(24, device="cuda") != 5
    for n in want:
        assert want[n][5].isinf().all() and torch.equal(back[n][5].double(), want[n][5])
        assert rel(back[n][rest], want[n][rest]) <= REL_BWD[dtype]
    assert back["dx"][1].isfinite().sum() == 0 and back["dx"][[0, 2]].isfinite().all()


@pytest.mark.parametrize("name,dtype", [("silu", "bf16"), ("gelu", "f16")])
@pytest.mark.parametrize("size", [(1, 64, 4744), (128, 64, 8192), (33, 40, 11008), (128, 512, 5128)])
def test_gradients_of_few_rows_and_many_hidden_units_are_rounded_once(size, name, dtype):
    """The bound of `test_gradients_of_few_rows_are_rounded_once`, with so many hidden units that their tiles fill the GPU."""
    M, C, F = size
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=M + F)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    _, grads = reference(x, wg, wu, dh, bg, bu, name)
    need = int(mod.lib.agent_attn_gated_workspace_bytes(mod._h, M, C, F, 1))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation=name, workspace=ws)
    assert mod.query_status() == 0
    eg, eu = hidden_errors(x, wg, wu, dh, bg, bu, name, 2.0 ** -16 + 1e-5, 6e-8 if dtype == "f16" else 0.0)
    xa = x.double().abs()
    left = dict(dx=eg @ wg.double().abs() + eu @ wu.double().abs(), dw_gate=eg.T @ xa, dw_up=eu.T @ xa, db_gate=eg.sum(0), db_up=eu.sum(0))
    for n, t in back.items():
        bound = STEP[dtype] * grads[n].abs() + left[n] + (6e-8 if dtype == "f16" else 0.0)
        assert ((t.double() - grads[n]).abs() <= bound).all(), (n, float(((t.double() - grads[n]).abs() / bound).max()))


LONG_SUMS = [("f32", 500000, 32, 128), ("f32", 300, 16384, 256), ("f32", 3000, 1032, 2048), ("f32", 2500, 64, 8192), ("f32", 20, 8192, 64),
             ("f16", 300, 65536, 256), ("f16", 3000, 16448, 2048), ("bf16", 3000, 16448, 2048), ("bf16", 2500, 64, 65536), ("f16", 3000000, 24, 72), ("bf16", 100, 20000, 64)]


@pytest.mark.parametrize("dtype,M,C,F", LONG_SUMS)
def test_sums_of_any_length(dtype, M, C, F):
    """Sums in tensor memory lose 3e-8 of themselves a step of 16, towards zero.  fp32: 32 steps, 1e-6, and the pieces' sum in fp32 another 1e-6 (thousands of
    pieces): the bounds of short sums hold.  16 bits: 1024 steps, 3e-5 in G and in U, which the activation's slope makes 8e-5 of H, beside its rounding."""
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=6)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    h, grads = reference(x, wg, wu, dh, bg, bu, "silu")
    args = dict(b_gate=bg, b_up=bu, activation="silu")
    got = mod.gated(x, wg, wu, **args)
    assert rel(got, h) <= (REL_FWD if dtype == "f32" else math.hypot(rel(h.to(DT[dtype]), h), 8e-5)), rel(got, h)
    need = int(mod.lib.agent_attn_gated_workspace_bytes(mod._h, M, C, F, 1))
    back = mod.gated_backward(x, wg, wu, dh, workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), **args)
    assert mod.query_status() == 0
    for n, t in back.items():
        assert torch.isfinite(t).all() and rel(t, grads[n]) <= REL_BWD[dtype], (n, rel(t, grads[n]))
    again = mod.gated_backward(x, wg, wu, dh, need_input_grad=False, **args)
    assert all(torch.equal(again[n], back[n]) for n in again)
    only = mod.gated_backward(x, wg, wu, dh, need_weight_grads=False, **args)
    assert torch.equal(only["dx"], back["dx"])


@pytest.mark.parametrize("M,C,F", [(9, 40, 136), (100, 320, 1280), (700, 320, 1280), (8192, 320, 1280)])
@pytest.mark.parametrize("kind", ["large", "small"])
def test_half_precision_gradients_over_their_whole_range(kind, M, C, F):
    """f16 results in range out of gradients of the projections that are not: far past 65504, or so small that f16 has a few bits left of them.  The bound of other
    magnitudes, and half a step of the smallest results (3e-8)."""
    x, wg, wu, dh, bg, bu = inputs(M, C, F, "f16", "gu", seed=M)
    if kind == "large":
        x, wg, wu, dh, bu = x * 1e-3, (wg.float() * 2e-3).half(), (wu.float() * 2e-3).half(), dh * 3000, bu * 100 + 30
    else:
        dh = (dh.float() * 1e-6).half()
    mod = AgentAttention(1, 1, 64, 1, 1, torch.float16)
    _, grads = reference(x, wg, wu, dh, bg, bu, "gelu")
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu, activation="gelu")
    assert mod.query_status() == 0
    if kind == "large":
        g, u = x.double() @ wg.double().T + bg.double(), x.double() @ wu.double().T + bu.double()
        assert float((dh.double() * u * act("gelu", g)).abs().max()) > 2e5                 # (what used to be infinite)
    for n, t in back.items():
        fits = grads[n].half().isfinite()
        clear = (grads[n].abs() / 65520 - 1).abs() > REL_BWD["f16"]                           # (not beside the first number that rounds to an infinity)
        assert torch.equal(t.isinf()[clear], ~fits[clear]) and (n[1] == "b" or fits.float().mean() > 0.99)
        fits &= t.isfinite()
        err, ref = (t.double() - grads[n])[fits], grads[n][fits]
        assert float(err.norm()) <= REL_BWD["f16"] * float(ref.norm()) + 3e-8 * fits.sum().item() ** 0.5, (n, float(err.norm() / ref.norm()))


def test_half_precision_gradients_beside_extreme_rows():
    """Rows of zeros, an infinite gradient or a NaN in an input leave the small gradients of the other rows what they are; no gradient at all gives zeros."""
    M, C, F = 300, 64, 136
    x, wg, wu, dh, bg, bu = inputs(M, C, F, "f16", "gu", seed=1)
    dh = (dh.float() * 1e-6).half()
    mod = AgentAttention(1, 1, 64, 1, 1, torch.float16)
    back = mod.gated_backward(x, wg, wu, torch.zeros_like(dh), b_gate=bg, b_up=bu)
    assert all((t == 0).all() for t in back.values())
    x[7], dh[8], dh[100, 3], x[200, 5] = 0, 0, math.inf, math.nan
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[[100, 200]] = False
    _, grads = reference(x[rows], wg, wu, dh[rows], bg, bu, "silu")
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu)
    err = back["dx"][rows].double() - grads["dx"]
    assert float(err.norm()) <= REL_BWD["f16"] * float(grads["dx"].norm()) + 3e-8 * err.numel() ** 0.5
    assert not back["dx"][100].isfinite().any() and back["dx"][200].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,C,F", [(129, 136, 264), (700, 64, 256), (8192, 320, 1280), (5200, 520, 1032)])
def test_two_terms_on_request(M, C, F, dtype):
    """Over any number of rows, the bound of `test_gradients_of_few_rows_are_rounded_once`."""
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=M)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    _, grads = reference(x, wg, wu, dh, bg, bu, "gelu")
    need = int(mod.lib.agent_attn_gated_workspace_bytes(mod._h, M, C, F, 2))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    args = dict(b_gate=bg, b_up=bu, activation="gelu")
    back = mod.gated_backward(x, wg, wu, dh, two_terms=True, workspace=ws, **args)
    assert mod.query_status() == 0
    eg, eu = hidden_errors(x, wg, wu, dh, bg, bu, "gelu", 2.0 ** -16 + 1e-5, 6e-8 if dtype == "f16" else 0.0)
    xa = x.double().abs()
    left = dict(dx=eg @ wg.double().abs() + eu @ wu.double().abs(), dw_gate=eg.T @ xa, dw_up=eu.T @ xa, db_gate=eg.sum(0), db_up=eu.sum(0))
    for n, t in back.items():
        bound = STEP[dtype] * grads[n].abs() + left[n] + (6e-8 if dtype == "f16" else 0.0)
        assert ((t.double() - grads[n]).abs() <= bound).all(), (n, float(((t.double() - grads[n]).abs() / bound).max()))
        assert rel(t, grads[n]) <= 1.05 * rel(grads[n].to(DT[dtype]), grads[n])
    one = mod.gated_backward(x, wg, wu, dh, **args)
    assert rel(one["dx"], grads["dx"]) > 1.2 * rel(back["dx"], grads["dx"])              # (what it is for)
    with pytest.raises(AgentAttnError) as e:                                             # the workspace of one term is too small
        mod.gated_backward(x, wg, wu, dh, two_terms=True, workspace=torch.empty(int(mod.lib.agent_attn_gated_workspace_bytes(mod._h, M, C, F, 1)), dtype=torch.uint8, device="cuda"), **args)
    assert e.value.status == 3


@pytest.mark.parametrize("dtype,M,C,F", [("f32", 63, 72, 200), ("bf16", 5, 40, 136), ("f16", 700, 64, 256), ("bf16", 9473, 136, 320)])
def test_gradient_of_a_bias_alone(dtype, M, C, F):
    x, wg, wu, dh, bg, bu = inputs(M, C, F, dtype, "gu", seed=3)
    mod = AgentAttention(1, 1, 64, 1, 1, DT[dtype])
    for name, args in (("db_gate", dict(b_gate=bg)), ("db_up", dict(b_up=bu))):
        _, grads = reference(x, wg, wu, dh, args.get("b_gate"), args.get("b_up"), "gelu")
        with pytest.warns(UserWarning, match="need_bias_grads"):
            silent = mod.gated_backward(x, wg, wu, dh, activation="gelu", **args)
        back = mod.gated_backward(x, wg, wu, dh, activation="gelu", need_bias_grads=True, **args)
        assert set(back) == {"dx", "dw_gate", "dw_up", name} and rel(back[name], grads[name]) <= REL_BWD[dtype]
        assert all(torch.equal(back[n], t) for n, t in silent.items())
        only = mod.gated_backward(x, wg, wu, dh, activation="gelu", need_bias_grads=True, need_input_grad=False, need_weight_grads=False, **args)
        assert list(only) == [name] and torch.equal(only[name], back[name])
    both = dict(b_gate=bg, b_up=bg)                          # one tensor for both is two biases
    _, grads = reference(x, wg, wu, dh, bg, bg, "silu")
    back = mod.gated_backward(x, wg, wu, dh, **both)
    assert all(rel(back[n], grads[n]) <= REL_BWD[dtype] for n in ("db_gate", "db_up"))
    assert set(mod.gated_backward(x, wg, wu, dh, need_bias_grads=False, **both)) == {"dx", "dw_gate", "dw_up"}
    assert set(mod.gated_backward(x, wg, wu, dh, need_bias_grads=True)) == {"dx", "dw_gate", "dw_up"}


@pytest.mark.parametrize("M,C,F", [(300, 16448, 256), (1000, 16448, 2048), (2500, 64, 20480), (100, 16448, 256)])
def test_small_half_precision_gradients_of_long_sums(M, C, F):
    """Both at once: the second pass over G and U that come in pieces, and results that are divided after their pieces have met."""
    x, wg, wu, dh, bg, bu = inputs(M, C, F, "f16", "gu", seed=8)
    dh = (dh.float() * 1e-6).half()
    mod = AgentAttention(1, 1, 64, 1, 1, torch.float16)
    _, grads = reference(x, wg, wu, dh, bg, bu, "silu")
    back = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu)
    assert mod.query_status() == 0
    for n, t in back.items():
        assert float((t.double() - grads[n]).norm()) <= REL_BWD["f16"] * float(grads[n].norm()) + 3e-8 * t.numel() ** 0.5, n
    again = mod.gated_backward(x, wg, wu, dh, b_gate=bg, b_up=bu)
    assert all(torch.equal(again[n], back[n]) for n in back)
