"""Queries and keys before the attention (`rotate`, `rotate_backward`): an RMS norm of each head and rotary positions, against the formulas in 64 bits.

Tolerances.  A pair (u, v) turned by t: the angle carries about 2^-24 of a turn (4e-7), cosine and sine 2 units in the last place (1.2e-7 each),
1 / sqrt 2^-22 (2.4e-7), the products and the sum 2^-24 each: below 1.5e-6 of |u| + |v| after norm and gain; 16-bit results are rounded once more
(by 2^-8 or 2^-11 of themselves at most).  Gradients have three factors 1 / sqrt and a mean of d products: 4e-6 of the largest gradient of the row;
a gain's gradient is a sum of such products: 4e-6 of the sum of their sizes.
"""
import ctypes

import pytest
import torch

from paper_2312_08874_b200 import AgentAttention, AgentAttnError, Rotary

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = {"f32": 0.0, "bf16": torch.finfo(torch.bfloat16).eps / 2, "f16": torch.finfo(torch.float16).eps / 2}


def pairs_of(channels, neighbours):
    first, second, axis, at = [], [], [], 0
    for a, seg in enumerate(channels):
        for j in range(seg // 2):
            first.append(at + (2 * j if neighbours else j))
            second.append(at + (2 * j + 1 if neighbours else j + seg // 2))
            axis.append(a)
        at += seg
    return first, second, axis


def grid_positions(extent):
    axes = [torch.arange(e, dtype=torch.float64) for e in extent]
    return torch.stack([m.reshape(-1) for m in torch.meshgrid(*axes, indexing="ij")], -1)[None]


def turned(x, positions, channels, freq, neighbours, sign=1.0):
    first, second, axis = pairs_of(channels, neighbours)
    if not first:
        return x.clone()
    t = (positions.double().cuda()[:, :, axis] * freq.double())[:, None] * sign
    y = x.clone()
    u, v = x[..., first], x[..., second]
    y[..., first], y[..., second] = u * t.cos() - v * t.sin(), u * t.sin() + v * t.cos()
    return y


def reference(x, positions, channels, freq, neighbours, gain, eps):
    y = x.double()
    if eps is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * (1.0 if gain is None else gain.double())
    out = turned(y, positions, channels, freq, neighbours)
    first, second, _ = pairs_of(channels, neighbours)
    size = y.abs()
    if first:
        size[..., first], size[..., second] = (y[..., first].abs() + y[..., second].abs(),) * 2
    return out, size


def check(got, ref, size, dtype):
    err = (got.double() - ref).abs()
    bound = 1.5e-6 * size + STEP[dtype] * ref.abs() + (6e-8 if dtype == "f16" else 0.0)      # (f16: half a step of its smallest numbers)
    assert torch.isfinite(got).all() and (err <= bound).all(), float((err - bound).max())


def views(kind, B, h, N, d, dt, gen, std=1.0):
    def draw(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)
    if kind == "dense":
        return draw(B, h, N, d), draw(B, h, N, d)
    if kind == "interleaved":
        qkv = draw(B, N, 3, h, d)
        return tuple(qkv[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    wide = draw(N, B, 2, h, d + 16)                          # token first, rows wider than a head
    return tuple(wide[:, :, i, :, :d].permute(1, 2, 0, 3) for i in range(2))


CASES = [
    # B, h, d, extent, channels, neighbours, norm, kind
    (2, 3, 64, (7, 9), (32, 32), False, True, "dense"),
    (2, 3, 64, (7, 9), (32, 32), True, True, "interleaved"),
    (1, 1, 64, (1,), (64,), False, True, "dense"),                     # one token
    (3, 2, 64, (2, 5, 3), (16, 24, 24), False, False, "interleaved"),  # segments of whole pieces in 16 bits
    (3, 2, 64, (2, 5, 3), (20, 20, 20), False, True, "interleaved"),   # of no whole pieces; four channels left
    (2, 2, 40, (3, 5), (20, 20), False, True, "dense"),                # idle lanes in a group
    (2, 2, 40, (3, 5), (20, 20), True, False, "apart"),
    (1, 4, 128, (33,), (128,), False, True, "apart"),
    (2, 1, 8, (5, 2), (2, 6), True, True, "dense"),
    (2, 2, 80, (4, 4), (0, 24), False, True, "interleaved"),           # an axis without channels
    (2, 2, 64, (4, 4), (6, 8), False, False, "dense"),
    (65, 1, 64, (31, 33), (32, 32), False, True, "dense"),             # several heads and entries to a block
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_matches_the_formula(case, dtype):
    B, h, d, extent, channels, neighbours, norm, kind = CASES[case]
    N, dt = int(torch.tensor(extent).prod()), DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(case)
    q, k = views(kind, B, h, N, d, dt, gen)
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2)] if norm else [None, None]
    eps = 1e-5 if norm else None
    freq = Rotary.frequencies(channels)
    rotary = Rotary(freq, channels, extent, pairs=neighbours)
    mod = AgentAttention(B, h, d, N, 1, dt)
    out = mod.rotate(q, k, rotary, q_gain=gains[0], k_gain=gains[1], eps=eps)
    for got, x, gain in zip(out, (q, k), gains):
        check(got, *reference(x, grid_positions(extent), channels, freq, neighbours, gain, eps), dtype)
    assert mod.last_launch_count() == 1
    # one tensor alone, in place, gives the same bits; the other stays as it is
    k_before = k.clone()
    only, none = mod.rotate(q, None, rotary, q_gain=gains[0], eps=eps, out=(q, None))
    assert none is None and torch.equal(only, out[0]) and torch.equal(k, k_before)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_backward_matches_the_formula(case, dtype):
    B, h, d, extent, channels, neighbours, norm, kind = CASES[case]
    N, dt = int(torch.tensor(extent).prod()), DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(100 + case)
    q, k = views(kind, B, h, N, d, dt, gen)
    grads = views(kind, B, h, N, d, torch.float32, gen)
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2)] if norm else [None, None]
    eps = 1e-5 if norm else None
    freq = Rotary.frequencies(channels)
    mod = AgentAttention(B, h, d, N, 1, dt)
    given = dict(q=q, k=k, q_gain=gains[0], k_gain=gains[1], eps=eps) if norm else {}
    got = mod.rotate_backward(*grads, Rotary(freq, channels, extent, pairs=neighbours), **given)
    for name, x, g, gain in zip("qk", (q, k), grads, gains):
        back = turned(g.double(), grid_positions(extent), channels, freq, neighbours, -1.0)
        if norm:
            xd, w = x.double(), gain.double()
            r = (xd.square().mean(-1, keepdim=True) + eps).rsqrt()
            ref = r * (back * w - xd * r * (back * w * xd * r).mean(-1, keepdim=True))
            terms = back * xd * r
            err = (got[f"d{name}_gain"].double() - terms.sum((0, 1, 2))).abs()
            assert (err <= 4e-6 * terms.abs().sum((0, 1, 2))).all()
        else:
            ref = back
        bound = 4e-6 * torch.maximum(ref.abs(), back.abs() * (r if norm else 1.0)).amax(-1, keepdim=True)
        assert ((got[f"d{name}"].double() - ref).abs() <= bound).all()
    again = mod.rotate_backward(*grads, Rotary(freq, channels, extent, pairs=neighbours), out=grads, **given)      # in place; sums in a fixed order
    assert all(torch.equal(again[n], got[n]) for n in got) and again["dq"] is grads[0]


def test_gradient_against_differences():
    """Central differences of the forward call in fp32: steps of 1e-2 leave 1e-4 of curvature and 1e-4 of rounding (1e-7 of values of one over 1e-2, in a sum)."""
    B, h, d, extent, channels = 2, 2, 32, (3, 4), (16, 16)
    N = 12
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k, wq, wk, tq, tk = (torch.randn((B, h, N, d), generator=gen, device="cuda") for _ in range(6))
    gq, gk, ug, vg = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(4))
    rotary, mod = Rotary(Rotary.frequencies(channels), channels, extent), AgentAttention(B, h, d, N, 1, torch.float32)

    def loss(s):
        a, b = mod.rotate(q + s * tq, k + s * tk, rotary, q_gain=gq + s * ug, k_gain=gk + s * vg, eps=1e-6)
        return float((a.double() * wq).sum() + (b.double() * wk).sum())
    got = mod.rotate_backward(wq, wk, rotary, q=q, k=k, q_gain=gq, k_gain=gk, eps=1e-6)
    slope = sum(float((got[n].double() * t).sum()) for n, t in (("dq", tq), ("dk", tk), ("dq_gain", ug), ("dk_gain", vg)))
    size = float(sum((got[n].double() * t).abs().sum() for n, t in (("dq", tq), ("dk", tk), ("dq_gain", ug), ("dk_gain", vg))))
    assert abs((loss(1e-2) - loss(-1e-2)) / 2e-2 - slope) <= 1e-3 * size


@pytest.mark.parametrize("batch", [1, 3])
def test_given_positions(batch):
    """Fractional, negative and very large positions, shared or an entry's own: a position of 3e5 at one radian a step keeps its accuracy."""
    B, h, d, N, channels = 3, 2, 64, 50, (32, 32)
    gen = torch.Generator(device="cuda").manual_seed(1)
    positions = (torch.rand((batch, N, 2), generator=gen, device="cuda") * 200 - 100)
    positions[0, :2] = torch.tensor([[300001.0, 65535.0], [-70000.25, 0.0]])
    q, k = views("dense", B, h, N, d, torch.float32, gen)
    freq = Rotary.frequencies(channels)
    mod = AgentAttention(B, h, d, N, 1, torch.float32)
    out = mod.rotate(q, k, Rotary(freq, channels, positions=positions))
    for got, x in zip(out, (q, k)):
        check(got, *reference(x, positions.cpu(), channels, freq, False, None, None), "f32")


def test_norm_alone_zero_rows_and_non_finite_values():
    mod = AgentAttention(1, 2, 64, 4, 1, torch.bfloat16)
    x = torch.randn((1, 2, 4, 64), device="cuda").bfloat16()
    x[0, 0, 1] = 0                                        # its norm is 0 / sqrt(eps)
    x[0, 1, 2, 3] = float("inf")
    x[0, 1, 3, 5] = float("nan")
    got, _ = mod.rotate(x, None, eps=1e-6)
    ref = x.double() / (x.double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
    assert (got[0, 0, 1] == 0).all()
    assert torch.isnan(got[0, 1, 2, 3]) and (got[0, 1, 2, :3] == 0).all() and torch.isnan(got[0, 1, 3]).all()
    fine = torch.ones((2, 4), dtype=torch.bool, device="cuda")
    fine[1, 2:] = False
    assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs())[0][fine].all()
    # without a norm what does not turn is handed through as it is, and only a partner of a non-finite value becomes non-finite
    rotary = Rotary(Rotary.frequencies((8,)), (8,), (4,))
    got, _ = mod.rotate(x, None, rotary)
    assert torch.equal(got[..., 8:], x[..., 8:])
    bad = ~torch.isfinite(got[0, 1])
    assert bad[2].nonzero().flatten().tolist() == [3, 7] and bad[3].nonzero().flatten().tolist() == [1, 5] and not bad[:2].any()


def test_other_streams_and_one_tensor_on_two_axes():
    B, h, d, extent, channels = 2, 8, 64, (24, 24), (32, 32)
    mod = AgentAttention(B, h, d, 576, 1, torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k = views("interleaved", B, h, 576, d, torch.bfloat16, gen)
    gq = torch.ones(d, device="cuda").bfloat16()
    g = views("dense", B, h, 576, d, torch.float32, gen)
    rotary = Rotary(Rotary.frequencies(channels), channels, extent)
    want = mod.rotate(q, k, rotary)
    want_b = mod.rotate_backward(*g, rotary, q=q, k=k, q_gain=gq, k_gain=gq, eps=1e-6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mod.rotate(q, k, rotary, stream=side)
    got_b = mod.rotate_backward(*g, rotary, q=q, k=k, q_gain=gq, k_gain=gq, eps=1e-6, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and all(torch.equal(want_b[n], got_b[n]) for n in want_b)


def test_refusals():
    mod = AgentAttention(2, 2, 64, 16, 1, torch.bfloat16)
    q = torch.zeros((2, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    g = torch.zeros((2, 2, 16, 64), device="cuda")
    freq = Rotary.frequencies((32, 32))
    fine = Rotary(freq, (32, 32), (4, 4))
    for bad in (lambda: Rotary(freq, (32, 31), (4, 4)), lambda: Rotary(freq, (32, 32), (16,)), lambda: Rotary(freq[:-1], (32, 32), (4, 4)),
                lambda: Rotary(freq, (32, 32), positions=torch.zeros((1, 16, 3), device="cuda")),
                lambda: mod.rotate(None, None, fine), lambda: mod.rotate(q.float(), None, fine), lambda: mod.rotate(q, q[:, :, :8], fine),
                lambda: mod.rotate(q, None, fine, q_gain=torch.ones(64, device="cuda").bfloat16()),
                lambda: mod.rotate(q, None, fine, q_gain=torch.ones(32, device="cuda").bfloat16(), eps=1e-6),
                lambda: mod.rotate(q, None, Rotary(freq, (32, 32), positions=torch.zeros((1, 15, 2), device="cuda"))),
                lambda: mod.rotate_backward(g, None, fine, eps=1e-6), lambda: mod.rotate_backward(g.bfloat16(), None, fine)):
        with pytest.raises(ValueError):
            bad()

    def status(call):
        with pytest.raises(AgentAttnError) as e:
            call()
        return e.value.status
    assert status(lambda: mod.rotate(q, None, Rotary(freq, (32, 32), (4, 5)))) == 1                        # another token count
    assert status(lambda: mod.rotate(q, None, Rotary(torch.cat([freq, freq]), (64, 64), (4, 4)))) == 1     # more channels than a head has
    assert status(lambda: mod.rotate(q, None, fine, eps=-1.0)) == 1
    assert status(lambda: mod.rotate(q, None, fine, eps=float("nan"))) == 1
    assert status(lambda: mod.rotate(q, q.clone(), fine, out=(torch.empty_like(q), q))) == 1               # a result over the other's input
    long = torch.zeros((2, 2, 17, 64), device="cuda", dtype=torch.bfloat16)
    assert status(lambda: mod.rotate(long, None, Rotary(freq, (32, 32), (1, 17)))) == 2
    odd = torch.zeros((2, 2, 16, 68), device="cuda", dtype=torch.bfloat16)[..., :64]                       # rows that are no multiple of 16 bytes
    assert status(lambda: mod.rotate(odd, None, fine)) == 1
    assert status(lambda: mod.rotate(q.expand(2, 2, 16, 64)[:, :1].expand(2, 2, 16, 64), None, fine)) == 1  # heads on one place
    lib, h = mod.lib, mod._h
    need = int(lib.agent_attn_rotate_workspace_bytes(h))
    small = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
    assert status(lambda: mod.rotate_backward(g, None, fine, q=q, eps=1e-6, workspace=small)) == 3
    assert lib.agent_attn_rotate(h, None, None, None, 16, None, None, None, None, None, None) == 1
    assert lib.agent_attn_rotate(h, q.data_ptr() + 2, None, None, 16, ctypes.byref(fine._c), None, q.data_ptr() + 2, None, None, None) == 1
    assert lib.agent_attn_rotate_backward(h, g.data_ptr(), None, None, None, None, None, 16, None, None, g.data_ptr(), None, None, g.data_ptr(), None,
                                          None, 0, None) == 1                                              # a gain's gradient without a norm
    assert b"gain" in lib.agent_attn_last_error(h)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [24, 40, 48, 56, 72, 80, 88, 104, 120])
def test_heads_whose_lanes_leave_some_of_a_warp_idle(d, dtype):
    """So many rows that a block works on more of them than its ring has stages, with groups of lanes that do not fill a warp: no lane may look past the
    ring.  Halves of segments that are no whole pieces."""
    B, h, extent, dt = 1, 16, (64, 64), DT[dtype]
    N = extent[0] * extent[1]
    gen = torch.Generator(device="cuda").manual_seed(d)
    q, k = views("dense", B, h, N, d, dt, gen)
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2)]
    mod = AgentAttention(B, h, d, N, 1, dt)
    for channels in ((d // 2, d // 2), (d // 2 - 2, d // 2 + 2)):           # partners of 16 bits by words, one by one
        freq = Rotary.frequencies(channels)
        rotary = Rotary(freq, channels, extent)
        for norm in (False, True):
            given = dict(q_gain=gains[0], k_gain=gains[1], eps=1e-5) if norm else {}
            for got, x, gain in zip(mod.rotate(q, k, rotary, **given), (q, k), gains):
                check(got, *reference(x, grid_positions(extent), channels, freq, False, gain if norm else None, 1e-5 if norm else None), dtype)


@pytest.mark.parametrize("norm", [False, True])
def test_offsets_past_32_bits(norm):
    """Batch entries more than 2^32 bytes, and 2^31 elements, apart, in place and back."""
    B, h, d, extent, dt = 2, 2, 64, (16, 8), torch.bfloat16
    N, apart = extent[0] * extent[1], (1 << 31) + 4096
    room = torch.empty(apart + 2 * N * h * d, dtype=dt, device="cuda")
    q, k = (room[i * N * h * d:].as_strided((B, h, N, d), (apart, d, h * d, 1)) for i in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t in (q, k):
        t.copy_(torch.randn((B, h, N, d), generator=gen, device="cuda"))
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2)]
    given = dict(q_gain=gains[0], k_gain=gains[1], eps=1e-5) if norm else {}
    freq = Rotary.frequencies((32, 32))
    mod, rotary = AgentAttention(B, h, d, N, 1, dt), Rotary(freq, (32, 32), extent)
    want = [reference(t.clone(), grid_positions(extent), (32, 32), freq, False, g if norm else None, 1e-5 if norm else None) for t, g in zip((q, k), gains)]
    mod.rotate(q, k, rotary, out=(q, k), **given)
    for got, (ref, size) in zip((q, k), want):
        check(got, ref, size, "bf16")


def gradients(x, g, positions, channels, freq, neighbours, gain, eps):
    """In 64 bits: dX, and the bound of an element's error (head of this file); the gain's gradient, and the sum of its summands' sizes."""
    xd, w = x.double(), 1.0 if gain is None else gain.double()
    back = turned(g.double(), positions, channels, freq, neighbours, -1.0)
    r = (xd.square().mean(-1, keepdim=True) + eps).rsqrt()
    dx = r * (back * w - xd * r * (back * w * xd * r).mean(-1, keepdim=True))
    terms = back * xd * r
    return dx, 4e-6 * torch.maximum(dx.abs(), back.abs() * r).amax(-1, keepdim=True), terms.sum((0, 1, 2)), terms.abs().sum((0, 1, 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("extent,d", [((14, 14), 64), ((1, 1), 64), ((14, 14), 40), ((3, 11), 128), ((1, 5), 8)])
def test_gradients_with_eps_of_zero(extent, d, dtype):
    """No row of the input is zero, so that every gradient is finite; rows past the last token of a tile are no rows."""
    B, h, dt = 2, 3, DT[dtype]
    N, channels = extent[0] * extent[1], (d // 4 * 2, d // 4 * 2)
    gen = torch.Generator(device="cuda").manual_seed(d + N)
    x, g = views("interleaved", B, h, N, d, dt, gen), views("dense", B, h, N, d, torch.float32, gen)
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2)]
    freq = Rotary.frequencies(channels)
    mod, rotary = AgentAttention(B, h, d, N, 1, dt), Rotary(freq, channels, extent)
    got = mod.rotate_backward(*g, rotary, q=x[0], k=x[1], q_gain=gains[0], k_gain=gains[1], eps=0.0)
    for i, n in enumerate("qk"):
        dx, bound, dgain, size = gradients(x[i], g[i], grid_positions(extent), channels, freq, False, gains[i], 0.0)
        assert ((got[f"d{n}"].double() - dx).abs() <= bound).all()
        assert ((got[f"d{n}_gain"].double() - dgain).abs() <= 4e-6 * size).all()
    for i, out in enumerate(mod.rotate(*x, rotary, q_gain=gains[0], k_gain=gains[1], eps=0.0)):
        check(out, *reference(x[i], grid_positions(extent), channels, freq, False, gains[i], 0.0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("channels,neighbours", [((16,), False), ((12,), False), ((8, 16), False), ((6, 8), True), ((0, 16), False)])
def test_non_finite_positions_reach_their_axis_alone(channels, neighbours, dtype):
    """A token whose position on an axis is infinite or NaN: the channels of that axis are lost; those of the others and those past the segments are not, nor
    is any other token."""
    B, h, d, N, axes = 2, 2, 64, 9, len(channels)
    gen = torch.Generator(device="cuda").manual_seed(5)
    positions = torch.rand((1, N, axes), generator=gen, device="cuda") * 20
    fine = positions.clone()
    positions[0, 2, 0], positions[0, 7, axes - 1] = float("inf"), float("nan")
    q, k = views("dense", B, h, N, d, DT[dtype], gen)
    g = views("dense", B, h, N, d, torch.float32, gen)
    freq = Rotary.frequencies(channels)
    mod = AgentAttention(B, h, d, N, 1, DT[dtype])
    lost = torch.zeros((N, d), dtype=torch.bool, device="cuda")
    lost[2, :channels[0]], lost[7, sum(channels[:-1]):sum(channels)] = True, True
    bad, good = (Rotary(freq, channels, positions=p, pairs=neighbours) for p in (positions, fine))
    for given in ({}, {"eps": 1e-5}):
        for got, want in zip(mod.rotate(q, k, bad, **given), mod.rotate(q, k, good, **given)):
            assert torch.equal(got[:, :, ~lost], want[:, :, ~lost]) and torch.isnan(got[:, :, lost]).all()
    for got, want in zip(mod.rotate_backward(*g, bad).values(), mod.rotate_backward(*g, good).values()):
        assert torch.equal(got[:, :, ~lost], want[:, :, ~lost]) and torch.isnan(got[:, :, lost]).all()
    # a norm's gradient takes the whole row with it
    row = lost.any(1)
    got, want = (mod.rotate_backward(*g, r, q=q, k=k, eps=1e-5) for r in (bad, good))
    for n in got:
        assert torch.equal(got[n][:, :, ~row], want[n][:, :, ~row]) and torch.isnan(got[n][:, :, row]).all()


def test_axes_past_what_fp32_counts_are_refused():
    """An odd coordinate past 2^24 is no fp32 number; up to there every token has its own angle, the last one too."""
    N, d = (1 << 24) + 2, 8
    mod, freq = AgentAttention(1, 1, d, N, 1, torch.bfloat16), torch.ones(1, device="cuda")
    q = torch.ones((1, 1, N, d), dtype=torch.bfloat16, device="cuda")
    for extent, channels in (((N,), (2,)), ((1, N), (0, 2))):
        with pytest.raises(AgentAttnError) as e:
            mod.rotate(q, None, Rotary(freq, channels, extent))
        assert e.value.status == 2
    with pytest.raises(AgentAttnError) as e:
        mod.rotate_backward(q.float(), None, Rotary(freq, (2,), (N,)))
    assert e.value.status == 2
    last = 1 << 24
    got, _ = mod.rotate(q[:, :, :last], None, Rotary(freq, (2,), (last,)))
    t = torch.arange(last - 100, last, dtype=torch.float64, device="cuda")
    assert ((got[0, 0, -100:, 0].double() - (t.cos() - t.sin())).abs() <= 2.0 ** -8 * 1.5).all()
    two = mod.rotate(q, None, Rotary(torch.ones(2, device="cuda"), (2, 2), (2, N // 2)))[0]        # two axes have room for more
    t = torch.tensor([N // 2 - 1], dtype=torch.float64, device="cuda")
    assert ((two[0, 0, -1, 2].double() - (t.cos() - t.sin())).abs() <= 2.0 ** -8 * 1.5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("N,d,neighbours", [(50, 64, False), (129, 40, True), (7, 128, False)])
def test_norms_and_gradients_over_given_positions(N, d, neighbours, own, dtype):
    """Positions of all entries, or each entry's own: runs of a block that go from one entry to the next change their angles there, in both directions."""
    B, h, channels, eps = 5, 3, (d // 4 * 2, d // 4 * 2), 1e-5
    gen = torch.Generator(device="cuda").manual_seed(N + d)
    positions = torch.rand((B if own else 1, N, 2), generator=gen, device="cuda") * 200 - 100
    x, g = views("interleaved", B, h, N, d, DT[dtype], gen), views("apart", B, h, N, d, torch.float32, gen)
    gains = [(1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(DT[dtype]) for _ in range(2)]
    freq = Rotary.frequencies(channels)
    mod, rotary = AgentAttention(B, h, d, N, 1, DT[dtype]), Rotary(freq, channels, positions=positions, pairs=neighbours)
    at = positions.cpu()
    for i, out in enumerate(mod.rotate(*x, rotary, q_gain=gains[0], k_gain=gains[1], eps=eps)):
        check(out, *reference(x[i], at, channels, freq, neighbours, gains[i], eps), dtype)
    got = mod.rotate_backward(*g, rotary, q=x[0], k=x[1], q_gain=gains[0], k_gain=gains[1], eps=eps)
    bare = mod.rotate_backward(*g, rotary)
    for i, n in enumerate("qk"):
        dx, bound, dgain, size = gradients(x[i], g[i], at, channels, freq, neighbours, gains[i], eps)
        assert ((got[f"d{n}"].double() - dx).abs() <= bound).all()
        assert ((got[f"d{n}_gain"].double() - dgain).abs() <= 4e-6 * size).all()
        check(bare[f"d{n}"], turned(g[i].double(), at, channels, freq, neighbours, -1.0), reference(g[i], at, channels, freq, neighbours, None, None)[1], "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_keys_alone_and_norms_without_gains(neighbours, dtype):
    """One tensor has the results that it has beside the other one.  (A gain's sum is shared out to other blocks then: inside its bound.)"""
    B, h, d, extent, channels, eps = 3, 2, 64, (9, 13), (20, 20), 1e-5
    N = extent[0] * extent[1]
    gen = torch.Generator(device="cuda").manual_seed(11)
    x, g = views("dense", B, h, N, d, DT[dtype], gen), views("interleaved", B, h, N, d, torch.float32, gen)
    gain = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(DT[dtype])
    freq = Rotary.frequencies(channels)
    mod, rotary = AgentAttention(B, h, d, N, 1, DT[dtype]), Rotary(freq, channels, extent, pairs=neighbours)
    for given in ({}, {"eps": eps}, {"eps": eps, "k_gain": gain}):
        both, alone = mod.rotate(*x, rotary, **given), mod.rotate(None, x[1], rotary, **given)
        assert alone[0] is None and torch.equal(alone[1], both[1])
        norm = "eps" in given
        ins = dict(q=x[0], k=x[1]) if norm else {}
        both, alone = mod.rotate_backward(*g, rotary, **ins, **given), mod.rotate_backward(None, g[1], rotary, k=x[1], **given)
        assert set(alone) == {"dk"} | ({"dk_gain"} if "k_gain" in given else set()) and torch.equal(alone["dk"], both["dk"])
        if not norm:
            continue
        for i, n in enumerate("qk"):
            dx, bound, dgain, size = gradients(x[i], g[i], grid_positions(extent), channels, freq, neighbours, given.get(f"{n}_gain"), eps)
            assert ((both[f"d{n}"].double() - dx).abs() <= bound).all()
        if "k_gain" in given:
            assert all(((t["dk_gain"].double() - dgain).abs() <= 4e-6 * size).all() for t in (both, alone))


def test_non_finite_gradients_stay_in_their_row():
    """An infinity or a NaN in the gradient of a result: its row of dX, and in the gain's gradient the two channels of its pair."""
    B, h, d, extent, channels, eps = 2, 2, 64, (5, 7), (32, 32), 1e-5
    N = 35
    for dtype in ("f32", "bf16"):
        gen = torch.Generator(device="cuda").manual_seed(12)
        x, g = views("dense", B, h, N, d, DT[dtype], gen), views("dense", B, h, N, d, torch.float32, gen)
        gain = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(DT[dtype])
        freq = Rotary.frequencies(channels)
        mod, rotary = AgentAttention(B, h, d, N, 1, DT[dtype]), Rotary(freq, channels, extent)
        dx, bound, dgain, size = gradients(x[0], g[0], grid_positions(extent), channels, freq, False, gain, eps)
        for value in (float("inf"), float("nan")):
            bad = g[0].clone()
            bad[1, 0, 11, 37] = value                        # of the pair 37, 53
            got = mod.rotate_backward(bad, g[1], rotary, q=x[0], k=x[1], q_gain=gain, k_gain=gain, eps=eps)
            rows, cols = torch.ones((B, h, N), dtype=torch.bool, device="cuda"), torch.ones(d, dtype=torch.bool, device="cuda")
            rows[1, 0, 11], cols[[37, 53]] = False, False
            assert not got["dq"][1, 0, 11].isfinite().any() and ((got["dq"].double() - dx).abs() <= bound)[rows].all()
            assert not got["dq_gain"][~cols].isfinite().any() and ((got["dq_gain"].double() - dgain).abs() <= 4e-6 * size)[cols].all()
            assert got["dk"].isfinite().all() and got["dk_gain"].isfinite().all()


@pytest.mark.parametrize("norm", [False, True])
def test_gradients_at_offsets_past_32_bits(norm):
    """Batch entries 2^31 elements apart, of the gradients (8 GB) and of the inputs, in place."""
    B, h, d, extent, channels, eps = 2, 2, 64, (16, 8), (32, 32), 1e-5
    N, apart = 128, (1 << 31) + 4096
    gen = torch.Generator(device="cuda").manual_seed(13)

    def far(dtype):
        room = torch.empty(apart + 2 * N * h * d, dtype=dtype, device="cuda")
        got = [room[i * N * h * d:].as_strided((B, h, N, d), (apart, d, h * d, 1)) for i in range(2)]
        for t in got:
            t.copy_(torch.randn((B, h, N, d), generator=gen, device="cuda"))
        return got
    g = far(torch.float32)
    x = far(torch.bfloat16) if norm else [None, None]
    freq = Rotary.frequencies(channels)
    mod, rotary = AgentAttention(B, h, d, N, 1, torch.bfloat16), Rotary(freq, channels, extent)
    if norm:
        gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        want = [gradients(a.clone(), b.clone(), grid_positions(extent), channels, freq, False, gain, eps) for a, b in zip(x, g)]
        got = mod.rotate_backward(*g, rotary, q=x[0], k=x[1], q_gain=gain, k_gain=gain, eps=eps, out=g)
        for n, t, (dx, bound, dgain, size) in zip("qk", g, want):
            assert ((t.double() - dx).abs() <= bound).all() and ((got[f"d{n}_gain"].double() - dgain).abs() <= 4e-6 * size).all()
    else:
        want = [(turned(t.double(), grid_positions(extent), channels, freq, False, -1.0), reference(t.clone(), grid_positions(extent), channels, freq, False, None, None)[1]) for t in g]
        mod.rotate_backward(*g, rotary, out=g)
        for t, (dx, size) in zip(g, want):
            check(t, dx, size, "f32")


def test_token_counts_that_32_bits_hold_but_not_their_tiles():
    """Refused before anything is launched: the pointers are of one token."""
    N = (1 << 31) - 100
    mod = AgentAttention(1, 1, 8, N, 1, torch.bfloat16)
    q, g = torch.zeros(8, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, device="cuda")
    ws = torch.empty(int(mod.lib.agent_attn_rotate_workspace_bytes(mod._h)), dtype=torch.uint8, device="cuda")
    norm = mod._norm(None, None, 1e-6)
    assert mod.lib.agent_attn_rotate(mod._h, q.data_ptr(), None, None, N, None, norm, q.data_ptr(), None, None, None) == 2
    assert mod.lib.agent_attn_rotate_backward(mod._h, g.data_ptr(), None, None, q.data_ptr(), None, None, N, None, norm, g.data_ptr(), None, None, None, None,
                                              ws.data_ptr(), ws.numel(), None) == 2
    assert b"32 bits" in mod.lib.agent_attn_last_error(mod._h)
