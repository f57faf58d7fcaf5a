"""Softmax attention over whole sequences and its gradient, against the formulas in 64 bits on the same inputs.

Bounds, element by element, u = half a step of the type (2^-8 bf16, 2^-11 f16, 2^-24 f32):
    result     u |o| (its rounding) + u sum p |v| (that of the probabilities, or of what an online softmax leaves in them) + e sum p |v|
    dV         u |dv| + (u + e) sum p |dO|
    dQ, dK     u |dq| + scale sum (|dS| (u + e) + p (u sum |dO O| + e (|dP| + |D|))) |k|: the rounding of dS, D out of a rounded result
e is the arithmetic in 32 bits: logits are sums of d products (their own rounding and that of the sum: 2^-23 of the products' magnitudes as a rule, which the
reference takes along), exponentials 2^-22, sums cut off 2^-23 of themselves every 16 summands on the tensor cores (2^-24 half of the time; at most 128
steps before they leave it in fp32, 1024 here in 16 bits).
"""
import pytest
import torch

from paper_2312_08874_b200 import AgentAttention, AgentAttnError

pytestmark = pytest.mark.gpu
BF, FH, F32 = torch.bfloat16, torch.float16, torch.float32


def u_of(t):
    return torch.finfo(t).eps / 2


def reference(q, k, v, causal, scale, do=None):
    """One sequence and head in 64 bits: result, log-sum-exp and bound's parts; with do the gradients."""
    q, k, v = q.double(), k.double(), v.double()
    n, m = q.shape[0], k.shape[0]
    s = q @ k.T * scale
    size = q.abs() @ k.abs().T * scale                          # what the logits' sums are made of
    if causal:
        seen = torch.arange(m, device=q.device)[None] <= torch.arange(n, device=q.device)[:, None] + m - n
    else:
        seen = torch.ones((n, m), dtype=torch.bool, device=q.device)
    some = seen.any(1, keepdim=True)
    s = s.masked_fill(~seen, -float("inf"))
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(some, lse[:, None], torch.zeros_like(lse[:, None]))), torch.zeros_like(s))
    r = {"o": p @ v, "lse": lse, "p": p, "size": torch.where(seen, size, torch.zeros_like(size)), "some": some}
    r["top"] = torch.cat([r["size"], torch.zeros_like(lse[:, None])], 1).amax(1)
    if do is not None:
        do = do.double()
        dp = do @ v.T
        d = (do * r["o"]).sum(1, keepdim=True)
        ds = p * (dp - d) * scale
        r.update(dq=ds @ k, dk=ds.T @ q, dv=p.T @ do, dp=do.abs() @ v.abs().T, d=(do.abs() * (p @ v.abs())).sum(1, keepdim=True), ds=ds, do=do)
    return r


def spans(q, k, q_offsets, k_offsets, q_lengths, k_lengths):
    if q_offsets is None:
        return [(b, 0, q.shape[2] if q_lengths is None else q_lengths[b], 0, k.shape[2] if k_lengths is None else k_lengths[b]) for b in range(q.shape[0])]
    return [(0, a, b - a, c, d - c) for a, b, c, d in zip(q_offsets, q_offsets[1:], k_offsets, k_offsets[1:])]


def check(q, k, v, causal=False, scale=None, q_offsets=None, k_offsets=None, q_lengths=None, k_lengths=None, grad=True, do=None, what=""):
    B, h, N, d = q.shape
    kv, M, dt = k.shape[1], k.shape[2], q.dtype
    u = u_of(dt)
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    args = dict(causal=causal, scale=scale, q_offsets=ints(q_offsets), k_offsets=ints(k_offsets), q_lengths=ints(q_lengths), k_lengths=ints(k_lengths))
    if k_offsets is None:
        k_offsets = q_offsets
    mod = AgentAttention(B, h, d, max(N, M), 1, dt)
    out, lse = mod.attend(q, k, v, need_lse=True, **args)
    assert out.shape == q.shape and torch.equal(mod.attend(q, k, v, **args), out), what
    g = None
    if grad:
        gen = torch.Generator(device="cuda").manual_seed(7)
        do = torch.randn(q.shape, generator=gen, device="cuda").to(dt) if do is None else do
        g = mod.attend_backward(q, k, v, out, lse, do, **args)
        again = mod.attend_backward(q, k, v, out, lse, do, **args)
        assert all(torch.equal(g[n], again[n]) for n in g), what
    assert mod.query_status() == 0
    sc = d ** -0.5 if scale is None else scale
    row_q, row_k = torch.zeros((B, N), dtype=torch.bool), torch.zeros((B, M), dtype=torch.bool)
    for b, q0, n, k0, m in spans(q, k, q_offsets, k_offsets, q_lengths, k_lengths):
        row_q[b, q0:q0 + n] = True
        row_k[b, k0:k0 + m] = True
        steps = 2.0 ** -24 * min(m / 16 + 8, 128 if dt is F32 else 4096)
        for hk in range(kv):
            sums = [torch.zeros((m, d), dtype=torch.float64, device="cuda") for _ in range(4)]
            for hq in range(hk * (h // kv), (hk + 1) * (h // kv)):
                rq = slice(q0, q0 + n)
                kk, vv = k[b, hk, k0:k0 + m], v[b, hk, k0:k0 + m]
                r = reference(q[b, hq, rq], kk, vv, causal, sc, do[b, hq, rq] if grad else None)
                e = 2.0 ** -21 + steps + 2.0 ** -22 * r["size"]                    # of a probability, relative
                pe = r["p"] * (e + (e * r["p"]).sum(1, keepdim=True))
                va = vv.double().abs()
                bound = u * (r["o"].abs() + r["p"] @ va) + pe @ va + 1e-7 * (dt is FH)
                err = (out[b, hq, rq].double() - r["o"]).abs()
                assert (err <= bound).all(), (what, "o", b, hq, float((err / bound).max()))
                ls, want = lse[b, hq, rq].double(), r["lse"]
                fin = r["some"][:, 0]
                assert torch.equal(ls[~fin], want[~fin])
                assert ((ls - want).abs()[fin] <= (2.0 ** -21 + steps + 2.0 ** -22 * r["top"] + 2.0 ** -23 * want.abs())[fin]).all(), (what, "lse")
                if not grad:
                    continue
                ka, qa = kk.double().abs(), q[b, hq, rq].double().abs()
                dsb = r["ds"].abs() * (u + e) + sc * r["p"] * (u * (r["do"].abs() * r["o"].abs()).sum(1, keepdim=True) * (dt is not F32) + (2 * e + 2 * u * (dt is F32)) * (r["dp"] + r["d"]))
                # f16: P is held times 2^15 and dP - D times a power of two that brings 2 max |dO| max |v| to at least 2^14 (dQ: of the row's dO, so of no
                # more): half a step of the smallest f16 numbers, 2^-25, is 2^-40 of P and at most 2^-25 2^-14 2 max |dO| max |v| of dS / scale
                most_do = do[b, hk * (h // kv):(hk + 1) * (h // kv), rq].double().norm(dim=-1).max() if n else 0.0
                held = (dt is FH) * 2.0 ** -38 * most_do * (vv.double().norm(dim=-1).max() if m else 0.0)
                dsb = dsb + sc * held * (r["p"] > 0)
                low = 3e-8 * (dt is FH)                                            # (half a step of the smallest f16 numbers)
                err, bound = (g["dq"][b, hq, rq].double() - r["dq"]).abs(), u * r["dq"].abs() + dsb @ ka + low
                assert (err <= bound).all(), (what, "dq", b, hq, float((err / bound).max()))
                for i, t in enumerate((r["dk"], dsb.T @ qa, r["dv"], (r["p"] * (u + 2 * e) + 2.0 ** -40 * (dt is FH)).T @ r["do"].abs())):
                    sums[i] += t
            if grad:
                for name, want, more in (("dk", sums[0], sums[1]), ("dv", sums[2], sums[3])):
                    err, bound = (g[name][b, hk, k0:k0 + m].double() - want).abs(), u * want.abs() + more + low
                    assert (err <= bound).all(), (what, name, b, hk, float((err / bound).max()))
    # rows of no sequence: zero in new results
    assert (out.transpose(1, 2)[~row_q.cuda()] == 0).all()
    if grad:
        assert (g["dq"].transpose(1, 2)[~row_q.cuda()] == 0).all() and all((g[n].transpose(1, 2)[~row_k.cuda()] == 0).all() for n in ("dk", "dv"))
    return out, lse, g


def make(B, h, kv, N, M, d, dt, seed=0, std=1.5, fused=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    if fused:
        x = rand(B, N, h + 2 * kv, d)
        x[:, :, :h] *= std
        return tuple(t.permute(0, 2, 1, 3) for t in x.to(dt).split([h, kv, kv], 2))
    return (rand(B, h, N, d) * std).to(dt), rand(B, kv, M, d).to(dt), rand(B, kv, M, d).to(dt)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,h,kv,N,M,d", [(1, 1, 1, 1, 1, 64), (2, 3, 3, 196, 196, 64), (1, 2, 1, 129, 257, 128), (1, 4, 2, 127, 63, 40), (2, 2, 2, 300, 300, 32),
                                          (1, 8, 1, 33, 700, 96), (1, 2, 2, 256, 256, 8), (1, 6, 2, 513, 129, 80), (3, 1, 1, 2, 3, 128), (1, 2, 2, 640, 641, 120)])
def test_dense(dt, causal, B, h, kv, N, M, d):
    check(*make(B, h, kv, N, M, d, dt), causal=causal)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("h,kv,d", [(2, 2, 64), (4, 1, 128), (3, 1, 40)])
def test_packed(dt, causal, h, kv, d):
    """Sequences of 0, 1 and up to 500 tokens, one with queries and no keys and one the other way round, rows before the first and behind the last."""
    lengths = [3, 128, 0, 1, 500, 255, 2, 129]
    at = [5]
    for n in lengths:
        at.append(at[-1] + n)
    N = at[-1] + 77
    q, k, v = make(1, h, kv, N, N, d, dt, fused=True)
    check(q, k, v, causal=causal, q_offsets=at)
    keys = [10, 0, 40, 1, 200, 300, 130, 129]
    ak = [0]
    for n in keys:
        ak.append(ak[-1] + n)
    q, k, v = make(1, h, kv, N, ak[-1] + 3, d, dt, seed=1)
    check(q, k, v, causal=causal, q_offsets=at, k_offsets=ak)


@pytest.mark.parametrize("dt", [BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("h,kv,d", [(2, 1, 64), (2, 2, 128)])
def test_long_packed_sequences(dt, causal, h, kv, d):
    """At least 512 rows a sequence on average, where the gradient's blocks take tiles by their work; empty and very short ones among them, more and fewer keys than queries."""
    def offsets(lengths):
        at = [2]
        for n in lengths:
            at.append(at[-1] + n)
        return at
    at = offsets([700, 0, 1500, 3, 900, 1, 640])
    q, k, v = make(1, h, kv, at[-1] + 9, at[-1] + 9, d, dt, fused=True)
    check(q, k, v, causal=causal, q_offsets=at)
    ak = offsets([1300, 40, 600, 0, 901, 1, 1024])
    q, k, v = make(1, h, kv, at[-1] + 9, ak[-1] + 9, d, dt, seed=1)
    check(q, k, v, causal=causal, q_offsets=at, k_offsets=ak)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("h,kv,d,N", [(8, 2, 128, 1), (4, 4, 64, 1), (2, 1, 40, 3), (24, 1, 64, 1), (4, 1, 128, 5), (2, 2, 64, 16), (1, 1, 32, 40)])
def test_few_queries_over_caches(dt, h, kv, d, N):
    """Caches of different fill, an empty and a short one among them, rows behind the fill not finite."""
    M, fill = 5000, [5000, 0, N, 1, 1025, 4097]
    q, k, v = make(len(fill), h, kv, N, M, d, dt)
    for b, n in enumerate(fill):
        k[b, :, n:] = float("nan")
        v[b, :, n:] = float("inf")
    for causal in (True, False):
        check(q, k, v, causal=causal, k_lengths=fill, grad=False)


@pytest.mark.parametrize("dt", [F32, BF, FH])
def test_padded_batch(dt):
    nq, nk = [200, 1, 0, 131, 77], [200, 260, 30, 0, 78]
    q, k, v = make(5, 4, 2, 200, 260, 64, dt)
    for b in range(5):
        q[b, :, nq[b]:] = float("nan")
        k[b, :, nk[b]:] = float("inf")
        v[b, :, nk[b]:] = float("nan")
    do = torch.randn(q.shape, device="cuda").to(dt)
    for b in range(5):
        do[b, :, nq[b]:] = float("nan")
    for causal in (False, True):
        check(q, k, v, causal=causal, q_lengths=nq, k_lengths=nk, do=do)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("d", [64, 128])
def test_neighbours_are_not_read_into_a_sequence(dt, d):
    """A sequence of NaNs between two others, at offsets that are no multiple of a tile."""
    at = [0, 70, 215, 400]
    q, k, v = make(1, 2, 1, 400, 400, d, dt, fused=True)
    mod = AgentAttention(1, 2, d, 400, 1, dt)
    o = torch.tensor(at, dtype=torch.int32, device="cuda")
    do = torch.randn(q.shape, device="cuda").to(dt)
    for causal in (False, True):
        want, lse = mod.attend(q, k, v, causal=causal, q_offsets=o, need_lse=True)
        g = mod.attend_backward(q, k, v, want, lse, do, causal=causal, q_offsets=o)
        q2, k2, v2, do2 = (t.clone() for t in (q, k, v, do))
        for t in (q2, k2, v2, do2):
            t[:, :, 70:215] = float("nan")
        got, lse2 = mod.attend(q2, k2, v2, causal=causal, q_offsets=o, need_lse=True)
        g2 = mod.attend_backward(q2, k2, v2, got, lse2, do2, causal=causal, q_offsets=o)
        for a, b in ((want, got), *((g[n], g2[n]) for n in g)):
            assert torch.equal(a[:, :, :70], b[:, :, :70]) and torch.equal(a[:, :, 215:], b[:, :, 215:])
            assert b[:, :, 70:215].isnan().all()


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("N,M,d", [(300, 300, 64), (200, 333, 128), (9, 2000, 64)])
def test_values_that_are_not_finite_reach_the_queries_that_see_them(dt, N, M, d):
    q, k, v = make(1, 2, 2, N, M, d, dt)
    mod = AgentAttention(1, 2, d, max(N, M), 1, dt)
    want = mod.attend(q, k, v, causal=True)
    j = M - N + N // 2                                                   # its first reader is query N // 2
    for bad in (float("nan"), float("inf")):
        v2, k2 = v.clone(), k.clone()
        v2[0, 0, j, 5] = bad
        k2[0, 1, j, 3] = float("nan")
        got = mod.attend(q, k2, v2, causal=True)
        assert torch.equal(got[:, :, :N // 2], want[:, :, :N // 2])
        assert torch.equal(got[0, 0, :, :5], want[0, 0, :, :5]) and torch.equal(got[0, 0, :, 6:], want[0, 0, :, 6:])
        assert not got[0, 0, N // 2:, 5].isfinite().any() and got[0, 1, N // 2:].isnan().all()


@pytest.mark.parametrize("dt", [F32, BF, FH])
def test_large_and_equal_logits(dt):
    """Logits of some 200: weights of one key; equal keys: weights that are exactly even."""
    q, k, v = make(1, 2, 2, 130, 260, 64, dt, std=16.0)
    check(q, k * 1.5, v)
    out = AgentAttention(1, 2, 64, 260, 1, dt).attend(q, k[:, :, :1].expand(1, 2, 260, 64).contiguous(), v)
    assert (out.double() - v.double().mean(2, keepdim=True)).abs().max() <= u_of(dt) * 2 + 1e-5


@pytest.mark.parametrize("dt", [F32, BF, FH])
def test_scale_and_strides(dt):
    """Heads first, tokens first, batch inside the tokens; results into views."""
    B, h, kv, N, d = 2, 4, 2, 150, 64
    q, k, v = make(B, h, kv, N, N, d, dt)
    q2 = q.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)          # [heads][B][N][d]
    k2 = k.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)          # [N][B][heads][d]
    v2 = torch.zeros((B, kv, N, d + 40), device="cuda").to(dt)[..., 8:8 + d]
    v2.copy_(v)
    out, lse, g = check(q2, k2, v2, causal=True, scale=0.3)
    mod = AgentAttention(B, h, d, N, 1, dt)
    wide = torch.full((B, N, h + 3, d), 5.0, device="cuda").to(dt)
    view = wide[:, :, 1:1 + h].permute(0, 2, 1, 3)
    assert mod.attend(q2, k2, v2, causal=True, scale=0.3, out=view) is view and torch.equal(view, out)
    assert (wide[:, :, 0] == 5).all() and (wide[:, :, 1 + h:] == 5).all()
    fused = torch.full((B, N, h + 2 * kv, d), 5.0, device="cuda").to(dt)
    views = [t.permute(0, 2, 1, 3) for t in fused.split([h, kv, kv], 2)]
    do = torch.randn((B, N, h, d), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").to(dt).permute(0, 2, 1, 3)
    dense = mod.attend_backward(q, k, v, out, lse, do.contiguous(), causal=True, scale=0.3)
    mod.attend_backward(q2, k2, v2, out, lse, do, causal=True, scale=0.3, grads=views)
    assert all(torch.equal(a, dense[n]) for a, n in zip(views, ("dq", "dk", "dv")))


def test_rows_of_no_sequence_stay_as_they_are():
    for dt in (F32, BF):
        q, k, v = make(1, 2, 2, 300, 300, 64, dt)
        mod = AgentAttention(1, 2, 64, 300, 1, dt)
        o = torch.tensor([10, 140, 140, 290], dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 3.0)
        _, lse = mod.attend(q, k, v, q_offsets=o, out=out, need_lse=True)
        grads = [torch.full_like(t, 3.0) for t in (q, k, v)]
        mod.attend_backward(q, k, v, out, lse, q, q_offsets=o, grads=grads)
        for t in [out] + grads:
            assert (t[:, :, :10] == 3).all() and (t[:, :, 290:] == 3).all() and (t[:, :, 10:290] != 3).any(-1).all()


@pytest.mark.parametrize("dt,few", [(F32, False), (BF, False), (FH, False), (BF, True)])
def test_gradient_against_differences(dt, few):
    """d(sum w o) along a direction, from the 64-bit formulas' difference: the gradient of what is computed, not only of the same formulas."""
    N, M, d = (2, 90, 64) if few else (70, 90, 64)
    q, k, v = make(1, 4, 2, N, M, d, dt, seed=3)
    w = torch.randn(q.shape, device="cuda").to(dt)
    mod = AgentAttention(1, 4, d, M, 1, dt)
    out, lse = mod.attend(q, k, v, causal=True, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, w, causal=True)

    def value(q, k, v):
        return sum((reference(q[0, i], k[0, i // 2], v[0, i // 2], True, d ** -0.5)["o"] * w[0, i].double()).sum() for i in range(4))
    for i, t in enumerate((q, k, v)):
        step = torch.randn(t.shape, device="cuda").double()
        args = [x.double() for x in (q, k, v)]
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * step, args[i] - 1e-5 * step
        slope, got = (value(*up) - value(*down)) / 2e-5, (g[("dq", "dk", "dv")[i]].double() * step).sum()
        # n independent errors of 2 u of the gradient's size each
        assert abs(slope - got) <= 6 * 2 * max(u_of(dt), 2e-6) * (g[("dq", "dk", "dv")[i]].double() * step).norm() + 1e-4


def test_small_gradients_in_f16():
    """Gradients around 1e-6 of the values: P and dS of a few times 1e-9 keep their bits."""
    q, k, v = make(1, 2, 1, 2000, 2000, 64, FH)
    do = (torch.randn(q.shape, device="cuda") * 64).half()
    mod = AgentAttention(1, 2, 64, 2000, 1, FH)
    out, lse = mod.attend(q, k, v, need_lse=True)
    big = mod.attend_backward(q, k, v, out, lse, do)
    small = mod.attend_backward(q, k, v, out, lse, do / 4096)            # (exact: a power of two of normal numbers)
    for n in big:
        a, b = big[n].double(), small[n].double() * 4096
        assert (a - b).norm() <= 1e-3 * a.norm() + 4096 * 3e-8 * a.numel() ** 0.5, n
    check(q, k, v, do=do)


@pytest.mark.parametrize("dt,d", [(F32, 12), (F32, 100), (BF, 24), (FH, 104), (BF, 56), (FH, 72)])
def test_head_sizes(dt, d):
    q, k, v = make(1, 4, 2, 150, 270, d, dt)
    check(q, k, v, causal=True)
    check(q[:, :, :2].contiguous(), k, v, grad=False)


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("d", [64, 128])
def test_sequences_of_one_to_a_few_keys(dt, d):
    """One key: a weight of one, whatever its logit, so exactly no gradient of queries and keys.  A few keys: slopes are differences of a few numbers, which keep the
    accuracy of theirs: two roundings (of dS and the result), each 0.44 u in the 2-norm, so 0.62 u, with room for chance 0.8 u."""
    lengths = [1, 1, 2, 2, 3, 1, 4, 2, 3, 5] * 20
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    q, k, v = make(1, 4, 2, at[-1], at[-1], d, dt, fused=True)
    mod = AgentAttention(1, 4, d, at[-1], 1, dt)
    o = torch.tensor(at, dtype=torch.int32, device="cuda")
    do = torch.randn(q.shape, device="cuda").to(dt)
    out, lse = mod.attend(q, k, v, q_offsets=o, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, do, q_offsets=o)
    want = {n: torch.zeros(t.shape, dtype=torch.float64, device="cuda") for n, t in (("dq", q), ("dk", k), ("dv", v))}
    for a, b in zip(at, at[1:]):
        for h in range(4):
            r = reference(q[0, h, a:b], k[0, h // 2, a:b], v[0, h // 2, a:b], False, d ** -0.5, do[0, h, a:b])
            want["dq"][0, h, a:b] = r["dq"]
            want["dk"][0, h // 2, a:b] += r["dk"]
            want["dv"][0, h // 2, a:b] += r["dv"]
        if b - a == 1:
            assert (g["dq"][:, :, a] == 0).all() and (g["dk"][:, :, a] == 0).all()
            # p = 1 within 2^-23, the same in the result's sum and its weights'; what is left are the roundings of p v, 1 / sum and their product, 2^-24 each and below half a
            # step of a 16-bit type
            value = v[0, :, a].repeat_interleave(2, 0)
            assert torch.equal(out[0, :, a], value) if dt is not F32 else ((out[0, :, a] - value).abs() <= 2.0 ** -22 * value.abs()).all()
    for n in g:
        rel = (g[n].double() - want[n]).norm() / want[n].norm()
        assert rel <= (0.8 * u_of(dt) if dt is not F32 else 4e-7), (n, float(rel))


def test_long_axis():
    """Offsets of a fused projection past 2^31 bytes and 2^31 elements (in halves), one query at the far end and keys all over."""
    d, M = 64, (1 << 25) + 17
    k = torch.zeros((1, 1, M, d), dtype=BF, device="cuda")
    v = torch.zeros((1, 1, M, d), dtype=BF, device="cuda")
    q = torch.ones((1, 1, 1, d), dtype=BF, device="cuda")
    k[0, 0, -1] = 8.0                                                   # logit 64 against 0: weight e^64 of 2^25
    v[0, 0, -1] = 1.0
    mod = AgentAttention(1, 1, d, M, 1, BF)
    out, lse = mod.attend(q, k, v, causal=True, need_lse=True)
    assert (out == 1).all() and abs(float(lse) - 64) <= 1e-4
    q = torch.ones((1, 1, 300, d), dtype=BF, device="cuda")
    out, lse = mod.attend(q, k, v, causal=True, need_lse=True)
    assert (out[0, 0, -1] == 1).all() and (out[0, 0, :-1] == 0).all()


def test_two_streams_and_graphs():
    """Calls on streams of their own, with buffers of their own; two captured calls with other offsets at the replay."""
    q, k, v = make(1, 4, 2, 700, 700, 64, BF)
    mod = AgentAttention(1, 4, 64, 700, 1, BF)
    o = torch.tensor([0, 100, 700], dtype=torch.int32, device="cuda")
    do = torch.randn(q.shape, device="cuda").to(BF)
    want = {}
    for cut in (100, 333):
        o[1] = cut
        want[cut] = mod.attend(q, k, v, causal=True, q_offsets=o, need_lse=True)
        want[cut] += tuple(mod.attend_backward(q, k, v, *want[cut], do, causal=True, q_offsets=o).values())
    q1 = q[:, :, :1].contiguous()
    few = mod.attend(q1, k, v)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        got.append((mod.attend(q, k, v, causal=True, q_offsets=o, stream=streams[i % 2]), mod.attend(q1, k, v, stream=streams[i % 2])))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[333][0]) and torch.equal(b, few) for a, b in got)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = mod.attend(q, k, v, causal=True, q_offsets=o, need_lse=True)
            grads = mod.attend_backward(q, k, v, out, lse, do, causal=True, q_offsets=o)
            one = mod.attend(q1, k, v)
        graphs.append((graph, (out, lse) + tuple(grads.values()), one))
    for cut in (100, 333):
        o[1] = cut
        for graph, _, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, results, one in graphs:
            assert all(torch.equal(a, b) for a, b in zip(results, want[cut])) and torch.equal(one, few)


def test_offsets_that_do_not_fit_stay_inside():
    """Offsets past the tensors, falling, negative: no access outside, and other sequences' rows are right."""
    q, k, v = make(1, 2, 2, 256, 256, 64, BF)
    mod = AgentAttention(1, 2, 64, 256, 1, BF)
    for at in ([0, 100, 1 << 30], [-5, 100, 300], [0, 200, 100, 256], [1 << 30, 1 << 30]):
        o = torch.tensor(at, dtype=torch.int32, device="cuda")
        out, lse = mod.attend(q, k, v, q_offsets=o, need_lse=True)
        mod.attend_backward(q, k, v, out, lse, q, q_offsets=o)
        if at[1] == 100:
            fit = mod.attend(q, k, v, q_offsets=torch.tensor([0, 100, 256], dtype=torch.int32, device="cuda"))
            assert torch.equal(out, fit)
    lengths = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    assert torch.equal(mod.attend(q, k, v, k_lengths=lengths, q_lengths=lengths), mod.attend(q, k, v))
    assert (mod.attend(q, k, v, k_lengths=-lengths) == 0).all()
    assert mod.query_status() == 0


def test_refusals():
    q, k, v = make(1, 4, 2, 64, 64, 64, BF)
    mod = AgentAttention(1, 4, 64, 64, 1, BF)
    o = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    out, lse = mod.attend(q, k, v, need_lse=True)
    bad = [dict(q=q.half()), dict(q=q.cpu()), dict(k=k[:, :1].expand(1, 3, 64, 64)), dict(v=v[:, :1]), dict(q=q[..., ::2]), dict(q=q[0]), dict(q=q[:, :2]),
           dict(q_offsets=o.long()), dict(q_offsets=o.cpu()), dict(k_offsets=o), dict(q_offsets=o, k_offsets=torch.cat([o, o])), dict(q_lengths=o), dict(scale=-1.0), dict(scale=0.0),
           dict(out=out[:, :2]), dict(out=out.float()), dict(q_offsets=o, k=k[:, :, :32], v=v[:, :, :32]), dict(workspace=torch.empty(16)), dict(scale=float("nan"))]
    for change in bad:
        with pytest.raises((ValueError, AgentAttnError)):
            mod.attend(**{**dict(q=q, k=k, v=v), **change})
    lengths = torch.tensor([64], dtype=torch.int32, device="cuda")
    status = [(dict(q_offsets=o, k_lengths=lengths), 1), (dict(q_offsets=o[:1]), 1), (dict(out=q), 1), (dict(k=k.expand(1, 2, 64, 64)[:, :1].expand(1, 2, 64, 64)), 1),
              (dict(scale=float("inf")), 1), (dict(q=q.new_zeros((1, 4, 64, 68))[..., :64]), 1),
              (dict(q=q.new_zeros((1, 4, 65, 64))), 2), (dict(q=q[:, :, :0]), 1), (dict(k=k[:, :, :0], v=v[:, :, :0]), 1)]
    for change, code in status:
        with pytest.raises(AgentAttnError) as e:
            mod.attend(**{**dict(q=q, k=k, v=v), **change})
        assert e.value.status == code, (change.keys(), str(e.value))
    do = torch.zeros_like(q)
    for change in (dict(lse=lse[:, :2]), dict(lse=lse.half()), dict(d_out=do[:, :2]), dict(grads=(do, k, v)), dict(grads=(do, torch.zeros_like(k))), dict(grads=(do, do, do)),
                   dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, AgentAttnError, TypeError)):
            mod.attend_backward(**{**dict(q=q, k=k, v=v, out=out, lse=lse, d_out=do), **change})
    batch = AgentAttention(2, 4, 64, 64, 1, BF)
    with pytest.raises(AgentAttnError) as e:
        batch.attend(q.expand(2, 4, 64, 64).contiguous(), k.expand(2, 2, 64, 64).contiguous(), v.expand(2, 2, 64, 64).contiguous(), q_offsets=o)
    assert e.value.status == 1
    few = AgentAttention(1, 4, 64, 40000, 1, BF)
    k2 = torch.zeros((1, 2, 40000, 64), dtype=BF, device="cuda")
    with pytest.raises(AgentAttnError) as e:
        few.attend(q[:, :, :1].contiguous(), k2, k2.clone(), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


@pytest.mark.parametrize("dt", [BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("N,M,d", [(64, (1 << 20) + 77, 64), (300, (1 << 20) + 77, 128), (300, (1 << 23) + 1, 64), (129, 16384 + 129, 64), (257, 32768, 128)])
def test_sums_over_long_axes(dt, causal, N, M, d):
    """Values of one and probabilities of all sizes: the result is one.  u of it and of the probabilities, 2^-14 of the tensor cores' sums (1024 steps of 2^-24), and of
    the sums in fp32 (32 of a tile, 128 tiles of a piece, the pieces) 2^-24 each, which the log-sum-exp has, too, with 2^-21 of exponentials and logarithm."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    q, k, v = torch.zeros((1, 1, N, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda"), torch.ones((1, 1, M, d), device="cuda")
    q[..., 0] = 1.0
    k[..., 0] = torch.randn(M, generator=gen, device="cuda") + torch.linspace(-3, 3, M, device="cuda")       # (the largest logit moves from piece to piece)
    q, k, v = q.to(dt), k.to(dt), v.to(dt)
    mod = AgentAttention(1, 1, d, M, 1, dt)
    out, lse = mod.attend(q, k, v, causal=causal, scale=1.0, need_lse=True)
    s = k[0, 0, :, 0].double()
    want = torch.stack([torch.logsumexp(s[:M - N + i + 1] if causal else s, 0) for i in range(N)]) if causal else torch.logsumexp(s, 0).expand(N)
    sums = 2.0 ** -24 * (32 + 128 + M / 16384)
    assert (out.double() - 1).abs().max() <= 2 * u_of(dt) + 2.0 ** -14 + sums, float((out.double() - 1).abs().max())
    assert ((lse[0, 0].double() - want).abs() <= sums + 2.0 ** -21 + 2.0 ** -23 * want.abs()).all(), float((lse[0, 0].double() - want).abs().max())
    assert mod.query_status() == 0


@pytest.mark.parametrize("dt", [BF, FH])
def test_single_queries_over_many_long_caches(dt):
    """Caches that fill the GPU without shares of their keys (windows of one buffer): sums of 2^22 keys come in pieces all the same.  Bounds as above."""
    B, kv, M, d = 150, 2, (1 << 22) + 5, 64
    rows = torch.ones((M + 3 * B, d), device="cuda")
    rows[:, 0] = torch.randn(M + 3 * B, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    k = rows.to(dt).as_strided((B, kv, M, d), (2 * d, d, d, 1))
    v = torch.ones((M + 3 * B, d), dtype=dt, device="cuda").as_strided((B, kv, M, d), (2 * d, d, d, 1))
    q = torch.zeros((B, 2, 1, d), dtype=dt, device="cuda")
    q[..., 0] = 1.0
    mod = AgentAttention(B, 2, d, M, 1, dt)
    out, lse = mod.attend(q, k, v, scale=1.0, need_lse=True)
    sums = 2.0 ** -24 * (1024 + 64 + M / 65536)
    assert (out.double() - 1).abs().max() <= 2 * u_of(dt) + 2.0 ** -14 + sums, float((out.double() - 1).abs().max())
    for b in (0, 77, 149):
        want = torch.stack([torch.logsumexp(k[b, h, :, 0].double(), 0) for h in range(2)])
        assert ((lse[b, :, 0].double() - want).abs() <= sums + 2.0 ** -21 + 2.0 ** -23 * want.abs()).all()
    assert mod.query_status() == 0


def rows_over_one_strong_key(N, M, below, dt, d=64, first=0):
    """Queries whose logit is 0 at one key and -below at the others; constant values (the result is 1), and a channel of the strong key alone."""
    q, k, v = torch.zeros((1, 1, N, d)), torch.zeros((1, 1, M, d)), torch.ones((1, 1, M, d))
    q[..., 0], k[..., 0] = 1.0, -below
    k[..., first, 0] = 0.0
    v[..., 1] = 0.0
    v[..., first, 1] = 1.0
    return tuple(t.to("cuda", dt) for t in (q, k, v))


@pytest.mark.parametrize("dt", [FH, BF])
@pytest.mark.parametrize("N,d", [(1, 64), (32, 64), (300, 64), (300, 128)])
def test_many_keys_far_below_one(dt, N, d):
    """65535 keys 16 to 18 below one: 2e-3 of the result, each of them below f16's normal numbers, or its last one; and 2^20 keys 19 to 21 below one.  Bound as above: u of
    the result, u of the probabilities, 2^-14 of the tensor cores' sums."""
    for below in (16.0, 17.0, 17.5, 18.0):
        check(*rows_over_one_strong_key(N, 65536, below, dt, d), scale=1.0, grad=False, what=below)
    for below in (19.0, 20.0, 21.0):
        q, k, v = rows_over_one_strong_key(N, 1 << 20, below, dt, d)
        got = AgentAttention(1, 1, d, 1 << 20, 1, dt).attend(q, k, v, scale=1.0).double()
        want = torch.softmax(k[0, 0, :, 0].double(), 0) @ v[0, 0].double()
        assert ((got - want).abs() <= (2 * u_of(dt) + 2.0 ** -14) * want).all(), (below, float((got / want - 1).abs().max()))


@pytest.mark.parametrize("N,M,below", [(1, 65536, 17.0), (64, 65536, 17.0), (300, 65536, 24.0), (2000, 20000, 12.0), (64, 1 << 20, 17.0), (300, (1 << 20) + 77, 20.0), (1, 1 << 23, 17.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_long_sums_in_fp32(N, M, below, d):
    """Equal probabilities beside a large one: their sums are rounded the same way at every step.  2^-24 for each of a piece's 128 steps and of the pieces, twice (the
    result's sum and the probabilities'), 2^-21 of exponentials."""
    q, k, v = rows_over_one_strong_key(N, M, below, F32, d)
    mod = AgentAttention(1, 1, d, M, 1, F32)
    out, lse = mod.attend(q, k, v, scale=1.0, need_lse=True)
    s = k[0, 0, :, 0].double()
    want, sums = torch.softmax(s, 0) @ v[0, 0].double(), 2.0 ** -24 * (8 + 128 + M / 4096)
    assert ((out.double() - want).abs() <= (2 * sums + 2.0 ** -21) * want).all(), float((out.double() / want - 1).abs().max())
    assert (lse.double() - torch.logsumexp(s, 0)).abs().max() <= sums + 2.0 ** -21


@pytest.mark.parametrize("dt", [FH, BF])
@pytest.mark.parametrize("h,N,M,d", [(1, (1 << 20) + 77, 130, 64), (2, 1 << 19, 70, 128), (4, 16384 + 5, 130, 64)])
def test_gradient_sums_over_many_queries(dt, h, N, M, d):
    """Gradients of keys and values that all queries add to with one sign.  Bound: u of the result, of P and of dS, u of a rounded result in D, 2^-14 of the tensor cores'
    sums and 2^-20 of a probability."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k, v, do = torch.zeros((1, h, N, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda"), torch.zeros((1, h, N, d), device="cuda")
    q[..., 0], k[..., 0] = rand(h, N), rand(M)
    q[..., 1] = do[..., 1] = torch.where(rand(h, N) > 0, 1.0, -1.0)
    v[..., 1], do[..., 2] = rand(M), 1.0
    q, k, v, do = (t.to(dt) for t in (q, k, v, do))
    mod = AgentAttention(1, h, d, N, 1, dt)
    out, lse = mod.attend(q, k, v, scale=1.0, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, do, scale=1.0)
    want = torch.zeros((4, M), dtype=torch.float64, device="cuda")         # dV, dK and what dK's errors are made of
    for i in range(h):
        for r in range(0, N, 1 << 17):
            p = torch.softmax(q[0, i, r:r + (1 << 17), :1].double() * k[0, 0, :, 0].double(), -1)
            mean = p @ v[0, 0, :, 1].double()
            slope = p * (v[0, 0, :, 1].double() - mean[:, None])
            want += torch.stack([p.sum(0), slope.sum(0), slope.abs().sum(0), (p * mean[:, None].abs()).sum(0)])
    u, e = u_of(dt), 2.0 ** -14 + 2.0 ** -20
    rel = (g["dv"][0, 0, :, 2].double() - want[0]).abs() / want[0]
    assert rel.max() <= 2 * u + e, float(rel.max())
    rel = (g["dk"][0, 0, :, 1].double() - want[1]).abs() / (want[1].abs() * u + want[2] * (u + e) + want[3] * (u + e))
    assert rel.max() <= 1, float(rel.max())
    assert mod.query_status() == 0


@pytest.mark.parametrize("dt", [FH, BF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("N,M,d", [(130, (1 << 20) + 77, 64), (70, (1 << 19) + 1, 128), (200, 16384 + 1, 64), (1, 1 << 20, 128)])
def test_gradient_sums_over_many_keys(dt, causal, N, M, d):
    """Gradients of queries that all keys add to with one sign: dQ = sum P (1 - D k).  Bounds as above."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    q, k, v, do = torch.zeros((1, 1, N, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda"), torch.zeros((1, 1, N, d), device="cuda")
    q[..., 0], k[..., 0] = 1.0, torch.randn(M, generator=gen, device="cuda")
    k[..., 1] = v[..., 1] = torch.where(torch.randn(M, generator=gen, device="cuda") > 0, 1.0, -1.0)
    do[..., 1] = 1.0
    q, k, v, do = (t.to(dt) for t in (q, k, v, do))
    mod = AgentAttention(1, 1, d, M, 1, dt)
    out, lse = mod.attend(q, k, v, causal=causal, scale=1.0, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, do, causal=causal, scale=1.0)
    s, sign = k[0, 0, :, 0].double(), k[0, 0, :, 1].double()
    for i in {0, N // 2, N - 1}:
        m = M - N + i + 1 if causal else M
        p = torch.softmax(s[:m], 0)
        mean = p @ sign[:m]
        want = p @ (sign[:m] * (sign[:m] - mean))
        err = float((g["dq"][0, 0, i, 1].double() - want).abs())
        assert err <= u_of(dt) * (want.abs() + 1 + 2 * mean.abs()) + (2.0 ** -14 + 2.0 ** -20) * (1 + mean.abs()), (i, err)
    assert mod.query_status() == 0


@pytest.mark.parametrize("h,N,M,d", [(1, 1 << 18, 70, 64), (2, 1 << 17, 33, 128), (4, 16384, 64, 32), (1, 70, 1 << 18, 64), (2, 33, 1 << 17, 128), (1, 1 << 16, 64, 96)])
def test_gradient_long_sums_in_fp32(h, N, M, d):
    """Equal summands, which are rounded the same way at every step: P = 1 / M, dO = 0.7, so dV = 0.7 N h / M; dK and dQ of slopes that are one number.  2^-24 for each of a
    piece's 128 steps of 32 columns and of the pieces, 2^-20 of probabilities, slopes and products."""
    q, k = torch.zeros((1, h, N, d), device="cuda"), torch.zeros((1, 1, M, d), device="cuda")
    v, do = torch.zeros((1, 1, M, d), device="cuda"), torch.zeros((1, h, N, d), device="cuda")
    q[..., 1], do[..., 1], do[..., 2] = 0.3, 0.9, 0.7
    sign = torch.where(torch.arange(M, device="cuda") % 3 == 0, 1.0, -1.0)
    v[..., 1] = sign
    mod = AgentAttention(1, h, d, max(N, M), 1, F32)
    k[..., 3] = sign                                                      # (q has nothing there: all logits are 0)
    out, lse = mod.attend(q, k, v, scale=1.0, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, do, scale=1.0)
    f = lambda x: float(torch.tensor(x))  # noqa: E731  (as it is in fp32)
    mean = float(sign.double().mean())
    slope = f(0.9) / M * (sign.double() - mean)
    sums = lambda columns: 2.0 ** -24 * (128 + columns / 4096) + 2.0 ** -20  # noqa: E731
    assert (g["dv"][0, 0, :, 2].double() * M / (f(0.7) * N * h) - 1).abs().max() <= sums(N * h)
    assert (g["dk"][0, 0, :, 1].double() / (slope * N * h * f(0.3)) - 1).abs().max() <= 4 * sums(N * h)       # (a slope: 2 / 3 or more of P, out of D with an error of P's)
    assert (g["dq"][0, :, :, 3].double() / (slope * sign.double()).sum() - 1).abs().max() <= 4 * sums(M)


@pytest.mark.parametrize("dt", [BF, FH, F32])
@pytest.mark.parametrize("N,M,d", [(1, 700, 64), (5, 700, 128), (200, 300, 64), (300, 200, 128)])
def test_infinite_logits(dt, N, M, d):
    """+infinity: a NaN row.  -infinity: weight 0 in 16 bits, what the formulas give; NaN in fp32.  A row of nothing but -infinity: NaN.  Other heads do not notice."""
    q, k, v = make(1, 2, 2, N, M, d, dt)
    q[..., 0] = q[..., 0].abs() + 1
    mod = AgentAttention(1, 2, d, max(N, M), 1, dt)
    plain, _ = mod.attend(q, k, v, need_lse=True)
    up, down = k.clone(), k.clone()
    up[0, 0, M // 2, 0] = float("inf")
    down[0, 0, [3, M // 2, M - 1], 0] = -float("inf")
    got = mod.attend(q, up, v)
    assert got[0, 0].isnan().all() and torch.equal(got[0, 1], plain[0, 1])
    got, lse = mod.attend(q, down, v, need_lse=True)
    assert torch.equal(got[0, 1], plain[0, 1])
    if dt is F32:
        assert got[0, 0].isnan().all()
    else:
        keep = torch.ones(M, dtype=torch.bool, device="cuda")
        keep[[3, M // 2, M - 1]] = False
        for i in {0, N - 1}:
            s = k[0, 0, keep].double() @ q[0, 0, i].double() * d ** -0.5
            p, w = torch.softmax(s, 0), v[0, 0, keep].double()
            assert ((got[0, 0, i].double() - p @ w).abs() <= 2 * u_of(dt) * (p @ w.abs()) + 1e-5).all()
            assert abs(float(lse[0, 0, i].double() - torch.logsumexp(s, 0))) <= 1e-5
    down[0, 0, :, 0] = -float("inf")
    assert mod.attend(q, down, v)[0, 0].isnan().all()
    assert mod.query_status() == 0


def test_a_scale_whose_units_of_log2_are_infinite_is_refused():
    q, k, v = make(1, 2, 2, 40, 40, 64, BF)
    mod = AgentAttention(1, 2, 64, 40, 1, BF)
    for scale in (2.5e38, 3.4e38):
        with pytest.raises(AgentAttnError) as e:
            mod.attend(torch.zeros_like(q), k, v, scale=scale)
        assert e.value.status == 1
    out = mod.attend(torch.zeros_like(q), k, v, scale=2.0 ** 126)                # (logits of zero: the mean)
    assert ((out.double() - v.double().mean(2, keepdim=True)).abs() <= 2 * u_of(BF) * v.double().abs().mean(2, keepdim=True)).all()


@pytest.mark.parametrize("dt", [F32, BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("h,kv,d", [(2, 2, 64), (8, 1, 128), (3, 1, 40)])
def test_few_queries_over_packed_keys(dt, causal, h, kv, d):
    """Up to three queries each of packed sequences of 0 to 9000 keys: several shares of the keys, some of them without a key of a sequence."""
    lengths, keys = [1, 2, 0, 1, 3, 1], [9000, 700, 30, 0, 2, 4001]
    at, ak = [1], [5]
    for n, m in zip(lengths, keys):
        at.append(at[-1] + n)
        ak.append(ak[-1] + m)
    q, k, v = make(1, h, kv, at[-1] + 2, ak[-1] + 3, d, dt)
    k[:, :, :5], v[:, :, ak[-1]:] = float("nan"), float("inf")
    check(q, k, v, causal=causal, q_offsets=at, k_offsets=ak, grad=False)


@pytest.mark.parametrize("dt", [BF, FH])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("S", [40, 128, 129])
def test_gradient_of_many_long_packed_sequences(dt, causal, S):
    """More sequences than a lane's first place holds, as many as take tiles by work, and one more."""
    gen = torch.Generator().manual_seed(S)
    lengths = [int(x) for x in torch.randint(1, 1200, (S,), generator=gen)]
    lengths[3] = lengths[S - 2] = 0
    at = [2]
    for n in lengths:
        at.append(at[-1] + n)
    assert at[-1] / S >= 512
    q, k, v = make(1, 2, 1, at[-1] + 9, at[-1] + 9, 64, dt, fused=True)
    check(q, k, v, causal=causal, q_offsets=at)


@pytest.mark.parametrize("dt", [BF, FH])
@pytest.mark.parametrize("d,N", [(64, 65), (64, 200), (128, 129), (128, 300), (64, 700)])
def test_first_rows_of_a_causal_sequence(dt, d, N):
    """The first rows see a few keys, as short sequences do: their slopes keep the accuracy of theirs (0.8 u in the 2-norm)."""
    lengths = [N] * 40
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    q, k, v = make(1, 4, 2, at[-1], at[-1], d, dt, fused=True)
    mod = AgentAttention(1, 4, d, at[-1], 1, dt)
    o = torch.tensor(at, dtype=torch.int32, device="cuda")
    do = torch.randn(q.shape, device="cuda").to(dt)
    out, lse = mod.attend(q, k, v, q_offsets=o, causal=True, need_lse=True)
    g = mod.attend_backward(q, k, v, out, lse, do, q_offsets=o, causal=True)
    few = 8
    want, got = torch.zeros((40, 4, few, d), dtype=torch.float64, device="cuda"), torch.zeros((40, 4, few, d), dtype=torch.float64, device="cuda")
    for i, a in enumerate(at[:-1]):
        for h in range(4):
            want[i, h] = reference(q[0, h, a:a + few], k[0, h // 2, a:a + few], v[0, h // 2, a:a + few], True, d ** -0.5, do[0, h, a:a + few])["dq"]
        got[i] = g["dq"][0, :, a:a + few].double()
    assert (got[:, :, 0] == 0).all()
    for r in range(1, few):
        rel = (got[:, :, r] - want[:, :, r]).norm() / want[:, :, r].norm()
        assert rel <= 0.8 * u_of(dt), (r, float(rel / u_of(dt)))
    assert mod.query_status() == 0
