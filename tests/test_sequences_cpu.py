"""Host side of softmax attention over whole sequences and of the layer norm that needs no GPU: null handles, struct layouts, checks of arguments."""
import os
import re
from types import SimpleNamespace

import pytest
import torch

import paper_2312_08874_b200 as pkg
from paper_2312_08874_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_null_handles():
    lib = pkg.load_library()
    assert lib.agent_attn_attend(None, None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_attend_backward(None, None, None, None, None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_attend_workspace_bytes(None, None, 0) == 0
    assert lib.agent_attn_layer_norm(None, None, None, None) == 1
    assert lib.agent_attn_layer_norm_backward(None, None, None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_layer_norm_workspace_bytes(None, 8, 8) == 0


def test_structs_match_the_header():
    text = open(os.path.join(ROOT, "include", "agent_attn.h")).read()
    for name, struct in (("agent_attn_sequences", binding.AgentAttnSequences), ("agent_attn_attend_grads", binding.AgentAttnAttendGrads),
                         ("agent_attn_layer_norm_args", binding.AgentAttnLayerNorm)):
        body = re.search(r"typedef struct \{((?:(?!typedef).)*?)\} %s;" % name, text, flags=re.S).group(1)
        body = re.sub(r"/\*.*?\*/|\*", " ", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
        fields = []
        for line in re.findall(r"(?:const\s+)?(?:long long|int|float|void)\b([^;]+);", body):
            fields += [re.sub(r"\[\d\]", "", f).strip() for f in line.split(",")]
        assert fields == [f[0] for f in struct._fields_], name


class OnDevice:
    """What the checks look at of a tensor, on any device."""

    def __init__(self, shape, dtype=torch.bfloat16, device=1, strides=None):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", device) if device >= 0 else torch.device("cpu")
        self._strides = strides or torch.empty(shape, device="meta").stride()

    def get_device(self):
        return self.device.index if self.device.type == "cuda" else -1

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def is_contiguous(self):
        return tuple(self._strides) == tuple(torch.empty(self.shape, device="meta").stride())

    def data_ptr(self):
        return 0


def handle(batch=1, heads=4, head_dim=64, max_tokens=256):
    h = SimpleNamespace(_index=1, device=torch.device("cuda", 1), dtype=torch.bfloat16, batch=batch, heads=heads, head_dim=head_dim, cfg=SimpleNamespace(max_tokens=max_tokens))
    for name in ("_view", "_numbers", "_tokens", "_sequences", "_chk_tensor", "_layer_norm"):
        setattr(h, name, getattr(pkg.AgentAttention, name).__get__(h))
    return h


def tensors(batch=1, heads=4, kv=2, n=64, m=64, d=64):
    return OnDevice((batch, heads, n, d)), OnDevice((batch, kv, m, d)), OnDevice((batch, kv, m, d))


def test_sequences_as_the_library_takes_them():
    h, (q, k, v) = handle(), tensors()
    s = h._sequences(q, k, v, True, None, None, None, None, None)
    assert (s.queries, s.keys, s.kv_heads, s.causal, s.scale, s.sequences) == (64, 64, 2, 1, 0.0, 0) and list(s.q_strides) == [64, 4096, 64]
    at = OnDevice((9,), torch.int32)
    s = h._sequences(q, k, v, False, 0.5, at, None, None, None)
    assert s.sequences == 8 and s.scale == 0.5
    assert not (s.q or s.q_offsets)                                  # (pointers are a call's own)
    one = OnDevice((1, 4, 1, 64), strides=(999, 128, 7, 1))          # strides of single entries are never used
    assert list(h._sequences(one, k, v, False, None, None, None, None, None).q_strides) == [64, 128, 64]


def test_refusals():
    h, (q, k, v) = handle(), tensors()
    at, long = OnDevice((9,), torch.int32), OnDevice((8,), torch.int32)
    none = (None,) * 4
    bad = [((OnDevice((1, 4, 64, 64), torch.float16), k, v), none), ((OnDevice((1, 4, 64, 64), device=0), k, v), none), ((OnDevice((1, 4, 64, 64), device=-1), k, v), none),
           ((OnDevice((1, 3, 64, 64)), k, v), none), ((q, OnDevice((1, 3, 64, 64)), v), none), ((q, OnDevice((1, 0, 64, 64)), v), none), ((q, k, OnDevice((1, 2, 65, 64))), none),
           ((OnDevice((1, 4, 64, 64), strides=(1, 1, 64, 2)), k, v), none), ((OnDevice((4, 64, 64)), k, v), none),
           ((q, k, v), (None, at, None, None)), ((q, k, v), (OnDevice((9,), torch.int64), None, None, None)), ((q, k, v), (OnDevice((9,), torch.int32, 0), None, None, None)),
           ((q, k, v), (at, long, None, None)), ((q, k, v), (None, None, at, None)), ((q, k, v), (None, None, None, at)), ((q, k, v), (OnDevice((3, 3), torch.int32), None, None, None)),
           ((q, k, v), (OnDevice((9,), torch.int32, strides=(2,)), None, None, None)), ((OnDevice((1, 4, 32, 64)), k, v), (at, None, None, None))]
    for (a, b, c), numbers in bad:
        with pytest.raises(ValueError):
            h._sequences(a, b, c, False, None, *numbers)
    for scale in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            h._sequences(q, k, v, False, scale, *none)
    big = OnDevice((1, 4, (1 << 32) + 4, 64))
    with pytest.raises(pkg.AgentAttnError) as e:
        h._sequences(big, k, v, False, None, *none)
    assert e.value.status == 2
    for x, w in ((OnDevice((8, 64), torch.float32), None), (OnDevice((8, 64), device=0), None), (OnDevice((8, 64), strides=(1, 8)), None), (OnDevice((8, 64)), OnDevice((32,))), (OnDevice(()), None)):
        with pytest.raises(ValueError):
            h._layer_norm(x, w, None, 1e-5)
    a = h._layer_norm(OnDevice((1 << 33, 8)), None, None, 1e-5)
    assert a.rows == 1 << 33 and a.channels == 8                     # (which the library refuses)



def test_numbers_of_a_kept_call_are_its_own():
    """What is kept for a call's shapes follows the scale's value and not the object that holds it."""
    h = handle()
    h._calls = {}
    q, k = OnDevice((1, 4, 32, 64)), OnDevice((1, 2, 32, 64))
    h._call = pkg.AgentAttention._call.__get__(h)
    scale, causal = torch.tensor(0.5), torch.tensor(True)
    for value, below in ((0.5, True), (0.25, False), (0.125, True)):
        scale.fill_(value)
        causal.fill_(below)
        s, _ = h._call(q, k, k, causal, scale, None, None, None, None)
        assert s.scale == value and s.causal == int(below)


def test_a_scale_that_is_zero_in_fp32_is_refused():
    h = handle()
    q, k = OnDevice((1, 4, 32, 64)), OnDevice((1, 2, 32, 64))
    with pytest.raises(ValueError):
        h._sequences(q, k, k, False, 1e-50, None, None, None, None)              # (0 means the default to the library)
    assert h._sequences(q, k, k, False, 1e39, None, None, None, None).scale == float("inf")      # (which the library refuses)
    assert h._sequences(q, k, k, False, 1e-30, None, None, None, None).scale > 0


def slots(offsets, unit, rows, most):
    """The kernels' search: which sequence and tile a slot has."""
    S = len(offsets) - 1
    clamp = lambda x: min(max(x, 0), most)  # noqa: E731
    base = lambda s: clamp(offsets[s]) * unit // rows + s  # noqa: E731
    found = []
    for slot in range(most * unit // rows + S):
        lo, hi = 0, S
        while hi - lo > 1:
            mid = (lo + hi) // 2
            lo, hi = (mid, hi) if base(mid) <= slot else (lo, mid)
        if slot < base(lo):
            continue
        first = clamp(offsets[lo])
        count = min(max(offsets[lo + 1], first), most) - first
        tile = slot - base(lo)
        assert tile <= most * unit // rows + 1                       # (a row number never leaves 31 bits)
        if tile * rows < count * unit:
            found.append((lo, tile))
    return found


@pytest.mark.parametrize("unit,rows", [(1, 256), (1, 128), (1, 64), (3, 16), (8, 64), (40, 16)])
def test_every_tile_of_packed_sequences_has_a_slot(unit, rows):
    gen = torch.Generator().manual_seed(unit * rows)
    for _ in range(60):
        n = int(torch.randint(1, 12, (1,), generator=gen))
        lengths = [int(x) for x in torch.randint(0, 300, (n,), generator=gen) * torch.randint(0, 2, (n,), generator=gen)]
        at = [int(torch.randint(0, 20, (1,), generator=gen))]
        for x in lengths:
            at.append(at[-1] + x)
        most = at[-1] + int(torch.randint(0, 9, (1,), generator=gen))
        if most == 0:
            continue
        want = [(s, t) for s, x in enumerate(lengths) for t in range((x * unit + rows - 1) // rows)]
        assert slots(at, unit, rows, most) == want


def test_offsets_that_do_not_rise_stay_inside():
    for at in ([0, 100, 1 << 30], [-5, 100, 300], [0, 200, 100, 256], [1 << 30, 1 << 30], [256, 0, 256, 0, 256], [-(1 << 31), (1 << 31) - 1]):
        for unit, rows in ((1, 256), (3, 16), (1, 64)):
            slots(at, unit, rows, 256)


def ranked(q_at, k_at, causal, keys, rows=128):
    """The gradient's order of a packed call's tiles, restated: (sequence, tile) of every slot.  A lane holds the sequences lane, lane + 32, ..."""
    nq, nk = [b - a for a, b in zip(q_at, q_at[1:])], [b - a for a, b in zip(k_at, k_at[1:])]
    S = len(nq)
    tiles = [((nk if keys else nq)[s] + rows - 1) // rows for s in range(S)]
    div = lambda a, b: int(a / b)  # noqa: E731  (towards zero, as in C)

    def at_least(s, units):
        if units <= 0 or not tiles[s]:
            return tiles[s]
        ahead, need = nk[s] - nq[s], (units - 1) * 128 + 1
        if not causal:
            return tiles[s] if (nq if keys else nk)[s] >= need else 0
        if keys:
            most = min(nq[s] - need, nq[s] - need + ahead)
            return 0 if most < 0 else min(tiles[s], div(max(0, nq[s] - need + ahead), rows) + 1)
        if nk[s] < need:
            return 0
        return tiles[s] - min(tiles[s] - 1, max(0, div(need - ahead + rows - 1, rows) - 1))
    count = lambda units: sum(at_least(s, units) for s in range(S))  # noqa: E731
    found, slot = [], 0
    while count(0) > slot:
        lo, hi = 0, (max(q_at[-1], k_at[-1]) + 127) // 128 + 1
        while hi - lo > 1:
            mid = (lo + hi) >> 1
            lo, hi = (mid, hi) if count(mid) > slot else (lo, mid)
        left, hit = slot - count(hi), None
        for i in range(4):                                               # (groups of 32 sequences, a lane's places)
            mine = [(s, at_least(s, lo) - at_least(s, hi), at_least(s, hi)) for s in range(32 * i, min(S, 32 * i + 32))]
            for s, some, more in mine:
                if hit is None and 0 <= left < some:
                    hit = (s, more + left if not causal or keys else tiles[s] - 1 - more - left)
                left -= some
        found.append(hit)
        slot += 1
    return found, [(s, t) for s in range(S) for t in range(tiles[s])]


@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("most", [1, 7, 33, 70, 128])
def test_ranked_tiles_are_found_once_each_and_fall_in_work(keys, causal, most):
    gen = torch.Generator().manual_seed(most * 4 + 2 * causal + keys)
    for trial in range(6):
        S = most if trial < 2 else int(torch.randint(1, most + 1, (1,), generator=gen))
        draw = lambda: [int(x) for x in torch.randint(0, 1500, (S,), generator=gen) * (torch.rand(S, generator=gen) < 0.8)]  # noqa: E731
        nq = draw()
        nk = nq if trial % 3 == 0 else draw() if trial % 3 == 1 else [a + b for a, b in zip(nq, draw())]
        q_at, k_at = [0], [0]
        for a, b in zip(nq, nk):
            q_at.append(q_at[-1] + a)
            k_at.append(k_at[-1] + b)
        if q_at[-1] == 0 or k_at[-1] == 0:
            continue
        found, want = ranked(q_at, k_at, causal, keys)
        assert sorted(found) == want

        def work(s, t):                                                  # columns in units of 128
            ahead = nk[s] - nq[s]
            if keys:
                n = nq[s] - (max(0, 128 * t - ahead) if causal else 0)
            else:
                n = min(nk[s], min(nq[s], 128 * t + 128) + ahead) if causal else nk[s]
            return max(0, n + 127) // 128 if n > 0 else 0
        works = [work(*x) for x in found]
        assert all(a >= b for a, b in zip(works, works[1:])), (q_at, k_at)
