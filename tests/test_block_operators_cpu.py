"""Host side of the operators around the attention that needs no GPU: null handles at the C ABI, struct layouts."""
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
    assert lib.agent_attn_rotate(None, None, None, None, 1, None, None, None, None, None, None) == 1
    assert lib.agent_attn_rotate_backward(None, None, None, None, None, None, None, 1, None, None, None, None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_rotate_workspace_bytes(None) == 0
    assert lib.agent_attn_gated(None, None, None, None, 0, None) == 1
    assert lib.agent_attn_gated_backward(None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_gated_workspace_bytes(None, 8, 8, 8, 1) == 0


def test_structs_match_the_header():
    text = open(os.path.join(ROOT, "include", "agent_attn.h")).read()
    for name, struct in (("agent_attn_rotary", binding.AgentAttnRotary), ("agent_attn_norm", binding.AgentAttnNorm),
                         ("agent_attn_gate", binding.AgentAttnGate), ("agent_attn_gate_grads", binding.AgentAttnGateGrads)):
        body = re.search(r"typedef struct \{((?:(?!typedef).)*?)\} %s;" % name, text, flags=re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [f for line in re.findall(r"(?:int|float|void|long long)\b\*?\s*([^;]+);", body) for f in re.findall(r"\b(\w+)(?:\[\d\])?\s*(?:,|$)", line.strip())]
        assert fields == [f[0] for f in struct._fields_], name


def test_sizes_past_32_bits_are_not_cut_off():
    """2^32 + 4 tokens or rows are not four: the first is refused here, the others reach the library as a number that it refuses."""
    big = (1 << 32) + 4
    handle = SimpleNamespace(cfg=SimpleNamespace(max_tokens=16), _chk_tensor=lambda *a: None)
    with pytest.raises(pkg.AgentAttnError) as e:
        pkg.AgentAttention._tokens(handle, torch.empty((1, 1, big, 8), device="meta"))
    assert e.value.status == 2
    assert pkg.AgentAttention._tokens(handle, torch.empty((1, 1, 16, 8), device="meta")) == 16
    for x, w in ((torch.empty((big, 8), device="meta"), torch.empty((16, 8), device="meta")), (torch.empty((2, 8), device="meta"), torch.empty((big, 8), device="meta")),
                 (torch.empty((1, big), device="meta"), torch.empty((16, big), device="meta"))):
        gate = pkg.AgentAttention._gate(handle, x, w, w, None, None, "silu")
        assert max(gate.rows, gate.channels, gate.hidden) == (1 << 31) - 1
    freq = SimpleNamespace(shape=(1,), dtype=torch.float32, is_cuda=True, is_contiguous=lambda: True, data_ptr=lambda: 0, device="cuda")
    for extent in ((big,), (0,), (-3,)):
        with pytest.raises(ValueError):
            pkg.Rotary(freq, (2,), extent)
    assert list(pkg.Rotary(freq, (2,), (16,))._c.extent)[:1] == [16]


class OnDevice:
    """What the checks look at of a tensor, on any device."""

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", device) if device >= 0 else torch.device("cpu")
        self.is_cuda = device >= 0

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0


def test_tensors_of_another_device_are_refused():
    """The kernels of a handle run on its device: a pointer of another one (or of the host) never reaches them."""
    handle = SimpleNamespace(_index=1, device=torch.device("cuda", 1), dtype=torch.float32, batch=1, heads=2, head_dim=8, _strides={}, cfg=SimpleNamespace(max_tokens=4))
    cls, shape = pkg.AgentAttention, (1, 2, 4, 8)
    checks = [lambda d: cls._chk_tensor(handle, OnDevice(shape, torch.float32, d), shape, "x"),
              lambda d: cls._chk_views(handle, ("q", "k"), (OnDevice(shape, torch.float32, 1), OnDevice(shape, torch.float32, d)), 4, torch.float32),
              lambda d: cls._chk_workspace(handle, OnDevice((64,), torch.uint8, d)),
              lambda d: pkg.Rotary(OnDevice((1,), torch.float32, d), (2,), (4,))._check(1, 4, handle._index)]
    for check in checks:
        check(1)
        for other in (0, 2, -1):
            with pytest.raises(ValueError):
                check(other)
    cls._chk_tensor(handle, OnDevice(shape, torch.float32, -1), shape, "x", cuda=False)
    with pytest.raises(ValueError):
        cls._chk_workspace(handle, torch.zeros(64, dtype=torch.uint8))


def test_null_handle_of_two_terms():
    lib = pkg.load_library()
    assert lib.agent_attn_gated_backward_two_terms(None, None, None, None, None, 0, None) == 1
    assert lib.agent_attn_gated_workspace_bytes(None, 8, 8, 8, 2) == 0
