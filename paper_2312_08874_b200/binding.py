"""Thin ctypes binding of `libagent_attn.so` (declared in `include/agent_attn.h`).

Argument marshalling only: every step of the forward pass runs in the library's CUDA kernels.
torch is used for device memory (`data_ptr()`), streams and dtype bookkeeping.  There is no
fallback: if the library is missing or no sm_100 GPU is present, construction raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional

import torch

from .build import LIB_PATH, build_library

AA_F32, AA_BF16, AA_F16 = 0, 1, 2
AA_PATH_AUTO, AA_PATH_SIMT, AA_PATH_UNFUSED, AA_PATH_QUEUE = 0, 1, 2, 3
STATUS_NAMES = {0: "AA_OK", 1: "AA_ERR_INVALID_ARG", 2: "AA_ERR_UNSUPPORTED", 3: "AA_ERR_WORKSPACE",
                4: "AA_ERR_CUDA", 5: "AA_ERR_TIMEOUT"}
_INT_MAX = 0x7fffffff                  # ctypes cuts larger numbers off without a word
_ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}
_DTYPES = {torch.float32: AA_F32, torch.bfloat16: AA_BF16, torch.float16: AA_F16}

EXPORTS = [
    "agent_attn_create", "agent_attn_destroy", "agent_attn_last_error", "agent_attn_workspace_bytes",
    "agent_attn_forward", "agent_attn_pool", "agent_attn_aggregate", "agent_attn_broadcast",
    "agent_attn_staging_bytes", "agent_attn_forward_host", "agent_attn_query_status",
    "agent_attn_last_launch_count", "agent_attn_aggregate_static", "agent_attn_static_scratch_bytes",
    "agent_attn_compose_bias", "agent_attn_forward_strided",
    "agent_attn_backward_workspace_bytes", "agent_attn_backward", "agent_attn_test_set_poll_limit",
    "agent_attn_test_set_stage_mask", "agent_attn_rotate", "agent_attn_rotate_backward", "agent_attn_rotate_workspace_bytes",
    "agent_attn_gated", "agent_attn_gated_backward", "agent_attn_gated_backward_two_terms", "agent_attn_gated_workspace_bytes",
]


class AgentAttnConfig(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("max_tokens", ctypes.c_int), ("max_agents", ctypes.c_int), ("dtype", ctypes.c_int),
                ("scale1", ctypes.c_float), ("scale2", ctypes.c_float), ("device", ctypes.c_int),
                ("path", ctypes.c_int)]


class AgentAttnBias(ctypes.Structure):
    _fields_ = [("b1", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class AgentAttnGrads(ctypes.Structure):
    _fields_ = [("dq", ctypes.c_void_p), ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p),
                ("db1", ctypes.c_void_p), ("db2", ctypes.c_void_p), ("dwd", ctypes.c_void_p)]


class AgentAttnRotary(ctypes.Structure):
    _fields_ = [("axes", ctypes.c_int), ("extent", ctypes.c_int * 3), ("channels", ctypes.c_int * 3), ("pairs", ctypes.c_int),
                ("freq", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_batch", ctypes.c_longlong)]


class AgentAttnNorm(ctypes.Structure):
    _fields_ = [("q_gain", ctypes.c_void_p), ("k_gain", ctypes.c_void_p), ("eps", ctypes.c_float)]


class AgentAttnGate(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("b_gate", ctypes.c_void_p),
                ("b_up", ctypes.c_void_p), ("rows", ctypes.c_int), ("channels", ctypes.c_int), ("hidden", ctypes.c_int),
                ("activation", ctypes.c_int)]


class AgentAttnGateGrads(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dw_gate", ctypes.c_void_p), ("dw_up", ctypes.c_void_p), ("db_gate", ctypes.c_void_p),
                ("db_up", ctypes.c_void_p)]


class AgentAttnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib: Optional[ctypes.CDLL] = None


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """dlopen the in-tree library (building it first if its sources are newer)."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing:
        try:
            build_library()
        except Exception:
            if not os.path.exists(LIB_PATH):
                raise
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2312_08874_b200.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.agent_attn_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(AgentAttnConfig)]
    lib.agent_attn_create.restype = ci
    lib.agent_attn_destroy.argtypes = [vp]
    lib.agent_attn_destroy.restype = ci
    lib.agent_attn_last_error.argtypes = [vp]
    lib.agent_attn_last_error.restype = ctypes.c_char_p
    lib.agent_attn_workspace_bytes.argtypes = [vp, ci, ci, ci]
    lib.agent_attn_workspace_bytes.restype = sz
    lib.agent_attn_forward.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ctypes.POINTER(AgentAttnBias), vp,
                                       vp, vp, sz, vp]
    lib.agent_attn_forward.restype = ci
    ll3 = ctypes.POINTER(ctypes.c_longlong)
    lib.agent_attn_forward_strided.argtypes = [vp, vp, vp, vp, vp, ll3, ci, ci, ci, ctypes.POINTER(AgentAttnBias), vp,
                                               vp, ll3, vp, ctypes.c_size_t, vp]
    lib.agent_attn_forward_strided.restype = ci
    lib.agent_attn_pool.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    lib.agent_attn_pool.restype = ci
    lib.agent_attn_aggregate.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp, sz, vp]
    lib.agent_attn_aggregate.restype = ci
    lib.agent_attn_broadcast.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, vp, vp]
    lib.agent_attn_broadcast.restype = ci
    lib.agent_attn_staging_bytes.argtypes = [vp, ci, ci, ci]
    lib.agent_attn_staging_bytes.restype = sz
    lib.agent_attn_forward_host.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ctypes.POINTER(AgentAttnBias), vp,
                                            vp, vp, sz, vp]
    lib.agent_attn_forward_host.restype = ci
    lib.agent_attn_query_status.argtypes = [vp, vp]
    lib.agent_attn_query_status.restype = ci
    lib.agent_attn_last_launch_count.argtypes = [vp]
    lib.agent_attn_last_launch_count.restype = ci
    lib.agent_attn_aggregate_static.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp]
    lib.agent_attn_aggregate_static.restype = ci
    lib.agent_attn_compose_bias.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, vp, vp]
    lib.agent_attn_compose_bias.restype = ci
    lib.agent_attn_backward_workspace_bytes.argtypes = [vp, ci, ci, ci]
    lib.agent_attn_backward_workspace_bytes.restype = sz
    lib.agent_attn_backward.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ctypes.POINTER(AgentAttnBias), vp,
                                        ctypes.POINTER(AgentAttnGrads), vp, sz, vp]
    lib.agent_attn_backward.restype = ci
    lib.agent_attn_test_set_stage_mask.argtypes = [vp, ctypes.c_uint]
    lib.agent_attn_test_set_stage_mask.restype = ci
    lib.agent_attn_test_set_poll_limit.argtypes = [vp, ctypes.c_uint]
    lib.agent_attn_test_set_poll_limit.restype = ci
    rot, nrm = ctypes.POINTER(AgentAttnRotary), ctypes.POINTER(AgentAttnNorm)
    lib.agent_attn_rotate.argtypes = [vp, vp, vp, ll3, ci, rot, nrm, vp, vp, ll3, vp]
    lib.agent_attn_rotate.restype = ci
    lib.agent_attn_rotate_workspace_bytes.argtypes = [vp]
    lib.agent_attn_rotate_workspace_bytes.restype = sz
    lib.agent_attn_rotate_backward.argtypes = [vp, vp, vp, ll3, vp, vp, ll3, ci, rot, nrm, vp, vp, ll3, vp, vp, vp, sz, vp]
    lib.agent_attn_rotate_backward.restype = ci
    gate, ggrads = ctypes.POINTER(AgentAttnGate), ctypes.POINTER(AgentAttnGateGrads)
    lib.agent_attn_gated_workspace_bytes.argtypes = [vp, ci, ci, ci, ci]
    lib.agent_attn_gated_workspace_bytes.restype = sz
    lib.agent_attn_gated.argtypes = [vp, gate, vp, vp, sz, vp]
    lib.agent_attn_gated.restype = ci
    for gradients in (lib.agent_attn_gated_backward, lib.agent_attn_gated_backward_two_terms):
        gradients.argtypes = [vp, gate, vp, ggrads, vp, sz, vp]
        gradients.restype = ci
    lib.agent_attn_static_scratch_bytes.argtypes = []
    lib.agent_attn_static_scratch_bytes.restype = sz
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _empty(shape, dtype: torch.dtype, device: torch.device, stream: torch.cuda.Stream) -> torch.Tensor:
    """Memory that work on `stream` may write at once: what the current stream's allocator hands out may still be read by earlier work there.  The
    current stream may use it, too, until it is freed."""
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _dense_like(t: Optional[torch.Tensor], stream=None):
    if t is None:
        return None
    if stream is None:                     # (half of the host time of torch.empty with type and device)
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return _empty(t.shape, t.dtype, t.device, stream)


def _dense(t: torch.Tensor, shape, stream=None):
    return t.new_empty(shape) if stream is None else _empty(shape, t.dtype, t.device, stream)


# torch.cuda.current_stream() builds a stream object (3.2 us); the raw handle costs 0.1 us
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream]):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _raw_device is not None:
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _bias(b1: Optional[torch.Tensor], b2: Optional[torch.Tensor]):
    return None if b1 is None and b2 is None else ctypes.byref(AgentAttnBias(_ptr(b1), _ptr(b2)))


class Rotary:
    """Rotary positions of a network's tokens (`agent_attn_rotary`): what `AgentAttention.rotate` turns queries and keys by.

    `channels` gives each axis (one to three: e.g. time, height, width) its number of channels of a head, an even one; `freq` the radians per
    unit of position of every pair, axis after axis, as an fp32 CUDA tensor of sum(channels) / 2 (`Rotary.frequencies` makes the usual ones).
    Positions are the tokens' places in the row-major grid `extent`, or `positions`, fp32 [B or 1, N, axes].  `pairs`: neighbouring channels
    form a pair; else channel i of an axis's segment and channel i + channels / 2.
    """

    def __init__(self, freq: torch.Tensor, channels, extent=None, positions: Optional[torch.Tensor] = None, pairs: bool = False):
        channels, axes = tuple(int(c) for c in channels), len(channels)
        if not 1 <= axes <= 3 or any(c < 0 or c % 2 for c in channels):
            raise ValueError(f"channels: expected one to three even numbers, got {channels}")
        if freq.shape != (sum(channels) // 2,) or freq.dtype is not torch.float32 or not freq.is_cuda or not freq.is_contiguous():
            raise ValueError(f"freq: expected a contiguous cuda float32 tensor of {sum(channels) // 2} values, got {tuple(freq.shape)} {freq.dtype} on {freq.device}")
        if positions is not None:
            if positions.dim() != 3 or positions.shape[2] != axes or positions.dtype is not torch.float32 or not positions.is_cuda or not positions.is_contiguous():
                raise ValueError(f"positions: expected a contiguous cuda float32 tensor [B or 1, N, {axes}], got {tuple(positions.shape)} {positions.dtype} on {positions.device}")
        elif extent is None or len(extent) != axes or any(not 0 < e <= _INT_MAX for e in extent):
            raise ValueError(f"extent: expected {axes} positive values of 32 bits, got {extent}")
        if positions is not None and positions.device != freq.device:
            raise ValueError(f"positions: expected them on {freq.device} with freq, got {positions.device}")
        self.freq, self.positions, self.channels, self.axes, self._index = freq, positions, channels, axes, None
        self.extent = (1,) * axes if extent is None else tuple(int(e) for e in extent)
        self._batch = 0 if positions is None else positions.shape[0]
        self._c = AgentAttnRotary(axes, (ctypes.c_int * 3)(*(self.extent if positions is None else ())), (ctypes.c_int * 3)(*channels), int(pairs), freq.data_ptr(), _ptr(positions),
                                  positions.shape[1] * axes if self._batch > 1 else 0)

    @staticmethod
    def frequencies(channels, theta: float = 100.0, device: int = 0) -> torch.Tensor:
        """theta ** (-i / pairs) for pair i of each axis."""
        return torch.tensor([theta ** (-i / (c // 2)) for c in channels for i in range(c // 2)], dtype=torch.float32, device=torch.device("cuda", device))

    def _check(self, batch: int, n_tokens: int, device: int):
        if self._index is None:
            self._index = self.freq.get_device()
        if self._index != device:
            raise ValueError(f"rotary: expected freq and positions on cuda:{device}, got {self.freq.device}")
        if self.positions is not None and (self.positions.shape[1] != n_tokens or self._batch not in (1, batch)):
            raise ValueError(f"positions: expected [{batch} or 1, {n_tokens}, {self.axes}], got {tuple(self.positions.shape)}")


class AgentAttention:
    """One `agent_attn_handle`.  Methods mirror the C entry points of the same names."""

    def __init__(self, batch: int, heads: int, head_dim: int, max_tokens: int, max_agents: int,
                 dtype: torch.dtype, scale1: float = 0.0, scale2: float = 0.0,
                 device: int = 0, path: int = AA_PATH_AUTO):
        self.lib = load_library()
        self.cfg = AgentAttnConfig(batch, heads, head_dim, max_tokens, max_agents, _DTYPES[dtype],
                                   scale1, scale2, device, path)
        self.dtype = dtype
        self.device, self._index = torch.device("cuda", device), device
        self.batch, self.heads, self.head_dim = batch, heads, head_dim
        self._h = ctypes.c_void_p()
        rc = self.lib.agent_attn_create(ctypes.byref(self._h), ctypes.byref(self.cfg))
        if rc != 0:
            self._h = ctypes.c_void_p()
            raise AgentAttnError(rc, "agent_attn_create failed (is an sm_100 GPU present?)")
        self._ws: Optional[torch.Tensor] = None
        self._staging: Optional[torch.Tensor] = None
        self._bytes: dict = {}             # scratch sizes by call shape: they depend on nothing else
        self._rotate_bytes: Optional[int] = None
        self._strides: dict = {}           # strides as the library takes them, by token count and strides

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self.lib.agent_attn_destroy(self._h)
            self._h = ctypes.c_void_p()

    __del__ = close

    # ------------------------------------------------------------------ helpers
    def _check(self, rc: int):
        if rc != 0:
            raise AgentAttnError(rc, self.lib.agent_attn_last_error(self._h).decode())

    def _chk_tensor(self, t: Optional[torch.Tensor], shape, name: str, cuda: bool = True):
        if t is None:
            return
        if t.shape != shape or t.dtype is not self.dtype or not t.is_contiguous() or t.get_device() != (self._index if cuda else -1):
            raise ValueError(f"{name}: expected contiguous {self.device if cuda else 'cpu'} {self.dtype} tensor of "
                             f"shape {tuple(shape)}, got {tuple(t.shape)} {t.dtype} on {t.device}")

    def _scratch_bytes(self, query: str, grid_h: int, grid_w: int, n_agents: int) -> int:
        key = (query, grid_h, grid_w, n_agents)
        need = self._bytes.get(key)
        if need is None:
            if len(self._bytes) >= 64:
                self._bytes.clear()
            need = self._bytes[key] = int(getattr(self.lib, query)(self._h, grid_h, grid_w, n_agents))
        return need

    def workspace_bytes(self, grid_h: int, grid_w: int, n_agents: int) -> int:
        return self._scratch_bytes("agent_attn_workspace_bytes", grid_h, grid_w, n_agents)

    def staging_bytes(self, grid_h: int, grid_w: int, n_agents: int) -> int:
        return self._scratch_bytes("agent_attn_staging_bytes", grid_h, grid_w, n_agents)

    def workspace(self, grid_h: int, grid_w: int, n_agents: int) -> torch.Tensor:
        need = self.workspace_bytes(grid_h, grid_w, n_agents)
        if need == 0:
            raise ValueError("shape not supported by this handle")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def intermediates(self, workspace: torch.Tensor, n_agents: int):
        """Views of the agents A and the agent features V_A ([B, heads, n, d] each) that `forward` left in its
        workspace: A occupies the first B*heads*n*d elements, V_A starts at the next multiple of 256 bytes."""
        count = self.batch * self.heads * n_agents * self.head_dim
        nbytes = count * workspace.new_empty(0, dtype=self.dtype).element_size()
        va_off = (nbytes + 255) // 256 * 256
        shape = (self.batch, self.heads, n_agents, self.head_dim)
        return (workspace[:nbytes].view(self.dtype).view(shape), workspace[va_off:va_off + nbytes].view(self.dtype).view(shape))

    def set_stage_mask(self, mask: int):
        """Measurement hook: which of the three streaming kernels `forward` launches (1 prep | 2 aggregation | 4 broadcast)."""
        self._check(self.lib.agent_attn_test_set_stage_mask(self._h, mask))

    def set_poll_limit(self, polls: int):
        """Test hook: polls of another block's counter before a wait of the task-queue kernel gives up."""
        self._check(self.lib.agent_attn_test_set_poll_limit(self._h, polls & 0xffffffff))

    def last_launch_count(self) -> int:
        return int(self.lib.agent_attn_last_launch_count(self._h))

    def query_status(self, stream=None) -> int:
        return int(self.lib.agent_attn_query_status(self._h, _stream_ptr(stream)))

    # ------------------------------------------------------------------ entry points
    def forward(self, q, k, v, grid_h: int, grid_w: int, n_agents: int, agents=None, b1=None, b2=None,
                dwc_weight=None, out=None, workspace=None, stream=None) -> torch.Tensor:
        B, h, d, N = self.batch, self.heads, self.head_dim, grid_h * grid_w
        for t, nm in ((q, "q"), (k, "k"), (v, "v")):
            self._chk_tensor(t, (B, h, N, d), nm)
        self._chk_tensor(agents, (B, h, n_agents, d), "agents")
        self._chk_tensor(b1, (h, n_agents, N), "b1")
        self._chk_tensor(b2, (h, N, n_agents), "b2")
        self._chk_tensor(dwc_weight, (h, d, 3, 3), "dwc_weight")
        if out is None:
            out = torch.empty_like(q)
        self._chk_tensor(out, (B, h, N, d), "out")
        ws = self.workspace(grid_h, grid_w, n_agents) if workspace is None else workspace
        self._check(self.lib.agent_attn_forward(
            self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(agents), grid_h, grid_w, n_agents,
            _bias(b1, b2), _ptr(dwc_weight), _ptr(out), _ptr(ws),
            ws.numel(), _stream_ptr(stream)))
        return out

    def forward_strided(self, q, k, v, grid_h: int, grid_w: int, n_agents: int, agents=None, b1=None, b2=None,
                        dwc_weight=None, out=None, workspace=None, stream=None) -> torch.Tensor:
        """Eq. 6 on VIEWS of shape [B, heads, N, d] with any batch / head / token strides (last dim contiguous).

        Typical use: `qkv` of shape [B, N, 3, heads, d] straight from a projection, passed as
        `qkv[:, :, i].permute(0, 2, 1, 3)`; `out` may be such a view of a [B, N, heads, d] tensor (that is
        what is allocated when `out` is None).  Q, K and V must share their strides.
        """
        B, h, d, N = self.batch, self.heads, self.head_dim, grid_h * grid_w
        for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
            if t is None:
                continue
            if t.shape != (B, h, N, d) or t.dtype is not self.dtype or t.get_device() != self._index or t.stride(3) != 1:
                raise ValueError(f"{nm}: expected a {self.device} {self.dtype} view of shape {(B, h, N, d)} with contiguous channels")
        if q.stride() != k.stride() or q.stride() != v.stride():
            raise ValueError("q, k and v must have the same strides")
        self._chk_tensor(agents, (B, h, n_agents, d), "agents")
        self._chk_tensor(b1, (h, n_agents, N), "b1")
        self._chk_tensor(b2, (h, N, n_agents), "b2")
        self._chk_tensor(dwc_weight, (h, d, 3, 3), "dwc_weight")
        if out is None:
            out = torch.empty((B, N, h, d), dtype=self.dtype, device=self.device).permute(0, 2, 1, 3)
        ws = self.workspace(grid_h, grid_w, n_agents) if workspace is None else workspace
        sin = (ctypes.c_longlong * 3)(q.stride(0), q.stride(1), q.stride(2))
        sout = (ctypes.c_longlong * 3)(out.stride(0), out.stride(1), out.stride(2))
        self._check(self.lib.agent_attn_forward_strided(
            self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(agents), sin, grid_h, grid_w, n_agents,
            _bias(b1, b2), _ptr(dwc_weight), _ptr(out), sout, _ptr(ws),
            ws.numel(), _stream_ptr(stream)))
        return out

    def backward_workspace(self, grid_h: int, grid_w: int, n_agents: int) -> torch.Tensor:
        nbytes = self._scratch_bytes("agent_attn_backward_workspace_bytes", grid_h, grid_w, n_agents)
        if nbytes == 0:
            raise AgentAttnError(2, f"backward does not support grid {grid_h}x{grid_w} with {n_agents} agents")
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def backward(self, q, k, v, d_out, grid_h: int, grid_w: int, n_agents: int, b1=None, b2=None,
                 dwc_weight=None, need_bias_grads: bool = True, need_filter_grad: bool = True,
                 workspace=None, stream=None) -> dict:
        """`agent_attn_backward`: fp32 gradients of Eq. 6 (pooled agents) for the upstream gradient `d_out`.

        Returns a dict with `dq`, `dk`, `dv` ([B, heads, N, d]) and, for the inputs that were given and asked
        for, `db1` ([heads, n, N]), `db2` ([heads, N, n]) and `dwd` ([heads, d, 3, 3]).
        """
        B, h, d, N = self.batch, self.heads, self.head_dim, grid_h * grid_w
        for t, nm in ((q, "q"), (k, "k"), (v, "v"), (d_out, "d_out")):
            if t is None:
                raise ValueError(f"{nm} is required")
            self._chk_tensor(t, (B, h, N, d), nm)
        self._chk_tensor(b1, (h, n_agents, N), "b1")
        self._chk_tensor(b2, (h, N, n_agents), "b2")
        self._chk_tensor(dwc_weight, (h, d, 3, 3), "dwc_weight")
        f32, like = torch.float32, torch.empty_like
        g = {"dq": like(q, dtype=f32), "dk": like(q, dtype=f32), "dv": like(q, dtype=f32)}
        if b1 is not None and need_bias_grads:
            g["db1"] = like(b1, dtype=f32)
        if b2 is not None and need_bias_grads:
            g["db2"] = like(b2, dtype=f32)
        if dwc_weight is not None and need_filter_grad:
            g["dwd"] = like(dwc_weight, dtype=f32)
        ws = self.backward_workspace(grid_h, grid_w, n_agents) if workspace is None else workspace
        grads = AgentAttnGrads(_ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]), _ptr(g.get("db1")), _ptr(g.get("db2")),
                               _ptr(g.get("dwd")))
        self._check(self.lib.agent_attn_backward(
            self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(d_out), grid_h, grid_w, n_agents,
            _bias(b1, b2), _ptr(dwc_weight), ctypes.byref(grads), _ptr(ws),
            ws.numel(), _stream_ptr(stream)))
        return g

    def pool(self, q, grid_h: int, grid_w: int, pool_h: int, pool_w: int, out=None, stream=None):
        B, h, d = self.batch, self.heads, self.head_dim
        self._chk_tensor(q, (B, h, grid_h * grid_w, d), "q")
        if out is None:
            out = torch.empty((B, h, pool_h * pool_w, d), dtype=self.dtype, device=self.device)
        self._chk_tensor(out, (B, h, pool_h * pool_w, d), "out")
        self._check(self.lib.agent_attn_pool(self._h, _ptr(q), grid_h, grid_w, pool_h, pool_w, _ptr(out),
                                             _stream_ptr(stream)))
        return out

    def aggregate(self, agents, k, v, b1=None, out=None, workspace=None, stream=None):
        B, h, d = self.batch, self.heads, self.head_dim
        n, N = agents.shape[2], k.shape[2]
        self._chk_tensor(agents, (B, h, n, d), "agents")
        self._chk_tensor(k, (B, h, N, d), "k")
        self._chk_tensor(v, (B, h, N, d), "v")
        self._chk_tensor(b1, (h, n, N), "b1")
        if out is None:
            out = torch.empty_like(agents)
        ws = self.workspace(1, N, n) if workspace is None else workspace
        self._check(self.lib.agent_attn_aggregate(self._h, _ptr(agents), _ptr(k), _ptr(v), _ptr(b1), N, n,
                                                  _ptr(out), _ptr(ws), ws.numel(), _stream_ptr(stream)))
        return out

    def aggregate_static(self, agents, k, v, b1=None, out=None, stream=None):
        """`agent_attn_aggregate_static`: the aggregation for callers that cannot allocate.

        Same result as `aggregate`, but the split partials live in the library's fixed 32 MiB
        array instead of a workspace, so this call allocates nothing when `out` is given.
        Calls that overlap on the GPU share that array and must be serialised.
        """
        B, h, d = self.batch, self.heads, self.head_dim
        n, N = agents.shape[2], k.shape[2]
        self._chk_tensor(agents, (B, h, n, d), "agents")
        self._chk_tensor(k, (B, h, N, d), "k")
        self._chk_tensor(v, (B, h, N, d), "v")
        self._chk_tensor(b1, (h, n, N), "b1")
        if out is None:
            out = torch.empty_like(agents)
        self._check(self.lib.agent_attn_aggregate_static(self._h, _ptr(agents), _ptr(k), _ptr(v), _ptr(b1),
                                                         N, n, _ptr(out), _stream_ptr(stream)))
        return out

    def broadcast(self, q, agents, va, v, grid_h: int, grid_w: int, b2=None, dwc_weight=None, out=None,
                  stream=None):
        B, h, d, N = self.batch, self.heads, self.head_dim, grid_h * grid_w
        n = agents.shape[2]
        self._chk_tensor(q, (B, h, N, d), "q")
        self._chk_tensor(agents, (B, h, n, d), "agents")
        self._chk_tensor(va, (B, h, n, d), "va")
        self._chk_tensor(v, (B, h, N, d), "v")
        self._chk_tensor(b2, (h, N, n), "b2")
        self._chk_tensor(dwc_weight, (h, d, 3, 3), "dwc_weight")
        if out is None:
            out = torch.empty_like(q)
        self._check(self.lib.agent_attn_broadcast(self._h, _ptr(q), _ptr(agents), _ptr(va), _ptr(v), _ptr(b2),
                                                  _ptr(dwc_weight), grid_h, grid_w, n, _ptr(out),
                                                  _stream_ptr(stream)))
        return out

    def compose_bias(self, col, row, blk, grid_h: int, grid_w: int, n_agents: int, transpose: bool = False,
                     out=None, stream=None):
        """`agent_attn_compose_bias`: dense B1 ([heads, n, N]) or B2 ([heads, N, n], transpose=True)
        from column [heads, n, w], row [heads, n, h] and block [heads, n, h0, w0] components (App. B)."""
        h, N = self.heads, grid_h * grid_w
        self._chk_tensor(col, (h, n_agents, grid_w), "col")
        self._chk_tensor(row, (h, n_agents, grid_h), "row")
        h0, w0 = (blk.shape[2], blk.shape[3]) if blk is not None else (1, 1)
        self._chk_tensor(blk, (h, n_agents, h0, w0), "blk")
        shape = (h, N, n_agents) if transpose else (h, n_agents, N)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        self._chk_tensor(out, shape, "out")
        self._check(self.lib.agent_attn_compose_bias(self._h, _ptr(col), _ptr(row), _ptr(blk), h0, w0, grid_h, grid_w,
                                                     n_agents, int(transpose), _ptr(out), _stream_ptr(stream)))
        return out

    def forward_host(self, q, k, v, grid_h: int, grid_w: int, n_agents: int, agents=None, b1=None, b2=None,
                     dwc_weight=None, out=None, stream=None, synchronize: bool = True, staging=None) -> torch.Tensor:
        """Eq. 6 on host (ideally pinned) tensors: copies in, runs, copies the result back.

        Everything is queued on `stream`.  `staging` is the device scratch of the call (uint8, at least
        `staging_bytes(...)`); calls that are in flight at the same time on different streams (to overlap one
        step's copies with the next) need a staging buffer each.  By default the module keeps one of its own.
        """
        B, h, d, N = self.batch, self.heads, self.head_dim, grid_h * grid_w
        for t, nm in ((q, "q"), (k, "k"), (v, "v")):
            self._chk_tensor(t, (B, h, N, d), nm, cuda=False)
        self._chk_tensor(agents, (B, h, n_agents, d), "agents", cuda=False)
        self._chk_tensor(b1, (h, n_agents, N), "b1", cuda=False)
        self._chk_tensor(b2, (h, N, n_agents), "b2", cuda=False)
        self._chk_tensor(dwc_weight, (h, d, 3, 3), "dwc_weight", cuda=False)
        if out is None:
            out = torch.empty((B, h, N, d), dtype=self.dtype).pin_memory()
        self._chk_tensor(out, (B, h, N, d), "out", cuda=False)
        need = self.staging_bytes(grid_h, grid_w, n_agents)
        if need == 0:
            raise ValueError("shape not supported by this handle")
        if staging is not None:
            if staging.dtype != torch.uint8 or not staging.is_cuda or staging.numel() < need:
                raise ValueError(f"staging must be a CUDA uint8 tensor of at least {need} bytes")
        else:
            if self._staging is None or self._staging.numel() < need:
                self._staging = torch.empty(need, dtype=torch.uint8, device=self.device)
            staging = self._staging
        s = torch.cuda.current_stream() if stream is None else stream
        self._check(self.lib.agent_attn_forward_host(
            self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(agents), grid_h, grid_w, n_agents,
            _bias(b1, b2), _ptr(dwc_weight), _ptr(out),
            _ptr(staging), staging.numel(), s.cuda_stream))
        if synchronize:
            s.synchronize()
        return out

    # ------------------------------------------------------------------ queries and keys before the attention
    def _chk_views(self, names, tensors, n_tokens: int, dtype: torch.dtype):
        """Views of shape [B, heads, N, d] that share their strides, or None; the strides as the library takes them (None: dense)."""
        shape, strides, dense = (self.batch, self.heads, n_tokens, self.head_dim), None, True
        for name, t in zip(names, tensors):
            if t is None:
                continue
            if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index:
                raise ValueError(f"{name}: expected a {self.device} {dtype} view of shape {shape} with contiguous channels, got {tuple(t.shape)} {t.dtype} on {t.device}")
            if not t.is_contiguous():
                dense = False
        if dense:
            return None
        for name, t in zip(names, tensors):
            if t is None:
                continue
            st = t.stride()
            if st == strides:
                continue
            if st[3] != 1:
                raise ValueError(f"{name}: expected contiguous channels, got strides {st}")
            if strides is not None and any(n > 1 and s != o for n, s, o in zip(shape, st, strides)):       # (of a single entry no stride is used)
                raise ValueError(f"{name}: expected the strides {strides} of the other tensor, got {st}")
            strides = st if strides is None else strides
        key = (n_tokens, strides)
        got = self._strides.get(key)
        if got is None:
            if len(self._strides) >= 64:
                self._strides.clear()
            got = self._strides[key] = (ctypes.c_longlong * 3)(*(s if n > 1 else self.head_dim for n, s in zip(shape, strides[:3])))
        return got

    def _tokens(self, t: torch.Tensor) -> int:
        N = t.shape[2] if t.dim() == 4 else 0
        if N > self.cfg.max_tokens:                        # (the library's count has 32 bits)
            raise AgentAttnError(2, f"N={N} exceeds the handle's max_tokens={self.cfg.max_tokens}")
        return N

    def _norm(self, q_gain, k_gain, eps):
        if eps is None:
            if q_gain is not None or k_gain is not None:
                raise ValueError("a gain belongs to a norm: give eps")
            return None
        self._chk_tensor(q_gain, (self.head_dim,), "q_gain")
        self._chk_tensor(k_gain, (self.head_dim,), "k_gain")
        return ctypes.byref(AgentAttnNorm(_ptr(q_gain), _ptr(k_gain), eps))

    def rotate(self, q, k, rotary: Optional[Rotary] = None, q_gain=None, k_gain=None, eps: Optional[float] = None, out=None, stream=None):
        """`agent_attn_rotate`: queries and keys as the attention takes them, with an RMS norm of each head (where `eps` is given) and rotary
        positions.

        `q` and `k` are views of shape [B, heads, N, d] with contiguous channels and the same strides (either may be None); `out` is a pair of
        such views, by default new dense tensors.  `out=(q, k)` works in place: `qkv[:, :, i].permute(0, 2, 1, 3)` of a fused projection can be
        prepared where `forward_strided` reads it.  Returns (q_out, k_out).
        """
        some = q if q is not None else k
        if some is None:
            raise ValueError("q or k is required")
        N = self._tokens(some)
        sin = self._chk_views(("q", "k"), (q, k), N, self.dtype)
        if rotary is not None:
            rotary._check(self.batch, N, self._index)
        norm = self._norm(q_gain, k_gain, eps)
        if out is None:
            out, sout = (_dense_like(q, stream), _dense_like(k, stream)), None
        else:
            if any((t is None) != (o is None) for t, o in zip((q, k), out)):
                raise ValueError("out: expected a tensor for each of q and k that is given")
            sout = self._chk_views(("out[0]", "out[1]"), out, N, self.dtype)
        self._check(self.lib.agent_attn_rotate(self._h, _ptr(q), _ptr(k), sin, N, None if rotary is None else ctypes.byref(rotary._c), norm,
                                               _ptr(out[0]), _ptr(out[1]), sout, _stream_ptr(stream)))
        return out[0], out[1]

    def rotate_backward(self, dq_out, dk_out, rotary: Optional[Rotary] = None, q=None, k=None, q_gain=None, k_gain=None,
                        eps: Optional[float] = None, out=None, workspace=None, stream=None) -> dict:
        """`agent_attn_rotate_backward`: from the fp32 gradients of `rotate`'s results (what `backward` returns as `dq`, `dk`), those of its inputs.

        `q`, `k` (the inputs of the forward call) are needed with a norm only.  Returns a dict with fp32 `dq`, `dk` ([B, heads, N, d]; `out`, a pair
        of views, which may be the gradients given) and, for the gains that were given, `dq_gain`, `dk_gain` ([d]).
        """
        some = dq_out if dq_out is not None else dk_out
        if some is None:
            raise ValueError("dq_out or dk_out is required")
        N = self._tokens(some)
        f32 = torch.float32
        sgrad = self._chk_views(("dq_out", "dk_out"), (dq_out, dk_out), N, f32)
        if rotary is not None:
            rotary._check(self.batch, N, self._index)
        norm = self._norm(q_gain, k_gain, eps)
        sin = None
        if norm is not None:
            if (dq_out is not None and q is None) or (dk_out is not None and k is None):
                raise ValueError("the gradient of a norm needs q and k")
            sin = self._chk_views(("q", "k"), (q, k), N, self.dtype)
        if out is None:
            out, sout = (_dense_like(dq_out, stream), _dense_like(dk_out, stream)), None
        else:
            if any((t is None) != (o is None) for t, o in zip((dq_out, dk_out), out)):
                raise ValueError("out: expected a tensor for each gradient that is given")
            sout = self._chk_views(("out[0]", "out[1]"), out, N, f32)
        got = {name: t for name, t in zip(("dq", "dk"), out) if t is not None}
        for name, gain, grad in (("dq_gain", q_gain, dq_out), ("dk_gain", k_gain, dk_out)):
            if gain is not None and grad is not None:
                got[name] = _dense(grad, (self.head_dim,), stream)
        if norm is None:
            workspace = None               # (not read)
        elif workspace is not None:
            self._chk_workspace(workspace)
        else:
            if self._rotate_bytes is None:
                self._rotate_bytes = int(self.lib.agent_attn_rotate_workspace_bytes(self._h))
            workspace = self._scratch(self._rotate_bytes, stream)
        self._check(self.lib.agent_attn_rotate_backward(
            self._h, _ptr(dq_out), _ptr(dk_out), sgrad, _ptr(q), _ptr(k), sin, N, None if rotary is None else ctypes.byref(rotary._c), norm,
            _ptr(out[0]), _ptr(out[1]), sout, _ptr(got.get("dq_gain")), _ptr(got.get("dk_gain")),
            _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_ptr(stream)))
        return got

    # ------------------------------------------------------------------ gated feed-forward product
    def _gate(self, x, w_gate, w_up, b_gate, b_up, activation):
        if activation not in _ACTIVATIONS:
            raise ValueError(f"activation: expected one of {sorted(_ACTIVATIONS)}, got {activation!r}")
        if x.dim() == 0 or w_gate.dim() != 2:
            raise ValueError(f"expected x [..., channels] and weights [hidden, channels], got {tuple(x.shape)} and {tuple(w_gate.shape)}")
        F, C = w_gate.shape
        self._chk_tensor(x, x.shape[:-1] + (C,), "x")
        for t, name in ((w_gate, "w_gate"), (w_up, "w_up")):
            self._chk_tensor(t, (F, C), name)
        if b_gate is not None:
            self._chk_tensor(b_gate, (F,), "b_gate")
        if b_up is not None:
            self._chk_tensor(b_up, (F,), "b_up")
        rows = x.numel() // C if C else 0
        if rows > _INT_MAX or C > _INT_MAX or F > _INT_MAX:
            rows, C, F = (min(n, _INT_MAX) for n in (rows, C, F))                              # (which the library refuses)
        return AgentAttnGate(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(b_gate), _ptr(b_up), rows, C, F, _ACTIVATIONS[activation])

    def _gate_workspace(self, gate, backward: int, workspace, stream):
        """The workspace of a call: the caller's, or a new one where one is needed."""
        if workspace is not None:
            self._chk_workspace(workspace)
            return workspace
        key = (gate.rows, gate.channels, gate.hidden, backward)
        need = self._bytes.get(key)
        if need is None:
            if len(self._bytes) >= 64:
                self._bytes.clear()
            need = self._bytes[key] = int(self.lib.agent_attn_gated_workspace_bytes(self._h, *key))
        return self._scratch(need, stream)

    def _chk_workspace(self, t: torch.Tensor):
        if t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"workspace: expected a contiguous {self.device} tensor, got one on {t.device}")

    def _scratch(self, nbytes: int, stream) -> Optional[torch.Tensor]:
        """Memory of one call on `stream`."""
        if nbytes == 0:
            return None
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device) if stream is None else _empty(nbytes, torch.uint8, self.device, stream)

    def gated(self, x, w_gate, w_up, b_gate=None, b_up=None, activation: str = "silu", out=None, workspace=None, stream=None) -> torch.Tensor:
        """`agent_attn_gated`: act(x w_gate^T + b_gate) * (x w_up^T + b_up) for x [..., channels] and weights [hidden, channels].

        `activation`: "silu", "gelu" (erf) or "gelu_tanh".  The halves of one fused weight [2 hidden, channels] are `weight.chunk(2)`.
        """
        gate = self._gate(x, w_gate, w_up, b_gate, b_up, activation)
        shape = x.shape[:-1] + (gate.hidden,)
        if out is None:
            out = _dense(x, shape, stream)
        else:
            self._chk_tensor(out, shape, "out")
        ws = self._gate_workspace(gate, 0, workspace, stream)
        self._check(self.lib.agent_attn_gated(self._h, ctypes.byref(gate), _ptr(out), _ptr(ws), 0 if ws is None else ws.numel(), _stream_ptr(stream)))
        return out

    def gated_backward(self, x, w_gate, w_up, d_out, b_gate=None, b_up=None, activation: str = "silu", need_input_grad: bool = True,
                       need_weight_grads: bool = True, workspace=None, stream=None, two_terms: bool = False, need_bias_grads: Optional[bool] = None) -> dict:
        """`agent_attn_gated_backward` (`…_two_terms`): gradients of `gated` for the upstream gradient `d_out`, in the element type.

        Returns a dict with `dx`, `dw_gate`, `dw_up` and `db_gate`, `db_up`: these by default with the weights' gradients and only where both
        biases are given (one alone: a warning); `need_bias_grads=True` returns that of each bias that is given, `False` none.
        `two_terms` (16-bit types): the projections' gradients are not rounded to the element type on the way, so that each result is rounded
        once; some 2.4 times the time.
        """
        gate = self._gate(x, w_gate, w_up, b_gate, b_up, activation)
        self._chk_tensor(d_out, x.shape[:-1] + (gate.hidden,), "d_out")
        g = {}
        dx = dw_gate = dw_up = db_gate = db_up = None
        if need_input_grad:
            g["dx"] = dx = _dense_like(x, stream)
        if need_weight_grads:
            g["dw_gate"], g["dw_up"] = dw_gate, dw_up = _dense_like(w_gate, stream), _dense_like(w_up, stream)
        one = (b_gate is None) != (b_up is None)
        if need_bias_grads is None:
            need_bias_grads = need_weight_grads and not one
            if need_weight_grads and one:
                warnings.warn("gated_backward: the gradient of a bias without the other one is returned with need_bias_grads=True only", stacklevel=2)
        some = b_up if b_gate is None else b_gate
        if need_bias_grads and some is not None:           # (the library sums both)
            db_gate, db_up = _dense_like(some, stream), _dense_like(some, stream)
            if b_gate is not None:
                g["db_gate"] = db_gate
            if b_up is not None:
                g["db_up"] = db_up
        grads = AgentAttnGateGrads(_ptr(dx), _ptr(dw_gate), _ptr(dw_up), _ptr(db_gate), _ptr(db_up))
        ws = self._gate_workspace(gate, 2 if two_terms else 1, workspace, stream)
        call = self.lib.agent_attn_gated_backward_two_terms if two_terms else self.lib.agent_attn_gated_backward
        self._check(call(self._h, ctypes.byref(gate), _ptr(d_out), ctypes.byref(grads), _ptr(ws), 0 if ws is None else ws.numel(), _stream_ptr(stream)))
        return g
