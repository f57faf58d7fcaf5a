"""Host side of the operators around the attention that needs no GPU: null handles at the C ABI, struct layouts."""
import os
import re

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
