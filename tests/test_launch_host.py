"""What the attention calls keep from one launch to the next, by reading their source: a failure of the
runtime is not for a test to bring about."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_03910_gb300", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_a_failure_is_not_kept():
    """The registers that a launch has are kept once they are known only, so that a call after one for
    which the runtime had no answer asks again."""
    for name in ("attn_chunk.cu", "attn_prompt.cu"):
        text = source(name)
        assert "if (launch_registers<kernel>() < kLaunchRegs) return NETKV_ECUDA;" in text
        assert "cudaFuncGetAttributes" not in text and "static const int" not in text
    text = source("kv_common.cuh")
    ask = text[text.index("int launch_registers("):]
    ask = ask[:ask.index("\n}\n")]
    got = ask.index("cudaFuncGetAttributes(&has, kKernel) == cudaSuccess")
    assert got < ask.index("known.store(") < ask.index("else") < ask.index("cudaGetLastError()")
