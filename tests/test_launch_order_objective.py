"""The launch rules of tik_ptx.cuh for the kernels of the policy loss, the log-probability gradient and the AdamW step."""
import os
import re

from paper_2609_35140_b200 import build


def _text(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def _kernels(name):
    """name -> body, without what follows a kernel in the file"""
    found = {}
    for part in _text(name).split("__global__")[1:]:
        head = re.search(r"\b(\w+_kernel)\s*\(", part)
        at = part.index("{", head.end())
        depth = 0
        for i in range(at, len(part)):
            depth += {"{": 1, "}": -1}.get(part[i], 0)
            if depth == 0:
                found[head.group(1)] = part[at:i + 1]
                break
    return found


def test_tensor_memory_is_taken_before_dependents_are_released():
    body = _kernels("tik_logprob_bwd.cu")["lpb_kernel"]
    take, wait, release = body.index("lpb_take_tensor_memory("), body.index("pdl_wait()"), body.index("pdl_launch_dependents()")
    assert take < wait < release and wait < body.index("__syncthreads()") < release
    assert body.count("pdl_wait()") == body.count("pdl_launch_dependents()") == 1
    helper = _text("tik_logprob_bwd.cu").split("lpb_take_tensor_memory(", 1)[1].split("}")[0]
    assert "tmem_alloc_pair(" in helper and "tmem_relinquish_pair(" in helper


def test_every_thread_waits_before_it_reads():
    """The wait stands in a kernel's outermost block behind no return, and nothing but parameters is touched before it."""
    for name in ("tik_loss.cu", "tik_logprob_bwd.cu", "tik_adamw.cu"):
        kernels = _kernels(name)
        assert kernels
        for kernel, body in kernels.items():
            before = body[:body.index("pdl_wait()")]
            assert before.count("{") - before.count("}") == 1 and "return" not in before, kernel
            assert not re.search(r"\bp\.(logprob|old_logprob|advantage|weight|ref|cu|count|part|ticket|target|lse|d_logprob|sum|norm|lr_device|step_device)\s*\[", before), kernel
            assert body.index("pdl_wait()") < body.index("pdl_launch_dependents()"), kernel
