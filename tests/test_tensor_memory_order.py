"""The order in which kernels take tensor memory, read from their sources.

A kernel that is the programmatic dependent of the one before it may start while that
one runs.  If it takes its columns first and then waits, a kernel that lets it start
early and allocates later can wait for those columns for ever; the same holds for a
kernel that lets the next one start before it has its own.  Neither can be run."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_06751_gb300", "csrc")


def kernels():
    """(file, name, head, body) of each kernel that takes tensor memory."""
    found = []
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"__global__", text):
            brace = text.index("{", m.start())
            head, depth, i = text[m.start():brace], 1, brace + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[i], 0)
                i += 1
            if "tensor_alloc<" in text[brace:i]:
                found.append((name, re.search(r"(\w+_kernel)\s*\(", head).group(1), head, text[brace:i], text))
    return found


@pytest.mark.parametrize("kernel", kernels(), ids=lambda k: f"{k[0]}:{k[1]}")
def test_columns_between_wait_and_trigger(kernel):
    _, name, head, body, text = kernel
    if "__cluster_dims__(2" in head:  # pairs: no other CTA fits on their SMs, whatever it holds
        if "kSmemMost" in text:
            assert "size_t smem = kSmemMost - kSmemBarriers;" in text
            smem = 1024 * (int(re.search(r"kSmemMost = (\d+) \* 1024", text).group(1)) - 1)
            assert re.search(r"kSmemBarriers = 1024\b", text)
        else:
            assert "size_t smem = kSmem;" in text
            smem = 1024 * int(re.search(r"kSmem = (\d+) \* 1024", text).group(1))
        # an SM has 228 KB; every CTA takes 1 KB besides its own, and these have barriers of some hundred bytes
        assert "__shared__ uint64_t full[kMaxStages]" in body
        assert 228 * 1024 - (smem + 1024 + 128) < 1024
        return
    at = [body.index(w) for w in ("griddep_wait()", "tensor_alloc<", "__syncthreads()", "griddep_launch_dependents()")]
    assert at == sorted(at), name
    for w in ("griddep_wait()", "tensor_alloc<", "griddep_launch_dependents()"):
        assert body.count(w) == 1, (name, w)
    free = body.index("tensor_free<")
    assert "cluster_sync()" not in body[:free], name  # given back before it waits for its cluster


def test_kernels_found():
    assert {k[1] for k in kernels()} == {"ffn_pair_kernel", "ffn_split_kernel", "ffn_parts_kernel"}
