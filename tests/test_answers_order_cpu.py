"""The order that the kernels over a model's answers keep on the device, read from their sources
(what goes wrong without it may be rare, or a fault): a block writes into another's shared memory
only after every block of the cluster has begun, and a kernel that may begin while the one before
it ends waits before it reads or writes."""
import os
import re

import pytest

from paper_2602_10729_gb300 import build as bld


def functions(name):
    """(name, body) of each device function and kernel of a source file, without comments."""
    with open(os.path.join(bld.CSRC, name)) as f:
        text = re.sub(r"//[^\n]*|__launch_bounds__\([^)]*\)", "", f.read())
    for m in re.finditer(r"__(?:global|device)__[^;{]*?(\w+)\s*\([^;{]*\)\s*(?:const\s*)?{", text):
        if m.group(1) in ("if", "for", "while"):
            continue
        depth, end = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield m.group(1), text[m.end():end]


@pytest.mark.parametrize("name,of", [
    ("logprobs.cu", {"token_logprobs_kernel", "token_logprobs_grad_kernel"}),
    ("scores.cu", {"cluster_join"})])
def test_peers_are_written_once_their_blocks_run(name, of):
    bodies = dict(functions(name))
    assert {n for n, b in bodies.items() if "store_peer(" in b or "add_peer(" in b} == of
    for n in of:
        first = re.search(r"store_peer\(|add_peer\(", bodies[n]).start()
        before = bodies[n][:first]
        assert "cluster_runs();" in before, n
        begin = bodies[n] if n != "cluster_join" else bodies["for_answers"]
        at = begin.index("cluster_begin();")
        assert at < begin.index("cluster_runs();" if n != "cluster_join" else "cluster_join("), n


@pytest.mark.parametrize("name", ["logprobs.cu", "scores.cu", "route.cu"])
def test_kernels_wait_before_they_read_or_write(name):
    """The wait is unconditional and comes before any access to an argument's array."""
    bodies = dict(functions(name))
    waiting = {n for n, b in bodies.items() if "pdl_wait();" in b}
    for n in waiting:
        assert bodies[n].count("pdl_wait();") == 1, n
        before = bodies[n][:bodies[n].index("pdl_wait();")]
        assert not re.search(r"\w\[|if \([^)]*\)\s*$|for \(", re.sub(r"__shared__[^;]*;", "", before)), n
    kernels = [n for n in bodies if n.endswith("_kernel")]
    assert len(kernels) >= 2
    for n in kernels:
        if n in waiting:
            continue
        first = re.search(r"\b(%s)(<\w+>)?\(" % "|".join(waiting), bodies[n])
        assert first, n
        assert not re.search(r"load_\w+\(|logit_at\(|A\.bias\[",
                             bodies[n][:first.start()].replace("begin_load(", "")), n
