"""Products of the workers' matrices: what holds without a GPU, by the sources, by arithmetic and by what the entry points refuse."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_22549_b200", "csrc")


def kernels():
    """(name, body) of every kernel of the library."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__\s+void[^{;]*?(\w+)\((?:[^(){};]|\([^()]*\))*\)\s*\{", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            yield m.group(1), text[m.end():at]


def test_no_kernel_lets_the_next_begin_before_its_blocks_have_their_tmem():
    """A block of the next kernel may take an SM's TMEM and hold it until this kernel ends: a block that has begun and not yet asked for its own would wait for ever."""
    bodies = dict(kernels())
    takers = {name for name, body in bodies.items() if "tcgen05.alloc" in body}
    assert {"gemm_kernel", "orth_small_kernel"} <= takers
    for name in takers:
        body = bodies[name]
        assert body.count("begin_and_let_next_begin()") == 1
        begin = body.index("begin_and_let_next_begin()")
        assert body.rindex("tcgen05.alloc") < begin < body.index("wait_for_earlier_kernels()"), f"{name}: the next kernel may begin before this block has its TMEM"
