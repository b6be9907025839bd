"""Products of the workers' matrices: what holds without a GPU, by the sources, by arithmetic and by what the entry points refuse."""
import glob
import os
import re

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_22549_b200", "csrc")


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


def test_where_the_header_says_that_singular_values_end():
    """The default triples, five steps, in exact arithmetic up to 64 bits: the smallest singular value of the statement, its range, and what smaller ones grow by."""
    text = " ".join(open(os.path.join(ROOT, "include", "desloc.h")).read().replace("\n *", " ").split())
    first, low, high = map(float, re.search(r"those of (\S+) and more of \|U\|_F within (\S+) \.\. (\S+) in five steps", text).groups())
    a, small, to = map(float, re.search(r"smaller ones grow by (\S+) a step at most \((\S+) to ([\d.]+)\)", text).groups())
    host = open(os.path.join(CSRC, "desloc_host.cu")).read()
    triple = [float(v) for v in re.search(r"kNewtonSchulz\[3\] = \{([^}]*)\}", host).group(1).replace("f", "").split(",")]

    def after(s, steps=5):
        for _ in range(steps):
            s = s * (triple[0] + s ** 2 * (triple[1] + s ** 2 * triple[2]))
        return s

    ends = after(np.exp(np.linspace(np.log(first), 0.0, 1_000_001)))
    assert low <= ends.min() < low + 0.01 and high - 0.01 < ends.max() <= high
    assert after(0.95 * first) < after(first) and after(np.array(small)) == np.clip(after(np.array(small)), to - 0.005, to + 0.005)
    below = np.exp(np.linspace(np.log(1e-7), np.log(first), 1001))
    assert a == triple[0] and np.all(after(below) <= a ** 5 * below)
