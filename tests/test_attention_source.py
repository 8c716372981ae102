"""What cannot be shown by running the kernels of rotary positions and of the attention over bf16 rows: read off their sources and the compiler's messages (no GPU)."""
import os
import re

from paper_2601_17818_b200.build import CSRC


def _code(name):
    with open(os.path.join(CSRC, name)) as fh:
        return re.sub(r"//.*", "", fh.read())


def _body(code, head):
    """A function's text, from its head to the brace that closes it."""
    at = code.index(head)
    begin = code.index("{", at)
    depth = 0
    for i in range(begin, len(code)):
        depth += (code[i] == "{") - (code[i] == "}")
        if depth == 0:
            return code[begin:i + 1]
    raise AssertionError(head)


def test_all_lanes_see_what_the_lane_that_asks_a_barrier_sees():
    """One lane asks, the others learn of it by a vote, which orders no memory: before any of them goes on, the warp's lanes have to be ordered."""
    code = _code("attention_tiles.cu")
    wait = _body(code, "bool warp_wait(")
    assert len(re.findall(r"return true", wait)) == 1
    assert re.search(r"if \(asked\(bar, parity\)\) \{\s*__syncwarp\(\);\s*return true;", wait)
    assert '"memory"' in _body(code, "bool asked(") and code.count("asked(") == 2              # (nothing else asks that way)


def test_nothing_is_read_as_constant_beside_a_kernel_that_may_write_it():
    """The kernels are launched while the one in front is still running: what it writes is not constant for as long as they run, as reads through the read-only cache
    ask for."""
    for name in ("rotary.cu", "attention.cu", "attention_tiles.cu", "attention.cuh"):
        assert not re.search(r"__ldg\(|ld\.global\.nc|__restrict__", _code(name)), name
