"""What the threads of kv_attention_rows.cu tell one another through shared memory, read off the source.

Two accesses without a barrier between them go wrong once in a great many runs, or on the next device, so no run shows their order.
"""
import os
import re

import pytest

from paper_2601_17818_b200.build import CSRC


@pytest.fixture(scope="module")
def kernel():
    """The kernel's body, without comments."""
    with open(os.path.join(CSRC, "kv_attention_rows.cu")) as fh:
        code = "".join(re.sub(r"//.*", "", line) for line in fh)
    start = code.index("cache_attention_rows_kernel(RowsArgs k) {")
    return code[start:code.index("row_anew(const AttArgs& a")]


def test_a_rows_two_sums_do_not_take_the_place_of_its_maxima(kernel):
    """A thread reads its partner's maximum behind a barrier and meets no other until the sums are written: they go elsewhere."""
    softmax = kernel[kernel.index("for (int i = 0; i < n; ++i)"):kernel.index("float* const turn")]
    written = re.findall(r"(\w+)\[half \* kRows \+ rl\] = (\w+);", softmax)
    read = re.findall(r"(\w+)\[\(half \^ 1\) \* kRows \+ rl\]", softmax)
    assert [value for _, value in written] == ["high", "sum"]
    assert written[0][0] != written[1][0] and [name for name, _ in written] == read
    with open(os.path.join(CSRC, "kv_attention_rows.cu")) as fh:
        at = dict(re.findall(r"static constexpr int (kPairs|kEnds|kTable) = (\w+ \+ \d+);", fh.read()))
    assert at == {"kPairs": "kBars + 256", "kEnds": "kPairs + 1024", "kTable": "kEnds + 1024"}      # (2 * 128 * 4 bytes each)


def test_the_row_of_ones_is_written_in_front_of_the_first_barrier(kernel):
    """A CTA without a tile turns its output in the bytes of the first stage, where the ones are, and meets no barrier on the way."""
    ones, barrier, turn = kernel.index("0x3C003C00u"), kernel.index("__syncthreads();"), kernel.index("float* const turn")
    assert ones < barrier < turn
