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


def test_sums_of_positions_stay_within_32_bits(tmp_path):
    """What a query sees of 32 rows, compiled for the host with signed overflow as an error: windows of 2^31 - 1 rows, rows in front of, inside and behind them, up to the
    most that K and V may have."""
    import subprocess
    shared, tiles = _code("attention.cuh"), _code("attention_tiles.cu")
    seen = "struct Seen<false> " + _body(shared, "struct Seen<false>") + ";"
    bits = re.search(r"[^\n]*bits_of\(const Seen<false>&[^\n]*", tiles).group(0)
    source = tmp_path / "seen.cpp"
    source.write_text("""
#include <algorithm>
#include <cstdint>
#include <cstdio>
using std::max; using std::min;
#define __device__
#define __forceinline__ inline
struct SeqArgs { int window, n_sink; };
struct Sample { int len, queries, base; };
template <bool TREE> struct Seen;
template <>
""" + seen + """
static uint32_t below(int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : ~0u >> (32 - x); }
""" + bits + """
int main() {
    const int most = 0x7fff0000, far = 0x7fffffff, windows[] = {0, 1, 100, most, far - 200, far - 1, far}, sinks[] = {0, 5, most, far}, ends[] = {1, 40, 1000, most};
    int wrong = 0;
    for (int window : windows) for (int n_sink : sinks) for (int len : ends) for (int t = 0; t < 300 && t < len; t += 7) {
        const int queries = min(len, 300);
        const SeqArgs a = {window, n_sink};
        const Sample s = {len, queries, len - queries};
        const Seen<false> sees(a, s, 0, t);
        const int64_t p = (int64_t)s.base + t;
        const int starts[] = {-96, 0, 32, s.base - 64, s.base, s.base + t - 16, s.base + 256, len - 32};
        for (int j0 : starts) if (j0 >= -96 && j0 + 32 <= most + 32) {
            const uint32_t got = bits_of(sees, j0);
            for (int e = 0; e < 32; ++e) {
                const int64_t j = (int64_t)j0 + e;
                if (j < 0 || j >= len) continue;
                const bool want = j <= p && (j < n_sink || j > p - window);
                wrong += (got >> e & 1) != want || sees((int)j) != want;
            }
        }
    }
    std::printf("%d\\n", wrong);
    return wrong != 0;
}
""")
    program = str(tmp_path / "seen")
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", str(source), "-o", program],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "0", (r.returncode, r.stdout)


def test_hardly_anything_is_spilled():
    """The kernel for many rows has no cache beside its shared memory: a reload takes some 600 cycles.  What the compiler says: a few words that are set once, in front of the
    loops (more of them, or of the kernel for few rows, would be a row's)."""
    import subprocess
    from paper_2601_17818_b200 import build
    for name, kernels, most in (("attention_tiles.cu", 4, 32), ("attention.cu", 10, 20)):
        r = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-Xptxas", "-v", "-cubin", os.path.join(build.CSRC, name), "-o", os.devnull], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        said = re.findall(r"Compiling entry function '\S*attention_(?:few|tiles)_kernel\S*'.*?(\d+) bytes spill stores, (\d+) bytes spill loads", r.stderr, re.S)
        assert len(said) == kernels
        assert all(int(stores) <= most and int(loads) <= most for stores, loads in said), said
