"""Rotary positions and attention over bf16 rows without a GPU: the oracle held to closed forms, and what the entry points refuse."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2601_17818_b200 import binding as vb
from paper_2601_17818_b200.build import build_library

NULL = None
A, K, V, OUT = (C.c_void_p(x << 20) for x in (16, 32, 48, 64))
LSE, WS, LEN = C.c_void_p(80 << 20), C.c_void_p(96 << 20), C.c_void_p(112 << 20)


@pytest.fixture(scope="module")
def L():
    build_library()
    return vb.lib()


# ---------------------------------------------------------------------------------------------- the oracle
def test_a_quarter_turn_swaps_the_halves():
    x = np.random.default_rng(0).standard_normal((1, 2, 3, 16))
    position = np.array([[[0, 1, 2]]])
    y, written = oa.rotary(x, position, [np.pi / 2] * 8, [0] * 8)
    assert written.all() and np.allclose(y[:, :, 0], x[:, :, 0])
    assert np.allclose(y[:, :, 1, :8], -x[:, :, 1, 8:]) and np.allclose(y[:, :, 1, 8:], x[:, :, 1, :8])
    assert np.allclose(y[:, :, 2], -x[:, :, 2])


def test_turning_back_is_the_inverse_and_the_gradient():
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((2, 2, 3, 3, 24))
    position, axis, f = rng.integers(-50, 20000, (3, 2, 3)), rng.integers(0, 3, 8), rng.uniform(0, 2, 8)
    y, _ = oa.rotary(x, position, f, axis)
    back, _ = oa.rotary(y, position, f, axis, inverse=True)
    assert np.allclose(back, x)
    dx, _ = oa.rotary(g, position, f, axis, inverse=True)
    step, u = 1e-6, rng.standard_normal(x.shape)
    plus, minus = (oa.rotary(x + e * u, position, f, axis)[0] for e in (step, -step))
    assert np.isclose(((plus - minus) / (2 * step) * g).sum(), (dx * u).sum())
    assert np.array_equal(y[..., 16:], x[..., 16:])


def test_rows_without_a_token_and_far_tokens():
    x = np.ones((1, 1, 4, 16))
    _, written = oa.rotary(x, np.zeros((1, 1, 2), int), [1.0] * 8, [0] * 8, token=np.array([[1, -1, 99, 0]]), seq_len=[3])
    assert written.tolist() == [[True, False, True, False]]


@pytest.mark.parametrize("window,n_sink,p,want", [(1, 0, 4, [4]), (0, 2, 4, [0, 1]), (3, 1, 5, [0, 3, 4, 5]), (9, 0, 2, [0, 1, 2]), (0, 0, 3, []),
                                                  (2, 99, 3, [0, 1, 2, 3]), (2 ** 31 - 1, 0, 1, [0, 1])])
def test_window_and_sinks(window, n_sink, p, want):
    assert np.flatnonzero(oa.seen_rows(8, 8, p, window, n_sink)).tolist() == want
    assert np.flatnonzero(oa.seen_rows(p + 1, 1, 0, window, n_sink)).tolist() == want


def test_a_tree_of_a_chain_is_causal_and_a_query_in_front_of_the_first_row_sees_nothing():
    for t in range(5):
        assert np.array_equal(oa.seen_rows(9, 5, t, tree=(2 << t) - 1), oa.seen_rows(9, 5, t, 10 ** 6))
    assert not oa.seen_rows(3, 5, 1, tree=-1).any() and not oa.seen_rows(3, 5, 1, 10 ** 6).any()
    assert oa.seen_rows(3, 5, 2, tree=1 << 4).tolist() == [False, False, True]


def test_attention_is_softmax():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((1, 2, 3, 64)), rng.standard_normal((1, 1, 7, 64)), rng.standard_normal((1, 1, 7, 64))
    out, lse, size, _ = oa.attention(q, k, v, [7], [3], 0.3, 10 ** 6)
    z = torch.from_numpy(0.3 * q[0] @ k[0, 0].T)
    z = z.masked_fill(torch.triu(torch.ones(3, 7), 5).bool(), -np.inf)
    assert np.allclose(out[0], torch.softmax(z, -1).numpy() @ v[0, 0]) and np.allclose(lse[0], torch.logsumexp(z, -1).numpy())
    assert np.all(size >= np.abs(out) - 1e-12)


# ---------------------------------------------------------------------------------------------- refusals
def test_lengths_of_the_workspace():
    assert vb.vitcop_workspace_bytes(vb.OP_ATTENTION, B=2, H=4, N=100, d=128, Nv=3, D=28) >= 256
    for dims, status in ((dict(H=-1), vb.ERR_INVALID_ARG), (dict(N=-1), vb.ERR_INVALID_ARG), (dict(d=-1), vb.ERR_INVALID_ARG),
                         (dict(B=65535, Nv=2 ** 20, D=2 ** 20), vb.ERR_UNSUPPORTED)):
        with pytest.raises(vb.VitcopError) as e:
            vb.vitcop_workspace_bytes(vb.OP_ATTENTION, **dims)
        assert e.value.status == status


def _attention(L, is_tree=False, **over):
    a = dict(q=A, K=K, V=V, B=2, Hq=8, H=4, Tq=3, d=128, N=64, qs=(8 * 3 * 128, 3 * 128, 128), ks=(4 * 64 * 128, 64 * 128, 128),
             vs=(4 * 64 * 128, 64 * 128, 128), cache_len=LEN, query_len=NULL, window=16, n_sink=4, tree=C.c_void_p(120 << 20), scale=0.1, out=OUT,
             os=(8 * 3 * 128, 3 * 128, 128), lse=LSE, ws=WS, bytes=1 << 20)
    a.update(over)
    head = (a["q"], a["K"], a["V"], a["B"], a["Hq"], a["H"], a["Tq"], a["d"], a["N"], *a["qs"], *a["ks"], *a["vs"], a["cache_len"], a["query_len"])
    tail = (a["scale"], a["out"], *a["os"], a["lse"], a["ws"], a["bytes"], NULL)
    return L.vitcop_tree_attention(*head, a["tree"], *tail) if is_tree else L.vitcop_window_attention(*head, a["window"], a["n_sink"], *tail)


@pytest.mark.parametrize("is_tree", [False, True])
def test_attention_refuses(L, is_tree):
    def status(**over):
        return _attention(L, is_tree, **over)
    inv, uns = vb.ERR_INVALID_ARG, vb.ERR_UNSUPPORTED
    odd = C.c_void_p((16 << 20) + 8)
    for name in ("q", "K", "V", "out"):
        assert status(**{name: NULL}) == inv, name
        assert status(**{name: odd}) == uns, name
    for name in ("B", "Hq", "H", "Tq", "N"):
        assert status(**{name: -1}) == inv, name
    for name in ("qs", "ks", "vs", "os"):
        for i in range(3):
            s = [8192 * 8, 8192, 128]
            s[i] = -8
            assert status(**{name: tuple(s)}) == inv, name
            s[i] = 100
            assert status(**{name: tuple(s)}) == uns, name
    assert status(d=0) == inv and status(d=96) == uns and status(d=32) == uns
    assert status(Hq=7) == inv and status(H=0) == inv
    for scale in (float("nan"), float("inf"), -float("inf"), 3e38):
        assert status(scale=scale) == inv
    assert status(os=(8 * 3 * 128, 128, 128)) == inv and status(os=(0, 3 * 128, 128)) == inv            # rows that share elements
    assert status(out=A) == inv and status(out=K) == inv and status(out=V) == inv and status(lse=A) == inv and status(ws=K) == inv
    assert status(lse=OUT) == inv and status(ws=OUT) == inv and status(lse=WS) == inv
    assert status(out=C.c_void_p((112 << 20) - 256)) == inv                                            # lengths in the output
    assert status(ws=NULL) == vb.ERR_WORKSPACE and status(bytes=8) == vb.ERR_WORKSPACE and status(ws=C.c_void_p((96 << 20) + 16)) == vb.ERR_WORKSPACE
    assert status(B=65536) == uns and status(Tq=2 ** 30, os=(2 ** 50, 2 ** 40, 128)) == uns and status(N=2 ** 31 - 1, ks=(0, 0, 0), vs=(0, 0, 0)) == uns
    if is_tree:
        assert status(tree=NULL) == inv and status(tree=C.c_void_p((120 << 20) + 4)) == uns and status(Tq=65) == uns
        assert status(tree=OUT) == inv
    else:
        assert status(window=-1) == inv and status(n_sink=-1) == inv


def _rotary(L, **over):
    a = dict(q=A, k=K, B=2, Hq=8, Hk=4, N=16, d=128, qs=(8 * 16 * 128, 16 * 128, 128), ks=(4 * 16 * 128, 16 * 128, 128), position=LEN, axes=3, n_pos=16,
             token=NULL, seq_len=NULL, inv_freq=C.c_void_p(113 << 20), axis=C.c_void_p(114 << 20), F=64, q_out=V, k_out=OUT)
    a["qo"], a["ko"] = a["qs"], a["ks"]
    a.update(over)
    return L.vitcop_rotary_axes(a["q"], a["k"], a["B"], a["Hq"], a["Hk"], a["N"], a["d"], *a["qs"], *a["ks"], a["position"], a["axes"], a["n_pos"], a["token"],
                                a["seq_len"], a["inv_freq"], a["axis"], a["F"], 0, a["q_out"], *a["qo"], a["k_out"], *a["ko"], NULL)


def test_rotary_refuses(L):
    inv, uns = vb.ERR_INVALID_ARG, vb.ERR_UNSUPPORTED
    odd = C.c_void_p((16 << 20) + 8)

    def status(**over):
        return _rotary(L, **over)
    assert status(q=NULL, k=NULL, q_out=NULL, k_out=NULL) == inv
    for name in ("q", "k", "q_out", "k_out", "position", "inv_freq", "axis"):
        assert status(**{name: NULL}) == inv, name
    for name in ("q", "k", "q_out", "k_out"):
        assert status(**{name: odd}) == uns, name
    for name in ("B", "Hq", "Hk", "N", "n_pos", "F"):
        assert status(**{name: -1}) == inv, name
    assert status(axes=0) == inv and status(d=0) == inv and status(n_pos=15) == inv and status(token=C.c_void_p(115 << 20), n_pos=0) == inv
    assert status(d=100) == uns and status(F=4) == uns and status(F=72) == uns and status(d=1024, F=264, qs=(0, 0, 0), ks=(0, 0, 0)) == uns
    assert status(d=4104, F=8) == uns and status(Hq=32768) == uns and status(Hk=40000) == uns and status(N=2 ** 31 - 1, token=C.c_void_p(115 << 20)) == uns
    assert status(token=C.c_void_p(115 << 20), n_pos=0, F=0) == inv
    assert status(B=65536) == uns and status(inv_freq=C.c_void_p((113 << 20) + 4)) == uns
    for name in ("qs", "ks", "qo", "ko"):
        for i in range(3):
            s = [8 * 16 * 128, 16 * 128, 128]
            s[i] = -8
            assert status(**{name: tuple(s)}) == inv, name
            s[i] = 100
            assert status(**{name: tuple(s)}) == uns, name
    assert status(q_out=K) == inv and status(k_out=A) == inv and status(k_out=V) == inv                # an output on the other's input, on the other output
    assert status(q_out=C.c_void_p((16 << 20) + 256)) == inv                                          # one row further
    assert status(q_out=A, qo=(8 * 16 * 128, 128, 8 * 128)) == inv                                     # in place in another order
    assert status(qo=(8 * 16 * 128, 16 * 128, 0)) == inv
    assert status(q_out=LEN) == inv and status(k_out=C.c_void_p(113 << 20)) == inv                     # positions, frequencies


def test_nothing_to_turn_is_nothing_to_do(L):
    assert _rotary(L, B=0) == vb.OK and _rotary(L, N=0) == vb.OK and _rotary(L, Hq=0, Hk=0) == vb.OK


@pytest.mark.parametrize("B,N", [(1, 16), (3, 16), (3, 1)])
@pytest.mark.parametrize("heads_outside", [False, True])
def test_keys_that_reach_into_the_queries_are_refused(L, B, N, heads_outside):
    """Queries and keys of one projection lie in one another's gaps; a head further down they share one.  (That side by side is not refused is
    seen on the GPU: the call goes through.)"""
    Hq, Hk, d = 8, 4, 128
    heads = Hq + 2 * Hk
    s, step = ((heads * N * d, N * d, d), N * d) if heads_outside else ((N * heads * d, d, heads * d), d)
    k = C.c_void_p((16 << 20) + (Hq - 1) * step * 2)
    assert _rotary(L, B=B, N=N, Hq=Hq, Hk=Hk, q=A, q_out=A, k=k, k_out=k, qs=s, qo=s, ks=s, ko=s) == vb.ERR_INVALID_ARG


def test_the_binding_refuses_other_tensors(L):
    f = torch.zeros
    with pytest.raises(ValueError):
        vb._module.window_attention(0, 0, f(1, 1, 1, 64), f(1, 1, 8, 64), f(1, 1, 8, 64), None, f(1, 1, 1, 64), None, 1.0, 4, 0, None, None)
    with pytest.raises(ValueError):
        vb._module.tree_attention(0, 0, None, None, None, None, None, None, None, 1.0, None, None)
    with pytest.raises(ValueError):
        vb._module.rotary_axes(0, 0, None, None, None, None, None, None, None, None, None, False)
    for name in ("window_attention", "tree_attention", "rotary_axes"):
        with pytest.raises(TypeError):
            getattr(vb._module, name)(0, 0)


def test_registers_that_change_hands_are_there():
    """The kernel for many query rows gives registers of some warps to others: the compiler's number a thread is the one that the exchange counts on (asked for and
    not there, they would be waited for without end), and its loop over blocks has no cache to spill to."""
    import re
    import subprocess
    from paper_2601_17818_b200 import build
    r = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-Xptxas", "-v", "-cubin", os.path.join(build.CSRC, "attention_tiles.cu"), "-o", os.devnull],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    used = re.findall(r"Compiling entry function '\S*attention_tiles_kernel\S*'.*?Used (\d+) registers", r.stderr, re.S)
    with open(os.path.join(build.CSRC, "attention_tiles.cu")) as fh:
        source = fh.read()
    softmax, other = (int(re.search(rf"{name} = (\d+)", source).group(1)) for name in ("kSoftmaxRegs", "kOtherRegs"))
    threads = int(re.search(r"kSoftmaxThreads = (\d+)", source).group(1))
    assert len(used) == 4 and set(used) == {str((threads * softmax + 128 * other) // (threads + 128))}
