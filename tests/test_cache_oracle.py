"""The K/V cache in 4 bits without a GPU: the oracle held to closed forms and to bounds, and what the entry points refuse."""
import ctypes as C
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2601_17818_b200 import binding as vb
from paper_2601_17818_b200.build import ROOT, build_library


@pytest.fixture(scope="module")
def L():
    build_library()
    return vb.lib()


def _bf16(rng, *shape, spread=1.0):
    return oc.round_bf16(rng.standard_normal(shape) * spread)


def test_rounding_to_bf16_is_torchs():
    x = np.random.default_rng(0).standard_normal(20000) * np.exp(np.random.default_rng(1).uniform(-80, 80, 20000))
    x[:6] = [0.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, np.inf, -np.inf, 2.0 ** -130 * 1.37]
    x = x.astype(np.float32)
    assert np.array_equal(oc.round_bf16(x), torch.from_numpy(x).bfloat16().double().numpy())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_pack_and_unpack_are_inverse(d):
    rng = np.random.default_rng(d)
    K, V = _bf16(rng, 2, 3, 64, d), _bf16(rng, 2, 3, 64, d, spread=5.0)
    cache = oc.pack(K, V)
    assert cache.shape == (2, 3, 2, 40 * d)
    for x, held in zip((K, V), oc.unpack(cache)):
        for a, b in zip(oc.quantise(x), held):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("offset,spread", [(0.0, 1.0), (100.0, 1.0), (-3.0, 0.01), (0.0, 1e30), (0.0, 1e-20)])
def test_values_are_as_near_as_the_step_allows(offset, spread):
    """At most half a step, the centre's own rounding (half of bf16's last place) and, at the ends, the scale's (15 / 2 steps of it)."""
    x = oc.round_bf16(np.random.default_rng(3).standard_normal((50, 128)) * spread + offset)
    s, m, code = oc.quantise(x)
    off = np.abs(oc.values(s, m, code) - x).reshape(50, 4, 32)
    assert code.min() >= 0 and code.max() <= 15
    assert np.all(off <= s[..., None] * (0.5 + 15 * 2.0 ** -8) + np.abs(m[..., None]) * 2.0 ** -8)


def test_codes_are_the_nearest_and_ties_go_to_the_even_one():
    rng = np.random.default_rng(4)
    x = rng.integers(-60, 61, (2000, 32)) / 4.0
    x[:, 0], x[:, 1] = -15.0, 15.0                         # s = 2, m = 1: borders at the even integers
    s, m, code = oc.quantise(x)
    assert np.all(s == 2.0) and np.all(m == 1.0)
    steps = np.arange(16)
    away = np.abs(x[..., None] - (1.0 + 2.0 * (steps - 8)))
    near = away.min(-1, keepdims=True)
    tied = (away == near).sum(-1) == 2
    assert tied.mean() > 0.05
    assert np.all(np.take_along_axis(away, code[:, 0, :, None], -1) == near)
    assert np.all(code[:, 0][tied] % 2 == 0)


def test_groups_that_are_special():
    x = np.zeros((6, 32))
    x[0] = 7.5                                             # constant: held exactly
    x[1, 3] = np.nan
    x[2, 4] = np.inf
    x[3, 5], x[3, 6] = 3.3e38, -3.3e38                     # further apart than fp32 reaches
    x[4, 0] = 2.0 ** -99                                   # a step below 2^-100 is none
    x[5, 0], x[5, 1] = 2.9e38, -1e37
    x = np.where(np.isfinite(x), oc.round_bf16(x), x)
    v = oc.values(*oc.quantise(x))
    assert np.all(v[0] == 7.5) and np.all(np.isnan(v[1:4])) and np.all(v[4] == 0.0)
    assert np.all(np.isfinite(v[5])) and np.abs(v[5] - x[5]).max() <= 2.9e38 / 15 * 0.6


def test_attention_oracle_closed_forms():
    rng = np.random.default_rng(5)
    K, V = rng.standard_normal((1, 2, 40, 64)), rng.standard_normal((1, 2, 40, 64))
    q = np.zeros((1, 4, 3, 64))
    out, lse = oc.attention(q, K, V, [10], 0.3, True)      # equal logits: means of the rows seen
    for t in range(3):
        assert np.allclose(out[0, 3, t], V[0, 1, :8 + t].mean(0)) and np.allclose(lse[0, :, t], np.log(8 + t))
    out, lse = oc.attention(q, K, V, [2], 0.3, True)       # the first of three queries sees nothing
    assert np.all(out[0, :, 0] == 0) and np.all(np.isneginf(lse[0, :, 0])) and np.allclose(out[0, 0, 1], V[0, 0, 0])
    out, lse = oc.attention(q, K, V, [0], 0.3, False)
    assert np.all(out == 0) and np.all(np.isneginf(lse))
    q = rng.standard_normal((1, 4, 1, 64))
    z = torch.from_numpy(np.einsum("hrd,hnd->hrn", q.reshape(2, 2, 64), K[0, :, :33]) * 0.7)
    want = torch.softmax(z, -1) @ torch.from_numpy(V[0, :, :33])
    out, lse = oc.attention(q, K, V, [33], 0.7, True)
    assert np.allclose(out.reshape(2, 2, 64), want.numpy()) and np.allclose(lse.reshape(2, 2), torch.logsumexp(z, -1).numpy())


# ---------------------------------------------------------------------------------------------- refusals (no device is touched)
A, B_, C_, D_, E_ = (0x1000000 * i for i in range(1, 6))
NULL = None


def _write(L, K=A, V=B_, B=2, H=2, N=40, d=64, ks=(5120, 2560, 64), vs=(5120, 2560, 64), seq=NULL, vis_start=0, vis=NULL, vu=0, keep=NULL,
           stride=0, nk=NULL, clen=NULL, cache=C_, Ncap=64, new=D_):
    return L.vitcop_cache_write(K, V, B, H, N, d, *ks, *vs, seq, vis_start, vis, vu, keep, stride, nk, clen, cache, Ncap, new, NULL)


@pytest.mark.parametrize("what,status", [
    (dict(K=NULL, V=NULL), vb.ERR_INVALID_ARG), (dict(cache=NULL), vb.ERR_INVALID_ARG), (dict(new=NULL), vb.ERR_INVALID_ARG),
    (dict(B=-1), vb.ERR_INVALID_ARG), (dict(N=-1), vb.ERR_INVALID_ARG), (dict(Ncap=-32), vb.ERR_INVALID_ARG),
    (dict(ks=(5120, -64, 64)), vb.ERR_INVALID_ARG), (dict(keep=E_, stride=8), vb.ERR_INVALID_ARG),
    (dict(keep=E_, stride=0, nk=E_ + 4096), vb.ERR_INVALID_ARG), (dict(keep=E_, stride=8, nk=E_ + 4096, vis_start=30, vu=11), vb.ERR_INVALID_ARG),
    (dict(keep=E_, stride=8, nk=E_ + 4096, vis_start=-1), vb.ERR_INVALID_ARG),
    (dict(clen=D_), vb.ERR_INVALID_ARG), (dict(seq=D_ + 4), vb.ERR_INVALID_ARG), (dict(cache=A), vb.ERR_INVALID_ARG),
    (dict(cache=B_ + 16), vb.ERR_INVALID_ARG), (dict(new=C_ + 64), vb.ERR_INVALID_ARG), (dict(clen=C_), vb.ERR_INVALID_ARG),
    (dict(d=96), vb.ERR_UNSUPPORTED), (dict(Ncap=48), vb.ERR_UNSUPPORTED), (dict(K=A + 8), vb.ERR_UNSUPPORTED),
    (dict(cache=C_ + 8), vb.ERR_UNSUPPORTED), (dict(vs=(5120, 2560, 68)), vb.ERR_UNSUPPORTED), (dict(B=65536, ks=(0, 0, 64), vs=(0, 0, 64), K=C_ << 16, V=C_ << 16), vb.ERR_UNSUPPORTED)])
def test_write_refuses(L, what, status):
    assert _write(L, **what) == status


def _read(L, cache=C_, B=2, H=2, Ncap=64, d=64, clen=NULL, begin=NULL, bu=0, K=A, V=B_, N=8):
    return L.vitcop_cache_read(cache, B, H, Ncap, d, clen, begin, bu, K, V, N, NULL)


@pytest.mark.parametrize("what,status", [
    (dict(cache=NULL), vb.ERR_INVALID_ARG), (dict(K=NULL, V=NULL), vb.ERR_INVALID_ARG), (dict(N=-1), vb.ERR_INVALID_ARG),
    (dict(bu=-1), vb.ERR_INVALID_ARG), (dict(K=C_ + 16), vb.ERR_INVALID_ARG), (dict(K=A, V=A), vb.ERR_INVALID_ARG),
    (dict(clen=A), vb.ERR_INVALID_ARG), (dict(d=32), vb.ERR_UNSUPPORTED), (dict(Ncap=65), vb.ERR_UNSUPPORTED),
    (dict(V=B_ + 2), vb.ERR_UNSUPPORTED)])
def test_read_refuses(L, what, status):
    assert _read(L, **what) == status


def _attend(L, q=A, cache=C_, B=2, Hq=4, H=2, Tq=1, d=64, Ncap=64, qs=(256, 64, 64), clen=NULL, out=B_, os=(256, 64, 64), lse=NULL, ws=D_,
            wsb=1 << 30):
    return L.vitcop_cache_attention(q, cache, B, Hq, H, Tq, d, Ncap, *qs, clen, 0.125, 1, out, *os, lse, ws, wsb, NULL)


@pytest.mark.parametrize("what,status", [
    (dict(q=NULL), vb.ERR_INVALID_ARG), (dict(cache=NULL), vb.ERR_INVALID_ARG), (dict(out=NULL), vb.ERR_INVALID_ARG),
    (dict(Hq=5), vb.ERR_INVALID_ARG), (dict(H=0), vb.ERR_INVALID_ARG), (dict(Tq=-1), vb.ERR_INVALID_ARG),
    (dict(qs=(256, -64, 64)), vb.ERR_INVALID_ARG), (dict(os=(256, 0, 64)), vb.ERR_INVALID_ARG), (dict(out=A), vb.ERR_INVALID_ARG),
    (dict(out=C_ + 128), vb.ERR_INVALID_ARG), (dict(lse=B_ + 8), vb.ERR_INVALID_ARG), (dict(ws=B_), vb.ERR_INVALID_ARG),
    (dict(clen=B_), vb.ERR_INVALID_ARG),
    (dict(d=80), vb.ERR_UNSUPPORTED), (dict(Ncap=16), vb.ERR_UNSUPPORTED), (dict(q=A + 4), vb.ERR_UNSUPPORTED),
    (dict(os=(256, 65, 64)), vb.ERR_UNSUPPORTED), (dict(ws=NULL), vb.ERR_WORKSPACE), (dict(wsb=8), vb.ERR_WORKSPACE),
    (dict(ws=D_ + 128), vb.ERR_WORKSPACE)])
def test_attention_refuses(L, what, status):
    assert _attend(L, **what) == status


def test_binding_refuses_what_is_not_on_the_device(L, monkeypatch):
    monkeypatch.setattr(vb, "_device", lambda: 0)
    monkeypatch.setattr(vb, "_raw_stream", lambda device: 0)
    cache = torch.zeros(1, 1, 1, 40 * 64, dtype=torch.uint8)
    x, n = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: vb.vitcop_cache_write(x, x, cache, n), lambda: vb.vitcop_cache_read(cache, n, x),
                 lambda: vb.vitcop_cache_attention(x, cache, n, x, cache[0, 0, 0], 1.0)):
        with pytest.raises(ValueError):
            call()
    for B, H, Ncap, d in ((1, 1, 33, 64), (1, 1, 32, 96)):
        with pytest.raises(ValueError):
            vb.alloc_cache(B, H, Ncap, d, device="cpu")
    assert vb.alloc_cache(2, 3, 64, 128, device="cpu").shape == (2, 3, 2, 5120)
    with pytest.raises(vb.VitcopError):
        vb.vitcop_workspace_bytes(vb.OP_CACHE_ATTENTION, B=1, H=-1)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_attention_refuses_a_scale_that_is_no_number(L, scale):
    assert L.vitcop_cache_attention(A, C_, 2, 4, 2, 1, 64, 64, 256, 64, 64, NULL, scale, 1, B_, 256, 64, 64, NULL, D_, 1 << 30, NULL) == vb.ERR_INVALID_ARG


def test_a_pointer_to_nothing_may_be_null(L):
    assert _write(L, K=NULL, V=NULL, B=0, cache=NULL, new=NULL) == vb.OK
    assert _read(L, B=0, cache=NULL, K=NULL, V=NULL) == vb.OK and _read(L, Ncap=0, cache=NULL, K=NULL, V=NULL, N=0) == vb.OK
    for nothing in (dict(Tq=0), dict(B=0), dict(H=0, Hq=0)):       # (as far as the workspace, which is asked for last)
        assert _attend(L, q=NULL, out=NULL, ws=NULL, cache=C_, **nothing) == vb.ERR_WORKSPACE
    assert _attend(L, cache=NULL, Ncap=0, ws=NULL) == vb.ERR_WORKSPACE


def test_codes_by_exact_fractions():
    """Elements of any size beside their centre, down to the last bf16 there is: the nearest code, computed with fractions."""
    from fractions import Fraction
    rng = np.random.default_rng(6)
    for trial in range(200):
        x = oc.round_bf16(rng.standard_normal(32) * np.exp2(-rng.integers(0, 130, 32).astype(np.float64)))
        x[:2] = [(-0.9375, 0.9375), (-15.0, 15.0), (-0.8125, 1.0625), (oc.round_bf16(rng.standard_normal()) - 2, 2.5)][trial % 4]
        x = oc.round_bf16(x)
        s, m, code = oc.quantise(x)
        for e in range(32):
            q = (Fraction(float(x[e])) - Fraction(float(m[0]))) / Fraction(float(s[0]))
            assert code[0, e] == min(max(round(q), -8), 7) + 8         # (Python's: halves to even)


@pytest.mark.parametrize("B,Hq,Tq,strides,shared", [
    (2, 4, 2, (256, 64, 64), True), (2, 4, 2, (512, 64, 64), True), (2, 4, 2, (64, 128, 512), False), (2, 4, 2, (448, 64, 256), True),
    (2, 4, 2, (0, 128, 64), True), (2, 1, 2, (64, 0, 64), True), (1, 4, 2, (0, 128, 120), True), (2, 4, 2, (1 << 62, 1 << 62, 64), True),
    (2, 4, 2, (512, 128, 64), False), (2, 4, 2, (512, 64, 256), False), (2, 4, 2, (64, 256, 128), False), (1, 1, 1, (0, 0, 0), False),
    (1, 4, 2, (0, 64, 256), False), (2, 1, 2, (128, 0, 64), False), (2, 4, 2, (1024, 72, 328), False)])
def test_attention_refuses_rows_of_the_output_that_share_elements(L, B, Hq, Tq, strides, shared):
    """Together too: head 1 of the first query, and the first head of query 1.  (What passes is asked for its workspace next.)"""
    status = _attend(L, B=B, Hq=Hq, H=min(Hq, 2), Tq=Tq, qs=(512, 128, 64), os=strides, ws=NULL)
    assert status == (vb.ERR_INVALID_ARG if shared else vb.ERR_WORKSPACE)


@pytest.mark.parametrize("scale,status", [(2.5e38, vb.ERR_INVALID_ARG), (-3.4e38, vb.ERR_INVALID_ARG), (2.0 ** 127, vb.ERR_WORKSPACE), (-1e38, vb.ERR_WORKSPACE),
                                          (1e-45, vb.ERR_WORKSPACE)])
def test_attention_refuses_a_scale_that_is_infinite_in_powers_of_two(L, scale, status):
    assert L.vitcop_cache_attention(A, C_, 2, 4, 2, 1, 64, 64, 256, 64, 64, NULL, scale, 1, B_, 256, 64, 64, NULL, NULL, 0, NULL) == status


@pytest.mark.parametrize("B,Hq,H,Tq,status", [(1, 1 << 30, 1, 1 << 30, vb.ERR_UNSUPPORTED), (4, 1 << 30, 1, 1 << 30, vb.ERR_UNSUPPORTED),
                                              (1 << 30, 1 << 30, 1 << 30, 16, vb.ERR_UNSUPPORTED), (2, 1 << 15, 1 << 15, 1 << 15, vb.ERR_UNSUPPORTED),
                                              (1, 1 << 15, 1, (1 << 16) - 1, vb.OK), (1, 0, 1, 1 << 30, vb.OK), (1, 4, 8, 1 << 28, vb.OK)])
def test_workspace_of_more_query_rows_than_are_counted(L, B, Hq, H, Tq, status):
    """In a process of its own: a product that loses its upper bits ended it with a division by zero."""
    code = (f"import ctypes as C\nfrom paper_2601_17818_b200 import binding as vb\nn = C.c_size_t(0)\n"
            f"print(vb.lib().vitcop_workspace_bytes(vb.OP_CACHE_ATTENTION, {B}, {H}, 64, 64, {Tq}, {Hq}, 0, C.byref(n)))")
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0 and int(run.stdout) == status, run.stderr
