"""Rotary positions and attention over bf16 rows where little is left to weigh, near the ends of fp32, over sizes on which the division of work turns, and beside the
other calls (``-m gpu``).  Tolerances as in test_gpu_attention.py, where they are derived; what is added to them is derived here beside its use.

Which path a call takes is asserted by its kernel's name and, of the kernel for many rows, by the number of CTAs that it has left in its status word.
"""
import numpy as np
import pytest
import torch

from paper_2601_17818_b200 import binding as vb
from test_gpu_attention import DEV, HALF, MANY, NO_WINDOW, _bf16, _case, _check_long, _f64, _i32, _kernels_of, _run

pytestmark = pytest.mark.gpu
FEW = {"attention_few_kernel"}
# B, H, R, Tq, N, kernel: a CTA a head, a cluster a head; items in turn, a cluster an item
PATHS = [(2, 100, 1, 1, 64, FEW), (2, 2, 2, 3, 600, FEW), (2, 8, 4, 300, 1500, MANY), (2, 1, 4, 300, 3000, MANY)]
PATHS = [(d, *path) for path in PATHS for d in (64, 128, 256) if d < 256 or path[-1] is FEW]
NAN, INF = float("nan"), float("inf")


def _plain(q, K, V, seen, scale):
    """(out, lse, tolerances of both) in fp64 by torch: of a causal call whose rows ``seen`` (bool [B, H, N]) weigh something, K and V finite there."""
    R, Tq, N, d = q.shape[1] // K.shape[1], q.shape[2], K.shape[2], q.shape[3]
    rows = lambda x: torch.where(seen[..., None], x, 0).double().repeat_interleave(R, 1)
    see = seen.repeat_interleave(R, 1)[:, :, None] & (torch.arange(N, device=DEV) <= N - Tq + torch.arange(Tq, device=DEV)[:, None])
    qd, k, v = q.double(), rows(K), rows(V)
    z = torch.where(see, qd @ k.mT * scale, -np.inf)
    lse = torch.logsumexp(z, -1)
    w = torch.exp(z - lse[..., None])
    w = torch.where(torch.isneginf(lse)[..., None], 0, w)
    want, size = w @ v, w @ v.abs()
    delta = 2.0 ** -22 * (d / 16 + 2) * abs(scale) * torch.where(see, qd.abs() @ k.abs().mT, 0).amax(-1, keepdim=True)
    return want, lse, HALF * (1 + HALF) * (size + 2 * want.abs()) + (torch.exp(2 * delta) - 1) * (size + want.abs()), delta[..., 0] + 2.0 ** -20 * (1 + lse.abs())


@pytest.mark.parametrize("d,B,H,R,Tq,N,kernel", PATHS)
def test_nothing_weighed_beside_values_that_are_no_numbers(d, B, H, R, Tq, N, kernel):
    """Logits of -inf alone: out = 0 and lse = -inf, whatever V holds and however a row's parts are joined.  (Where others weigh something, 0 times what is no number
    is none.)"""
    rng, q, K, V = _case(N + d, B, H, R, Tq, d, N)
    q[..., 0] = 1.0
    K[0, ..., 0] = -INF
    V[0, :, ::7], V[0, :, 1::9], V[0, :, N - 2] = NAN, INF, -INF
    K[1, :, ::3, 0] = -INF
    V[1, :, 3, 5], V[1, :, N // 2 // 3 * 3, 9] = NAN, -INF
    out, lse, names = _kernels_of(q, K, V, None, d ** -0.5)
    assert names == kernel
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    assert torch.isnan(out[1][..., [5, 9]]).all()
    seen = torch.arange(N, device=DEV).expand(B, H, N) % 3 != 0
    want, wlse, tol, lse_tol = _plain(q, K, V, seen, d ** -0.5)
    rest = [e for e in range(d) if e not in (5, 9)]
    assert ((out[1].double() - want[1]).abs() <= tol[1])[..., rest].all()
    assert ((lse[1].double() - wlse[1]).abs() <= lse_tol[1]).all()


@pytest.mark.parametrize("bad", [INF, -INF])
@pytest.mark.parametrize("d,B,H,R,Tq,N,kernel", PATHS)
def test_infinite_keys_of_rows_that_are_seen(bad, d, B, H, R, Tq, N, kernel):
    """One infinite element: its logit is +inf, and the output no number, or -inf, and the row weighs nothing, as its query's element has the same sign or the other."""
    rng, q, K, V = _case(N + d + 1, B, H, R, Tq, d, N)
    at = torch.zeros(N, dtype=torch.bool, device=DEV)
    at[[1, N // 3, N // 2, N - Tq]] = True                 # (all of them seen by all queries)
    K[:, :, at, 2] = bad
    q[..., 2] = torch.where(torch.rand(q.shape[:-1], device=DEV) < 0.5, 1.0, -1.0).bfloat16()
    out, lse, names = _kernels_of(q, K, V, None, d ** -0.5)
    assert names == kernel
    want, wlse, tol, lse_tol = _plain(q, K, V, ~at.expand(B, H, N), d ** -0.5)
    nan = q[..., 2].float() * bad > 0
    assert nan.any() and torch.isnan(out[nan]).all() and torch.isnan(lse[nan]).all()
    assert ((out.double() - want).abs() <= tol)[~nan].all() and ((lse.double() - wlse).abs() <= lse_tol)[~nan].all()


def _us(B, H, R, Tq, d, N):
    rng, q, K, V = _case(N, B, H, R, Tq, d, N)
    out, ws = torch.empty_like(q), vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=N, d=d, Nv=Tq, D=H * R)
    graph, times = torch.cuda.CUDAGraph(), []
    vb.vitcop_window_attention(q, K, V, None, out, ws, d ** -0.5, NO_WINDOW)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for _ in range(20):
            vb.vitcop_window_attention(q, K, V, None, out, ws, d ** -0.5, NO_WINDOW)
    for _ in range(8):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        times.append(begin.elapsed_time(end) * 50)
    return min(times)


@pytest.mark.parametrize("heads", [(15, 16), (16, 17), (17, 18), (18, 19), (33, 34), (36, 37), (37, 38)])
def test_a_head_more_does_not_bring_clusters_that_wait_for_others(heads):
    """An item a head, a cluster an item: one that does not run beside the others begins when they end, and the call takes twice as long (smaller clusters, and the half of a
    step of them: a head more may cost half as much again)."""
    fewer, more = (_us(1, h, 1, 256, 128, 1500) for h in heads)
    assert max(fewer, more) <= 1.5 * min(fewer, more)


@pytest.mark.parametrize("d,fewer,more", [(256, 16, 24), (256, 34, 64), (128, 24, 34), (64, 24, 64)])
def test_a_token_over_fewer_heads_takes_no_longer(d, fewer, more):
    """The same of the kernel for few rows (8 % for the clock)."""
    assert _us(1, fewer, 1, 1, d, 4160) <= 1.08 * _us(1, more, 1, 1, d, 4160)


# (the same paths, with rows enough for a maximum that moves late)
LATE = [(2, 100, 1, 1, 400, FEW), (2, 2, 2, 3, 600, FEW), (2, 8, 4, 300, 1500, MANY), (2, 1, 4, 300, 3000, MANY)]
LATE = [(d, *path) for path in LATE for d in (64, 128, 256) if d < 256 or path[-1] is FEW]


@pytest.mark.parametrize("rise", [10.0, 16.25, 16.5, 30.0])
@pytest.mark.parametrize("d,B,H,R,Tq,N,kernel", LATE)
def test_large_values_under_a_maximum_that_rises_late(rise, d, B, H, R, Tq, N, kernel):
    """Logits of 0, then of ``rise`` (14 to 43 powers of two): the mean of rows of 2^127 is 2^127, however many of them weigh as much as one can."""
    rng, q, K, V = _case(3, B, H, R, Tq, d, N)
    q[..., 0], K[..., 0] = 1.0, rise
    q[..., 1:], K[:, :, :200, 0] = 0.0, 0.0
    V[:] = 2.0 ** 127
    V[1, ..., ::2] *= -1
    out, lse, names = _kernels_of(q, K, V, None, 1.0)
    assert names == kernel
    want, wlse, tol, lse_tol = _plain(q, K, V, torch.ones(B, H, N, dtype=torch.bool, device=DEV), 1.0)
    assert ((out.double() - want).abs() <= tol).all() and ((lse.double() - wlse).abs() <= lse_tol).all()


@pytest.mark.parametrize("power", [-80, -95])
@pytest.mark.parametrize("d,B,H,R,Tq,N,kernel", LATE)
def test_small_values_keep_their_digits(power, d, B, H, R, Tq, N, kernel):
    """The largest weight may be 2^-(24 + b), b the bits of N, and a product with V, or a sum of them, is off by 2^-149 besides its own rounding: N 2^(b - 125) of the output
    each."""
    rng, q, K, V = _case(5, B, H, R, Tq, d, N)
    V *= 2.0 ** power
    out, lse, names = _kernels_of(q, K, V, None, d ** -0.5)
    assert names == kernel
    want, wlse, tol, lse_tol = _plain(q, K, V, torch.ones(B, H, N, dtype=torch.bool, device=DEV), d ** -0.5)
    assert ((out.double() - want).abs() <= tol + N * 2.0 ** (N.bit_length() - 124)).all() and ((lse.double() - wlse).abs() <= lse_tol).all()


@pytest.mark.parametrize("B,Hq,Hk,N", [(0, 4, 2, 8), (2, 4, 2, 0), (2, 0, 2, 8), (2, 4, 0, 8), (2, 0, 0, 8)])
def test_turning_tensors_of_no_elements(B, Hq, Hk, N):
    rng = np.random.default_rng(1)
    q, k = _bf16(rng, B, Hq, N, 64), _bf16(rng, B, Hk, N, 64)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    args = torch.zeros(1, B, N, dtype=torch.int32, device=DEV), torch.ones(32, dtype=torch.float64, device=DEV), torch.zeros(32, dtype=torch.int32, device=DEV)
    vb.vitcop_rotary_axes(q, k, *args, qo, ko)
    assert torch.equal(q, qo) and torch.equal(k, ko)      # (position 0 turns nothing)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 200, 2 ** 30])
@pytest.mark.parametrize("B,H,R,Tq,N", [(16, 16, 1, 300, 300), (1, 2, 2, 5, 90)])
def test_windows_near_the_end_of_32_bits(window, B, H, R, Tq, N):
    """All of them are no window at all."""
    rng, q, K, V = _case(2, B, H, R, Tq, 64, N)
    out, lse, names = _kernels_of(q, K, V, None, 0.125, window, 0)
    assert names == (MANY if Tq > 5 else FEW)
    _check_long(q, K, V, [N] * B, [Tq] * B, 0.125, out, lse, window, 0)


@pytest.mark.parametrize("d", [64, 128])
def test_one_axis_is_the_table_of_the_key_projection(d):
    """Keys turned by their projection, and keys projected and then turned.  The latter are rounded in front of the turn as well: half a place of |a| + |b|, next to the half
    place of either result; the table is rounded to fp32, and so are the products (2^-20 of |a| + |b|)."""
    B, N, Dh, H, F = 2, 75, 128, 3, d // 2
    rng = np.random.default_rng(d)
    hidden, W = _bf16(rng, B, N, Dh), _bf16(rng, H * d, Dh, spread=Dh ** -0.5)
    position, f = rng.integers(0, 4000, (B, N)), 10000.0 ** (-np.arange(F) / F)
    table = np.arange(4000)[:, None] * f
    cos, sin = (torch.tensor(g(table), dtype=torch.float32, device=DEV) for g in (np.cos, np.sin))
    ws = vb.alloc_workspace(vb.OP_KPROJ, B=B, H=H, N=N, d=d)
    K, turned, of_axes = (torch.zeros(B, H, N, d, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    vb.vitcop_kproj_knorm(hidden, W, H, d, K, ws)
    vb.vitcop_kproj_knorm(hidden, W, H, d, turned, ws, rope_cos=cos, rope_sin=sin, position_ids=_i32(position))
    vb.vitcop_rotary_axes(None, K, _i32(position[None]), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(np.zeros(F)), None, of_axes)
    size = (K[..., :F].double().abs() + K[..., F:].double().abs()).repeat(1, 1, 1, 2)
    tol = (HALF * (1 + HALF) + 2.0 ** -20) * size + HALF * (turned.double().abs() + of_axes.double().abs())
    assert ((turned.double() - of_axes.double()).abs() <= tol).all()
    assert not torch.equal(turned, K)


def _turn(seed, B=2, Hq=4, Hk=2, N=90, d=64, F=32):
    rng = np.random.default_rng(seed)
    q, k, position = _bf16(rng, B, N, Hq, d).transpose(1, 2), _bf16(rng, B, Hk, N, d), _i32(rng.integers(0, 9000, (3, B, N)))
    return q, k, position, torch.tensor(10000.0 ** (-np.arange(F) / F), dtype=torch.float64, device=DEV), _i32(np.arange(F) * 3 // F)


def test_turning_on_two_streams_and_in_a_graph():
    """Two streams at once; a captured turn, and the one back beside it, replayed on other rows and positions."""
    cases = [_turn(s) for s in (1, 2)]
    want = [vb.vitcop_rotary_axes(*c, *(torch.zeros_like(x) for x in c[:2])) for c in cases]
    outs = [tuple(torch.zeros_like(x) for x in c[:2]) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, o, s in zip(cases, outs, streams):
            with torch.cuda.stream(s):
                vb.vitcop_rotary_axes(*c, *o)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o, w in zip(outs, want) for x, y in zip(o, w))
    held, out, back = [x.clone() for x in cases[0]], [torch.zeros_like(x) for x in cases[0][:2]], [torch.zeros_like(x) for x in cases[0][:2]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vitcop_rotary_axes(*held, *out)
        vb.vitcop_rotary_axes(*out, *held[2:], *back, inverse=True)
    for c, w in ((cases[1], want[1]), (cases[0], want[0])):
        for x, y in zip(held, c):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for x, y, z, b in zip(out, w, c[:2], back):
            assert torch.equal(x, y)
            # (two roundings of half a place, of the size of either element of a pair)
            size = (z[..., :32].double().abs() + z[..., 32:].double().abs()).repeat(1, 1, 1, 2)
            assert ((b.double() - z.double()).abs() <= 2 * HALF * size + 2.0 ** -20 * size).all()


def test_tables_that_the_kernel_in_front_writes():
    """Positions and frequencies of a turn come from the kernel right in front of it, which the turn may be launched beside; nothing waits between the calls."""
    q, k, position, f, axis = _turn(3)
    zeros = [torch.zeros_like(x) for x in (q, k)]
    tables = [(position * n % 7000, f * (1 + n / 8), (axis + n) % 3) for n in range(1, 9)]
    want = [[x.clone() for x in vb.vitcop_rotary_axes(q, k, *t, *zeros)] for t in tables]
    held, outs = [x.clone() for x in tables[0]], [[torch.zeros_like(x) for x in (q, k)] for _ in tables]
    torch.cuda.synchronize()
    for t, o in zip(tables, outs):
        for x, y in zip(held, t):
            x.copy_(y)
        vb.vitcop_rotary_axes(q, k, *held, *o)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o, w in zip(outs, want) for x, y in zip(o, w))


@pytest.mark.parametrize("Tq", [3, 300])
def test_two_graphs_that_share_a_workspace(Tq):
    """Replayed in turn on one stream, each in either order."""
    B, H, R, d, N = 2, 2, 4, 128, 900
    ws = vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=N, d=d, Nv=Tq, D=H * R)
    cases = [_case(s, B, H, R, Tq, d, N)[1:] for s in (1, 2)]
    want = [_run(*c, None, 0.1, 500, 4)[0] for c in cases]
    outs, graphs = [torch.zeros_like(c[0]) for c in cases], [torch.cuda.CUDAGraph() for _ in cases]
    for c, o, g in zip(cases, outs, graphs):
        with torch.cuda.graph(g):
            vb.vitcop_window_attention(*c, None, o, ws, 0.1, 500, 4)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for o in outs:
            o.zero_()
        for i in order:
            graphs[i].replay()
        assert vb.vitcop_poll_status(ws) == vb.OK
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
