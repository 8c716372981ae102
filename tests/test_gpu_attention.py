"""Rotary positions with several axes and attention over bf16 rows on the GPU, against fp64 (``-m gpu``).

Rotary: the angle is a double's turns less the whole ones, in fp32 (2^-24 of half a turn: 2^-23 pi, 2^-48 |position| of the product's digits are less); sine,
cosine, two products and a sum in fp32, 2^-22 of |a| + |b| with the angle's; the result rounded to bf16, 2^-8 of it.
Attention, with HALF = 2^-8, half of bf16's last place:
  logits   fp32 sums of D exact products, in any order and with truncation: off by DELTA = 2^-22 D / 16 of scale sum |q k|, and 2^-21 of themselves
           on their way to the power of two
  weights  exp of that: exp(2 DELTA) - 1 (numerator and sum); rounded to bf16 (HALF), which counts towards the mean of V as sum p |v|, and, as
           the sum is of the weights as they were rounded, towards the quotient as |out|
  out      bf16 (HALF)
  lse      DELTA, and 2^-20 of 1 + |lse| for the logarithm and its products
"""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from paper_2601_17818_b200 import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = 2.0 ** -8
NO_WINDOW = 2 ** 31 - 1


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _bf16(rng, *shape, spread=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * spread).astype(np.float32)).bfloat16().to(DEV)


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------- rotary
def _rotary_case(seed, B, Hq, Hk, N, d, F, axes, n_pos=None, far=20000):
    rng = np.random.default_rng(seed)
    q, k = _bf16(rng, B, N, Hq, d).transpose(1, 2), _bf16(rng, B, Hk, N, d)
    position = rng.integers(-far, far, (axes, B, n_pos or N))
    inv_freq = 10000.0 ** (-np.arange(F) / max(F, 1))
    axis = rng.integers(0, axes, F)
    return rng, q, k, position, inv_freq, axis


def _check_rotary(x, y, before, position, inv_freq, axis, token=None, seq_len=None, inverse=False):
    F = len(inv_freq)
    want, written = oa.rotary(_f64(x), position, inv_freq, axis, token, seq_len, inverse)
    got, x = _f64(y), _f64(x)
    size = np.zeros(x.shape)
    size[..., :F] = size[..., F:2 * F] = np.abs(x[..., :F]) + np.abs(x[..., F:2 * F])
    off = np.abs(got - want)
    w = written[:, None, :, None] & np.ones(x.shape, bool)
    assert np.all(off[w] <= (HALF * np.abs(want) + 2.0 ** -21 * size)[w])
    assert np.array_equal(got[~w], _f64(before)[~w])
    copied = w & (np.arange(x.shape[3]) >= 2 * F)
    assert np.array_equal(got[copied], x[copied])


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("B,Hq,Hk,N,d,F,axes", [(1, 1, 1, 1, 16, 8, 1), (1, 32, 32, 1, 128, 64, 3), (2, 7, 1, 37, 128, 64, 3), (3, 4, 2, 130, 64, 16, 2),
                                                (1, 3, 5, 5, 72, 32, 4), (2, 2, 2, 9, 256, 128, 3), (1, 2, 2, 3, 512, 256, 2), (1, 2, 2, 6, 64, 0, 1),
                                                (5, 28, 4, 67, 128, 64, 3), (1, 300, 2, 3, 64, 32, 3), (65, 2, 1, 2, 64, 32, 3)])
def test_rows_are_turned(B, Hq, Hk, N, d, F, axes, inverse):
    _, q, k, position, f, axis = _rotary_case(N + d, B, Hq, Hk, N, d, F, axes)
    qo = torch.full((B, N, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    ko = torch.full((B, Hk, N, d), 7.0, dtype=torch.bfloat16, device=DEV)
    qb, kb = qo.clone(), ko.clone()
    vb.vitcop_rotary_axes(q, k, _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis), qo, ko, inverse=inverse)
    _check_rotary(q, qo, qb, position, f, axis, inverse=inverse)
    _check_rotary(k, ko, kb, position, f, axis, inverse=inverse)


def test_rows_take_the_positions_of_their_tokens_and_others_stay():
    B, N, n_pos = 4, 45, 99
    rng, q, k, position, f, axis = _rotary_case(3, B, 4, 2, N, 64, 32, 3, n_pos)
    token = rng.integers(-1, n_pos + 3, (B, N))
    token[0, :5] = [-7, n_pos - 1, n_pos, 2 ** 31 - 1, -2 ** 31]
    seq_len = [45, 0, 17, 400]
    args = _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis)
    for tk, sl in ((token, None), (token, seq_len), (None, seq_len)):
        qo, ko = (torch.full_like(x, 5.0, memory_format=torch.contiguous_format) for x in (q, k))
        qb, kb = qo.clone(), ko.clone()
        vb.vitcop_rotary_axes(q, k, *args, qo, ko, token=None if tk is None else _i32(tk), seq_len=None if sl is None else _i32(sl))
        _check_rotary(q, qo, qb, position, f, axis, tk, sl)
        _check_rotary(k, ko, kb, position, f, axis, tk, sl)
        for x, o, b, pair in ((q, qo, qb, 0), (k, ko, kb, 1)):                 # one of the two alone: the same
            alone = b.clone()
            vb.vitcop_rotary_axes(*((x, None) if pair == 0 else (None, x)), *args, *((alone, None) if pair == 0 else (None, alone)),
                                  token=None if tk is None else _i32(tk), seq_len=None if sl is None else _i32(sl))
            assert torch.equal(alone, o)


@pytest.mark.parametrize("heads_outside", [False, True])
@pytest.mark.parametrize("B,N", [(1, 21), (3, 21), (3, 1)])
def test_in_place_inside_one_projection(heads_outside, B, N):
    rng = np.random.default_rng(N)
    Hq, Hk, d, F = 4, 2, 64, 32
    qkv = _bf16(rng, B, Hq + 2 * Hk, N, d) if heads_outside else _bf16(rng, B, N, Hq + 2 * Hk, d).transpose(1, 2)
    before = qkv.clone()
    position, f, axis = rng.integers(0, 3000, (3, B, N)), 10000.0 ** (-np.arange(F) / F), np.arange(F) % 3
    args = _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    vb.vitcop_rotary_axes(q, k, *args, q, k)
    _check_rotary(before[:, :Hq], q, q, position, f, axis)
    _check_rotary(before[:, Hq:Hq + Hk], k, k, position, f, axis)
    assert torch.equal(qkv[:, Hq + Hk:], before[:, Hq + Hk:])
    apart = [torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k)]
    vb.vitcop_rotary_axes(before[:, :Hq], before[:, Hq:Hq + Hk], *args, *apart)
    assert torch.equal(apart[0], q) and torch.equal(apart[1], k)


def test_far_positions_keep_their_angle_and_one_axis_is_the_table_of_the_key_projection():
    """At positions up to 2^31 an angle in fp32 would be off by turns."""
    B, N, d, F = 1, 64, 128, 64
    rng, q, _, position, f, axis = _rotary_case(5, B, 3, 1, N, d, F, 1, far=2 ** 31 - 1)
    qo = torch.zeros_like(q)
    vb.vitcop_rotary_axes(q, None, _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis), qo, None)
    # (2^31 of the frequency's own digits: 2^-22 of a turn)
    want, _ = oa.rotary(_f64(q), position, f, axis)
    size = np.abs(_f64(q)[..., :F]) + np.abs(_f64(q)[..., F:])
    assert np.all(np.abs(_f64(qo) - want) <= HALF * np.abs(want) + 2.0 ** -18 * np.concatenate([size, size], -1))


def test_a_rotation_and_its_gradient_agree_with_differences():
    """Sum of g y has the gradient that turning g back gives; differences of the oracle along a direction say the same."""
    B, N, d, F = 2, 11, 64, 32
    rng, g, _, position, f, axis = _rotary_case(6, B, 4, 1, N, d, F, 3)
    dq = torch.empty_like(g, memory_format=torch.contiguous_format)
    vb.vitcop_rotary_axes(g, None, _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis), dq, None, inverse=True)
    x, u, step = rng.standard_normal((2, B, 4, N, d)).tolist(), rng.standard_normal((B, 4, N, d)), 1e-4
    x = np.array(x[0])
    plus, minus = (oa.rotary(x + e * u, position, f, axis)[0] for e in (step, -step))
    slope = ((plus - minus) / (2 * step) * _f64(g)).sum()
    bound = (np.abs(u) * (HALF + 2.0 ** -20) * 2 * np.abs(_f64(g)).max()).sum()
    assert abs((_f64(dq) * u).sum() - slope) <= bound


# ---------------------------------------------------------------------------------------------- attention
def _run(q, K, V, lens, scale, window=NO_WINDOW, n_sink=0, counts=None, tree=None, out=None, lse=None, workspace=None):
    B, Hq, Tq, d = q.shape
    H, N = K.shape[1], K.shape[2]
    out = torch.full((B, Tq, Hq, d), 9.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2) if out is None else out
    lse = torch.full((B, Hq, Tq), 9.0, device=DEV) if lse is None else lse
    ws = vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=N, d=d, Nv=Tq, D=Hq) if workspace is None else workspace
    length = None if lens is None else _i32(lens)
    count = None if counts is None else _i32(counts)
    if tree is None:
        vb.vitcop_window_attention(q, K, V, length, out, ws, scale, window, n_sink, query_len=count, lse=lse)
    else:
        vb.vitcop_tree_attention(q, K, V, length, torch.from_numpy(np.asarray(tree, np.int64)).to(DEV), out, ws, scale, query_len=count, lse=lse)
    assert vb.vitcop_poll_status(ws) == vb.OK
    return out, lse


def _check(q, K, V, lens, scale, out, lse, window=NO_WINDOW, n_sink=0, counts=None, tree=None):
    B, Hq, Tq, d = q.shape
    lens = [K.shape[2]] * B if lens is None else lens
    counts = [Tq] * B if counts is None else counts
    want, wlse, size, logit = oa.attention(_f64(q), _f64(K), _f64(V), lens, counts, scale, window, n_sink, tree)
    got, glse = _f64(out), lse.cpu().numpy().astype(np.float64)
    behind = np.isnan(want).all(-1) & np.isnan(wlse)
    behind &= np.arange(Tq) >= np.clip(counts, 0, Tq)[:, None, None]
    assert np.all(got[behind] == 9.0) and np.all(glse[behind] == 9.0)
    empty = np.isneginf(wlse)
    assert np.all(got[empty] == 0.0) and np.all(np.isneginf(glse[empty]))
    nan = np.isnan(wlse) & ~behind
    assert np.all(np.isnan(got[nan])) and np.all(np.isnan(glse[nan]))
    rest = ~(behind | empty | nan)
    delta = (2.0 ** -22 * (d / 16 + 2) * logit)[..., None]
    with np.errstate(invalid="ignore"):
        tol = HALF * (1 + HALF) * (size + 2 * np.abs(want)) + (np.exp(2 * delta) - 1) * (size + np.abs(want)) + 1e-37
        fine = np.abs(got - want) <= tol
    fine |= (np.isnan(want) & np.isnan(got)) | (np.isinf(want) & ((got == want) | np.isnan(got)))
    assert np.all(fine[rest])
    wlse, glse = np.where(rest, wlse, 0), np.where(rest, glse, 0)
    assert np.all(np.abs(glse - wlse)[rest] <= (delta[..., 0] + 2.0 ** -20 * (1 + np.abs(wlse)))[rest])


def _case(seed, B, H, R, Tq, d, N, spread=1.0):
    rng = np.random.default_rng(seed)
    K, V = _bf16(rng, B, H, N, d, spread=spread), _bf16(rng, B, N, H, d).transpose(1, 2)
    return rng, _bf16(rng, B, Tq, H * R, d).transpose(1, 2), K, V


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,R,Tq,N,window,n_sink", [(2, 1, 1, 70, NO_WINDOW, 0), (1, 7, 1, 300, 64, 4), (2, 4, 5, 129, 33, 16), (1, 1, 17, 64, 1, 0), (2, 2, 9, 40, 0, 3),
                                                    (1, 3, 11, 257, 100, 35), (1, 1, 1, 1, 5, 5), (1, 16, 3, 515, 256, 130), (2, 8, 40, 200, 50, 200)])
def test_windows_and_sinks(d, H, R, Tq, N, window, n_sink):
    B = 5
    rng, q, K, V = _case(N + d, B, H, R, Tq, d, N)
    lens = [N, max(0, N - 13), Tq, Tq // 2, 0]             # (more queries than rows, no rows)
    for le in (lens, None):
        out, lse = _run(q, K, V, le, d ** -0.5, window, n_sink)
        _check(q, K, V, le, d ** -0.5, out, lse, window, n_sink)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,R,N,window,n_sink", [(2, 1, 150, 40, 4), (1, 4, 77, NO_WINDOW, 0), (2, 3, 200, 64, 130), (1, 7, 33, 1, 0), (1, 1, 400, 130, 0)])
def test_prompts_of_a_padded_batch(d, H, R, N, window, n_sink):
    B = 4
    rng, q, K, V = _case(N * d, B, H, R, N, d, N)
    lens = [N, N - 17, 1, 0]
    for b in range(B):                                     # what lies behind a sequence is anything
        K[b, :, lens[b]:] = float("nan")
        V[b, :, lens[b]:] = float("inf")
        q[b, :, lens[b]:] = float("nan")
    out, lse = _run(q, K, V, lens, d ** -0.5, window, n_sink, counts=lens)
    _check(q, K, V, lens, d ** -0.5, out, lse, window, n_sink, counts=lens)


def test_query_counts_of_all_kinds():
    B, H, R, Tq, d, N = 6, 2, 2, 12, 64, 90
    rng, q, K, V = _case(1, B, H, R, Tq, d, N)
    lens, counts = [90, 50, 3, 400, -5, 90], [12, 5, 12, 1, 7, -3]
    out, lse = _run(q, K, V, lens, 0.2, 20, 2, counts=counts)
    _check(q, K, V, lens, 0.2, out, lse, 20, 2, counts=counts)


def _tree(rng, B, T, empty=True):
    words = np.zeros((B, T), np.uint64)
    for b in range(B):
        for t in range(T):
            parent = int(rng.integers(-1, t)) if t else -1
            words[b, t] = (words[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1 << t)
        if empty:
            words[b, int(rng.integers(0, T))] = 0
    return words.view(np.int64)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,R,Tq,N", [(2, 1, 25, 120), (1, 7, 60, 333), (2, 4, 64, 64), (1, 1, 1, 40), (1, 2, 33, 500), (1, 1, 7, 9)])
def test_trees(d, H, R, Tq, N):
    B = 5
    rng, q, K, V = _case(N + Tq, B, H, R, Tq, d, N)
    tree = _tree(rng, B, Tq)
    tree[0, 0] = -1                                        # all drafted tokens, those that come later too
    lens = [N, max(Tq, N - 20), Tq, max(Tq - 3, 0), 0]
    out, lse = _run(q, K, V, lens, d ** -0.5, tree=tree)
    _check(q, K, V, lens, d ** -0.5, out, lse, tree=tree)
    counts = [Tq, Tq // 2, 1, Tq, Tq]
    out, lse = _run(q, K, V, lens, d ** -0.5, tree=tree, counts=counts)
    _check(q, K, V, lens, d ** -0.5, out, lse, tree=tree, counts=counts)


def test_a_chain_is_causal():
    B, H, R, Tq, d, N = 2, 2, 4, 30, 128, 300
    rng, q, K, V = _case(2, B, H, R, Tq, d, N)
    tree = np.tile(np.array([(2 << t) - 1 for t in range(Tq)], np.int64), (B, 1))
    # (not the same bits: a tile of window rows ends at its last query's own row, one of a tree at the last drafted one, and parts are cut by that)
    for out, lse in (_run(q, K, V, [300, 100], 0.1, tree=tree), _run(q, K, V, [300, 100], 0.1)):
        _check(q, K, V, [300, 100], 0.1, out, lse, tree=tree)
        _check(q, K, V, [300, 100], 0.1, out, lse)


@pytest.mark.parametrize("Tq,R", [(6, 2), (40, 8), (300, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_that_are_no_numbers_reach_only_those_who_see_them(bad, d, Tq, R):
    B, H, N, window, n_sink = 2, 1, 330, 90, 5
    rng, q, K, V = _case(4, B, H, R, Tq, d, N)
    at = [0, 3, 4, 5, 40, 41, 200, 250, 285, 300, 328, 329]
    V[:, :, at] = bad
    V[1, 0, 290, 7] = bad
    out, lse = _run(q, K, V, None, d ** -0.5, window, n_sink)
    _check(q, K, V, None, d ** -0.5, out, lse, window, n_sink)
    V = _case(4, B, H, R, Tq, d, N)[3]
    K[:, :, at] = bad
    K[0, 0, 295, 0] = bad
    keep = torch.ones(N, dtype=torch.bool)
    out, lse = _run(q, K, V, None, d ** -0.5, window, n_sink)
    hidden = np.array([[not oa.seen_rows(N, Tq, t, window, n_sink)[at + [295]].any() for t in range(Tq)]] * B)
    got, clean = _f64(out), _f64(_run(q, torch.nan_to_num(K, 0.0, 0.0, 0.0), V, None, d ** -0.5, window, n_sink)[0])
    assert keep.all() and np.array_equal(got.transpose(0, 2, 1, 3)[hidden], clean.transpose(0, 2, 1, 3)[hidden])
    if bad != bad:
        sees = ~hidden
        sees[1] = [oa.seen_rows(N, Tq, t, window, n_sink)[at].any() for t in range(Tq)]
        assert np.isnan(got.transpose(0, 2, 1, 3)[sees]).all()


@pytest.mark.parametrize("Tq", [20, 200])
def test_drafted_rows_that_are_no_numbers(Tq):
    B, H, R, d, N = 1, 2, 4, 128, 260
    T = min(Tq, 64)
    rng, q, K, V = _case(5, B, H, R, T, d, N)
    tree = _tree(rng, B, T)
    V[:, :, N - T + 3::5] = float("nan")
    out, lse = _run(q, K, V, None, 0.1, tree=tree)
    _check(q, K, V, None, 0.1, out, lse, tree=tree)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0, 1e-30, 60.0])
@pytest.mark.parametrize("Tq", [3, 150])
def test_scales_and_sharp_logits(scale, Tq):
    B, H, R, d, N = 2, 1, 3, 64, 210
    rng, q, K, V = _case(6, B, H, R, Tq, d, N)
    out, lse = _run(q, K, V, [210, 170], scale, 100, 3)
    _check(q, K, V, [210, 170], scale, out, lse, 100, 3)


@pytest.mark.parametrize("Tq", [2, 140])
def test_logits_that_rise_and_fall_by_thousands(Tq):
    """The running maximum moves many times, and what came before it is gone."""
    B, H, R, d, N = 1, 1, 2, 128, 1000
    rng, q, K, V = _case(7, B, H, R, Tq, d, N)
    K *= torch.from_numpy(np.linspace(0.1, 40, N)[rng.permutation(N)].astype(np.float32)).bfloat16().to(DEV).view(1, 1, N, 1)
    out, lse = _run(q, K, V, None, 1.0, 700, 8)
    _check(q, K, V, None, 1.0, out, lse, 700, 8)


@pytest.mark.parametrize("Tq", [1, 130])
def test_strides_and_shared_tensors(Tq):
    """Keys and values side by side in one tensor, one stored head for all samples (stride 0), rows of the output apart."""
    rng = np.random.default_rng(8)
    B, H, R, d, N = 3, 2, 2, 64, 150
    kv = _bf16(rng, B, N, 2, H, d)
    K, V = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    q = _bf16(rng, B, H * R, Tq, 2 * d)[..., d:]
    wide = torch.full((B, H * R, Tq, 3 * d), 9.0, dtype=torch.bfloat16, device=DEV)
    out, lse = _run(q, K, V, [150, 149, 140], 0.1, 60, 7, out=wide[..., d:2 * d])
    _check(q, K, V, [150, 149, 140], 0.1, out, lse, 60, 7)
    assert (wide[..., :d] == 9.0).all() and (wide[..., 2 * d:] == 9.0).all()
    for one in (_bf16(rng, 1, 1, N, d).expand(B, H, N, d), _bf16(rng, 1, H, N, d).expand(B, H, N, d), _bf16(rng, B, H, 1, d).expand(B, H, N, d)):
        out, lse = _run(q, one, V, None, 0.1, 60, 7)
        _check(q, one, V, None, 0.1, out, lse, 60, 7)
        out, lse = _run(q, K, one, None, 0.1, 60, 7)
        _check(q, K, one, None, 0.1, out, lse, 60, 7)


@pytest.mark.parametrize("Tq", [1, 200])
def test_rows_beyond_32_bits(Tq):
    """A cache of 2^25 rows of 64 elements: offsets of 2^31 elements and more."""
    d, N = 64, (1 << 25) + 1000
    K = torch.zeros(1, 1, N, d, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros(1, 1, N, d, dtype=torch.bfloat16, device=DEV)
    rng, q, k, v = _case(9, 1, 1, 2, Tq, d, 600)
    K[:, :, -600:], V[:, :, -600:] = k, v
    K[:, :, :8], V[:, :, :8] = k[:, :, :8], v[:, :, :8]
    out, lse = _run(q, K, V, None, 0.1, 300, 8)
    near = torch.cat([k[:, :, :8], k[:, :, 600 - Tq - 300:]], 2), torch.cat([v[:, :, :8], v[:, :, 600 - Tq - 300:]], 2)
    _check(q, *near, None, 0.1, out, lse, 300, 8)
    del K, V
    torch.cuda.empty_cache()


def _check_long(q, K, V, lens, counts, scale, out, lse, window=NO_WINDOW, n_sink=0, tree=None):
    """As _check, by torch in fp64 on the GPU, a head at a time.  Rows of V that are no numbers count with those who see them alone."""
    B, Hq, Tq, d = q.shape
    R = Hq // K.shape[1]
    for b in range(B):
        n, m = min(max(lens[b], 0), K.shape[2]), min(max(counts[b], 0), Tq)
        j, p = torch.arange(n, device=DEV)[None], n - m + torch.arange(m, device=DEV)[:, None]
        if tree is None:
            seen = (j <= p) & ((j < n_sink) | (j + window > p))
        else:
            seen = (j < n - m) | ((tree[b, :m, None] >> (j - (n - m)).clamp(0, 63)) & 1 == 1)
        seen &= p >= 0
        for h in range(Hq):
            qd, k, v = q[b, h, :m].double(), K[b, h // R, :n].double(), V[b, h // R, :n].double()
            z = torch.where(seen, qd @ k.T * scale, -np.inf)
            wlse = torch.logsumexp(z, -1)
            w = torch.exp(z - wlse[:, None])
            empty = torch.isneginf(wlse)
            w[empty] = 0
            odd = (seen.double() @ (~torch.isfinite(v)).double() > 0) | torch.isnan(wlse)[:, None]
            v = v.nan_to_num(0.0, 0.0, 0.0)
            want, size = w @ v, w @ v.abs()
            delta = 2.0 ** -22 * (d / 16 + 2) * abs(scale) * torch.where(seen, qd.abs() @ k.abs().T, 0).amax(-1, keepdim=True) if n else torch.zeros(m, 1, device=DEV)
            tol = HALF * (1 + HALF) * (size + 2 * want.abs()) + (torch.exp(2 * delta) - 1) * (size + want.abs()) + 1e-37
            got = out[b, h, :m].double()
            assert (((got - want).abs() <= tol) | odd).all()
            assert (~torch.isfinite(got) == odd).all()
            assert (got[empty] == 0).all() and torch.isneginf(lse[b, h, :m][empty]).all()
            off, fine = (lse[b, h, :m].double() - wlse).abs(), ~empty & ~torch.isnan(wlse)
            assert (off <= delta[:, 0] + 2.0 ** -20 * (1 + wlse.abs()))[fine].all()
            assert torch.isnan(lse[b, h, :m][torch.isnan(wlse)]).all()
        assert (out[b, :, m:] == 9.0).all() and (lse[b, :, m:] == 9.0).all()


def _kernels_of(*args, **kw):
    """(out, lse, names of the kernels that a call has launched)"""
    vb.vitcop_kernel_timing_begin()
    try:
        out, lse = _run(*args, **kw)
    finally:
        names = set(vb.vitcop_kernel_timing_end())
    return out, lse, names


MANY = {"attention_tiles_kernel"}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,R,Tq,N,window,n_sink", [(16, 32, 1, 256, 300, 1, 0), (16, 32, 1, 256, 290, 0, 3), (16, 32, 1, 200, 301, 0, 0), (12, 32, 1, 260, 259, 40, 1000),
                                                      (2, 8, 4, 300, 2300, 1700, 35), (3, 4, 7, 129, 1999, 1024, 0), (4, 8, 5, 515, 1500, 333, 130), (4, 4, 64, 50, 1500, 900, 9),
                                                      (9, 32, 1, 131, 140, NO_WINDOW, 0)])
def test_many_rows_windows_and_sinks(d, B, H, R, Tq, N, window, n_sink):
    rng, q, K, V = _case(N + d, B, H, R, Tq, d, N)
    lens = ([N, max(0, N - 13), Tq // 2, 0, 1, Tq, Tq - 1] * 3)[:B]            # (more queries than rows, no rows)
    out, lse, names = _kernels_of(q, K, V, lens, d ** -0.5, window, n_sink)
    assert names == MANY
    _check_long(q, K, V, lens, [Tq] * B, d ** -0.5, out, lse, window, n_sink)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("B,H,R,N,window,n_sink", [(5, 16, 2, 700, 256, 35), (6, 8, 7, 400, 100, 5), (3, 4, 4, 1100, NO_WINDOW, 0)])
def test_many_rows_padded_behind_with_anything(bad, B, H, R, N, window, n_sink):
    d = 128
    rng, q, K, V = _case(N, B, H, R, N, d, N)
    lens = [N, N - 17, N // 2, 1, 0, N // 3][:B]
    for b in range(B):
        K[b, :, lens[b]:], V[b, :, lens[b]:], q[b, :, lens[b]:] = bad, bad, float("nan")
    out, lse, names = _kernels_of(q, K, V, lens, d ** -0.5, window, n_sink, counts=lens)
    assert names == MANY
    _check_long(q, K, V, lens, lens, d ** -0.5, out, lse, window, n_sink)


@pytest.mark.parametrize("B,H,R,N", [(31, 8, 2, 600), (32, 16, 1, 550), (33, 16, 1, 550), (40, 3, 7, 300)])
def test_many_rows_every_sample_its_own_number(B, H, R, N):
    """Also none at all, in samples in front, behind and between."""
    d = 64
    rng, q, K, V = _case(B, B, H, R, N, d, N)
    counts = rng.integers(0, N + 1, B)
    counts[[0, 3, 4, B - 1]], counts[5] = [0, -2, 0, 0], N + 7
    lens = np.minimum(N, np.clip(counts, 0, N) + rng.integers(0, 90, B)).tolist()
    counts = counts.tolist()
    out, lse, names = _kernels_of(q, K, V, lens, d ** -0.5, 130, 9, counts=counts)
    assert names == MANY
    _check_long(q, K, V, lens, counts, d ** -0.5, out, lse, 130, 9)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,R,Tq,N,window,n_sink", [(2, 8, 4, 300, 1500, 700, 40), (16, 32, 1, 256, 400, 90, 5)])
def test_many_rows_and_values_that_are_no_numbers(bad, d, B, H, R, Tq, N, window, n_sink):
    """A single element, whole rows, at the edges of windows and sinks, one after the other."""
    rng, q, K, V = _case(d, B, H, R, Tq, d, N)
    at = sorted({0, 4, n_sink - 1, n_sink, N - Tq - window, N - Tq - window + 1, N - Tq - window + 60, N - Tq, N - Tq + 77, N - 130, N - 129, N - 2})
    V[:, :, at] = bad
    V[1, 0, N - 140, 7] = bad
    out, lse, names = _kernels_of(q, K, V, None, d ** -0.5, window, n_sink)
    assert names == MANY
    _check_long(q, K, V, [N] * B, [Tq] * B, d ** -0.5, out, lse, window, n_sink)


def test_many_rows_and_keys_that_are_no_numbers():
    B, H, R, Tq, d, N, window, n_sink = 2, 8, 4, 300, 128, 1500, 700, 40
    rng, q, K, V = _case(3, B, H, R, Tq, d, N)
    K[0, :, [3, N - 200, N - 1]] = float("nan")
    K[1, 2, N - 900, 5] = float("inf")
    q[1, 9, 17, 3] = float("nan")
    out, lse, names = _kernels_of(q, K, V, None, d ** -0.5, window, n_sink)
    assert names == MANY
    j, p = torch.arange(N, device=DEV)[None], N - Tq + torch.arange(Tq, device=DEV)[:, None]
    seen = (j <= p) & ((j < n_sink) | (j + window > p))
    hit = seen[:, [3, N - 200, N - 1]].any(1)
    assert torch.isnan(out[0, :, hit]).all() and torch.isfinite(out[0, :, ~hit]).all()
    assert torch.isnan(out[1, 9, 17]).all()
    clean = K.nan_to_num(0.0, 0.0, 0.0)
    want, _ = _run(q.nan_to_num(0.0), clean, V, None, d ** -0.5, window, n_sink)
    same = [h for h in range(H * R) if h // R != 2 and h != 9]
    assert torch.equal(out[1, same], want[1, same])


@pytest.mark.parametrize("scale", [0.0, -0.3, 60.0])
def test_many_rows_scales_and_values_near_the_end(scale):
    B, H, R, Tq, d, N = 2, 8, 4, 260, 64, 1400
    rng, q, K, V = _case(6, B, H, R, Tq, d, N)
    V[0] *= 2.0 ** 125 / V[0].abs().max()
    out, lse, names = _kernels_of(q, K, V, [N, N - 70], scale, 1000, 3)
    assert names == MANY
    _check_long(q, K, V, [N, N - 70], [Tq] * B, scale, out, lse, 1000, 3)


def test_many_rows_strides_and_shared_tensors():
    """One stored head for all samples, or heads; queries and output apart, the latter at odd multiples of 16 bytes; a row for all tokens, which the other
    kernel takes."""
    rng = np.random.default_rng(8)
    B, H, R, d, N, Tq = 3, 4, 4, 128, 1500, 270
    V = _bf16(rng, B, N, H, d).transpose(1, 2)
    q = _bf16(rng, B, H * R, Tq, 2 * d)[..., d:]
    wide = torch.full((B, H * R, Tq, 2 * d + 8), 9.0, dtype=torch.bfloat16, device=DEV)
    lens = [N, N - 1, 1000]
    for one in (_bf16(rng, 1, H, N, d).expand(B, H, N, d), _bf16(rng, 1, 1, N, d).expand(B, H, N, d), _bf16(rng, B, 1, N, d).expand(B, H, N, d)):
        for k, v in ((one, V), (V, one)):
            wide.fill_(9.0)
            out, lse, names = _kernels_of(q, k, v, lens, 0.1, 900, 7, out=wide[..., 8:d + 8])
            assert names == MANY
            _check_long(q, k, v, lens, [Tq] * B, 0.1, out, lse, 900, 7)
            assert (wide[..., :8] == 9.0).all() and (wide[..., d + 8:] == 9.0).all()
    one = _bf16(rng, B, H, 1, d).expand(B, H, N, d)
    out, lse, names = _kernels_of(q, one, V, lens, 0.1, 900, 7)
    assert names == {"attention_few_kernel"}
    _check_long(q, one, V, lens, [Tq] * B, 0.1, out, lse, 900, 7)
    shared = _bf16(rng, 1, H * R, Tq, d).expand(B, H * R, Tq, d)
    out, lse, names = _kernels_of(shared, V, V, lens, 0.1, 900, 7)
    assert names == MANY
    _check_long(shared, V, V, lens, [Tq] * B, 0.1, out, lse, 900, 7)


@pytest.mark.parametrize("bad", [0.0, float("nan")])
@pytest.mark.parametrize("B,H,R,Tq,N,d", [(8, 4, 7, 60, 3000, 128), (8, 8, 8, 64, 2500, 64), (16, 32, 1, 64, 1300, 128)])
def test_many_rows_of_trees(bad, B, H, R, Tq, N, d):
    rng, q, K, V = _case(N, B, H, R, Tq, d, N)
    lens = ([N, N - 1, Tq, Tq - 3, 5, 0, N - 64, N // 2] * 2)[:B]
    tree = torch.from_numpy(_tree(rng, B, Tq)).to(DEV)
    tree[0, 0] = -1
    for b in range(B):
        V[b, :, max(0, lens[b] - Tq + 2):lens[b]:5] += bad
    out, lse, names = _kernels_of(q, K, V, lens, d ** -0.5, tree=tree.cpu().numpy())
    assert names == MANY
    _check_long(q, K, V, lens, [Tq] * B, d ** -0.5, out, lse, tree=tree)


@pytest.mark.parametrize("B,H,R,N,d,window,n_sink", [(1, 1, 7, 2990, 128, 700, 64), (2, 2, 2, 1501, 64, 900, 0), (3, 8, 8, 901, 128, 200, 16), (1, 2, 1, 5000, 128, NO_WINDOW, 0),
                                                     (1, 1, 7, 3333, 64, 2000, 130), (5, 16, 1, 1290, 64, 300, 4), (1, 1, 64, 600, 128, 333, 3), (1, 1, 65, 90, 128, 33, 3)])
def test_long_prompts(B, H, R, N, d, window, n_sink):
    """Many blocks an item, many items a CTA."""
    rng, q, K, V = _case(N, B, H, R, N, d, N)
    lens = [N, 3 * N // 4, N // 5, N - 1, 1][:B]
    out, lse = _run(q, K, V, lens, d ** -0.5, window, n_sink, counts=lens)
    _check_long(q, K, V, lens, lens, d ** -0.5, out, lse, window, n_sink)
    out, lse = _run(q[:, :, :N // 3], K, V, lens, d ** -0.5, window, n_sink)   # a chunk of a prompt, longer than some sequences
    _check_long(q[:, :, :N // 3], K, V, lens, [N // 3] * B, d ** -0.5, out, lse, window, n_sink)


@pytest.mark.parametrize("B,H,R,Tq,N,d", [(8, 4, 7, 60, 4672, 128), (1, 2, 8, 64, 16000, 64), (3, 32, 1, 64, 1111, 128), (2, 1, 7, 5, 9000, 128), (1, 4, 7, 1, 16512, 128)])
def test_long_caches_and_large_trees(B, H, R, Tq, N, d):
    rng, q, K, V = _case(N, B, H, R, Tq, d, N)
    lens = [N, N - 1, Tq + 7, N // 2, N // 3, 77, N - 64, N // 4][:B]
    tree = torch.from_numpy(_tree(rng, B, Tq)).to(DEV)
    out, lse = _run(q, K, V, lens, d ** -0.5, tree=tree.cpu().numpy())
    _check_long(q, K, V, lens, [Tq] * B, d ** -0.5, out, lse, tree=tree)
    for window, n_sink in ((N // 2, 64), (130, 0)):
        out, lse = _run(q, K, V, lens, d ** -0.5, window, n_sink)
        _check_long(q, K, V, lens, [Tq] * B, d ** -0.5, out, lse, window, n_sink)


@pytest.mark.parametrize("roles", [1, 2, 4])
@pytest.mark.parametrize("B,N,Tq,window", [(1, 3000, 300, 2500), (16, 900, 900, 500)])
def test_a_wait_that_ran_out_is_reported(roles, B, N, Tq, window):
    """One role of every CTA gives up at once, with copies and products of the others in flight (CTAs of a cluster on one item; CTAs with items in
    turn); the next call is right again."""
    H, R, d = 2, 4, 128
    rng, q, K, V = _case(15, B, H, R, Tq, d, N)
    ws, out = vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=N, d=d, Nv=Tq, D=H * R), torch.zeros_like(q)
    try:
        vb.vitcop_set_wait_limit(0, roles)
        vb.vitcop_window_attention(q, K, V, None, out, ws, d ** -0.5, window, 4)
        assert vb.vitcop_poll_status(ws) == vb.ERR_TIMEOUT
    finally:
        vb.vitcop_set_wait_limit(0, 0)
    out, lse = _run(q, K, V, None, d ** -0.5, window, 4, workspace=ws)
    again, lse2 = _run(q, K, V, None, d ** -0.5, window, 4)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    _check_long(q[:1], K[:1], V[:1], [N], [Tq], d ** -0.5, out, lse, window, 4)


def test_no_rows_and_nothing_to_do():
    rng, q, K, V = _case(10, 2, 2, 2, 3, 64, 40)
    out, lse = _run(q, K[:, :, :0], V[:, :, :0], None, 0.1)
    assert (out == 0).all() and torch.isneginf(lse).all()
    for e in (q[:0], q[:, :, :0]):
        ws = vb.alloc_workspace(vb.OP_ATTENTION)
        ws.fill_(255)
        vb.vitcop_window_attention(e, K[:e.shape[0]], V[:e.shape[0]], None, torch.empty_like(e), ws, 0.1, 5)
        assert vb.vitcop_poll_status(ws) == vb.OK


def test_without_lse_and_the_same_bits_again():
    rng, q, K, V = _case(11, 3, 2, 4, 20, 128, 700)
    ws = vb.alloc_workspace(vb.OP_ATTENTION, B=3, H=2, N=700, d=128, Nv=20, D=8)
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    vb.vitcop_window_attention(q, K, V, None, a, ws, 0.1, 300, 4)
    want, _ = _run(q, K, V, None, 0.1, 300, 4)
    for _ in range(5):
        vb.vitcop_window_attention(q, K, V, None, b, ws, 0.1, 300, 4)
        assert torch.equal(a, b) and torch.equal(a, want)


@pytest.mark.parametrize("Tq", [1, 256])
def test_streams_and_graphs(Tq):
    """Two streams with a workspace each; a captured call replayed on other lengths, beside an eager one; other queries the next time."""
    B, H, R, d, N = 2, 2, 2, 128, 600
    rng, q, K, V = _case(12, B, H, R, Tq, d, N)
    q2 = _case(13, B, H, R, Tq, d, N)[1]
    want = [_run(x, K, V, [600, 333], 0.1, 200, 4)[0].clone() for x in (q, q2)]
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=N, d=d, Nv=Tq, D=H * R) for _ in range(2)]
    outs, lens = [torch.zeros_like(q) for _ in range(2)], _i32([600, 333])
    torch.cuda.synchronize()
    for _ in range(10):
        for x, s, w, o in zip((q, q2), streams, ws, outs):
            with torch.cuda.stream(s):
                vb.vitcop_window_attention(x, K, V, lens, o, w, 0.1, 200, 4)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    x, o, length = q.clone(), torch.zeros_like(q), lens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vitcop_window_attention(x, K, V, length, o, ws[0], 0.1, 200, 4)
    for case in ((q, [600, 333]), (q2, [400, 260]), (q2, [600, 333])):
        x.copy_(case[0])
        length.copy_(_i32(case[1]))
        graph.replay()
        eager = torch.zeros_like(q)
        vb.vitcop_window_attention(case[0], K, V, _i32(case[1]), eager, ws[1], 0.1, 200, 4)
        torch.cuda.synchronize()
        assert torch.equal(o, eager)
    assert vb.vitcop_poll_status(ws[0]) == vb.OK


def test_a_pruned_sequence_goes_on():
    """The run of them: queries and keys turned on the grid, a prompt attended over, the sequence pruned, what is left turned anew by the positions it
    had, a token and a tree of drafted ones attended over it."""
    rng = np.random.default_rng(14)
    B, H, R, d, T, n, budget = 2, 2, 2, 64, 10, 144, 40
    N, Dh, F = n + T, 64, 32
    Hq, front = H * R, T // 2
    hidden = _bf16(rng, B, N, Dh)
    q, k, V = _bf16(rng, B, Hq, N, d), _bf16(rng, B, H, N, d), _bf16(rng, B, H, N, d)
    position = np.zeros((3, B, N), np.int64)
    for i in range(N):
        r = i - front
        position[:, :, i] = [[i]] * 3 if r < 0 else ([[front], [front + r // 12], [front + r % 12]] if r < n else [[front + 12 + r - n]] * 3)
    f, axis = 10000.0 ** (-np.arange(F) / F), np.arange(F) * 3 // F
    pos, inv, ax = _i32(position), torch.tensor(f, dtype=torch.float64, device=DEV), _i32(axis)
    qt, kt = torch.empty_like(q), torch.empty_like(k)
    vb.vitcop_rotary_axes(q, k, pos, inv, ax, qt, kt)
    _check_rotary(q, qt, qt, position, f, axis)
    out, lse = _run(qt, kt, V, None, d ** -0.5, 64, front)
    _check(qt, kt, V, None, d ** -0.5, out, lse, 64, front)
    # a Stage III step, on the keys as they are cached
    Ncap = T + budget + 14
    ho, Ko, Vo = torch.zeros(B, Ncap, Dh, dtype=torch.bfloat16, device=DEV), *(torch.zeros(B, H, Ncap, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    out_len, kept = _i32([0] * B), torch.full((B, Ncap), -1, dtype=torch.int32, device=DEV)
    ws = vb.alloc_workspace(vb.OP_PRUNE_STEP, B=B, Nv=n)
    vb.vitcop_prune_step(hidden, kt, V, front, n, n, budget, ho, Ko, Vo, out_len, ws, kept_pos=kept)
    assert out_len.tolist() == [T + budget] * B
    # the next layer's rows of what is left
    q2, k2 = _bf16(rng, B, Hq, Ncap, d), _bf16(rng, B, H, Ncap, d)
    q3, k3 = q2.clone(), k2.clone()
    vb.vitcop_rotary_axes(q3, k3, pos, inv, ax, q3, k3, token=kept)
    _check_rotary(q2, q3, q2, position, f, axis, kept.cpu().numpy())
    _check_rotary(k2, k3, k2, position, f, axis, kept.cpu().numpy())
    # the token of a step over the pruned cache, then a tree of drafted ones
    Ko[:, :, T + budget:], Vo[:, :, T + budget:] = _bf16(rng, B, H, 14, d), _bf16(rng, B, H, 14, d)
    x = _bf16(rng, B, Hq, 1, d)
    o, ls = _run(x, Ko, Vo, (out_len + 1).tolist(), d ** -0.5, 32, front)
    _check(x, Ko, Vo, (out_len + 1).tolist(), d ** -0.5, o, ls, 32, front)
    x, tree = _bf16(rng, B, Hq, 12, d), _tree(rng, B, 12, empty=False)
    o, ls = _run(x, Ko, Vo, (out_len + 12).tolist(), d ** -0.5, tree=tree)
    _check(x, Ko, Vo, (out_len + 12).tolist(), d ** -0.5, o, ls, tree=tree)
