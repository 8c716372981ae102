"""The K/V cache in 4 bits on the GPU, against fp64 (``-m gpu``): rows written and read back, attention over it, and the run of
them behind a pruning step.

Codes, scales and centres have to be the oracle's.  Values read back are its values rounded to bf16 (half of the last place, 2^-8 of
the value; bf16 of an fp32 that was itself rounded: the same and 2^-23).  Attention:
  logits   fp32 sums of products in which a code stands as up to 271 / 2 + 136 and is brought back to its centre: every product and partial sum
           is off by at most 2^-20 of sum |q| (280 s + |m|) per group, all of them together by DELTA below
  weights  enter the products in bf16 (2^-8): those of the centres once, those of the codes once more with the scale; or, where
           there are many query rows, the weights once and the values of V, as they are read back (2^-8).  Either way the part
           that a row adds is off by at most 2^-8 (2 |code - 8| s + |m|) + 2^-8 (|code - 8| s + |m|), and the products of the two
  out      bf16 (2^-8), and the weights' own error, exp(2 delta) - 1
"""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2601_17818_b200 import binding as vb
from paper_2601_17818_b200 import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = 2.0 ** -8                                           # half of bf16's last place


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _bf16(rng, *shape, spread=1.0, offset=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * spread + offset).astype(np.float32)).bfloat16().to(DEV)


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def _cache(B, H, Ncap, d, byte=0xFF):
    """Full of NaN scales and centres (or another byte), as memory that nobody wrote may be."""
    return torch.full((B, H, Ncap // 32, 40 * d), byte, dtype=torch.uint8, device=DEV)


def _same_rows(cache, b, rows, K, V):
    """Rows ``rows`` of sample b hold what the oracle makes of K, V [H, len(rows), d]."""
    held = oc.unpack(cache.cpu().numpy()[b:b + 1])
    for x, (s, m, code) in zip((K, V), held):
        if x is None:
            continue
        ws, wm, wc = oc.quantise(x)
        assert np.array_equal(s[0][:, rows], ws, equal_nan=True) and np.array_equal(m[0][:, rows], wm)
        assert np.array_equal(code[0][:, rows], wc)


def _untouched(before, after, b, rows, K=True, V=True):
    """Bytes of sample b outside the rows (and halves) written are as they were."""
    d = before.shape[3] // 40
    G = d // 32
    owner = np.zeros(40 * d, np.int64)                     # token of every byte of a block
    for half in (0, 20 * d):
        for r in range(32):
            owner[half + r * d // 2: half + (r + 1) * d // 2] = r
            owner[half + 16 * d + 2 * r * G: half + 16 * d + 2 * (r + 1) * G] = r
    owner[18 * d:20 * d] = np.repeat(np.arange(32), 2 * G)
    owner[38 * d:40 * d] = np.tile(np.repeat(np.arange(32), 2), G)
    token = owner[None, :] + 32 * np.arange(before.shape[2])[:, None]
    written = np.isin(token, np.asarray(rows, np.int64))
    written[:, :20 * d] &= K
    written[:, 20 * d:] &= V
    x, y = before.cpu().numpy()[b], after.cpu().numpy()[b]
    assert np.array_equal(x[:, ~written], y[:, ~written])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("N,lens", [(1, [0, 31, 32]), (33, [0, 5, 64]), (100, [0, 1, 96]), (7, [95, 96, 92]), (0, [3, 0, 96]), (40, None)])
def test_rows_are_written_as_the_oracle_holds_them(d, N, lens):
    rng = np.random.default_rng(d + N)
    B, H, Ncap = 3, 2, 96
    K, V = _bf16(rng, B, N, H, d).transpose(1, 2), _bf16(rng, B, H, N, d, spread=3.0, offset=0.7)
    if N > 2:                                              # few bits: values in the middle between two steps
        K[0] = torch.from_numpy(rng.integers(-8, 9, (H, N, d)) / 4.0).bfloat16().to(DEV)
        V[1, 0, 0, :32] = 0.0
    cache, new_len = _cache(B, H, Ncap, d), _i32([-5] * B)
    before = cache.clone()
    vb.vitcop_cache_write(K, V, cache, new_len, cache_len=None if lens is None else _i32(lens))
    lens = lens or [0] * B
    assert new_len.tolist() == [n + N for n in lens]
    for b in range(B):
        rows = [lens[b] + i for i in range(N) if lens[b] + i < Ncap]
        _same_rows(cache, b, rows, _f64(K)[b, :, :len(rows)], _f64(V)[b, :, :len(rows)])
        _untouched(before, cache, b, rows)


def test_write_of_one_half_and_of_short_sequences():
    rng = np.random.default_rng(1)
    B, H, N, d, Ncap = 4, 3, 70, 64, 128
    K, V, seq = _bf16(rng, B, H, N, d), _bf16(rng, B, H, N, d), [70, 0, 33, 500]
    for k, v in ((K, None), (None, V)):
        cache, new_len = _cache(B, H, Ncap, d, 0x5A), _i32([0] * B)
        before = cache.clone()
        vb.vitcop_cache_write(k, v, cache, new_len, cache_len=_i32([10, 10, -7, 127]), seq_len=_i32(seq))
        assert new_len.tolist() == [80, 10, 33, 197]
        for b, (start, n) in enumerate(((10, 70), (10, 0), (0, 33), (127, 1))):
            rows = list(range(start, start + n))
            _same_rows(cache, b, rows, None if k is None else _f64(K)[b, :, :n], None if v is None else _f64(V)[b, :, :n])
            _untouched(before, cache, b, rows, K=k is not None, V=v is not None)


def test_special_groups_are_held_as_stated():
    d, N = 64, 8
    x = torch.zeros(1, 1, N, d)
    x[0, 0, 0] = 7.5
    x[0, 0, 1, 3], x[0, 0, 2, 40], x[0, 0, 3, 5] = float("nan"), float("inf"), float("-inf")
    x[0, 0, 4, 5], x[0, 0, 4, 6] = 3.3e38, -3.3e38
    x[0, 0, 5, 0] = 2.0 ** -99
    x[0, 0, 6, 0], x[0, 0, 6, 1] = 2.9e38, -1e37
    x[0, 0, 7] = torch.arange(d) * 1e-5 - 3e-4
    x = x.bfloat16().to(DEV)
    cache, n = _cache(1, 1, 32, d, 0), _i32([0])
    vb.vitcop_cache_write(x, x, cache, n)
    rows = list(range(N))
    _same_rows(cache, 0, rows, _f64(x)[0], _f64(x)[0])
    K, V = torch.zeros_like(x), torch.zeros_like(x)
    vb.vitcop_cache_read(cache, n, K, V)
    want = oc.round_bf16(oc.values(*oc.quantise(_f64(x))))
    assert np.array_equal(_f64(K), want, equal_nan=True) and np.array_equal(_f64(V), want, equal_nan=True)
    assert torch.isnan(K[0, 0, 1, :32]).all() and not torch.isnan(K[0, 0, 1, 32:]).any()


@pytest.mark.parametrize("vis_start,vis_len,T_behind", [(0, 40, 0), (5, 40, 9), (7, [40, 3, 0, 25], 4)])
def test_a_keep_list_gives_the_rows_of_the_compaction(vis_start, vis_len, T_behind):
    rng = np.random.default_rng(vis_start)
    B, H, d, cap, stride = 4, 2, 128, 40, 17
    lens = [vis_len] * B if isinstance(vis_len, int) else vis_len
    N = vis_start + cap + T_behind
    seq = [vis_start + n + T_behind for n in lens]
    n_keep = [min(n, k) for n, k in zip(lens, (17, 1, 0, 12))]
    keep = np.zeros((B, stride), np.int64)
    for b in range(B):
        keep[b, :n_keep[b]] = np.sort(rng.permutation(lens[b])[:n_keep[b]])
    K, V = _bf16(rng, B, H, N, d), _bf16(rng, B, H, N, d)
    Ncap = 64
    K_out, V_out, out_len = torch.zeros(B, H, Ncap, d, dtype=torch.bfloat16, device=DEV), torch.zeros(B, H, Ncap, d, dtype=torch.bfloat16, device=DEV), _i32([0] * B)
    vl = vis_len if isinstance(vis_len, int) else _i32(vis_len)
    vb.vitcop_compact_kv(None, K, V, vis_start, vl, _i32(keep), _i32(n_keep), None, K_out, V_out, out_len, seq_len=_i32(seq))
    cache, new_len = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, new_len, cache_len=_i32([0, 3, 0, 1]), seq_len=_i32(seq), vis_start=vis_start, vis_len=vl,
                          keep_idx=_i32(keep), n_keep=_i32(n_keep))
    rows = out_len.tolist()
    assert new_len.tolist() == [n + s for n, s in zip(rows, (0, 3, 0, 1))]
    for b, start in enumerate((0, 3, 0, 1)):
        _same_rows(cache, b, list(range(start, start + rows[b])), _f64(K_out)[b, :, :rows[b]], _f64(V_out)[b, :, :rows[b]])


def test_indices_out_of_the_span_stay_inside():
    rng = np.random.default_rng(8)
    K = _bf16(rng, 1, 1, 30, 64)
    cache, n = _cache(1, 1, 32, 64), _i32([0])
    vb.vitcop_cache_write(K, K, cache, n, vis_start=4, vis_len=20, keep_idx=_i32([[-3, 5, 90000]]), n_keep=_i32([50]))
    assert n.tolist() == [13]
    src = [0, 1, 2, 3, 4, 9, 23] + list(range(24, 30))
    _same_rows(cache, 0, list(range(13)), _f64(K)[0][:, src], _f64(K)[0][:, src])


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_come_back(d):
    rng = np.random.default_rng(d)
    B, H, Ncap, N_out = 4, 2, 96, 50
    Kv, Vv = oc.round_bf16(rng.standard_normal((B, H, Ncap, d))), oc.round_bf16(rng.standard_normal((B, H, Ncap, d)) * 4 + 1)
    cache = torch.from_numpy(oc.pack(Kv, Vv)).to(DEV)
    want = [oc.values(*oc.quantise(x)) for x in (Kv, Vv)]
    lens = [96, 0, 33, 500]
    for begin in (0, 3, 95, 96, 200, [0, 4, 32, 90]):
        first = begin if isinstance(begin, list) else [begin] * B
        for which in ((True, True), (True, False), (False, True)):
            out = [torch.full((B, H, N_out, d), 9.0, dtype=torch.bfloat16, device=DEV) if on else None for on in which]
            vb.vitcop_cache_read(cache, _i32(lens), out[0], out[1], row_begin=_i32(begin) if isinstance(begin, list) else begin)
            for o, w in zip(out, want):
                if o is None:
                    continue
                for b in range(B):
                    n = max(0, min(N_out, min(lens[b], Ncap) - first[b]))
                    exact = w[b, :, first[b]:first[b] + n]
                    assert np.all(np.abs(_f64(o)[b, :, :n] - exact) <= (HALF + 2.0 ** -23) * np.abs(exact))
                    assert np.all(_f64(o)[b, :, n:] == 9.0)
    K = torch.zeros(B, H, Ncap, d, dtype=torch.bfloat16, device=DEV)
    vb.vitcop_cache_read(cache, None, K)                   # no lengths: all of it
    assert np.all(np.abs(_f64(K) - want[0]) <= (HALF + 2.0 ** -23) * np.abs(want[0]))


# ---------------------------------------------------------------------------------------------- attention
def _bounds(q, K, V, lens, scale, causal):
    """(out, lse, what out may be off by, what lse may be off by); K, V: (s, m, code) of the rows."""
    B, Hq, Tq, d = q.shape
    H, N = K[0].shape[1], K[0].shape[2]
    Kv, Vv = oc.values(*K), oc.values(*V)
    out, lse = oc.attention(q, Kv, Vv, lens, scale, causal)
    tol, ltol = np.zeros(out.shape), np.zeros(lse.shape)
    absq = np.abs(q).reshape(B, Hq, Tq, d // 32, 32).sum(-1)
    rounded = (HALF * (1 + HALF) * (2 * np.abs(V[2] - 8) * V[0][..., None] + 2 * np.abs(V[1])[..., None])).reshape(B, H, N, d)
    for b in range(B):
        n = int(min(max(lens[b], 0), N))
        for h in range(Hq):
            g = h // (Hq // H)
            for t in range(Tq):
                seen = max(0, n - Tq + t + 1) if causal else n
                if seen == 0:
                    continue
                delta = (scale * 2.0 ** -20 * (absq[b, h, t] * (280 * K[0][b, g, :seen] + np.abs(K[1][b, g, :seen]))).sum(-1)).max()
                w = np.exp(scale * (Kv[b, g, :seen] @ q[b, h, t]) - lse[b, h, t])
                off = np.expm1(2 * delta) + 2.0 ** -20 * 8     # (sums of the weights in fp32)
                tol[b, h, t] = HALF * np.abs(out[b, h, t]) + (w @ rounded[b, g, :seen] + off * (w @ np.abs(Vv[b, g, :seen]))) * (1 + HALF)
                ltol[b, h, t] = delta + 2.0 ** -20 * (1 + abs(lse[b, h, t]))
    return out, lse, tol + 1e-30, ltol


def _problem(seed, B, H, R, Tq, d, Ncap, lens, spread=1.0, offset=0.3):
    rng = np.random.default_rng(seed)
    K = oc.round_bf16(rng.standard_normal((B, H, Ncap, d)) + offset * rng.standard_normal((1, H, 1, d)))
    V = oc.round_bf16(rng.standard_normal((B, H, Ncap, d)) * 2)
    cache = oc.pack(K, V)
    for b in range(B):                                     # behind the last row: whatever the memory held
        n = min(max(lens[b], 0), Ncap)
        rows = np.arange(Ncap).reshape(-1, 32)
        held = cache[b].reshape(H, Ncap // 32, -1)
        for blk in range(Ncap // 32):
            if rows[blk, 0] >= n:
                held[:, blk] = 0xFF
    return _bf16(rng, B, Tq, H * R, d, spread=spread).transpose(1, 2), torch.from_numpy(cache).to(DEV), oc.quantise(K), oc.quantise(V)


def _poison(cache, lens):
    """Rows behind a sample's last, inside its last block too: every byte 0xFF (NaN scales and centres)."""
    B, H, blocks, width = cache.shape
    d = width // 40
    G = d // 32
    for b in range(B):
        for r in range(min(max(lens[b], 0), blocks * 32), blocks * 32):
            blk, t = r // 32, r % 32
            for half in (0, 20 * d):
                cache[b, :, blk, half + t * d // 2:half + (t + 1) * d // 2] = 0xFF
                cache[b, :, blk, half + 16 * d + 2 * t * G:half + 16 * d + 2 * (t + 1) * G] = 0xFF
            cache[b, :, blk, 18 * d + 2 * t * G:18 * d + 2 * (t + 1) * G] = 0xFF
            for g in range(G):
                cache[b, :, blk, 38 * d + 2 * (32 * g + t):38 * d + 2 * (32 * g + t) + 2] = 0xFF


def _attend(q, cache, lens, scale, causal=True, lse=True, strided=True, ws=None):
    B, Hq, Tq, d = q.shape
    _, H, blocks, _ = cache.shape
    out = torch.full((B, Tq, Hq, d) if strided else (B, Hq, Tq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    out = out.transpose(1, 2) if strided else out
    L = torch.full((B, Hq, Tq), 7.0, device=DEV) if lse else None
    if ws is None:
        ws = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=B, H=H, N=blocks * 32, d=d, Nv=Tq, D=Hq)
        ws.fill_(0xFF)
    vb.vitcop_cache_attention(q, cache, lens if lens is None else _i32(lens), out, ws, scale, causal=causal, lse=L)
    assert vb.vitcop_poll_status(ws) == vb.OK
    return out, L


def _check(q, cache, K, V, lens, scale, causal, out, lse):
    w, wl, tol, ltol = _bounds(_f64(q), K, V, lens, scale, causal)
    got = _f64(out)
    worst = (np.abs(got - w) / tol).max()
    assert worst <= 1, worst
    if lse is not None:
        g = _f64(lse)
        empty = np.isneginf(wl)
        assert np.array_equal(np.isneginf(g), empty) and np.all(got[empty] == 0)
        assert np.all(np.abs(g[~empty] - wl[~empty]) <= ltol[~empty]), (np.abs(g[~empty] - wl[~empty]) / ltol[~empty]).max()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("R,Tq,causal", [(1, 1, True), (7, 1, True), (8, 1, False), (4, 5, True), (3, 17, True), (1, 40, False), (16, 4, True)])
def test_attention_matches_fp64(d, R, Tq, causal):
    B, H, Ncap = 6, 2, 160
    lens = [0, 1, 31, 33, 160, 77]
    q, cache, K, V = _problem(d + R + Tq, B, H, R, Tq, d, Ncap, lens)
    _poison(cache, lens)
    out, lse = _attend(q, cache, lens, d ** -0.5, causal)
    _check(q, cache, K, V, lens, d ** -0.5, causal, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,lens", [(1, 1, 1, 1, 128, [5000]), (2, 2, 7, 1, 128, [4097, 31]), (3, 1, 4, 6, 64, [3000, 1, 1500]),
                                             (1, 32, 1, 1, 128, [257]), (2, 1, 8, 33, 128, [900, 40]), (40, 3, 1, 1, 64, list(range(40))),
                                             (1, 2, 5, 1, 256, [2500]), (2, 2, 2, 130, 128, [515, 100])])
def test_attention_over_long_and_ragged_caches(B, H, R, Tq, d, lens):
    Ncap = (max(lens) + 63) // 32 * 32
    q, cache, K, V = _problem(sum(lens), B, H, R, Tq, d, Ncap, lens, spread=2.0)
    _poison(cache, lens)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    _check(q, cache, K, V, lens, d ** -0.5, True, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,lens,causal", [
    (3, 1, 8, 33, 128, 2688, [2688, 31, 0], True),          # pieces of two lengths, a sample that sees nothing, one with more queries than rows
    (2, 1, 4, 33, 64, 8192, [8100, 65], True), (2, 2, 1, 40, 128, 12800, [129, 12799], False), (1, 1, 7, 19, 128, 16512, [16500], True),
    (66, 4, 2, 64, 64, 64, [(7 * b) % 65 for b in range(66)], True),   # more heads than SMs: a CTA has all of one
    (52, 3, 2, 70, 128, 96, [(11 * b) % 97 for b in range(52)], False)])
def test_many_query_rows(B, H, R, Tq, d, Ncap, lens, causal):
    q, cache, K, V = _problem(Tq + d, B, H, R, Tq, d, Ncap, lens, spread=1.5)
    if B < 10:
        _poison(cache, lens)
    out, lse = _attend(q, cache, lens, d ** -0.5, causal)
    _check(q, cache, K, V, lens, d ** -0.5, causal, out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_many_query_rows_and_rows_that_are_no_numbers(d):
    """Values that are no numbers reach the queries that see them, in their group, and no others; keys all of those queries' output."""
    rng = np.random.default_rng(d)
    n, Tq, R, Ncap = 300, 48, 4, 11008
    K, V = _bf16(rng, 1, 1, n, d), _bf16(rng, 1, 1, n, d)
    V[0, 0, 290, 3], V[0, 0, 280, 40] = float("inf"), float("nan")
    cache, lens = _cache(1, 1, Ncap, d), _i32([0])
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, 1, R, Tq, d)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    first = n - Tq                                         # position of the first query
    for t in range(Tq):
        bad = [first + t >= 290, first + t >= 280]
        for g in range(d // 32):
            part = out[:, :, t, 32 * g:32 * g + 32]
            assert torch.isnan(part).all() if g < 2 and bad[g] else torch.isfinite(part).all()
    assert torch.isfinite(lse).all()
    K[0, 0, 270, 5] = float("nan")
    vb.vitcop_cache_write(K, _bf16(rng, 1, 1, n, d), cache, lens, cache_len=None)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    seen = 270 - first
    assert torch.isfinite(out[:, :, :seen]).all() and torch.isnan(out[:, :, seen:]).all()
    assert torch.isfinite(lse[:, :, :seen]).all() and torch.isnan(lse[:, :, seen:]).all()


@pytest.mark.parametrize("up", [True, False])
def test_many_query_rows_over_values_that_grow(up):
    """Values of V a million times larger, or smaller, at the end than at the beginning."""
    n, d, R, Tq, Ncap = 700, 128, 8, 24, 10944
    rng = np.random.default_rng(21)
    size = np.exp2(np.linspace(-10, 10, n) * (1 if up else -1))[None, None, :, None]
    K, V = _bf16(rng, 1, 1, n, d), torch.from_numpy((rng.standard_normal((1, 1, n, d)) * size).astype(np.float32)).bfloat16().to(DEV)
    cache, lens = _cache(1, 1, Ncap, d), _i32([0])
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, 1, R, Tq, d)
    for length in (n, 65):
        out, lse = _attend(q, cache, [length], d ** -0.5)
        _check(q, cache, oc.quantise(_f64(K)), oc.quantise(_f64(V)), [length], d ** -0.5, True, out, lse)


@pytest.mark.parametrize("roles", [1, 2, 4])
def test_many_query_rows_report_a_wait_that_ran_out(roles):
    """One role of every CTA gives up at once, with products and copies of the others in flight; the next call is right again."""
    B, H, R, Tq, d, Ncap = 1, 2, 8, 16, 128, 8192
    q, cache, K, V = _problem(99, B, H, R, Tq, d, Ncap, [Ncap])
    ws = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=B, H=H, N=Ncap, d=d, Nv=Tq, D=H * R)
    out = torch.zeros(B, H * R, Tq, d, dtype=torch.bfloat16, device=DEV)
    try:
        vb.vitcop_set_wait_limit(0, roles)
        vb.vitcop_cache_attention(q, cache, _i32([Ncap]), out, ws, d ** -0.5)
        assert vb.vitcop_poll_status(ws) == vb.ERR_TIMEOUT
    finally:
        vb.vitcop_set_wait_limit(0, 0)
    out, lse = _attend(q, cache, [Ncap], d ** -0.5, ws=ws)
    again, lse2 = _attend(q, cache, [Ncap], d ** -0.5)
    assert torch.equal(out, again) and torch.equal(lse, lse2) and torch.isfinite(out).all()


def test_attention_without_lengths_lse_or_strides_and_beyond_the_capacity():
    q, cache, K, V = _problem(3, 2, 2, 4, 2, 64, 96, [96, 96])
    for lens, strided in ((None, False), ([96, 4000], True), ([96, 96], False)):
        out, _ = _attend(q, cache, lens, 0.125, lse=False, strided=strided)
        _check(q, cache, K, V, [96, 96], 0.125, True, out, None)
    out, lse = _attend(q.contiguous(), cache, [-4, 96], 0.125)
    _check(q, cache, K, V, [-4, 96], 0.125, True, out, lse)


def test_sharp_and_flat_logits():
    """Logits of hundreds, where one row takes all, and of nothing; both signs of the scale, and zero."""
    q, cache, K, V = _problem(5, 1, 2, 4, 3, 128, 320, [300], spread=40.0)
    for scale in (0.5, -0.5, 0.0, 1e-6):
        out, lse = _attend(q, cache, [300], scale)
        w, wl, tol, ltol = _bounds(_f64(q), K, V, [300], abs(scale), True)
        w, wl = oc.attention(_f64(q), oc.values(*K), oc.values(*V), [300], scale, True)
        if scale < 0:                                      # (the bound's weights for this sign)
            _, _, tol, ltol = _bounds(-_f64(q), K, V, [300], -scale, True)
        assert np.all(np.abs(_f64(out) - w) <= tol) and np.all(np.abs(_f64(lse) - wl) <= ltol)


def test_large_offsets_in_values():
    """Centres far from zero: what the codes add is small beside them."""
    rng = np.random.default_rng(9)
    K, V = oc.round_bf16(rng.standard_normal((1, 1, 128, 64)) + 20.0), oc.round_bf16(rng.standard_normal((1, 1, 128, 64)) * 0.5 - 50.0)
    cache = torch.from_numpy(oc.pack(K, V)).to(DEV)
    q = _bf16(rng, 1, 3, 1, 64)
    out, lse = _attend(q, cache, [100], 0.125)
    _check(q, cache, oc.quantise(K), oc.quantise(V), [100], 0.125, True, out, lse)


def test_a_row_that_is_no_number_is_seen_only_by_those_that_see_it():
    rng = np.random.default_rng(10)
    K, V = _bf16(rng, 1, 1, 50, 64), _bf16(rng, 1, 1, 50, 64)
    V[0, 0, 48, 3] = float("inf")                          # seen by the last two of four queries, in one group
    cache, n = _cache(1, 1, 64, 64), _i32([0])
    vb.vitcop_cache_write(K, V, cache, n)
    q = _bf16(rng, 1, 2, 4, 64)
    out, lse = _attend(q, cache, [50], 0.125)
    assert torch.isfinite(out[:, :, :2]).all() and torch.isfinite(out[:, :, :, 32:]).all() and torch.isfinite(lse).all()
    assert torch.isnan(out[:, :, 2:, :32]).all()
    K[0, 0, 47, 40] = float("nan")                         # a key: seen by the last three, in all of their output
    vb.vitcop_cache_write(K, _bf16(rng, 1, 1, 50, 64), cache, n)
    out, lse = _attend(q, cache, [50], 0.125)
    assert torch.isfinite(out[:, :, :1]).all() and torch.isnan(out[:, :, 1:]).all() and torch.isnan(lse[:, :, 1:]).all()


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GB: the last rows written, read and attended over."""
    B, H, Ncap, d = 2, 32, 425984, 128
    cache = torch.empty((B, H, Ncap // 32, 40 * d), dtype=torch.uint8, device=DEV)
    assert cache.numel() > 2 ** 32
    rng = np.random.default_rng(11)
    K, V = _bf16(rng, B, H, 45, d), _bf16(rng, B, H, 45, d)
    n, start = _i32([0] * B), _i32([Ncap - 45, 0])
    vb.vitcop_cache_write(K, V, cache, n, cache_len=start)
    K_out, V_out = torch.zeros_like(K), torch.zeros_like(V)
    vb.vitcop_cache_read(cache, n, K_out, V_out, row_begin=start)
    want = [oc.round_bf16(oc.values(*oc.quantise(_f64(x)))) for x in (K, V)]
    assert np.array_equal(_f64(K_out), want[0]) and np.array_equal(_f64(V_out), want[1])
    q = _bf16(rng, B, H, 1, d)
    out, lse = _attend(q, cache, [0, 45], d ** -0.5)       # (sample 1 starts beyond 2^31 bytes, its last head beyond 2^32)
    Kq, Vq = oc.quantise(_f64(K)), oc.quantise(_f64(V))
    _check(q, cache, Kq, Vq, [0, 45], d ** -0.5, True, out, lse)


def test_the_order_of_calls_and_the_workspace_do_not_change_results():
    """Twice the same bits, on another stream too, with a workspace that another problem left behind."""
    q, cache, _, _ = _problem(12, 2, 2, 7, 3, 128, 1280, [1280, 700], spread=2.0)
    ws = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=2, H=2, N=1280, d=128, Nv=3, D=14)
    first, l1 = _attend(q, cache, [1280, 700], 0.09, ws=ws)
    _attend(q, cache, [64, 1111], 0.5, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, l2 = _attend(q, cache, [1280, 700], 0.09, ws=ws)
    side.synchronize()
    assert torch.equal(first, again) and torch.equal(l1, l2)


@pytest.mark.parametrize("H,R", [(4, 1), (2, 7)])
def test_a_pruned_sequence_goes_on_token_by_token(H, R):
    """K-norm, selection and the kept rows to the cache; then tokens, each appended and attended from; then the same as graphs."""
    rng = np.random.default_rng(13)
    B, d, n, T, budget, steps = 3, 128, 120, 10, 37, 5
    N, vis_start = n + T, 4
    K, V = _bf16(rng, B, H, N, d), _bf16(rng, B, H, N, d)
    score = torch.zeros(B, n, device=DEV)
    keep, n_keep = torch.zeros(B, budget, dtype=torch.int32, device=DEV), _i32([0] * B)
    vb.vitcop_knorm_score(K, vis_start, n, score)
    vb.vitcop_select(score, n, budget, keep, n_keep, vb.alloc_workspace(vb.OP_SELECT, B=B, Nv=n))
    Ncap = 64
    cache, lens = _cache(B, H, Ncap, d), [_i32([0] * B), _i32([0] * B)]
    vb.vitcop_cache_write(K, V, cache, lens[0], vis_start=vis_start, vis_len=n, keep_idx=keep, n_keep=n_keep)
    assert lens[0].tolist() == [T + budget] * B
    order = [[*range(vis_start), *(vis_start + i for i in k), *range(vis_start + n, N)] for k in keep.tolist()]
    rows_K = [_f64(K)[b][:, order[b]] for b in range(B)]
    rows_V = [_f64(V)[b][:, order[b]] for b in range(B)]
    pruned, first_len = cache.clone(), lens[0].clone()
    tokens = [(_bf16(rng, B, H, 1, d), _bf16(rng, B, H, 1, d), _bf16(rng, B, H * R, 1, d, spread=2.0)) for _ in range(steps)]
    ws = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=B, H=H, N=Ncap, d=d, Nv=1, D=H * R)
    k, v, q = (torch.zeros_like(x) for x in tokens[0])
    out, lse = torch.zeros_like(q), torch.zeros(B, H * R, 1, device=DEV)

    def step(old, new):
        vb.vitcop_cache_write(k, v, cache, new, cache_len=old)
        vb.vitcop_cache_attention(q, cache, new, out, ws, d ** -0.5, lse=lse)

    outs = []
    for i, token in enumerate(tokens):
        for x, y in zip((k, v, q), token):
            x.copy_(y)
        step(lens[i % 2], lens[1 - i % 2])
        outs.append((out.clone(), lse.clone()))
        rows_K = [np.concatenate([r, _f64(token[0])[b]], 1) for b, r in enumerate(rows_K)]
        rows_V = [np.concatenate([r, _f64(token[1])[b]], 1) for b, r in enumerate(rows_V)]
        length = T + budget + i + 1
        assert lens[1 - i % 2].tolist() == [length] * B
        _check(q, cache, oc.quantise(np.stack(rows_K)), oc.quantise(np.stack(rows_V)), [length] * B, d ** -0.5, True, *outs[-1])
    cache.copy_(pruned)
    lens[0].copy_(first_len)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(lens[i], lens[1 - i])
        graphs.append(g)
    for i, token in enumerate(tokens):
        for x, y in zip((k, v, q), token):
            x.copy_(y)
        graphs[i % 2].replay()
        assert torch.equal(out, outs[i][0]) and torch.equal(lse, outs[i][1])


def test_a_budget_of_the_longest_sequence_in_one_step():
    """A real pruning step's list and counts (the one-call Stage III), its K and V compacted both ways."""
    w = W.workload("tiny")
    K_b, V_b = W.make_kv(w, 0, w.Nv)
    K, V, hid = vb.bf16_tensor(K_b), vb.bf16_tensor(V_b), vb.bf16_tensor(np.ascontiguousarray(W.make_hidden(w)))
    B, H, N, d = K.shape
    if d not in (64, 128, 256):
        K, V = (x.repeat(1, 1, 1, 64 // d + 1)[..., :64].contiguous() for x in (K, V))
        d = 64
    budget = w.budgets[0]
    Ncap = (w.T + budget + 31) // 32 * 32
    K_out, V_out = (torch.zeros(B, H, Ncap, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hid_out, out_len = torch.zeros(B, Ncap, hid.shape[2], dtype=torch.bfloat16, device=DEV), _i32([0] * B)
    keep, n_keep = torch.zeros(B, w.Nv, dtype=torch.int32, device=DEV), _i32([0] * B)
    vb.vitcop_prune_step(hid, K, V, w.vis_start, w.Nv, w.Nv, budget, hid_out, K_out, V_out, out_len,
                         vb.alloc_workspace(vb.OP_PRUNE_STEP, B=B, Nv=w.Nv), keep_idx_out=keep, n_keep_out=n_keep)
    cache, new_len = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, new_len, vis_start=w.vis_start, vis_len=w.Nv, keep_idx=keep, n_keep=n_keep)
    assert new_len.tolist() == out_len.tolist()
    for b, n in enumerate(new_len.tolist()):
        _same_rows(cache, b, list(range(n)), _f64(K_out)[b, :, :n], _f64(V_out)[b, :, :n])


def test_what_the_binding_refuses():
    x, n = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16, device=DEV), _i32([0, 0])
    cache = _cache(2, 2, 32, 64)
    ws = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=2, H=2, N=32, d=64, Nv=4, D=2)
    y = torch.zeros_like(x)
    for call in (lambda: vb.vitcop_cache_write(x.float(), x, cache, n), lambda: vb.vitcop_cache_write(x[:1], x, cache, n),
                 lambda: vb.vitcop_cache_write(x, x[..., ::2], cache, n), lambda: vb.vitcop_cache_write(x, x, cache, n.long()),
                 lambda: vb.vitcop_cache_write(x, x, cache[:, :, :, 1:], n), lambda: vb.vitcop_cache_write(x, x, cache, n[:1]),
                 lambda: vb.vitcop_cache_write(x, x, cache, n, vis_len=4, keep_idx=n, n_keep=n.clone()),
                 lambda: vb.vitcop_cache_write(None, None, cache, n), lambda: vb.vitcop_cache_read(cache, n, x.transpose(0, 1)),
                 lambda: vb.vitcop_cache_read(cache, n), lambda: vb.vitcop_cache_read(cache.int(), n, x),
                 lambda: vb.vitcop_cache_attention(x, cache, n, y.half(), ws, 1.0), lambda: vb.vitcop_cache_attention(x, cache, n, y[:, :1], ws, 1.0),
                 lambda: vb.vitcop_cache_attention(x, cache, n, y, ws, 1.0, lse=torch.zeros(2, 2, device=DEV)),
                 lambda: vb.vitcop_cache_attention(x, cache, n, y, ws.int(), 1.0)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: vb.vitcop_cache_write(x, x, cache, n, cache_len=n), lambda: vb.vitcop_cache_attention(x, cache, n, x, ws, 1.0)):
        with pytest.raises(vb.VitcopError):
            call()


def test_no_rows_no_samples_no_capacity():
    x = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16, device=DEV)
    empty, n, to = vb.alloc_cache(2, 2, 0, 64), _i32([5, 0]), _i32([9, 9])
    vb.vitcop_cache_write(x[:, :2], x[:, :2], empty, to, cache_len=n)      # (nothing fits)
    assert to.tolist() == [8, 3]
    vb.vitcop_cache_read(empty, n, torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device=DEV))
    out, lse = _attend(x, empty, [5, 0], 1.0)
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))
    cache, _ = _cache(2, 2, 64, 64), _attend(x[:, :, :0], empty, [5, 0], 1.0)
    assert _attend(x[:, :, :0], cache, [5, 0], 1.0)[0].shape == (2, 4, 0, 64)
    none, no_len = vb.alloc_cache(0, 2, 64, 64), _i32([])
    vb.vitcop_cache_write(x[:0, :2], x[:0, :2], none, no_len)
    vb.vitcop_cache_read(none, no_len, x[:0, :2])
    _attend(x[:0], none, [], 1.0)
    with pytest.raises(ValueError):
        vb.vitcop_cache_attention(x, cache, n, torch.zeros_like(x), vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=2, H=2, N=64, d=64, Nv=3, D=4),
                                  1.0, causal=n)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,n", [(1, 2, 4, 1, 64, 64, 50), (1, 2, 7, 2, 128, 2048, 1999), (70, 2, 1, 1, 256, 128, 128),
                                               (1, 1, 4, 48, 128, 11008, 1500), (40, 4, 2, 20, 64, 352, 300)])
def test_values_near_the_end_of_the_range(B, H, R, Tq, d, Ncap, n):
    """Values of which a handful add up to more than fp32 holds; their mean is one of them."""
    rng = np.random.default_rng(n)
    K, V = _bf16(rng, B, H, n, d), torch.from_numpy((2e38 + 3e36 * rng.standard_normal((B, H, n, d))).astype(np.float32)).bfloat16().to(DEV)
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, [n] * B, d ** -0.5)
    _check(q, cache, oc.quantise(_f64(K)), oc.quantise(_f64(V)), [n] * B, d ** -0.5, True, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,n", [(1, 1, 4, 48, 128, 11008, 1500), (1, 2, 7, 48, 64, 2048, 300), (40, 4, 2, 20, 128, 352, 300), (40, 4, 2, 20, 64, 352, 300)])
def test_many_query_rows_and_values_of_other_sizes(B, H, R, Tq, d, Ncap, n):
    """Values at the end of the range that some of the queries do not see, and groups far apart in size, are everybody's own."""
    rng = np.random.default_rng(n + d)
    K, V = _bf16(rng, B, H, n, d), _bf16(rng, B, H, n, d)
    V[0, 0, n - 5, :32] = 3.38e38
    V[0, 0, n - 15] *= 2.0 ** 100
    V[B - 1, H - 1, :, 32:64] *= 2.0 ** -40
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, [n] * B, d ** -0.5)
    _check(q, cache, oc.quantise(_f64(K)), oc.quantise(_f64(V)), [n] * B, d ** -0.5, True, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap", [(3, 8, 7, 1, 128, 2048), (2, 4, 4, 40, 128, 4096), (1, 2, 4, 1, 64, 512), (80, 2, 2, 20, 64, 320)])
def test_two_streams_at_once_and_replays_with_other_lengths(B, H, R, Tq, d, Ncap):
    """Calls on two streams, each with its workspace, at the same time; a captured call takes the lengths that it finds when it runs."""
    lens = [Ncap - 37 * b % 300 for b in range(B)]
    q, cache, _, _ = _problem(B + d, B, H, R, Tq, d, Ncap, lens)
    shared = q[:, :1, :1].expand(B, H * R, Tq, d)          # (one row for all of a sample's queries)
    n = _i32(lens)
    ws = [vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=B, H=H, N=Ncap, d=d, Nv=Tq, D=H * R) for _ in range(3)]
    outs = [torch.empty_like(q, memory_format=torch.contiguous_format) for _ in range(3)]
    want = [_attend(x, cache, ln, 0.1, strided=False)[0] for x, ln in ((q, lens), (shared, lens), (q, [x // 2 for x in lens]))]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, x, o, w in zip(streams, (q, shared), outs, ws):
            with torch.cuda.stream(s):
                vb.vitcop_cache_attention(x, cache, n, o, w, 0.1)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    assert all(vb.vitcop_poll_status(w) == vb.OK for w in ws[:2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vitcop_cache_attention(q, cache, n, outs[2], ws[2], 0.1)
    for ln, w in ((lens, want[0]), ([x // 2 for x in lens], want[2]), ([0] * B, torch.zeros_like(want[0]))):
        n.copy_(_i32(ln))
        outs[2].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[2], w) and vb.vitcop_poll_status(ws[2]) == vb.OK


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,lens,causal", [(4, 4, 1, 60, 64, 6304, [6300, 0, 31, 4097], True), (2, 6, 2, 32, 128, 8192, [8192, 100], False)])
def test_half_a_tile_of_query_rows(B, H, R, Tq, d, Ncap, lens, causal):
    q, cache, K, V = _problem(Tq + d, B, H, R, Tq, d, Ncap, lens, spread=1.5)
    _poison(cache, lens)
    out, lse = _attend(q, cache, lens, d ** -0.5, causal)
    _check(q, cache, K, V, lens, d ** -0.5, causal, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap", [
    (2, 64, 1, 1, 128, 1536), (5, 32, 1, 1, 64, 1024), (9, 32, 1, 1, 128, 896), (16, 32, 1, 1, 64, 800), (11, 64, 1, 1, 128, 896), (1, 8, 1, 1, 128, 1024),
    (3, 32, 4, 4, 128, 1280), (8, 32, 4, 4, 64, 1024), (12, 32, 4, 5, 64, 864), (2, 4, 8, 5, 128, 1056), (3, 64, 4, 2, 256, 832), (2, 4, 8, 4, 64, 4096)])
def test_however_heads_are_given_to_ctas(B, H, R, Tq, d, Ncap):
    """A CTA a head (of four warps or of eight, all at once or not), or blocks shared out: lengths from none to all."""
    rng = np.random.default_rng(B * H + Tq)
    K, V = _bf16(rng, 1, H, Ncap, d).expand(B, H, Ncap, d), _bf16(rng, 1, H, Ncap, d).expand(B, H, Ncap, d)
    cache, n = _cache(B, H, Ncap, d), _i32([0] * B)
    lens = [0, Ncap, 33, Ncap - 1, 1, 257, Ncap // 2, 5, 700, 130, 64, 31, 500, 96, Ncap, 3][:B]
    vb.vitcop_cache_write(K, V, cache, n, seq_len=_i32(lens))
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    heads = sorted({0, 1, H // 2, H - 1})                  # (the oracle looks at some of them)
    rows = [h * R + i for h in heads for i in range(R)]
    held = [tuple(np.repeat(x, B, 0) for x in oc.quantise(_f64(t[:1, heads]))) for t in (K, V)]
    _check(q[:, rows], cache, *held, lens, d ** -0.5, True, out[:, rows], lse[:, rows])
    for h in range(H):                                     # and the others against it: the cache is the same for all calls
        if h % 7 == 3:
            one, _ = _attend(q[:, h * R:(h + 1) * R], cache[:, h:h + 1].contiguous(), lens, d ** -0.5)
            # (each is off by at most HALF (|out| + 2 |code - 8| s + 2 |m|), and values reach 5)
            assert (one.float() - out[:, h * R:(h + 1) * R].float()).abs().max() <= 2 * HALF * 3 * 5


@pytest.mark.parametrize("d", [64, 128])
def test_many_query_rows_of_one_tile(d):
    """CTAs that have one tile of tokens, whose maximum always moves; logits far enough from 0 that another's would show."""
    B, H, R, Tq, Ncap = 66, 4, 2, 64, 256
    lens = [[64, 33, 1, 40, 63][b % 5] for b in range(B)]
    q, cache, K, V = _problem(d + 7, B, H, R, Tq, d, Ncap, lens, spread=3.0)
    out, lse = _attend(q, cache, lens, d ** -0.5, False)
    _check(q, cache, K, V, lens, d ** -0.5, False, out, lse)
    for _ in range(30):
        again, lse2 = _attend(q, cache, lens, d ** -0.5, False)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,Ncap", [(66, 4, 256), (2, 4, 4096)])
def test_many_query_rows_and_samples_without_a_tile(d, B, H, Ncap):
    """CTAs that see no token (all of a head, or a piece of one) write zeros."""
    R, Tq = 2, 64
    lens = [[0, 64, 0, 5][b % 4] for b in range(B)]
    q, cache, K, V = _problem(d + 8, B, H, R, Tq, d, Ncap, lens)
    for _ in range(30):
        out, lse = _attend(q, cache, lens, d ** -0.5, False)
        for b in range(0, B, 2):
            assert torch.all(out[b] == 0) and torch.all(torch.isneginf(lse[b]))
    _check(q, cache, K, V, lens, d ** -0.5, False, out, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_elements_far_below_the_centre_fall_to_their_side_of_a_border(d):
    """Where the centre is a whole number of steps and a half away from 0, an element's sign decides, however small it is; 0 itself is a tie."""
    rng = np.random.default_rng(d)
    N = 64
    x = rng.choice([1.0, -1.0, 0.0], (1, 2, N, d)) * np.exp2(-rng.integers(17, 118, (1, 2, N, d)).astype(np.float64))
    group = x.reshape(-1, 32)
    ends = rng.integers(0, 4, len(group))
    lo, hi = np.array([-0.9375, -0.8125, -1.0, -15.0])[ends], np.array([0.9375, 1.0625, 0.875, 15.0])[ends]
    group[np.arange(len(group)), rng.integers(0, 16, len(group))] = lo
    group[np.arange(len(group)), rng.integers(16, 32, len(group))] = hi
    s, m, _ = oc.quantise(x)
    assert (2 * m / s % 2 == 1).mean() > 0.6               # (three of the four pairs of ends; the other has its centre at 0)
    x = torch.from_numpy(x.astype(np.float32)).bfloat16().to(DEV)
    cache, n = _cache(1, 2, N, d), _i32([0])
    vb.vitcop_cache_write(x, x, cache, n)
    _same_rows(cache, 0, list(range(N)), _f64(x)[0], _f64(x)[0])


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,n", [(1, 1, 4, 48, 128, 11008, 1500), (1, 2, 7, 48, 64, 4096, 300), (40, 4, 4, 20, 128, 352, 300)])
def test_a_token_of_next_to_no_value_costs_other_rows_nothing(B, H, R, Tq, d, Ncap, n):
    """Padding or a sink whose values are 2^-45 of the others': rows that look elsewhere are not done anew in fp32 (they are the bits that they
    are with zeros there), those that look at nothing else are right."""
    rng = np.random.default_rng(n + d)
    K, V = _bf16(rng, B, H, n, d), _bf16(rng, B, H, n, d)
    q = _bf16(rng, B, H * R, Tq, d)
    K[:, :, 2] = 4.0                                       # the token that the odd queries look at
    q[:, :, 1::2] = (0.3 * q[:, :, 1::2].float() + 3.0).bfloat16()
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    V[:, :, 2] = 0.0
    vb.vitcop_cache_write(K, V, cache, lens)
    zeros, _ = _attend(q, cache, [n] * B, d ** -0.5)
    V[:, :, 2] = _bf16(rng, B, H, d, spread=2.0 ** -45)
    vb.vitcop_cache_write(K, V, cache, lens)
    out, lse = _attend(q, cache, [n] * B, d ** -0.5)
    _check(q, cache, oc.quantise(_f64(K)), oc.quantise(_f64(V)), [n] * B, d ** -0.5, True, out, lse)
    assert torch.equal(out[:, :, ::2], zeros[:, :, ::2])


def test_many_small_weights_on_large_values():
    """A thousand tokens of 2^-33 of a row's weight each, with values 2^20 times those of the token that it looks at: a tenth of its output."""
    B, H, n, d, R, Tq, Ncap = 37, 4, 1000, 128, 4, 48, 1024       # (more tiles of rows than SMs: a CTA has all tokens)
    K = torch.zeros(B, H, n, d, dtype=torch.bfloat16, device=DEV)
    V = torch.full((B, H, n, d), 2.0 ** 20, dtype=torch.bfloat16, device=DEV)
    K[:, :, 7], V[:, :, 7] = 1.015625, 1.0
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = torch.full((B, H * R, Tq, d), 2.0, dtype=torch.bfloat16, device=DEV)
    out, lse = _attend(q, cache, [n] * B, d ** -0.5, causal=False)
    z = 2 * 1.015625 * d ** 0.5
    w = (n - 1) * np.exp(-z)
    want = (1 + w * 2.0 ** 20) / (1 + w)
    assert want > 1.1
    # (all of the sums are exact but for the weights: 2^-8 each at most, and the rounding of the output)
    assert (out.double() - want).abs().max() <= want * (2 * HALF + HALF ** 2)
    assert (lse.double() - z - np.log1p(w)).abs().max() <= 2.0 ** -20 * (1 + z)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,lens", [
    (1, 32, 1, 1, 128, 16512, [256]), (4, 32, 1, 1, 128, 16512, [1500, 33, 0, 700]), (3, 2, 4, 5, 256, 8192, [40, 500, 1]),
    (1, 4, 7, 64, 128, 16512, [300]), (2, 2, 4, 40, 64, 16512, [1, 129]), (40, 4, 1, 1, 64, 4096, [3 * b for b in range(40)])])
def test_short_sequences_in_long_caches(B, H, R, Tq, d, Ncap, lens):
    """A cache has room for the longest conversation; what is in it may be a hundredth of that."""
    n = max(lens)
    rng = np.random.default_rng(B + Ncap)
    K, V = _bf16(rng, B, H, n, d), _bf16(rng, B, H, n, d)
    cache, to = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, to, seq_len=_i32(lens))
    q = _bf16(rng, B, H * R, Tq, d, spread=1.5)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    _check(q, cache, oc.quantise(_f64(K)), oc.quantise(_f64(V)), lens, d ** -0.5, True, out, lse)


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap", [(16, 32, 1, 1, 64, 800), (2, 64, 1, 1, 128, 1536), (12, 32, 4, 2, 64, 864), (2, 4, 8, 5, 128, 1056), (1, 8, 4, 3, 64, 4096)])
def test_every_head_however_heads_are_given_to_ctas(B, H, R, Tq, d, Ncap):
    """All heads against fp64, outputs and sums: a piece of a head that is lost or counted twice shows in lse."""
    rng = np.random.default_rng(B * H + Tq + 1)
    K, V = _bf16(rng, 1, H, Ncap, d), _bf16(rng, 1, H, Ncap, d)
    cache, n = _cache(B, H, Ncap, d), _i32([0] * B)
    lens = [Ncap, 0, Ncap - 1, 33, 257, Ncap // 2, 1, 700, 5, 130, 64, 31, 500, 96, Ncap, 3][:B]
    vb.vitcop_cache_write(K.expand(B, H, Ncap, d), V.expand(B, H, Ncap, d), cache, n, seq_len=_i32(lens))
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    k, v = oc.quantise(_f64(K)), oc.quantise(_f64(V))
    for b in range(B):
        _check(q[b:b + 1], cache, k, v, lens[b:b + 1], d ** -0.5, True, out[b:b + 1], lse[b:b + 1])


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,lens", [(1, 2, 8, 48, 128, 5440, [5400]), (2, 1, 7, 24, 64, 8192, [777, 8100]), (40, 4, 4, 20, 128, 352, [(37 * b) % 353 for b in range(40)])])
def test_many_query_rows_hold_eleven_bits(B, H, R, Tq, d, Ncap, lens):
    """Weights and values of V in fp16: each off by 2^-11 at most, and the sum of the weights, which the output is divided by, too."""
    q, cache, K, V = _problem(Tq + d + 1, B, H, R, Tq, d, Ncap, lens)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    qq, Kv, Vv = _f64(q), oc.values(*K), oc.values(*V)
    absq = np.abs(qq).reshape(B, H * R, Tq, d // 32, 32).sum(-1)
    for b in range(0, B, max(1, B // 4)):
        w, _ = oc.attention(qq[b:b + 1], Kv[b:b + 1], Vv[b:b + 1], lens[b:b + 1], d ** -0.5, True)
        size, _ = oc.attention(qq[b:b + 1], Kv[b:b + 1], np.abs(Vv[b:b + 1]), lens[b:b + 1], d ** -0.5, True)
        reach = (280 * K[0][b] + np.abs(K[1][b])).max(1)[:, None, None]                  # [H, 1, 1, G]
        delta = d ** -0.5 * 2.0 ** -20 * (absq[b].reshape(H, R, Tq, -1) * reach).sum(-1).reshape(1, H * R, Tq, 1)
        off = np.expm1(2 * delta) + 2.0 ** -17
        eleven = 2.0 ** -11 * (1 + 2.0 ** -10)
        tol = HALF * np.abs(w) + (1 + HALF) * ((2 * eleven + off) * size + eleven * np.abs(w)) + 1e-30
        worst = (np.abs(_f64(out)[b:b + 1] - w) / tol).max()
        assert worst <= 1, worst


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,R,Tq,Ncap,n", [(1, 2, 4, 3, 128, 100), (1, 2, 1, 1, 4096, 3000), (1, 1, 8, 40, 8192, 300)])
def test_a_query_that_is_no_number_is_its_own(B, H, R, Tq, Ncap, n, d):
    """NaN and infinities in a query: all of its output is NaN, and no other's changes; one that sees nothing stays at zero."""
    rng = np.random.default_rng(n + d)
    K, V = _bf16(rng, B, H, n, d), _bf16(rng, B, H, n, d)
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    bad = torch.zeros(B, H * R, Tq, dtype=torch.bool, device=DEV)
    p = q.clone()
    for i, what in enumerate((float("nan"), float("inf"), float("-inf"))):
        at = (0, (i * R) % (H * R) + min(i, R - 1) if R > 1 else i % (H * R), (i * 7) % Tq)
        p[at][5 + 20 * i], bad[at] = what, True
    out2, lse2 = _attend(p, cache, [n], d ** -0.5)
    assert torch.isnan(out2[bad]).all() and torch.isnan(lse2[bad]).all()
    assert torch.equal(out2[~bad], out[~bad]) and torch.equal(lse2[~bad], lse[~bad])
    out3, lse3 = _attend(p, cache, [0], d ** -0.5)
    assert torch.all(out3 == 0) and torch.all(torch.isneginf(lse3))


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,n", [(1, 2, 4, 3, 128, 128, 100), (1, 2, 1, 1, 256, 4096, 3000), (1, 1, 8, 40, 64, 8192, 300)])
def test_logits_beyond_the_range_are_their_rows_own(B, H, R, Tq, d, Ncap, n):
    """Products that pass what fp32 holds: NaN where a logit is infinite upwards, and nothing in other rows."""
    rng = np.random.default_rng(n + d)
    K, V = _bf16(rng, B, H, n, d, spread=0.1, offset=1.0), _bf16(rng, B, H, n, d)
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    p = q.clone()
    p[:, 0, Tq - 1] = 3e38
    out2, lse2 = _attend(p, cache, [n], d ** -0.5)
    assert torch.isnan(out2[:, 0, Tq - 1]).all()
    rest = torch.ones(B, H * R, Tq, dtype=torch.bool, device=DEV)
    rest[:, 0, Tq - 1] = False
    assert torch.equal(out2[rest], out[rest]) and torch.equal(lse2[rest], lse[rest])


@pytest.mark.parametrize("R,Tq,Ncap,n", [(1, 4, 96, 60), (8, 4, 96, 60), (4, 40, 4096, 700), (1, 2, 8192, 5000)])
def test_wide_heads_and_rows_that_are_no_numbers(R, Tq, Ncap, n):
    """d = 256: a row of V that is no number reaches the queries that see it, in its group; a key all of their output."""
    rng, d = np.random.default_rng(n), 256
    K, V = _bf16(rng, 1, 1, n, d), _bf16(rng, 1, 1, n, d)
    q = _bf16(rng, 1, R, Tq, d)
    cache, lens = _cache(1, 1, Ncap, d), _i32([0])
    V[0, 0, n - 1, 200], V[0, 0, n - 2, 7] = float("inf"), float("nan")
    vb.vitcop_cache_write(K, V, cache, lens)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    assert torch.isfinite(lse).all()
    nan = torch.isnan(out)
    for t in range(Tq):
        for g in range(8):
            sees = (g == 6 and t >= Tq - 1) or (g == 0 and t >= Tq - 2)
            assert nan[:, :, t, 32 * g:32 * g + 32].all() if sees else not nan[:, :, t, 32 * g:32 * g + 32].any()
    K[0, 0, n - 2, 99] = float("-inf")
    vb.vitcop_cache_write(K, _bf16(rng, 1, 1, n, d), cache, lens)
    out, lse = _attend(q, cache, [n], d ** -0.5)
    assert torch.isfinite(out[:, :, :Tq - 2]).all() and torch.isnan(out[:, :, max(0, Tq - 2):]).all() and torch.isnan(lse[:, :, max(0, Tq - 2):]).all()


@pytest.mark.parametrize("B,H,R,Tq,d,Ncap,n", [(1, 2, 4, 3, 128, 128, 100), (1, 1, 8, 40, 64, 8192, 300)])
def test_a_scale_of_zero_is_a_product(B, H, R, Tq, d, Ncap, n):
    """Zero times a query that is no number is no number either."""
    rng = np.random.default_rng(n + d + 1)
    K, V = _bf16(rng, B, H, n, d), _bf16(rng, B, H, n, d)
    cache, lens = _cache(B, H, Ncap, d), _i32([0] * B)
    vb.vitcop_cache_write(K, V, cache, lens)
    q = _bf16(rng, B, H * R, Tq, d)
    q[0, 1, 2, 5], q[0, H * R - 1, 0, 0] = float("nan"), float("inf")
    out, lse = _attend(q, cache, [n], 0.0, causal=False)
    bad = torch.zeros(B, H * R, Tq, dtype=torch.bool, device=DEV)
    bad[0, 1, 2] = bad[0, H * R - 1, 0] = True
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all() and torch.isfinite(out[~bad]).all()
    assert (lse[~bad] - np.log(n)).abs().max() <= 2.0 ** -20 * 8


@pytest.mark.parametrize("R,Tq,d,Ncap", [(1, 1, 128, 3008), (4, 4, 64, 4000), (4, 5, 128, 4800), (1, 1, 256, 3008)])
def test_more_heads_than_sms_and_blocks_shared_out(R, Tq, d, Ncap):
    """160 heads of long caches: blocks of all heads shared out, samples from empty to full."""
    B, H, rng = 5, 32, np.random.default_rng(Ncap + d)
    K, V = _bf16(rng, 1, H, Ncap, d), _bf16(rng, 1, H, Ncap, d)
    cache, n = _cache(B, H, Ncap, d), _i32([0] * B)
    lens = [Ncap, 0, 1000, 33, Ncap - 1]
    vb.vitcop_cache_write(K.expand(B, H, Ncap, d), V.expand(B, H, Ncap, d), cache, n, seq_len=_i32(lens))
    q = _bf16(rng, B, H * R, Tq, d)
    out, lse = _attend(q, cache, lens, d ** -0.5)
    k, v = oc.quantise(_f64(K)), oc.quantise(_f64(V))
    for b in range(B):
        _check(q[b:b + 1], cache, k, v, lens[b:b + 1], d ** -0.5, True, out[b:b + 1], lse[b:b + 1])
