"""The operators of the K/V cache in 4 bits: what is measured, in plain torch and as the framework's calls.

A model that prunes its visual tokens decodes on what is left of its K/V cache.  Held in 4 bits, the cache takes rows as they
are made ("write": a prompt, or one token a step) or as a pruning step leaves them ("prune": the rows of a keep list), gives
them back ("read"), and is what the queries of a decoding step, of a few guessed tokens or of a question attend over
("attend").

The cache, uint8 [B, H, Ncap / 32, 40 d]: a group is 32 elements of a row (one token, one head), lo and hi its smallest and
largest, s = bf16((hi - lo) / 15), m = bf16(lo + 8 s), code = clamp(round((x - m) / s) + 8, 0, 15), and it stands for
m + (code - 8) s.  A block holds 32 tokens r of a head, G = d / 32 groups, K before V:
    K codes   [r][e / 8][G][4 bytes]   element e of a group: nibble e % 8, low first
    K s, m    bf16 [r][G], bf16 [r][G]
    V codes   [r][e / 4][G][2 bytes]   element e of a group: nibble e % 4
    V s, m    bf16 [r][G], bf16 [G][r]

Sizes: LLaVA-1.5-like images (576 tokens, 192 kept), AnyRes images (2880, 640 kept), clips (4608, 1152 kept) and long videos
with grouped heads (16384), with the text around them; heads of 128 and 64.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the next token of one chat about one pruned image: the smallest call, where latency counts
        _attend("attend_image_b1", 1, 32, 1, 1, 128, 256, False),
        # a serving batch of such chats, every one at another length
        _attend("attend_image_b16", 16, 32, 1, 1, 128, 777, True),
        # high-resolution images that were not pruned: the most bytes
        _attend("attend_anyres_b8", 8, 32, 1, 1, 128, 2944, True),
        # two long videos, seven query heads to a stored one: few rows over a long axis
        _attend("attend_long_b2", 2, 4, 7, 1, 128, 16512, False),
        # the question behind a pruned clip, all its tokens at once
        _attend("attend_question_b4", 4, 4, 7, 64, 128, 1280, False),
        # five guessed tokens checked at once, narrow heads
        _attend("attend_guess_b8", 8, 8, 4, 5, 64, 733, True),
        # one token more: the smallest write
        _write("write_token_b1", 1, 32, 1, 128, 255, False),
        # one token more in each of a batch, every sample at another length
        _write("write_token_b16", 16, 32, 1, 128, 777, True),
        # the prompts of two long videos, keys and values as the projection leaves them (heads inside tokens)
        _write("write_long_b2", 2, 4, 16512, 128, 0, False),
        # what a pruning step keeps of high-resolution images, text around it
        dict(name="prune_anyres_b8", kind="prune", B=8, H=32, d=128, n=2880, T=64, keep=640),
        # a pruned image read back
        dict(name="read_image_b1", kind="read", B=1, H=32, d=128, len=256, ragged=False),
        # a batch of high-resolution images read back
        dict(name="read_anyres_b8", kind="read", B=8, H=32, d=128, len=2944, ragged=True),
    ]


def draw(rng):
    while True:
        kind = rng.choice(["attend", "attend", "attend", "attend", "write", "write", "prune", "read"])
        B = int(_log_uniform(rng, 1, 16))
        H, d = rng.choice([4, 8, 16, 32]), rng.choice([64, 128])
        ragged = rng.random() < 0.6
        if kind == "attend":
            R, Tq = rng.choice([1, 1, 4, 7, 8]), rng.choice([1, 1, 1, 2, 5, 17, 64])
            case = _attend("", B, H, R, Tq, d, int(_log_uniform(rng, max(64, 2 * Tq), 16512)), ragged)
        elif kind == "write":
            if rng.random() < 0.5:
                case = _write("", B, H, rng.choice([1, 1, 3]), d, int(_log_uniform(rng, 64, 16512)), ragged)
            else:
                case = _write("", B, H, int(_log_uniform(rng, 17, 16512)), d, rng.choice([0, 0, 35]), False)
        elif kind == "prune":
            n = int(_log_uniform(rng, 64, 16384))
            case = dict(kind="prune", B=B, H=H, d=d, n=n, T=rng.randint(2, 128), keep=max(1, int(n * rng.uniform(0.06, 0.5))))
        else:
            case = dict(kind="read", B=B, H=H, d=d, len=int(_log_uniform(rng, 64, 16512)), ragged=ragged)
        case.pop("name", None)
        # no dearer than the dearest of the list, and memory for several states
        w = work(case)
        rows = case.get("n", 0) + case.get("N", 0) + case.get("len", 0)
        if w["bytes"] <= 3e8 and w["flops"] <= 5e9 and B * H * rows * d <= 1 << 27 and B * H * case.get("R", 1) * case.get("Tq", 1) * rows <= 1 << 26:
            return case


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))


def _attend(name, B, H, R, Tq, d, length, ragged):
    return dict(name=name, kind="attend", B=B, H=H, R=R, Tq=Tq, d=d, len=length, ragged=ragged)


def _write(name, B, H, N, d, before, ragged):
    return dict(name=name, kind="write", B=B, H=H, N=N, d=d, before=before, ragged=ragged)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _keys(g, B, H, N, d):
    """bf16 [B, H, N, d]: channels with an offset of their own, a few of them large, and one log-normal scale per token."""
    offset = 0.5 * _randn(g, 1, H, 1, d) * (1 + 7 * (torch.rand(1, H, 1, d, generator=g, device="cuda") < 0.04))
    return ((_randn(g, B, H, N, d) + offset) * torch.exp(0.25 * _randn(g, B, 1, N, 1))).bfloat16()


def _lengths(g, B, length, ragged):
    less = torch.randint(0, length * 3 // 4 + 1 if ragged else 1, (B,), generator=g, device="cuda")
    return (length - less).int()


def _groups(x):
    """(s, m, code) of bf16 rows [..., d]: bf16 [..., G], bf16 [..., G], int64 [..., G, 32]."""
    x = x.double().unflatten(-1, (-1, 32))
    lo, hi = x.amin(-1), x.amax(-1)
    s = ((hi - lo) / 15).bfloat16()
    s = torch.where(s < 2.0 ** -100, 0, s)
    m = (lo + 8 * s.double()).bfloat16()
    step = torch.where(s > 0, s.double(), 1)[..., None]
    code = (torch.round((x - m.double()[..., None]) / step) + 8).clamp_(0, 15).long()
    return s, m, code


def _nibbles(code, unit):
    """int64 [..., unit] codes -> uint8 [..., unit / 2], low nibble first."""
    pair = code.unflatten(-1, (unit // 2, 2))
    return (pair[..., 0] + 16 * pair[..., 1]).to(torch.uint8)


def _bytes(x):
    return x.contiguous().view(torch.uint8).flatten(3)


def _packed(K, V):
    """Rows [B, H, Ncap, d] as the cache holds them."""
    B, H, N, d = K.shape
    G = d // 32
    parts = []
    for x, unit in ((K, 8), (V, 4)):
        s, m, code = _groups(x)
        code = _nibbles(code.unflatten(-1, (32 // unit, unit)), unit)                    # [B, H, N, G, 32 / unit, unit / 2]
        parts.append(_bytes(code.transpose(3, 4).reshape(B, H, N // 32, 32, 32 // unit, G, unit // 2)))
        parts.append(_bytes(s.reshape(B, H, N // 32, 32, G)))
        m = m.reshape(B, H, N // 32, 32, G)
        parts.append(_bytes(m if unit == 8 else m.transpose(3, 4)))
    return torch.cat(parts, 3).contiguous()


def prepare(case, seed):
    c, s = case, {"case": case}
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, B, H, d = c["kind"], c["B"], c["H"], c["d"]
    if kind in ("attend", "read"):
        cap = (c["len"] + 63) // 32 * 32                                                 # room for some tokens more
        s["len"] = _lengths(g, B, c["len"], c["ragged"])
        K, V = _keys(g, B, H, cap, d), _randn(g, B, H, cap, d).bfloat16()
        if kind == "attend":
            Hq, Tq = H * c["R"], c["Tq"]
            q = _randn(g, B, Tq, Hq, d)
            # a few tokens that the query looks at
            at = (torch.rand(B, Tq, Hq, 1, generator=g, device="cuda") * s["len"].view(B, 1, 1, 1)).long()
            seen = K.repeat_interleave(c["R"], 1).transpose(1, 2).gather(1, at.expand(-1, -1, -1, d))
            s["q"] = (q + 0.4 * seen).bfloat16().transpose(1, 2)                         # heads inside tokens, as projected
            s["out"] = torch.zeros(B, Tq, Hq, d, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
            s["lse"] = torch.zeros(B, Hq, Tq, device="cuda")
            s["scale"] = d ** -0.5
            if own:
                from paper_2601_17818_b200 import binding as vb
                s["workspace"] = vb.alloc_workspace(vb.OP_CACHE_ATTENTION, B=B, H=H, N=cap, d=d, Nv=Tq, D=Hq)
        else:
            s["K_out"], s["V_out"] = (torch.zeros(B, H, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["cache"] = _packed(K, V)
        return s
    if kind == "write":
        N = c["N"]
        s["K"], s["V"] = (_keys(g, B, N, H, d).transpose(1, 2), _randn(g, B, N, H, d).bfloat16().transpose(1, 2))
        s["len"] = _lengths(g, B, c["before"], c["ragged"])
        cap, rows = (c["before"] + N + 63) // 32 * 32, N
    else:
        n, T = c["n"], c["T"]
        s["K"], s["V"] = _keys(g, B, H, n + T, d), _randn(g, B, H, n + T, d).bfloat16()
        s["len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        # the quotas of clusters leave every sample a little less than the budget
        s["n_keep"] = (c["keep"] - torch.randint(0, c["keep"] // 16 + 1, (B,), generator=g, device="cuda")).int()
        order = torch.rand(B, n, generator=g, device="cuda").argsort(1)
        order = torch.where(torch.arange(n, device="cuda") < s["n_keep"][:, None], order, n)
        s["keep_idx"] = order.sort(1).values[:, :c["keep"]].clamp(max=n - 1).int().contiguous()
        cap, rows = (T + c["keep"] + 63) // 32 * 32, T + c["keep"]
    s["cache"] = torch.zeros(B, H, cap // 32, 40 * d, dtype=torch.uint8, device="cuda")
    s["K_out"], s["V_out"] = (torch.zeros(B, H, rows, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    kind = c["kind"]
    if kind == "attend":
        return _attention(s, c)
    if kind == "read":
        K, V = _unpacked(s["cache"], c["d"])
        there = (torch.arange(K.shape[2], device="cuda") < s["len"][:, None])[:, None, :, None]
        return {"K": torch.where(there, K, 0).bfloat16(), "V": torch.where(there, V, 0).bfloat16()}
    K, V, count = s["K"], s["V"], c.get("N")
    if kind == "prune":
        K, V, count = _kept(s, c)
    K, V = _values(K), _values(V)
    if kind == "prune":
        there = (torch.arange(K.shape[2], device="cuda") < count[:, None])[:, None, :, None]
        K, V = torch.where(there, K, 0), torch.where(there, V, 0)
    return {"K": K.bfloat16(), "V": V.bfloat16(), "new_len": (s["len"] + count).int()}


def _run_own(s, c):
    from paper_2601_17818_b200 import binding as vb
    kind = c["kind"]
    if kind == "attend":
        vb.vitcop_cache_attention(s["q"], s["cache"], s["len"], s["out"], s["workspace"], s["scale"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "read":
        vb.vitcop_cache_read(s["cache"], s["len"], s["K_out"], s["V_out"])
        return {"K": s["K_out"], "V": s["V_out"]}
    if kind == "prune":
        vb.vitcop_cache_write(s["K"], s["V"], s["cache"], s["new_len"], vis_start=c["T"] // 2, vis_len=c["n"], keep_idx=s["keep_idx"],
                              n_keep=s["n_keep"])
    else:
        vb.vitcop_cache_write(s["K"], s["V"], s["cache"], s["new_len"], cache_len=s["len"])
    # (what stands in the cache is compared as the values it stands for)
    vb.vitcop_cache_read(s["cache"], s["new_len"], s["K_out"], s["V_out"], row_begin=s["len"])
    return {"K": s["K_out"], "V": s["V_out"], "new_len": s["new_len"]}


def _kept(s, c):
    """Rows that stay, in their order: text in front, kept visual tokens, text behind; how many there are."""
    n, T, keep, front = c["n"], c["T"], c["keep"], c["T"] // 2
    r, kept = torch.arange(T + keep, device="cuda")[None], s["n_keep"][:, None].long()
    visual = front + s["keep_idx"].gather(1, (r - front).clamp(0, keep - 1).expand(c["B"], -1)).long()
    src = torch.where(r < front, r, torch.where(r < front + kept, visual, r - kept + n)).clamp(max=n + T - 1)
    src = src[:, None, :, None].expand(-1, c["H"], -1, c["d"])
    return s["K"].gather(2, src), s["V"].gather(2, src), T + s["n_keep"]


def _values(x):
    """What the cache holds of bf16 rows, as the values it stands for; 64 bits, because a code next to a border between two
    steps falls to the wrong one otherwise."""
    s, m, code = _groups(x)
    return (m.double()[..., None] + (code - 8) * s.double()[..., None]).flatten(-2)


def _unpacked(cache, d):
    """The values of K and V, fp32 [B, H, Ncap, d]."""
    B, H, blocks, _ = cache.shape
    G, out, at = d // 32, [], 0
    for unit in (8, 4):
        code = cache[..., at:at + 16 * d].unflatten(-1, (32, 32 // unit, G, unit // 2)).transpose(4, 5)
        code = torch.stack([code & 15, code >> 4], -1).reshape(B, H, blocks * 32, G, 32).float() - 8
        s = cache[..., at + 16 * d:at + 18 * d].contiguous().view(torch.bfloat16).reshape(B, H, blocks * 32, G, 1).float()
        m = cache[..., at + 18 * d:at + 20 * d].contiguous().view(torch.bfloat16)
        m = m.unflatten(-1, (32, G)) if unit == 8 else m.unflatten(-1, (G, 32)).transpose(3, 4)
        out.append((m.reshape(B, H, blocks * 32, G, 1).float() + code * s).flatten(-2))
        at += 20 * d
    return out


def _attention(s, c):
    B, H, R, Tq, d = c["B"], c["H"], c["R"], c["Tq"], c["d"]
    K, V = _unpacked(s["cache"], d)
    N = K.shape[2]
    q = s["q"].float().reshape(B, H, R * Tq, d)
    logits = (q @ K.transpose(2, 3)).view(B, H, R, Tq, N) * s["scale"]
    # query t stands at position len - Tq + t and sees what is not behind it
    last = s["len"].view(B, 1, 1, 1, 1) - Tq + torch.arange(Tq, device="cuda").view(1, 1, 1, Tq, 1)
    seen = torch.arange(N, device="cuda") <= last
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    V = torch.where(torch.arange(N, device="cuda").view(1, 1, N, 1) < s["len"].view(B, 1, 1, 1), V, 0)
    out = (p.view(B, H, R * Tq, N) @ V).view(B, H, R, Tq, d) / torch.where(total == 0, 1, total)
    return {"out": out.bfloat16().view(B, H * R, Tq, d), "lse": (top + torch.log(total)).view(B, H * R, Tq)}


# ---------------------------------------------------------------------------------------------- from the definition, in 64 bits
def _nearest(x):
    """Values that bf16 rows are held as: of the sixteen that a group has, the nearest, the even code of two that are as near."""
    x = x.double().unflatten(-1, (x.shape[-1] // 32, 32))
    lo = x.min(-1, keepdim=True).values
    s = ((x.max(-1, keepdim=True).values - lo) / 15).bfloat16().double()
    m = (lo + 8 * s).bfloat16().double()
    best, away = m - 8 * s, (x - (m - 8 * s)).abs()
    best = best.expand_as(x)
    for code in range(1, 16):
        value = m + (code - 8) * s
        off = (x - value).abs()
        nearer = (off < away) | ((off == away) & (code % 2 == 0))
        best, away = torch.where(nearer, value, best), torch.minimum(off, away)
    return best.flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, B, H, d = c["kind"], c["B"], c["H"], c["d"]
    length = s["len"].long()
    if kind in ("attend", "read"):
        # the rows that prepare packed, made again from the seed
        g = torch.Generator(device="cuda").manual_seed(seed)
        _lengths(g, B, c["len"], c["ragged"])
        cap = s["cache"].shape[2] * 32
        K = _nearest(_keys(g, B, H, cap, d))
        V = _nearest(_randn(g, B, H, cap, d).bfloat16())
        behind = torch.arange(cap, device="cuda")[None] >= length[:, None]
        if kind == "read":
            return {"K": K.masked_fill(behind[:, None, :, None], 0), "V": V.masked_fill(behind[:, None, :, None], 0)}
        R, Tq = c["R"], c["Tq"]
        q = s["q"].double().unflatten(1, (H, R))
        z = torch.einsum("bhrtd,bhnd->bhrtn", q, K) * s["scale"]
        t = torch.arange(Tq, device="cuda")
        later = torch.arange(cap, device="cuda")[None, None] > (length[:, None] - Tq + t[None])[..., None]      # [B, Tq, N]
        z = z.masked_fill(later[:, None, None], -math.inf)
        lse = torch.logsumexp(z, -1)
        w = torch.exp(z - lse[..., None]).nan_to_num(0.0)
        out = torch.einsum("bhrtn,bhnd->bhrtd", w, V)
        return {"out": out.flatten(1, 2), "lse": lse.flatten(1, 2)}
    if kind == "write":
        return {"K": _nearest(s["K"]), "V": _nearest(s["V"]), "new_len": None}
    n, T, front = c["n"], c["T"], c["T"] // 2
    K = torch.zeros(B, H, T + c["keep"], d, dtype=torch.float64, device="cuda")
    V = torch.zeros_like(K)
    for b in range(B):
        kept = int(s["n_keep"][b])
        rows = torch.cat([torch.arange(front, device="cuda"), front + s["keep_idx"][b, :kept].long(),
                          torch.arange(front + n, n + T, device="cuda")])
        K[b, :, :len(rows)], V[b, :, :len(rows)] = _nearest(s["K"][b, :, rows]), _nearest(s["V"][b, :, rows])
    return {"K": K, "V": V, "new_len": None}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    kind, B, H, d = c["kind"], c["B"], c["H"], c["d"]
    row, held = 4 * d, 5 * d // 4                                                        # K and V of a row: in bf16, in the cache
    if kind in ("attend", "read"):
        rows = B * H * c["len"] * (5 / 8 if c["ragged"] else 1)
        if kind == "read":
            return {"bytes": int(rows * (held + row)), "flops": int(rows * 4 * d)}
        queries = B * H * c["R"] * c["Tq"]
        return {"bytes": int(rows * held) + queries * (4 * d + 4), "flops": int(rows * c["R"] * c["Tq"] * 4 * d)}
    # bf16 rows in, the cache written and read, values out
    rows = B * H * (c["N"] if kind == "write" else c["T"] + c["keep"])
    return {"bytes": rows * (2 * row + 2 * held), "flops": rows * 2 * d * 10}
