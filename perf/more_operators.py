"""Rotary positions on a grid and attention over K and V in bf16: what is measured, in plain torch and as the framework's calls.

A pruned sequence goes on through the model.  Its queries and keys are turned by positions of several axes (time, height, width),
every kept token by those that it had ("rope"); its tokens attend over K and V with a window and a few first tokens that stay
visible, a whole prompt at once or one token a step ("window"); and drafted tokens that form a tree are checked at once ("tree").

rope    pair (e, e + F) of a row, F = n_freq, turns by position[axis[e]] * inv_freq[e]: (a, b) -> (a cos - b sin, b cos + a sin),
        the other way round for gradients; what is behind 2 F is copied.  Row r of sample b is token[b][r] (none: r); rows without a
        token, or behind the sequence, stay as they were.
window  query t of sample b, t < query_len[b], stands at p = cache_len[b] - query_len[b] + t and sees rows j <= p of K and V with
        j < n_sink or j > p - window.
tree    query t sees the rows in front of cache_len[b] - query_len[b], and row i behind that where bit i of tree[b][t] is set.

Sizes: LLaVA-1.5-like images (576 tokens, 192 kept), AnyRes images (2880, 640 kept), clips (4608) and long videos with grouped
heads (16384), with the text around them; heads of 128 and 64.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the token of one chat's step: the smallest call, where latency counts
        _rope("rope_token_b1", 1, 32, 32, 128, 1, 64, 3, False, False),
        # what a pruning step keeps of high-resolution images, turned in the next layer by the positions that it had
        _rope("rope_kept_b8", 8, 32, 32, 128, 704, 64, 3, True, False),
        # clips before pruning, grouped heads: the most bytes
        _rope("rope_clip_b4", 4, 28, 4, 128, 4672, 64, 3, False, False),
        # the gradient of the same, narrow heads of which half is turned, height and width alone
        _rope("rope_gradient_b2", 2, 16, 16, 64, 2943, 16, 2, False, True),
        # the next token of one chat about one image
        _window("window_token_b1", 1, 32, 1, 1, 128, 640, 256, 35, False, False),
        # a serving batch on long videos, seven query heads to a stored one, every chat at another length
        _window("window_token_b16", 16, 4, 7, 1, 128, 16512, 4096, 64, True, False),
        # the questions behind pruned clips, narrow heads
        _window("window_question_b4", 4, 8, 4, 64, 64, 1501, 512, 16, True, False),
        # prompts with pruned images, every one of another length, padded behind
        _window("window_prompt_b8", 8, 32, 1, 704, 128, 704, 256, 35, True, True),
        # two clips' prompts, grouped heads
        _window("window_clip_b2", 2, 4, 7, 4672, 128, 4672, 1024, 64, False, True),
        # a long video's prompt: the most work
        _window("window_long_b1", 1, 4, 7, 16512, 128, 16512, 4096, 64, False, True),
        # a tree of 25 drafted tokens of one chat
        _tree("tree_b1", 1, 32, 1, 25, 128, 640, False),
        # larger trees in a batch of chats about clips, grouped heads, every one at another length
        _tree("tree_b8", 8, 4, 7, 60, 128, 4672, True),
    ]


def draw(rng):
    while True:
        kind = rng.choice(["rope", "rope", "window", "window", "window", "window", "tree", "tree"])
        B, d = int(_log_uniform(rng, 1, 16)), rng.choice([64, 128, 128])
        H, R = rng.choice([(32, 1), (4, 7), (8, 4), (4, 4), (16, 1), (12, 1), (2, 8)])
        ragged = rng.random() < 0.6
        if kind == "rope":
            N = rng.choice([1, int(_log_uniform(rng, 1, 16512)), int(_log_uniform(rng, 64, 16512))])
            case = _rope("", B, H * R, H, d, N, rng.choice([d // 2, d // 2, d // 4]), rng.choice([1, 2, 3, 3]), rng.random() < 0.4, rng.random() < 0.3)
        elif kind == "window":
            length = int(_log_uniform(rng, 64, 16512))
            Tq = rng.choice([1, 1, 1, 2, 5, 17, 64, length, length, int(_log_uniform(rng, 64, length))])
            case = _window("", B, H, R, min(Tq, length), d, length, int(_log_uniform(rng, 32, 8192)), rng.choice([0, 4, 35, 64, 130]), ragged,
                           Tq == length)
        else:
            Tq = rng.choice([2, 7, 16, 25, 33, 60, 64])
            case = _tree("", B, H, R, Tq, d, int(_log_uniform(rng, max(64, 5 * Tq), 16512)), ragged)
        case.pop("name", None)
        # no dearer than the dearest of the list, and memory for several states
        w = work(case)
        rows = case["N"] if kind == "rope" else case["len"]
        if w["bytes"] <= 3e8 and w["flops"] <= 9e11 and B * H * R * rows * d <= 1 << 27 and B * H * R * case.get("Tq", 1) * rows <= 1 << 32:
            return case


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))


def _rope(name, B, Hq, Hk, d, N, F, axes, kept, gradient):
    return dict(name=name, kind="rope", B=B, Hq=Hq, H=Hk, d=d, N=N, F=F, axes=axes, kept=kept, gradient=gradient)


def _window(name, B, H, R, Tq, d, length, window, n_sink, ragged, prompt):
    return dict(name=name, kind="window", B=B, H=H, R=R, Tq=Tq, d=d, len=length, window=window, n_sink=n_sink, ragged=ragged, prompt=prompt)


def _tree(name, B, H, R, Tq, d, length, ragged):
    return dict(name=name, kind="tree", B=B, H=H, R=R, Tq=Tq, d=d, len=length, ragged=ragged)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _grid_positions(g, axes, B, n):
    """int32 [axes, B, n]: text, frames of 12 x 12 tokens, text again; every sample's conversation began somewhere else."""
    start = torch.randint(0, 20000, (B, 1), generator=g, device="cuda")
    front = min(n // 8, 35)
    side, i = 12, torch.arange(n, device="cuda")
    v = (n - 2 * front) // (side * side) * side * side                                  # visual tokens
    r = (i - front).clamp(0, max(v - 1, 0))
    tyx = torch.stack([r // (side * side), r // side % side, r % side])
    text = torch.where(i < front, i, front + max(v // (side * side), side if v else 0) + i - front - v)
    at = torch.where((i >= front) & (i < front + v), front + tyx, text)                  # [3, n]
    return (at[[0, 1, 2][-axes:], None] + start).int().contiguous()


def _keys(g, B, H, N, d):
    """bf16 [B, H, N, d]: channels with an offset of their own, a few of them large, and one log-normal scale per token."""
    offset = 0.5 * _randn(g, 1, H, 1, d) * (1 + 7 * (_rand(g, 1, H, 1, d) < 0.04))
    return ((_randn(g, B, H, N, d) + offset) * torch.exp(0.25 * _randn(g, B, 1, N, 1))).bfloat16()


def _trees(g, B, T):
    """int64 [B, T]: bit i of word t is set where drafted token i is t or an ancestor of it; a few chains and what branches off."""
    word = torch.zeros(B, T, dtype=torch.int64, device="cuda")
    back = (1 + 4 * _rand(g, B, T) ** 2).long()
    for t in range(T):
        parent = (t - back[:, t]).clamp(min=-1)
        above = torch.where(parent >= 0, word.gather(1, parent.clamp(min=0)[:, None])[:, 0], 0)
        # (bit 63 is the sign)
        word[:, t] = above | (1 << t if t < 63 else -(1 << 63))
    return word


def prepare(case, seed):
    c, s = case, {"case": case}
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, d = c["B"], c["H"], c["d"]
    if c["kind"] == "rope":
        N, F = c["N"], c["F"]
        s["q"], s["k"] = (_randn(g, B, N, h, d).bfloat16().transpose(1, 2) for h in (c["Hq"], H))      # heads inside tokens, as projected
        n = N if not c["kept"] else 2 * N + 71
        s["position"] = _grid_positions(g, c["axes"], B, n)
        # frequencies in sections, one an axis, as even as they go
        s["axis"] = (torch.arange(F, device="cuda") * c["axes"] // F).int()
        s["inv_freq"] = 1e6 ** (-torch.arange(F, device="cuda", dtype=torch.float64) / F)
        s["token"] = None
        if c["kept"]:
            # which tokens the rows are: some of them, in their order; less in some samples
            order = _rand(g, B, n).argsort(1)[:, :N].sort(1).values
            rows = N - torch.randint(0, N // 16 + 1, (B, 1), generator=g, device="cuda")
            s["token"] = torch.where(torch.arange(N, device="cuda") < rows, order, -1).int()
        s["q_out"], s["k_out"] = (torch.zeros(B, h, N, d, dtype=torch.bfloat16, device="cuda") for h in (c["Hq"], H))
        return s
    R, Tq, length = c["R"], c["Tq"], c["len"]
    Hq, cap = H * R, (length + 63) // 32 * 32                                            # room for some tokens more
    less = torch.randint(0, (length - Tq if not c.get("prompt") else length // 2) * 3 // 4 + 1 if c["ragged"] else 1, (B,), generator=g, device="cuda")
    s["len"] = (length - less).int()
    s["query_len"] = s["len"] if c.get("prompt") else None
    s["K"], s["V"] = _keys(g, B, H, cap, d), _randn(g, B, H, cap, d).bfloat16()
    # a token that each query looks at
    at = _rand(g, B, Tq, Hq, 1) * s["len"].view(B, 1, 1, 1)
    if c.get("prompt"):
        at = at * (torch.arange(Tq, device="cuda") + 1).view(1, Tq, 1, 1) / length
    q = _randn(g, B, Tq, Hq, d)
    for h in range(Hq):
        q[:, :, h] += 0.4 * s["K"][:, h // R].gather(1, at[:, :, h].long().expand(-1, -1, d))
    s["q"] = q.bfloat16().transpose(1, 2)                                                # heads inside tokens, as projected
    s["scale"] = d ** -0.5
    if c["kind"] == "tree":
        s["tree"] = _trees(g, B, Tq)
    s["out"] = torch.zeros(B, Tq, Hq, d, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    s["lse"] = torch.zeros(B, Hq, Tq, device="cuda")
    if own:
        from paper_2601_17818_b200 import binding as vb
        s["workspace"] = vb.alloc_workspace(vb.OP_ATTENTION, B=B, H=H, N=cap, d=d, Nv=Tq, D=Hq)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "rope":
        return _rotated(s, c)
    # as many queries at a time as a gigabyte of logits holds
    B, Hq, Tq, d = s["q"].shape
    chunk = max(1, (1 << 28) // (B * Hq * s["K"].shape[2]))
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    for t in range(0, Tq, chunk):
        _attention(s, c, t, min(Tq, t + chunk), out, lse)
    return {"out": out, "lse": lse}


def _run_own(s, c):
    from paper_2601_17818_b200 import binding as vb
    if c["kind"] == "rope":
        vb.vitcop_rotary_axes(s["q"], s["k"], s["position"], s["inv_freq"], s["axis"], s["q_out"], s["k_out"], token=s["token"],
                              inverse=c["gradient"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "window":
        vb.vitcop_window_attention(s["q"], s["K"], s["V"], s["len"], s["out"], s["workspace"], s["scale"], c["window"], c["n_sink"],
                                   query_len=s["query_len"], lse=s["lse"])
    else:
        vb.vitcop_tree_attention(s["q"], s["K"], s["V"], s["len"], s["tree"], s["out"], s["workspace"], s["scale"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _rotated(s, c):
    F, position, token = c["F"], s["position"], s["token"]
    if token is not None:
        position = position.gather(2, token.clamp(min=0).long().expand(c["axes"], -1, -1))
    # (64 bits: a position of 20000 leaves 32 of them three digits of the turn)
    angle = position[s["axis"].long()].double() * s["inv_freq"].view(F, 1, 1)            # [F, B, N]
    cos, sin = angle.cos().float().permute(1, 2, 0)[:, None], angle.sin().float().permute(1, 2, 0)[:, None]
    if c["gradient"]:
        sin = -sin
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        a, b = x[..., :F], x[..., F:2 * F]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * F:]], -1)
        if token is not None:
            y = torch.where((token >= 0)[:, None, :, None], y, 0)
        out[name] = y.bfloat16()
    return out


def _attention(s, c, t0, t1, out, lse):
    """Queries t0 .. t1 - 1, all of whose logits are held at a time."""
    B, H, R, d = c["B"], c["H"], c["R"], c["d"]
    K, V, length = s["K"], s["V"], s["len"].view(B, 1, 1)
    count = length if s["query_len"] is not None else torch.full_like(length, c["Tq"])
    t = torch.arange(t0, t1, device="cuda").view(1, -1, 1)
    j = torch.arange(K.shape[2], device="cuda")
    if c.get("prompt"):
        # (positions are the rows' own: what no query of these sees is left out)
        first = max(c["n_sink"], t0 - c["window"] + 1)
        j = torch.cat([j[:min(c["n_sink"], t1)], j[first:t1]])
        K, V = K[:, :, j], V[:, :, j]
    p = length - count + t
    if c["kind"] == "window":
        seen = (j <= p) & ((j < c["n_sink"]) | (j > p - c["window"]))
    else:
        i = j - (length - count)
        seen = (i < 0) | ((i < count) & ((s["tree"][:, t0:t1, None] >> i.clamp(0, 63)) & 1 == 1))
    seen = (seen & (j < length))[:, None, None]
    q = s["q"][:, :, t0:t1].float().reshape(B, H, R * (t1 - t0), d)
    logits = (q @ K.float().transpose(2, 3)).view(B, H, R, t1 - t0, -1) * s["scale"]
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    w = torch.exp(logits - top)
    total = w.sum(-1, keepdim=True)
    V = torch.where((j < length).view(B, 1, -1, 1), V, 0).float()
    o = (w.view(B, H, R * (t1 - t0), -1) @ V).view(B, H, R, t1 - t0, d) / torch.where(total == 0, 1, total)
    there = (t < count).view(B, 1, -1, 1)
    out[:, :, t0:t1] = torch.where(there, o.flatten(1, 2), 0).bfloat16()
    lse[:, :, t0:t1] = torch.where(there[..., 0], (top + torch.log(total)).flatten(1, 2)[..., 0], 0)


# ---------------------------------------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, H, d = c["B"], c["H"], c["d"]
    if c["kind"] == "rope":
        F = c["F"]
        out = {}
        for name in ("q", "k"):
            x = s[name].double()
            y = torch.zeros_like(x, memory_format=torch.contiguous_format)
            for b in range(B):
                there = torch.arange(c["N"], device="cuda")
                which = there
                if s["token"] is not None:
                    there = (s["token"][b] >= 0).nonzero()[:, 0]
                    which = s["token"][b, there].long()
                at = torch.stack([s["position"][int(a), b, which] for a in s["axis"]], 1).double()   # [rows, F]
                turn = torch.polar(torch.ones_like(at), (-at if c["gradient"] else at) * s["inv_freq"])
                z = torch.complex(x[b, :, there, :F], x[b, :, there, F:2 * F]) * turn
                y[b][:, there, :F], y[b][:, there, F:2 * F], y[b][:, there, 2 * F:] = z.real, z.imag, x[b, :, there, 2 * F:]
            out[name] = y
        return out
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    R = c["R"]
    for b in range(B):
        n = int(s["len"][b])
        Tq = n if c.get("prompt") else c["Tq"]
        base = n - Tq
        for t0 in range(0, Tq, 1024):
            t1 = min(Tq, t0 + 1024)
            if c["kind"] == "window":
                begin = max(0, base + t0 - c["window"] + 1)
                rows = sorted(set(range(min(c["n_sink"], base + t1))) | set(range(begin, base + t1)))
            else:
                rows = range(n)
            rows = torch.tensor(list(rows), device="cuda")
            p = base + torch.arange(t0, t1, device="cuda")[:, None]
            if c["kind"] == "window":
                hidden = (rows > p) | ((rows >= c["n_sink"]) & (rows + c["window"] <= p))
            else:
                words = s["tree"][b].tolist()
                hidden = torch.tensor([[i >= base and not words[t] >> (i - base) & 1 for i in range(n)] for t in range(t0, t1)], device="cuda")
            for h in range(H):
                k, v = s["K"][b, h, rows].double(), s["V"][b, h, rows].double()
                for r in range(R):
                    z = (s["q"][b, h * R + r, t0:t1].double() @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
                    total = torch.logsumexp(z, -1)
                    lse[b, h * R + r, t0:t1] = total
                    out[b, h * R + r, t0:t1] = torch.exp(z - total[:, None]) @ v
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    B, H, d = c["B"], c["H"], c["d"]
    if c["kind"] == "rope":
        rows = B * c["N"]
        return {"bytes": rows * ((c["Hq"] + H) * d * 4 + 4 * c["axes"]), "flops": rows * (c["Hq"] + H) * c["F"] * 6}
    R, Tq, length = c["R"], c["Tq"], c["len"]
    mean = length * (5 / 8 if c["ragged"] and not c.get("prompt") else 1)
    if c["kind"] == "tree":
        rows, pairs = mean, Tq * mean
    else:
        rows = min(mean, c["n_sink"] + c["window"] + Tq)
        if c.get("prompt"):
            # (a ragged batch has 13/16 of the rows on average)
            n = length * (13 / 16 if c["ragged"] else 1)
            w, rows = min(c["window"] + c["n_sink"], n), n
            pairs = w * (w + 1) / 2 + (n - w) * w
            Tq = n
        else:
            pairs = Tq * min(mean, c["n_sink"] + c["window"])
    return {"bytes": int(B * H * rows * 4 * d + B * H * R * Tq * (4 * d + 4)), "flops": int(B * H * R * pairs * 4 * d)}
