"""Operators of models with normalised queries and keys, and of serving with drafted tokens, as cases that can be timed.

A case is a dict of plain values.
  kind    "norm"    queries and keys normalised head by head (root mean square, a weight for every column) and rotated by their positions, and
                    the gradients of both and of the weights (a training step on either side of the attention): B, H, KV, N rows, d, dims
                    (rotated columns), pairs, factor, q_off, far, layout; w32 (weights in fp32)
          "append"  new tokens of S sequences: queries and keys normalised and rotated, keys and values written to their pages
          "tree"    attention of drafted tokens over their sequences' pages: all of the context, and of the new tokens those that a mask names
                    (of sequences with more new tokens than a mask has bits, 64 x words: those before)
          "plan"    what a step's calls read, from the lengths of the requests: starts, lengths, pages, slots, positions, masks of the trees
          "keep"    the accepted ones of the drafted tokens moved together, in every layer's pages
  Those of a cache: S, H, KV, d, dtype, page (rows of a page), pool ("head": [pages, heads, rows, d]; "seq": [pages, rows, heads, d] seen with
  heads first); sequence lengths (with the new tokens) from len_lo to len_hi and new tokens from new_lo to new_hi, spread evenly over
  their logarithm by the whole number `mix`; words; bushy (a drafted token hangs on one of so many before it).
Values are N(0, 1), weights 1 + N(0, 1) / 8 (trained norms stay near 1)."""
import math
import random

import torch

own = False

_BASE = 10000.0
_EPS = 1e-6


def _norm(name=None, dtype="bf16", B=1, H=32, KV=8, N=4096, d=128, dims=128, pairs="half", factor=1.0, q_off=0, far=0, layout="head", w32=False):
    c = dict(kind="norm", dtype=dtype, B=B, H=H, KV=KV, N=N, d=d, dims=dims, pairs=pairs, factor=factor, q_off=q_off, far=far, layout=layout, w32=w32)
    return dict(c, name=name) if name else c


def _cache(kind, name=None, dtype="bf16", S=1, H=32, KV=8, d=128, page=64, pool="head", len_lo=4096, len_hi=4096, new_lo=1, new_hi=1, mix=1, words=1,
           bushy=4, window=0, dims=128, pairs="half", factor=1.0, layers=1, trees=True, ended=0):
    c = dict(kind=kind, S=S, page=page, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi, mix=mix, words=words, bushy=bushy)
    if kind == "plan":
        c.update(trees=trees, ended=ended)
    else:
        c.update(dtype=dtype, H=H, KV=KV, d=d, pool=pool)
        c.update(dict(dims=dims, pairs=pairs, factor=factor) if kind == "append" else dict(window=window) if kind == "tree" else dict(layers=layers))
    return dict(c, name=name) if name else c


def listed():
    return [
        # A training step's layer on the last rank of the benchmark's ring, grouped heads.
        _norm("norm_last_rank", q_off=7 * 4096),
        # Sequence-major activations of a batch, interleaved pairs, a stretched context, weights kept in fp32, no round number of rows.
        _norm("norm_seq_major_scaled", B=2, H=16, KV=16, N=1501, d=64, dims=64, pairs="interleaved", factor=4.0, layout="seq", w32=True),
        # fp32, part of a head that is neither 64 nor 128 wide, positions up to a million; the host's calls are what counts.
        _norm("norm_f32_far_partial", dtype="f32", H=8, KV=2, N=333, d=80, dims=32, far=1 << 20),
        # One token for each of 64 sequences: a step of serving.
        _cache("append", "append_single_tokens", S=64, page=16, len_lo=100, len_hi=4000),
        # Trees of some sequences and chunks of others' prompts, packed together, into a cache that lies sequence-major.
        _cache("append", "append_trees_and_chunks", S=12, pool="seq", len_lo=2048, len_hi=8192, new_lo=8, new_hi=2048, dims=64, pairs="interleaved", factor=8.0),
        # One user, a long context, a tree of the most tokens that a mask's first word names.
        _cache("tree", "tree_one_long", len_lo=32768, len_hi=32768, new_lo=64, new_hi=64),
        # A batch as a server has it: lengths from a few hundred to 16K, small and large trees.
        _cache("tree", "tree_ragged_batch", S=32, page=16, len_lo=300, len_hi=16384, new_lo=4, new_hi=48),
        # fp32, every head with keys of its own, 64 wide, short contexts, a few drafted tokens.
        _cache("tree", "tree_f32_few", dtype="f32", S=8, H=8, KV=8, d=64, page=32, pool="seq", len_lo=40, len_hi=2000, new_lo=3, new_hi=12, bushy=2),
        # A step of single tokens: nearly nothing to do, many times a second.
        _cache("plan", "plan_single_tokens", S=256, page=64, len_lo=16, len_hi=16384, trees=False),
        # Trees of many sequences, prompts of others, and sequences that have ended.
        _cache("plan", "plan_trees_and_prompts", S=400, page=16, len_lo=64, len_hi=8192, new_lo=4, new_hi=2000, ended=20),
        # Four users, two layers: over before the next launch.
        _cache("keep", "keep_few", S=4, page=16, len_lo=200, len_hi=3000, new_lo=8, new_hi=24, layers=2),
        # All layers' pages of a batch at once.
        _cache("keep", "keep_batch", S=96, pool="seq", len_lo=300, len_hi=2000, new_lo=8, new_hi=64, layers=24, bushy=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "append", "tree", "tree", "tree", "plan", "keep"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([128, 128, 64, 64, 96, 80, 32])
        KV, group = rng.choice([1, 2, 4, 8, 8, 32]), rng.choice([1, 1, 2, 4, 4, 8])
        H = KV * group
        dims, pairs, factor = rng.choice([d, d, d // 2, 16]), rng.choice(["half", "half", "interleaved"]), rng.choice([1.0, 1.0, 4.0, 16.0])
        if kind == "norm":
            far = rng.choice([0, 0, 1 << 20])
            c = _norm(dtype=dtype, B=rng.choice([1, 1, 2, 3]), H=H, KV=KV, N=_log(rng, 16, 8192), d=d, dims=dims, pairs=pairs, factor=factor,
                      q_off=0 if far else rng.choice([0, rng.randrange(1 << 18)]), far=far, layout=rng.choice(["head", "seq"]), w32=rng.random() < 0.4)
        else:
            c = _cache(kind, dtype=dtype, S=_log(rng, 1, 512 if kind == "plan" else 96), H=H, KV=KV, d=d, page=rng.choice([16, 32, 64, 128]),
                       pool=rng.choice(["head", "seq"]), mix=rng.randrange(1 << 20), bushy=rng.choice([1, 2, 4, 8]), words=rng.choice([1, 1, 1, 2, 4]))
            c["len_hi"] = _log(rng, 1, 32768 if kind == "tree" else 8192)
            c["len_lo"] = c["len_hi"] if rng.random() < 0.3 else _log(rng, 1, c["len_hi"])
            c["new_hi"] = min(c["len_hi"], _log(rng, 1, 64 * c["words"])) if kind in ("tree", "keep") or rng.random() < 0.6 else _log(rng, 1, c["len_hi"])
            c["new_lo"] = c["new_hi"] if rng.random() < 0.3 else _log(rng, 1, c["new_hi"])
            if kind == "append":
                c.update(dims=dims, pairs=pairs, factor=factor)
            elif kind == "tree":
                if rng.random() < 0.2:
                    c["window"] = _log(rng, 64, 8192)
                if rng.random() < 0.2:                          # chunks of prompts among them
                    c.update(words=1, new_hi=_log(rng, 1, min(512, c["len_hi"])))
                    c["new_lo"] = min(c["new_lo"], c["new_hi"])
            elif kind == "plan":
                c.update(trees=rng.random() < 0.6, ended=rng.choice([0, 0, c["S"] // 8]))
            elif kind == "keep":
                c["layers"] = _log(rng, 1, 24)
        if _affordable(c):
            return c


def _affordable(c):
    """No more than the largest listed case of its kind costs, the plain form's padding included."""
    w = work(c)
    if c["kind"] == "norm":
        return 1e6 < w["bytes"] < 3e8
    n, L = max(_news(c)), max(_lengths(c))
    if c["kind"] == "plan":
        return sum(_news(c)) < 300000
    pool = 4.0 * sum(_lengths(c)) * c["KV"] * c["d"] * c.get("layers", 1) * (1 if c["dtype"] == "bf16" else 2)
    if c["kind"] in ("append", "keep"):
        return w["bytes"] < 2e8 and pool < 1.2e10 and sum(_news(c)) < 100000
    return c["S"] * c["H"] * n * L <= 32 * 48 * 32 * 16384 and c["S"] * c["KV"] * L * c["d"] <= 64 * 8 * 16384 * 128 and w["flops"] < 1e12


def _spread(c, lo, hi, salt):
    rng = random.Random(2 * c["mix"] + salt)
    at = [i / max(1, c["S"] - 1) for i in range(c["S"])]
    rng.shuffle(at)
    return [int(round(math.exp(math.log(lo) + x * (math.log(hi) - math.log(lo))))) for x in at]


def _lengths(c):
    return _spread(c, c["len_lo"], c["len_hi"], 0)


def _news(c):
    """New tokens of each sequence: its last ones."""
    return [min(n, L) for n, L in zip(_spread(c, c["new_lo"], c["new_hi"], 1), _lengths(c))]


def work(case):
    """Every input read once and every output written once.  norm: x and y, then x, g and dx, 30 operations a value.  tree: the keys
    and values that some new token sees, 4 d operations a visible pair and query head (half of a tree's pairs taken for visible).  plan: what a
    sequence and a row have in the arrays, and the table's entries that rows lie in.  keep: moved rows (taken as three a sequence)."""
    c = case
    if c["kind"] == "plan":
        T, S = sum(_news(c)), c["S"]
        return {"bytes": 20.0 * S + T * (16.0 + (4 + 8 * c["words"] if c["trees"] else 0)) + 4.0 * (T // c["page"] + S), "flops": 2.0 * T}
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "norm":
        n = 1.0 * c["B"] * (c["H"] + c["KV"]) * c["N"] * c["d"]
        return {"bytes": 5 * n * e, "flops": 30 * n}
    if c["kind"] == "keep":
        return {"bytes": 12.0 * c["S"] * c["layers"] * c["KV"] * c["d"] * e, "flops": 0.0}
    T = sum(_news(c))
    if c["kind"] == "append":
        return {"bytes": 2.0 * T * (c["H"] + 2 * c["KV"]) * c["d"] * e, "flops": 10.0 * T * (c["H"] + c["KV"]) * c["d"]}
    keys = pairs = 0
    for n, L in zip(_news(c), _lengths(c)):
        w = min(c["window"] or L, L - n)
        keys += w + n
        pairs += n * (w + (n + 1) / 2)
    return {"bytes": 2.0 * keys * c["KV"] * c["d"] * e + T * c["H"] * (2.0 * c["d"] * e + 4), "flops": 4.0 * c["d"] * c["H"] * pairs}


# ------------------------------------------------------------------------------- inputs
def _turns(dims, factor, original=4096):
    """Turns per position of every pair, 64 bits.  factor > 1: pairs that turn more than 32 times over the original length keep
    their speed, those that turn less than once are slowed by the factor, the others are between."""
    t = _BASE ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims) / (2 * math.pi)
    keep = ((original * t - 1) / 31).clamp(0, 1)
    return t if factor == 1.0 else t * keep + t / factor * (1 - keep)


def _amplitude(factor):
    return 1.0 if factor == 1.0 else 0.1 * math.log(factor) + 1.0


def _parents(c, rng, n):
    """The token that each drafted one hangs on: one of the `bushy` before it; the first one (the last token that is sure) on none."""
    return [-1] + [rng.randrange(max(0, t - c["bushy"]), t) for t in range(1, n)]


def _branch(parents, t):
    """A token and those that it hangs on, the first one first."""
    path = []
    while t >= 0:
        path.append(t)
        t = parents[t]
    return path[::-1]


def _signed(mask, words):
    parts = [(mask >> (64 * w)) & ((1 << 64) - 1) for w in range(words)]
    return [p - (1 << 64) if p >> 63 else p for p in parts]


def _trees(c, seed, news):
    """For every sequence the parents of its tokens (a chunk's: none)."""
    rng = random.Random(seed)
    return [_parents(c, rng, n) if n <= 64 * c["words"] else None for n in news]


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if c["kind"] == "plan":
        return _prepare_plan(c, seed, gen)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    rand = lambda *shape: torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(dt)  # noqa: E731
    weight = lambda t: (1 + torch.randn(c["d"], generator=gen, device=dev) / 8).to(t)  # noqa: E731
    s = {k: c[k] for k in ("kind", "d", "H", "KV")}
    if c["kind"] in ("norm", "append"):
        s.update(turns=_turns(c["dims"], c["factor"]).to(dev), interleaved=c["pairs"] == "interleaved", amplitude=_amplitude(c["factor"]))
        s["w"] = [weight(torch.float32 if c.get("w32") else dt) for _ in range(2)]
    if c["kind"] == "norm":
        def rows(heads):
            if c["layout"] == "seq":
                return rand(c["B"], c["N"], heads, c["d"]).transpose(1, 2)
            return rand(c["B"], heads, c["N"], c["d"])
        s["x"] = [rows(h).requires_grad_(True) for h in (c["H"], c["KV"])]
        s["g"] = [rows(h) for h in (c["H"], c["KV"])]
        s["w"] = [w.requires_grad_(True) for w in s["w"]]
        s["offset"] = c["q_off"]
        s["positions"] = torch.randint(c["far"], (c["B"], c["N"]), generator=gen, device=dev) if c["far"] else None
        return s
    news, lengths = _news(c), _lengths(c)
    T, S, page = sum(news), c["S"], c["page"]
    per = [-(-L // page) for L in lengths]
    pages = sum(per) + 3
    pool = (lambda: rand(pages, page, c["KV"], c["d"]).transpose(1, 2)) if c["pool"] == "seq" else (lambda: rand(pages, c["KV"], page, c["d"]))
    layers = c.get("layers", 1)
    s["k_pages"], s["v_pages"] = [pool() for _ in range(layers)], [pool() for _ in range(layers)]
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu()
    table = torch.full((S, max(per)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s.update(table=table.to(dev), lengths=i32(lengths), starts=i32(starts), max_new=max(news))
    trees = _trees(c, seed, news)
    if c["kind"] == "keep":
        rng = random.Random(seed + 1)
        kept = [_branch(p, rng.randrange(len(p))) if p else list(range(n)) for p, n in zip(trees, news)]
        most = max(len(p) for p in kept)
        s.update(kept=i32([p + [0] * (most - len(p)) for p in kept]), counts=i32([len(p) for p in kept]))
        return s
    branches = [[_branch(p, t) for t in range(n)] if p else [range(t + 1) for t in range(n)] for p, n in zip(trees, news)]
    if c["kind"] == "tree":
        masks = [_signed(sum(1 << j for j in b), c["words"]) if p else [0] * c["words"] for p, bs in zip(trees, branches) for b in bs]
        s.update(q=rand(T, c["H"], c["d"]), tree=torch.tensor(masks, dtype=torch.int64, device=dev), scale=c["d"] ** -0.5, window=c["window"])
        return s
    qkv = rand(T, c["H"] + 2 * c["KV"], c["d"])
    s["q"], s["k"], s["v"] = qkv.split([c["H"], c["KV"], c["KV"]], dim=1)
    s["positions"] = torch.tensor([L - n + len(b) - 1 for L, n, bs in zip(lengths, news, branches) for b in bs], dtype=torch.int64, device=dev)
    rows = [(i, L - n + t) for i, (L, n) in enumerate(zip(lengths, news)) for t in range(n)]
    s["slots"] = torch.tensor([int(table[i, p // page]) * page + p % page for i, p in rows], dtype=torch.int64, device=dev)
    return s


def _prepare_plan(c, seed, gen):
    """The table of the last step (pages up to the lengths without the new tokens), and the other pages on the stack."""
    dev, S, page = "cuda", c["S"], c["page"]
    news, lengths = _news(c), _lengths(c)
    rng = random.Random(seed)
    ended = set(rng.sample(range(S), c["ended"]))
    have = [-(-(L - n) // page) for L, n in zip(lengths, news)]
    pages = sum(-(-L // page) for L in lengths) + S
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu()
    table = torch.full((S, max(-(-L // page) for L in lengths) + 5), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(have):
        table[i, :n] = order[at:at + n]
        at += n
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    free = torch.cat([order[at:], torch.zeros(at, dtype=torch.int32)])
    s = dict(kind="plan", page=page, new=i32([-1 if i in ended else n for i, n in enumerate(news)]), lengths=i32([L - n for L, n in zip(lengths, news)]),
             table=table.to(dev), free=free.to(dev), count=i32([pages - at]), rows=sum(news), words=c["words"], parents=None)
    if c["trees"]:
        trees = _trees(c, seed, news)
        most = max([len(p) for p in trees if p] + [1])
        s["parents"] = i32([(p or []) + [-1] * (most - len(p or [])) for p in trees])
    return s


# ------------------------------------------------------------------------------- one pass
def run(state):
    s = state
    if own:
        return _run_own(s)
    return {"norm": _norm_plain, "append": _append_plain, "tree": _tree_plain, "plan": _plan_plain, "keep": _keep_plain}[s["kind"]](s)


def _run_own(s):
    if s["kind"] == "norm":
        from paper_2403_09347_amd.rotary import burst_norm_rotary
        y = burst_norm_rotary(s["x"], s["w"], s["turns"], _EPS, offset=s["offset"], positions=s["positions"], interleaved=s["interleaved"],
                              amplitude=s["amplitude"])
        return [t.detach() for t in y] + list(torch.autograd.grad(y, s["x"] + s["w"], s["g"]))
    from paper_2403_09347_amd import paged
    if s["kind"] == "append":
        k, v = s["k_pages"][0], s["v_pages"][0]
        q = paged.burst_cache_append(s["k"], s["v"], k, v, s["table"], s["lengths"], s["starts"], q=s["q"], turns=s["turns"], interleaved=s["interleaved"],
                                     amplitude=s["amplitude"], q_norm=s["w"][0], k_norm=s["w"][1], eps=_EPS, slots=s["slots"], positions=s["positions"])
        return [q, k, v]
    if s["kind"] == "tree":
        return list(paged.burst_paged_attention(s["q"], s["k_pages"][0], s["v_pages"][0], s["table"], s["lengths"], s["starts"], scale=s["scale"],
                                                window=s["window"], max_new=s["max_new"], tree=s["tree"]))
    if s["kind"] == "plan":
        p = paged.burst_cache_plan(s["new"], s["lengths"], s["table"], s["free"], s["count"], s["page"], s["rows"], parents=s["parents"], words=s["words"])
        return [t for t in p if t is not None] + [s["table"], s["free"], s["count"]]
    lengths = paged.burst_cache_keep(s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["starts"], s["kept"], s["counts"])
    return [lengths] + s["k_pages"] + s["v_pages"]


def _rotated(f, cos, sin, interleaved):
    """The first columns of f (32 bits), in pairs, turned by the angles of cos and sin [..., pairs]."""
    n = cos.shape[-1]
    a, b = (f[..., 0:2 * n:2], f[..., 1:2 * n:2]) if interleaved else (f[..., :n], f[..., n:2 * n])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, f[..., 2 * n:]], -1)


def _angles(positions, s):
    """cos and sin at the positions, computed in 64 bits, rounded to 32."""
    turn = positions.double().unsqueeze(-1) * s["turns"]
    a = (turn - turn.round()) * (2 * math.pi)
    return (torch.cos(a) * s["amplitude"]).float(), (torch.sin(a) * s["amplitude"]).float()


def _root(f):
    return torch.rsqrt((f * f).mean(-1, keepdim=True) + _EPS)


def _norm_plain(s):
    x, g, w = s["x"], s["g"], s["w"]
    at = s["positions"] if s["positions"] is not None else s["offset"] + torch.arange(x[0].shape[2], device=x[0].device).unsqueeze(0)
    cos, sin = (t.unsqueeze(1) for t in _angles(at, s))

    def forward(x, w):
        f = x.float()
        return _rotated(f * _root(f) * w.float(), cos, sin, s["interleaved"]).to(x.dtype)

    def backward(x, w, g):
        f, h = x.float(), _rotated(g.float(), cos, -sin, s["interleaved"])
        r = _root(f)
        f = f * r
        u = h * w.float()
        dx = r * (u - f * (u * f).mean(-1, keepdim=True))
        return dx.to(x.dtype), (h * f).sum((0, 1, 2)).to(w.dtype)

    with torch.no_grad():
        y = [forward(x[0], w[0]), forward(x[1], w[1])]
        (dq, dwq), (dk, dwk) = backward(x[0], w[0], g[0]), backward(x[1], w[1], g[1])
    return y + [dq, dk, dwq, dwk]


def _append_plain(s):
    cos, sin = (t.unsqueeze(1) for t in _angles(s["positions"], s))
    K, V = s["k_pages"][0], s["v_pages"][0]
    page = K.shape[2]
    at, slot = s["slots"] // page, s["slots"] % page
    q, k = s["q"].float(), s["k"].float()
    K[at, :, slot] = _rotated(k * _root(k) * s["w"][1].float(), cos, sin, s["interleaved"]).to(K.dtype)
    V[at, :, slot] = s["v"]
    return [_rotated(q * _root(q) * s["w"][0].float(), cos, sin, s["interleaved"]).to(K.dtype), K, V]


def _tree_plain(s):
    q, table, starts, lengths = s["q"], s["table"].long(), s["starts"].long(), s["lengths"].long()
    S, KV, d, G, n = table.shape[0], s["KV"], s["d"], s["H"] // s["KV"], s["max_new"]
    keys, values = (p[0][table].permute(0, 2, 1, 3, 4).reshape(S, KV, -1, d).float() for p in (s["k_pages"], s["v_pages"]))
    L = keys.shape[2]
    nth = torch.arange(n, device=q.device)
    new = starts[1:] - starts[:-1]
    rows = (starts[:-1, None] + nth).clamp(max=q.shape[0] - 1)
    x = q[rows].float().view(S, n, KV, G, d).permute(0, 2, 3, 1, 4).reshape(S, KV, G * n, d)
    score = torch.matmul(x, keys.transpose(2, 3).contiguous()).mul_(s["scale"]).view(S, KV, G, n, L)
    bits = (s["tree"][rows].unsqueeze(-1) >> torch.arange(64, device=q.device)) & 1          # [S, n, words, 64]
    bits = bits.flatten(2).bool()
    most = bits.shape[2]
    is_tree = (new <= most)[:, None, None]
    base, key = (lengths - new)[:, None, None], torch.arange(L, device=q.device)
    pos = base + torch.where(is_tree, bits.sum(-1, keepdim=True) - 1, nth[:, None])
    among = (key - base).expand(S, n, L)
    named = torch.gather(bits, 2, among.clamp(0, most - 1)) & (among < most)
    seen = torch.where(is_tree, (among < 0) | named, key <= base + nth[:, None]) & (key < lengths[:, None, None])
    if s["window"]:
        seen = seen & ((key > pos - s["window"]) | (is_tree & (among >= 0)))
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(S, KV, G * n, L), values).view(S, KV, G, n, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = (top + torch.log(total)).squeeze(-1)
    row = torch.arange(q.shape[0], device=q.device)
    seq = torch.searchsorted(starts, row, right=True) - 1
    at = row - starts[seq]
    return [out[seq, :, :, at].reshape(-1, s["H"], d).to(q.dtype), lse[seq, :, :, at].reshape(-1, s["H"])]


def _plan_plain(s):
    """(There are pages and rows enough in these cases.)"""
    table, free, count, page = s["table"], s["free"], s["count"], s["page"]
    dev, (S, width) = table.device, table.shape
    new, old, column = s["new"].long(), s["lengths"].long(), torch.arange(width, device=dev)
    ended = new < 0
    # pages that go back: to the places of the stack behind its end, in their order
    back = (ended[:, None] & (table >= 0)).flatten()
    stack = torch.cat([free, free.new_zeros(1)])
    stack[torch.where(back, count.long() - 1 + back.cumsum(0), free.numel())] = table.flatten()
    free.copy_(stack[:-1])
    table.masked_fill_(ended[:, None], -1)
    n, base = new.clamp(min=0), torch.where(ended, 0, old)
    total = base + n
    wanted = ((column >= (base // page)[:, None]) & (column < ((total + page - 1) // page)[:, None]) & (table < 0)).flatten()
    left = count.long() + back.sum()
    got = free[(left - wanted.cumsum(0)).clamp(min=0)]
    table.copy_(torch.where(wanted, got, table.flatten()).view(S, width))
    count.copy_(left - wanted.sum())
    starts = torch.cat([n.new_zeros(1), n.cumsum(0)])
    row = torch.arange(s["rows"], device=dev)
    seq = (torch.searchsorted(starts, row, right=True) - 1).clamp(max=S - 1)
    there = row < starts[-1]
    nth = torch.where(there, row - starts[seq], 0)
    place = base[seq] + nth
    at = table[seq, (place // page).clamp(max=width - 1)].long()
    slots = torch.where(there, at * page + place % page, -1)
    out = [starts.int(), total.int(), slots]
    if s["parents"] is None:
        return out + [torch.where(there, place, -1), table, free, count]
    # the branch of every token: parents of parents, twice as far each time
    W, most = s["words"], s["parents"].shape[1]
    token = torch.arange(most, device=dev)
    up = torch.where((s["parents"] >= 0) & (s["parents"] < token), s["parents"].long(), most)
    up = torch.cat([up, torch.full((S, 1), most, device=dev)], 1)
    sees = torch.cat([torch.eye(most, dtype=torch.bool, device=dev), torch.zeros(1, most, dtype=torch.bool, device=dev)]).expand(S, most + 1, most)
    for _ in range(max(1, (most - 1).bit_length())):
        sees = sees | torch.gather(sees, 1, up[:, :, None].expand(S, most + 1, most))
        up = torch.gather(up, 1, up)
    tree = (there & (n[seq] <= 64 * W))[:, None]
    sees = sees[seq, nth.clamp(max=most - 1)] & tree
    named = torch.cat([sees, torch.zeros(row.numel(), 64 * W - most, dtype=torch.bool, device=dev)], 1) if most < 64 * W else sees
    masks = (named.view(-1, W, 64).long() << torch.arange(64, device=dev)).sum(-1)
    at = torch.where(tree[:, 0], base[seq] + sees.sum(-1) - 1, place)
    return out + [torch.where(there, at, -1), masks, table, free, count]


def _keep_plain(s):
    page, starts = s["k_pages"][0].shape[2], s["starts"].long()
    base = s["lengths"].long() - (starts[1:] - starts[:-1])
    kept, j = s["kept"].long(), torch.arange(s["kept"].shape[1], device=starts.device)
    some = j < s["counts"][:, None]                             # (behind the last kept one: the first one's move again)
    frm, to = base[:, None] + torch.where(some, kept, kept[:, :1]), base[:, None] + torch.where(some, j, 0)
    place = lambda p: (torch.gather(s["table"].long(), 1, p // page), p % page)  # noqa: E731
    (fp, fr), (tp, tr) = place(frm), place(to)
    for pages in s["k_pages"] + s["v_pages"]:
        pages[tp, :, tr] = pages[fp, :, fr]
    return [(base + s["counts"]).int()] + s["k_pages"] + s["v_pages"]


# ------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    return {"norm": _exact_norm, "append": _exact_append, "tree": _exact_tree, "keep": _exact_keep}[case["kind"]](case, seed, s)


def _exact_rotation(x, positions, s):
    """Column pairs as complex numbers, times amplitude x e^(i angle)."""
    n = s["turns"].numel()
    i = torch.arange(0, 2 * n, 2, device="cuda") if s["interleaved"] else torch.arange(n, device="cuda")
    j = i + 1 if s["interleaved"] else i + n
    angle = torch.remainder(positions.double()[..., None] * s["turns"], 1.0) * (2 * math.pi)
    z = torch.complex(x[..., i], x[..., j]) * torch.polar(torch.full_like(angle, s["amplitude"]), angle)
    return x.index_copy(-1, i, z.real).index_copy(-1, j, z.imag)


def _exact_normed(x, w):
    return x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt() * w


def _exact_norm(c, seed, s):
    N = c["N"]
    at = s["positions"] if s["positions"] is not None else torch.arange(s["offset"], s["offset"] + N, device="cuda").expand(c["B"], N)
    ys, dxs, dws = [], [], []
    for x, w, g in zip(s["x"], s["w"], s["g"]):
        x, w = x.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
        y = _exact_rotation(_exact_normed(x, w), at[:, None], s)
        dx, dw = torch.autograd.grad(y, [x, w], g.double())
        ys.append(y.detach())
        dxs.append(dx)
        dws.append(dw)
    return ys + dxs + dws


def _exact_append(c, seed, s):
    K, V = s["k_pages"][0].double(), s["v_pages"][0].double()
    at = s["positions"][:, None]
    q = _exact_rotation(_exact_normed(s["q"].double(), s["w"][0].double()), at, s)
    k = _exact_rotation(_exact_normed(s["k"].double(), s["w"][1].double()), at, s)
    row = 0
    for i, (n, L) in enumerate(zip(_news(c), _lengths(c))):
        pos = torch.arange(L - n, L, device="cuda")
        pages = s["table"][i].long()[torch.div(pos, c["page"], rounding_mode="floor")]
        K[pages, :, pos % c["page"]] = k[row:row + n]
        V[pages, :, pos % c["page"]] = s["v"][row:row + n].double()
        row += n
    return [q, K, V]


def _exact_tree(c, seed, s):
    O = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(O.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, L, parents) in enumerate(zip(_news(c), _lengths(c), _trees(c, seed, _news(c)))):
        pages = s["table"][i, :-(-L // c["page"])].long()
        branches = [_branch(parents, t) if parents else list(range(t + 1)) for t in range(n)]
        seen = torch.zeros(n, L, dtype=torch.bool)
        for t, b in enumerate(branches):
            first = max(0, L - n + len(b) - c["window"]) if c["window"] else 0
            seen[t, first:L - n] = True
            b = b if parents or not c["window"] else b[max(0, len(b) - c["window"]):]
            seen[t, [L - n + j for j in b]] = True
        seen = seen.cuda()
        for h in range(c["KV"]):
            K, V = (p[0][pages, h].reshape(-1, c["d"])[:L].double() for p in (s["k_pages"], s["v_pages"]))
            for j in range(h * (c["H"] // c["KV"]), (h + 1) * (c["H"] // c["KV"])):
                z = (s["q"][at:at + n, j].double() @ K.t().contiguous()) * s["scale"]
                z = z.masked_fill(~seen, -math.inf)
                lse[at:at + n, j] = torch.logsumexp(z, -1)
                O[at:at + n, j] = torch.softmax(z, -1) @ V
        at += n
    return [O, lse]


def _exact_keep(c, seed, s):
    pools = [p.double() for p in s["k_pages"] + s["v_pages"]]
    kept, counts, table = s["kept"].tolist(), s["counts"].tolist(), s["table"].tolist()
    frm, to, lengths = [], [], []
    for i, (n, L) in enumerate(zip(_news(c), _lengths(c))):
        frm += [(table[i][p // c["page"]], p % c["page"]) for p in (L - n + t for t in kept[i][:counts[i]])]
        to += [(table[i][p // c["page"]], p % c["page"]) for p in range(L - n, L - n + counts[i])]
        lengths.append(L - n + counts[i])
    (fp, fr), (tp, tr) = (torch.tensor(list(zip(*v)), device="cuda") for v in (frm, to))
    for p in pools:
        p[tp, :, tr] = p[fp, :, fr].clone()
    return [torch.tensor(lengths, dtype=torch.int32, device="cuda")] + pools
