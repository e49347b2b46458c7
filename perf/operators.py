"""The operators beside the attention walks, as cases that can be timed: the rotation of queries and keys by their positions,
appending keys and values to a paged cache, and attention of new tokens over such a cache.

A case is a dict of plain values.
  kind    "rotary"  queries and keys rotated, and the gradients brought back (what a training step does on either side of the
                    attention): B, H, KV, N rows, d, dims (rotated columns), pairs ("half" / "interleaved"), factor (yarn, 1 = not
                    scaled), q_off (position of row 0), far (0, or positions drawn below it), layout
          "append"  new tokens of S sequences rotated and written to their pages, the queries rotated besides
          "attend"  attention of the new tokens of S sequences over their pages
  Both of a cache: S, H, KV, d, dtype, page (rows of a page), pool ("head": [pages, heads, rows, d]; "seq": [pages, rows, heads,
  d] seen with heads first), packed (the tokens' q, k, v are views of one projection); sequence lengths (with the new tokens)
  from len_lo to len_hi and new tokens from new_lo to new_hi, spread evenly over their logarithm by the whole number `mix`.
Values are N(0, 1), as everywhere in this repository (activations of a normalised layer)."""
import math
import random

import torch

own = False

_BASE = 10000.0


def _rotary(name=None, dtype="bf16", B=1, H=32, KV=32, N=4096, d=128, dims=128, pairs="half", factor=1.0, q_off=0, far=0, layout="head"):
    c = dict(kind="rotary", dtype=dtype, B=B, H=H, KV=KV, N=N, d=d, dims=dims, pairs=pairs, factor=factor, q_off=q_off, far=far, layout=layout)
    return dict(c, name=name) if name else c


def _cache(kind, name=None, dtype="bf16", S=1, H=32, KV=8, d=128, page=64, pool="head", packed=True, len_lo=4096, len_hi=4096, new_lo=1,
           new_hi=1, mix=1, window=0, dims=128, pairs="half", factor=1.0):
    c = dict(kind=kind, dtype=dtype, S=S, H=H, KV=KV, d=d, page=page, pool=pool, packed=packed, len_lo=len_lo, len_hi=len_hi,
             new_lo=new_lo, new_hi=new_hi, mix=mix)
    c.update(dict(dims=dims, pairs=pairs, factor=factor) if kind == "append" else dict(window=window))
    return dict(c, name=name) if name else c


def listed():
    return [
        # A training step's layer on the last rank of the benchmark's ring (32 heads, 32K tokens on 8 devices).
        _rotary("rotary_last_rank", q_off=7 * 4096),
        # Grouped heads in sequence-major activations, a context stretched four times, a length that is no multiple of anything.
        _rotary("rotary_grouped_scaled", KV=8, N=3001, factor=4.0, layout="seq"),
        # fp32, interleaved pairs in part of a head that is neither 64 nor 128 wide, positions up to a million.
        _rotary("rotary_f32_far_partial", dtype="f32", B=2, H=8, KV=8, N=777, d=80, dims=32, pairs="interleaved", far=1 << 20),
        # One token for each of four sequences: the call is over before the launch of the next one.
        _cache("append", "append_few_tokens", S=4, page=16, len_lo=100, len_hi=3000),
        # Prompts of different lengths, prefilled together into a cache that lies sequence-major.
        _cache("append", "append_prompts", S=7, pool="seq", len_lo=300, len_hi=4096, new_lo=300, new_hi=4096, dims=64, pairs="interleaved", factor=8.0),
        # One user, a long context, one token: the whole chip reads one sequence's cache.
        _cache("attend", "decode_one_long", len_lo=32768, len_hi=32768),
        # A batch as a server has it: lengths from a few tokens to 16K.
        _cache("attend", "decode_ragged_batch", S=64, page=16, len_lo=16, len_hi=16384),
        # fp32, every head with keys of its own, 64 wide, short contexts.
        _cache("attend", "decode_f32_heads", dtype="f32", S=8, H=8, KV=8, d=64, page=32, pool="seq", packed=False, len_lo=1, len_hi=2000),
        # A chunk of a long prompt.
        _cache("attend", "chunk_long_prompt", len_lo=32768, len_hi=32768, new_lo=2048, new_hi=2048),
        # Chunks of some prompts and single tokens of other sequences in one call.
        _cache("attend", "chunk_mixed_batch", S=12, H=32, KV=32, page=16, len_lo=600, len_hi=8000, new_lo=1, new_hi=512),
        # Sliding window, 64-wide heads, sequence-major cache.
        _cache("attend", "chunk_window_d64", S=4, H=16, KV=4, d=64, page=32, pool="seq", len_lo=3000, len_hi=9000, new_lo=300, new_hi=900, window=1024),
        # fp32 chunks of odd sizes, heads 96 wide.
        _cache("attend", "chunk_f32_ragged", dtype="f32", S=3, H=8, KV=2, d=96, page=16, len_lo=400, len_hi=1500, new_lo=30, new_hi=300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotary", "append", "attend", "attend", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([128, 128, 64, 64, 96, 80, 32])
        KV, group = rng.choice([1, 2, 4, 8, 8, 32]), rng.choice([1, 1, 2, 4, 4, 8])
        H = KV * group
        dims, pairs, factor = rng.choice([d, d, d // 2, 16]), rng.choice(["half", "half", "interleaved"]), rng.choice([1.0, 1.0, 4.0, 16.0])
        if kind == "rotary":
            far = rng.choice([0, 0, 1 << 20])
            c = _rotary(dtype=dtype, B=rng.choice([1, 1, 2, 3]), H=H, KV=KV, N=_log(rng, 16, 8192), d=d, dims=dims, pairs=pairs, factor=factor,
                        q_off=0 if far else rng.choice([0, rng.randrange(1 << 18)]), far=far, layout=rng.choice(["head", "seq"]))
        else:
            c = _cache(kind, dtype=dtype, S=_log(rng, 1, 64), H=H, KV=KV, d=d, page=rng.choice([16, 32, 64, 128]), pool=rng.choice(["head", "seq"]),
                       packed=rng.random() < 0.7, mix=rng.randrange(1 << 20))
            c["len_hi"] = _log(rng, 1, 32768 if kind == "attend" else 4096)
            c["len_lo"] = c["len_hi"] if rng.random() < 0.3 else _log(rng, 1, c["len_hi"])
            if kind == "append":
                c["new_hi"] = rng.choice([1, c["len_hi"]])
                c["new_lo"] = 1 if c["new_hi"] == 1 else c["len_lo"]
                c.update(dims=dims, pairs=pairs, factor=factor)
            else:
                c["new_hi"] = 1 if rng.random() < 0.5 else _log(rng, 2, min(2048, max(2, c["len_hi"])))
                c["new_lo"] = 1 if rng.random() < 0.5 else _log(rng, 1, c["new_hi"])
                if rng.random() < 0.25:
                    c["window"] = _log(rng, 16, 8192)
        if _affordable(c):
            return c


def _affordable(c):
    """No more than the largest listed case costs, the plain form's padding included."""
    w = work(c)
    if c["kind"] == "rotary":
        return 1e6 < w["bytes"] < 6e8
    n, L = max(_news(c)), max(_lengths(c))
    if c["kind"] == "append":
        return w["bytes"] < 4e8
    return c["S"] * c["H"] * n * L <= 32 * 2048 * 32768 and c["S"] * c["KV"] * L * c["d"] <= 64 * 8 * 16384 * 128 and w["flops"] < 1.2e12


def _spread(c, lo, hi, salt):
    rng = random.Random(2 * c["mix"] + salt)
    at = [i / max(1, c["S"] - 1) for i in range(c["S"])]
    rng.shuffle(at)
    return [int(round(math.exp(math.log(lo) + x * (math.log(hi) - math.log(lo))))) for x in at]


def _lengths(c):
    return _spread(c, c["len_lo"], c["len_hi"], 0)


def _news(c):
    """New tokens of each sequence: its last ones."""
    if (c["new_lo"], c["new_hi"]) == (c["len_lo"], c["len_hi"]):
        return _lengths(c)
    return [min(n, L) for n, L in zip(_spread(c, c["new_lo"], c["new_hi"], 1), _lengths(c))]


def work(case):
    """Every input read once and every output written once.  attend: the keys and values that some new token sees, 4 d operations a
    visible pair and query head; the rotation: 6 operations a pair of columns (its angle is shared by all heads)."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        n = c["B"] * (c["H"] + c["KV"]) * c["N"]
        return {"bytes": 4.0 * n * c["d"] * e, "flops": 6.0 * n * c["dims"]}
    T = sum(_news(c))
    if c["kind"] == "append":
        return {"bytes": 2.0 * T * (c["H"] + 2 * c["KV"]) * c["d"] * e, "flops": 3.0 * T * (c["H"] + c["KV"]) * c["dims"]}
    keys = pairs = 0
    for n, L in zip(_news(c), _lengths(c)):
        w = c["window"] or L
        keys += min(L, w + n - 1)
        pairs += sum(min(w, p + 1) for p in range(L - n, L))
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


def prepare(case, seed):
    c, dev = case, "cuda"
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(dt)  # noqa: E731
    s = {k: c[k] for k in ("kind", "d", "H", "KV")}
    if c["kind"] != "attend":
        s.update(turns=_turns(c["dims"], c["factor"]).to(dev), interleaved=c["pairs"] == "interleaved", amplitude=_amplitude(c["factor"]))
    if c["kind"] == "rotary":
        def rows(heads):
            if c["layout"] == "seq":
                return rand(c["B"], c["N"], heads, c["d"]).transpose(1, 2)
            return rand(c["B"], heads, c["N"], c["d"])
        s["x"] = [rows(h).requires_grad_(True) for h in (c["H"], c["KV"])]
        s["g"] = [rows(h) for h in (c["H"], c["KV"])]
        s["offset"] = c["q_off"]
        s["positions"] = torch.randint(c["far"], (c["B"], c["N"]), generator=gen, device=dev) if c["far"] else None
        return s
    news, lengths = _news(c), _lengths(c)
    T, S, page = sum(news), c["S"], c["page"]
    if c["packed"]:
        qkv = rand(T, c["H"] + 2 * c["KV"], c["d"])
        s["q"], s["k"], s["v"] = qkv.split([c["H"], c["KV"], c["KV"]], dim=1)
    else:
        s["q"], s["k"], s["v"] = (rand(T, h, c["d"]) for h in (c["H"], c["KV"], c["KV"]))
    per = [-(-L // page) for L in lengths]
    pages = sum(per) + 3
    pool = (lambda: rand(pages, page, c["KV"], c["d"]).transpose(1, 2)) if c["pool"] == "seq" else (lambda: rand(pages, c["KV"], page, c["d"]))
    s["k_pages"], s["v_pages"] = pool(), pool()
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu()
    table = torch.full((S, max(per)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    s.update(table=table.to(dev), lengths=torch.tensor(lengths, dtype=torch.int32, device=dev),
             starts=torch.tensor(starts, dtype=torch.int32, device=dev), max_new=max(news))
    if c["kind"] == "attend":
        s.update(scale=c["d"] ** -0.5, window=c["window"])
    return s


# ------------------------------------------------------------------------------- one pass
def run(state):
    s = state
    if own:
        return _run_own(s)
    return {"rotary": _rotary_plain, "append": _append_plain, "attend": _attend_plain}[s["kind"]](s)


def _run_own(s):
    if s["kind"] == "rotary":
        from paper_2403_09347_amd.rotary import burst_rotary
        y = burst_rotary(s["x"], s["turns"], offset=s["offset"], positions=s["positions"], interleaved=s["interleaved"], amplitude=s["amplitude"])
        return [t.detach() for t in y] + list(torch.autograd.grad(y, s["x"], s["g"]))
    from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention
    if s["kind"] == "append":
        q = burst_cache_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["starts"], q=s["q"], turns=s["turns"],
                               interleaved=s["interleaved"], amplitude=s["amplitude"])
        return [q, s["k_pages"], s["v_pages"]]
    return list(burst_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["starts"], scale=s["scale"],
                                      window=s["window"], max_new=s["max_new"]))


def _rotate(x, cos, sin, interleaved):
    """The first columns of x, in pairs, turned by the angles of cos and sin [..., pairs]; 32 bits, the type of x again at the end."""
    n = cos.shape[-1]
    f = x.float()
    a, b = (f[..., 0:2 * n:2], f[..., 1:2 * n:2]) if interleaved else (f[..., :n], f[..., n:2 * n])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, f[..., 2 * n:]], -1).to(x.dtype)


def _angles(positions, s):
    """cos and sin at the positions, computed in 64 bits, rounded to 32."""
    turn = positions.double().unsqueeze(-1) * s["turns"]
    a = (turn - turn.round()) * (2 * math.pi)
    return (torch.cos(a) * s["amplitude"]).float(), (torch.sin(a) * s["amplitude"]).float()


def _rotary_plain(s):
    x, g = s["x"], s["g"]
    at = s["positions"] if s["positions"] is not None else s["offset"] + torch.arange(x[0].shape[2], device=x[0].device).unsqueeze(0)
    cos, sin = (t.unsqueeze(1) for t in _angles(at, s))
    with torch.no_grad():
        return [_rotate(t, cos, sin, s["interleaved"]) for t in x] + [_rotate(t, cos, -sin, s["interleaved"]) for t in g]


def _owners(s):
    """Sequence, place in it and position of every new token."""
    T = s["q"].shape[0]
    row = torch.arange(T, device=s["q"].device)
    starts, lengths = s["starts"].long(), s["lengths"].long()
    seq = torch.searchsorted(starts, row, right=True) - 1
    nth = row - starts[seq]
    return seq, nth, lengths[seq] - (starts[seq + 1] - starts[seq]) + nth


def _append_plain(s):
    seq, _, pos = _owners(s)
    cos, sin = (t.unsqueeze(1) for t in _angles(pos, s))
    page = s["k_pages"].shape[2]
    at, slot = s["table"][seq, pos // page].long(), pos % page
    s["k_pages"][at, :, slot] = _rotate(s["k"], cos, sin, s["interleaved"])
    s["v_pages"][at, :, slot] = s["v"]
    return [_rotate(s["q"], cos, sin, s["interleaved"]), s["k_pages"], s["v_pages"]]


def _attend_plain(s):
    q, table, starts, lengths = s["q"], s["table"].long(), s["starts"].long(), s["lengths"].long()
    S, KV, d, G, n = table.shape[0], s["KV"], s["d"], s["H"] // s["KV"], s["max_new"]
    keys, values = (p[table].permute(0, 2, 1, 3, 4).reshape(S, KV, -1, d).float() for p in (s["k_pages"], s["v_pages"]))
    L = keys.shape[2]
    nth = torch.arange(n, device=q.device)
    new = starts[1:] - starts[:-1]
    rows = (starts[:-1, None] + nth).clamp(max=q.shape[0] - 1)
    x = q[rows].float().view(S, n, KV, G, d).permute(0, 2, 3, 1, 4).reshape(S, KV, G * n, d)
    score = torch.matmul(x, keys.transpose(2, 3).contiguous()).mul_(s["scale"]).view(S, KV, G, n, L)
    pos, key = (lengths - new)[:, None, None] + nth[:, None], torch.arange(L, device=q.device)
    hidden = (key > pos) | (key >= lengths[:, None, None])
    if s["window"]:
        hidden = hidden | (key <= pos - s["window"])
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(S, KV, G * n, L), values).view(S, KV, G, n, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = (top + torch.log(total)).squeeze(-1)
    seq, at, _ = _owners(s)
    return [out[seq, :, :, at].reshape(-1, s["H"], d).to(q.dtype), lse[seq, :, :, at].reshape(-1, s["H"])]


# ------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        if case["kind"] == "rotary":
            N = case["N"]
            at = s["positions"] if s["positions"] is not None else torch.arange(s["offset"], s["offset"] + N, device="cuda").expand(case["B"], N)
            turned = [_exact_rotation(t.detach(), at[:, None], s, 1) for t in s["x"]]
            return turned + [_exact_rotation(t, at[:, None], s, -1) for t in s["g"]]
        return (_exact_append if case["kind"] == "append" else _exact_attend)(case, s)


def _exact_rotation(x, positions, s, sign):
    """Column pairs as complex numbers, times amplitude x e^(i angle)."""
    n = s["turns"].numel()
    y = x.double().clone()
    first = slice(0, 2 * n, 2) if s["interleaved"] else slice(0, n)
    second = slice(1, 2 * n, 2) if s["interleaved"] else slice(n, 2 * n)
    angle = torch.remainder(positions.double()[..., None] * s["turns"], 1.0) * (2 * math.pi * sign)
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(angle, s["amplitude"]), angle)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(c, s):
    K, V = s["k_pages"].double(), s["v_pages"].double()
    q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, L) in enumerate(zip(_news(c), _lengths(c))):
        pos = torch.arange(L - n, L, device="cuda")
        k = _exact_rotation(s["k"][at:at + n], pos[:, None], s, 1)
        q[at:at + n] = _exact_rotation(s["q"][at:at + n], pos[:, None], s, 1)
        pages = s["table"][i].long()[torch.div(pos, c["page"], rounding_mode="floor")]
        K[pages, :, pos % c["page"]] = k
        V[pages, :, pos % c["page"]] = s["v"][at:at + n].double()
        at += n
    return [q, K, V]


def _exact_attend(c, s):
    O = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(O.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, L) in enumerate(zip(_news(c), _lengths(c))):
        pages = s["table"][i, :-(-L // c["page"])].long()
        pos, key = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")
        seen = key <= pos
        if c["window"]:
            seen = seen & (key > pos - c["window"])
        for h in range(c["KV"]):
            K, V = (p[pages, h].reshape(-1, c["d"])[:L].double() for p in (s["k_pages"], s["v_pages"]))
            for j in range(h * (c["H"] // c["KV"]), (h + 1) * (c["H"] // c["KV"])):
                z = (s["q"][at:at + n, j].double() @ K.t().contiguous()) * s["scale"]
                z = z.masked_fill(~seen, -math.inf)
                lse[at:at + n, j] = torch.logsumexp(z, -1)
                O[at:at + n, j] = torch.softmax(z, -1) @ V
        at += n
    return [O, lse]
