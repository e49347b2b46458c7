"""Appending to a paged cache and attention over it, against 64 bits: lengths from none to long, odd groups and sizes, masks that leave rows
empty, values that must not matter, pages that are none, streams, captured replays, shards of a sequence."""
import numpy as np
import pytest
import torch

from paged_util import Batch, check_rotation, default_turns, f64, rotation
from paper_2403_09347_amd import binding as B
from paper_2403_09347_amd.harness import PagedWalk, RingWalk
from paper_2403_09347_amd.paged import burst_cache_append, burst_paged_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def attend(b, **kw):
    return burst_paged_attention(b.q, *b.args(), **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [128, 64, 96, 80, 32, 8])
def test_single_tokens_of_all_lengths(dtype, d):
    lengths = [1, 0, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 500, 1025]
    b = Batch(lengths, [1] * len(lengths), 4, 2, d, dtype=dtype, seed=d)
    O, lse = attend(b, max_new=1)
    b.check(O, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,KV", [(1, 1), (6, 2), (7, 1), (16, 1), (17, 1), (40, 2), (8, 8), (33, 1)])
@pytest.mark.parametrize("new", [1, 3, 50])
def test_groups(dtype, H, KV, new):
    b = Batch([70, 300, 5], [new, min(new, 2), 1], H, KV, 64, page=32, dtype=dtype, seed=H + new)
    O, lse = attend(b)
    b.check(O, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_groups_of_more_heads_than_a_block_has_rows(dtype):
    b = Batch([90, 300], [2, 1], 150, 1, 32, dtype=dtype, seed=1)
    for max_new in (0, 2):
        O, lse = attend(b, max_new=max_new)
        b.check(O, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_new_tokens_than_the_caller_said(dtype):
    """max_new chooses the kernel: one that is too small changes no result beyond rounding."""
    b = Batch([300, 70, 5], [45, 1, 5], 4, 2, 64, dtype=dtype)
    O, lse = attend(b, max_new=1)
    b.check(O, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
def test_a_cache_without_pages(dtype, new):
    b = Batch([100], [new], 4, 2, 64, dtype=dtype)
    none = b.k_pages[:0].contiguous()
    O, lse = burst_paged_attention(b.q, none, none, b.table, b.lengths, b.starts)
    assert (O == 0).all() and torch.isneginf(lse).all()
    O, lse = burst_paged_attention(b.q, b.k_pages, b.v_pages, b.table[:, :0], b.lengths, b.starts)
    assert (O == 0).all() and torch.isneginf(lse).all()
    burst_cache_append(b.k, b.v, none, none.clone(), b.table, b.lengths, b.starts)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,pool,packed", [(16, "head", False), (16, "seq", True), (32, "seq", False), (64, "head", True), (128, "seq", True), (1024, "head", False)])
@pytest.mark.parametrize("d", [128, 64])
def test_chunks_and_layouts(dtype, page, pool, packed, d):
    b = Batch([400, 200, 64, 333, 1], [37, 200, 64, 1, 1], 8, 2, d, page=page, dtype=dtype, seed=page, pool=pool, packed=packed)
    O, lse = attend(b)
    b.check(O, lse)
    again = attend(b, max_new=200)
    assert torch.equal(O, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 65, 200, 1 << 40])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(dtype, window, causal):
    b = Batch([500, 130, 90, 17], [1, 130, 40, 2], 4, 2, 96, dtype=dtype, seed=window % 1000)
    O, lse = attend(b, causal=causal, window=window)
    b.check(O, lse, causal, window)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_all_keys_visible(dtype):
    b = Batch([500, 130, 0, 17], [1, 130, 0, 2], 4, 1, 128, dtype=dtype)
    O, lse = attend(b, causal=False)
    b.check(O, lse, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_without_a_position_see_nothing(dtype):
    """More new tokens than the sequence is long: the first ones are before its start.  No tokens at all, no sequences."""
    b = Batch([10, 0, 40], [30, 5, 40], 2, 1, 64, dtype=dtype)
    O, lse = attend(b)
    b.check(O, lse)
    assert torch.isneginf(lse[:20]).all() and (O[:20] == 0).all() and torch.isneginf(lse[30:35]).all()
    e = Batch([10, 20], [0, 0], 2, 1, 64, dtype=dtype)
    assert attend(e)[0].shape == (0, 2, 64)
    n = burst_paged_attention(b.q, b.k_pages, b.v_pages, b.table[:0], b.lengths[:0], b.starts[:1])
    assert n[0].shape == b.q.shape


@pytest.mark.parametrize("new", [1, 20])
def test_rows_behind_the_last_sequence_are_left(new):
    b = Batch([100, 50], [new, 1], 4, 2, 64, spare_rows=9)
    out, lse = torch.full_like(b.q, 7.0), torch.full((b.q.shape[0], 4), 7.0, device=DEV)
    O, l = attend(b, out=out, lse=lse)
    assert O is out or O.data_ptr() == out.data_ptr()
    b.check(O, l)
    assert (out[new + 1:] == 7).all() and (lse[new + 1:] == 7).all()


def test_outputs_of_other_types_and_layouts():
    b = Batch([100, 50, 700], [30, 1, 2], 4, 2, 64)
    O, lse = attend(b)
    wide = torch.full((33, 6, 64), 9.0, device=DEV)
    O32, l32 = attend(b, out=wide[:, 1:5])
    assert torch.equal(O32.to(BF16), O) and torch.equal(l32, lse) and (wide[:, 0] == 9).all() and (wide[:, 5] == 9).all()
    b.check(O32, l32)
    narrow = torch.empty(4, 33, 64, dtype=BF16, device=DEV).transpose(0, 1)
    assert torch.equal(attend(b, out=narrow)[0], O)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("new", [1, 40])
def test_hidden_values_do_not_matter(dtype, value, new):
    """Non-finite values behind a sequence's end, in pages of nobody, after a token's position and before its window."""
    b = Batch([100, 203, 64], [new, new, 1], 4, 2, 128, dtype=dtype, seed=4)
    for i, L in enumerate(b.lengths_list):
        if L % 16:
            last = int(b.table[i, (L - 1) // 16])
            b.k_pages[last, :, L % 16:] = value
            b.v_pages[last, :, L % 16:] = value
    for f in b.free:
        b.k_pages[f] = value
        b.v_pages[f] = value
    O, lse = attend(b)
    b.check(O, lse)
    at = lambda s, p: (int(b.table[s, p // 16]), slice(None), p % 16)
    for p in (0, 3, 100):                                     # before the windows of all tokens of sequence 1
        b.k_pages[at(1, p)], b.v_pages[at(1, p)] = value, value
    O, lse = attend(b, window=60)
    b.check(O, lse, window=60)
    if new > 1:                                               # the last key: its own token sees it, the others do not
        c = Batch([100, 64], [new, 1], 4, 2, 128, dtype=dtype, seed=5)
        page, _, row = int(c.table[0, 99 // 16]), 0, 99 % 16
        clean = attend(c)
        c.v_pages[page, :, row] = value
        O, lse = attend(c)
        keep = [i for i in range(new + 1) if i != new - 1]
        O_ref, _, O_err, _ = c_reference(c, clean)
        assert np.all(np.abs(f64(O)[keep] - O_ref[keep]) <= 2 * O_err[keep])
        assert not torch.isfinite(O[new - 1]).any()


def c_reference(c, clean):
    """Values and bounds of a batch whose reference cannot be taken any more: from its run before."""
    O = f64(clean[0])
    err = np.abs(O) * 2.0 ** -6 + 2.0 ** -6
    return O, None, err, None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
def test_visible_infinities(dtype, new):
    b = Batch([100], [new], 2, 2, 64, dtype=dtype)
    page = int(b.table[0, 0])
    b.v_pages[page, 0, 3, 5] = float("inf")
    O, lse = attend(b)
    assert torch.isinf(O[:, 0, 5]).all() and torch.isfinite(O[:, 0, :5]).all() and torch.isfinite(O[:, 1]).all() and torch.isfinite(lse).all()
    b.k_pages[page, 1, 2] = float("nan")
    O, lse = attend(b)
    assert torch.isnan(O[:, 1]).all() and torch.isnan(lse[:, 1]).all() and torch.isfinite(lse[:, 0]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
def test_pages_that_are_none_hold_no_keys(dtype, new):
    b = Batch([200, 90], [new, new], 4, 2, 64, dtype=dtype)
    b.table[0, 1], b.table[0, 5], b.table[1, 0] = -1, b.k_pages.shape[0], 1 << 30
    O, lse = attend(b)
    b.check(O, lse)
    b.table[:] = -7
    O, lse = attend(b)
    assert torch.isneginf(lse).all() and (O == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_arrays_that_hold_anything(dtype):
    """Nothing is written outside the outputs whatever the three arrays say (their arithmetic is tested on the host)."""
    b = Batch([200, 90, 33], [20, 1, 5], 4, 2, 64, dtype=dtype)
    guard = torch.full((26 + 20, 4, 64), 5.0, dtype=dtype, device=DEV)
    lse = torch.full((26 + 20, 4), 5.0, device=DEV)
    for lengths, starts in (([1 << 30, -5, 1000], [0, 20, 21, 26]), ([200, 90, 33], [-3, 50, 10, 1 << 30]), ([7, 7, 7], [26, 0, 0, -1])):
        b.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        b.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        attend(b, out=guard[10:36], lse=lse[10:36])
        assert (guard[:10] == 5).all() and (guard[36:] == 5).all() and (lse[:10] == 5).all() and (lse[36:] == 5).all()
        k0 = b.k_pages.clone()
        burst_cache_append(b.k, b.v, *b.args(), turns=default_turns(64))
        used = set(b.table.flatten().tolist())
        for f in set(range(b.k_pages.shape[0])) - used:
            assert torch.equal(k0[f], b.k_pages[f])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths,news,H,KV", [([5000], [1], 8, 2), ([5000], [1], 4, 4), ([3000, 1, 700, 20, 2500], [1, 1, 1, 1, 1], 4, 1),
                                               ([3000, 70, 700, 2500], [64, 70, 1, 3], 8, 1), ([2000], [700], 2, 1)])
def test_long_caches_are_cut_into_runs(dtype, lengths, news, H, KV):
    b = Batch(lengths, news, H, KV, 128, page=64, dtype=dtype, seed=9)
    O, lse = attend(b)
    b.check(O, lse)
    for _ in range(2):
        again = attend(b)
        assert torch.equal(O, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("sequences", [65, 200])
def test_many_sequences(sequences):
    rng = np.random.default_rng(sequences)
    lengths = rng.integers(0, 120, sequences).tolist()
    for news in ([min(1, L) for L in lengths], [min(int(rng.integers(0, 40)), L) for L in lengths]):
        b = Batch(lengths, news, 4, 2, 64, seed=sequences)
        O, lse = attend(b)
        b.check(O, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("size", [30.0, 1e4])
def test_large_scores(dtype, new, size):
    b = Batch([300, 90], [new, new], 4, 2, 64, dtype=dtype, scale_qk=size)
    O, lse = attend(b)
    if size < 100:
        b.check(O, lse)
    assert torch.isfinite(O).all() and torch.isfinite(lse).all()


def test_a_cache_beyond_32_bit_offsets():
    """A pool of 2^31 elements and more, whose used pages are its last ones."""
    page, KV, d, L = 1024, 8, 128, 3000
    pages = (1 << 31) // (page * KV * d) + 4
    k_pages, v_pages = (torch.zeros(pages, KV, page, d, dtype=BF16, device=DEV) for _ in range(2))
    assert k_pages.numel() > 1 << 31
    for new in (1, 70):
        b = Batch([L], [new], 16, KV, d, page=page, seed=new)
        for i in range(-(-L // page)):
            k_pages[pages - 1 - i], v_pages[pages - 1 - i] = b.k_pages[int(b.table[0, i])], b.v_pages[int(b.table[0, i])]
        want = attend(b)
        table = torch.arange(pages - 1, pages - 4, -1, dtype=torch.int32, device=DEV).view(1, 3)
        got = burst_paged_attention(b.q, k_pages, v_pages, table, b.lengths, b.starts)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        burst_cache_append(b.k, b.v, k_pages, v_pages, table, b.lengths, b.starts)
        assert torch.equal(k_pages[pages - 3, :, (L - 1) % page], b.k[-1]) and torch.equal(v_pages[pages - 3, :, (L - 1) % page], b.v[-1])


def expected_pages(b, turns, interleaved, amplitude, offsets=None):
    """Where the new tokens go: {(page, row): token}."""
    return {(int(b.table[s, p // b.page]), p % b.page): (i, p + (0 if offsets is None else offsets[s]))
            for i, (s, p) in enumerate(b.positions()) if p >= 0 and 0 <= int(b.table[s, p // b.page]) < b.k_pages.shape[0]}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pool,packed", [("head", False), ("seq", True)])
@pytest.mark.parametrize("d,dims,interleaved", [(128, 128, False), (64, 32, True), (80, 40, False), (96, 0, False), (32, 32, True)])
def test_append(dtype, pool, packed, d, dims, interleaved):
    b = Batch([100, 17, 1, 40, 3], [30, 1, 1, 40, 0], 6, 2, d, dtype=dtype, pool=pool, packed=packed, spare_rows=3, seed=d)
    b.table[3, 1] = -1                                        # a page that is none: its tokens are left out
    k0, v0 = b.k_pages.clone(), b.v_pages.clone()
    turns = default_turns(dims) if dims else None
    offsets = [1000, 0, 7, 1 << 33, 3]
    got = burst_cache_append(b.k, b.v, *b.args(), q=b.q if dims else None, turns=turns, interleaved=interleaved, amplitude=1.5,
                             offsets=torch.tensor(offsets, device=DEV))
    if dims:
        pos = np.array([p + offsets[s] for s, p in b.positions()])
        T = len(pos)
        check_rotation("q", got[:T], b.q[:T], pos[:, None], f64(turns), interleaved, 1.5)
    else:
        assert got is None
    want = expected_pages(b, turns, interleaved, 1.5, offsets)
    touched = torch.zeros(b.k_pages.shape[0], b.page, dtype=torch.bool)
    for (page, row), (i, p) in want.items():
        touched[page, row] = True
        assert torch.equal(b.v_pages[page, :, row], b.v[i])
        if dims:
            check_rotation("k", b.k_pages[page, :, row], b.k[i], np.array([p]), f64(turns), interleaved, 1.5)
        else:
            assert torch.equal(b.k_pages[page, :, row], b.k[i])
    left = ~touched.to(DEV)[:, None, :, None].expand_as(b.k_pages)
    assert torch.equal(b.k_pages[left], k0[left]) and torch.equal(b.v_pages[left], v0[left])


def test_append_of_nothing_and_of_tokens_without_a_position():
    b = Batch([0, 10], [0, 0], 2, 1, 64)
    k0 = b.k_pages.clone()
    assert burst_cache_append(b.k, b.v, *b.args()) is None
    c = Batch([2, 5], [6, 5], 2, 1, 64, spare_rows=2)
    q = burst_cache_append(c.k, c.v, *c.args(), q=c.q, turns=default_turns(64))
    assert torch.equal(k0, b.k_pages) and q.shape == c.q.shape
    check_rotation("q", q[4:11], c.q[4:11], np.array([0, 1, 0, 1, 2, 3, 4])[:, None], f64(default_turns(64)))
    assert torch.equal(c.v_pages[int(c.table[0, 0]), :, 1], c.v[5])


def serving(dtype, steps, H=4, KV=2, d=64, page=16, seed=3):
    """Prompts of two sequences, then single tokens: the batches of each step, sharing one cache."""
    gen = torch.Generator().manual_seed(seed)
    total = [37, 90]
    rand = lambda *s: torch.randn(s, generator=gen).to(dtype).to(DEV)
    tokens = [{n: rand(L + steps, h, d) for n, h in (("q", H), ("k", KV), ("v", KV))} for L in total]
    pages = 20
    pool = [torch.full((pages, KV, page, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    table = torch.randperm(pages, generator=gen)[:16].view(2, 8).to(torch.int32).to(DEV)
    return tokens, total, pool, table


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_served_sequence_is_the_whole_sequence(dtype):
    """Prompt and single tokens through PagedWalk, against the rotated sequence in 64 bits; the cache starts as NaN."""
    steps, d = 5, 64
    tokens, total, pool, table = serving(dtype, steps)
    turns = default_turns(d)
    walk = PagedWalk(*pool, d ** -0.5, turns)
    done = [0, 0]
    got = [[], []]
    for step in range(steps + 1):
        news = total if step == 0 else [1, 1]
        take = lambda n: torch.cat([tokens[s][n][done[s]:done[s] + news[s]] for s in range(2)])
        lengths = torch.tensor([done[s] + news[s] for s in range(2)], dtype=torch.int32, device=DEV)
        starts = torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device=DEV)
        O, lse = walk.step(take("q"), take("k"), take("v"), table, lengths, starts, max_new=max(news))
        for s, part in enumerate(O.split(news)):
            got[s].append(part)
            done[s] += news[s]
    # q and k are rounded once more after their rotation: relative 2^-8 (2^-24) of either, on scores of at most 12 here
    tol = (2.0 ** -8 + 2 * 12 * 2.0 ** -8) if dtype == BF16 else 1e-4
    for s in range(2):
        n = done[s]
        see = np.tril(np.ones((n, n), bool))
        out = f64(torch.cat(got[s]))
        for h in range(4):
            q = rotation(f64(tokens[s]["q"][:, h]), np.arange(n), f64(turns))[0]
            k = rotation(f64(tokens[s]["k"][:, h // 2]), np.arange(n), f64(turns))[0]
            v = f64(tokens[s]["v"][:, h // 2])
            z = np.where(see, q @ k.T * d ** -0.5, -np.inf)
            p = np.exp(z - z.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            assert np.abs(z[see]).max() < 12
            assert np.all(np.abs(out[:, h] - p @ v) <= tol * (p @ np.abs(v)) + 1e-6)


def test_a_walk_and_the_cache_agree():
    """The keys of a walk's chunk, put into pages, and the paged attention of the walk's queries."""
    Q, K, V = (torch.randn(1, h, 200, 128, device=DEV, generator=torch.Generator(DEV).manual_seed(h)).to(BF16) for h in (8, 2, 2))
    walk = RingWalk(Q, 128 ** -0.5, True, 0, kv_heads=2)
    O, lse = walk.forward([K], [V], [0])
    pages = [torch.zeros(13, 2, 16, 128, dtype=BF16, device=DEV) for _ in range(2)]
    table = torch.arange(13, dtype=torch.int32, device=DEV).view(1, 13)
    lengths, starts = torch.tensor([200], dtype=torch.int32, device=DEV), torch.tensor([0, 200], dtype=torch.int32, device=DEV)
    burst_cache_append(K[0].transpose(0, 1), V[0].transpose(0, 1), *pages, table, lengths, starts)
    O2, lse2 = burst_paged_attention(Q[0].transpose(0, 1), *pages, table, lengths, starts)
    # (two roundings of P and of O each; values of size 4)
    assert (O2.transpose(0, 1) - O[0]).abs().max().item() <= 4 * 2.0 ** -6
    assert (lse2.t() - lse[0]).abs().max().item() <= 1e-2     # (the walk's l sums rounded probabilities)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 30])
def test_shards_of_a_sequence_are_joined_by_merge_state(dtype, new):
    """The last `new` tokens on the device that appends them, the others' keys all visible."""
    b = Batch([300], [new], 4, 2, 64, dtype=dtype)
    whole, lse = attend(b)
    part = [Batch([n], [new], 4, 2, 64, dtype=dtype) for n in (144, 156)]
    for p, first in zip(part, (0, 9)):
        p.q, p.k_pages, p.v_pages = b.q, b.k_pages, b.v_pages
        p.table = b.table[:, first:].contiguous()
    states = []
    for p, causal in zip(part, (False, True)):
        out = torch.empty(new, 4, 64, device=DEV)
        _, l = attend(p, causal=causal, out=out)
        states.append((out.view(1, 1, -1, 64), l.view(1, 1, -1).clone(), torch.ones(1, 1, new * 4, device=DEV)))
    params = B.params(1, 1, new * 4, 0, 64, "f32", 1.0)
    B.burst_merge_state(*states[0], *states[1], params)
    O, m, l = states[0]
    b.check((O / l[..., None]).view(new, 4, 64).to(dtype), (m + l.log()).view(new, 4))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streams_and_two_calls_at_once(dtype):
    bs = [Batch([900, 300], [1, 40], 8, 2, 64, dtype=dtype, seed=s) for s in range(3)]
    want = [attend(b) for b in bs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in bs]
    got = []
    for b, st in zip(bs, streams):
        with torch.cuda.stream(st):
            got.append([attend(b) for _ in range(3)])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for x in g:
            assert torch.equal(x[0], w[0]) and torch.equal(x[1], w[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("max_new", [1, 60])
def test_a_captured_step_is_replayed_with_other_sequences(dtype, max_new):
    """Appending and attention recorded once; every replay has other tokens, lengths and tables, with eager work in between."""
    S, H, KV, d, page, width = 3, 4, 2, 64, 16, 40
    rows = S * max_new
    gen = torch.Generator(DEV).manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen, device=DEV).to(dtype)
    pools = [rand(130, KV, page, d) for _ in range(2)]
    walk = PagedWalk(*pools, d ** -0.5, default_turns(d))
    q, k, v = rand(rows, H, d), rand(rows, KV, d), rand(rows, KV, d)
    table = torch.randperm(130, generator=gen, device=DEV)[:S * width].view(S, width).to(torch.int32)
    lengths = torch.full((S,), max_new, dtype=torch.int32, device=DEV)
    starts = torch.arange(S + 1, dtype=torch.int32, device=DEV) * max_new
    walk.step(q, k, v, table, lengths, starts, max_new)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):                                        # two graphs of the same step, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(walk.step(q, k, v, table, lengths, starts, max_new))
        graphs.append(g)
    for i, (L, n) in enumerate([((600, 17, max_new), (1, 1, max_new)), ((1, 640, 0), (1, 1, 0)), ((300, 300, 300), (max_new,) * 3), ((64, 65, 63), (0, 1, 1))]):
        q.copy_(rand(rows, H, d)); k.copy_(rand(rows, KV, d)); v.copy_(rand(rows, KV, d))
        table.copy_(torch.randperm(130, generator=gen, device=DEV)[:S * width].view(S, width))
        lengths.copy_(torch.tensor(L, dtype=torch.int32))
        starts.copy_(torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32))
        T = sum(n)
        before = [p.clone() for p in pools]
        eager = walk.step(q, k, v, table, lengths, starts, max_new)
        after = [p.clone() for p in pools]
        for p, x in zip(pools, before):
            p.copy_(x)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, x) for p, x in zip(pools, after))
        assert torch.equal(outs[i % 2][0][:T], eager[0][:T]) and torch.equal(outs[i % 2][1][:T], eager[1][:T])


def test_nothing_is_written_outside_the_workspace_and_outputs():
    """The C call with a workspace of exactly the size that it asks for, between guards."""
    for dtype, news in ((BF16, [1, 1]), (BF16, [70, 20]), (F32, [1, 1]), (F32, [70, 20])):
        b = Batch([900, 500], news, 4, 2, 64, dtype=dtype)
        p = B.paged_params(sum(news), 4, 2, 64, dtype, b.k_pages, b.table, b.lengths, b.starts, b.scale)
        need = B.burst_paged_workspace_bytes(p)
        assert need > 0
        ws = torch.full((need + 8192,), 77, dtype=torch.uint8, device=DEV)
        O = torch.full((sum(news) + 8, 4, 64), 3.0, dtype=dtype, device=DEV)
        lse = torch.full((sum(news) + 8, 4), 3.0, device=DEV)
        B.burst_paged_fwd(b.q.contiguous(), b.k_pages, b.v_pages, O[4:-4], lse[4:-4], p, ws[4096:4096 + need])
        b.check(O[4:-4], lse[4:-4])
        assert (ws[:4096] == 77).all() and (ws[4096 + need:] == 77).all()
        assert (O[:4] == 3).all() and (O[-4:] == 3).all() and (lse[:4] == 3).all() and (lse[-4:] == 3).all()
        with pytest.raises(B.BurstError):
            B.burst_paged_fwd(b.q.contiguous(), b.k_pages, b.v_pages, O[4:-4], lse[4:-4], p, ws[4096:4096 + need - 16])


def test_random_batches():
    rng = np.random.default_rng(11)
    for i in range(40):
        S, KV = int(rng.integers(1, 7)), int(rng.choice([1, 2, 3]))
        H = KV * int(rng.choice([1, 2, 3, 4, 8]))
        d = int(rng.choice([8, 24, 32, 64, 72, 128]))
        lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(700), S))]
        news = [min(L, int(np.exp(rng.uniform(0, np.log(100))))) if rng.random() < 0.6 else min(L, 1) for L in lengths]
        dtype = BF16 if rng.random() < 0.6 else F32
        b = Batch(lengths, news, H, KV, d, page=int(rng.choice([16, 32, 256])), dtype=dtype, seed=i, pool=str(rng.choice(["head", "seq"])), packed=bool(rng.random() < 0.5))
        causal, window = bool(rng.random() < 0.8), int(rng.choice([0, 0, 5, 100]))
        O, lse = attend(b, causal=causal, window=window, max_new=max(news) if rng.random() < 0.5 else 0)
        b.check(O, lse, causal, window, name=f"case {i}: {lengths} {news} H {H} KV {KV} d {d} {dtype} {causal} {window}")


def test_tensors_that_do_not_fit_are_refused():
    b = Batch([20, 30], [2, 1], 4, 2, 64)
    t = dict(q=b.q, k_pages=b.k_pages, v_pages=b.v_pages, table=b.table, lengths=b.lengths, starts=b.starts)

    def refuses(call=burst_paged_attention, **kw):
        with pytest.raises((ValueError, B.BurstError)):
            call(**dict(t, **kw))
    refuses(q=b.q[:, :3])                                     # 3 heads over 2
    refuses(q=b.q[0])
    refuses(q=b.q.float())
    refuses(q=b.q.cpu())
    refuses(q=b.q.clone().requires_grad_(True))
    refuses(v_pages=b.v_pages[:-1])
    refuses(v_pages=b.v_pages.float())
    refuses(k_pages=b.k_pages[:, :, :7], v_pages=b.v_pages[:, :, :7])
    refuses(k_pages=b.k_pages.half(), v_pages=b.v_pages.half())
    refuses(k_pages=b.k_pages[..., ::2], v_pages=b.v_pages[..., ::2], q=b.q[..., ::2])
    refuses(table=b.table.long())
    refuses(table=b.table[:1])
    refuses(table=b.table.cpu())
    refuses(lengths=b.lengths[:1])
    refuses(starts=b.starts[:2])
    refuses(scale=0.0)
    refuses(window=-1)
    refuses(max_new=-1)
    refuses(out=torch.empty(3, 4, 32, dtype=BF16, device=DEV))
    refuses(out=torch.empty(3, 4, 64, dtype=torch.half, device=DEV))
    refuses(out=torch.empty(3, 4, 65, dtype=BF16, device=DEV)[..., 1:])
    refuses(lse=torch.empty(3, 4, dtype=BF16, device=DEV))
    a = dict(k=b.k, v=b.v, k_pages=b.k_pages, v_pages=b.v_pages, table=b.table, lengths=b.lengths, starts=b.starts)
    t.clear()
    t.update(a)
    refuses(burst_cache_append, k=b.k[:, :1])
    refuses(burst_cache_append, v=b.v[:2])
    refuses(burst_cache_append, q=b.q)                        # no turns
    refuses(burst_cache_append, turns=default_turns(64).float())
    refuses(burst_cache_append, turns=default_turns(66))
    refuses(burst_cache_append, q=b.q[:2], turns=default_turns(64))
    refuses(burst_cache_append, offsets=b.lengths)
    refuses(burst_cache_append, k=b.k.clone().requires_grad_(True))
    refuses(burst_cache_append, k_pages=b.k_pages.clone().requires_grad_(True))
    with torch.no_grad():
        burst_cache_append(**dict(a, k=b.k.clone().requires_grad_(True)))


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 70), (False, 0)])
def test_sequences_of_many_blocks(causal, window):
    """More than 64 blocks of 16 tokens in one sequence, few in the next."""
    b = Batch([1500, 40, 900], [1400, 40, 800], 8, 1, 32, seed=31)
    O, lse = attend(b, causal=causal, window=window)
    b.check(O, lse, causal, window)
    b = Batch([1200, 40], [1100, 2], 8, 1, 32, dtype=F32, seed=32)
    O, lse = attend(b, causal=causal, window=window)
    b.check(O, lse, causal, window)


@pytest.mark.parametrize("new", [1, 4096])
def test_starts_that_decrease(new):
    """The same rows in 32 sequences of 2^29 keys each would be more work than 32 bits count: nothing is done."""
    q = torch.ones(4096, 2, 64, dtype=BF16, device=DEV)
    none = torch.empty(0, 2, 1 << 26, 64, dtype=BF16, device=DEV)
    table = torch.full((64, 8), -1, dtype=torch.int32, device=DEV)
    lengths = torch.full((64,), 1 << 30, dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 4096] * 32 + [0], dtype=torch.int32, device=DEV)
    O, lse = torch.full_like(q, 5), torch.full((4096, 2), 5.0, device=DEV)
    burst_paged_attention(q, none, none, table, lengths, starts, out=O, lse=lse, max_new=new)
    assert (O == 5).all() and (lse == 5).all()


def test_expanded_pages_are_refused():
    b = Batch([20, 30], [2, 1], 4, 2, 64)
    for shape in ((1, 1, 1, 64), (1, 2, 16, 64), (6, 1, 16, 64), (6, 2, 1, 64)):
        p = torch.zeros(shape, dtype=BF16, device=DEV).expand(6, 2, 16, 64)
        with pytest.raises(ValueError, match="rows that lie in memory"):
            burst_paged_attention(b.q, p, p, b.table, b.lengths, b.starts)
        with pytest.raises(ValueError, match="rows that lie in memory"):
            burst_cache_append(b.k, b.v, p, p, b.table, b.lengths, b.starts)


@pytest.mark.parametrize("new", [1, 30])
def test_sequences_that_share_pages(new):
    """A common beginning lies in the same pages."""
    b = Batch([400, 300, 270], [new] * 3, 4, 2, 64, seed=33)
    b.table[1:, :10] = b.table[0, :10]
    O, lse = attend(b)
    b.check(O, lse)
