"""A cache of keys and values in pages, and attention of new tokens over it: what serves a sequence token by token (or a prompt
chunk by chunk) after, or instead of, the walks over resident chunks.  Marshalling is native (csrc/burst_torch.cpp), the
kernels are csrc/burst_rotary.hip, csrc/burst_norm.hip, csrc/burst_paged.hip and csrc/burst_plan.hip.

Several sequences at once: token tensors [rows, heads, d] hold the new tokens of sequence s in rows starts[s] .. starts[s + 1] - 1
(views of a packed projection are read in place); lengths[s] counts all tokens of the sequence, the new ones among them; position p of
it is row p % page of page table[s, p // page] of k_pages and v_pages [pages, kv_heads, page, d] (any strides with a contiguous last
dimension; page: a power of two, 16 or more).  table, lengths and starts are int32 tensors on the device and are read there, so
that a captured call can be replayed with other contents (they are not to change while a call runs); values outside their
ranges are cut to them, a page that is not one of the pages holds no keys, nor does a position behind the table's row (new tokens there are
not kept, and see the keys that are), and attention with starts that decrease writes nothing.

A step of serving with drafted tokens: burst_cache_plan (once), burst_cache_append and burst_paged_attention (in every layer), and when it is
known which branch of every tree is right, burst_cache_keep (once, for all layers)."""
from typing import NamedTuple, Optional

import torch

from . import binding as B


def burst_cache_append(k, v, k_pages, v_pages, table, lengths, starts, q=None, turns=None, interleaved=False, amplitude=1.0, offsets=None, q_norm=None,
                       k_norm=None, eps=1e-6, slots=None, positions=None):
    """Writes the new tokens' k and v [rows, kv_heads, d] to their pages, k rotated by its positions (turns, interleaved, amplitude: see
    rotary.burst_rotary; None: not rotated); q [rows, H, d], if given, is rotated likewise and returned as a new tensor (rows behind the
    last sequence are not written).  offsets: int64 [sequences], added to the positions of the rotation (what of the
    sequence lies on the ring's other devices).  q_norm, k_norm [d] (of the pages' type or float32): q, k are normalised first, as
    rotary.burst_norm_rotary does, with these weights and eps (None: not normalised, which a norm without weights is not: that has ones).  slots: int64 [rows], the places of the tokens' keys and values (row slots[i] %
    page of page slots[i] // page, no two of them one place; negative or no page: left out) instead of those that the table says; positions: int64 [rows], the positions of the rotation
    instead of the places in the sequences (a tree's tokens have those of their depth; negative: the row is left out).  With both, the batch's three arrays
    are not read.  One launch; no gradient."""
    try:
        return B.load_torch_module().cache_append(k, v, k_pages, v_pages, table, lengths, starts, q, turns, bool(interleaved), float(amplitude), offsets,
                                                  q_norm, k_norm, float(eps), slots, positions)
    except RuntimeError as e:
        raise B.from_native(e) from None


def burst_paged_attention(q, k_pages, v_pages, table, lengths, starts, scale=None, causal=True, window=0, max_new=0, out=None, lse=None, full_p=False, tree=None):
    """Attention of the new tokens q [rows, H, d] (H a multiple of kv_heads) over the keys of their sequences up to their own positions (causal =
    False: all of them), the last `window` of them if that is not 0.  Returns (O [rows, H, d], lse [rows, H] fp32): new tensors, or out
    (of q's type or float32) and lse; rows behind the last sequence are not written, tokens that see no key get 0 and -inf.
    max_new: the most new tokens of any sequence, if the caller knows it (chooses the kernel only: single tokens, with up to 16 query heads for each
    of keys and values, have one that is made for them).  0: not known; 1 is taken where there are no more rows than sequences.
    O as float32, lse and a sum of 1 are a state that binding.burst_merge_state joins with those of
    the ring's other devices.  full_p (bfloat16): probabilities enter the product with the values with 16 bits in any call; otherwise the kernel
    of longer chunks rounds them to 8 at d = 64 and d = 128, as the walks do.
    tree: int64 [rows, words], the masks of drafted tokens: new token t of a sequence sees all keys before the sequence's new tokens, and new token j if bit
    j % 64 of word j // 64 of its row is set (its own among them).  A window then counts back from the first new token's position + the token's
    depth (bits - 1) among the keys before; the mask alone says which new tokens are seen (masks of a burst_cache_plan with the same window: those in it).  Sequences with more than 64 * words new tokens are chunks of
    prompts, as without masks.  No gradient."""
    scale = float(scale) if scale is not None else q.shape[-1] ** -0.5
    try:
        return B.load_torch_module().paged_attention(q, k_pages, v_pages, table, lengths, starts, scale, bool(causal), int(window), int(max_new), out, lse,
                                                      bool(full_p), tree)
    except RuntimeError as e:
        raise B.from_native(e) from None


class _Arrays(NamedTuple):
    starts: torch.Tensor
    lengths: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor
    tree: Optional[torch.Tensor]


class CachePlan(_Arrays):
    """What a step's calls read: starts [sequences + 1] and lengths [sequences] (int32; lengths with the new tokens), slots and positions [rows] (int64) of
    burst_cache_append, and tree [rows, words] (int64; None without parents) of burst_paged_attention.
    Beside the arrays: window, which the masks are made for (0: none), and longest, the most tokens that a branch can have (None: as many as bits)."""
    window, longest = 0, None

    def masks_for(self, window):
        """Whether the masks are those of attention with this window."""
        if self.tree is None:
            return True
        longest = self.longest or 64 * self.tree.shape[1]
        return min(self.window or longest, longest) == min(window or longest, longest)


def burst_cache_plan(new, lengths, table, free, count, page, rows, parents=None, words=1, window=0):
    """Plans a step on the device, from int32 tensors: new [sequences], the new tokens of each (negative: the sequence has ended), lengths [sequences], the tokens
    that each has in the cache, table [sequences, width] (-1: no page; a page is one entry's, or the stack's), free [pages] and count [1], a stack of the pages that are free, its top at
    count - 1.  rows: of the step's token tensors (up to 2^20 - 1; at most 4096 sequences).
    Sequences are served in their order; one whose new tokens do not fit into the rows that are left, whose tokens do not fit into a row of the table, or that
    lacks more pages than are free, is passed over (it has no new tokens in starts).  Entries of the table in which new tokens lie get a page where they
    have none; ended sequences give theirs back first.  table, free and count are written; the same call again changes nothing.
    parents: int32 [sequences, most], the new token (one before it) that each new token hangs on, -1: none; then the plan has the trees' masks of 64 * words bits,
    and positions go by depth; sequences with more new tokens than that are chunks of prompts.  window: of the attention that the masks are for, which sees that much of a branch (0: all of
    it; layers with other windows have a plan of their own, made by the same call again).  Returns a CachePlan; rows behind the last
    sequence have slot and position -1.  One launch, two of more than 2048 rows."""
    try:
        plan = CachePlan(*B.load_torch_module().cache_plan(new, lengths, table, free, count, int(page), int(rows), parents, int(words), int(window)))
    except RuntimeError as e:
        raise B.from_native(e) from None
    if parents is not None:
        plan.window, plan.longest = int(window), max(1, min(64 * int(words), parents.shape[1], int(rows)))
    return plan


def burst_cache_keep(k_pages, v_pages, table, lengths, starts, kept, counts):
    """Keeps some of the new tokens of every sequence (a branch of its tree), in all layers at once: k_pages, v_pages, a tensor or a list of every layer's,
    which lie alike; kept: int32 [sequences, most], the numbers of the tokens that are kept among the new ones, increasing; counts: int32 [sequences], how many.  Their
    keys and values move to where the first new tokens were; returns the new lengths [sequences], int32 (the pages behind them stay in the table, for the next
    tokens).  One launch (400 tensors each); no gradient."""
    ks, vs = ([p] if isinstance(p, torch.Tensor) else list(p) for p in (k_pages, v_pages))
    try:
        return B.load_torch_module().cache_keep(ks, vs, table, lengths, starts, kept, counts)
    except RuntimeError as e:
        raise B.from_native(e) from None
