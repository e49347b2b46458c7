"""A cache of keys and values in pages, and attention of new tokens over it: what serves a sequence token by token (or a prompt
chunk by chunk) after, or instead of, the walks over resident chunks.  Marshalling is native (csrc/burst_torch.cpp), the
kernels are csrc/burst_rotary.hip and csrc/burst_paged.hip.

Several sequences at once: token tensors [rows, heads, d] hold the new tokens of sequence s in rows starts[s] .. starts[s + 1] - 1
(views of a packed projection are read in place); lengths[s] counts all tokens of the sequence, the new ones among them; position p of
it is row p % page of page table[s, p // page] of k_pages and v_pages [pages, kv_heads, page, d] (any strides with a contiguous last
dimension; page: a power of two, 16 or more).  table, lengths and starts are int32 tensors on the device and are read there, so
that a captured call can be replayed with other contents (they are not to change while a call runs); values outside their
ranges are cut to them, a page that is not one of the pages holds no keys, nor does a position behind the table's row (new tokens there are
not kept, and see the keys that are), and attention with starts that decrease writes nothing."""
from . import binding as B


def burst_cache_append(k, v, k_pages, v_pages, table, lengths, starts, q=None, turns=None, interleaved=False, amplitude=1.0, offsets=None):
    """Writes the new tokens' k and v [rows, kv_heads, d] to their pages, k rotated by its positions (turns, interleaved, amplitude: see
    rotary.burst_rotary; None: not rotated); q [rows, H, d], if given, is rotated likewise and returned as a new tensor (rows behind the
    last sequence are not written).  offsets: int64 [sequences], added to the positions of the rotation (what of the
    sequence lies on the ring's other devices).  One launch; no gradient."""
    try:
        return B.load_torch_module().cache_append(k, v, k_pages, v_pages, table, lengths, starts, q, turns, bool(interleaved), float(amplitude), offsets)
    except RuntimeError as e:
        raise B.from_native(e) from None


def burst_paged_attention(q, k_pages, v_pages, table, lengths, starts, scale=None, causal=True, window=0, max_new=0, out=None, lse=None, full_p=False):
    """Attention of the new tokens q [rows, H, d] (H a multiple of kv_heads) over the keys of their sequences up to their own positions (causal =
    False: all of them), the last `window` of them if that is not 0.  Returns (O [rows, H, d], lse [rows, H] fp32): new tensors, or out
    (of q's type or float32) and lse; rows behind the last sequence are not written, tokens that see no key get 0 and -inf.
    max_new: the most new tokens of any sequence, if the caller knows it (chooses the kernel only: single tokens, with up to 16 query heads for each
    of keys and values, have one that is made for them).  0: not known; 1 is taken where there are no more rows than sequences.
    O as float32, lse and a sum of 1 are a state that binding.burst_merge_state joins with those of
    the ring's other devices.  full_p (bfloat16): probabilities enter the product with the values with 16 bits in any call; otherwise the kernel
    of longer chunks rounds them to 8 at d = 64 and d = 128, as the walks do.  No gradient."""
    scale = float(scale) if scale is not None else q.shape[-1] ** -0.5
    try:
        return B.load_torch_module().paged_attention(q, k_pages, v_pages, table, lengths, starts, scale, bool(causal), int(window), int(max_new), out, lse,
                                                      bool(full_p))
    except RuntimeError as e:
        raise B.from_native(e) from None
