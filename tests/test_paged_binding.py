"""The binding's calls of the rotation and the paged cache: what its parameter blocks cannot say is refused before any device call.  A block
holds addresses, sizes and strides only, so that each of these tensors would be read or written beyond its end."""
import pytest
import torch

from paper_2403_09347_amd import binding as B

BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
R = B.BurstRotary(4096, 16, 0, 1.0, 0)                        # (addresses that nothing reads)


def test_rotated_tensors_and_positions():
    x, at = torch.zeros(2, 3, 5, 16), torch.zeros(2, 5, dtype=I64)
    for bad in (at[:, :1].expand(2, 5),                       # one position for all rows, which a block has no stride for
                at[:1, :1].expand(2, 5), torch.zeros(2, 10, dtype=I64)[:, ::2], at[:1], at[:, :4], at[0], at.int()):
        with pytest.raises(ValueError, match="positions: int64"):
            B.burst_rotate([x], [x], R, positions=[bad])
    for good in (at, at[:1].expand(2, 5), at[:, :1]):         # these are fine: it is x that is refused
        y = x[:, :, :good.shape[1]]
        with pytest.raises(ValueError, match="device tensor"):
            B.burst_rotate([y], [y], R, positions=[good])
    one = torch.zeros(1, 1, 1, 16).expand(2, 3, 5, 16)        # its strides are 0, which a block takes for dense ones
    for a, b in ((one, x), (x, one), (x, x[:1].expand(2, 3, 5, 16)), (x, x[:, :1].expand(2, 3, 5, 16)), (x, x[:, :, :1].expand(2, 3, 5, 16))):
        with pytest.raises(ValueError, match="not one row for all"):
            B.burst_rotate([a], [b], R)
    with pytest.raises(ValueError, match="device tensor"):    # heads that share rows are read as they are
        B.burst_rotate([x[:, :1].expand(2, 3, 5, 16)], [x], R)
    for other in (torch.zeros(2, 3, 5, 8), x.to(BF16), x[0]):
        with pytest.raises(ValueError, match="of one type and d"):
            B.burst_rotate([x, other], [x, other], R)
    with pytest.raises(ValueError, match="of one type and d"):
        B.burst_rotate([x.half()], [x.half()], R)
    for kw in (dict(ys=[x]), dict(offsets=[1]), dict(positions=[None])):
        with pytest.raises(ValueError, match="as many"):
            B.burst_rotate([x, x], **dict(dict(ys=[x, x], r=R), **kw))


def cache(**kw):
    t = dict(k_pages=torch.zeros(5, 2, 16, 64, dtype=BF16), table=torch.zeros(3, 4, dtype=I32), lengths=torch.zeros(3, dtype=I32),
             starts=torch.zeros(4, dtype=I32))
    t.update(kw)
    return t


def block(**kw):
    return B.paged_params(6, 4, 2, 64, BF16, **cache(**kw))


def test_arrays_of_a_batch():
    t = cache()
    for bad in (dict(table=t["table"].long()), dict(lengths=t["lengths"].long()), dict(starts=t["starts"].long()), dict(table=t["table"][0]),
                dict(lengths=t["lengths"][:2]), dict(starts=t["starts"][:3]), dict(table=t["table"][:2])):
        with pytest.raises(ValueError, match="int32 tensors"):
            block(**bad)
    for bad in (dict(table=t["table"][:1].expand(3, 4)),      # a stride of 0 would mean rows that lie one after the other
                dict(table=torch.zeros(4, 3, dtype=I32).t()), dict(lengths=torch.zeros(6, dtype=I32)[::2]), dict(starts=t["starts"][:1].expand(4))):
        with pytest.raises(ValueError, match="contiguous"):
            block(**bad)
    assert block().table_stride in (0, 4) and block(table=torch.zeros(3, 9, dtype=I32)[:, :4]).table_stride == 9
    one = block(table=torch.zeros(1, 4, dtype=I32).expand(1, 4), lengths=t["lengths"][:1], starts=t["starts"][:2])
    assert one.table_stride in (0, 4)


def test_pages():
    t = cache()["k_pages"]
    for bad in (t[:1].expand(5, 2, 16, 64), t[:1, :1, :1].expand(5, 2, 16, 64), t[:, :1].expand(5, 2, 16, 64)):
        with pytest.raises(ValueError, match="one after the other"):
            block(k_pages=bad)
    for bad in (t[:, :1], t[..., :32], t[0], torch.zeros(5, 2, 16, 128, dtype=BF16)[..., ::2]):
        with pytest.raises(ValueError, match="k_pages"):
            block(k_pages=bad)
    assert list(block().page_strides) == [0, 0, 0]
    assert list(block(k_pages=torch.zeros(5, 16, 2, 64, dtype=BF16).transpose(1, 2)).page_strides) == [2048, 64, 128]


def test_tensors_of_a_block():
    pages, p = cache()["k_pages"], block()
    q, kv, lse = torch.zeros(6, 4, 64, dtype=BF16), torch.zeros(6, 2, 64, dtype=BF16), torch.zeros(6, 4)

    def fwd(p=p, **kw):
        B.burst_paged_fwd(**dict(dict(Q=q, k_pages=pages, v_pages=pages, O=q, lse=lse, p=p), **kw))

    def append(p=p, **kw):
        B.burst_cache_append(**dict(dict(K=kv, V=kv, k_pages=pages, v_pages=pages, Q=None, Q_out=None, offsets=None, r=None, p=p), **kw))

    with pytest.raises(ValueError, match="device tensor"):    # nothing but that they lie on the host
        fwd()
    with pytest.raises(ValueError, match="device tensor"):
        append()
    wide = torch.zeros(6, 8, 64, dtype=BF16)
    for bad in (q[:5], q[:, :3], q.float(), q[0], wide[:, :4], q[:1].expand(6, 4, 64)):
        with pytest.raises(ValueError, match="Q: "):
            fwd(Q=bad)
    for bad in (kv[:5], kv[:, :1], kv.float(), wide[:, :2]):
        with pytest.raises(ValueError, match="K: "):
            append(K=bad)
    strided = block()
    strided.q_strides[:] = [512, 64]
    with pytest.raises(ValueError, match="Q: strides"):
        fwd(strided)
    with pytest.raises(ValueError, match="device tensor"):
        fwd(strided, Q=wide[:, :4])
    with pytest.raises(ValueError, match="lse"):
        fwd(lse=lse[:5])
    with pytest.raises(ValueError, match="v_pages"):
        B._pages(pages[:4], p, "v_pages")
    with pytest.raises(ValueError, match="v_pages"):
        B._pages(torch.zeros(5, 16, 2, 64, dtype=BF16).transpose(1, 2), p, "v_pages")
    with pytest.raises(ValueError, match="offsets"):
        B._offsets(torch.zeros(2, dtype=I64), p)
    assert B._offsets(None, p) is None


def test_tensors_of_another_device(monkeypatch):
    """The library launches on the current device."""
    class Elsewhere:
        is_cuda, device = True, torch.device("cuda", 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        B._here(Elsewhere(), "x")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    B._here(Elsewhere(), "x")


def test_blocks_keep_what_they_point_to(monkeypatch):
    t = cache()
    p = block(**t)
    assert all(a is b for a, b in zip(p.holds, (t["starts"], t["lengths"], t["table"])))
    monkeypatch.setattr(B, "_ptr", lambda t: t.data_ptr())
    turns = torch.zeros(8, dtype=torch.float64)
    assert B.rotary(turns).holds is turns
