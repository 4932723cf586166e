"""Refusals of the attention, rotary and cache entry points, before anything is launched: all device addresses are made up."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2210_09603_amd import binding as hb

INVALID, UNSUPPORTED, ALIGN = 1, 2, 3
OK = 0


def heads(data=0x1000, batch=1 << 20, head=1 << 14, row=64):
    return hb.hidet_heads_t(data, batch, head, row)


def options(**kw):
    o = hb.hidet_attention_options_t()
    o.struct_size = ctypes.sizeof(o)
    o.scale = 0.125
    for n, v in kw.items():
        setattr(o, n, v)
    return o


def attention(**kw):
    a = dict(dtype=hb.HIDET_F16, batch=2, heads=4, kv=2, sq=16, sk=16, dim=64, q=heads(), k=heads(), v=heads(), out=heads(0x100000),
             lse=None, o=options(), ws=None, wb=0)
    a.update(kw)
    return hb.lib().hidet_attention(a["dtype"], a["batch"], a["heads"], a["kv"], a["sq"], a["sk"], a["dim"], a["q"], a["k"], a["v"],
                                    a["out"], a["lse"], a["o"], a["ws"], a["wb"], None)


def backward(**kw):
    a = dict(dtype=hb.HIDET_F16, batch=2, heads=4, kv=2, sq=16, sk=16, dim=64, g=heads(), q=heads(), k=heads(), v=heads(), out=heads(),
             lse=0x1000, gq=heads(0x100000), gk=heads(0x200000), gv=heads(0x300000), o=options(), ws=0x10000, wb=1 << 20)
    a.update(kw)
    return hb.lib().hidet_attention_backward(a["dtype"], a["batch"], a["heads"], a["kv"], a["sq"], a["sk"], a["dim"], a["g"], a["q"], a["k"],
                                             a["v"], a["out"], a["lse"], a["gq"], a["gk"], a["gv"], a["o"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("call", [attention, backward])
def test_attention_refusals(call):
    assert call(dtype=3) == INVALID and call(dtype=-1) == INVALID
    assert call(dtype=hb.HIDET_F32) == UNSUPPORTED
    for n in ("batch", "heads", "kv", "sq", "sk", "dim", "wb"):
        assert call(**{n: -1}) == INVALID, n
    assert call(dim=0) == INVALID
    assert call(dim=60) == UNSUPPORTED and call(dim=136) == UNSUPPORTED
    assert call(heads=5) == INVALID and call(kv=0) == INVALID
    assert call(q=None) == INVALID and call(k=None) == INVALID and call(out=heads(None)) == INVALID
    assert call(q=heads(0x1001)) == ALIGN and call(v=heads(0x1001)) == ALIGN
    assert call(lse=0x1002) == ALIGN and call(ws=0x1008, wb=1 << 20) == ALIGN
    assert call(k=heads(row=-64)) == INVALID and call(q=heads(head=-1)) == INVALID
    assert call(k=heads(row=1 << 23)) == UNSUPPORTED
    assert call(q=heads(batch=1 << 47)) == UNSUPPORTED
    assert call(sq=1 << 29) == UNSUPPORTED and call(sk=1 << 29) == UNSUPPORTED and call(sq=1 << 28) == UNSUPPORTED  # (two heads a key head)
    assert call(o=None) == INVALID and call(o=options(struct_size=8)) == INVALID
    assert call(o=options(scale=math.nan)) == INVALID and call(o=options(scale=math.inf)) == INVALID
    assert call(o=options(softcap=-1.0)) == INVALID and call(o=options(softcap=math.inf)) == INVALID
    assert call(o=options(window=-1)) == INVALID and call(o=options(causal=2)) == INVALID
    assert call(o=options(ranges=0x1000, causal=1)) == INVALID and call(o=options(ranges=0x1000, window=4)) == INVALID
    assert call(o=options(slopes=0x1002)) == ALIGN and call(o=options(ranges=0x1001)) == ALIGN


def test_what_is_written_must_not_overlap_itself():
    assert attention(out=heads(row=0)) == INVALID and attention(out=heads(row=32)) == INVALID and attention(out=heads(batch=0)) == INVALID
    for n in ("gq", "gk", "gv"):
        assert backward(**{n: heads(head=0)}) == INVALID, n
    assert backward(lse=None) == INVALID and backward(ws=None) == INVALID
    n = hb.lib().hidet_attention_backward_workspace_bytes(2, 4, 2, 16, 16, 64)
    assert n > 0 and backward(wb=n - 1) == INVALID


def test_empty_calls_do_nothing():
    assert attention(batch=0) == OK and attention(sq=0) == OK and attention(heads=0, kv=0) == OK
    assert backward(batch=0) == OK and backward(sq=0, sk=0) == OK


def test_workspace_sizes():
    f = hb.lib().hidet_attention_workspace_bytes
    assert f(8, 32, 32, 4096, 4096, 128) == 0  # (fills the device)
    assert f(1, 8, 8, 1, 100000, 128) > 0 and f(1, 8, 8, 1, 100000, 128) % 8 == 0
    assert f(1, 8, 3, 1, 100, 128) == 0 and f(0, 8, 8, 1, 100, 128) == 0 and f(1, 8, 8, 1, 100, 256) == 0


def rope(**kw):
    a = dict(dtype=hb.HIDET_F16, batch=2, heads=4, seq=16, dim=64, rotary=64, x=heads(), y=heads(0x100000), f=0x1000, p=None, ps=0, first=0,
             inter=0, inv=0)
    a.update(kw)
    return hb.lib().hidet_rope(a["dtype"], a["batch"], a["heads"], a["seq"], a["dim"], a["rotary"], a["x"], a["y"], a["f"], a["p"], a["ps"],
                               a["first"], a["inter"], a["inv"], 1.0, None)


def test_rope_refusals():
    assert rope(dtype=5) == INVALID and rope(rotary=63) == INVALID and rope(rotary=66) == INVALID and rope(rotary=0) == INVALID
    assert rope(seq=-1) == INVALID and rope(inter=2) == INVALID and rope(inv=-1) == INVALID and rope(ps=-1) == INVALID
    assert rope(x=None) == INVALID and rope(f=None) == INVALID and rope(y=heads(None)) == INVALID
    assert rope(dim=4104, rotary=64) == UNSUPPORTED and rope(seq=1 << 29) == UNSUPPORTED and rope(first=1 << 40) == UNSUPPORTED
    assert rope(x=heads(0x1001)) == ALIGN and rope(dtype=hb.HIDET_F32, y=heads(0x1002)) == ALIGN and rope(f=0x1004) == ALIGN
    assert rope(p=0x1002) == ALIGN and rope(y=heads(row=32)) == INVALID
    assert rope(batch=0) == OK


def test_rope_frequencies():
    d = 128
    plain = hb.hidet_rope_frequencies(d).numpy()
    assert np.allclose(plain, 10000.0 ** (-2.0 * np.arange(d // 2) / d), rtol=1e-14)
    assert np.allclose(hb.hidet_rope_frequencies(d, scaling=hb.HIDET_ROPE_LINEAR, factor=4.0).numpy(), plain / 4, rtol=1e-14)
    base = hb.hidet_rope_frequencies(d, scaling=hb.HIDET_ROPE_BASE, factor=4.0).numpy()
    assert base[0] == 1.0 and abs(base[-1] / (plain[-1] / 4) - 1) < 1e-12  # fastest kept, slowest divided
    bands = hb.hidet_rope_frequencies(d, scaling=hb.HIDET_ROPE_BANDS, factor=8.0, low_turns=1.0, high_turns=4.0, original_length=8192).numpy()
    turns = 8192 * plain / (2 * np.pi)
    assert np.array_equal(bands[turns >= 4], plain[turns >= 4]) and np.allclose(bands[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all(bands[mid] < plain[mid]) and np.all(bands[mid] > plain[mid] / 8)
    f = hb.lib().hidet_rope_frequencies
    out = (ctypes.c_double * 64)()
    assert f(7, 1e4, 0, 1, 1, 4, 8192, out) == INVALID and f(8, 0.0, 0, 1, 1, 4, 8192, out) == INVALID and f(8, 1e4, 4, 1, 1, 4, 8192, out) == INVALID
    assert f(8, 1e4, 1, 0, 1, 4, 8192, out) == INVALID and f(2, 1e4, 2, 2, 1, 4, 8192, out) == INVALID and f(8, 1e4, 3, 2, 4, 4, 8192, out) == INVALID
    assert f(8, 1e4, 0, 1, 1, 4, 8192, None) == INVALID


def cache(**kw):
    c = hb.hidet_cache_t()
    c.struct_size = ctypes.sizeof(c)
    v = dict(dtype=hb.HIDET_F16, k=0x10000, v=0x20000, num_pages=8, page_size=16, heads=2, head_dim=64, stride_page=16 * 128, stride_slot=128,
             stride_head=64, tables=0x1000, table_width=4, table_stride=4, lengths=0x1000, seqs=3)
    v.update(kw)
    for n, x in v.items():
        setattr(c, n, x)
    return c


def append(c=None, tokens=5, max_new=4, k=heads(row=128, head=64), v=heads(row=128, head=64), starts=0x1000):
    return hb.lib().hidet_cache_append(c or cache(), tokens, max_new, k, v, starts, None)


def cache_attention(c=None, n_heads=4, tokens=5, max_new=4, q=heads(row=256, head=64), out=heads(0x90000, row=256, head=64), starts=0x1000,
                    o=None, ws=None, wb=0):
    return hb.lib().hidet_cache_attention(c or cache(), n_heads, tokens, max_new, q, out, None, starts, o or options(causal=1), ws, wb, None)


@pytest.mark.parametrize("call", [append, cache_attention])
def test_cache_refusals(call):
    for bad in (dict(struct_size=8), dict(dtype=7), dict(num_pages=-1), dict(page_size=0), dict(head_dim=0), dict(seqs=-1), dict(table_width=-1),
                dict(lengths=None), dict(tables=None), dict(k=None), dict(stride_slot=-1), dict(stride_slot=32), dict(stride_page=0),
                dict(table_stride=3), dict(heads=-1)):
        assert call(cache(**bad)) == INVALID, bad
    for bad in (dict(head_dim=60), dict(num_pages=1 << 31), dict(stride_page=1 << 46)):
        assert call(cache(**bad)) == UNSUPPORTED, bad
    for bad in (dict(k=0x10001), dict(lengths=0x1002), dict(tables=0x1001)):
        assert call(cache(**bad)) == ALIGN, bad
    assert call(tokens=-1) == INVALID and call(max_new=-1) == INVALID and call(starts=None) == INVALID and call(starts=0x1002) == ALIGN
    assert call(tokens=1 << 29) == UNSUPPORTED
    assert call(tokens=0) == OK and call(max_new=0) == OK and call(cache(seqs=0)) == OK


def test_cache_attention_refusals():
    assert cache_attention(cache(dtype=hb.HIDET_F32)) == UNSUPPORTED and cache_attention(
        cache(head_dim=136, stride_head=136, stride_slot=272, stride_page=16 * 272)) == UNSUPPORTED
    assert cache_attention(n_heads=3) == INVALID and cache_attention(n_heads=-2) == INVALID and cache_attention(wb=-1) == INVALID
    assert cache_attention(o=options()) == INVALID and cache_attention(o=options(causal=1, ranges=0x1000)) == INVALID
    assert cache_attention(out=heads(0x90000, row=32, head=64)) == INVALID
    assert cache_attention(ws=0x1004, wb=64) == ALIGN
    assert append(k=heads(None)) == INVALID and append(v=None) == INVALID and append(k=heads(0x1001)) == ALIGN
    assert append(cache(dtype=hb.HIDET_F32), v=heads(0x1002, row=128, head=64)) == ALIGN


def test_ranges_refusals():
    f = hb.lib().hidet_attention_ranges
    assert f(-1, 4, 4, None, None, 1, 0, 0x1000, None) == INVALID and f(1, 4, 4, None, None, 2, 0, 0x1000, None) == INVALID
    assert f(1, 4, 4, None, 0x1000, 1, 3, 0x1000, None) == INVALID and f(1, 4, 4, None, None, 1, -3, 0x1000, None) == INVALID
    assert f(1, 4, 4, None, None, 1, 0, None, None) == INVALID and f(1, 1 << 29, 4, None, None, 1, 0, 0x1000, None) == UNSUPPORTED
    assert f(1, 4, 4, 0x1001, None, 1, 0, 0x1000, None) == ALIGN and f(0, 4, 4, None, None, 1, 0, None, None) == OK


def test_the_binding_refuses_what_it_cannot_describe():
    q, k = torch.zeros(1, 2, 4, 64, dtype=torch.float16), torch.zeros(1, 2, 6, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="on the GPU"):
        hb.hidet_attention(q, k, k, q.clone())
    for bad in (dict(lse=torch.zeros(1, 2, 4, dtype=torch.float64)), dict(slopes=torch.zeros(3)), dict(ranges=torch.zeros(1, 4, 2))):
        with pytest.raises(ValueError):
            hb.hidet_attention(q, k, k, q.clone(), **bad)
    for args in ((q, k, k[:, :1], q), (q, k, k, q[:, :, :2]), (q.float(), k, k, q), (q[0], k, k, q)):
        with pytest.raises(ValueError):
            hb.hidet_attention(*args)
    pages = torch.zeros(4, 16, 2, 64, dtype=torch.float16)
    tables, lengths = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args in ((pages, pages[:2], tables, lengths), (pages, pages.float(), tables, lengths), (pages, pages, tables.long(), lengths),
                 (pages, pages, tables, lengths[:2]), (pages, pages.transpose(0, 1).contiguous().transpose(0, 1), tables, lengths)):
        with pytest.raises(ValueError):
            hb.make_cache(*args)
    c = hb.make_cache(pages, pages.clone(), tables, lengths)
    x = torch.zeros(5, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        hb.hidet_cache_append(c, x, x, torch.zeros(3, dtype=torch.int32), 1)
    with pytest.raises(ValueError):
        hb.hidet_cache_append(c, x[:, :1], x[:, :1], torch.zeros(4, dtype=torch.int32), 1)
    with pytest.raises(ValueError):
        hb.hidet_cache_attention(c, x.float(), x, torch.zeros(4, dtype=torch.int32), 1)
    with pytest.raises(ValueError):
        hb.hidet_rope(q, q, torch.zeros(32))


def test_workspaces_that_are_not_dense_are_refused():
    """(A strided one holds elements that are not its own, an expanded one has fewer bytes than elements.)"""
    q, k = torch.zeros(1, 2, 3, 16, dtype=torch.float16), torch.zeros(1, 2, 4, 16, dtype=torch.float16)
    lse = torch.zeros(1, 2, 3)
    pages, i32 = torch.zeros(2, 4, 2, 16, dtype=torch.float16), lambda *shape: torch.zeros(shape, dtype=torch.int32)
    cache = hb.make_cache(pages, pages.clone(), i32(1, 2), i32(1))
    rows = torch.zeros(3, 2, 16, dtype=torch.float16)
    for ws in (torch.zeros(64)[::2], torch.zeros(1).expand(1 << 20)):
        for f, args in ((hb.hidet_attention, (q, k, k, q)), (hb.hidet_attention_backward, (q, q, k, k, q, lse, q, k, k)),
                        (hb.hidet_cache_attention, (cache, rows, rows, i32(2), 3))):
            with pytest.raises(ValueError, match="dense"):
                f(*args, workspace=ws)


def test_sizes_at_and_beyond_the_limits_are_answered():
    """Each size within its own limit, their product far beyond: a query of a workspace answers 0, a call refuses; sizes that a call
    takes have workspaces that are counted in 64 bits."""
    L = hb.lib()
    big = [(1 << 24, 1 << 20, 1 << 20, 1 << 20, 4096, 64), (1 << 24, 1 << 24, 1 << 24, 1 << 13, 1, 64), (1 << 24, 1 << 24, 1 << 24, 1 << 28, 1, 128),
           (1 << 24, 2, 2, 5, 1 << 28, 64), (1, 1 << 28, 1, 2, 4096, 64), (2, 4, 2, 16, 1 << 62, 64), (1 << 62, 4, 2, 16, 16, 64), (1, 1 << 62, 1 << 62, 1, 1, 64),
           (1, 1 << 62, 1, 1, 1, 64)]
    for b, h, kv, n, m, d in big:
        assert L.hidet_attention_workspace_bytes(b, h, kv, n, m, d) == 0, (b, h, kv, n, m, d)
        assert L.hidet_attention_backward_workspace_bytes(b, h, kv, n, m, d) == 0, (b, h, kv, n, m, d)
        near = heads(batch=128, head=128, row=128)
        for call in (attention, backward):
            kw = dict(q=near, k=near, v=near, out=heads(0x100000, 128, 128, 128), wb=1 << 62, ws=0x10000)
            if call is backward:
                kw.update(g=near, gq=heads(0x100000, 128, 128, 128), gk=near, gv=near)
            assert call(batch=b, heads=h, kv=kv, sq=n, sk=m, dim=d, **kw) == UNSUPPORTED, (b, h, kv, n, m, d)
    # rows and keys at their limits, for entries at theirs
    most = L.hidet_attention_backward_workspace_bytes(1 << 12, 1 << 12, 1 << 12, (1 << 29) - 1, 1, 128)
    assert most >= (1 << 24) * ((1 << 29) - 1) * 32
    for seqs, kv, h, new in ((1 << 24, 1 << 20, 1 << 20, 1 << 13), (1 << 24, 1 << 24, 1 << 24, 1 << 13), (1 << 13, 1 << 12, 1 << 12, 4), (1 << 24, 2, 2, 1 << 28)):
        c = cache(seqs=seqs, heads=kv, stride_head=64, stride_slot=64, stride_page=64)
        assert L.hidet_cache_attention_workspace_bytes(c, h, new, 0) == 0
        assert cache_attention(c, n_heads=h, max_new=new, q=heads(row=64, head=64), out=heads(0x90000, row=64, head=64)) == UNSUPPORTED
    # (so many rows that the second kernel of equal pieces had no grid for them)
    c = cache(seqs=1024, heads=1 << 14, stride_head=64, stride_slot=64, stride_page=64, table_width=4096, table_stride=4096)
    assert L.hidet_cache_attention_workspace_bytes(c, 1 << 19, 1, 0) == 0


@pytest.mark.parametrize("call", [attention, backward])
def test_factors_that_pass_fp32_are_refused(call):
    for o in (dict(softcap=1e-39), dict(scale=2e38), dict(scale=-2e38), dict(scale=1e20, softcap=1e-19), dict(scale=1e38, softcap=0.5)):
        assert call(o=options(**o)) == UNSUPPORTED, o


def test_rope_in_place_under_other_strides_is_refused():
    """(It would read what it has written, and leave what it had to move.)"""
    here = heads(0x100000)
    for other in (heads(0x100000, row=128), heads(0x100000, head=1 << 15), heads(0x100000, batch=1 << 21), heads(0x100000, batch=0)):
        assert rope(x=other, y=here) == INVALID
    # (strides of dimensions that have one entry do not count: what is left to refuse is the alignment)
    assert rope(batch=1, heads=1, x=heads(0x100000, batch=5, head=7), y=here, f=0x1004) == ALIGN
