"""The paged cache: append (exact copies) and attention of ragged batches over pages, against the float64 oracle."""
import numpy as np
import pytest
import torch

from attention_helpers import TYPES, assert_within, bounds, f64
from oracle import attention as oa
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Batch:
    """A ragged batch over a cache whose pages are dealt at random: lengths (with the new tokens) and new tokens of every sequence."""

    def __init__(self, seed, dtype, lengths, new, heads, kv_heads, dim, page, layout="dense", pad=0, width=None):
        g = self.g = np.random.Generator(np.random.PCG64(seed))
        self.dtype, self.lengths, self.new, self.heads, self.kv_heads, self.dim, self.page = dtype, lengths, new, heads, kv_heads, dim, page
        t = TYPES[dtype]
        used = [-(-n // page) for n in lengths]
        pages = sum(used) + 3
        if layout == "dense":
            both = [torch.empty(pages, page, kv_heads, dim, dtype=t, device="cuda") for _ in range(2)]
        elif layout == "heads first":  # [pages][heads][page_size][dim]
            both = [torch.empty(pages, kv_heads, page, dim, dtype=t, device="cuda").transpose(1, 2) for _ in range(2)]
        else:  # keys and values of a page side by side, rows of odd length
            wide = torch.zeros(pages, 2, page, kv_heads, dim + 5, dtype=t, device="cuda")
            both = [wide[:, i, :, :, 1:dim + 1] for i in range(2)]
        self.k_pages, self.v_pages = both
        for x in both:
            x.copy_(torch.from_numpy(g.standard_normal((pages, page, kv_heads, dim)).astype(np.float32)))
        deal = g.permutation(pages)
        table = np.full((len(lengths), width or max(max(used), 1)), -7, dtype=np.int32)
        at = 0
        for s, n in enumerate(used):
            table[s, :n] = deal[at:at + n]
            at += n
        self.table = table
        self.tables, self.lens = torch.from_numpy(table).cuda(), _ints(lengths)
        starts = np.concatenate([[0], np.cumsum(new)])
        self.starts, self.total = _ints(starts.tolist()), int(starts[-1])
        self.tokens = self.total + pad
        self.cache = hb.make_cache(self.k_pages, self.v_pages, self.tables, self.lens)

    def rows(self, heads):
        x = self.g.standard_normal((self.tokens, heads, self.dim)).astype(np.float32)
        return torch.from_numpy(x).to(TYPES[self.dtype]).cuda()

    def check(self, q, out, lse, scale=None, window=0, softcap=0.0, slopes=None, at_most=None, what=""):
        k, v = f64(self.k_pages), f64(self.v_pages)
        s0 = 0
        for s, (length, n) in enumerate(zip(self.lengths, self.new)):
            rows = slice(s0, s0 + n)
            s0 += n
            if n == 0:
                continue
            done = n if at_most is None else min(n, at_most)
            kk, there = oa.cache_rows(k, self.table[s], length)
            vv, _ = oa.cache_rows(v, self.table[s], length)
            see = oa.sees(n, length, causal=True, window=window) & there[None, :]
            # (weights of keys below a running maximum that is up to 2^8 stale, splits: the bound of the weights does not change)
            want, bound = bounds(self.dtype, f64(q[rows]).transpose(1, 0, 2)[None], kk[None], vv[None], see[None],
                                 self.dim ** -0.5 if scale is None else scale, softcap, slopes)
            got = f64(out[rows]).transpose(1, 0, 2)[None]
            assert_within(got[:, :, :done], want[0][:, :, :done], bound[0][:, :, :done], "%s sequence %d out" % (what, s))
            if lse is not None:
                assert_within(f64(lse[rows]).T[None][:, :, :done], want[1][:, :, :done], bound[1][:, :, :done], "%s sequence %d lse" % (what, s))

    def run(self, max_new=None, workspace=True, **kw):
        q = self.rows(self.heads)
        out = torch.full_like(q, 7.0)
        lse = torch.full((self.tokens, self.heads), 7.0, device="cuda")
        max_new = max(self.new) if max_new is None else max_new
        ws = None
        if workspace:
            size = hb.hidet_cache_attention_workspace_bytes(self.cache, q, max_new, kw.get("window", 0))
            ws = torch.full((size // 4 + 1,), float("nan"), device="cuda")[:size // 4] if size else None
        hb.hidet_cache_attention(self.cache, q, out, self.starts, max_new, lse=lse, workspace=ws, **kw)
        torch.cuda.synchronize()
        assert bool((out[self.total:] == 7.0).all()) and bool((lse[self.total:] == 7.0).all())  # rows behind the last sequence
        return q, out, lse


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 100])
def test_single_tokens(page, dtype):
    b = Batch(page, dtype, [1, 2, 15, 16, 17, 63, 64, 65, 130, 400, 33, 129], [1] * 12, 8, 2, 64, page, pad=2)
    q, out, lse = b.run()
    b.check(q, out, lse)
    q, out, lse = b.run(workspace=False)
    b.check(q, out, lse)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (7, 1, 128), (32, 4, 128), (6, 6, 40), (40, 1, 96), (64, 1, 8)])
def test_heads_and_dims(heads, kv_heads, dim, dtype):
    for layout in ("dense", "heads first", "odd"):
        b = Batch(heads + dim, dtype, [70, 5, 300], [1, 1, 1], heads, kv_heads, dim, 16, layout=layout, pad=1)
        q, out, lse = b.run()
        b.check(q, out, lse, what=layout)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_chunks(dim, dtype):
    # a whole prompt, a chunk behind a cached beginning, a single token, no new token, nothing at all
    b = Batch(dim, dtype, [90, 400, 77, 50, 0, 261], [90, 130, 1, 0, 0, 2], 6, 2, dim, 32, pad=5)
    for kw in (dict(), dict(window=50), dict(softcap=3.0), dict(window=1), dict(scale=0.3)):
        q, out, lse = b.run(**kw)
        b.check(q, out, lse, what=str(kw), **kw)
    slopes = torch.tensor([2.0 ** -(i + 1) for i in range(6)], device="cuda")
    q, out, lse = b.run(slopes=slopes, softcap=8.0)
    b.check(q, out, lse, softcap=8.0, slopes=f64(slopes))


def test_long_contexts_are_split_and_give_the_same_bits_twice():
    for dtype, lengths, new, window in (("bf16", [9000], [1], 0), ("f16", [6000, 37], [40, 1], 0), ("bf16", [20000], [2], 3000)):
        b = Batch(len(lengths) + new[0], dtype, lengths, new, 4, 1, 128, 64)
        q = b.rows(4)
        size = hb.hidet_cache_attention_workspace_bytes(b.cache, q, max(new), window)
        assert size > 0
        outs = []
        for _ in range(2):
            out, lse = torch.zeros_like(q), torch.zeros(b.tokens, 4, device="cuda")
            ws = torch.full((size // 4,), float("nan"), device="cuda")
            hb.hidet_cache_attention(b.cache, q, out, b.starts, max(new), lse=lse, window=window, workspace=ws)
            outs.append((out, lse))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        b.check(q, *outs[0], window=window)


def test_what_lies_behind_a_sequence_and_on_no_page_is_not_seen():
    b = Batch(3, "bf16", [40, 130, 20], [1, 70, 20], 4, 2, 64, 16)
    k, v = b.k_pages, b.v_pages
    used = set()
    for s, length in enumerate(b.lengths):
        for t in range(length):
            used.add((int(b.table[s, t // 16]), t % 16))
    for page in range(k.shape[0]):
        for slot in range(16):
            if (page, slot) not in used:
                k[page, slot], v[page, slot] = float("nan"), float("inf")
    q, out, lse = b.run()
    b.check(q, out, lse)
    # pages that were given back, numbers of no page
    b.tables[1, 1] = -1
    b.tables[1, 4] = k.shape[0]
    b.tables[2, 0] = 2 ** 31 - 1
    b.table = b.tables.cpu().numpy()
    b2 = b.table.copy()
    b2[b2 >= k.shape[0]] = -1
    b.table = b2
    q, out, lse = b.run()
    b.check(q, out, lse)
    q, out, lse = b.run(window=30)
    b.check(q, out, lse, window=30)


def test_lists_that_make_no_sense_reach_nothing():
    """Starts that descend or leave the batch, lengths that are negative or pass the table: no row outside the sequences that make
    sense is written, and nothing outside the tensors is touched."""
    b = Batch(4, "f16", [40, 30, 50], [1, 1, 1], 2, 1, 64, 16, pad=3)
    q = b.rows(2)
    k = b.rows(1)
    before = b.k_pages.clone()
    for starts, lengths in (([0, 1, 1, 2], [-5, 30, 2 ** 31 - 1]), ([5, 3, 9000, -4], [40, 30, 50]), ([-3, -2, -1, 0], [40, 30, 50]),
                            ([0, 0, 0, 0], [0, 0, 0])):
        b.starts.copy_(_ints(starts))
        b.lens.copy_(_ints(lengths))
        out = torch.full_like(q, 7.0)
        hb.hidet_cache_attention(b.cache, q, out, b.starts, 1)
        hb.hidet_cache_append(b.cache, k, k, b.starts, 1)
        torch.cuda.synchronize()
    b.starts.copy_(_ints([0, 0, 0, 0]))
    b.k_pages.copy_(before)
    out = torch.full_like(q, 7.0)
    hb.hidet_cache_attention(b.cache, q, out, b.starts, 1)
    hb.hidet_cache_append(b.cache, k, k, b.starts, 1)
    assert bool((out == 7.0).all()) and torch.equal(b.k_pages, before)


# ---- a ragged batch of many entries: equal pieces of all its keys ----
RAGGED = [0, 1, 2, 31, 32, 33, 3000, 64, 65, 700, 5, 1, 0, 2100, 96, 97, 300, 301, 12, 40, 41, 42, 1500, 3, 8, 9, 10, 128, 129, 1000, 6, 700]


def _ragged(seed, dtype, dim, poison=False, **kw):
    """32 sequences of 0 to 3000 tokens, 0 to 4 of them new, 8 kv heads; one of them without a page in its middle."""
    new = [min(n, (i * 7) % 5) for i, n in enumerate(RAGGED)]
    new[4] = new[30] = 0
    b = Batch(seed, dtype, RAGGED, new, 16, 8, dim, 48, pad=3, width=350, **kw)
    b.table[9, 3] = -1
    b.tables.copy_(torch.from_numpy(b.table))
    if poison:  # (whatever no sequence owns)
        own = torch.zeros(b.k_pages.shape[:2], dtype=torch.bool)
        for s, n in enumerate(RAGGED):
            for t in range(n):
                if b.table[s, t // 48] >= 0:
                    own[int(b.table[s, t // 48]), t % 48] = True
        for x in (b.k_pages, b.v_pages):
            x[~own.cuda()] = float("nan")
    return b


@pytest.mark.parametrize("dtype,dim,poison", [("f16", 64, False), ("bf16", 128, False), ("bf16", 40, True), ("f16", 128, True)])
def test_ragged_batches_in_equal_pieces(dtype, dim, poison):
    b = _ragged(dim, dtype, dim, poison)
    slopes = torch.tensor([2.0 ** -(i / 2 + 1) for i in range(16)], device="cuda")
    for kw in (dict(), dict(window=100), dict(window=2500), dict(softcap=5.0, slopes=slopes)):
        if poison and "window" not in kw and kw:
            continue
        for workspace in (True, False):
            q, out, lse = b.run(workspace=workspace, **kw)
            b.check(q, out, lse, what=str(kw), **{k: f64(v) if k == "slopes" else v for k, v in kw.items()})


def test_ragged_pieces_of_one_token_and_of_a_wide_table():
    """One long sequence among short ones, a table that would hold a hundred times as many tokens."""
    lengths = [9000 if i == 13 else 1 + i % 70 for i in range(64)]
    b = Batch(3, "bf16", lengths, [1] * 64, 32, 8, 128, 16, width=4096)
    q, out, lse = b.run()
    b.check(q, out, lse)
    again = torch.zeros_like(out)
    ws = torch.full((hb.hidet_cache_attention_workspace_bytes(b.cache, q, 1) // 4,), 3e38, device="cuda")
    hb.hidet_cache_attention(b.cache, q, again, b.starts, 1, workspace=ws)
    assert torch.equal(out, again)


def test_ragged_pieces_under_a_wide_window():
    lengths = [20000 if i == 3 else 17100 if i == 20 else 1 + 9 * i for i in range(32)]
    b = Batch(4, "f16", lengths, [1 + i % 2 for i in range(31)] + [0], 8, 8, 64, 64)
    q, out, lse = b.run(window=17000)
    b.check(q, out, lse, window=17000)


def test_ragged_pieces_captured_while_lengths_grow():
    b = _ragged(11, "f16", 64)
    q = b.rows(16)
    ws = torch.empty(hb.hidet_cache_attention_workspace_bytes(b.cache, q, 4), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]
    call = lambda out: hb.hidet_cache_attention(b.cache, q, out, b.starts, 4, workspace=ws)
    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    for shrink in (0, 100, 500, 3, 0):
        b.lens.copy_(_ints([n if i % 3 else max(n - shrink, min(n, 4)) for i, n in enumerate(RAGGED)]))
        outs[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        outs[0].zero_()
        call(outs[0])
        torch.cuda.synchronize()
        assert torch.equal(*outs), shrink


def test_ragged_lists_that_make_no_sense_reach_nothing():
    """Starts and lengths out of any order: no index leaves its tensor, and nothing hangs."""
    b = _ragged(12, "bf16", 64)
    q = b.rows(16)
    g = np.random.Generator(np.random.PCG64(5))
    ws = torch.empty(hb.hidet_cache_attention_workspace_bytes(b.cache, q, 4), dtype=torch.uint8, device="cuda")
    for lengths, starts, table in ((2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), (10 ** 4, 100, 60)):
        b.lens.copy_(torch.from_numpy(g.integers(-lengths, lengths, size=32).astype(np.int32)))
        b.starts.copy_(torch.from_numpy(g.integers(-starts, starts, size=33).astype(np.int32)))
        b.tables.copy_(torch.from_numpy(g.integers(-table, table, size=b.table.shape).astype(np.int32)))
        buf = torch.full((q.numel() + 512,), 7.0, dtype=q.dtype, device="cuda")
        out = buf[256:-256].view(q.shape)
        hb.hidet_cache_attention(b.cache, q, out, b.starts, 4, workspace=ws)
        torch.cuda.synchronize()
        assert bool((buf[:256] == 7.0).all()) and bool((buf[-256:] == 7.0).all())


def test_at_most_max_new_tokens_of_a_sequence():
    b = Batch(6, "bf16", [40, 60], [9, 4], 2, 2, 64, 16)
    q, out, lse = b.run(max_new=5)
    b.check(q, out, lse, at_most=5)
    assert bool((out[5:9] == 7.0).all())
    k, v = b.rows(2), b.rows(2)
    before = b.k_pages.clone()
    hb.hidet_cache_append(b.cache, k, v, b.starts, 5)
    for t in range(31, 40):
        page, slot = int(b.table[0, t // 16]), t % 16
        assert torch.equal(b.k_pages[page, slot], k[t - 31] if t - 31 < 5 else before[page, slot])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("page,heads,dim,layout", [(1, 1, 8, "dense"), (16, 8, 128, "dense"), (7, 3, 40, "odd"), (64, 2, 200, "heads first"),
                                                   (256, 16, 64, "odd")])
def test_append(page, heads, dim, layout, dtype):
    b = Batch(page + dim, dtype, [300, 17, 1, 0, 64, 1500, 90], [300, 16, 1, 0, 1, 1400, 0], heads, heads, dim, page, layout=layout, pad=4)
    b.table[4, 0] = -3  # no page: nothing is written
    b.tables.copy_(torch.from_numpy(b.table))
    wide = torch.zeros(b.tokens, 2, heads, dim + 3, dtype=TYPES[dtype], device="cuda")
    k, v = wide[:, 0, :, 3:], wide[:, 1, :, 2:-1]
    k.copy_(b.rows(heads))
    v.copy_(b.rows(heads))
    want = [b.k_pages.clone(), b.v_pages.clone()]
    starts = b.starts.tolist()
    for s, (length, n) in enumerate(zip(b.lengths, b.new)):
        for i in range(n):
            page_no, slot = int(b.table[s, (length - n + i) // page]), (length - n + i) % page
            if page_no >= 0:
                want[0][page_no, slot], want[1][page_no, slot] = k[starts[s] + i], v[starts[s] + i]
    hb.hidet_cache_append(b.cache, k, v, b.starts, max(b.new))
    torch.cuda.synchronize()
    assert torch.equal(b.k_pages, want[0]) and torch.equal(b.v_pages, want[1])


def test_many_sequences():
    n = 700
    b = Batch(9, "f16", [3 + i % 5 for i in range(n)], [1 + i % 2 for i in range(n)], 1, 1, 64, 4, pad=1)
    k, v = b.rows(1), b.rows(1)
    hb.hidet_cache_append(b.cache, k, v, b.starts, 2)
    starts = b.starts.tolist()
    kp = b.k_pages.cpu()
    for s in range(n):
        for i in range(b.new[s]):
            t = b.lengths[s] - b.new[s] + i
            assert torch.equal(kp[int(b.table[s, t // 4]), t % 4], k[starts[s] + i].cpu())


def test_offsets_beyond_32_bits():
    """Pages 2^28 elements apart: the tenth begins 2.6e9 elements behind the first."""
    apart, page, dim = 2 ** 28 + 64, 16, 64
    bufs = [torch.zeros(11 * apart + page * dim, dtype=torch.float16, device="cuda") for _ in range(2)]
    k_pages, v_pages = (torch.as_strided(x, (12, page, 1, dim), (apart, dim, dim, 1)) for x in bufs)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (k_pages, v_pages):
        x.copy_(torch.randn(12, page, 1, dim, device="cuda", generator=g))
    table = np.array([[11, 3, 10, 9]], dtype=np.int32)
    cache = hb.make_cache(k_pages, v_pages, torch.from_numpy(table).cuda(), _ints([60]))
    new = torch.randn(40, 1, dim, device="cuda", generator=g).half()
    hb.hidet_cache_append(cache, new, -new, _ints([0, 40]), 40)
    for t in range(20, 60):
        assert torch.equal(k_pages[int(table[0, t // page]), t % page], new[t - 20])
        assert torch.equal(v_pages[int(table[0, t // page]), t % page], -new[t - 20])
    kk, _ = oa.cache_rows(f64(k_pages), table[0], 60)
    vv, _ = oa.cache_rows(f64(v_pages), table[0], 60)
    for n in (1, 40):  # both kernels
        q = torch.randn(n, 1, dim, device="cuda", generator=g).half()
        out = torch.empty_like(q)
        hb.hidet_cache_attention(cache, q, out, _ints([0, n]), n)
        want, bound = bounds("f16", f64(q).transpose(1, 0, 2)[None], kk[None], vv[None], oa.sees(n, 60, causal=True)[None], dim ** -0.5)
        assert_within(f64(out).transpose(1, 0, 2)[None], want[0], bound[0], "%d rows" % n)


def test_a_serving_step_captured_and_replayed():
    """rope -> append -> attention of growing sequences, from one graph, against eager calls and the oracle."""
    b = Batch(12, "bf16", [20, 45, 3], [1, 1, 1], 8, 2, 64, 16, width=6)
    table = np.arange(18, dtype=np.int32).reshape(3, 6)
    pages = torch.zeros(2, 18, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    pages.copy_(torch.randn(pages.shape, device="cuda"))
    other = pages.clone()
    b.table = table
    tables, lengths = torch.from_numpy(table).cuda(), _ints([20, 45, 3])
    qkv = torch.randn(3, 12, 64, device="cuda").bfloat16()  # 8 query, 2 key, 2 value heads of every token
    f = hb.hidet_rope_frequencies(64).cuda()
    starts, pos = _ints([0, 1, 2, 3]), torch.zeros(1, 3, dtype=torch.int32, device="cuda")

    def state(p):
        c = hb.make_cache(p[0], p[1], tables, lengths)
        q = torch.empty(3, 8, 64, dtype=torch.bfloat16, device="cuda")
        size = hb.hidet_cache_attention_workspace_bytes(c, q, 1)
        return c, torch.empty(3, 10, 64, dtype=torch.bfloat16, device="cuda"), q, torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    def step(c, qk, out, ws):
        hb.hidet_rope(qkv[:, :10].transpose(0, 1)[None], qk.transpose(0, 1)[None], f, positions=pos)
        hb.hidet_cache_append(c, qk[:, 8:], qkv[:, 10:], starts, 1)
        hb.hidet_cache_attention(c, qk[:, :8], out, starts, 1, workspace=ws)

    eager, captured = state(pages), state(other)
    step(*captured)
    other.copy_(pages)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for t in range(5):
        lengths.add_(1)
        pos.copy_((lengths - 1)[None])
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        graph.replay()
        step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(eager[2], captured[2]) and torch.equal(pages, other), t
        b.lengths, b.new, b.k_pages, b.v_pages = lengths.tolist(), [1, 1, 1], pages[0], pages[1]
        b.check(eager[1][:, :8], eager[2], None, what="step %d" % t)
    side = torch.cuda.Stream()
    out = torch.zeros_like(eager[2])
    hb.hidet_cache_attention(eager[0], eager[1][:, :8], out, starts, 1, workspace=eager[3], stream=side)
    side.synchronize()
    assert torch.equal(out, eager[2])


LAST = 2 ** 31 - 1  # the longest sequence that a length can state


def _one_page_everywhere(new, values):
    """A sequence of 2^31 - 1 tokens of 8 dimensions whose pages are all the same one, of 2^20 slots that hold `values`."""
    page = 1 << 20
    k, v = (torch.from_numpy(x).to(torch.float16).cuda().view(1, page, 1, 8) for x in values)
    cache = hb.make_cache(k, v, torch.zeros(1, 2048, dtype=torch.int32, device="cuda"), _ints([LAST]))
    return cache, k, v, _ints([0, new])


@pytest.mark.parametrize("new,window", [(1, 3000), (1, 33), (3, 50), (2000, 3000)])
def test_windows_at_the_last_positions_that_a_length_can_state(new, window):
    """Tiles of keys that end behind 2^31 - 1 (few rows, and 2000 in tiles of 128): the keys that the queries see are the last ones."""
    g = np.random.Generator(np.random.PCG64(41))
    cache, k, v, starts = _one_page_everywhere(new, [g.standard_normal((1 << 20, 8)).astype(np.float32) for _ in range(2)])
    q = torch.from_numpy(g.standard_normal((new, 2, 8)).astype(np.float32)).half().cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((new, 2), 7.0, device="cuda")
    size = hb.hidet_cache_attention_workspace_bytes(cache, q, new, window)
    ws = torch.full((size // 4 + 4,), float("nan"), device="cuda")
    hb.hidet_cache_attention(cache, q, out, starts, new, lse=lse, window=window, workspace=ws)
    keys = new + window
    slots = (LAST - keys + torch.arange(keys)) % (1 << 20)
    kk, vv = (f64(x[0, :, 0].cpu()[slots])[None, None] for x in (k, v))
    see = oa.sees(new, keys, causal=True, window=window)[None]
    want, bound = bounds("f16", f64(q).transpose(1, 0, 2)[None], kk, vv, see, 8 ** -0.5)
    assert_within(f64(out).transpose(1, 0, 2)[None], want[0], bound[0], "out")
    assert_within(f64(lse).T[None], want[1], bound[1], "lse")


def test_every_key_up_to_the_last_position_that_a_length_can_state():
    """Scores of 0 and values of -1, 0 and 1: weights are 1 and all partial sums whole numbers of fp32, so that the mean is off by the
    divisions and roundings of its end alone (2^-11, and a few of 2^-24)."""
    g = np.random.Generator(np.random.PCG64(42))
    v = g.integers(-1, 2, (1 << 20, 8)).astype(np.float32)
    v[:, 0] = 1.0
    cache, _, _, starts = _one_page_everywhere(1, [np.ones((1 << 20, 8), np.float32), v])
    q = torch.zeros(1, 1, 8, dtype=torch.float16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((1, 1), 7.0, device="cuda")
    size = hb.hidet_cache_attention_workspace_bytes(cache, q, 1)
    assert size > 0
    ws = torch.full((size // 4,), float("nan"), device="cuda")
    hb.hidet_cache_attention(cache, q, out, starts, 1, lse=lse, workspace=ws)
    want = (2048 * v.astype(np.float64).sum(0) - v[-1]) / LAST
    assert np.all(np.abs(f64(out)[0, 0] - want) <= (2.0 ** -11 + 2.0 ** -20) * np.abs(want) + 2.0 ** -25), (f64(out), want)
    assert abs(float(lse[0, 0]) - np.log(LAST)) <= 1e-5


@pytest.mark.parametrize("starts", [[0, 9], [-4, 5], [-4, 9, 2 ** 31 - 1], [0, 3, 9], [-2 ** 31, 2, 2 ** 31 - 1], [1, 4, 70]])
@pytest.mark.parametrize("max_new", [9, 2])
def test_starts_that_leave_the_batch_are_cut_to_it(starts, max_new):
    """5 rows of tokens: append writes those of a sequence to its last positions, counted from the cut starts, where the attention that
    follows looks for them."""
    tokens, seqs, page = 5, len(starts) - 1, 16
    b = Batch(43, "f16", [40, 33][:seqs], [1] * seqs, 2, 1, 64, page)
    b.tokens = tokens
    k, v, q = b.rows(1), b.rows(1), b.rows(2)
    b.starts.copy_(_ints([max(min(x, 2 ** 31 - 1), -2 ** 31) for x in starts]))
    cut = [min(max(x, 0), tokens) for x in starts]
    want = [b.k_pages.clone(), b.v_pages.clone()]
    for s in range(seqs):
        n = cut[s + 1] - cut[s]
        for i in range(min(n, max_new)):
            at = b.lengths[s] - n + i
            for x, new in zip(want, (k, v)):
                x[int(b.table[s, at // page]), at % page] = new[cut[s] + i]
    hb.hidet_cache_append(b.cache, k, v, b.starts, max_new)
    assert torch.equal(b.k_pages, want[0]) and torch.equal(b.v_pages, want[1])
    out, lse = torch.full_like(q, 7.0), torch.full((tokens, 2), 7.0, device="cuda")
    hb.hidet_cache_attention(b.cache, q, out, b.starts, max_new, lse=lse)
    for s in range(seqs):
        n = cut[s + 1] - cut[s]
        rows = slice(cut[s], cut[s] + min(n, max_new))
        kk, vv = (oa.cache_rows(f64(x), b.table[s], b.lengths[s])[0] for x in want)
        see = oa.sees(n, b.lengths[s], causal=True)[:min(n, max_new)]
        if not len(see):
            continue
        w, e = bounds("f16", f64(q[rows]).transpose(1, 0, 2)[None], kk[None], vv[None], see[None], 64 ** -0.5)
        assert_within(f64(out[rows]).transpose(1, 0, 2)[None], w[0], e[0], "sequence %d" % s)
    written = np.zeros(tokens, bool)
    for s in range(seqs):
        written[cut[s]:cut[s] + min(cut[s + 1] - cut[s], max_new)] = True
    assert bool((out[torch.from_numpy(~written).cuda()] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("softcap", [64.0, 1e4, 1e30])
def test_large_caps(softcap, dtype):
    slopes = torch.tensor([0.5, 0.25, 0.125, 1.0], device="cuda")
    for new, dim in (([1, 1, 1], 64), ([200, 3, 77], 128)):
        b = Batch(44, dtype, [300, 1000, 77], new, 4, 2, dim, 16, pad=1)
        for sl in (None, slopes):
            q, out, lse = b.run(softcap=softcap, slopes=sl)
            b.check(q, out, lse, softcap=softcap, slopes=None if sl is None else f64(sl))
    b = _ragged(64, dtype, 64)
    q, out, lse = b.run(softcap=softcap)
    b.check(q, out, lse, softcap=softcap)


@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 128), ("bf16", 40)])
@pytest.mark.parametrize("kind", ["single tokens", "chunks", "long chunks", "pieces"])
def test_values_that_are_not_finite_reach_the_queries_that_see_them_alone(kind, dtype, dim):
    """A dimension in which a query sees infinities or a NaN is their sum, and every other result has the bits that it has without them --
    wherever the pages lie, the one that stands for no page among them."""
    g = np.random.Generator(np.random.PCG64(45))
    if kind == "pieces":
        b = _ragged(45, dtype, dim)
    else:
        new = {"single tokens": [1, 1, 1, 1], "chunks": [200, 3, 77, 40], "long chunks": [300, 3, 77, 500]}[kind]
        b = Batch(45, dtype, [300, 1700, 77, 500], new, 4, 2, dim, 24, pad=1)
        b.table[1, 2] = -1
        b.tables.copy_(torch.from_numpy(b.table))
    before = b.v_pages.clone()
    state = b.g.bit_generator.state
    _, clean, lse_clean = b.run()
    places = [tuple(int(g.integers(n)) for n in before.shape) + ((np.inf, -np.inf, np.nan)[int(g.integers(3))],) for _ in range(200)]
    places += [(0, 1, 0, 3, np.inf), (0, 2, 1, 5, np.nan)]  # (of page 0)
    for p, slot, h, d, x in places:
        b.v_pages[p, slot, h, d] = x
    b.g.bit_generator.state = state
    _, out, lse = b.run()
    assert torch.equal(lse, lse_clean)
    want, group, first = clean.clone(), b.heads // b.kv_heads, 0
    values = f64(b.v_pages)
    for s, (length, n) in enumerate(zip(b.lengths, b.new)):
        vv, there = oa.cache_rows(values, b.table[s], length)
        see = oa.sees(n, length, causal=True) & there[None, :]
        for h in range(b.heads):
            v = np.where(there[:, None], vv[h // group], 0.0)
            for j, d in zip(*np.nonzero(~np.isfinite(v))):
                for i in np.flatnonzero(see[:, j]):
                    old = want[first + i, h, d]
                    want[first + i, h, d] = float(v[j, d]) if bool(torch.isfinite(old)) else old + float(v[j, d])
        first += n
    assert torch.equal(torch.nan_to_num(out, 11.0, 12.0, 13.0), torch.nan_to_num(want, 11.0, 12.0, 13.0))
    assert not torch.equal(torch.nan_to_num(out, 11.0, 12.0, 13.0), clean)
