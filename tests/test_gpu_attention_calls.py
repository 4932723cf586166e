"""The extension module that serves the plain calls of attention, rotary positions and the cache against the general path: both are
handed entry points that only write down what they get (nothing runs on the GPU), over every form of tensors and options, the
refused ones among them."""
import ctypes
import types

import pytest
import torch

from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu

NAMES = ("hidet_attention", "hidet_attention_backward", "hidet_attention_ranges", "hidet_rope", "hidet_cache_append", "hidet_cache_attention")
F16, BF16, F32, I32 = torch.float16, torch.bfloat16, torch.float32, torch.int32


class Recorder:
    """Structures are handed over by pointers of their own type: what they hold is read while the call lasts."""

    def __init__(self, monkeypatch, status=0):
        real, self.calls, self.status, self.keep = hb.lib(), [], status, []
        stub = types.SimpleNamespace(hidet_status_string=real.hidet_status_string)
        for name in NAMES:
            fn = ctypes.CFUNCTYPE(ctypes.c_int32, *getattr(real, name).argtypes)(lambda *a, name=name: self.write(name, a))
            self.keep.append(fn)
            setattr(stub, name, fn)
        monkeypatch.setattr(hb, "_lib", stub)
        monkeypatch.setattr(hb, "_attention_calls", hb._load_attention_calls(stub))

    def write(self, name, args):
        self.calls.append((name, tuple((bytes(a.contents) if a else None) if isinstance(a, ctypes._Pointer) else a for a in args)))
        return self.status

    def outcome(self, f, *args):
        self.calls.clear()
        try:
            f(*args)
            raised = None
        except Exception as e:
            raised = (type(e), str(e))
        return list(self.calls), raised


def both(rec, name, args, served):
    """What the public function and the general path do; `served`: whether the extension module has to take the call, or leave it."""
    fast = getattr(hb._attention_calls, name[6:])
    what = "%s(%s)" % (name, ", ".join("%s%s %s" % (type(x).__name__, tuple(x.shape), x.dtype) if isinstance(x, torch.Tensor) else repr(x) for x in args))
    public = rec.outcome(getattr(hb, name), *args)
    general = rec.outcome(getattr(hb, name[5:]), *args)
    same = public == general
    assert same, what
    rec.calls.clear()
    status = fast(*args)
    assert (status >= 0) == served, what
    assert len(rec.calls) == int(served), what
    return public[1]


def t(*shape, dtype=F16, device="cuda"):
    return torch.zeros(shape, dtype=dtype, device=device)


def changed(args, i, x):
    return args[:i] + (x,) + args[i + 1:]


def refused(rec, name, args, at):
    """Each wrong argument: refused by both alike, or left to the general path."""
    for i, x in at:
        both(rec, name, changed(args, i, x), False)


def test_attention(monkeypatch):
    rec = Recorder(monkeypatch)
    q, k, v, out = t(2, 4, 5, 16), t(2, 2, 7, 16), t(2, 2, 7, 16), t(2, 4, 5, 16)
    plain = (q, k, v, out, None, None, False, 0, 0.0, None, None, None, None)
    full = (q, k, v, out, t(2, 4, 5, dtype=F32), 0.5, True, 3, 30, t(4, dtype=F32), t(2, 5, 2, dtype=I32), t(64, dtype=F32), torch.cuda.Stream())
    for args in (plain, full, changed(plain, 5, 2), changed(plain, 7, 1 << 40)):
        assert both(rec, "hidet_attention", args, True) is None
    both(rec, "hidet_attention", changed(plain, 6, 1), False)  # (flags are bools)
    tokens = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    wide = t(2, 4, 5, 40)[..., 3:19]
    for x in (tokens(q), wide, t(2, 4, 5, 16, dtype=F16), q[:1].expand(2, 4, 5, 16), torch.nn.Parameter(q)):
        assert both(rec, "hidet_attention", changed(plain, 0, x), True) is None
    for dim in range(1, 130):  # (the scale that is not given)
        a, b = t(1, 1, 1, dim), t(1, 1, 2, dim)
        assert both(rec, "hidet_attention", (a, b, b, a) + plain[4:], True) is None
    for dtype in (BF16, F32):
        a, b = t(2, 4, 5, 16, dtype=dtype), t(2, 2, 7, 16, dtype=dtype)
        assert both(rec, "hidet_attention", (a, b, b, a) + plain[4:], True) is None
    refused(rec, "hidet_attention", full, [
        (0, t(2, 4, 5, 16, dtype=BF16)), (0, t(2, 4, 5, 16, dtype=torch.float64)), (0, t(4, 5, 16)), (0, t(2, 4, 5, 32)[..., ::2]), (0, q.cpu()),
        (1, t(2, 2, 8, 16)), (1, t(3, 2, 7, 16)), (1, t(2, 2, 7, 8)), (2, t(2, 2, 7, 16, dtype=BF16)), (3, t(2, 4, 6, 16)), (3, out.cpu()),
        (4, t(2, 4, 5)), (4, t(2, 5, 4, dtype=F32).transpose(1, 2)), (4, t(2, 4, 6, dtype=F32)), (5, "scale"), (6, "causal"), (7, 1.5), (8, None),
        (9, t(5, dtype=F32)), (9, t(4)), (9, t(8, dtype=F32)[::2]), (10, t(2, 5, 2)), (10, t(2, 5, 2, dtype=I32).cpu()), (10, t(2, 6, 2, dtype=I32)),
        (11, t(128, dtype=F32)[::2]), (11, t(1, dtype=F32).expand(1 << 20)), (11, t(64, device="cpu")), (0, None), (0, 7)])
    assert both(rec, "hidet_attention", changed(full, 11, t(64, dtype=torch.int8)), True) is None
    with torch.cuda.stream(torch.cuda.Stream()):  # (the current stream)
        assert both(rec, "hidet_attention", plain, True) is None
    monkeypatch.undo()
    assert both(Recorder(monkeypatch, status=3), "hidet_attention", plain, True)[0] is hb.HidetError


def test_attention_backward(monkeypatch):
    rec = Recorder(monkeypatch)
    q, k = t(2, 4, 5, 16), t(2, 2, 7, 16)
    args = (q.clone(), q, k, k.clone(), q.clone(), t(2, 4, 5, dtype=F32), q.clone(), k.clone(), k.clone(), t(64, dtype=F32), None, True, 0, 0.0,
            None, None, None)
    for a in (args, changed(args, 14, t(4, dtype=F32)), changed(changed(args, 11, False), 15, t(2, 5, 2, dtype=I32)), changed(args, 10, 0.25),
              changed(args, 5, None), changed(args, 9, None), changed(args, 16, torch.cuda.Stream())):
        assert both(rec, "hidet_attention_backward", a, True) is None
    for i in (0, 1, 4, 6):
        assert both(rec, "hidet_attention_backward", changed(args, i, t(2, 5, 4, 16).transpose(1, 2)), True) is None
        refused(rec, "hidet_attention_backward", args, [(i, t(2, 4, 6, 16)), (i, t(2, 4, 5, 16, dtype=BF16)), (i, q.cpu()), (i, None)])
    for i in (2, 3, 7, 8):
        assert both(rec, "hidet_attention_backward", changed(args, i, t(2, 7, 2, 16).transpose(1, 2)), True) is None
        refused(rec, "hidet_attention_backward", args, [(i, t(2, 2, 6, 16)), (i, t(2, 2, 7, 16, dtype=BF16)), (i, t(2, 2, 7, 32)[..., ::2])])
    refused(rec, "hidet_attention_backward", args, [(5, t(2, 4, 5)), (9, t(64, dtype=F32)[::2]), (14, t(3, dtype=F32)), (15, t(2, 4, 2, dtype=I32))])


def test_ranges(monkeypatch):
    rec = Recorder(monkeypatch)
    args = (t(2, 5, 2, dtype=I32), 9, t(2, 9, dtype=I32), t(2, dtype=I32), True, 0, None)
    for a in (args, changed(args, 2, None), changed(args, 3, None), changed(args, 6, torch.cuda.Stream()), changed(args, 5, 4)):
        assert both(rec, "hidet_attention_ranges", a, True) is None
    refused(rec, "hidet_attention_ranges", args, [(0, t(2, 5, 3, dtype=I32)), (0, t(2, 5, 2)), (0, t(5, 2, dtype=I32)), (1, 8), (1, 9.0), (0, None),
                                                  (2, t(2, 9)), (2, t(9, 2, dtype=I32).t()), (2, t(2, 9, dtype=I32).cpu()), (3, t(3, dtype=I32))])


def test_rope(monkeypatch):
    rec = Recorder(monkeypatch)
    x, f = t(2, 4, 5, 16), t(8, dtype=torch.float64)
    args = (x, x, f, None, 0, False, False, 1.0, None)
    for a in (args, changed(args, 3, t(2, 5, dtype=I32)), changed(args, 3, t(5, dtype=I32)), changed(args, 3, t(2, 9, dtype=I32)[:, 2:7]),
              changed(args, 4, 1 << 30), changed(args, 5, True), changed(args, 6, True), changed(args, 7, 2), changed(args, 1, t(2, 5, 4, 16).transpose(1, 2)),
              changed(args, 2, t(0, dtype=torch.float64)), changed(args, 8, torch.cuda.Stream())):
        assert both(rec, "hidet_rope", a, True) is None
    refused(rec, "hidet_rope", args, [(0, t(2, 4, 6, 16)), (0, t(2, 4, 5, 16, dtype=BF16)), (1, t(4, 5, 16)), (2, t(8, dtype=F32)), (2, f.cpu()),
                                      (2, t(16, dtype=torch.float64)[::2]), (3, t(2, 6, dtype=I32)), (3, t(3, 5, dtype=I32)), (3, t(2, 5)),
                                      (3, t(2, 10, dtype=I32)[:, ::2]), (4, 0.5), (7, "one")])


def _cache(device="cuda", dtype=F16):
    return hb.make_cache(t(6, 4, 2, 16, dtype=dtype, device=device), t(6, 4, 2, 16, dtype=dtype, device=device), t(3, 2, dtype=I32, device=device),
                         t(3, dtype=I32, device=device))


def test_cache(monkeypatch):
    rec = Recorder(monkeypatch)
    cache, starts = _cache(), t(4, dtype=I32)
    append = (cache, t(5, 2, 16), t(5, 2, 16), starts, 3, None)
    attend = (cache, t(5, 4, 16), t(5, 4, 16), starts, 3, None, 0, 0.0, None, None, None, None)
    for a in (append, changed(append, 1, t(5, 40)[:, 4:36].view(5, 2, 16)), changed(append, 5, torch.cuda.Stream())):
        assert both(rec, "hidet_cache_append", a, True) is None
    for a in (attend, changed(attend, 5, 0.3), changed(attend, 6, 9), changed(attend, 7, 2.0), changed(attend, 8, t(4, dtype=F32)),
              changed(attend, 9, t(5, 4, dtype=F32)), changed(attend, 10, t(64, dtype=F32)), changed(attend, 11, torch.cuda.Stream())):
        assert both(rec, "hidet_cache_attention", a, True) is None
    bad = [(1, t(5, 4, 8)), (1, t(5, 2, 16, dtype=BF16)), (1, t(2, 5, 2, 16)), (2, t(6, 2, 16)), (2, t(5, 4, 32)[..., ::2]), (3, t(5, dtype=I32)),
           (3, t(4)), (3, starts.cpu()), (4, 1.5), (0, _cache("cpu")), (0, _cache(dtype=BF16))]
    refused(rec, "hidet_cache_append", append, bad + [(1, t(5, 3, 16))])
    refused(rec, "hidet_cache_attention", attend, bad + [(8, t(3, dtype=F32)), (9, t(5, 4)), (10, t(64, dtype=F32)[::2]), (10, t(64, device="cpu"))])


def test_pages_on_another_device_than_the_tables_are_refused():
    cache = hb.make_cache(t(6, 4, 2, 16), t(6, 4, 2, 16), t(3, 2, dtype=I32, device="cpu"), t(3, dtype=I32))
    with pytest.raises(ValueError, match="on the GPU"):
        hb.hidet_cache_append(cache, t(5, 2, 16), t(5, 2, 16), t(4, dtype=I32), 3)
