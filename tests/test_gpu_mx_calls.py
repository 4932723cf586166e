"""The extension module that serves the plain calls of norms, block-scaled matrices and their products against the general path: both
are handed entry points that only write down what they get (nothing runs on the GPU), the refused forms among them."""
import ctypes
import types

import pytest
import torch

from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu

NAMES = ("hidet_rms_norm", "hidet_rms_norm_backward", "hidet_mx_quantize", "hidet_mx_dequantize", "hidet_mx_gemm")
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


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
        monkeypatch.setattr(hb, "_mx_calls", hb._load_mx_calls(stub))

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
    what = "%s(%s)" % (name, ", ".join("%s %s" % (tuple(x.shape), x.dtype) if isinstance(x, torch.Tensor) else repr(x) for x in args))
    public, general = rec.outcome(getattr(hb, name), *args), rec.outcome(getattr(hb, name[5:]), *args)
    assert public == general, what
    rec.calls.clear()
    status = getattr(hb._mx_calls, name[6:])(*args)
    assert (status >= 0) == served and len(rec.calls) == int(served), what
    return public[1]


def t(*shape, dtype=F16, device="cuda"):
    return torch.zeros(shape, dtype=dtype, device=device)


def mx(rows, cols, fmt=0, device="cuda"):
    return hb.make_mx(rows, cols, fmt, device=device)


def test_rms_norm(monkeypatch):
    rec = Recorder(monkeypatch)
    x, w = t(6, 100), t(100)

    def call(x=x, w=w, y=t(6, 100), r=None, s=None, q=None, rstd=None, eps=1e-5, offset=0.0, stream=None):
        return x, w, y, r, s, q, rstd, eps, offset, stream

    wide = t(6, 128)
    for args in (call(), call(r=t(6, 100), s=t(6, 100), rstd=t(6, dtype=F32)), call(y=None, q=mx(6, 100, 2)), call(w=t(100, dtype=F32), eps=0, offset=1),
                 call(x=wide[:, :100], y=wide[:, 20:120]), call(x=t(2, 3, 100), y=t(2, 3, 100), rstd=t(2, 3, dtype=F32)), call(x=t(100), y=t(100)),
                 call(stream=torch.cuda.Stream())):
        assert both(rec, "hidet_rms_norm", args, True) is None
    for args in (call(y=t(6, 99)), call(y=t(6, 100, dtype=BF16)), call(w=t(99)), call(w=t(200)[::2]), call(rstd=t(6)), call(rstd=t(5, dtype=F32)),
                 call(q=mx(6, 101)), call(q=mx(6, 100, device="cpu")), call(x=t(100, 6).t(), y=t(6, 100)), call(x=t(6, 100, device="cpu")),
                 call(y=t(6, 100, device="cpu")), call(x=t(4, 6, 100)[::2, :3], y=t(2, 3, 100))):
        assert both(rec, "hidet_rms_norm", args, False) is not None


def test_rms_norm_backward(monkeypatch):
    rec = Recorder(monkeypatch)

    def call(gy=t(6, 100), h=t(6, 100), rstd=t(6, dtype=F32), w=t(100), gh=t(6, 100), gw=t(100), ws=t(64), gs=None, offset=0.0, stream=None):
        return gy, h, rstd, w, gh, gw, ws, gs, offset, stream

    for args in (call(), call(gs=t(6, 100), offset=1.0), call(gw=None, ws=None), call(w=t(100, dtype=F32), gw=t(100, dtype=F32))):
        assert both(rec, "hidet_rms_norm_backward", args, True) is None
    for args in (call(rstd=t(6)), call(gy=t(5, 100)), call(gw=t(100, dtype=F32)), call(gw=t(99)), call(ws=t(64, 4)[:, :2]), call(gh=t(6, 100, dtype=F32)),
                 call(w=t(100, device="cpu"))):
        assert both(rec, "hidet_rms_norm_backward", args, False) is not None


def test_quantize_and_dequantize(monkeypatch):
    rec = Recorder(monkeypatch)
    for args in ((t(5, 70), mx(5, 70), None, None), (t(5, 70, dtype=F32), None, mx(70, 5, 1), None), (t(5, 96)[:, 3:73], mx(5, 70, 2), mx(70, 5, 0), None)):
        assert both(rec, "hidet_mx_quantize", args, True) is None
    for args in ((t(5, 70), mx(70, 5), None, None), (t(5, 70), None, mx(5, 70), None), (t(70, 5).t(), mx(5, 70), None, None), (t(5, 7, 10), mx(5, 70), None, None),
                 (t(5, 70, dtype=torch.float64), mx(5, 70), None, None), (t(5, 70), mx(5, 70, device="cpu"), None, None)):
        assert both(rec, "hidet_mx_quantize", args, False) is not None
    for y, ok in ((t(5, 70), True), (t(5, 96, dtype=BF16)[:, 1:71], True), (t(5, 71), False), (t(70, 5).t(), False), (t(5, 70, device="cpu"), False)):
        assert (both(rec, "hidet_mx_dequantize", (mx(5, 70, 2), y, None), ok) is None) == ok


def test_gemm(monkeypatch):
    rec = Recorder(monkeypatch)
    a, b = mx(6, 100, 0), mx(9, 100, 2)
    e = hb.make_epilogue(bias=t(9), bias_axis=hb.HIDET_BIAS_PER_COL, residual=t(6, 9), relu=True)
    for args in ((a, b, t(6, 9), None, None, None), (a, b, t(6, 16, dtype=BF16)[:, 2:11], None, t(64), None), (a, b, t(6, 9), e, None, None),
                 (a, b, t(6, 9), None, None, torch.cuda.Stream())):
        assert both(rec, "hidet_mx_gemm", args, True) is None
    # (another device's bias; a head-split map is the library's to refuse, through the general path)
    cpu = hb.make_epilogue(bias=t(9, device="cpu"), bias_axis=hb.HIDET_BIAS_PER_COL)
    for x, axis in ((t(6), hb.HIDET_BIAS_PER_COL), (t(9), hb.HIDET_BIAS_PER_ROW), (t(9, dtype=F32), hb.HIDET_BIAS_PER_COL)):
        assert both(rec, "hidet_mx_gemm", (a, b, t(6, 9), hb.make_epilogue(bias=x, bias_axis=axis), None, None), False) is not None
    for r in (t(5, 9), t(6, 9, dtype=BF16)):
        assert both(rec, "hidet_mx_gemm", (a, b, t(6, 9), hb.make_epilogue(residual=r), None, None), False) is not None
    for args in ((a, b, t(6, 8), None, None, None), (a, mx(9, 99), t(6, 9), None, None, None), (a, b, t(9, 6).t(), None, None, None), (a, b, t(54), None, None, None),
                 (a, b, t(6, 9), cpu, None, None), (a, b, t(6, 9), None, t(64, 4)[:, :2], None), (a, mx(9, 100, device="cpu"), t(6, 9), None, None, None)):
        assert both(rec, "hidet_mx_gemm", args, False) is not None
    assert both(rec, "hidet_mx_gemm", (a, b, t(6, 9), hb.make_epilogue(head_split=(3, 3)), None, None), False) is None


def test_a_status_is_raised_once(monkeypatch):
    rec = Recorder(monkeypatch, status=2)
    with pytest.raises(hb.HidetError) as e:
        hb.hidet_mx_quantize(t(5, 70), by_rows=mx(5, 70))
    assert e.value.status == 2 and len(rec.calls) == 1
