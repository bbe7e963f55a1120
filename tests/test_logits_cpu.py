"""The calls on logits without a GPU: what they refuse (nothing is launched, the addresses passed are
never read), and that empty calls are fine."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

INV = 1


@pytest.fixture(scope="module")
def emo():
    from paper_2607_12324_amd import emo as mod
    return mod


F32, F16, BF16, U8, I32, I64 = range(6)
SIZE = {F32: 4, F16: 2, BF16: 2, U8: 1, I32: 4, I64: 8}


class Memory:
    """Addresses of pretended device buffers, apart from each other."""

    def __init__(self, emo):
        self.emo, self.next = emo, 1 << 32

    def __call__(self, rows, cols, dtype=F32, row_stride=None, col_stride=1, data=None):
        rs = cols if row_stride is None else row_stride
        if data is None:
            data, self.next = self.next, self.next + ((max(rows * rs, 1) * SIZE[dtype] + 4095) // 4096 + 1) * 4096
        return self.emo.Tensor(data, rows, cols, rs, col_stride, dtype, 0)


@pytest.fixture
def mem(emo):
    return Memory(emo)


def ref(t):
    return None if t is None else ctypes.byref(t)


ADJUST = ("logits", "history", "lengths", "repetition", "frequency", "presence", "bias", "inv_temperature", "mask", "noise",
          "out", "choice")


def adjust(emo, rows, vocab, ws=None, size=0, **kw):
    return emo.lib.emo_adjust_logits(rows, vocab, *[ref(kw.get(k)) for k in ADJUST], ws, size, None)


def refused(emo, status, *words):
    assert status == INV, status
    text = emo.lib.emo_last_error().decode()
    for w in words:
        assert w in text, text


def test_adjust_refuses(emo, mem):
    R, V = 6, 100
    ok = {"logits": mem(R, V), "out": mem(R, V)}
    W = (V + 31) // 32

    def bad(words, rows=R, vocab=V, **kw):
        refused(emo, adjust(emo, rows, vocab, **{**ok, **kw}), *words)

    bad(["rows"], rows=-1)
    bad(["rows"], rows=1 << 31)
    bad(["vocab"], vocab=0)
    bad(["vocab"], vocab=1 << 31)
    bad(["logits"], logits=None)
    bad(["logits", "type"], logits=mem(R, V, I32))
    bad(["logits", "columns"], logits=mem(R, V - 1))
    bad(["logits", "divide"], logits=mem(4, V))
    bad(["logits", "divide"], logits=mem(2 * R, V))
    bad(["logits", "divide"], logits=mem(0, V))
    bad(["logits", "col_stride"], logits=mem(R, V, row_stride=2 * V, col_stride=2))
    bad(["logits", "strides"], logits=mem(R, V, row_stride=-V))
    bad(["logits", "strides"], logits=mem(R, V, row_stride=1 << 41, data=1 << 33))
    bad(["logits", "aligned"], logits=mem(R, V, data=(1 << 33) + 2))
    bad(["logits", "no data"], logits=mem(R, V, data=0))
    bad(["type"], logits=emo.Tensor(1 << 33, R, V, V, 1, 7, 0))
    bad(["type"], logits=emo.Tensor(1 << 33, R, V, V, 1, -1, 0))
    bad(["mask", "columns"], mask=mem(R, W + 1, I32))
    bad(["mask", "type"], mask=mem(R, W, I64))
    bad(["bias", "type"], bias=mem(1, V, BF16))
    bad(["noise", "columns"], noise=mem(1, 1))
    bad(["history"], lengths=mem(R, 1, I32))
    bad(["history"], repetition=mem(R, 1))
    bad(["history"], frequency=mem(R, 1))
    bad(["history"], presence=mem(R, 1))
    bad(["history", "type"], history=mem(R, 9))
    bad(["history", "columns"], history=mem(1, (1 << 30) + 1, I32, row_stride=0, col_stride=0, data=1 << 33))
    bad(["lengths", "type"], history=mem(R, 9, I32), lengths=mem(R, 1, I64))
    bad(["presence", "columns"], history=mem(R, 9, I32), presence=mem(R, 2))
    bad(["inv_temperature", "divide"], inv_temperature=mem(4, 1))
    bad(["out", "rows"], out=mem(1, V))
    bad(["out", "overlap"], out=mem(R, V, row_stride=V - 1))
    bad(["out", "overlap"], out=mem(R, V, row_stride=0))
    bad(["out", "type"], out=mem(R, V, F16))
    bad(["out", "type"], out=mem(R, V, I32))
    bad(["choice", "type"], choice=mem(R, 1, F32))
    bad(["choice", "rows"], choice=mem(1, 1, I32))
    bad(["choice", "overlap"], choice=mem(R, 1, I32, row_stride=0))
    refused(emo, adjust(emo, R, 256, logits=mem(R, 256), choice=mem(R, 1, U8)), "byte")


def test_reserved_fields_are_zero(emo, mem):
    """A record that was not cleared is refused, whichever operand it is."""
    R, V = 6, 100
    W = (V + 31) // 32
    kw = {"logits": mem(R, V), "history": mem(R, 9, I32), "lengths": mem(R, 1, I32), "repetition": mem(R, 1), "frequency": mem(R, 1),
          "presence": mem(R, 1), "bias": mem(1, V), "inv_temperature": mem(R, 1), "mask": mem(R, W, I32), "noise": mem(R, V),
          "out": mem(R, V), "choice": mem(R, 1, I32)}
    for k, t in kw.items():
        t.reserved = 1
        refused(emo, adjust(emo, R, V, **kw), k, "reserved")
        t.reserved = 0


def test_adjust_refuses_overlaps(emo, mem):
    R, V = 6, 100
    x = mem(R, V)
    one = mem(1, V)
    for kw in ({"logits": x, "out": emo.Tensor(x.data + 4, R, V, V, 1, F32, 0)},           # shifted by an element
               {"logits": x, "out": emo.Tensor(x.data, R, V, V + 1, 1, F32, 0)},           # another stride
               {"logits": mem(R, V, F16, data=x.data), "out": x},                          # another type
               {"logits": one, "out": emo.Tensor(one.data, R, V, V, 1, F32, 0)},           # repeated rows
               {"logits": x, "bias": emo.Tensor(1 << 34, 1, V, V, 1, F32, 0), "out": emo.Tensor(1 << 34, R, V, V, 1, F32, 0)},
               {"logits": x, "choice": emo.Tensor(x.data + 8, R, 1, 1, 1, I32, 0)},
               {"logits": x, "out": emo.Tensor(1 << 34, R, V, V, 1, F32, 0), "choice": emo.Tensor(1 << 34, R, 1, 1, 1, I32, 0)}):
        refused(emo, adjust(emo, R, V, **kw), "overlaps")


def test_adjust_in_place_frees_no_other_operand(emo, mem):
    """The adjusted logits may be the logits, not the noise or the bias, whichever records describe them."""
    R, V = 6, 100
    x = mem(R, V)
    again = emo.Tensor(x.data, R, V, V, 1, F32, 0)
    choice = mem(R, 1, I32)
    for out in (x, again):
        for other in (x, again):
            refused(emo, adjust(emo, R, V, logits=x, noise=other, out=out, choice=choice), "out overlaps noise")
            refused(emo, adjust(emo, R, V, logits=x, bias=other, out=out, choice=choice), "out overlaps bias")
            refused(emo, adjust(emo, R, V, logits=mem(R, V), noise=other, out=out, choice=choice), "out overlaps noise")


DIST = ("logits", "ids", "teacher")


def forward(emo, rows, vocab, t, tau=1.0, mask=None, loss=None, stats=None, ws=None, size=0):
    return emo.lib.emo_distill_forward(rows, vocab, *[ref(t.get(k)) for k in DIST], tau, ref(mask), ref(loss), ref(stats), ws, size, None)


def backward(emo, rows, vocab, t, tau=1.0, stats=None, scale=None, mask=None, grad=None):
    return emo.lib.emo_distill_backward(rows, vocab, ref(t["logits"]), ref(stats), ref(t["ids"]), ref(t["teacher"]), tau, ref(scale),
                                        ref(mask), ref(grad), None)


def step(emo, rows, vocab, t, tau=1.0, scale=None, mask=None, loss=None, grad=None, ws=None, size=0):
    return emo.lib.emo_distill_step(rows, vocab, *[ref(t.get(k)) for k in DIST], tau, ref(scale), ref(mask), ref(loss), ref(grad), ws,
                                    size, None)


def test_distill_refuses(emo, mem):
    N, V, K = 6, 100, 5
    t = {"logits": mem(N, V), "ids": mem(N, K, I32), "teacher": mem(N, K)}
    loss, stats, grad = mem(N, 1), mem(N, 2), mem(N, V)
    calls = (lambda u, **kw: forward(emo, kw.pop("rows", N), kw.pop("vocab", V), u, loss=loss, stats=stats, **kw),
             lambda u, **kw: backward(emo, kw.pop("rows", N), kw.pop("vocab", V), u, stats=stats, grad=grad, **kw),
             lambda u, **kw: step(emo, kw.pop("rows", N), kw.pop("vocab", V), u, loss=loss, grad=grad, **kw))
    for call in calls:
        for tau in (0.0, -1.0, 1e-30, 1e30, float("inf"), float("nan")):
            refused(emo, call(t, tau=tau), "temperature")
        refused(emo, call(t, rows=-1), "rows")
        refused(emo, call(t, vocab=0), "vocab")
        for k in DIST:
            refused(emo, call({**t, k: None}), "NULL")
        refused(emo, call({**t, "logits": mem(3, V)}), "logits", "rows")
        refused(emo, call({**t, "ids": mem(N, 1025, I32)}), "ids", "1025")
        refused(emo, call({**t, "ids": mem(N, K)}), "ids", "type")
        refused(emo, call({**t, "ids": mem(4, K, I32)}), "ids", "divide")
        refused(emo, call({**t, "teacher": mem(N, K + 1)}), "teacher", "columns")
        refused(emo, call({**t, "teacher": mem(N, K, I32)}), "teacher", "type")
        refused(emo, call(t, mask=mem(N, 3, I32)), "mask", "columns")
    refused(emo, forward(emo, N, V, t, loss=mem(1, 1)), "loss", "rows")
    refused(emo, forward(emo, N, V, t, loss=loss, stats=mem(N, 1)), "stats", "columns")
    refused(emo, forward(emo, N, V, t, loss=loss, stats=mem(N, 2, data=loss.data)), "overlaps")
    refused(emo, backward(emo, N, V, t, stats=None, grad=grad), "NULL")
    refused(emo, backward(emo, N, V, t, stats=stats, grad=None), "NULL")
    refused(emo, backward(emo, N, V, t, stats=mem(1, 2), grad=grad), "stats", "rows")
    refused(emo, backward(emo, N, V, t, stats=stats, grad=mem(N, V, BF16)), "gradient", "type")
    refused(emo, backward(emo, N, V, t, stats=stats, grad=grad, scale=mem(4, 1)), "scale", "divide")
    refused(emo, step(emo, N, V, t, loss=loss, grad=None), "NULL")
    refused(emo, step(emo, N, V, t, grad=mem(N, V, data=t["logits"].data + 4)), "overlaps")
    refused(emo, step(emo, N, V, t, grad=mem(N, V, data=t["teacher"].data)), "overlaps")


def test_distill_in_place_frees_no_other_operand(emo, mem):
    """The gradient may be the logits, not the teacher, whichever records describe them."""
    N, V = 6, 5
    x = mem(N, V)
    again = emo.Tensor(x.data, N, V, V, 1, F32, 0)
    for grad in (x, again):
        for teacher in (x, again):
            t = {"logits": x, "ids": mem(N, V, I32), "teacher": teacher}
            refused(emo, step(emo, N, V, t, loss=mem(N, 1), grad=grad), "gradient overlaps teacher")
            refused(emo, backward(emo, N, V, t, stats=mem(N, 2), grad=grad), "gradient overlaps teacher")


def test_outputs_between_the_rows_of_others(emo, mem):
    """What shares no byte is no overlap.  Another type than the logits' in the output, looked for after the
    overlaps, keeps the accepted layouts from being run."""
    R, V, at = 6, 100, 1 << 33

    def out(logits, data, row_stride, words, rows=R, **kw):
        t = emo.Tensor(data, rows, V, row_stride, 1, F16, 0)
        refused(emo, adjust(emo, rows, V, logits=logits, out=t, **kw), *words)

    apart, meet = ("out must have the logits' type",), ("out overlaps",)
    half = emo.Tensor(at, R, V, 2 * V, 1, F32, 0)
    out(half, at + 4 * V, 4 * V, apart)                             # the right half of the logits' rows
    out(half, at + 6 * V, 4 * V, apart)                             # its last 2 V bytes
    out(half, at + 6 * V + 2, 4 * V, meet)                          # 2 bytes into the next row's logits
    out(half, at + 4 * V - 2, 4 * V, meet)
    out(half, at - 4 * V, 4 * V, apart)                             # the half before the first row
    out(half, at - 2 * V, 4 * V, apart)
    out(half, at - 2 * V + 2, 4 * V, meet)
    out(half, at + 4 * V, 4 * V + 2, meet)                          # the strides drift
    out(half, at + 4 * V, 8 * V, apart)                             # every other row's right half
    out(half, at + 4 * V, 2 * V, meet)                              # twice as many rows as the buffer's
    out(emo.Tensor(at, 1, V, V, 1, F32, 0), at + 4 * V, 4 * V, apart)
    out(emo.Tensor(at, 1, V, V, 1, F32, 0), at - 4 * V, 4 * V, apart)   # one row in the others' gap
    out(emo.Tensor(at, 1, V, V, 1, F32, 0), at - 2 * V, 4 * V, apart)
    out(emo.Tensor(at, 1, V, V, 1, F32, 0), at - 2 * V + 2, 4 * V, meet)
    out(emo.Tensor(at, 1, V, V, 1, F32, 0), at, 4 * V, meet)
    # a history read through a transposed view of the buffer's last rows, and one that the output's rows cross
    half16 = emo.Tensor(at, R, 9, 1, 4 * V, I32, 0)
    rate = mem(R, 1)
    out(mem(R, V), at + 64, 8 * V, apart, history=half16, presence=rate)
    out(mem(R, V), at + 20, 8 * V, meet, history=half16, presence=rate)
    # the elements of two by turns
    turns = emo.Tensor(at, R, 9, 18, 2, I32, 0)
    choice = emo.Tensor(at + 4, R, 1, 18, 1, I32, 0)
    refused(emo, adjust(emo, R, V, logits=mem(R, V), history=turns, presence=rate, choice=choice, out=mem(R, V, F16)), *apart)
    choice = emo.Tensor(at + 8, R, 1, 18, 1, I32, 0)
    refused(emo, adjust(emo, R, V, logits=mem(R, V), history=turns, presence=rate, choice=choice, out=mem(R, V, F16)), "choice overlaps")
    # a workspace among the elements of a strided column, and in the gap between two rows
    long, n = 1 << 22, ctypes.c_int64(0)
    assert emo.lib.emo_adjust_workspace(R, long, ctypes.byref(n)) == 0 and n.value > 64
    kw = {"logits": mem(R, long), "ws": at, "size": n.value}
    refused(emo, adjust(emo, R, long, choice=emo.Tensor(at + 8, R, 1, 2, 1, I64, 0), **kw), "overlaps")
    refused(emo, adjust(emo, R, long, choice=emo.Tensor(at - 8, R, 1, (n.value + 15) // 8, 1, I64, 0), out=mem(R, long, F16), **kw), *apart)
    t = {"logits": half, "ids": mem(R, 5, I32), "teacher": mem(R, 5)}
    for data, words in ((at + 4 * V, "type"), (at + 4 * V - 2, "overlaps")):
        g = emo.Tensor(data, R, V, 4 * V, 1, F16, 0)
        refused(emo, step(emo, R, V, t, loss=mem(R, 1), grad=g), words)
        refused(emo, backward(emo, R, V, t, stats=mem(R, 2), grad=g), words)


def test_workspaces(emo, mem):
    n = ctypes.c_int64(-1)
    for fn in (emo.lib.emo_adjust_workspace, emo.lib.emo_distill_workspace):
        refused(emo, fn(1, 1, None), "bytes")
        refused(emo, fn(-1, 1, ctypes.byref(n)), "rows")
        refused(emo, fn(1, 0, ctypes.byref(n)), "vocab")
        for rows, vocab in ((0, 1), (1, 1), (1, 1 << 20), (1, (1 << 31) - 1), (4096, 131072), ((1 << 31) - 1, 16)):
            assert fn(rows, vocab, ctypes.byref(n)) == 0 and 0 <= n.value <= 1 << 26
    # a call that needs one refuses to go without, with too little, misaligned, or overlapping its operands
    rows, V = 1, 1 << 22
    x = mem(rows, V)
    assert emo.lib.emo_adjust_workspace(rows, V, ctypes.byref(n)) == 0
    need = n.value
    if need:
        kw = {"logits": x, "choice": mem(rows, 1, I64)}
        refused(emo, adjust(emo, rows, V, **kw), "workspace")
        refused(emo, adjust(emo, rows, V, ws=1 << 40, size=need - 1, **kw), "workspace")
        refused(emo, adjust(emo, rows, V, ws=(1 << 40) + 8, size=need, **kw), "workspace", "aligned")
        refused(emo, adjust(emo, rows, V, ws=x.data + 64, size=need, **kw), "overlaps")
    assert emo.lib.emo_distill_workspace(rows, V, ctypes.byref(n)) == 0
    need = n.value
    if need:
        t = {"logits": x, "ids": mem(rows, 5, I32), "teacher": mem(rows, 5)}
        refused(emo, forward(emo, rows, V, t, loss=mem(rows, 1)), "workspace")
        refused(emo, step(emo, rows, V, t, loss=mem(rows, 1), grad=mem(rows, V), ws=1 << 40, size=need - 1), "workspace")
        refused(emo, step(emo, rows, V, t, grad=mem(rows, V), ws=t["teacher"].data, size=need), "overlaps")


def test_empty_calls(emo, mem):
    t = {"logits": mem(0, 7), "ids": mem(0, 3, I32), "teacher": mem(0, 3)}
    assert adjust(emo, 0, 7, logits=mem(0, 7), out=mem(0, 7)) == 0
    assert adjust(emo, 5, 7, logits=mem(5, 7)) == 0                    # no output asked for
    assert forward(emo, 0, 7, t, loss=mem(0, 1), stats=mem(0, 2)) == 0
    assert backward(emo, 0, 7, t, stats=mem(0, 2), grad=mem(0, 7)) == 0
    assert step(emo, 0, 7, t, loss=mem(0, 1), grad=mem(0, 7)) == 0


def test_binding_refuses_host_tensors(emo):
    import torch
    x = torch.zeros((2, 3))
    for call in (lambda: emo.adjust_logits(x), lambda: emo.distill_forward(x, x, x), lambda: emo.distill_step(x, x, x),
                 lambda: emo.distill_backward(x, x, x, x)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="rows"):
        emo.adjust_logits(x[0])
    assert ctypes.sizeof(emo.Tensor) == 48 and np.dtype(np.int64).itemsize == 8


@pytest.mark.parametrize("source", ["emo_logits.hip", "emo_distill.hip"])
def test_no_access_claims_an_alignment_that_rows_lack(source):
    """Rows start at any element: a pointer into one is never taken for a more aligned one."""
    from paper_2607_12324_amd import build as b
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *b.HIPCC_FLAGS, "-I", b.INCLUDE, "-I", b.CSRC, "--cuda-device-only",
           "-fsyntax-only", "-Werror=align-mismatch", os.path.join(b.CSRC, source)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
