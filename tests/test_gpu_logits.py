"""Calls on logits on the GPU against the oracle (needs an MI355X).

Adjusted logits and choices are compared to the bit.  Distillation is compared with fp64 within bounds
made of the roundings its fp32 sums do (EPS = 2^-24, half a step of fp32):
  s      a sum of V exponentials: at most V / 256 + 64 additions follow each other (a thread's share, then
         waves and workgroups), each exponential is off by 3 roundings of its argument d / tau (which counts
         e^-|d| |d| <= 1 of it) and one step;
  loss   log s and the distances are each off by a rounding or two of their own size, a probability by
         K + 8 roundings and 3 of its argument;
  grad   q by s's error, 3 roundings of its own argument and 4 of its value, p likewise; then the output
         type's half step.
"""
import numpy as np
import pytest

from oracle import logits as orc

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


@pytest.fixture(scope="module")
def emo(torch):
    from paper_2607_12324_amd import emo as mod
    return mod


def types(torch):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "u8": torch.uint8, "i32": torch.int32,
            "i64": torch.int64}


def dev(torch, a, dtype=None, stride=None, offset=0):
    """A device tensor of a [n, V] array, its rows `stride` elements apart, `offset` elements in; the memory
    around it holds NaN (or -1)."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a))
    t = t.to(types(torch)[dtype]) if dtype else t
    if stride is None and not offset:
        return t.cuda()
    n, V = t.shape
    stride = stride or V
    fill = float("nan") if t.dtype.is_floating_point else -1
    big = torch.full((offset + n * stride + 64,), fill, dtype=t.dtype).cuda()
    view = big.as_strided((n, V), (stride, 1), offset)
    view.copy_(t)
    return view


def as_f32(torch, a, dtype):
    """What an array holds once it is of a type."""
    return torch.from_numpy(a).to(types(torch)[dtype]).float().numpy()


def bits_equal(torch, got, want, dtype, what):
    w = torch.from_numpy(want).to(types(torch)[dtype])
    g = got.cpu()
    same = (g == w) | (g.isnan() & w.isnan())
    assert bool(same.all()), f"{what}: {int((~same).sum())} of {same.numel()} differ, first {torch.nonzero(~same)[0].tolist()}"


def make_adjust(rng, R, V, distinct, L, ids, nan=True):
    x = (rng.normal(size=(distinct, V)) * 3).astype(np.float32)
    if V > 4:       # ties, infinities, NaN and the lowest value, some of them masked below
        x[rng.random(x.shape) < 0.2] = np.float32(1.5)
        x[rng.random(x.shape) < 0.02] = -np.inf
        if nan:
            x[rng.random(x.shape) < 0.02] = np.nan
            x[rng.random(x.shape) < 0.01] = np.finfo(np.float32).min
    h = ln = None
    if L is not None:
        h = rng.integers(-2, V + 2, size=(R, L)) if ids != "u8" else rng.integers(0, min(V + 2, 256), size=(R, L))
        if L:
            h[:, : L // 2] = rng.integers(0, max(1, min(V, 200) // 8 + 1), size=(R, L // 2))     # repeats
        ln = rng.integers(-1, L + 2, size=R).astype(np.int32)
        ln[-1] = L
    return x, h, ln


def check_adjust(torch, emo, rng, R, V, dtype="f32", out="f32", choice="i32", distinct=None, L=None, ids="i32", mask=0, noise=0, bias=0,
                 lengths=True, stride=None, offset=0, in_place=False, stream=None):
    distinct = distinct or R
    print(f"[case] adjust R={R} V={V} {dtype}->{out} distinct={distinct} L={L} {ids} mask={mask} noise={noise} bias={bias} stride={stride}"
          f" offset={offset} in_place={in_place}", flush=True)
    x, h, ln = make_adjust(rng, R, V, distinct, L, ids)
    x = as_f32(torch, x, dtype)
    kw = {"inv_temperature": rng.uniform(0.5, 2, size=R).astype(np.float32)}
    if L is not None:
        kw.update(repetition=rng.uniform(1, 1.5, size=R).astype(np.float32), frequency=rng.uniform(0, 0.5, size=1).astype(np.float32),
                  presence=rng.uniform(0, 0.5, size=R).astype(np.float32))
    allowed = None
    if mask:
        allowed = rng.random((mask, V)) < 0.6
        if mask > 1:
            allowed[0] = False
        kw["mask"] = orc.mask_words(allowed)
    if noise:
        kw["noise"] = rng.gumbel(size=(noise, V)).astype(np.float32)
    if bias:
        kw["bias"] = rng.normal(size=(bias, V)).astype(np.float32)
    want, wchoice = orc.adjust(R, x, history=h, lengths=ln if lengths else None, **kw)
    X = dev(torch, x, dtype, stride, offset)
    dkw = {k: dev(torch, v) for k, v in kw.items()}
    if noise and stride:
        dkw["noise"] = dev(torch, kw["noise"], None, stride + 3, 1)
    if L is not None:
        dkw["history"] = dev(torch, h, ids)
        if lengths:
            dkw["lengths"] = dev(torch, ln)
    O = None
    if out:
        O = X if in_place else dev(torch, np.zeros((R, V), np.float32), out, stride, offset)
    C = torch.full((R,), 77, dtype=types(torch)[choice], device="cuda") if choice else None
    torch.cuda.synchronize()
    got, gc = emo.adjust_logits(X, rows=R, out=O, choice=C, stream=stream, **dkw)
    torch.cuda.synchronize()
    if out:
        assert got.data_ptr() == O.data_ptr()
        bits_equal(torch, got, want, out, "adjusted logits")
        if stride and not in_place:     # the memory between and behind the rows still holds NaN
            flat = torch.as_strided(got, (offset + R * stride + 64,), (1,), 0)
            keep = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
            keep.as_strided((R, V), (stride, 1), offset)[:] = False
            assert bool(flat[keep].isnan().all())
    if choice:
        w = torch.from_numpy(wchoice).to(types(torch)[choice])
        assert torch.equal(gc.cpu(), w), (gc.cpu()[gc.cpu() != w][:5], w[gc.cpu() != w][:5])


EDGES = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 2047, 2048, 2049,
         4095, 4096, 4097, 8191, 8192, 8193, 16385, 32768, 40001]


@pytest.mark.parametrize("V", EDGES)
def test_adjust_sizes(torch, emo, V):
    rng = np.random.default_rng(V)
    choice = "u8" if V <= 255 else "i32"
    check_adjust(torch, emo, rng, 5, V, choice=choice)
    check_adjust(torch, emo, rng, 6, V, "bf16", "bf16", choice="i64", distinct=3, L=20, mask=2, noise=6, bias=1)
    check_adjust(torch, emo, rng, 4, V, "f16", "f32", choice=choice, L=9, ids="i64", mask=1, bias=4, stride=V + 5, offset=3)


@pytest.mark.parametrize("R,V,distinct", [(1, 1, 1), (1, 8, 1), (64, 8, 64), (4096, 16, 64), (1001, 11, 7), (3000, 24, 1000), (777, 64, 777),
                                          (2500, 5, 1), (300, 300, 100), (9, 100003, 3), (1, 1 << 20, 1), (2, 1000003, 1), (70, 20000, 70)])
def test_adjust_rows(torch, emo, R, V, distinct):
    rng = np.random.default_rng(R + V)
    check_adjust(torch, emo, rng, R, V, out="", choice="u8" if V <= 255 else "i64", distinct=distinct, mask=distinct, noise=R)
    check_adjust(torch, emo, rng, R, V, "bf16", "f32", choice="", distinct=distinct, mask=1, bias=1, L=33)


@pytest.mark.parametrize("V", [(1 << 20) + 1, 3 * (1 << 20) + 77])
def test_adjust_choices_among_more_than_256_tiles(torch, emo, V):
    """Ties of the greatest value in tiles far apart, in a tile, at a row's ends; none; noise on all of it."""
    rng = np.random.default_rng(V)
    x = np.minimum(rng.normal(size=(6, V)).astype(np.float32), np.float32(4))
    far = 4096 * 255
    for r, at in enumerate(([far + 7, far - 1], [V - 1, far + 1], [V - 1], [0, V - 1, far], [], [])):
        x[r, at] = 9.0
    x[4] = np.nan
    for kw in ({}, {"noise": rng.gumbel(size=(1, V)).astype(np.float32)}):
        _, wc = orc.adjust(6, x, **kw)
        C = torch.empty(6, dtype=torch.int64, device="cuda")
        emo.adjust_logits(dev(torch, x), choice=C, **{k: dev(torch, v) for k, v in kw.items()})
        assert C.cpu().tolist() == wc.tolist()
        if not kw:
            assert wc[:5].tolist() == [far - 1, far + 1, V - 1, 0, -1]


@pytest.mark.parametrize("L", [0, 1, 2, 63, 64, 65, 1000, 5000, 70000])
@pytest.mark.parametrize("V", [6, 200, 3000, 30011])
def test_adjust_histories(torch, emo, L, V):
    rng = np.random.default_rng(L)
    check_adjust(torch, emo, rng, 3, V, "bf16", "f32", L=L, ids="i32")
    check_adjust(torch, emo, rng, 2, V, "f32", "f32", L=L, ids="u8" if V <= 200 else "i64", lengths=False, noise=2)


@pytest.mark.parametrize("L", [2048, 2049, 6000])
@pytest.mark.parametrize("R,V", [(300, 8193), (3, 8193), (3, 32769), (5, 100003), (1, 1 << 20)])
def test_adjust_long_histories_of_wide_rows(torch, emo, R, V, L):
    rng = np.random.default_rng(V + L)
    check_adjust(torch, emo, rng, R, V, "bf16", "f32", L=L, ids="i32", mask=1, bias=1)
    check_adjust(torch, emo, rng, min(R, 3), V, "f16", "f16", L=L, ids="i64", choice="", in_place=True, stride=V + 3, offset=1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [9, 64, 1031, 50021])
def test_adjust_in_place_and_strides(torch, emo, dtype, V):
    rng = np.random.default_rng(V)
    check_adjust(torch, emo, rng, 7, V, dtype, dtype, L=12, mask=7, in_place=True)
    check_adjust(torch, emo, rng, 7, V, dtype, dtype, L=12, mask=7, in_place=True, stride=V + 1, offset=1)
    check_adjust(torch, emo, rng, 3, V, dtype, dtype, noise=3, stride=V + 7, offset=5)


def test_adjust_strided_operands(torch, emo):
    """History read through a transposed view, parameters of one row, expanded logits."""
    rng = np.random.default_rng(8)
    R, V, L = 40, 16, 30
    x, h, _ = make_adjust(rng, R, V, 1, L, "u8", nan=False)
    rep = np.float32([1.3])
    want, wc = orc.adjust(R, x, history=h, repetition=rep)
    H = dev(torch, np.ascontiguousarray(h.T), "u8").t()
    assert not H.is_contiguous()
    for X in (dev(torch, x), dev(torch, x).expand(R, V)):
        C = torch.empty(2 * R, dtype=torch.uint8, device="cuda")[::2]
        O, C = emo.adjust_logits(X, rows=R, history=H, repetition=dev(torch, rep), out=torch.empty((R, V), device="cuda"), choice=C)
        bits_equal(torch, O, want, "f32", "adjusted")
        assert C.cpu().numpy().tolist() == (wc % 256).tolist()


@pytest.mark.parametrize("V", [5, 16, 64, 71, 3001, 9001])
def test_operands_of_fewer_rows(torch, emo, V):
    """Every operand repeats over the call's rows by its own count, 1 and all among them; strided lists and outputs."""
    rng = np.random.default_rng(V)
    R = 12
    counts = {"history": 4, "lengths": 6, "repetition": 3, "frequency": 1, "presence": 12, "bias": 2, "inv_temperature": 4,
              "mask": 6, "noise": 3}
    for turn in range(2):
        x = rng.normal(size=(2 if turn else 4, V)).astype(np.float32)
        kw = {k: rng.uniform(0.5, 1.5, size=n).astype(np.float32) for k, n in counts.items()
              if k in ("repetition", "frequency", "presence", "inv_temperature")}
        kw["history"] = rng.integers(-1, V + 1, size=(counts["history"], 10))
        kw["lengths"] = rng.integers(0, 11, size=counts["lengths"]).astype(np.int32)
        kw["bias"] = rng.normal(size=(counts["bias"], V)).astype(np.float32)
        kw["noise"] = rng.gumbel(size=(counts["noise"], V)).astype(np.float32)
        kw["mask"] = orc.mask_words(rng.random((counts["mask"], V)) < 0.7)
        want, wc = orc.adjust(R, x, **kw)
        d = {k: dev(torch, v) for k, v in kw.items()}
        d["history"] = torch.stack([d["history"], d["history"] + 7], 2)[:, :, 0]        # every other element
        O, C = emo.adjust_logits(dev(torch, x), rows=R, out=torch.empty((R, V), device="cuda"),
                                 choice=torch.empty((R, 3), dtype=torch.int32, device="cuda")[:, 1], **d)
        bits_equal(torch, O, want, "f32", "adjusted")
        assert C.cpu().tolist() == wc.tolist()
        counts = {k: 12 // n for k, n in counts.items()}
    N, K = 12, 7
    x = rng.normal(size=(N, V)).astype(np.float32)
    i, t = rng.integers(0, V, size=(3, K)), rng.normal(size=(4, K)).astype(np.float32)
    words, scale = orc.mask_words(rng.random((6, V)) < 0.8), rng.uniform(size=2).astype(np.float32)
    w = orc.distill(x, i, t, 1.3, words, scale)
    _, tl, tg = bounds(w, V, K, 1.3, 1.3 * np.tile(scale, 6).astype(np.float64), "f32")
    I = torch.stack([dev(torch, i, "i64")] * 2, 2)[:, :, 0]
    T = torch.stack([dev(torch, t)] * 3, 2)[:, :, 2]
    loss, stats = torch.empty((N, 2), device="cuda")[:, 1], torch.empty((N, 5), device="cuda")[:, 2:4]
    X, M, S = dev(torch, x), dev(torch, words), dev(torch, scale)
    emo.distill_forward(X, I, T, 1.3, mask=M, loss=loss, stats=stats)
    g = emo.distill_backward(X, stats, I, T, 1.3, scale=S, mask=M)
    loss2, g2 = emo.distill_step(X, I, T, np.float32(1.3), scale=S, mask=M)
    for a, b in ((loss, g), (loss2, g2)):
        check_near(a.cpu().numpy(), w["loss"], tl, "loss")
        check_near(b.cpu().numpy(), w["grad"], tg, "gradient")


def test_adjust_defaults_and_refusals(torch, emo):
    x = torch.randn(4, 300, device="cuda", dtype=torch.float16)
    out, choice = emo.adjust_logits(x)
    assert torch.equal(out, x) and choice is None and out.dtype == x.dtype
    with pytest.raises(emo.EmoError, match="divide"):
        emo.adjust_logits(x, rows=6)
    with pytest.raises(emo.EmoError, match="byte"):
        emo.adjust_logits(x, choice=torch.empty(4, dtype=torch.uint8, device="cuda"))
    with pytest.raises(emo.EmoError, match="overlaps"):
        emo.adjust_logits(x[:3], out=x[1:])
    with pytest.raises(ValueError, match="mask"):
        emo.adjust_logits(x, mask=torch.zeros((4, 10), dtype=torch.int32))
    with pytest.raises(ValueError, match="type"):
        emo.adjust_logits(x.double())
    e, c = emo.adjust_logits(x[:0], choice=torch.empty(0, dtype=torch.int32, device="cuda"))
    assert e is None and c.numel() == 0


@pytest.mark.parametrize("V", [3, 5, 61, 70, 2051])
def test_adjust_odd_rates(torch, emo, V):
    """Rates of any value: a negative, zero or infinite temperature turns no padding behind a row into an entry."""
    rng = np.random.default_rng(V)
    x = rng.normal(size=(6, V)).astype(np.float32)
    x[:, 0] = -np.inf
    h = rng.integers(0, V, size=(6, 4))
    kw = {"repetition": np.float32([0, -1, np.inf, np.nan, 1, 2]), "frequency": np.float32([0, -1, np.inf, 1, 0, 0]),
          "presence": np.float32([0, 1, -1, 0, -np.inf, 0]), "inv_temperature": np.float32([-1, -2, 0, np.inf, -0.5, np.nan])}
    for mask in (None, orc.mask_words(rng.random((6, V)) < 0.5)):
        want, wc = orc.adjust(6, x, history=h, mask=mask, **kw)
        O, C = emo.adjust_logits(dev(torch, x), history=dev(torch, h, "i32"), mask=dev(torch, mask), out=torch.empty((6, V), device="cuda"),
                                 choice=torch.empty(6, dtype=torch.int32, device="cuda"), **{k: dev(torch, v) for k, v in kw.items()})
        bits_equal(torch, O, want, "f32", "adjusted")
        assert C.cpu().tolist() == wc.tolist()


@pytest.mark.parametrize("L", [20, 1500, 40000])
@pytest.mark.parametrize("V", [40, 70, 3001, 9001, 40001])
def test_adjust_rates_that_are_no_number(torch, emo, V, L):
    """A penalty of any NaN, that of all ones among them, makes the entry NaN: the ids, of the greatest logits, are
    the history's last, each once."""
    rng = np.random.default_rng(V)
    x = rng.normal(size=(4, V)).astype(np.float32)
    h = np.full((4, L), -1)
    for r in range(4):
        h[r, -20:] = rng.choice(V, 20, replace=False)
        x[r, h[r, -20:]] += 20
    nans = np.array([0xffffffff, 0x7fffffff, 0x7fc00000, 0xffc00001], np.uint32).view(np.float32)
    for name in ("repetition", "frequency", "presence"):
        want, wc = orc.adjust(4, x, history=h, **{name: nans})
        assert np.isnan(want).sum() == 80
        O, C = emo.adjust_logits(dev(torch, x), history=dev(torch, h, "i32"), out=torch.empty((4, V), device="cuda"),
                                 choice=torch.empty(4, dtype=torch.int32, device="cuda"), **{name: dev(torch, nans)})
        bits_equal(torch, O, want, "f32", f"adjusted, {name}")
        assert C.cpu().tolist() == wc.tolist()


@pytest.mark.parametrize("V", [2, 7, 40, 61, 75, 2500, 9003, 33001])
def test_adjust_odd_noise_bias_and_mask_ends(torch, emo, V):
    """Infinities and NaN in noise and bias; mask bits behind the last entry, which are nobody's."""
    rng = np.random.default_rng(V)
    x = rng.normal(size=(4, V)).astype(np.float32)
    noise, bias = rng.gumbel(size=(4, V)).astype(np.float32), rng.normal(size=(1, V)).astype(np.float32)
    for a, row in ((noise, 0), (noise, 1), (bias, 0)):
        a[row][rng.random(V) < 0.2] = [np.nan, -np.inf, np.nan][row]
    noise[2][rng.random(V) < 0.3] = np.inf
    noise[3] = np.nan
    bias[0, V - 1] = -np.inf
    W = (V + 31) // 32
    words = orc.mask_words(rng.random((4, V)) < 0.7).copy()
    if V % 32:
        words[:, W - 1] |= np.int32(-1) << np.int32(V % 32)
    for kw in ({"noise": noise}, {"noise": noise, "bias": bias, "mask": words}, {"mask": words}):
        want, wc = orc.adjust(4, x, **kw)
        O, C = emo.adjust_logits(dev(torch, x), out=torch.empty((4, V), device="cuda"),
                                 choice=torch.empty(4, dtype=torch.int64, device="cuda"), **{k: dev(torch, v) for k, v in kw.items()})
        bits_equal(torch, O, want, "f32", "adjusted")
        assert C.cpu().tolist() == wc.tolist()
    i, t = rng.integers(0, V, size=(4, 9)), rng.normal(size=(4, 9)).astype(np.float32)
    w = orc.distill(x, i, t, 1.0, words)
    _, tl, tg = bounds(w, V, 9, 1.0, np.ones(4), "f32")
    loss, g = emo.distill_step(dev(torch, x), dev(torch, i, "i64"), dev(torch, t), mask=dev(torch, words))
    check_near(loss.cpu().numpy(), w["loss"], tl, "loss")
    check_near(g.cpu().numpy(), w["grad"], tg, "gradient")


def test_distill_teachers_of_nan_and_infinity(torch, emo):
    """A NaN or an infinity in a teacher's list that counts makes the loss NaN; one at an id that does not, nothing."""
    for V in (16, 40, 300, 9000):
        x = np.zeros((5, V), np.float32)
        i = np.tile(np.arange(4), (5, 1))
        t = np.zeros((5, 4), np.float32)
        t[0, 1], t[1, 2], t[2] = np.nan, np.inf, np.nan
        t[3, 3], i[3, 3] = np.nan, -1
        X, I, T = dev(torch, x), dev(torch, i, "i32"), dev(torch, t)
        loss, stats = emo.distill_forward(X, I, T)
        loss2, g = emo.distill_step(X, I, T)
        g3 = emo.distill_backward(X, stats, I, T)
        for a in (loss, loss2):
            a = a.cpu().numpy()
            assert np.isnan(a[:3]).all() and abs(a[3:] - np.log(V)).max() < 1e-5
        for b in (g, g3):
            b = b.cpu().numpy()
            assert np.isnan(b[:3, 1]).all() and np.isfinite(b[3:]).all()


def test_workspaces_of_the_caller(torch, emo):
    """A workspace given serves call after call whatever it holds; too small a one is refused."""
    import ctypes
    for call, size in ((lambda x, w: emo.adjust_logits(x, choice=torch.empty(len(x), dtype=torch.int64, device="cuda"), workspace=w)[1],
                        emo.lib.emo_adjust_workspace),
                       (lambda x, w: emo.distill_forward(x, torch.full((1, 1), 5, device="cuda"), torch.zeros((1, 1), device="cuda"),
                                                         workspace=w)[0], emo.lib.emo_distill_workspace),
                       (lambda x, w: emo.distill_step(x, torch.full((1, 1), 5, device="cuda"), torch.zeros((1, 1), device="cuda"),
                                                      workspace=w)[1], emo.lib.emo_distill_workspace)):
        n = ctypes.c_int64(0)
        for V in (200000, 70001):
            x = torch.randn((3, V), device="cuda")
            assert size(3, V, ctypes.byref(n)) == 0 and n.value > 0
            w = torch.full((n.value,), 255, dtype=torch.uint8, device="cuda")
            want = call(x, None)
            for _ in range(2):
                assert torch.equal(call(x, w), want)
            with pytest.raises(emo.EmoError, match="workspace"):
                call(x, w[: n.value - 1])
            with pytest.raises(ValueError, match="workspace"):
                call(x, torch.zeros(2 * n.value, dtype=torch.uint8, device="cuda")[::2])


def test_adjust_masks_that_leave_little(torch, emo):
    """Nothing, only -inf, only the lowest value, only NaN; a byte choice without an entry is 255."""
    for V in (5, 70, 5000):
        x = np.zeros((5, V), np.float32)
        allowed = np.zeros((5, V), bool)
        allowed[1:, V - 1] = True
        x[1, V - 1], x[2, V - 1], x[3, V - 1], x[4, V - 1] = -np.inf, np.finfo(np.float32).min, np.nan, np.inf
        x[0, 0] = np.nan
        X, M = dev(torch, x), dev(torch, orc.mask_words(allowed))
        C = torch.zeros(5, dtype=torch.uint8 if V < 256 else torch.int64, device="cuda")
        O, _ = emo.adjust_logits(X, mask=M, out=torch.empty_like(X), choice=C)
        want, wc = orc.adjust(5, x, mask=orc.mask_words(allowed))
        bits_equal(torch, O, want, "f32", "adjusted")
        none = 255 if V < 256 else -1
        assert C.cpu().tolist() == [none, none, V - 1, none, V - 1]


# ------------------------------------------------------------------------------ distillation

HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}


def bounds(w, V, K, tau, c, dtype):
    """Bounds of (s relative, loss, gradient) made of the roundings, see the head of this file."""
    rel_s = (V / 256 + 64 + 3) * EPS
    rel_p = (K + 8 + 3 * w["spread"]) * EPS
    loss = tau * tau * (rel_s + (K + 16 + 3 * np.minimum(w["spread"], 1.0) + 4) * EPS * w["term"])
    q = w["q"] * (rel_s + (3 * w["away"] + 4) * EPS)
    g = np.abs(c)[:, None] * (q + w["p"] * rel_p[:, None] + 3 * EPS * np.abs(w["q"] - w["p"]))
    return rel_s, loss, g + (np.abs(w["grad"]) + g) * HALF[dtype] + TINY[dtype]


def check_near(got, want, tol, what):
    got = np.asarray(got, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{what}: infinities"
    off = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0))
    tol = np.broadcast_to(tol, off.shape)
    bad = fine & ~(off <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]} (bound {tol[bad][0]})"


def make_distill(torch, rng, N, V, K, dtype, ids, mask, teacher="f32", shared=False):
    x = as_f32(torch, (rng.normal(size=(N, V)) * 3).astype(np.float32), dtype)
    hi = min(V, 256) if ids == "u8" else V
    i = rng.integers(0, hi, size=(N, K))
    if ids != "u8" and K > 1:
        i[:, -1] = rng.choice([-1, V, V + 7, 0], size=N)        # padding
    t = as_f32(torch, (rng.normal(size=(1 if shared else N, K)) * 2).astype(np.float32), teacher)
    if K > 2:
        t[:, 1] = -np.inf
    words = None
    if mask:
        allowed = rng.random((mask, V)) < 0.7
        if mask > 1:
            allowed[1] = False
        words = orc.mask_words(allowed)
        x[rng.random(x.shape) < 0.02] = -np.inf
        if V > 8:                       # masked places hold anything
            for r in range(N):
                hidden = np.flatnonzero(~allowed[r % mask])
                if len(hidden):
                    x[r, hidden[: len(hidden) // 2 + 1]] = np.nan
    return x, i, t, words


def check_distill(torch, emo, rng, N, V, K, dtype="f32", ids="i32", mask=0, tau=1.0, teacher="f32", shared=False, grad=None, stride=None,
                  offset=0, in_place=False, scaled=True, x=None):
    grad = grad or dtype
    print(f"[case] distill N={N} V={V} K={K} {dtype}->{grad} {ids} mask={mask} tau={tau} teacher={teacher} shared={shared} stride={stride}"
          f" offset={offset} in_place={in_place}", flush=True)
    made, i, t, words = make_distill(torch, rng, N, V, K, dtype, ids, mask, teacher, shared)
    x = made if x is None else x
    scale = rng.uniform(-2, 2, size=N).astype(np.float32) if scaled else None
    w = orc.distill(x, i, t, tau, words, scale)
    c = tau * (np.ones(N) if scale is None else scale.astype(np.float64))
    rel_s, tol_loss, tol_grad = bounds(w, V, K, tau, c, grad)
    I = dev(torch, i, ids)
    if ids == "u8":
        I = dev(torch, np.ascontiguousarray(i.T), ids).t()
    T, M, S = dev(torch, t, teacher), dev(torch, words), dev(torch, scale)

    def logits():
        return dev(torch, x, dtype, stride, offset)

    def gradient(X):
        return X if in_place else dev(torch, np.zeros((N, V), np.float32), grad, stride, offset)

    X = logits()
    loss, stats = emo.distill_forward(X, I, T, tau, mask=M)
    got = stats.cpu().numpy().astype(np.float64)
    check_near(got[:, 0], w["stats"][:, 0], 0.0, "m")
    check_near(got[:, 1], w["stats"][:, 1], rel_s * np.abs(np.nan_to_num(w["stats"][:, 1], posinf=0)), "s")
    check_near(loss.cpu().numpy(), w["loss"], tol_loss, "loss")
    g = emo.distill_backward(X, stats, I, T, tau, scale=S, mask=M, grad=gradient(X))
    check_near(g.float().cpu().numpy(), w["grad"], tol_grad, "gradient")
    X = logits()
    loss2, g2 = emo.distill_step(X, I, T, tau, scale=S, mask=M, grad=gradient(X))
    check_near(loss2.cpu().numpy(), w["loss"], tol_loss, "step's loss")
    check_near(g2.float().cpu().numpy(), w["grad"], tol_grad, "step's gradient")
    if stride and not in_place:
        for y in (g, g2):
            flat = torch.as_strided(y, (offset + N * stride + 64,), (1,), 0)
            keep = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
            keep.as_strided((N, V), (stride, 1), offset)[:] = False
            assert bool(flat[keep].isnan().all())
    # the same call, the same bits
    X = logits()
    loss3, g3 = emo.distill_step(X, I, T, tau, scale=S, mask=M, grad=gradient(X))
    assert torch.equal(loss3.nan_to_num(7), loss2.nan_to_num(7)) and torch.equal(g3.float().nan_to_num(7), g2.float().nan_to_num(7))
    return w


@pytest.mark.parametrize("V", EDGES)
def test_distill_sizes(torch, emo, V):
    rng = np.random.default_rng(V + 1)
    check_distill(torch, emo, rng, 5, V, 6)
    check_distill(torch, emo, rng, 4, V, 33, "bf16", "i64", mask=4, tau=2.0)
    check_distill(torch, emo, rng, 3, V, 17, "f16", "u8", mask=1, tau=0.5, grad="f32", shared=True, stride=V + 5, offset=3)


@pytest.mark.parametrize("V", [32768, 131072])
def test_distill_long_sums(torch, emo, V):
    """Rows of one value below the greatest, whose exponential a long running sum would round the same way every
    time: of 131,072 entries such a sum is off by 105 half steps.  Its additions here follow each other by 4 within 16
    bytes, 8 times 16 bytes, V / 8,192 steps, 6 in a wave, 4 waves; an exponential is off by its argument's 3
    roundings (the argument is below 0.02) and a step, two half steps."""
    steps = 2.0 ** 15                   # of a sum from 256 on: one below the next half, so that it is rounded down
    e = (np.floor(0.99 * steps) + 0.45) / steps
    x = np.full((1, V), np.log(e), np.float32)
    x[0, :1024] = 0.0                   # 16 bytes of every thread
    X = dev(torch, x).expand(2048, V)
    I, T = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1, 1), device="cuda")
    loss, stats = emo.distill_forward(X, I, T)
    w = orc.distill(x, np.zeros((1, 1), int), np.zeros((1, 1)), 1.0)
    near = (4 + 8 + V / 8192 + 6 + 4 + 3 * 0.02 + 2) * EPS
    check_near(stats[:, 1].cpu().numpy(), np.full(2048, w["stats"][0, 1]), near * w["stats"][0, 1], "s")
    # log s is off by s's error and a rounding of its own, the distance and the product by one each
    check_near(loss.cpu().numpy(), np.full(2048, w["loss"][0]), near + 4 * EPS * w["loss"][0], "loss")


@pytest.mark.parametrize("K", [0, 1, 2, 63, 64, 65, 100, 255, 256, 257, 1000, 1024])
@pytest.mark.parametrize("V", [3, 16, 300, 9001])
def test_distill_entries(torch, emo, K, V):
    rng = np.random.default_rng(K)
    check_distill(torch, emo, rng, 3, V, K, "bf16", "i32", mask=1)
    check_distill(torch, emo, rng, 3, V, K, "f32", "u8", tau=1.5, teacher="bf16")


@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (1, 8, 32), (64, 8, 32), (4099, 16, 64), (1001, 11, 33), (777, 64, 5), (300, 700, 20),
                                   (1, 131072, 64), (2, 100003, 64), (1, 1000003, 10), (40, 32768, 32), (300, 5000, 40)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_rows(torch, emo, N, V, K, dtype):
    rng = np.random.default_rng(N + V)
    check_distill(torch, emo, rng, N, V, K, dtype, "i32", mask=N if V < 1000 else 1, tau=2.0)


@pytest.mark.parametrize("N,V", [(4200, 2500), (2100, 4200), (1100, 8300), (8300, 2051), (4200, 4097), (2100, 8193)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_many_rows(torch, emo, N, V, dtype):
    """More rows than the card holds at once: against the two passes on every row, the oracle on some."""
    rng = np.random.default_rng(N)
    x = torch.from_numpy(rng.normal(size=(N, V)).astype(np.float32) * 3).to(types(torch)[dtype])
    i, t = rng.integers(-1, V, size=(N, 9)), rng.normal(size=(N, 9)).astype(np.float32)
    i[:, 3] = i[:, 5]
    words = orc.mask_words(rng.random((1, V)) < 0.8)
    X, I, T, M = x.cuda(), dev(torch, i, "i32"), dev(torch, t), dev(torch, words)
    loss, stats = emo.distill_forward(X, I, T, mask=M)
    g = emo.distill_backward(X, stats, I, T, mask=M)
    loss2, g2 = emo.distill_step(X, I, T, mask=M)
    some = rng.choice(N, 6, replace=False)
    w = orc.distill(x.float().numpy()[some], i[some], t[some], 1.0, words)
    _, tl, tg = bounds(w, V, 9, 1.0, np.ones(6), dtype)
    for a, b in ((loss, g), (loss2, g2)):
        check_near(a.cpu().numpy()[some], w["loss"], tl, "loss")
        check_near(b.float().cpu().numpy()[some], w["grad"], tg, "gradient")
    # the two differ by their roundings: each is within the bounds of the exact values, s by V / 256 + 67 steps
    near = 2 * (V / 256 + 67 + 60) * EPS
    assert bool(((loss - loss2).abs() <= near * (1 + loss.abs())).all())
    q = g.float().abs() + 1e-3
    assert bool(((g.float() - g2.float()).abs() <= q * (near + 2 * HALF[dtype])).all())


@pytest.mark.parametrize("V", [65537, 100003, 131072])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_distill_widest_rows_held(torch, emo, V, dtype):
    """Rows of 65,537 to 131,072 2-byte entries that a workgroup holds: more than 32 of them."""
    rng = np.random.default_rng(V)
    check_distill(torch, emo, rng, 33, V, 40, dtype, mask=1, scaled=False)
    check_distill(torch, emo, rng, 34, V, 20, dtype, "i64", grad="f32", stride=V + 3, offset=1)
    check_distill(torch, emo, rng, 35, V, 7, dtype, mask=35, tau=2.0, in_place=True)


@pytest.mark.parametrize("N,V,dtype", [(4200, 2049, "bf16"), (4200, 4096, "f16"), (8300, 2500, "f32")])
def test_distill_many_rows_of_long_lists(torch, emo, N, V, dtype):
    """More rows than the card holds at once with lists longer than a sixteenth of the row: a wave a row and a
    table of probabilities.  Against the two passes on every row, the oracle on some."""
    rng = np.random.default_rng(N)
    K = 300
    x = torch.from_numpy(rng.normal(size=(N, V)).astype(np.float32) * 3).to(types(torch)[dtype])
    i, t = rng.integers(-1, V, size=(N, K)), rng.normal(size=(N, K)).astype(np.float32)
    i[:, 100:200] = rng.integers(0, 3, size=(N, 100)) * (V // 2)
    words = orc.mask_words(rng.random((1, V)) < 0.8)
    X, I, T, M = x.cuda(), dev(torch, i, "i32"), dev(torch, t), dev(torch, words)
    loss, stats = emo.distill_forward(X, I, T, mask=M)
    g = emo.distill_backward(X, stats, I, T, mask=M)
    loss2, g2 = emo.distill_step(X, I, T, mask=M)
    some = rng.choice(N, 6, replace=False)
    w = orc.distill(x.float().numpy()[some], i[some], t[some], 1.0, words)
    _, tl, tg = bounds(w, V, K, 1.0, np.ones(6), dtype)
    for a, b in ((loss, g), (loss2, g2)):
        check_near(a.cpu().numpy()[some], w["loss"], tl, "loss")
        check_near(b.float().cpu().numpy()[some], w["grad"], tg, "gradient")
    # the two differ by their roundings: of s and, at an entry's summed probability, of the list
    near = 2 * (V / 256 + 67 + 60 + K + 8) * EPS
    assert bool(((loss - loss2).abs() <= near * (1 + loss.abs())).all())
    assert bool(((g.float() - g2.float()).abs() <= (g.float().abs() + 1e-3) * (near + 2 * HALF[dtype])).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [9, 64, 1031, 50021, 140001])
def test_distill_in_place_and_strides(torch, emo, dtype, V):
    rng = np.random.default_rng(V)
    check_distill(torch, emo, rng, 3, V, 12, dtype, in_place=True, scaled=False)
    check_distill(torch, emo, rng, 3, V, 40, dtype, teacher="f16", in_place=True, stride=V + 1, offset=1, mask=3)
    check_distill(torch, emo, rng, 2, V, 12, dtype, stride=V + 9, offset=7)


def test_distill_one_id_many_times(torch, emo):
    """Every entry of the list names the same few ids, the first, the last, one on each side of a border."""
    rng = np.random.default_rng(2)
    for V in (16, 300, 5000, 20000, 70000):
        x = rng.normal(size=(2, V)).astype(np.float32)
        i = rng.choice([0, V - 1, V // 2, V // 2 - 1, 7, 8], size=(2, 512))
        t = rng.normal(size=(2, 512)).astype(np.float32)
        w = orc.distill(x, i, t, 1.0)
        _, _, tol = bounds(w, V, 512, 1.0, np.ones(2), "f32")
        loss, g = emo.distill_step(dev(torch, x), dev(torch, i, "i32"), dev(torch, t))
        check_near(g.cpu().numpy(), w["grad"], tol, f"gradient V={V}")
        # q and the summed p both add up to 1: so does the gradient to 0, within the bounds' sum
        assert abs(g.double().sum(-1).cpu().numpy()).max() <= tol.sum(-1).max()


def test_distill_gradient_is_the_difference(torch, emo):
    rng = np.random.default_rng(4)
    N, V, K, tau = 3, 21, 9, 1.7
    x = rng.normal(size=(N, V)).astype(np.float32)
    i = rng.integers(-1, V, size=(N, K))
    t = rng.normal(size=(N, K)).astype(np.float32)
    words = orc.mask_words(rng.random((N, V)) < 0.8)
    w = orc.distill(x, i, t, tau, words)
    _, _, tol = bounds(w, V, K, tau, np.full(N, tau), "f32")
    _, g = emo.distill_step(dev(torch, x), dev(torch, i, "i64"), dev(torch, t), tau, mask=dev(torch, words))
    for r in range(N):
        for v in range(V):
            # the difference itself is good to 1e-7 (the oracle's own test)
            assert abs(float(g[r, v]) - orc.loss_difference(x, i, t, tau, words, r, v)) < 1e-7 + tol[r, v]


@pytest.mark.parametrize("V", [12, 500, 6000, 90000])
def test_distill_specials(torch, emo, V):
    """Rows of NaN, infinities and nothing: each keeps to itself, the row beside it is as alone."""
    rng = np.random.default_rng(V)
    x = rng.normal(size=(9, V)).astype(np.float32)
    i = rng.integers(0, V, size=(9, 4))
    t = rng.normal(size=(9, 4)).astype(np.float32)
    i[0] = -1                                   # a row without a teacher, whatever its logits
    x[0] = np.nan
    x[1] = -np.inf                              # no distribution
    x[2, V - 1] = np.inf
    x[3, 0] = np.nan
    i[3] = 1
    t[4] = -np.inf                              # no valid entry
    x[5, :] = -np.inf                           # one entry left, the teacher on it
    x[5, 3], i[5] = 0.5, 3
    x[6, i[6]] = -np.inf                        # the teacher on what the student excludes
    x[6, (i[6].max() + 1) % V] = 1.0
    x[7] = np.finfo(np.float32).min             # the lowest value everywhere
    w = orc.distill(x, i, t, 1.0)
    _, tol_loss, tol = bounds(w, V, 4, 1.0, np.ones(9), "f32")
    X, I, T = dev(torch, x), dev(torch, i, "i32"), dev(torch, t)
    loss, stats = emo.distill_forward(X, I, T)
    g = emo.distill_backward(X, stats, I, T)
    loss2, g2 = emo.distill_step(X, I, T)
    assert w["loss"][0] == 0 and np.isnan(w["loss"][[1, 2, 3]]).all() and w["loss"][4] == 0 and w["loss"][6] == np.inf
    for a, b in ((loss, g), (loss2, g2)):
        check_near(a.cpu().numpy(), w["loss"], tol_loss, "loss")
        b = b.cpu().numpy()
        check_near(b[[0, 1, 2, 3, 4, 5, 6, 7, 8]], w["grad"], tol, "gradient")
        assert not b[[0, 4]].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [12, 60, 500, 6000, 90000])
def test_distill_teachers_on_the_lowest_value(torch, emo, V, dtype):
    """The teacher on logits of the type's lowest value, as masks by addition leave them: the distance in
    temperatures is no fp32 number below a temperature of 1, but the loss, temperature times the distance, is."""
    rng = np.random.default_rng(V)
    N, K, tau = 40, 5, 0.25
    x = as_f32(torch, rng.normal(size=(N, V)).astype(np.float32), dtype)
    i = np.stack([rng.choice(V, K, replace=False) for _ in range(N)])
    t = rng.normal(size=(N, K)).astype(np.float32) * 0.25
    for r in range(N):
        x[r, i[r, :1 + r % 4]] = float(torch.finfo(types(torch)[dtype]).min)
    w = orc.distill(x, i, t, tau)
    assert np.isfinite(w["loss"]).all() and w["loss"].min() > 1e33
    _, tl, tg = bounds(w, V, K, tau, np.full(N, tau), dtype)
    X, I, T = dev(torch, x, dtype), dev(torch, i, "i32"), dev(torch, t)
    loss, stats = emo.distill_forward(X, I, T, tau)
    g = emo.distill_backward(X, stats, I, T, tau)
    loss2, g2 = emo.distill_step(X, I, T, tau)
    for a, b in ((loss, g), (loss2, g2)):
        check_near(a.cpu().numpy(), w["loss"], tl, "loss")
        check_near(b.float().cpu().numpy(), w["grad"], tg, "gradient")


def test_streams_and_graphs(torch, emo):
    """Calls on side streams at once, each with its own operands, and captured graphs replayed between eager
    calls give the same bits as the eager calls."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)

    def operands(N, V):
        x = torch.randn((N, V), generator=gen, device="cuda").bfloat16()
        return {"x": x, "i": torch.randint(0, V, (N, 20), generator=gen, device="cuda", dtype=torch.int32),
                "t": torch.randn((N, 20), generator=gen, device="cuda"), "n": torch.randn((N, V), generator=gen, device="cuda"),
                "h": torch.randint(0, V, (N, 50), generator=gen, device="cuda"), "f": torch.full((N,), 0.3, device="cuda")}

    def eager(o):
        a, c = emo.adjust_logits(o["x"], history=o["h"], frequency=o["f"], noise=o["n"], out=torch.empty_like(o["x"]),
                                 choice=torch.empty(len(o["x"]), dtype=torch.int64, device="cuda"))
        l, s = emo.distill_forward(o["x"], o["i"], o["t"], 2.0)
        g = emo.distill_backward(o["x"], s, o["i"], o["t"], 2.0)
        l2, g2 = emo.distill_step(o["x"], o["i"], o["t"], 2.0)
        return [a, c, l, s, g, l2, g2]

    sets = [operands(1, 1 << 20), operands(3, 200003), operands(64, 8), operands(40, 4096)]
    want = [[y.clone() for y in eager(o)] for o in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for o, st in zip(sets, streams):
        with torch.cuda.stream(st):
            got.append(eager(o))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for u, v in zip(a, b):
            assert torch.equal(u, v)
    # two graphs captured on one stream, replayed on two streams at once
    graphs = []
    st = torch.cuda.Stream()
    for o in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            outs = eager(o)
        graphs.append((g, outs))
    for turn in range(3):
        for _, outs in graphs:
            for y in outs:
                y.zero_()
        torch.cuda.synchronize()
        for (g, _), s2 in zip(graphs, streams):
            with torch.cuda.stream(s2):
                g.replay()
        mixed = eager(sets[turn])
        torch.cuda.synchronize()
        for u, v in zip(want[turn], mixed):
            assert torch.equal(u, v)
        for (_, outs), a in zip(graphs, want):
            for u, v in zip(a, outs):
                assert torch.equal(u, v), f"replay {turn}"
    # the stream argument, with the workspace and outputs made by the call
    side = torch.cuda.Stream()
    o = sets[0]
    c = torch.empty(1, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    emo.adjust_logits(o["x"], history=o["h"], frequency=o["f"], noise=o["n"], choice=c, stream=side)
    l, s = emo.distill_forward(o["x"], o["i"], o["t"], 2.0, stream=side)
    side.synchronize()
    assert torch.equal(c, want[0][1]) and torch.equal(l, want[0][2]) and torch.equal(s, want[0][3])


@pytest.mark.parametrize("V", [8, 40, 300, 9001, 70001])
def test_outputs_beside_each_other(torch, emo, V):
    """Outputs as columns of one buffer, between the rows of the logits, beside the noise: the values of the same
    call on memory of its own, and nothing else written."""
    N, K = 5, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V)
    I = torch.randint(0, V, (N, K), generator=gen, device="cuda", dtype=torch.int32)
    T = torch.randn((N, K), generator=gen, device="cuda")
    both = torch.randn((N, 2 * V + 1), generator=gen, device="cuda")
    X, Y = both[:, :V], both[:, V + 1:]
    alone = X.contiguous()
    loss, stats = emo.distill_forward(alone, I, T)
    kept = torch.full((N, 4), 7.0, device="cuda")
    emo.distill_forward(X, I, T, loss=kept[:, 0], stats=kept[:, 2:])
    assert torch.equal(kept[:, 0], loss) and torch.equal(kept[:, 2:], stats) and bool((kept[:, 1] == 7).all())
    want = emo.distill_backward(alone, stats, I, T)
    emo.distill_backward(X, stats, I, T, grad=Y)
    assert torch.equal(Y, want) and torch.equal(X, alone)
    loss, want = emo.distill_step(alone, I, T)
    wide = torch.cat([both, both.new_full((N, 1), 7.0)], 1)
    X, Y = wide[:, :V], wide[:, V:2 * V]
    emo.distill_step(X, I, T, loss=wide[:, 2 * V + 1], grad=Y)
    assert torch.equal(Y, want) and torch.equal(wide[:, 2 * V + 1], loss) and torch.equal(X, alone)
    assert torch.equal(wide[:, 2 * V], both[:, 2 * V])
    # the adjusted logits in the noise's buffer, the choice in the last column of another
    noise = torch.randn((N, V), generator=gen, device="cuda")
    mixed = torch.cat([noise, noise], 1)
    chosen = torch.full((N, V + 2), 7, dtype=torch.int32, device="cuda")
    want, wc = emo.adjust_logits(alone, noise=noise, out=torch.empty_like(alone),
                                 choice=torch.empty(N, dtype=torch.int32, device="cuda"))
    emo.adjust_logits(alone, noise=mixed[:, :V], out=mixed[:, V:], choice=chosen[:, V])
    assert torch.equal(mixed[:, V:], want) and torch.equal(mixed[:, :V], noise) and torch.equal(chosen[:, V], wc)
    assert bool((chosen[:, :V] == 7).all()) and bool((chosen[:, V + 1] == 7).all())


def test_offsets_past_32_bits(torch, emo):
    """Rows whose first elements lie beyond 2^31 elements and 2^32 bytes."""
    N, V, stride = 3, 1000, (1 << 30) + 4099
    big = torch.empty(2 * stride + V + 8, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((N, V), (stride, 1), 5)
    rng = np.random.default_rng(1)
    vals = as_f32(torch, rng.normal(size=(N, V)).astype(np.float32), "bf16")
    x.copy_(torch.from_numpy(vals))
    C = torch.empty(N, dtype=torch.int32, device="cuda")
    emo.adjust_logits(x, out=x, choice=C)
    want, wc = orc.adjust(N, vals)
    bits_equal(torch, x, want, "bf16", "adjusted")
    assert C.cpu().tolist() == wc.tolist()
    i, t = rng.integers(0, V, size=(N, 8)), rng.normal(size=(N, 8)).astype(np.float32)
    w = orc.distill(vals, i, t, 1.0)
    _, tl, tg = bounds(w, V, 8, 1.0, np.ones(N), "bf16")
    loss, g = emo.distill_step(x, dev(torch, i, "i32"), dev(torch, t), grad=x)
    check_near(loss.cpu().numpy(), w["loss"], tl, "loss")
    check_near(g.float().cpu().numpy(), w["grad"], tg, "gradient")


@pytest.mark.parametrize("tau", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
@pytest.mark.parametrize("V", [9, 300, 9001, 70001])
def test_distill_temperatures_at_their_limits(torch, emo, V, tau):
    rng = np.random.default_rng(V)
    check_distill(torch, emo, rng, 3, V, 12, tau=tau, mask=1)
    check_distill(torch, emo, rng, 3, V, 5, "bf16", tau=tau, grad="f32", scaled=False)


def test_calls_of_several_launches(torch, emo):
    """More workgroups than a launch takes (2^21): the last rows are what they are alone."""
    rng = np.random.default_rng(0)
    N, V, K = (1 << 21) + 5, 70, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    X = torch.randn((N, V), generator=gen, device="cuda").bfloat16()
    I = torch.randint(0, V, (N, K), generator=gen, device="cuda", dtype=torch.int32)
    T = torch.randn((N, K), generator=gen, device="cuda")
    loss, stats = emo.distill_forward(X, I, T)
    g = emo.distill_backward(X, stats, I, T)
    loss2, g2 = emo.distill_step(X, I, T)
    C = torch.empty(N, dtype=torch.int64, device="cuda")
    O, _ = emo.adjust_logits(X, history=I, presence=T[:1, 0], out=torch.empty_like(X), choice=C)
    for rows in (slice(0, 3), slice((1 << 21) - 2, N)):
        x, i, t = X[rows].float().cpu().numpy(), I[rows].cpu().numpy(), T[rows].cpu().numpy()
        w = orc.distill(x, i, t, 1.0)
        _, tl, tg = bounds(w, V, K, 1.0, np.ones(len(x)), "bf16")
        for a, b in ((loss, g), (loss2, g2)):
            check_near(a[rows].cpu().numpy(), w["loss"], tl, "loss")
            check_near(b[rows].float().cpu().numpy(), w["grad"], tg, "gradient")
        want, wc = orc.adjust(len(x), x, history=i, presence=T[:1, 0].cpu().numpy())
        bits_equal(torch, O[rows], want, "bf16", "adjusted")
        assert C[rows].cpu().tolist() == wc.tolist()
    del X, I, T, g, g2, O
    # rows of several tiles, choices joined; 3 rows of logits in turn
    R, V = (1 << 21) + 1, 16400
    x = rng.normal(size=(3, V)).astype(np.float32)
    C = torch.empty(R, dtype=torch.int32, device="cuda")
    emo.adjust_logits(dev(torch, x), rows=R, choice=C)
    assert R % 3 == 0 and bool((C.view(-1, 3) == torch.from_numpy(orc.adjust(3, x)[1]).cuda()).all())
    # rows of a few entries
    N, V, K = (1 << 27) + 70, 4, 5
    x, i, t = rng.normal(size=(1, V)).astype(np.float32), rng.integers(0, V, size=(1, K)), rng.normal(size=(1, K)).astype(np.float32)
    loss, g = emo.distill_step(dev(torch, x).expand(N, V), dev(torch, i, "i32"), dev(torch, t))
    w = orc.distill(x, i, t, 1.0)
    _, tl, tg = bounds(w, V, K, 1.0, np.ones(1), "f32")
    check_near(loss[:1].cpu().numpy(), w["loss"], tl, "loss")
    check_near(g[:1].cpu().numpy(), w["grad"], tg, "gradient")
    assert bool((loss == loss[0]).all()) and bool((g == g[0]).all())


@pytest.mark.parametrize("V", [5, 300, 9001])
def test_counts_past_24_bits(torch, emo, V):
    """One id (2^24 + 3 times, read at a column stride of 0): the count is rounded to fp32 as the oracle's is."""
    L = (1 << 24) + 3
    x = np.random.default_rng(V).normal(size=(2, V)).astype(np.float32)
    h, rate = np.array([[V - 1], [2]]), np.float32([1.0, 0.37])
    want, wc = orc.adjust(2, x, history=np.broadcast_to(h, (2, L)), frequency=rate)
    O, C = emo.adjust_logits(dev(torch, x), history=dev(torch, h, "i32").expand(2, L), frequency=dev(torch, rate),
                             out=torch.empty((2, V), device="cuda"), choice=torch.empty(2, dtype=torch.int32, device="cuda"))
    bits_equal(torch, O, want, "f32", "adjusted")
    assert C.cpu().tolist() == wc.tolist() and want[0, V - 1] < -1.6e7


def test_nearly_2_31_rows(torch, emo):
    """Candidates for 2,047 packs, 2^20 of them: row r reads row r % 2047 up to the last."""
    P, B, V = 2047, 1 << 20, 8
    x = np.random.default_rng(3).normal(size=(P, V)).astype(np.float32)
    C = torch.full((B * P,), 77, dtype=torch.uint8, device="cuda")
    emo.adjust_logits(dev(torch, x), rows=B * P, choice=C)
    want = torch.from_numpy(orc.adjust(P, x)[1]).to(torch.uint8).cuda()
    for part in C.view(B, P).split(B // 8):
        assert bool((part == want).all())


def test_nearly_2_31_entries(torch, emo):
    """A row of 2^31 - 1 entries: indexes, offsets and sums to its end."""
    V = (1 << 31) - 1
    far = [V - 1, (1 << 30) + 3, 7]
    X = torch.zeros((1, V), dtype=torch.bfloat16, device="cuda")
    X[0, far] = 4.0
    X[0, V // 2] = 3.0
    words = torch.full((1, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    C = torch.empty(1, dtype=torch.int32, device="cuda")
    assert int(emo.adjust_logits(X, choice=C)[1]) == 7
    words[0, 0] &= ~(1 << 7)
    assert int(emo.adjust_logits(X, mask=words, choice=C)[1]) == (1 << 30) + 3
    H = torch.tensor([[V - 1, far[1], -1, V - 1, 9]], device="cuda")
    rate = torch.tensor([1.5], device="cuda")
    O, _ = emo.adjust_logits(X, history=H, presence=rate, frequency=rate, mask=words, out=torch.empty_like(X), choice=C)
    assert int(C) == V // 2
    assert O[0, [V - 1, far[1], 7, 9, 8, V - 2]].tolist() == [-0.5, 1.0, -float("inf"), -3.0, 0.0, 0.0]
    del O
    I = torch.tensor([[V - 1, 12, V // 2]], device="cuda")
    T = torch.tensor([[1.0, 0.0, 2.0]], device="cuda")
    loss, stats = emo.distill_forward(X, I, T)
    s = 3 + np.exp(-1.0) + (V - 4) * np.exp(-4.0)
    p = np.exp([1.0, 0.0, 2.0]) / np.exp([1.0, 0.0, 2.0]).sum()
    near = (8 + 4 + 128 + 6 + 4 + 32 + 6 + 16) * EPS        # chunks, steps, a wave, waves, a row's parts, a wave; the exponents
    check_near(stats.cpu().numpy(), np.array([[4.0, s]]), np.array([[0.0, near * s]]), "statistics")
    want = np.log(s) + (p * [0.0, 4.0, 1.0]).sum()
    check_near(loss.cpu().numpy(), np.array([want]), near + 16 * EPS * want, "loss")
    for g in (emo.distill_backward(X, stats, I, T), emo.distill_step(X, I, T, grad=X)[1]):
        at = [V - 1, 12, V // 2, far[1], 7, 0, V - 2]
        q = np.exp([0.0, -4.0, -1.0, 0.0, 0.0, -4.0, -4.0]) / s
        w = q - np.concatenate([p, np.zeros(4)])
        check_near(g[0, at].float().cpu().numpy(), w, np.abs(w) * (near + 2 * HALF["bf16"]), "gradient")
        others = sum(int((part != g[0, 0]).sum()) for part in g[0].split(1 << 28))
        assert others == 5          # all but the teacher's entries and the three greatest


def test_a_learned_search(torch, emo):
    """The calls together, as a search uses them: levels drawn from the packs' logits under a mask, evaluated
    where they lie, the best candidates' levels as the teacher; each step against the oracle."""
    import oracle
    from paper_2607_12324_amd import synth
    g = synth.config_graph(1)
    P, F, B, K = g.num_packs, g.num_levels, 512, 32
    gh = emo.EmoGraph(g, device=0)
    rng = np.random.default_rng(0)
    logits = torch.zeros((P, F), device="cuda")
    allowed = np.ones((P, F), bool)
    allowed[2, 0] = False                       # a pack that may not run at the lowest level
    words = orc.mask_words(allowed)
    M = dev(torch, words)
    top = np.full((1, P), F - 1, np.uint8)
    target = float(np.float32(1.2 * oracle.eval_batch(g, top)[0][0]))
    for _ in range(3):
        noise = rng.gumbel(size=(B * P, F)).astype(np.float32)
        before = logits.cpu().numpy()
        levels = torch.empty((B, P), dtype=torch.uint8, device="cuda")
        emo.adjust_logits(logits, rows=B * P, mask=M, noise=dev(torch, noise), choice=levels.view(-1))
        _, wc = orc.adjust(B * P, before, mask=words, noise=noise)
        lv = levels.cpu().numpy()
        assert np.array_equal(lv.reshape(-1), wc)
        T, E = gh.eval_policies(levels)
        To, Eo = oracle.eval_batch(g, lv)
        assert np.array_equal(T.cpu().numpy().astype(np.float64), To)
        cost = torch.where(T <= target, E, E * 4)
        best = torch.topk(-cost, K)[1]
        elite = levels[best]                    # [K, P] level bytes, read as [P, K]
        t = -cost[best] / cost.mean()
        loss, grad = emo.distill_step(logits, elite.t(), t, mask=M)
        w = orc.distill(before, elite.cpu().numpy().T.astype(np.int64), t.cpu().numpy()[None], 1.0, words)
        _, tl, tg = bounds(w, F, K, 1.0, np.ones(P), "f32")
        check_near(loss.cpu().numpy(), w["loss"], tl, "loss")
        check_near(grad.cpu().numpy(), w["grad"], tg, "gradient")
        logits -= 0.5 * grad
    # a pack with no level allowed gives byte 255: the evaluator's invalid level
    none = orc.mask_words(np.zeros((1, F), bool))
    levels = torch.empty((1, P), dtype=torch.uint8, device="cuda")
    emo.adjust_logits(logits, mask=dev(torch, none), choice=levels.view(-1))
    assert levels.unique().tolist() == [255] and bool(gh.eval_policies(levels)[0].isnan().all())
    # a batch's own feasibility mask as the mask of a draw among its candidates
    res, feas = gh.select_policy(dev(torch, lv), target)
    T, E = gh.eval_policies(dev(torch, lv))
    cost = -E.view(1, -1)
    pick, sel = torch.empty(1, dtype=torch.int64, device="cuda"), emo.parse_selection(res)
    emo.adjust_logits(cost, mask=feas, choice=pick)
    assert sel.num_feasible > 0 and int(pick) == sel.index      # the greatest -energy is the least energy
