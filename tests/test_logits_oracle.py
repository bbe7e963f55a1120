"""The oracle of the calls on logits against values worked out by hand and against differences."""
import numpy as np
import pytest

from oracle import logits as orc

INF = np.float32(np.inf)


def test_mask_words_round_trip():
    rng = np.random.default_rng(0)
    for V in (1, 31, 32, 33, 100):
        a = rng.random((3, V)) < 0.5
        w = orc.mask_words(a)
        assert w.shape == (3, (V + 31) // 32) and w.dtype == np.int32
        for r in range(3):
            assert np.array_equal(orc.allowed_bits(w[r], V), a[r])
    assert orc.mask_words(np.array([[True] + [False] * 30 + [True, True]]))[0].view(np.uint32).tolist() == [0x80000001, 1]


def test_adjust_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.0]], np.float32)
    out, c = orc.adjust(1, x, history=np.array([[0, 0, 1, 9, -1]]), repetition=np.float32([2]), frequency=np.float32([0.25]),
                        presence=np.float32([0.5]), bias=np.float32([[0, 0, 0, 3]]), inv_temperature=np.float32([2]))
    # 2 / 2 - 2 * .25 - .5 = 0;  -2 * 2 - .25 - .5 = -4.75;  doubled
    assert out[0].tolist() == [0.0, -9.5, 2.0, 6.0] and c[0] == 3
    out, c = orc.adjust(2, x, mask=orc.mask_words([[True, True, True, False], [False] * 4]), noise=np.float32([[0, 4.5, 0, 9]]))
    assert out[0].tolist() == [2.0, -2.0, 1.0, -INF] and c.tolist() == [1, -1]


def test_choice_ties_and_nans():
    x = np.float32([[1, 3, 3, np.nan], [-INF, -INF, np.nan, -INF], [-INF, -3.4e38, -INF, -INF], [0.0, -0.0, 0, 0]])
    assert orc.adjust(4, x)[1].tolist() == [1, -1, 1, 0]


def test_distill_by_hand():
    # two entries, the teacher on the first: loss = log(1 + e^(b - a)), gradient (q - p)
    r = orc.distill(np.array([[1.0, 0.0]]), np.array([[0]]), np.array([[5.0]]), 1.0)
    assert np.isclose(r["loss"][0], np.log1p(np.exp(-1.0)))
    q = 1 / (1 + np.exp(-1.0))
    assert np.allclose(r["grad"][0], [q - 1, 1 - q])
    # equal ids add up: as if listed once
    a = orc.distill(np.array([[0.3, -1.0, 2.0]]), np.array([[1, 1, 2]]), np.array([[0.0, 0.0, np.log(2.0)]]), 1.0)
    b = orc.distill(np.array([[0.3, -1.0, 2.0]]), np.array([[1, 2]]), np.array([[0.0, 0.0]]), 1.0)
    assert np.allclose(a["grad"], b["grad"]) and np.allclose(a["loss"], b["loss"])


def test_padding_and_masks():
    x = np.array([[0.5, 1.0, -np.inf, np.nan]])
    mask = orc.mask_words([[True, True, True, False]])
    r = orc.distill(x, np.array([[3, -1, 7]]), np.array([[1.0, 1.0, 1.0]]), 2.0, mask)
    assert r["loss"][0] == 0 and not r["grad"].any()
    r = orc.distill(x, np.array([[1, 3, 0]]), np.array([[1.0, 9.0, -np.inf]]), 2.0, mask)
    assert np.isfinite(r["loss"][0]) and r["grad"][0, 3] == 0 and r["grad"][0, 2] == 0
    assert r["p"][0].tolist() == [0, 1, 0, 0]


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_gradient_is_the_difference(tau):
    rng = np.random.default_rng(3)
    N, V, K = 4, 9, 6
    x = rng.normal(size=(N, V))
    ids = rng.integers(-1, V, size=(N, K))
    t = rng.normal(size=(N, K))
    mask = orc.mask_words(rng.random((N, V)) < 0.8)
    res = orc.distill(x, ids, t, tau, mask)
    for r in range(N):
        for v in range(V):
            # central differences: the loss's third derivative times h^2 / 6, and 1e-16 / h of rounding
            assert abs(orc.loss_difference(x, ids, t, tau, mask, r, v) - res["grad"][r, v]) < 1e-7
