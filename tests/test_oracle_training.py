"""The oracle of token scores, experts' rows and AdamW: its gradients against
differences, its formats against their definitions."""

import numpy as np
import pytest

from oracle import training_oracle as O


def test_scores_gradient_is_the_difference():
    r = np.random.default_rng(0)
    x, y = r.standard_normal((5, 9)) * 2, np.array([3, -1, 0, 8, 2])
    x[3, :4] = -np.inf
    a, b = r.standard_normal(5), r.standard_normal(5)
    a[2] = b[4] = 0

    def loss(x):
        q = O.log_probabilities(x, 0.7)
        h = O.entropy(q)
        return sum(a[t] * q[t, y[t]] + b[t] * h[t] for t in range(5) if y[t] >= 0)
    g = O.scores_gradient(x, y, a, b, 0.7)
    for t in range(5):
        for v in range(9):
            if np.isinf(x[t, v]):
                assert g[t, v] == 0
                continue
            d = np.zeros_like(x)
            d[t, v] = 1e-5
            # central difference: rounding 1e-11, third derivative 1e-10
            assert abs((loss(x + d) - loss(x - d)) / 2e-5 - g[t, v]) < 1e-8


def test_entropy_and_top():
    assert abs(O.entropy(O.log_probabilities(np.zeros((1, 8))))[0] - np.log(8)) < 1e-14
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0]])
    assert O.top(x, 6).tolist() == [[1, 2, 4, 0, -1, -1]]


def test_routes():
    choice = np.array([[2, 0], [0, -1], [5, 2], [0, 0]])
    place, slot, offsets = O.route(choice, 4)
    assert offsets.tolist() == [0, 4, 4, 6, 6]
    assert slot.tolist() == [1, 2, 6, 7, 0, 5, -1, -1]
    assert place.tolist() == [[4, 0], [1, -1], [-1, 5], [2, 3]]


def test_join_gradient_is_the_difference():
    r = np.random.default_rng(1)
    rows, w, dy = r.standard_normal((6, 3)), r.standard_normal((3, 2)), r.standard_normal((3, 3))
    place = np.array([[4, 0], [1, -1], [9, 5]])
    drows, dw, _ = O.join_grad(dy, rows, place, w)
    f = lambda rows, w: (O.join(rows, place, w)[0] * dy).sum()  # noqa: E731
    for r_ in range(6):
        for c in range(3):
            d = np.zeros_like(rows)
            d[r_, c] = 1e-4
            # linear: rounding alone
            assert abs((f(rows + d, w) - f(rows - d, w)) / 2e-4 - (drows[r_][c] if r_ in drows else 0.0)) < 1e-9
    for t in range(3):
        for j in range(2):
            d = np.zeros_like(w)
            d[t, j] = 1e-4
            assert abs((f(rows, w + d) - f(rows, w - d)) / 2e-4 - dw[t, j]) < 1e-9


def test_formats():
    m, v = O.decode_m(np.arange(0x79)), O.decode_v(np.arange(256))
    assert (np.diff(m) > 0).all() and m[-1] == 256 and m[8] == 2.0 ** -6 and m[1] == 2.0 ** -9
    assert (np.diff(v) > 0).all() and v[255] == 32 and v[127] == 0.125 and v[1] == 1.25 * 2.0 ** -19 and v[0] == 0
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8)
    ours = O.decode_m(codes.numpy())
    theirs = codes.view(torch.float8_e4m3fn).float().numpy()
    keep = ~np.isnan(theirs)
    assert (ours[keep] == theirs[keep]).all()


def test_chances_are_even():
    """Of 2^20 elements the mean of 16 bits is within five standard deviations of their middle, the
    halves of a word do not go together, nor do neighbours, tensors or steps."""
    n = 1 << 20
    h = O.chances(7, 3, 1, np.arange(n, dtype=np.uint64))
    sigma = 5 / np.sqrt(n)
    unit = lambda h: ((h & np.uint64(0xffff)).astype(np.float64) + 0.5) / 65536 - 0.5  # noqa: E731
    a, b = unit(h) * np.sqrt(12), unit(h >> np.uint64(16)) * np.sqrt(12)
    others = [unit(O.chances(*k, np.arange(n, dtype=np.uint64))) * np.sqrt(12) for k in ((7, 4, 1), (7, 3, 2), (8, 3, 1))]
    high = unit(O.chances(7, 3, 1, (1 << 32) + np.arange(n, dtype=np.uint64))) * np.sqrt(12)
    assert abs(a.mean()) < sigma and abs(b.mean()) < sigma and abs(a.var() - 1) < sigma
    for other in [b, np.roll(a, 1), np.roll(a, 2), np.roll(a, 256), high] + others:
        assert abs((a * other).mean()) < sigma
    counts = np.bincount((h & np.uint64(0xff)).astype(np.int64), minlength=256)
    assert abs(counts - n / 256).max() < 6 * np.sqrt(n / 256)


@pytest.mark.parametrize("which", ["m", "v"])
def test_rounding_is_even_handed(which):
    """The mean of many roundings of one value is the value: within five
    standard deviations of at most half a step each, and half a 65536th step."""
    codes = O.decode_m(np.arange(0x79)) if which == "m" else O.decode_v(np.arange(256))
    n = 1 << 16
    h = O.chances(1, 1, 1, np.arange(n, dtype=np.uint64)) & np.uint64(0xffff)
    for y in [1.0, 1.03, 17.77, 0.3001, 0.0171, 31.9]:
        got = codes[O.encode(np.full(n, y), 1.0, codes, h)]
        low = np.searchsorted(codes, y, side="right") - 1
        step = codes[low + 1] - codes[low]
        assert set(got) <= {codes[low], codes[low + 1]}
        assert abs(got.mean() - y) <= step * (5 * 0.5 / np.sqrt(n) + 2.0 ** -17)


def test_adamw_moves_against_the_gradient():
    p, m, v = O.adamw(np.array([1.0]), np.array([0.5]), np.zeros(1), np.zeros(1), 1, lr=0.1, decay=0.0)
    assert abs(p[0] - (1.0 - 0.1 * 0.5 / (0.5 + 1e-8))) < 1e-12     # the first step is lr whatever the gradient
