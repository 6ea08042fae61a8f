"""Pins of the feed-forward operators' 64-bit forms: gradients against
differences, the group formats against exhaustive search, closed forms, and
planted mistakes that the pins have to see."""
import numpy as np
import pytest

from oracle import ffn


def rng(seed):
    return np.random.default_rng(seed)


def numeric(f, x, h=1e-6):
    """Central differences of a scalar function."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        u, v = x.copy(), x.copy()
        u[i] += h
        v[i] -= h
        g[i] = (f(u) - f(v)) / (2 * h)
    return g


# a difference of step h errs by h^2 times a third derivative and by 2^-53 / h
# of the values: some 1e-9 here; 1e-6 leaves room for both
DIFF = 1e-6


@pytest.mark.parametrize("T,D", [(1, 1), (2, 5), (3, 33)])
def test_norm_gradient_against_differences(T, D):
    r = rng(T * 100 + D)
    h, w, dy, dh = r.standard_normal((T, D)), 1 + 0.1 * r.standard_normal(D), *r.standard_normal((2, T, D))
    eps = 1e-3
    rstd = ffn.rmsnorm(h, w, eps)[1]

    def loss(hh, ww):
        return (ffn.rmsnorm(hh, ww, eps)[2] * dy).sum() + (hh * dh).sum()

    # the formula treats mean(h^2) + eps = rstd^-2
    dx, dw = ffn.rmsnorm_bwd(dy, h, w, rstd, dh)
    assert np.allclose(dx, numeric(lambda v: loss(v, w), h), atol=DIFF)
    assert np.allclose(dw, numeric(lambda v: loss(h, v), w), atol=DIFF)
    wrong = ffn.rmsnorm_bwd(dy, h, w, rstd * 1.01, dh)[0]
    assert not np.allclose(wrong, numeric(lambda v: loss(v, w), h), atol=DIFF)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(2, 5, 2), (3, 9, 4), (1, 3, 3)])
def test_route_gradient_against_differences(T, E, k, renorm, score):
    r = rng(E * 10 + k)
    logits, dw = r.standard_normal((T, E)), r.standard_normal((T, k))
    ids = ffn.route(logits, k, score=score, renorm=renorm, scale=1.7)[0]

    def loss(v):
        s = np.stack([ffn.scores(row, score)[0] for row in v])
        w = np.take_along_axis(s, ids.astype(np.int64), 1)
        w = 1.7 * (w / (w.sum(1, keepdims=True) + 1e-20) if renorm else w)
        return (w * dw).sum()

    got = ffn.route_bwd(dw, logits, ids, score, renorm, 1.7)
    assert np.allclose(got, numeric(loss, logits), atol=DIFF)
    other = "sigmoid" if score == "softmax" else "softmax"
    if not (renorm and k == E and score == "softmax"):
        assert not np.allclose(ffn.route_bwd(dw, logits, ids, other, renorm, 1.7), numeric(loss, logits), atol=DIFF)


def test_route_choice_rules():
    l = np.array([[1.0, 3.0, 3.0, 2.0], [-np.inf, -np.inf, 0.0, np.nan], [-np.inf] * 4])
    ids, w, offsets, order = ffn.route(l, 2)
    assert ids.tolist() == [[1, 2], [2, -1], [-1, -1]]  # a tie to the lowest; a masked expert never
    assert np.allclose(w, [[0.5, 0.5], [1, 0], [0, 0]])
    assert offsets.tolist() == [0, 0, 1, 3, 3] and order.tolist() == [0, 1, 2, -1, -1, -1]
    # groups by the sum of their two best: (5 + 0) < (3 + 3), though 5 is the largest
    l = np.array([[5.0, -9.0, 3.0, 3.0]])
    ids, _, _, _ = ffn.route(l, 2, bias=np.array([0.5, 0, 0.5, 0.5]), score="sigmoid", groups=2, keep=1)
    assert ids.tolist() == [[2, 3]]
    # the bias chooses and does not weigh
    ids, w, _, _ = ffn.route(np.array([[0.0, 0.0]]), 1, bias=np.array([0.0, 1.0]), score="sigmoid", renorm=False)
    assert ids.tolist() == [[1]] and np.allclose(w, 0.5)


def test_formats_exhaustively():
    codes = np.arange(256, dtype=np.uint8)
    v = ffn.e4m3_values(codes)
    assert np.isnan(v[[127, 255]]).all() and np.nanmax(v) == 448.0 and v[1] == 2.0 ** -9
    assert np.all(np.diff(v[:127]) > 0) and np.array_equal(-v[:127], v[128:255])
    w = ffn.fp4_values(np.array([[0x10, 0x32, 0x54, 0x76, 0x98, 0xba, 0xdc, 0xfe]], dtype=np.uint8),
                       np.array([[128]], dtype=np.uint8), 16)
    assert w[0].tolist() == [0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12]


@pytest.mark.parametrize("top", [6.0, 448.0])
def test_group_scale_is_the_smallest_that_fits(top):
    r = rng(5)
    v = r.standard_normal((50, 32)) * np.exp(r.uniform(-20, 20, (50, 1)))
    v[0], v[1, 0], v[2, 0] = 0, np.inf, np.nan
    v[3] = 0
    v[3, 7] = top * 4  # exactly a scale's top
    e = ffn.scale_exponents(v, top)[:, 0]
    assert e[0] == -127 and e[1] == e[2] == 128 and e[3] == 2
    for i in range(4, 50):
        a = np.abs(v[i]).max()
        assert a <= top * 2.0 ** e[i] and a > top * 2.0 ** (e[i] - 1)


def test_quantize_is_nearest():
    r = rng(6)
    w = r.standard_normal((20, 65))
    codes, b = ffn.fp4_quantize(w)
    assert codes.shape == (20, 33) and b.shape == (20, 3)
    v = ffn.fp4_values(codes, b, 65)
    scale = np.repeat(ffn.scale_values(b), 32, axis=-1)[:, :65]
    grid = np.concatenate([-ffn.FP4, ffn.FP4])
    best = np.abs(w[..., None] / scale[..., None] - grid).min(axis=-1)
    assert np.allclose(np.abs(w - v) / scale, best, atol=1e-12)
    ties, _ = ffn.fp4_quantize(np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]]))
    assert ffn.fp4_values(ties, np.array([[127]], np.uint8), 8).tolist() == [[0, 1, 1, 2, 2, 4, 4, 6]]


def test_products():
    r = rng(7)
    w, x = r.standard_normal((3, 4, 6)), r.standard_normal((2, 6))
    x[0, 2] = 0
    w[:, 1, 2] = np.nan
    y, _ = ffn.product(w[0], x[:1], skip=True)
    assert np.isfinite(y).all()
    assert np.isnan(ffn.product(w[0], x[:1])[0][0, 1])
    ids = np.array([[2, -1], [0, 2]])
    y, _ = ffn.routed(w, x, ids)
    assert np.allclose(y[0, 0, 0], w[2, 0] @ x[0]) and (y[0, 1] == 0).all() and np.isnan(y[1, 0, 1])
