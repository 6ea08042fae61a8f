"""Pins of the 64-bit forms of the operators that train a routed block: gradients
against differences, the polynomial against the singular values, and planted
mistakes that the pins have to see."""
import numpy as np
import pytest

from oracle import train

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def rng(seed):
    return np.random.default_rng(seed)


def numeric(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        u, v = x.copy(), x.copy()
        u[i] += h
        v[i] -= h
        g[i] = (f(u) - f(v)) / (2 * h)
    return g


# a difference of step h errs by h^2 times a third derivative (0 here, but across a
# rectifier's border) and by 2^-53 / h of the values, some 1e-9
DIFF = 1e-7


def case(seed, T, k, E, N, K, shared):
    r = rng(seed)
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)])
    ids[r.random(ids.shape) < 0.15] = -1
    return (r.standard_normal((T, K) if shared else (T, k, K)), r.standard_normal((E, N, K)), ids, r.random(ids.shape))


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("form", ["plain", "relu", "combine"])
def test_gradients_against_differences(shared, form):
    x, w, ids, s = case(3, 4, 2, 3, 5, 6, shared)
    relu, weights = form == "relu", s if form == "combine" else None
    y, _ = train.expert_linear(x, w, ids, relu, weights)
    dy = rng(5).standard_normal(y.shape)
    got = train.expert_linear_bwd(dy, x, w, ids, y if relu else None, weights)
    f = lambda x_, w_, s_: (train.expert_linear(x_, w_, ids, relu, s_)[0] * dy).sum()  # noqa: E731
    assert np.abs(got["dx"][0] - numeric(lambda v: f(v, w, weights), x)).max() < DIFF
    assert np.abs(got["dw"][0] - numeric(lambda v: f(x, v, weights), w)).max() < DIFF
    if weights is not None:
        empty = ids < 0
        assert np.abs(got["dweights"][0] - numeric(lambda v: f(x, w, v), s))[~empty].max() < DIFF
        assert (got["dweights"][0][empty] == 0).all()
    for value, size in got.values():
        assert (np.abs(value) <= size * (1 + 1e-12)).all()


def test_differences_see_mistakes():
    x, w, ids, s = case(3, 4, 2, 3, 5, 6, False)
    y, _ = train.expert_linear(x, w, ids, False, s)
    dy = rng(5).standard_normal(y.shape)
    want = numeric(lambda v: (train.expert_linear(v, w, ids, False, s)[0] * dy).sum(), x)
    unweighted = train.expert_linear_bwd(np.repeat(dy[:, None], 2, 1), x, w, ids)["dx"][0]
    assert np.abs(unweighted - want).max() > 0.01
    swapped = train.expert_linear_bwd(dy, x, w, np.where(ids == 0, 1, np.where(ids == 1, 0, ids)), None, s)["dx"][0]
    assert np.abs(swapped - want).max() > 0.01


def test_lists():
    ids = np.array([[2, 0], [-1, 2], [0, 1], [7, -1]])
    offsets, order = train.lists(ids, 3)
    assert offsets.tolist() == [0, 2, 3, 5] and order.tolist() == [1, 4, 5, 0, 3, -1, -1, -1]


@pytest.mark.parametrize("M,N", [(1, 1), (1, 7), (5, 5), (6, 20), (20, 6)])
def test_orthogonalize_is_a_polynomial_of_the_singular_values(M, N):
    g = rng(M * 100 + N).standard_normal((M, N))
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-7)
    for a, b, c in [COEFFICIENTS] * 5:
        s = s * (a + b * s ** 2 + c * s ** 4)
    got = train.orthogonalize(g, [COEFFICIENTS] * 5, 1e-7)
    assert np.abs(got - (u * s) @ vt).max() < 1e-9
    other = train.orthogonalize(g, [COEFFICIENTS] * 4 + [(3.4445, -4.7750, 2.0)], 1e-7)
    assert np.abs(other - got).max() > 1e-6  # a coefficient's third digit shows


def test_rounded_operands_err_as_stated():
    """2e-3 of the result's norm at most: what the header says."""
    r = rng(8)
    for M, N, rank in ((64, 64, 0), (200, 500, 0), (300, 100, 8), (128, 128, 4)):
        g = r.standard_normal((M, N)) * (0.1 if rank else 1.0)
        if rank:
            g += r.standard_normal((M, rank)) @ r.standard_normal((rank, N))
        exact, rounded = (train.orthogonalize(g, [COEFFICIENTS] * 5, 1e-7, v) for v in (False, True))
        err = np.linalg.norm(rounded - exact) / np.linalg.norm(exact)
        assert 1e-5 < err < 2e-3, (M, N, rank, err)


# What the rounded operands cost, of the result's norm, as the header has it: steps, Frobenius norm, 2-norm.  Sides
# from 65 on: operands in fp16.  The form below was tried on 70 to 105 matrices of each of eight shapes with sides from
# 64 on: 2.7e-3 and 6.0e-3 were the most after 5 steps, 4.0e-3 and 2.0e-2 after 8, 3.3e-2 and 0.22 after 16, 6.2e-2
# and 0.40 after 64; a half more for others and for other roundings of the same size.
ERRORS = [(5, 4e-3, 1e-2), (8, 8e-3, 4e-2), (16, 6e-2, 0.4), (64, 0.12, 0.7)]
# A side of at most 64: operands in two parts.  On 35 to 210 matrices of each of nine shapes from 1 x 1 to 64 x 300 the
# most were 2.6e-5 and 3.8e-5 after 5 steps, 9.3e-5 and 1.6e-4 after 8; fp32 sums add about as much.
SMALL_ERRORS = [(5, 1e-4, 2e-4), (8, 4e-4, 8e-4)]


def draws(M, N, seeds):
    """Noise, and a few strong directions over it, some with rows of unlike lengths."""
    for seed in range(seeds):
        r = rng(seed * 7919 + M * 31 + N)
        rank, noise = [(0, 1), (1, .1), (4, .1), (16, .1), (16, .01), (3, .01), (1, .003)][seed % 7]
        g = r.standard_normal((M, N)) * noise
        if rank:
            g = g + r.standard_normal((M, rank)) @ r.standard_normal((rank, N))
        yield g * np.exp(r.standard_normal((M, 1)) * 2) if seed % 5 == 4 else g


@pytest.mark.parametrize("steps,frobenius,spectral", ERRORS)
@pytest.mark.parametrize("shape", [(65, 65), (65, 300), (100, 100), (130, 66), (200, 300)], ids=str)
def test_rounded_operands_err_by_steps(shape, steps, frobenius, spectral):
    for g in draws(*shape, 21):
        exact, rounded = (train.orthogonalize(g, [COEFFICIENTS] * steps, 1e-7, v) for v in (False, True))
        assert np.linalg.norm(rounded - exact) < frobenius * np.linalg.norm(exact)
        assert np.linalg.norm(rounded - exact, 2) < spectral * np.linalg.norm(exact, 2)


@pytest.mark.parametrize("steps,frobenius,spectral", SMALL_ERRORS)
@pytest.mark.parametrize("shape", [(1, 1), (2, 2), (2, 3), (3, 5), (1, 40), (8, 8), (16, 300), (32, 500), (64, 64), (130, 64)], ids=str)
def test_operands_in_two_parts_err_by_steps(shape, steps, frobenius, spectral):
    for g in draws(*shape, 21):
        exact, rounded = (train.orthogonalize(g, [COEFFICIENTS] * steps, 1e-7, v) for v in (False, "parts"))
        assert np.linalg.norm(rounded - exact) < frobenius * np.linalg.norm(exact)
        assert np.linalg.norm(rounded - exact, 2) < spectral * np.linalg.norm(exact, 2)


def test_small_matrices_need_more_than_fp16():
    """Few singular values, no averaging: 2 x 3 with fp16 operands is off by more than 1e-2 after five steps, and
    with two parts by less than 1e-4."""
    most = [max(np.linalg.norm(train.orthogonalize(g, [COEFFICIENTS] * 5, 1e-7, v) - exact) / np.linalg.norm(exact)
                for g in draws(2, 3, 60) for exact in [train.orthogonalize(g, [COEFFICIENTS] * 5, 1e-7)]) for v in (True, "parts")]
    assert most[0] > 1e-2 and most[1] < 1e-4
