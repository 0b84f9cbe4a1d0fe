"""Pins for the oracle's sequence block (layer norm, gated linear recurrence, dropout): against numpy, closed forms, the compositing
recursion it generalises, and finite differences."""
import numpy as np
import pytest

import oracle


def _differences(f, x, h=1e-6):
    """Gradient of the scalar f by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        was = x[i]
        x[i] = was + h
        up = f()
        x[i] = was - h
        g[i] = (up - f()) / (2 * h)
        x[i] = was
    return g


# ------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("N,W", [(1, 1), (3, 2), (5, 7), (2, 64)])
def test_norm_against_numpy(N, W):
    rng = np.random.default_rng(W)
    x, gamma, beta = rng.standard_normal((N, W)) * 3 + 1, rng.standard_normal(W), rng.standard_normal(W)
    want = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + 1e-5) * gamma + beta
    np.testing.assert_allclose(oracle.layer_norm_fwd(x, gamma, beta, 1e-5), want, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(oracle.layer_norm_fwd(x, None, None, 1e-5) * gamma + beta, want, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("with_gamma", [True, False])
def test_norm_gradient_is_that_of_differences(with_gamma):
    rng = np.random.default_rng(1)
    x, gamma, beta, dy = rng.standard_normal((4, 6)), rng.standard_normal(6), rng.standard_normal(6), rng.standard_normal((4, 6))
    used = gamma if with_gamma else None
    f = lambda: float(np.sum(dy * oracle.layer_norm_fwd(x, used, beta, 1e-2)))
    dx, dgamma, dbeta = oracle.layer_norm_bwd(x, used, dy, 1e-2)
    np.testing.assert_allclose(dx, _differences(f, x), rtol=1e-7, atol=1e-8)
    np.testing.assert_allclose(dbeta, _differences(f, beta), rtol=1e-7, atol=1e-8)
    if with_gamma:
        np.testing.assert_allclose(dgamma, _differences(f, gamma), rtol=1e-7, atol=1e-8)


def test_norm_gradient_does_not_move_mean_or_scale():
    # y does not change when x is shifted, nor (eps = 0) when it is scaled: dx is orthogonal to both directions
    rng = np.random.default_rng(2)
    x, gamma, dy = rng.standard_normal((5, 9)), rng.standard_normal(9), rng.standard_normal((5, 9))
    dx, _, _ = oracle.layer_norm_bwd(x, gamma, dy, 0.0)
    np.testing.assert_allclose(dx.sum(1), 0.0, atol=1e-12)
    np.testing.assert_allclose((dx * x).sum(1), 0.0, atol=1e-12)


# ------------------------------------------------------------------ recurrence
FIRST = np.array([0, 3, 3, 4, 9], np.uint32)        # three tokens, none, one, five


def _inputs(rng, N=9, W=2, n_seq=4):
    return [rng.standard_normal(s) for s in ((N, W), (N, W), (n_seq, W), (N, W), (n_seq, W))]


def test_recurrence_of_one_gate_is_a_running_mean_with_weights():
    # h_T = h0 prod a + sum_t (1 - a_t) u_t prod_{s > t} a_s
    rng = np.random.default_rng(3)
    z, u, h0, _, _ = _inputs(rng, 9, 2, 1)
    y, last = oracle.recurrence_fwd(z, u, [0, 9], h0=h0)
    a = 1 / (1 + np.exp(-z))
    for T in range(1, 10):
        want = h0[0] * np.prod(a[:T], 0) + sum((1 - a[t]) * u[t] * np.prod(a[t + 1:T], 0) for t in range(T))
        np.testing.assert_allclose(y[T - 1], want, rtol=1e-12)
    np.testing.assert_array_equal(last[0], y[-1])


def test_recurrence_back_to_front_composites():
    # with a = exp(-sigma delta), the weights of the samples of a ray gone through back to front are those of Eq. 3
    rng = np.random.default_rng(4)
    sigma, delta, rgb = rng.random(12) * 3, rng.random(12), rng.random((12, 3))
    a = np.exp(-sigma * delta)
    z = np.repeat(np.log(a / (1 - a))[:, None], 3, 1)
    y, last = oracle.recurrence_fwd(z, rgb, [0, 12], reverse=True)
    C, _ = oracle.composite_fwd_ragged(sigma, rgb, delta, [0, 12])
    np.testing.assert_allclose(last[0], C[0], rtol=1e-12)
    np.testing.assert_array_equal(y[0], last[0])


@pytest.mark.parametrize("reverse", [False, True])
def test_recurrence_of_segments_merges(reverse):
    rng = np.random.default_rng(5)
    z, u, h0, _, _ = _inputs(rng, 9, 2, 1)
    y, last = oracle.recurrence_fwd(z, u, [0, 9], reverse, h0)
    near, far = slice(0, 4), slice(4, 9)
    order = (far, near) if reverse else (near, far)
    parts, h = {}, h0
    for sl in order:
        parts[sl.start], h = oracle.recurrence_fwd(z[sl], u[sl], [0, sl.stop - sl.start], reverse, h)
    np.testing.assert_array_equal(np.concatenate([parts[0], parts[4]]), y)
    np.testing.assert_array_equal(h, last)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("carry", [False, True])
def test_recurrence_gradient_is_that_of_differences(reverse, carry):
    rng = np.random.default_rng(6)
    z, u, h0, dy, dlast = _inputs(rng)

    def f():
        y, last = oracle.recurrence_fwd(z, u, FIRST, reverse, h0 if carry else None)
        return float(np.sum(dy * y) + np.sum(dlast * last) * carry)

    dz, du, dh0 = oracle.recurrence_bwd(z, u, FIRST, dy, reverse, h0 if carry else None, dlast if carry else None)
    np.testing.assert_allclose(dz, _differences(f, z), rtol=1e-6, atol=1e-8)
    np.testing.assert_allclose(du, _differences(f, u), rtol=1e-6, atol=1e-8)
    if carry:
        np.testing.assert_allclose(dh0, _differences(f, h0), rtol=1e-6, atol=1e-8)
        np.testing.assert_array_equal(dh0[1], dlast[1])             # the sequence without a token


def test_recurrence_shut_gates_look_at_nothing():
    inf, nan = np.inf, np.nan
    z, u = np.array([[0.0], [inf], [-inf], [88.0], [-88.0]]), np.array([[1.0], [nan], [2.0], [inf], [3.0]])
    y, last = oracle.recurrence_fwd(z, u, [0, 5], h0=[[5.0]])
    np.testing.assert_array_equal(y[:, 0], [3.0, 3.0, 2.0, 2.0, 3.0])
    y, _ = oracle.recurrence_fwd(z, u, [0, 5], h0=[[nan]])
    np.testing.assert_array_equal(y[:, 0], [nan, nan, 2.0, 2.0, 3.0])
    dz, du, dh0 = oracle.recurrence_bwd(z, u, [0, 5], np.ones((5, 1)), h0=[[5.0]])
    np.testing.assert_array_equal(dz[:, 0], [0.5 * 0.5 * 4.0 * 2.0, 0, 0, 0, 0])
    np.testing.assert_array_equal(du[:, 0], [0.5 * 2.0, 0, 2.0, 0, 1.0])
    assert dh0[0, 0] == 1.0


def test_recurrence_leaves_other_rows_alone():
    rng = np.random.default_rng(7)
    z, u, _, dy, _ = _inputs(rng)
    y, _ = oracle.recurrence_fwd(z, u, [2, 4, 7])
    assert np.array_equal(np.isnan(y[:, 0]), [True] * 2 + [False] * 5 + [True] * 2)


# ------------------------------------------------------------------ dropout
def test_dropout_mask_of_known_words():
    keep, factor = oracle.dropout_mask(7, 3, 10, 0.25)
    lib = oracle.lib()
    lib.dgo_rand64.restype, lib.dgo_rand64.argtypes = oracle.C.c_uint64, [oracle.C.c_uint64] * 2
    fields = [(lib.dgo_rand64(7, 3 + i // 4) >> 16 * (i % 4)) & 0xffff for i in range(10)]
    assert list(keep) == [f >= 16384 for f in fields] and factor == 4 / 3


@pytest.mark.parametrize("p", [0.0, 1.0, 0.1, 0.5, 1e-6])
def test_dropout_share(p):
    n = 1 << 18
    keep, factor = oracle.dropout_mask(11, 0, n, p)
    below = np.floor(p * 65536 + 0.5)
    share = 1 - below / 65536
    # six standard deviations of a binomial
    assert abs(keep.mean() - share) <= 6 * np.sqrt(share * (1 - share) / n)
    assert factor == (0.0 if share == 0 else 1 / share)


def test_dropout_masks_of_other_seeds_and_offsets_are_unrelated():
    n = 1 << 16
    a, _ = oracle.dropout_mask(1, 0, n, 0.5)
    for seed, offset in ((2, 0), (1, n // 4), (1 << 40, 0)):
        b, _ = oracle.dropout_mask(seed, offset, n, 0.5)
        assert abs((a == b).mean() - 0.5) <= 6 * 0.5 / np.sqrt(n)
    b, _ = oracle.dropout_mask(1, 5, n, 0.5)
    np.testing.assert_array_equal(a[20:], b[:-20])                  # the words of a stretch are its own
