"""Pins for the oracle's block with an associative memory (root-mean-square norm, rows in 8 bits, gated delta rule): against numpy, torch's own type,
closed forms and finite differences."""
import numpy as np
import pytest
import torch

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


# ------------------------------------------------------------------ root-mean-square norm
@pytest.mark.parametrize("N,W", [(1, 1), (3, 2), (5, 7), (2, 64)])
def test_norm_against_numpy(N, W):
    rng = np.random.default_rng(W)
    x, gamma = rng.standard_normal((N, W)) * 3 + 1, rng.standard_normal(W)
    want = x / np.sqrt((x * x).mean(1, keepdims=True) + 1e-5)
    np.testing.assert_allclose(oracle.rms_norm_fwd(x, gamma, 1e-5), want * gamma, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(oracle.rms_norm_fwd(x, None, 1e-5), want, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("with_gamma", [True, False])
def test_norm_gradient_is_that_of_differences(with_gamma):
    rng = np.random.default_rng(1)
    x, gamma, dy = rng.standard_normal((4, 6)), rng.standard_normal(6), rng.standard_normal((4, 6))
    used = gamma if with_gamma else None
    f = lambda: float(np.sum(dy * oracle.rms_norm_fwd(x, used, 1e-2)))
    dx, dgamma = oracle.rms_norm_bwd(x, used, dy, 1e-2)
    np.testing.assert_allclose(dx, _differences(f, x), rtol=1e-7, atol=1e-8)
    if with_gamma:
        np.testing.assert_allclose(dgamma, _differences(f, gamma), rtol=1e-7, atol=1e-8)


# ------------------------------------------------------------------ rows in 8 bits
def test_rows_are_the_nearest_of_the_type():
    """With scales of 1 the values are those that torch rounds to; ties go to even."""
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.standard_normal(500) * 10.0 ** rng.integers(-4, 3, 500), np.arange(-64, 64) / 1024.0, np.arange(1, 60) * 0.75])
    x = np.clip(x, -440, 440).astype(np.float32)
    blocks = [np.concatenate([x[i:i + 127], [448.0]]) for i in range(0, x.size, 127)]
    for b in blocks:
        q, s = oracle.e4m3_rows(b[None])
        assert s.tolist() == [[127]]
        np.testing.assert_array_equal(q[0], torch.from_numpy(b.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy())


def test_rows_scales():
    x = np.zeros((1, 400))
    x[0, 0], x[0, 128], x[0, 256], x[0, 390] = 448.0, -448.5, 2.0 ** -140, 3.0e38
    x[0, 1], x[0, 2] = np.inf, np.nan
    q, s = oracle.e4m3_rows(x)
    assert s.tolist() == [[127, 128, 0, 247]]
    assert np.isnan(q[0, 1:3]).all() and q[0, 0] == 448.0 and q[0, 128] == -224.0 and q[0, 256] == 0.0
    assert q[0, 390] == 224.0                # 225.7, in steps of 16


# ------------------------------------------------------------------ gated delta rule
FIRST = np.array([0, 3, 3, 4, 9], np.uint32)        # three tokens, none, one, five


def _inputs(rng, N=9, Hk=1, H=2, Dk=3, Dv=2, n_seq=4):
    q, k = rng.standard_normal((N, Hk, Dk)), rng.standard_normal((N, Hk, Dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return dict(q=q, k=k, v=rng.standard_normal((N, H, Dv)), g=-rng.random((N, H)), beta=rng.random((N, H)), s0=rng.standard_normal((n_seq, H, Dk, Dv)))


@pytest.mark.parametrize("reverse", [False, True])
def test_delta_rule_against_numpy(reverse):
    a = _inputs(np.random.default_rng(3), Hk=2, H=4)
    o, last = oracle.delta_rule_fwd(a["q"], a["k"], a["v"], a["g"], a["beta"], FIRST, 0.5, reverse, a["s0"])
    for j in range(4):
        for h in range(4):
            S = a["s0"][j, h]
            rows = range(FIRST[j], FIRST[j + 1])
            for i in (reversed(rows) if reverse else rows):
                k = a["k"][i, h // 2]
                S = np.exp(a["g"][i, h]) * S
                S = S + a["beta"][i, h] * np.outer(k, a["v"][i, h] - S.T @ k)
                np.testing.assert_allclose(o[i, h], 0.5 * S.T @ a["q"][i, h // 2], rtol=1e-12, atol=1e-12)
            np.testing.assert_allclose(last[j, h], S, rtol=1e-12, atol=1e-12)


def test_delta_rule_gives_back_what_it_stored():
    """Keys at right angles, rate 1, nothing forgotten: a query that is a key reads that key's value, and storing under a key again replaces it."""
    k = np.eye(4)[[0, 1, 2, 3, 1]][:, None, :]
    v = np.random.default_rng(4).standard_normal((5, 1, 3))
    q = np.eye(4)[[0, 0, 1, 0, 1]][:, None, :]
    o, _ = oracle.delta_rule_fwd(q, k, v, np.zeros((5, 1)), np.ones((5, 1)), [0, 5])
    np.testing.assert_allclose(o[:, 0], v[[0, 0, 1, 0, 4], 0], atol=1e-15)


def test_delta_rule_forgets_with_a_shut_gate():
    a = _inputs(np.random.default_rng(5), n_seq=1)
    a["g"][4] = -np.inf
    a["g"][6] = -105.0
    o, last = oracle.delta_rule_fwd(a["q"], a["k"], a["v"], a["g"], a["beta"], [0, 9], 1.0, False, a["s0"])
    o2, last2 = oracle.delta_rule_fwd(*(a[n][4:] for n in ("q", "k", "v", "g", "beta")), [0, 2, 5])
    np.testing.assert_array_equal(o[4:], o2)
    np.testing.assert_array_equal(last[0], last2[1])


@pytest.mark.parametrize("reverse,carry", [(False, False), (True, True)])
def test_delta_rule_gradient_is_that_of_differences(reverse, carry):
    rng = np.random.default_rng(6)
    a = _inputs(rng)
    do, dl = rng.standard_normal(a["v"].shape), rng.standard_normal(a["s0"].shape)
    s0, ds_last = (a["s0"], dl) if carry else (None, None)

    def f():
        o, last = oracle.delta_rule_fwd(a["q"], a["k"], a["v"], a["g"], a["beta"], FIRST, 0.7, reverse, s0)
        return float(np.sum(o * do) + (np.sum(last * dl) if carry else 0.0))

    got = oracle.delta_rule_bwd(a["q"], a["k"], a["v"], a["g"], a["beta"], FIRST, do, 0.7, reverse, s0, ds_last)
    for name, d in zip(("q", "k", "v", "g", "beta", "s0"), got):
        if name != "s0" or carry:
            np.testing.assert_allclose(d, _differences(f, a[name]), rtol=1e-6, atol=1e-8, err_msg=name)


def test_delta_rule_rows_of_no_sequence():
    a = _inputs(np.random.default_rng(7))
    args = [a[n] for n in ("q", "k", "v", "g", "beta")]
    o, _ = oracle.delta_rule_fwd(*args, [2, 5, 8])
    held = np.isfinite(o).all((1, 2))
    assert held.tolist() == [False] * 2 + [True] * 6 + [False]
    dv = oracle.delta_rule_bwd(*args, [2, 5, 8], np.ones_like(o))[2]
    assert np.isnan(dv[~held]).all() and np.isfinite(dv[held]).all()
