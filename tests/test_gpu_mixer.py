"""The sequence block as a whole on the GPU: against the oracle's operators put together in 64 bits, sample by sample, and learning."""
import sys

import numpy as np
import pytest
import torch

import oracle
from paper_2405_04416_amd.binding import DistGridError
from paper_2405_04416_amd.mixer import EPS, RayMixer, train_example

from gpu_util import DEV

pytestmark = pytest.mark.gpu

# fp32: a norm is off by some 40 half units of values up to 4, a gate by a quarter of what its argument is, and a state gathers the errors
# of the some 20 tokens that it remembers: 800 half units of the largest value, 1000 with the rest
TOL = 1000 * 2.0 ** -24


def say(*what):
    print("[case]", *what)
    sys.stdout.flush()


def _close(got, want):
    got = got.double().cpu().numpy()
    assert np.abs(got - want).max() <= TOL * max(1.0, np.abs(want).max())


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("first", [None, [0, 7, 7, 40, 64, 90]], ids=["even", "ragged"])
def test_block_against_the_oracle(first, reverse):
    say("block", first, reverse)
    rng = np.random.default_rng(0)
    N, W, n_seq = 90, 24, 5
    offsets = np.arange(6) * 18 if first is None else np.array(first)
    x, dy = rng.standard_normal((N, W)).astype(np.float32), rng.standard_normal((N, W)).astype(np.float32)
    h0, dlast = rng.standard_normal((n_seq, W)).astype(np.float32), rng.standard_normal((n_seq, W)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).to(DEV)
    block = RayMixer(W, torch.float32, p=0.25, reverse=reverse, seed=77, device=DEV)
    params = rng.standard_normal((4, W)).astype(np.float32) * 0.3 + 1.0
    block.params.copy_(dev(params).reshape(-1))
    f = None if first is None else dev(np.array(first, np.int32))
    h_last, dh0 = torch.zeros(n_seq, W, device=DEV), torch.zeros(n_seq, W, device=DEV)
    block.forward(dev(x), n_seq, f)                                 # a pass before: other words of the generator from here on
    used = block.drawn
    y = block.forward(dev(x), n_seq, f, dev(h0), h_last)
    dx = block.backward(dev(dy), dev(dlast), dh0)
    z, u = oracle.layer_norm_fwd(x, params[0], params[1], EPS), oracle.layer_norm_fwd(x, params[2], params[3], EPS)
    m, last = oracle.recurrence_fwd(z, u, offsets, reverse, h0)
    keep, factor = oracle.dropout_mask(77, used, N * W, 0.25)
    mask = keep.reshape(N, W) * factor
    _close(y, x + mask * m)
    _close(h_last, last)
    dz, du, g0 = oracle.recurrence_bwd(z, u, offsets, dy * mask, reverse, h0, dlast)
    dx_z, dgz, dbz = oracle.layer_norm_bwd(x, params[0], dz, EPS)
    dx_u, dgu, dbu = oracle.layer_norm_bwd(x, params[2], du, EPS)
    _close(dx, dy + dx_z + dx_u)
    _close(dh0, g0)
    _close(block.grads.view(4, W), np.stack([dgz, dbz, dgu, dbu]))


def test_block_sample_by_sample():
    """Without dropout, a ray read one sample after the other gives the ray read at once."""
    say("block steps")
    torch.manual_seed(0)
    n_seq, S, W = 6, 12, 32
    x = torch.randn(n_seq, S, W, device=DEV)
    block = RayMixer(W, torch.float32, device=DEV)
    last = torch.zeros(n_seq, W, device=DEV)
    whole = block.forward(x.reshape(n_seq * S, W), n_seq, h_last=last, training=False).clone().view(n_seq, S, W)
    h = torch.zeros(n_seq, W, device=DEV)
    for t in range(S):
        y = block.advance(x[:, t].contiguous(), h)
        _close(y, whole[:, t].double().cpu().numpy())
    _close(h, last.double().cpu().numpy())


def test_block_across_two_partitions():
    """The state that leaves one segment enters the next one: the same as the whole ray, gradients included."""
    say("block partitions")
    torch.manual_seed(1)
    n_seq, S, W = 4, 32, 16
    x, dy = torch.randn(n_seq, 2 * S, W, device=DEV), torch.randn(n_seq, 2 * S, W, device=DEV)
    flat = lambda t: t.reshape(-1, W).contiguous()
    whole, near, far = (RayMixer(W, torch.float32, p=0.0, device=DEV) for _ in range(3))
    y = whole.forward(flat(x), n_seq).view(n_seq, 2 * S, W)
    state, back = torch.zeros(n_seq, W, device=DEV), torch.zeros(n_seq, W, device=DEV)
    y_near = near.forward(flat(x[:, :S]), n_seq, h_last=state).view(n_seq, S, W)
    y_far = far.forward(flat(x[:, S:]), n_seq, h0=state).view(n_seq, S, W)
    _close(torch.cat([y_near, y_far], 1), y.double().cpu().numpy())
    dx = whole.backward(flat(dy)).view(n_seq, 2 * S, W)
    dx_far = far.backward(flat(dy[:, S:]), dh0=back).view(n_seq, S, W)
    dx_near = near.backward(flat(dy[:, :S]), dh_last=back).view(n_seq, S, W)
    _close(torch.cat([dx_near, dx_far], 1), dx.double().cpu().numpy())
    _close(near.grads + far.grads, whole.grads.double().cpu().numpy())


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.bfloat16])
def test_block_learns(dtype):
    """The same training in autograd takes the error from 0.64 to 0.23; half is left for dropout and for other random numbers."""
    say("block learns", dtype)
    first, last = train_example(rays=512, samples=48, iterations=120, dtype=dtype, report=None)
    assert np.isfinite(last) and last < 0.5 * first


def test_block_on_its_own_result():
    """A result that goes in again is not overwritten before the gradient has used it."""
    say("block twice")
    torch.manual_seed(2)
    n_seq, S, W = 5, 30, 24
    x, dy = torch.randn(n_seq * S, W, device=DEV), torch.randn(n_seq * S, W, device=DEV)
    got, want = [], []
    for out, again in ((got, lambda y: y), (want, lambda y: y.clone())):
        block = RayMixer(W, torch.float32, p=0.2, seed=3, device=DEV)
        for _ in range(3):
            y = again(block.forward(x, n_seq))
            z = block.forward(y, n_seq)
            out += [z.clone(), block.backward(dy).clone(), block.grads.clone()]
            out += [block.forward(again(block.backward(dy)), n_seq).clone(), block.backward(dy).clone(), block.grads.clone()]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_gradient_is_of_the_pass_that_was():
    """A schedule may change p before the gradient is taken."""
    say("block p")
    torch.manual_seed(3)
    n_seq, S, W = 4, 20, 16
    x, dy = torch.randn(n_seq * S, W, device=DEV), torch.randn(n_seq * S, W, device=DEV)
    out = []
    for later in (0.3, 0.9):
        block = RayMixer(W, torch.float32, p=0.3, device=DEV)
        block.forward(x, n_seq)
        block.p = later
        out.append((block.backward(dy).clone(), block.grads.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_block_refuses_states_in_place_in_training():
    """The gradient needs the state that went in."""
    say("block h0")
    n_seq, S, W = 4, 20, 16
    x, h = torch.randn(n_seq * S, W, device=DEV), torch.randn(n_seq, W, device=DEV)
    block = RayMixer(W, torch.float32, device=DEV)
    for last in (h, h.view(-1), h.view(n_seq, W)):
        with pytest.raises(DistGridError):
            block.forward(x, n_seq, h0=h, h_last=last)
    block.forward(x, n_seq, h0=h, h_last=h, training=False)
    block.forward(x, n_seq, h0=h, h_last=torch.empty_like(h))
    both = torch.zeros(2, n_seq, W, device=DEV)
    block.forward(x, n_seq, h0=both[0], h_last=both[1])
    assert both[1].any() and not both[0].any()
