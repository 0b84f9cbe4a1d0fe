"""The sequence block as a whole on the GPU: against the oracle's operators put together in 64 bits, sample by sample, and learning."""
import sys

import numpy as np
import pytest
import torch

import dg_inputs as di
import oracle
from paper_2405_04416_amd import binding as B
from paper_2405_04416_amd.binding import DistGridError
from paper_2405_04416_amd.mixer import EPS, RayMixer, train_example

from gpu_util import DEV, dev, host, rel_err

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


def test_a_graph_outlives_passes_of_other_sizes():
    """What a captured pass works in is not given back when passes of other sizes need other buffers."""
    say("block, sizes between replays")
    torch.manual_seed(5)
    n_seq, S, W = 6, 200, 48
    x, dy = torch.randn(n_seq * S, W, device=DEV), torch.randn(n_seq * S, W, device=DEV)
    block, twin = (RayMixer(W, torch.float32, p=0.0, device=DEV) for _ in range(2))
    step = lambda b: [b.forward(x, n_seq), b.backward(dy), b.grads]
    step(block)                                     # its buffers are there before the graph is
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step(block)
    for n in (600, 12, 2400):
        z = torch.randn(n, W, device=DEV)
        block.forward(z, n_seq)
        block.backward(z)
        block.advance(z[:n_seq], torch.zeros(n_seq, W, device=DEV))
    others = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for size in [1 << 10, 1 << 14, 1 << 17, 1 << 18, 1 << 19, 1 << 21] for _ in range(40)]
    for _ in range(3):
        for z in (x, dy): z.copy_(torch.randn(z.shape, device=DEV))
        for z in results: z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, step(twin)): assert torch.equal(a, b)
        for z in others: assert bool((z == 7).all())


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


def test_block_between_the_encode_and_the_networks():
    """Features of a hash grid, the samples of a segment one after the other, through the block to the field networks and back to the table: every
    hand-over against the oracle on what the stage before it gave.  A stage rounds to fp16 some eight times, 2^-11 of values up to twice its
    result's: 0.01 of it."""
    say("block in the field")
    rng = np.random.default_rng(6)
    n_seg, S, scale = 41, 32, 64.0
    N = n_seg * S
    u = di.make_unit_coords(N, seed=7)
    growth = B.dg_growth_factor(16, 512, 16)
    grid, ref_grid = B.dg_grid_desc_init(16, 2, 14, 16, growth, [1.0, 1.0, 1.0]), oracle.grid_init(16, 2, 14, 16, growth, [1.0, 1.0, 1.0])
    table = di.make_table(ref_grid.n_entries, 2, 1.0, seed=8)
    order = B.dg_order_desc_init(grid, N)
    ordered, pieces = torch.zeros(N, 4, device=DEV), torch.zeros(B.dg_order_pieces_words(order, N), dtype=torch.int32, device=DEV)
    B.dg_order_samples(order, dev(u), N, ordered, pieces, torch.zeros(B.dg_order_workspace_bytes(order) // 4, dtype=torch.int32, device=DEV))
    feat = torch.empty(N, 32, dtype=torch.float16, device=DEV)
    B.dg_hashgrid_encode_fwd_ordered(grid, dev(table), ordered, N, feat)
    assert rel_err(host(feat).astype(np.float64), oracle.encode_fwd(ref_grid, table, u)) <= 2.0 ** -10
    block = RayMixer(32, torch.float16, p=0.0, device=DEV)
    params = (rng.standard_normal((4, 32)) * 0.2 + 1.0).astype(np.float32)
    block.params.copy_(dev(params).reshape(-1))
    y = block.forward(feat, n_seg)
    x64, offsets = host(feat).astype(np.float64), np.arange(n_seg + 1) * S
    z, v = oracle.layer_norm_fwd(x64, params[0], params[1], EPS), oracle.layer_norm_fwd(x64, params[2], params[3], EPS)
    assert rel_err(host(y).astype(np.float64), x64 + oracle.recurrence_fwd(z, v, offsets)[0]) <= 0.01
    mlp, ref_mlp = B.dg_mlp_desc(32, 64, 16, 16, 64, 2, 1), oracle.mlp_desc(32, 64, 16, 16, 64, 2, 1)
    weights, dirs = (rng.standard_normal(9408) * 0.2).astype(np.float16), rng.standard_normal((n_seg, 16)).astype(np.float16)
    dsigma, drgb = rng.standard_normal(N).astype(np.float32) * 0.01, rng.standard_normal((N, 3)).astype(np.float32) * 0.01
    sigma, rgb, dfeat = torch.zeros(N, device=DEV), torch.zeros(N, 3, device=DEV), torch.zeros(N, 32, device=DEV)
    dW, largest = torch.zeros(9408, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.dg_mlp_fwd_rows(mlp, dev(weights), y, dev(dirs), None, S, N, sigma, rgb)
    B.dg_mlp_bwd_rows(mlp, dev(weights), y, dev(dirs), None, S, N, dev(dsigma), dev(drgb), 256.0, 16, dfeat, largest, dW,
                      torch.zeros(B.dg_mlp_bwd_app_workspace_bytes(mlp, N, S) // 4 + 64, device=DEV))
    y64 = host(y).astype(np.float64)
    w_sigma, w_rgb = oracle.mlp_fwd(ref_mlp, weights, y64, dirs, S)
    assert rel_err(host(sigma), w_sigma) <= 0.01 and rel_err(host(rgb), w_rgb) <= 0.01
    assert rel_err(host(dfeat), oracle.mlp_bwd(ref_mlp, weights, y64, dirs, S, dsigma, drgb, 256.0)[0]) <= 0.01
    dy = (dfeat * scale).half()                                     # the networks give their gradient in fp32
    dx = block.backward(dy)
    dy64 = host(dy).astype(np.float64)
    dz, dv, _ = oracle.recurrence_bwd(z, v, offsets, dy64)
    w_dx = dy64 + oracle.layer_norm_bwd(x64, params[0], dz, EPS)[0] + oracle.layer_norm_bwd(x64, params[2], dv, EPS)[0]
    assert rel_err(host(dx).astype(np.float64), w_dx) <= 0.01
    dtable, ws = torch.zeros(ref_grid.n_entries, 2, device=DEV), torch.zeros(B.dg_hashgrid_encode_bwd_workspace_bytes(grid, N) // 4 + 64, device=DEV)
    B.dg_hashgrid_encode_bwd(grid, dev(u), (dx.float() / scale).view(N, 16, 2).transpose(0, 1).contiguous(), N, dtable, ws)     # and it is read in planes
    assert rel_err(host(dtable), oracle.encode_bwd(ref_grid, u, host(dx).astype(np.float64) / scale)) <= 0.01
