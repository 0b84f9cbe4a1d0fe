"""The block with an associative memory as a whole on the GPU: against the oracle's operators put together in 64 bits, sample by sample, in a graph, and its example."""
import numpy as np
import pytest
import torch

import dg_inputs as di
import oracle
from paper_2405_04416_amd import binding as B
from paper_2405_04416_amd.binding import DistGridError
from paper_2405_04416_amd.memory import EPS, KEY_EPS, DeltaMixer, train_example

from gpu_util import DEV, dev, host, rel_err
from test_gpu_memory import worth
from test_gpu_sequence import TYPES, f32, got, rounded, say

pytestmark = pytest.mark.gpu

# Results go through some eight roundings to 16 bits (bf16: 2^-8 at most, 2^-9 in the mean) and up to four to 8 bits, which the reference makes as well; but a value within the
# error of the former of a step's edge falls on its other side, 2^-3 of the value away at most.  With errors of 8 2^-9 = 2^-6 that happens to one in eight at most, to 2^-3 sqrt(1/8) =
# 0.044 of the values in root mean square each time, 0.09 over four; fp16 errors are an eighth, and 0.03 covers them.
TOL = {"fp16": 0.03, "bf16": 0.09}


def close(what, value, want, dtype):
    err, size = np.linalg.norm(got(value).reshape(want.shape) - want), np.linalg.norm(want)
    assert err <= TOL[dtype] * size, "%s: off by %.3g of %.3g" % (what, err, size)


def in_8_bits(x):
    q, s = oracle.e4m3_rows(x)
    return q * np.repeat(np.exp2(s.astype(np.float64) - 127.0), 128, axis=1)[:, :x.shape[1]]


def the_oracles(block, x, r, g, beta, offsets, s0, dt, dout, ds_last):
    """(t, out, s_last, dx, dgamma, dg, dbeta, ds0) in 64 bits, rounded to 8 bits where the block is."""
    Hk, H, Dk, Dv, wq = block.Hk, block.H, block.Dk, block.Dv, block.wq
    N = len(x)
    w_qv, w_k, w_o = (worth(*w) for w in block.forth)
    b_qv, b_k, b_o = (worth(*w) for w in block.back)
    gamma, unit, eps, key_eps = got(block.gamma), got(block.unit), float(np.float32(EPS)), float(np.float32(KEY_EPS))
    t = x + r
    n8 = in_8_bits(oracle.rms_norm_fwd(t, gamma, eps))
    qv, raw = n8 @ w_qv.T, (n8 @ w_k.T).reshape(N * Hk, Dk)
    q, v, k = qv[:, :wq].reshape(N, Hk, Dk), qv[:, wq:].reshape(N, H, Dv), oracle.rms_norm_fwd(raw, unit, key_eps).reshape(N, Hk, Dk)
    scale = float(np.float32(block.scale))
    o, s_last = oracle.delta_rule_fwd(q, k, v, g, beta, offsets, scale, block.reverse, s0)
    out = in_8_bits(np.nan_to_num(o).reshape(N, -1)) @ w_o.T
    do = (in_8_bits(dout) @ b_o.T).reshape(N, H, Dv)
    dq, dk, dv, dg, dbeta, ds0 = oracle.delta_rule_bwd(q, k, v, g, beta, offsets, do, scale, block.reverse, s0, ds_last)
    draw, _ = oracle.rms_norm_bwd(raw, unit, dk.reshape(N * Hk, Dk), key_eps)
    dqv = np.concatenate([dq.reshape(N, -1), np.nan_to_num(dv).reshape(N, -1)], 1)
    dn = in_8_bits(dqv) @ b_qv.T + in_8_bits(draw.reshape(N, wq)) @ b_k.T
    dx, dgamma = oracle.rms_norm_bwd(t, gamma, dn, eps)
    return t, out, s_last, dx + dt, dgamma, np.nan_to_num(dg), np.nan_to_num(dbeta), ds0


def make(rng, N, n_seq, block, dtype):
    T = TYPES[dtype]
    rows = {n: rounded(rng.standard_normal((N, block.width)), T) for n in ("x", "r", "dt", "dout")}
    g, beta = -0.3 * rng.random((N, block.H)).astype(np.float32), rng.random((N, block.H)).astype(np.float32)
    s0, ds = (rng.standard_normal((n_seq, block.H, block.Dk, block.Dv)).astype(np.float32) for _ in range(2))
    return {n: t.to(DEV) for n, (t, _) in rows.items()}, {n: a for n, (_, a) in rows.items()}, g, beta, s0, ds


SHAPES = [dict(width=96, heads=2, d_key=32, d_value=32), dict(width=200, heads=4, key_heads=2, d_key=64, d_value=48), dict(width=64, heads=3, key_heads=1, d_key=16, d_value=24)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape", range(3))
@pytest.mark.parametrize("first", [None, [0, 7, 7, 40, 64, 88]], ids=["even", "ragged"])
def test_block_against_the_oracle(first, shape, reverse, dtype):
    say("memory block", first, shape, reverse, dtype)
    rng = np.random.default_rng(shape)
    N, n_seq = 90, 5
    offsets = np.arange(6) * 18 if first is None else np.array(first)
    block = DeltaMixer(dtype=TYPES[dtype], reverse=reverse, seed=5, **SHAPES[shape])
    block.gamma.copy_(f32(1.0 + 0.3 * rng.standard_normal(block.width)))
    rows, rows64, g, beta, s0, ds = make(rng, N, n_seq, block, dtype)
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV)
    s_last, ds0 = torch.zeros(s0.shape, device=DEV), torch.zeros(s0.shape, device=DEV)
    t, out = block.forward(rows["x"], rows["r"], f32(g), f32(beta), n_seq, f, f32(s0), s_last)
    dx, dg, dbeta = block.backward(rows["dt"], rows["dout"], f32(ds), ds0)
    want = the_oracles(block, rows64["x"], rows64["r"], g.astype(np.float64), beta.astype(np.float64), offsets, s0, rows64["dt"], rows64["dout"], ds)
    for name, value, w in zip(("t", "out", "s_last", "dx", "dgamma", "dg", "dbeta", "ds0"), (t, out, s_last, dx, block.dgamma, dg, dbeta, ds0), want): close(name, value, w, dtype)
    if first is not None: assert not out[88:].any() and not dg[88:].any()
    # the way without training: the same results, with the memories in place
    memory = f32(s0)
    t2, out2 = block.forward(rows["x"], rows["r"], f32(g), f32(beta), n_seq, f, memory, memory, training=False)
    close("out", out2, want[1], dtype)
    close("memory", memory, want[2], dtype)
    with pytest.raises(DistGridError):
        block.backward(rows["dt"], rows["dout"])


@pytest.mark.parametrize("shape", range(3))
def test_sample_by_sample_is_the_whole(shape):
    say("memory block advance", shape)
    rng = np.random.default_rng(shape)
    n_seq, S = 6, 12
    block = DeltaMixer(dtype=torch.float16, seed=1, **SHAPES[shape])
    rows, _, g, beta, s0, _ = make(rng, n_seq * S, n_seq, block, "fp16")
    g, beta, memory, last = f32(g), f32(beta), f32(s0), torch.zeros(s0.shape, device=DEV)
    t, out = (z.clone() for z in block.forward(rows["x"], rows["r"], g, beta, n_seq, None, f32(s0), last))
    at = lambda z, i: z.view(n_seq, S, -1)[:, i].contiguous()
    for i in range(S):
        ti, oi = block.advance(at(rows["x"], i), at(rows["r"], i), at(g, i), at(beta, i), memory)
        assert torch.equal(ti, at(t, i))
        close("out", oi, got(at(out, i)), "fp16")
    close("memory", memory, got(last), "fp16")


def test_blocks_in_a_stack_and_a_graph():
    """Two blocks one after the other, forward and backward captured, replayed with other inputs: what they give when called one by one."""
    say("memory blocks in a graph")
    rng = np.random.default_rng(3)
    N, n_seq = 96, 4
    blocks = [DeltaMixer(dtype=torch.bfloat16, seed=i, **SHAPES[0]) for i in range(2)]
    rows, _, g, beta, _, _ = make(rng, N, n_seq, blocks[0], "bf16")
    x, dout, g, beta = rows["x"], rows["dout"], f32(g), f32(beta)

    def step():
        t, out = blocks[0].forward(x, None, g, beta, n_seq)
        t, out = blocks[1].forward(t, out, g, beta, n_seq)
        dx, dg1, _ = blocks[1].backward(dout, dout)
        dx, dg0, _ = blocks[0].backward(dx, dx)
        return [z for z in (t, out, dx, dg0, dg1, blocks[0].dgamma, blocks[1].dgamma)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for i in range(4):
        for z in (x, dout): z.copy_(torch.randn(z.shape, device=DEV))
        want = [z.clone() for z in step()]
        for z in results: z.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, want): assert torch.equal(a, b)


@pytest.mark.parametrize("way", ["forward", "training", "advance"])
def test_own_results_go_in_again_without_a_residual(way):
    """t is x: the pass must not write its other result there."""
    say("memory block again", way)
    rng = np.random.default_rng(7)
    n_seq, S = (5, 1) if way == "advance" else (3, 20)
    block, other = (DeltaMixer(dtype=torch.float16, seed=2, **SHAPES[0]) for _ in range(2))
    rows, _, g, beta, s0, _ = make(rng, n_seq * S, n_seq, block, "fp16")
    g, beta, memories = f32(g), f32(beta), [f32(s0), f32(s0)]

    def go(b, x, memory):
        if way == "advance": return b.advance(x, None, g, beta, memory)
        return b.forward(x, None, g, beta, n_seq, training=way == "training")

    x, y = rows["x"], rows["x"].clone()
    for i in range(4):
        was = x.clone()
        t, x = go(block, x, memories[0])
        assert torch.equal(t, was) and x.data_ptr() != t.data_ptr()
        ty, out = go(other, y, memories[1])                 # the same with a copy
        assert torch.equal(t, ty) and torch.equal(x, out)
        y = out.clone()


@pytest.mark.parametrize("shape,N", [(SHAPES[0], 1536), (dict(width=1024, heads=1, d_key=64, d_value=64), 160)], ids=["rows", "products in parts"])
def test_a_graph_outlives_passes_of_other_sizes(shape, N):
    """What a captured pass works in is not given back when others, or this one, need buffers of other sizes."""
    say("memory block, sizes between replays", N)
    rng = np.random.default_rng(11)
    n_seq = 4
    block, twin = (DeltaMixer(dtype=torch.bfloat16, seed=3, **shape) for _ in range(2))
    rows, _, g, beta, s0, _ = make(rng, N, n_seq, block, "bf16")
    g, beta, s0 = f32(g), f32(beta), f32(s0)

    def step(b):
        t, out = b.forward(rows["x"], rows["r"], g, beta, n_seq, None, s0)
        return [t, out, *b.backward(rows["dt"], rows["dout"]), b.dgamma]

    step(block)                                     # its buffers are there before the graph is
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step(block)
    for n in (800, 12, 2400):
        x = rows["x"][:1].expand(n, -1).contiguous()
        block.forward(x, x, g[:1].expand(n, -1).contiguous(), beta[:1].expand(n, -1).contiguous(), n_seq)
        block.backward(x, x)
        block.advance(rows["x"][:n_seq], rows["r"][:n_seq], g[:n_seq].contiguous(), beta[:n_seq].contiguous(), s0.clone())
    others = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for size in [1 << 10, 1 << 14, 1 << 17, 1 << 19, 1 << 21, 1 << 23] for _ in range(40)]
    for _ in range(3):
        for z in (rows["x"], rows["dout"]): z.copy_(torch.randn(z.shape, device=DEV))
        for z in results: z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, step(twin)): assert torch.equal(a, b)
        for z in others: assert bool((z == 7).all())


def test_more_samples_than_a_product_takes():
    """Segments do not know of each other: those around row 2^24, where products are cut, and the last ones give what they give alone."""
    say("memory block of 2^24 samples and more")
    S, n_seq, some = 37, 453600, 300
    N = S * n_seq
    assert N > (1 << 24) + 1000
    block, alone = (DeltaMixer(16, 1, d_key=8, d_value=8, seed=4) for _ in range(2))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x, dout = (torch.randn(N, 16, device=DEV, generator=gen).half() for _ in range(2))
    g, beta = -torch.rand(N, 1, device=DEV, generator=gen), torch.rand(N, 1, device=DEV, generator=gen)
    t, out = block.forward(x, None, g, beta, n_seq)
    dx, dg, dbeta = block.backward(None, dout)
    for seq in ((1 << 24) // S - some // 2, n_seq - some):
        rows = slice(seq * S, (seq + some) * S)
        _, out1 = alone.forward(x[rows].contiguous(), None, g[rows].contiguous(), beta[rows].contiguous(), some)
        for name, a, b in zip(("out", "dx", "dg", "dbeta"), (out1, *alone.backward(None, dout[rows].contiguous())), (out, dx, dg, dbeta)): close(name, a, got(b[rows]), "fp16")


def test_block_between_the_encode_and_the_networks():
    """Features of a hash grid, the samples of a segment one after the other, through the block to the field networks and back to the table: every hand-over against the oracle on
    what the stage before it gave.  A stage of the field rounds to fp16 some eight times, 2^-11 of values up to twice its result's: 0.01 of it."""
    say("memory block in the field")
    rng = np.random.default_rng(6)
    n_seg, S, field = 41, 32, 0.01
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
    block = DeltaMixer(32, 2, d_key=16, d_value=16, dtype=torch.float16, seed=3)
    block.gamma.copy_(f32(1.0 + 0.3 * rng.standard_normal(32)))
    length = rng.exponential(size=(N, 1))                           # of steps: what is stored fades with the way
    g, beta = (-0.2 * np.repeat(length, 2, 1)).astype(np.float32), rng.random((N, 2)).astype(np.float32)
    t, out = block.forward(feat, None, f32(g), f32(beta), n_seg)
    y = torch.empty_like(out)
    B.dg_dropout_fwd(out, t, 0.0, 0, 0, y)                          # the residual's addition
    zeros = lambda *shape: np.zeros(shape)
    x64, offsets = got(feat), np.arange(n_seg + 1) * S
    want = lambda dt, dout: the_oracles(block, x64, zeros(N, 32), g.astype(np.float64), beta.astype(np.float64), offsets, None, dt, dout, None)
    close("y", y, x64 + want(zeros(N, 32), zeros(N, 32))[1], "fp16")
    mlp, ref_mlp = B.dg_mlp_desc(32, 64, 16, 16, 64, 2, 1), oracle.mlp_desc(32, 64, 16, 16, 64, 2, 1)
    weights, dirs = (rng.standard_normal(9408) * 0.2).astype(np.float16), rng.standard_normal((n_seg, 16)).astype(np.float16)
    dsigma, drgb = rng.standard_normal(N).astype(np.float32) * 0.01, rng.standard_normal((N, 3)).astype(np.float32) * 0.01
    sigma, rgb, dfeat = torch.zeros(N, device=DEV), torch.zeros(N, 3, device=DEV), torch.zeros(N, 32, device=DEV)
    dW, largest = torch.zeros(9408, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.dg_mlp_fwd_rows(mlp, dev(weights), y, dev(dirs), None, S, N, sigma, rgb)
    B.dg_mlp_bwd_rows(mlp, dev(weights), y, dev(dirs), None, S, N, dev(dsigma), dev(drgb), 256.0, 16, dfeat, largest, dW,
                      torch.zeros(B.dg_mlp_bwd_app_workspace_bytes(mlp, N, S) // 4 + 64, device=DEV))
    y64, scale = got(y), 64.0
    w_sigma, w_rgb = oracle.mlp_fwd(ref_mlp, weights, y64, dirs, S)
    assert rel_err(host(sigma), w_sigma) <= field and rel_err(host(rgb), w_rgb) <= field
    assert rel_err(host(dfeat), oracle.mlp_bwd(ref_mlp, weights, y64, dirs, S, dsigma, drgb, 256.0)[0]) <= field
    dy = (dfeat * scale).half()                                     # the networks give their gradient in fp32
    dx, dg, dbeta = block.backward(dy, dy)
    _, _, _, w_dx, w_dgamma, w_dg, w_dbeta, _ = want(got(dy), got(dy))
    for name, value, w in zip(("dx", "dgamma", "dg", "dbeta"), (dx, block.dgamma, dg, dbeta), (w_dx, w_dgamma, w_dg, w_dbeta)): close(name, value, w, "fp16")
    dtable, ws = torch.zeros(ref_grid.n_entries, 2, device=DEV), torch.zeros(B.dg_hashgrid_encode_bwd_workspace_bytes(grid, N) // 4 + 64, device=DEV)
    B.dg_hashgrid_encode_bwd(grid, dev(u), (dx.float() / scale).view(N, 16, 2).transpose(0, 1).contiguous(), N, dtable, ws)     # and it is read in planes
    assert rel_err(host(dtable), oracle.encode_bwd(ref_grid, u, got(dx) / scale)) <= field


def test_refusals():
    with pytest.raises(DistGridError):
        DeltaMixer(32, 2, weights=[torch.zeros(4, 4)] * 3, device=DEV)
    block = DeltaMixer(32, 2, d_key=16, d_value=16)
    x, g, s0 = torch.zeros(4, 32, dtype=torch.float16, device=DEV), torch.zeros(4, 2, device=DEV), torch.zeros(1, 2, 16, 16, device=DEV)
    with pytest.raises(DistGridError):
        block.backward(x, x)
    with pytest.raises(DistGridError):
        block.forward(x, None, g, g, 1, None, s0, s0)
    with pytest.raises(DistGridError):
        block.forward(x, None, g, g, 3)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_example_runs(dtype):
    say("memory example", dtype)
    errors = train_example(rays=40, samples=16, iterations=3, dtype=dtype, report=None)
    assert np.isfinite(errors).all()
