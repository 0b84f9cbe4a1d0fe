"""A block with an associative memory on the features of the samples of rays: call sequencing only.

Where RayMixer keeps one number for each channel along a ray, a head of this block keeps a matrix: a sample stores a value under a key, in place of what the
key had, and reads with a query.  As the block of a residual stack whose additions are left to the norms that follow:

    t = x + r;   n = rms_norm(t; gamma);   q, v = n W_qv^T;   k = n W_k^T, each head's to length one;
    o = gated delta rule(q, k, v; decays, rates);   r' = o W_o^T                 the next block gets (t, r')

The projections are given, and stay: they are kept in 8 bits, as are the rows that go through them, and so are the gradients on their way back through them.  What is
learned are gamma and what makes the gates: logarithms of decays g <= 0 and rates beta in [0, 1], [samples, heads] each, which the caller computes, for instance from the
distances of samples, and of which it gets the gradients.

Rows are samples, segment after segment: all of one length, or with the offsets `first` that dg_march_segments writes.  A segment can start from the memory in
which another one ended, as partitions do along a ray.  Every arithmetic step happens inside libdistgrid; this file allocates, slices and calls.
As RayMixer, the block stands between the encode and the networks in a program of its own: fp16 rows of features go in as they are, and t + out goes to the networks.

    python -m paper_2405_04416_amd.memory       trains a block to give back, at the end of each ray, what its samples stored
"""
import torch

from . import binding as B
from .mixer import _overlap, keep_captured

EPS = 1e-5
KEY_EPS = 1e-6
MOST_ROWS = 1 << 24     # of a product


def rows_in_8_bits(x):
    """x [N, W] -> (values, scales), as dg_e4m3_rows writes them."""
    N, W = x.shape
    q, s = room_in_8_bits(N, W, x.device)
    B.dg_e4m3_rows(x, q, s)
    return q, s


def room_in_8_bits(N, W, device):
    """Rows begin at multiples of 16 bytes."""
    q = torch.empty(N, -(-W // 16) * 16, dtype=torch.float8_e4m3fn, device=device)[:, :W]
    return q, torch.empty(N, -(-W // 128), dtype=torch.float8_e8m0fnu, device=device)


class DeltaMixer:
    def __init__(self, width, heads, key_heads=None, d_key=64, d_value=64, dtype=torch.float16, reverse=False, weights=None, seed=0, device="cuda:0"):
        """width: features per sample; heads: memories of d_key x d_value, `key_heads` of which (all, if None) have keys and queries of their own; dtype: fp16 or bf16;
        reverse: back to front; weights: None (drawn from `seed`), or (W_qv [key_heads d_key + heads d_value, width], W_k [key_heads d_key, width], W_o [width, heads d_value])."""
        self.width, self.H, self.Hk, self.Dk, self.Dv = width, heads, key_heads or heads, d_key, d_value
        self.dtype, self.reverse, self.dev = dtype, reverse, torch.device(device)
        self.wq, self.wv = self.Hk * d_key, heads * d_value
        if weights is None:
            gen = torch.Generator(device=self.dev)
            gen.manual_seed(seed)
            draw = lambda n, m: torch.randn(n, m, generator=gen, device=self.dev) * m ** -0.5
            weights = draw(self.wq + self.wv, width), draw(self.wq, width), draw(width, self.wv)
        weights = [w.to(self.dev) for w in weights]
        for w, shape in zip(weights, ((self.wq + self.wv, width), (self.wq, width), (width, self.wv))):
            if tuple(w.shape) != shape:
                raise B.DistGridError("expected weights %s, got %s" % (shape, tuple(w.shape)))
        self.forth = [rows_in_8_bits(w.contiguous()) for w in weights]              # qv, k, o
        self.back = [rows_in_8_bits(w.t().contiguous()) for w in weights]           # for gradients
        self.gamma, self.dgamma = torch.ones(width, dtype=torch.float32, device=self.dev), torch.zeros(width, dtype=torch.float32, device=self.dev)
        self.unit = torch.full((d_key,), d_key ** -0.5, dtype=torch.float32, device=self.dev)
        self.scale = d_key ** -0.5
        self.opt = None
        self.saved = None
        self.buffers, self.captured = {}, []

    def _buffer(self, name, shape, dtype=None):
        """A buffer that this block keeps from pass to pass, replaced when a pass needs another size."""
        t, shape, dtype = self.buffers.get(name), torch.Size(shape), dtype or self.dtype
        if t is None or t.shape != shape or t.dtype != dtype:
            keep_captured(self.captured, [t])           # products of other sizes have other workspaces within a pass
            t = self.buffers[name] = torch.empty(shape, dtype=dtype, device=self.dev)
        return t

    def _workspace(self, name, n_bytes):
        return self._buffer(name, [n_bytes], torch.uint8) if n_bytes else None

    def _room8(self, name, N, W):
        t = self.buffers.get(name)
        if t is None or t[0].shape != (N, W):
            keep_captured(self.captured, [t])
            t = self.buffers[name] = room_in_8_bits(N, W, self.dev)
        return t

    def _part_with(self, *inputs):
        """A result of this block that goes in again is needed until its gradient has been taken, and is a result again where there is no residual: other buffers take its place."""
        for name in ("t", "out", "dx"):
            t = self.buffers.get(name)
            if t is not None and any(x is not None and x.untyped_storage().data_ptr() == t.untyped_storage().data_ptr() for x in inputs):
                del self.buffers[name]

    def _product(self, a, b, y):
        M, N, K = a[0].shape[0], b[0].shape[0], a[0].shape[1]
        for i in range(MOST_ROWS, M, MOST_ROWS):            # more rows than a product takes, some after the others
            self._product([z[i:i + MOST_ROWS] for z in a], b, y[i:i + MOST_ROWS])
        if M > MOST_ROWS: M, a, y = MOST_ROWS, [z[:MOST_ROWS] for z in a], y[:MOST_ROWS]
        B.dg_e4m3_product(*a, *b, y, self._workspace("ws_product", B.dg_e4m3_product_workspace_bytes(M, N, K)))

    def _rows8(self, name, x):
        q = self._room8(name, *x.shape)
        B.dg_e4m3_rows(x, *q)
        return q

    def _mix(self, x, r, g, beta, n_seq, first, s0, s_last, saved):
        self.saved = None               # what a backward pass would need is overwritten
        if r is None:
            self._part_with(x)          # x is the first result
        N = x.shape[0]
        t, n8 = (x if r is None else self._buffer("t", x.shape)), self._room8("n8", N, self.width)
        B.dg_rms_norm_e4m3_fwd(x, r, self.gamma, EPS, None if r is None else t, *n8)
        qv, raw, k = self._buffer("qv", [N, self.wq + self.wv]), self._buffer("raw", [N * self.Hk, self.Dk]), self._buffer("k", [N, self.wq])
        self._product(n8, self.forth[0], qv)
        self._product(n8, self.forth[1], raw.view(N, self.wq))
        B.dg_rms_norm_fwd(raw, None, self.unit, KEY_EPS, None, k.view(N * self.Hk, self.Dk))
        o, out = self._buffer("o", [N, self.wv]), self._buffer("out", [N, self.width])
        if first is not None: o.zero_()         # rows of no segment are left as they are, and read by the projection
        B.dg_delta_rule_fwd(qv[:, :self.wq], k, qv[:, self.wq:], g, beta, self.Hk, n_seq, first, self.reverse, self.scale, s0, o, s_last, saved,
                            self._workspace("ws_delta", B.dg_delta_rule_fwd_least_workspace_bytes(N, n_seq, self.H, self.Dk, self.Dv, saved is not None)))
        self._product(self._rows8("o8", o), self.forth[2], out)
        keep_captured(self.captured, self.buffers.values())
        return t, out

    def forward(self, x, r, g, beta, n_seq, first=None, s0=None, s_last=None, training=True):
        """x, r [N, width] (r may be None) -> (t, out) for the next block.  g, beta [N, heads] fp32; n_seq segments of N / n_seq samples each, or of the rows that `first`
        gives them (of rows of none `out` is 0).  s0, s_last [n_seq, heads, d_key, d_value] fp32 or None: memories in and out (s_last may be s0 outside training).
        The results are buffers that the next pass overwrites, unless that is a training pass on them, or one without r (where t is x).  backward reads x, g, beta and first again: they
        have to stay as they are until then."""
        N = x.shape[0]
        saved = None
        if training:
            if s0 is not None and s_last is not None and _overlap(s0, s_last):
                raise B.DistGridError("s_last must not lie in the memory of s0, of which ds0 is the gradient")
            self._part_with(x, r)
            saved = self._workspace("saved", max(B.dg_delta_rule_saved_bytes(N, n_seq, self.H, self.Dk, self.Dv), 16))
        t, out = self._mix(x, r, g, beta, n_seq, first, s0, s_last, saved)
        if training:
            self.saved = (t, g, beta, n_seq, first, saved)
        return t, out

    def backward(self, dt, dout, ds_last=None, ds0=None):
        """Gradient of the last training pass, from those of its results (dt may be None): returns (dx, dg, dbeta), dx that of x and of r alike, and overwrites `dgamma`.
        ds_last, ds0 [n_seq, heads, d_key, d_value] fp32 or None."""
        if self.saved is None:
            raise B.DistGridError("the last pass was not a training pass")
        t, g, beta, n_seq, first, saved = self.saved
        N, buf = t.shape[0], self.buffers
        do, dqv, dk, draw = self._buffer("do", [N, self.wv]), self._buffer("dqv", [N, self.wq + self.wv]), self._buffer("dk", [N, self.wq]), self._buffer("draw", [N * self.Hk, self.Dk])
        dg, dbeta = self._buffer("dg", g.shape, torch.float32), self._buffer("dbeta", g.shape, torch.float32)
        if first is not None:           # rows of no segment are left as they are, and read by what follows
            for z in (dqv, dk, dg, dbeta): z.zero_()
        self._product(self._rows8("dout8", dout), self.back[2], do)
        B.dg_delta_rule_bwd(buf["qv"][:, :self.wq], buf["k"], buf["qv"][:, self.wq:], g, beta, self.Hk, n_seq, first, self.reverse, self.scale, saved, do, ds_last,
                            dqv[:, :self.wq], dk, dqv[:, self.wq:], dg, dbeta, ds0,
                            self._workspace("ws_back", B.dg_delta_rule_workspace_bytes(N, n_seq, self.Hk, self.H, self.Dk, self.Dv)))
        B.dg_rms_norm_bwd(buf["raw"], self.unit, dk.view(N * self.Hk, self.Dk), None, KEY_EPS, draw, None)
        part, dn, dx = (self._buffer(n, [N, self.width]) for n in ("part", "dn", "dx"))
        self._product(self._rows8("dqv8", dqv), self.back[0], part)
        self._product(self._rows8("dk8", draw.view(N, self.wq)), self.back[1], dn)
        B.dg_dropout_fwd(part, dn, 0.0, 0, 0, dn)           # without dropping: the sum
        B.dg_rms_norm_bwd(t, self.gamma, dn, dt, EPS, dx, self.dgamma, self._workspace("ws_norm", B.dg_rms_norm_bwd_workspace_bytes(N, self.width)))
        keep_captured(self.captured, self.buffers.values())
        return dx, dg, dbeta

    def advance(self, x, r, g, beta, memory):
        """One more sample for every segment, x, r [n_seq, width]; the memories [n_seq, heads, d_key, d_value] fp32 are updated in place."""
        return self._mix(x, r, g, beta, x.shape[0], None, memory, memory, None)

    def optimiser_step(self, iteration, lr):
        """Adam on gamma; consumes the gradient.  iteration counts from 0."""
        if self.opt is None:
            self.opt = torch.zeros_like(self.gamma), torch.zeros_like(self.gamma)
        B.dg_adam_step(self.gamma, self.dgamma, *self.opt, lr, iteration + 1)


def train_example(rays=256, samples=32, width=64, heads=2, iterations=100, dtype=torch.float16, seed=0, report=print):
    """Each sample of the first half of a ray stores its features; the second half shows the same samples again through noise, and the block is to give back what they were.  It learns
    the gains of the features, and for each head how fast it forgets and how much it writes.  Returns the mean squared errors of the first and the last iteration."""
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    block = DeltaMixer(width, heads, d_key=32, d_value=32, dtype=dtype, seed=seed + 1, device=dev)
    gates = torch.zeros(2, heads, device=dev)               # logits of decays and rates
    grads, opt = torch.zeros_like(gates), (torch.zeros_like(gates), torch.zeros_like(gates))
    errors, N, half = [], rays * samples, samples // 2
    for i in range(iterations):
        clean = torch.randn(rays, half, width, device=dev, generator=gen)
        noisy = clean + 0.5 * torch.randn(clean.shape, device=dev, generator=gen)
        x = torch.cat([clean, noisy], 1).reshape(N, width).to(dtype)
        keep, rate = torch.sigmoid(gates[0] + 3.0), torch.sigmoid(gates[1])
        g, beta = keep.log().expand(N, heads).contiguous(), rate.expand(N, heads).contiguous()
        _, out = block.forward(x, None, g, beta, rays)
        off = (out.float().view(rays, samples, width) - torch.cat([torch.zeros_like(clean), clean - noisy], 1))
        off[:, :half] = 0.0                                 # what the first half adds is of no interest
        errors.append(off.square().mean())
        _, dg, dbeta = block.backward(None, off.reshape(N, width).to(dtype))
        grads[0], grads[1] = dg.sum(0) * (1.0 - keep), dbeta.sum(0) * rate * (1.0 - rate)
        lr = B.dg_cosine_lr(0.02, 0.002, i, iterations)
        block.optimiser_step(i, lr)
        B.dg_adam_step(gates.view(-1), grads.view(-1), *(o.view(-1) for o in opt), lr, i + 1)
        if report and (i % 25 == 0 or i == iterations - 1):
            report("iteration %4d  mean squared error %.4f" % (i, float(errors[-1])))
    return float(errors[0]), float(errors[-1])


if __name__ == "__main__":
    train_example()
