"""A sequence block on the features of the samples of rays: call sequencing only.

Sec. 4.3 composites the samples of a ray by one recurrence, with the transmittance as its gate, and merges segments by carrying
the state across.  `RayMixer` sends rows of features through such a recurrence, with a gate for each channel that is learned, as the
residual block of a sequence model:

    y = x + dropout(recurrence(gates = norm(x; gamma_z, beta_z), inputs = norm(x; gamma_u, beta_u)))

Rows are samples, segment after segment: all of one length, or with the offsets `first` that dg_march_segments writes.  A segment
can start from the state in which another one ended, as partitions do along a ray.  Every arithmetic step happens inside
libdistgrid; this file allocates, slices and calls.

A program of its own puts the block between the encode and the networks; TrainStep has no place for it.  fp16 rows of 32 features as
dg_hashgrid_encode_fwd_ordered writes them, in the samples' own order, go in as they are, and the result goes to dg_mlp_fwd_rows as it
is.  On the way back the caller converts twice: dg_mlp_bwd_rows with n_merged = 16 gives rows in fp32 (scaled, they fit fp16), and
dg_hashgrid_encode_bwd reads planes in fp32.

    python -m paper_2405_04416_amd.mixer        trains a block to clean noisy features along rays
"""
import torch

from . import binding as B

EPS = 1e-5


def _overlap(a, b):
    """Whether two contiguous tensors share memory."""
    begin, end = (lambda t: t.data_ptr()), (lambda t: t.data_ptr() + t.numel() * t.element_size())
    return begin(a) < end(b) and begin(b) < end(a)


class RayMixer:
    def __init__(self, width, dtype=torch.float16, p=0.1, reverse=False, seed=0, device="cuda:0"):
        """width: features per sample; p: share that dropout takes during training; reverse: back to front; seed: of dropout, not
        one that samplers draw from."""
        self.width, self.dtype, self.p, self.reverse, self.seed, self.dev = width, dtype, p, reverse, seed, torch.device(device)
        f32 = dict(dtype=torch.float32, device=self.dev)
        # gamma_z, beta_z, gamma_u, beta_u one after the other, so that one launch of the optimiser serves them
        self.params, self.grads = torch.zeros(4 * width, **f32), torch.zeros(4 * width, **f32)
        self.gamma_z, self.beta_z, self.gamma_u, self.beta_u = self.params.view(4, width)
        self.gamma_z.fill_(1.0), self.gamma_u.fill_(1.0), self.beta_z.fill_(1.0)       # gates that keep three quarters
        self.opt = None
        self.drawn = 0              # words of the generator that earlier passes have used
        self.saved = None
        self.buffers = {}

    def _buffer(self, name, shape, dtype):
        """A buffer that this block keeps from pass to pass, replaced when a pass needs another size."""
        t = self.buffers.get(name)
        if t is None or t.shape != shape or t.dtype != dtype:
            t = self.buffers[name] = torch.empty(shape, dtype=dtype, device=self.dev)
        return t

    def _rows(self, name, x):
        return self._buffer(name, x.shape, self.dtype)

    def _part_with(self, x):
        """A result of this block that goes in again is needed until its gradient has been taken: other buffers take its place."""
        for name in ("y", "dx"):
            t = self.buffers.get(name)
            if t is not None and t.untyped_storage().data_ptr() == x.untyped_storage().data_ptr():
                del self.buffers[name]

    def _workspace(self, name, n_bytes):
        return self._buffer(name, torch.Size([n_bytes]), torch.uint8) if n_bytes else None

    def _recur(self, x, n_seq, first, h0, h_last, states):
        self.saved = None           # what a backward pass would need is overwritten
        z, u, m = self._rows("z", x), self._rows("u", x), self._rows("m", x)
        B.dg_layer_norm_fwd(x, self.gamma_z, self.beta_z, EPS, z)
        B.dg_layer_norm_fwd(x, self.gamma_u, self.beta_u, EPS, u)
        N, W = x.shape
        B.dg_recurrence_fwd(z, u, n_seq, first, self.reverse, h0, m, h_last, states, self._workspace("ws_scan", B.dg_recurrence_workspace_bytes(N, n_seq, W)))
        return m

    def forward(self, x, n_seq, first=None, h0=None, h_last=None, training=True):
        """x [N, width] -> y.  n_seq segments of N / n_seq samples each, or of the rows that `first` gives them.  h0, h_last
        [n_seq, width] fp32 or None: states in and out (h_last is written, it may be h0 outside training).  The result is a buffer that the next
        pass overwrites, unless that is a training pass on it.  backward reads x, first and h0 again: they have to stay as they are until then."""
        N, W = x.shape
        if training:
            if h0 is not None and h_last is not None and _overlap(h0, h_last):
                raise B.DistGridError("the gradient needs h0: h_last must not lie in its memory")
            self._part_with(x)
        states = self._buffer("states", torch.Size([B.dg_recurrence_state_count(N, W)]), torch.float32) if training else None
        m, y = self._recur(x, n_seq, first, h0, h_last, states), self._rows("y", x)
        p = self.p if training else 0.0
        B.dg_dropout_fwd(m, x, p, self.seed, self.drawn, y)
        if training:
            self.saved = (x, n_seq, first, h0, states, p, self.drawn)
            self.drawn += -(-x.numel() // 4)
        return y

    def backward(self, dy, dh_last=None, dh0=None):
        """Gradient of the last training pass: returns dx, overwrites `grads`.  dh_last, dh0 [n_seq, width] fp32 or None."""
        if self.saved is None:
            raise B.DistGridError("the last pass was not a training pass")
        x, n_seq, first, h0, states, p, drawn = self.saved
        N, W = x.shape
        dm, dz, du, dx, part = (self._rows(n, x) for n in ("dm", "dz", "du", "dx", "part"))
        B.dg_dropout_bwd(dy, p, self.seed, drawn, dm)
        B.dg_recurrence_bwd(self.buffers["z"], self.buffers["u"], n_seq, first, self.reverse, h0, states, dm, dh_last, dz, du, dh0,
                            self._workspace("ws_scan", B.dg_recurrence_workspace_bytes(N, n_seq, W)))
        ws = self._workspace("ws_norm", B.dg_layer_norm_bwd_workspace_bytes(N, W))
        g = self.grads.view(4, W)
        B.dg_layer_norm_bwd(x, self.gamma_z, dz, EPS, part, g[0], g[1], ws)
        # Without dropping: dx = dy + part.  In 16 bits dx is rounded at both sums, each once to half a unit: less than dz and du are already off by.
        B.dg_dropout_fwd(part, dy, 0.0, 0, 0, dx)
        B.dg_layer_norm_bwd(x, self.gamma_u, du, EPS, part, g[2], g[3], ws)
        B.dg_dropout_fwd(part, dx, 0.0, 0, 0, dx)
        return dx

    def advance(self, x, h):
        """One more sample for every segment, x [n_seq, width]; the states h [n_seq, width] fp32 are updated in place."""
        m, y = self._recur(x, x.shape[0], None, h, h, None), self._rows("y", x)
        B.dg_dropout_fwd(m, x, 0.0, 0, 0, y)
        return y

    def optimiser_step(self, iteration, lr):
        """Adam on the four vectors; consumes the gradients.  iteration counts from 0."""
        if self.opt is None:
            self.opt = torch.zeros_like(self.params), torch.zeros_like(self.params)
        B.dg_adam_step(self.params, self.grads, *self.opt, lr, iteration + 1)


def train_example(rays=4096, samples=48, width=32, iterations=200, dtype=torch.float16, seed=0, report=print):
    """Features that change slowly along a ray, seen through noise one and a half times as large: what the block adds to a sample is to be
    its clean features.  It learns for how long each channel has to remember.  Returns the mean squared errors of what it adds in the
    first and in the last iteration."""
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    block = RayMixer(width, dtype, p=0.05, seed=seed + 1, device=dev)
    errors = []
    for i in range(iterations):
        start, slope = (torch.randn(rays, 1, width, device=dev, generator=gen) for _ in range(2))
        t = torch.linspace(0.0, 1.0, samples, device=dev)[None, :, None]
        clean = (start + 0.3 * slope * t).reshape(rays * samples, width)
        noisy = (clean + 1.5 * torch.randn(clean.shape, device=dev, generator=gen)).to(dtype)
        off = block.forward(noisy, rays).float() - noisy.float() - clean
        errors.append(off.square().mean())
        block.backward(off.to(dtype))               # gradient of half the sum of squares; Adam does not mind its scale
        block.optimiser_step(i, B.dg_cosine_lr(0.02, 0.002, i, iterations))
        if report and (i % 50 == 0 or i == iterations - 1):
            report("iteration %4d  mean squared error %.4f" % (i, float(errors[-1])))
    return float(errors[0]), float(errors[-1])


if __name__ == "__main__":
    train_example()
