"""Cases that time the operators of a sequence block along the samples of a ray: layer norm, a gated linear recurrence and
dropout.

A case is one pass of a user's program through one operator on one GPU: the call alone ("fwd": rendering, serving), or the
call and its gradient ("train").  `own` False computes the same in elementary torch operations in 32 bits, rounded once at
the end; True calls the package's entry points.  Inputs are synthetic and made on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
EPS = 1e-5
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
LARGEST = 1 << 28       # elements of one input


def _norm(name, way, dtype, rows, width):
    c = dict(op="norm", way=way, dtype=dtype, rows=rows, width=width)
    return dict(c, name=name) if name else c


def _recurrence(name, way, dtype, seqs, tokens, width, ragged=False, joint=False, carry=False, reverse=False):
    """tokens: of each sequence, or of the longest one (ragged).  joint: gates and inputs are halves of one projection's rows.
    carry: the state comes from outside and goes on (a segment's end is the next one's start).  reverse: back to front."""
    c = dict(op="recurrence", way=way, dtype=dtype, seqs=seqs, tokens=tokens, width=width, ragged=ragged, joint=joint, carry=carry, reverse=reverse)
    return dict(c, name=name) if name else c


def _dropout(name, way, dtype, rows, width, residual, p):
    c = dict(op="dropout", way=way, dtype=dtype, rows=rows, width=width, residual=residual, p=p)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the samples of a small batch of segments, 4 levels of 2 features: launch latency
        _norm("norm_small", "fwd", "fp16", 1024, 8),
        # the features (16 levels of 2) of all samples of a training batch
        _norm("norm_features", "train", "fp16", (1 << 17) * 64, 32),
        # odd sizes: an odd number of samples a ray, a width that no vector load divides
        _norm("norm_odd", "train", "fp32", 5003 * 37, 37),
        # tokens of a wide sequence model
        _norm("norm_wide", "train", "bf16", 8192, 4096),
        # one more token for every sequence that is being served: the state goes in and out
        _recurrence("recurrence_token", "fwd", "bf16", 256, 1, 1024, joint=True, carry=True),
        # the feature channels along the samples of every ray of a training batch
        _recurrence("recurrence_rays", "train", "fp16", 1 << 17, 64, 32),
        # segments of very different lengths, as the occupancy-guided sampler makes them, some without a sample; back to front
        _recurrence("recurrence_ragged", "train", "fp32", 20011, 96, 64, ragged=True, reverse=True),
        # one long sequence read in: few channels, all the work lies along it
        _recurrence("recurrence_long", "fwd", "bf16", 1, 1 << 17, 256, joint=True, carry=True),
        # a training batch of long sequences of a wide model
        _recurrence("recurrence_batch", "train", "bf16", 4, 16384, 1024, joint=True),
        # a small batch of segments' features with the residual: latency again
        _dropout("dropout_small", "fwd", "fp16", 1024, 32, True, 0.1),
        # all features of a training batch, the residual added
        _dropout("dropout_features", "train", "fp16", (1 << 17) * 64, 32, True, 0.1),
        # odd sizes, no residual
        _dropout("dropout_odd", "train", "fp32", 5003 * 37, 37, False, 0.25),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths that models have, and any width."""
    usual = [w for w in (8, 16, 32, 48, 64, 96, 128, 256, 384, 512, 768, 1024, 1536, 2048, 4096, 8192) if lo <= w <= hi]
    return rng.choice(usual) if rng.random() < 0.6 else _log_uniform(rng, lo, hi)


def draw(rng):
    op = rng.choice(["norm", "recurrence", "recurrence", "dropout"])
    way, dtype = rng.choice(["fwd", "train"]), rng.choice(["fp32", "fp16", "bf16"])
    most = LARGEST >> 1
    if op == "norm":
        width = _width(rng, 8, 8192)
        return _norm(None, way, dtype, _log_uniform(rng, 64, min(most // width, 1 << 23)), width)
    if op == "dropout":
        width = _width(rng, 8, 4096)
        return _dropout(None, way, dtype, _log_uniform(rng, 64, min(most // width, 1 << 23)), width, rng.random() < 0.6, rng.choice([0.05, 0.1, 0.2, 0.5]))
    width = _width(rng, 8, 2048)
    tokens = 1 if rng.random() < 0.15 else _log_uniform(rng, 2, 1 << 17)
    tokens = min(tokens, most // width)
    seqs = _log_uniform(rng, 1, min(max(1, most // (2 * width * tokens)), 1 << 17))
    return _recurrence(None, way, dtype, seqs, tokens, width, ragged=tokens > 1 and rng.random() < 0.35, joint=rng.random() < 0.4,
                       carry=tokens == 1 or rng.random() < 0.5, reverse=rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the sequences before they are shuffled: all the same, or 0, 1, 2, ... up to the longest and again."""
    if not case["ragged"]:
        return [case["tokens"]] * case["seqs"]
    m = case["tokens"] + 1
    return [case["tokens"]] + [j % m for j in range(case["seqs"] - 1)]


def prepare(case, seed):
    dtype = TYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=gen, dtype=torch.float32)      # noqa: E731
    empty = lambda *shape, dt=dtype: torch.empty(*shape, device=DEV, dtype=dt)                       # noqa: E731
    s = dict(case=case, train=case["way"] == "train")
    width = case["width"]
    if case["op"] == "norm":
        rows = case["rows"]
        s.update(x=(normal(rows, width) * 1.5 + 0.5).to(dtype), gamma=1.0 + 0.2 * normal(width), beta=0.2 * normal(width), y=empty(rows, width))
        if s["train"]:
            s.update(dy=normal(rows, width).to(dtype), dx=empty(rows, width), dgamma=empty(width, dt=torch.float32), dbeta=empty(width, dt=torch.float32))
    elif case["op"] == "dropout":
        rows = case["rows"]
        s.update(x=normal(rows, width).to(dtype), seed=seed * 1000003 + 17, offset=seed % 7, y=empty(rows, width))
        if case["residual"]:
            s.update(residual=normal(rows, width).to(dtype))
        if s["train"]:
            s.update(dy=normal(rows, width).to(dtype), dx=empty(rows, width))
    else:
        seqs = case["seqs"]
        lengths = torch.tensor(_lengths(case), device=DEV)
        if case["ragged"]:
            lengths = lengths[torch.randperm(seqs, device=DEV, generator=gen)]
        ends = torch.cumsum(lengths, 0)
        N = sum(_lengths(case))
        s.update(N=N, first=torch.cat([ends.new_zeros(1), ends]).to(torch.int32))
        # gates around one that keeps three quarters of the state, now and then one that lets all or nothing through
        z, u = (normal(N, width) * 2 + 1).to(dtype), normal(N, width).to(dtype)
        s["zu"] = torch.cat([z, u], 1) if case["joint"] else (z, u)
        s["y"] = empty(N, width)
        if case["carry"]:
            s.update(h0=normal(seqs, width), h_last=empty(seqs, width, dt=torch.float32))
        if s["train"]:
            s["dy"] = normal(N, width).to(dtype)
            s["dzu"] = empty(N, 2 * width) if case["joint"] else (empty(N, width), empty(N, width))
            if case["carry"]:
                s.update(dh_last=normal(seqs, width), dh0=empty(seqs, width, dt=torch.float32))
    return s


def _halves(case, both):
    return (both[:, :case["width"]], both[:, case["width"]:]) if case["joint"] else both


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"norm": _run_norm, "recurrence": _run_recurrence, "dropout": _run_dropout}[state["case"]["op"]](state)


def _run_norm(s):
    if own:
        from paper_2405_04416_amd import binding as B
        B.dg_layer_norm_fwd(s["x"], s["gamma"], s["beta"], EPS, s["y"])
        if not s["train"]:
            return {"y": s["y"]}
        if "ws" not in s:
            s["ws"] = torch.empty(B.dg_layer_norm_bwd_workspace_bytes(*s["x"].shape), dtype=torch.uint8, device=DEV)
        B.dg_layer_norm_bwd(s["x"], s["gamma"], s["dy"], EPS, s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return {k: s[k] for k in ("y", "dx", "dgamma", "dbeta")}
    x = s["x"].float()
    centred = x - x.mean(1, keepdim=True)
    scale = 1.0 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xh = centred * scale
    out = {"y": (xh * s["gamma"] + s["beta"]).to(s["x"].dtype)}
    if s["train"]:
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = scale * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        out.update(dx=dx.to(s["x"].dtype), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    return out


def _mask64(seed, offset, n):
    """16 random bits for each of n elements: word offset + i / 4 of the counter-based generator, field i % 4."""
    words = -(-n // 4)
    golden, m1, m2 = (v - (1 << 64) for v in (0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB))
    right = lambda v, k: (v >> k) & ((1 << (64 - k)) - 1)        # noqa: E731   logical shift of signed words
    z = (torch.arange(words, device=DEV, dtype=torch.int64) + (offset + 1)) * golden + seed
    z = (z ^ right(z, 30)) * m1
    z = (z ^ right(z, 27)) * m2
    z = z ^ right(z, 31)
    fields = (z[:, None] >> torch.tensor([0, 16, 32, 48], device=DEV)) & 0xffff
    return fields.reshape(-1)[:n]


def _run_dropout(s):
    p = s["case"]["p"]
    if own:
        from paper_2405_04416_amd import binding as B
        B.dg_dropout_fwd(s["x"], s.get("residual"), p, s["seed"], s["offset"], s["y"])
        if not s["train"]:
            return {"y": s["y"]}
        B.dg_dropout_bwd(s["dy"], p, s["seed"], s["offset"], s["dx"])
        return {"y": s["y"], "dx": s["dx"]}
    x = s["x"]
    below = math.floor(p * 65536 + 0.5)
    kept = (_mask64(s["seed"], s["offset"], x.numel()) >= below).reshape(x.shape)
    scale = 65536.0 / (65536 - below)
    zero = torch.zeros((), device=DEV)
    y = torch.where(kept, x.float() * scale, zero)
    if "residual" in s:
        y = y + s["residual"].float()
    out = {"y": y.to(x.dtype)}
    if s["train"]:
        out["dx"] = torch.where(kept, s["dy"].float() * scale, zero).to(x.dtype)
    return out


def _scan(a, b, longest):
    """h[t] = a[t] h[t-1] + b[t] down the rows, no state before the first; no chain of non-zero a is longer than `longest`.
    Pairs (a, b) of neighbours are combined over distances 1, 2, 4, ..."""
    step = 1
    while step < longest:
        b = torch.cat([b[:step], b[step:] + a[step:] * b[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _run_recurrence(s):
    case = s["case"]
    z, u = _halves(case, s["zu"])
    h0, dh_last = s.get("h0"), s.get("dh_last")
    if own:
        from paper_2405_04416_amd import binding as B
        first = s["first"] if case["ragged"] else None
        if "ws" not in s:
            s["ws"] = torch.empty(B.dg_recurrence_workspace_bytes(s["N"], case["seqs"], case["width"]), dtype=torch.uint8, device=DEV)
            s["states"] = torch.empty(B.dg_recurrence_state_count(s["N"], case["width"]), device=DEV) if s["train"] else None
        B.dg_recurrence_fwd(z, u, case["seqs"], first, case["reverse"], h0, s["y"], s.get("h_last"), s["states"], s["ws"])
        out = {"y": s["y"]}
        if s["train"]:
            dz, du = _halves(case, s["dzu"])
            B.dg_recurrence_bwd(z, u, case["seqs"], first, case["reverse"], h0, s["states"], s["dy"], dh_last, dz, du, s.get("dh0"), s["ws"])
            out["dzu"] = s["dzu"]
        out.update({k: s[k] for k in ("h_last", "dh0") if k in s})
        return out
    dtype, longest, back = z.dtype, case["tokens"], case["reverse"]
    first = s["first"].long()
    some = first[1:] > first[:-1] if case["ragged"] else slice(None)        # the sequences that have tokens
    begin, end = first[:-1][some], first[1:][some] - 1
    if back:        # the same on rows in the opposite order
        begin, end = s["N"] - 1 - end, s["N"] - 1 - begin
    turn = (lambda t: t.flip(0)) if back else (lambda t: t)
    z, u = turn(z.float()), turn(u.float())
    a, c = 1.0 / (1.0 + torch.exp(-z)), 1.0 / (1.0 + torch.exp(z))
    b, chain = c * u, a.clone()
    if h0 is not None:
        b[begin] += a[begin] * h0[some]
    chain[begin] = 0.0
    h = _scan(chain, b, longest)
    out = {"y": turn(h).to(dtype)}
    if h0 is not None:
        out["h_last"] = h0.clone()
        out["h_last"][some] = h[end]
    if s["train"]:
        before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
        before[begin] = 0.0 if h0 is None else h0[some]
        g = turn(s["dy"].float()).clone()
        if dh_last is not None:
            g[end] += dh_last[some]
        after = torch.cat([a[1:], torch.zeros_like(a[:1])])
        after[end] = 0.0
        g = _scan(after.flip(0), g.flip(0), longest).flip(0)
        dz, du = turn(g * a * c * (before - u)).to(dtype), turn(g * c).to(dtype)
        out["dzu"] = torch.cat([dz, du], 1) if case["joint"] else (dz, du)
        if h0 is not None:
            out["dh0"] = dh_last.clone()
            out["dh0"][some] = (a * g)[begin]
    return out


# ---------------------------------------------------------------------------------------------------- work, exact values
def work(case):
    """Each input read once, each output written once."""
    item, train = torch.empty(0, dtype=TYPES[case["dtype"]]).element_size(), case["way"] == "train"
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        return {"bytes": n * item * (4 if train else 2) + case["width"] * (16 if train else 8), "flops": n * (19 if train else 8)}
    if case["op"] == "dropout":
        n = case["rows"] * case["width"]
        return {"bytes": n * item * ((4 if train else 2) + case["residual"]), "flops": n * (8 if train else 6)}
    n, per_seq = sum(_lengths(case)) * case["width"], case["seqs"] * case["width"]
    size = n * item * (6 if train else 3) + (per_seq * (16 if train else 8) if case["carry"] else 0) + (4 * case["seqs"] if case["ragged"] else 0)
    return {"bytes": size, "flops": n * (24 if train else 8)}


def exact(case, seed):
    """The definitions in 64 bits: gradients of the norm by differentiation, the recurrence token after token, random bits on the host."""
    s = prepare(case, seed)
    train = s["train"]
    if case["op"] == "norm":
        x, gamma, beta = (s[k].double().requires_grad_(train) for k in ("x", "gamma", "beta"))
        mean = x.sum(1, keepdim=True) / case["width"]
        variance = ((x - mean) ** 2).sum(1, keepdim=True) / case["width"]
        y = (x - mean) / torch.sqrt(variance + EPS) * gamma + beta
        out = {"y": y.detach()}
        if train:
            out["dx"], out["dgamma"], out["dbeta"] = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
        return out
    if case["op"] == "dropout":
        n = case["rows"] * case["width"]
        with np.errstate(over="ignore"):
            word = np.uint64(s["seed"]) + np.uint64(0x9E3779B97F4A7C15) * (np.arange(-(-n // 4), dtype=np.uint64) + np.uint64(s["offset"] + 1))
            word ^= word >> np.uint64(30)
            word *= np.uint64(0xBF58476D1CE4E5B9)
            word ^= word >> np.uint64(27)
            word *= np.uint64(0x94D049BB133111EB)
            word ^= word >> np.uint64(31)
        below = int(np.floor(case["p"] * 65536 + 0.5))
        keep = torch.from_numpy((word.view(np.uint16)[:n] >= below).reshape(case["rows"], case["width"])).to(DEV)
        factor = keep.double() * (65536 / (65536 - below))
        y = s["x"].double() * factor
        if case["residual"]:
            y += s["residual"].double()
        out = {"y": y}
        if train:
            out["dx"] = s["dy"].double() * factor
        return out
    return _exact_recurrence(case, s)


def _exact_recurrence(case, s):
    # tokens beside each other, sequence after sequence, padded to the longest with gates that keep the state
    width, seqs, T, N, train = case["width"], case["seqs"], case["tokens"], s["N"], s["train"]
    first = s["first"].long()
    if T * (2 if train else 1) * (3 if case["ragged"] else 1) > 300000:      # steps that would take too long
        return None
    if seqs * T > 1 << 24 or seqs * T * width > 3 * LARGEST:
        return None
    length = first[1:] - first[:-1]
    place = torch.arange(T, device=DEV)[None, :]
    held = place < length[:, None]                                   # [seqs, T]
    at = torch.where(held, first[:-1, None] + (length[:, None] - 1 - place if case["reverse"] else place), 0)
    z, u = (t.double() for t in _halves(case, s["zu"]))
    a_all = torch.sigmoid(z)
    h = s["h0"].double() if case["carry"] else torch.zeros(seqs, width, device=DEV, dtype=torch.float64)
    y = torch.empty(N, width, device=DEV, dtype=torch.float64)
    before = torch.empty(N, width, device=DEV, dtype=torch.float64) if train else None
    even = not case["ragged"]
    for t in range(T):
        who = slice(None) if even else held[:, t].nonzero()[:, 0]
        rows = at[who, t]
        a = a_all[rows]
        was = h[who]
        now = torch.addcmul(u[rows], a, was - u[rows])               # u + a (h - u) = a h + (1 - a) u
        if train:
            before[rows] = was
        y[rows] = now
        if even:
            h = now
        else:
            h[who] = now
    out = {"y": y}
    if case["carry"]:
        out["h_last"] = h
    if train:
        g = s["dh_last"].double() if case["carry"] else torch.zeros(seqs, width, device=DEV, dtype=torch.float64)
        dz, du = torch.empty_like(y), torch.empty_like(y)
        dy = s["dy"].double()
        for t in reversed(range(T)):
            who = slice(None) if even else held[:, t].nonzero()[:, 0]
            rows = at[who, t]
            a, total = a_all[rows], g[who] + dy[rows]
            dz[rows] = total * (before[rows] - u[rows]) * a * torch.sigmoid(-z[rows])
            du[rows] = total * torch.sigmoid(-z[rows])
            if even:
                g = total * a
            else:
                g[who] = total * a
        out["dzu"] = torch.cat([dz, du], 1) if case["joint"] else (dz, du)
        if case["carry"]:
            out["dh0"] = g
    return out
