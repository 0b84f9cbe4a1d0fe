"""Cases that time the operators of a block with an associative memory: root-mean-square norm with the residual's addition, rows in
8-bit floating point with a scale for each block of 128 columns, the matrix product of such rows, and the gated delta rule.

A case is one pass of a user's program through one operator on one GPU: the call alone ("fwd": rendering, serving), or the
call and its gradient ("train").  `own` False computes the same in elementary torch operations in 32 bits, rounded once at
the end; True calls the package's entry points.  Inputs are synthetic and made on the GPU from the seed.
"""
import math

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu      # values, and scales that are powers of two
BLOCK = 128             # columns that share a scale
CHUNK = 64              # tokens that the plain delta rule takes at once
SHUT = -200.0           # exp of it is 0 in 32 bits: logarithms of decays below it are as good
LARGEST = 1 << 28       # elements of one input


def _norm(name, way, dtype, rows, width, residual):
    c = dict(op="norm", way=way, dtype=dtype, rows=rows, width=width, residual=residual)
    return dict(c, name=name) if name else c


def _rows8(name, dtype, rows, width, norm, residual):
    """norm: the rows are normed first, and with residual the residual is added before that."""
    c = dict(op="rows8", way="fwd", dtype=dtype, rows=rows, width=width, norm=norm, residual=residual)
    return dict(c, name=name) if name else c


def _product(name, dtype, rows, columns, depth):
    c = dict(op="product", way="fwd", dtype=dtype, rows=rows, columns=columns, depth=depth)
    return dict(c, name=name) if name else c


def _delta(name, way, dtype, seqs, tokens, heads_k, heads, dk, dv, ragged=False, joint=False, carry=False, reverse=False):
    """tokens: of each sequence, or of the longest one (ragged).  joint: q, k and v are ranges of columns of one projection.
    carry: the memory comes from outside and goes on.  reverse: back to front."""
    c = dict(op="delta", way=way, dtype=dtype, seqs=seqs, tokens=tokens, heads_k=heads_k, heads=heads, dk=dk, dv=dv, ragged=ragged, joint=joint, carry=carry,
             reverse=reverse)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the features (16 levels of 2) of a small batch's samples: launch latency
        _norm("norm_small", "fwd", "fp16", 1024, 32, True),
        # tokens of a wide sequence model, the residual stream through it
        _norm("norm_wide", "train", "bf16", 8192, 4096, True),
        # what goes into a projection in 8 bits: the sum with the residual, normed
        _rows8("norm_in_8_bits", "bf16", 16384, 2048, True, True),
        # weights of a projection whose rows are no multiple of a block, laid out for the product
        _rows8("weights_in_8_bits", "fp32", 5003, 1000, False, False),
        # a projection for the few sequences that are being served: all of the weights for a few rows
        _product("product_token", "bf16", 8, 8192, 4096),
        # odd sizes
        _product("product_odd", "fp16", 1003, 1213, 968),
        # a projection of many tokens that are read in at once
        _product("product_batch", "bf16", 16384, 4096, 4096),
        # one more token for every sequence that is being served: the memories go in and out
        _delta("delta_token", "fwd", "bf16", 256, 1, 8, 16, 128, 128, joint=True, carry=True),
        # the features along the samples of every ray of a training batch, two heads of 16
        _delta("delta_rays", "train", "fp16", 1 << 16, 64, 2, 2, 16, 16),
        # segments of very different lengths, as the occupancy-guided sampler makes them, some without a sample; back to front
        _delta("delta_ragged", "train", "fp32", 2003, 96, 1, 3, 24, 40, ragged=True, carry=True, reverse=True),
        # one long sequence read in: few heads, all the work lies along it
        _delta("delta_long", "fwd", "bf16", 1, 1 << 16, 8, 8, 128, 128, joint=True, carry=True),
        # a training batch of long sequences of a wide model, two value heads to a key head
        _delta("delta_batch", "train", "bf16", 2, 8192, 8, 16, 128, 128, joint=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths that models have, and any width."""
    usual = [w for w in (8, 16, 32, 48, 64, 96, 128, 256, 384, 512, 768, 1024, 1536, 2048, 4096, 8192) if lo <= w <= hi]
    return rng.choice(usual) if rng.random() < 0.6 else _log_uniform(rng, lo, hi)


def draw(rng):
    op = rng.choice(["norm", "rows8", "product", "delta", "delta", "delta"])
    way, dtype = rng.choice(["fwd", "train"]), rng.choice(["fp32", "fp16", "bf16"])
    if op == "norm":
        width = _width(rng, 8, 8192)
        return _norm(None, way, dtype, _log_uniform(rng, 64, min((1 << 25) // width, 1 << 21)), width, rng.random() < 0.6)
    if op == "rows8":
        width, norm = _width(rng, 8, 8192), rng.random() < 0.6
        return _rows8(None, dtype, _log_uniform(rng, 64, min((1 << 25) // width, 1 << 20)), width, norm, norm and rng.random() < 0.6)
    if op == "product":
        rows, columns = _log_uniform(rng, 1, 16384), _width(rng, 64, 8192)
        depth = min(_width(rng, 64, 8192), (16384 * 4096 * 4096) // (rows * columns))
        return _product(None, rng.choice(["fp16", "bf16"]), rows, columns, depth)
    dk, dv = (rng.choice([16, 32, 64, 128]) if rng.random() < 0.6 else rng.randint(8, 128) for _ in range(2))
    heads_k, group = _log_uniform(rng, 1, 16), rng.choice([1, 1, 2, 3, 4])
    heads = heads_k * group
    tokens = 1 if rng.random() < 0.15 else _log_uniform(rng, 2, 1 << 16)
    # limits: products of the whole case, values that a chunk's matrices hold, values of all memories
    most = min(2 * 8192 * 16 * 128 * 128 // (heads * dk * dv), (1 << 22) // heads) // tokens
    seqs = _log_uniform(rng, 1, max(1, min(most, (1 << 26) // (heads * dk * dv), 1 << 16)))
    if most < 1:
        tokens = max(2, tokens * most)
        tokens = max(2, min(2 * 8192 * 16 * 128 * 128 // (heads * dk * dv), (1 << 22) // heads))
    return _delta(None, way, dtype, seqs, tokens, heads_k, heads, dk, dv, ragged=tokens > 1 and rng.random() < 0.35, joint=rng.random() < 0.4,
                  carry=tokens == 1 or rng.random() < 0.5, reverse=rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the sequences before they are shuffled: all the same, or 0, 1, 2, ... up to the longest and again."""
    if not case["ragged"]:
        return [case["tokens"]] * case["seqs"]
    m = case["tokens"] + 1
    return [case["tokens"]] + [j % m for j in range(case["seqs"] - 1)]


def _blocks(width):
    return -(-width // BLOCK)


def _empty8(rows, width):
    """Room for rows of 8-bit values, a multiple of 16 bytes apart as the product reads them."""
    return torch.empty(rows, -(-width // 16) * 16, device=DEV, dtype=torch.uint8).view(E4M3)[:, :width]


def _in_8_bits(y):
    """Rows of 32-bit values: the nearest 8-bit values, and for each block of columns the smallest power of two that brings them into range."""
    rows, width = y.shape
    blocks = _blocks(width)
    y = torch.cat([y, y.new_zeros(rows, blocks * BLOCK - width)], 1).reshape(rows, blocks, BLOCK)
    fraction, exponent = torch.frexp(y.abs().amax(2))       # largest = fraction 2^exponent, 448 = 0.875 2^9
    e = (exponent - 9 + (fraction > 0.875)).clamp(-127, 127)
    e = torch.where(fraction == 0, -127, e)
    q = torch.ldexp(y, -e[:, :, None].to(y.dtype))
    return q.reshape(rows, blocks * BLOCK)[:, :width].float().to(E4M3), (e + 127).to(torch.uint8).view(E8M0)


def prepare(case, seed):
    dtype = TYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=gen, dtype=torch.float32)      # noqa: E731
    empty = lambda *shape, dt=dtype: torch.empty(*shape, device=DEV, dtype=dt)                       # noqa: E731
    s = dict(case=case, train=case["way"] == "train")
    if case["op"] in ("norm", "rows8"):
        rows, width = case["rows"], case["width"]
        # channels of different size, as a residual stream has them
        s["x"] = (normal(rows, width) * torch.exp(normal(width))).to(dtype)
        if case["op"] == "norm" or case["norm"]:
            s.update(gamma=1.0 + 0.2 * normal(width))
        if case["residual"]:
            s.update(residual=normal(rows, width).to(dtype), total=empty(rows, width))
        if case["op"] == "rows8":
            s.update(q=_empty8(rows, width), scales=torch.empty(rows, _blocks(width), device=DEV, dtype=torch.uint8).view(E8M0))
            return s
        s.update(y=empty(rows, width))
        if s["train"]:
            s.update(dy=normal(rows, width).to(dtype), dx=empty(rows, width), dgamma=empty(width, dt=torch.float32))
            if case["residual"]:
                s.update(dtotal=normal(rows, width).to(dtype))
        return s
    if case["op"] == "product":
        for name, rows in (("a", case["rows"]), ("b", case["columns"])):
            q, scales = _in_8_bits(normal(rows, case["depth"]) * torch.exp(normal(case["depth"])))
            room = _empty8(rows, case["depth"])
            room.copy_(q)
            s[name] = room, scales
        s["y"] = empty(case["rows"], case["columns"])
        return s
    seqs, heads_k, heads, dk, dv = (case[k] for k in ("seqs", "heads_k", "heads", "dk", "dv"))
    lengths = torch.tensor(_lengths(case), device=DEV)
    if case["ragged"]:
        lengths = lengths[torch.randperm(seqs, device=DEV, generator=gen)]
    ends = torch.cumsum(lengths, 0)
    N = sum(_lengths(case))
    s.update(N=N, first=torch.cat([ends.new_zeros(1), ends]).to(torch.int32))
    parts = [normal(N, heads_k, dk), normal(N, heads_k, dk), normal(N, heads, dv)]
    parts[:2] = [t / torch.sqrt((t * t).sum(2, keepdim=True) + 1e-12) for t in parts[:2]]       # queries and keys of length one
    parts = [t.reshape(N, t.shape[1] * t.shape[2]).to(dtype) for t in parts]
    s["qkv"] = torch.cat(parts, 1) if case["joint"] else tuple(parts)
    # decays that keep from half to nearly all of the memory, now and then one that forgets all; rates between 0 and 1
    u = torch.rand(N, heads, device=DEV, generator=gen)
    s["g"] = torch.where(torch.rand(N, heads, device=DEV, generator=gen) < 1e-3, -math.inf, -torch.exp(-0.4 - 6.0 * u))
    s["beta"] = 1.0 / (1.0 + torch.exp(-1.5 * normal(N, heads)))
    s["o"] = empty(N, heads * dv)
    if case["carry"]:
        s.update(s0=normal(seqs, heads, dk, dv) * 0.5, s_last=empty(seqs, heads, dk, dv, dt=torch.float32))
    if s["train"]:
        s.update(do=normal(N, heads * dv).to(dtype), dg=empty(N, heads, dt=torch.float32), dbeta=empty(N, heads, dt=torch.float32))
        widths = [t.shape[1] for t in parts]
        s["dqkv"] = empty(N, sum(widths)) if case["joint"] else tuple(empty(N, w) for w in widths)
        if case["carry"]:
            s.update(ds_last=normal(seqs, heads, dk, dv) * 0.1, ds0=empty(seqs, heads, dk, dv, dt=torch.float32))
    return s


def _thirds(case, rows):
    """q, k and v of a joint projection, or of three."""
    if not case["joint"]:
        return rows
    a, b = case["heads_k"] * case["dk"], 2 * case["heads_k"] * case["dk"]
    return rows[:, :a], rows[:, a:b], rows[:, b:]


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"norm": _run_norm, "rows8": _run_rows8, "product": _run_product, "delta": _run_delta}[state["case"]["op"]](state)


def _run_norm(s):
    with_total = "residual" in s
    if own:
        from paper_2405_04416_amd import binding as B
        B.dg_rms_norm_fwd(s["x"], s.get("residual"), s["gamma"], EPS, s.get("total"), s["y"])
        out = {"y": s["y"]}
        if with_total:
            out["total"] = s["total"]
        if s["train"]:
            if "ws" not in s:
                s["ws"] = torch.empty(B.dg_rms_norm_bwd_workspace_bytes(*s["x"].shape), dtype=torch.uint8, device=DEV)
            B.dg_rms_norm_bwd(s["total"] if with_total else s["x"], s["gamma"], s["dy"], s.get("dtotal"), EPS, s["dx"], s["dgamma"], s["ws"])
            out.update(dx=s["dx"], dgamma=s["dgamma"])
        return out
    total, out = s["x"], {}
    if with_total:
        total = out["total"] = (s["x"].float() + s["residual"].float()).to(total.dtype)
    x = total.float()
    scale = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    xh = x * scale
    out["y"] = (xh * s["gamma"]).to(total.dtype)
    if s["train"]:
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = scale * (g - xh * (g * xh).mean(1, keepdim=True))
        out.update(dx=(dx + s["dtotal"].float() if with_total else dx).to(total.dtype), dgamma=(dy * xh).sum(0))
    return out


def _run_rows8(s):
    norm, with_total = s["case"]["norm"], "residual" in s
    if own:
        from paper_2405_04416_amd import binding as B
        if norm:
            B.dg_rms_norm_e4m3_fwd(s["x"], s.get("residual"), s["gamma"], EPS, s.get("total"), s["q"], s["scales"])
        else:
            B.dg_e4m3_rows(s["x"], s["q"], s["scales"])
        out = {"q": s["q"], "scales": s["scales"]}
        if with_total:
            out["total"] = s["total"]
        return out
    total, out = s["x"], {}
    if with_total:
        total = out["total"] = (s["x"].float() + s["residual"].float()).to(total.dtype)
    y = total.float()
    if norm:
        y = y * (1.0 / torch.sqrt((y * y).mean(1, keepdim=True) + EPS)) * s["gamma"]
    out["q"], out["scales"] = _in_8_bits(y)
    return out


def _values(q, scales):
    """What 8-bit rows stand for."""
    return q.float() * scales.float().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _run_product(s):
    if own:
        from paper_2405_04416_amd import binding as B
        if "ws" not in s:
            s["ws"] = torch.empty(B.dg_e4m3_product_workspace_bytes(*(s["case"][k] for k in ("rows", "columns", "depth"))), dtype=torch.uint8, device=DEV)
        B.dg_e4m3_product(*s["a"], *s["b"], s["y"], s["ws"])
        return {"y": s["y"]}
    return {"y": (_values(*s["a"]) @ _values(*s["b"]).t()).to(s["y"].dtype)}


def _run_delta(s):
    case, (q, k, v) = s["case"], _thirds(s["case"], s["qkv"])
    if own:
        from paper_2405_04416_amd import binding as B
        seqs, heads_k, heads, dk, dv = (case[n] for n in ("seqs", "heads_k", "heads", "dk", "dv"))
        first, scale = s["first"] if case["ragged"] else None, dk ** -0.5
        if "ws" not in s:
            s["ws"] = torch.empty(B.dg_delta_rule_workspace_bytes(s["N"], seqs, heads_k, heads, dk, dv), dtype=torch.uint8, device=DEV)
            s["saved"] = torch.empty(B.dg_delta_rule_saved_bytes(s["N"], seqs, heads, dk, dv), dtype=torch.uint8, device=DEV) if s["train"] else None
        B.dg_delta_rule_fwd(q, k, v, s["g"], s["beta"], heads_k, seqs, first, case["reverse"], scale, s.get("s0"), s["o"], s.get("s_last"), s["saved"], s["ws"])
        out = {"o": s["o"]}
        if s["train"]:
            B.dg_delta_rule_bwd(q, k, v, s["g"], s["beta"], heads_k, seqs, first, case["reverse"], scale, s["saved"], s["do"], s.get("ds_last"),
                                *_thirds(case, s["dqkv"]), s["dg"], s["dbeta"], s.get("ds0"), s["ws"])
            out.update(dqkv=s["dqkv"], dg=s["dg"], dbeta=s["dbeta"])
        out.update({n: s[n] for n in ("s_last", "ds0") if n in s})
        return out
    return _plain_delta(s, case, q, k, v)


def _places(case, s, multiple):
    """Rows of the sequences' tokens beside each other, [seqs, T] with T a multiple of `multiple`, in the order that they are taken, and which are any."""
    T = -(-case["tokens"] // multiple) * multiple
    first = s["first"].long()
    length = first[1:] - first[:-1]
    place = torch.arange(T, device=DEV)[None, :]
    held = place < length[:, None]
    return torch.where(held, first[:-1, None] + (length[:, None] - 1 - place if case["reverse"] else place), 0), held


def _plain_delta(s, case, q, k, v):
    """Chunk after chunk.  S is the memory before a chunk, D[i, j] how much of what token j left is there at token i, U what the tokens write:
        (1 + A) U = beta (V - e^G K S),  A[i, j] = beta[i] D[i, j] k[i] k[j] below the diagonal,
        O = e^G Q S + P U,  P[i, j] = D[i, j] q[i] k[j] up to the diagonal,  S' = e^G[last] S + K^T (e^(G[last] - G) U)."""
    seqs, heads_k, heads, dk, dv = (case[n] for n in ("seqs", "heads_k", "heads", "dk", "dv"))
    dtype, N, group = v.dtype, s["N"], case["heads"] // case["heads_k"]
    at, held = _places(case, s, CHUNK)
    chunks, BH = at.shape[1] // CHUNK, seqs * heads

    def spread(rows, n, d, times=1):            # [N, n d] -> [chunks, seqs heads, CHUNK, d], nothing where no token is
        t = rows.float().reshape(N, n, d)[at] * held[:, :, None, None]
        return t.repeat_interleave(times, 2).reshape(seqs, chunks, CHUNK, heads, d).permute(1, 0, 3, 2, 4).reshape(chunks, BH, CHUNK, d)

    def gather(t):                              # and back
        t = t.reshape(chunks, seqs, heads, CHUNK, -1).permute(1, 0, 3, 2, 4).reshape(seqs, chunks * CHUNK, heads, -1)
        out = t.new_empty(N, heads, t.shape[3])
        out[at[held]] = t[held]
        return out

    Q, K, V = spread(q, heads_k, dk, group) * dk ** -0.5, spread(k, heads_k, dk, group), spread(v, heads, dv)
    beta = spread(s["beta"], heads, 1)
    G = torch.cumsum(spread(s["g"].clamp_min(SHUT), heads, 1).double(), 2)
    lower = torch.ones(CHUNK, CHUNK, device=DEV, dtype=torch.bool).tril()
    D = torch.where(lower, torch.exp(torch.where(lower, G - G.transpose(2, 3), 0.0).float()), 0.0)
    since, until = torch.exp(G.float()), torch.exp((G[:, :, -1:] - G).float())
    whole = since[:, :, -1:]
    kk = torch.where(lower.tril(-1), D * (K @ K.transpose(2, 3)), 0.0)
    P, A = D * (Q @ K.transpose(2, 3)), beta * kk
    inverse = torch.eye(CHUNK, device=DEV).expand_as(A).clone()
    for i in range(1, CHUNK):
        inverse[:, :, i, :i] = -(A[:, :, i, :i, None] * inverse[:, :, :i, :i]).sum(2)
    S = s["s0"].reshape(BH, dk, dv) if "s0" in s else torch.zeros(BH, dk, dv, device=DEV)
    O, U, before = torch.empty_like(V), torch.empty_like(V), []
    for c in range(chunks):
        before.append(S)
        U[c] = inverse[c] @ (beta[c] * (V[c] - since[c] * (K[c] @ S)))
        O[c] = since[c] * (Q[c] @ S) + P[c] @ U[c]
        S = whole[c] * S + K[c].transpose(1, 2) @ (until[c] * U[c])
    out = {"o": gather(O).reshape(N, heads * dv).to(dtype)}
    if "s_last" in s:
        out["s_last"] = S.reshape(seqs, heads, dk, dv)
    if not s["train"]:
        return out
    dO = spread(s["do"], heads, dv)
    dS = s["ds_last"].reshape(BH, dk, dv) if "ds_last" in s else torch.zeros(BH, dk, dv, device=DEV)
    dQ, dK, dV, dbeta, dG = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V), torch.empty_like(beta), torch.empty_like(beta)
    for c in reversed(range(chunks)):
        S, UU = before[c], until[c] * U[c]
        dU = P[c].transpose(1, 2) @ dO[c] + until[c] * (K[c] @ dS)
        dR = inverse[c].transpose(1, 2) @ dU
        E = dR @ U[c].transpose(1, 2)
        M = dO[c] @ U[c].transpose(1, 2)
        read_q, read_k, write_k = since[c] * (dO[c] @ S.transpose(1, 2)), -beta[c] * since[c] * (dR @ S.transpose(1, 2)), UU @ dS.transpose(1, 2)
        MD, ED = torch.where(lower, M * D[c], 0.0), torch.where(lower.tril(-1), -beta[c] * E * D[c], 0.0)
        dQ[c] = read_q + MD @ K[c]
        dK[c] = read_k + write_k + MD.transpose(1, 2) @ Q[c] + ED @ K[c] + ED.transpose(1, 2) @ K[c]
        dV[c] = beta[c] * dR
        dbeta[c] = (dR * V[c]).sum(2, keepdim=True) - since[c] * (K[c] * (dR @ S.transpose(1, 2))).sum(2, keepdim=True) - (kk[c] * E).sum(2, keepdim=True)
        both = M * P[c] - E * A[c]
        at_end = (k_write := K[c] * write_k).sum(2, keepdim=True)
        dG[c] = (Q[c] * read_q).sum(2, keepdim=True) + (K[c] * read_k).sum(2, keepdim=True) - at_end + both.sum(2, keepdim=True) - both.sum(1)[:, :, None]
        dG[c, :, -1] += k_write.sum((1, 2))[:, None] + whole[c, :, 0] * (S * dS).sum((1, 2))[:, None]
        dS = whole[c] * dS + Q[c].transpose(1, 2) @ (since[c] * dO[c]) - K[c].transpose(1, 2) @ (beta[c] * since[c] * dR)
    dg = dG.flip(2).cumsum(2).flip(2)
    share = lambda t: gather(t).reshape(N, heads_k, group, dk).sum(2).reshape(N, heads_k * dk).to(dtype)         # noqa: E731
    grads = share(dQ * dk ** -0.5), share(dK), gather(dV).reshape(N, heads * dv).to(dtype)
    out.update(dqkv=torch.cat(grads, 1) if case["joint"] else grads, dg=gather(dg)[:, :, 0], dbeta=gather(dbeta)[:, :, 0])
    if "ds0" in s:
        out["ds0"] = dS.reshape(seqs, heads, dk, dv)
    return out


# ---------------------------------------------------------------------------------------------------- work, exact values
def work(case):
    """Each input read once, each output written once; what the delta rule takes token by token."""
    item, train = torch.empty(0, dtype=TYPES[case["dtype"]]).element_size(), case["way"] == "train"
    if case["op"] == "norm":
        n, with_total = case["rows"] * case["width"], case["residual"]
        arrays = (2 + 2 * with_total) + ((2 + with_total) if train else 0)
        return {"bytes": n * item * arrays + case["width"] * (8 if train else 4), "flops": n * ((15 if train else 4) + with_total * (2 if train else 1))}
    if case["op"] == "rows8":
        n = case["rows"] * case["width"]
        return {"bytes": n * (item * (1 + 2 * case["residual"]) + 1) + case["rows"] * _blocks(case["width"]) + 4 * case["width"] * case["norm"],
                "flops": n * (2 + 4 * case["norm"] + case["residual"])}
    if case["op"] == "product":
        rows, columns, depth = case["rows"], case["columns"], case["depth"]
        return {"bytes": (rows + columns) * (depth + _blocks(depth)) + 2 * rows * columns, "flops": 2 * rows * columns * depth}
    N, seqs, heads_k, heads, dk, dv = sum(_lengths(case)), *(case[n] for n in ("seqs", "heads_k", "heads", "dk", "dv"))
    qk, vs, memory = N * heads_k * dk * item, N * heads * dv * item, seqs * heads * dk * dv * 4
    size = (4 * qk + 2 * vs + 2 * vs + 4 * N * heads * 4 + 0) if train else (2 * qk + 2 * vs + 2 * N * heads * 4)
    return {"bytes": size + case["carry"] * memory * (4 if train else 2) + 4 * (seqs + 1) * case["ragged"], "flops": N * heads * dk * dv * (20 if train else 6)}


def exact(case, seed):
    """The definitions in 64 bits: gradients of the norm by differentiation, the delta rule token after token."""
    if case["op"] == "delta" and case["tokens"] * (40 if case["way"] == "train" else 12) * (
            1e-5 + 16.0 * case["seqs"] * case["heads"] * case["dk"] * case["dv"] / 2.5e12) > 15:
        return None
    s = prepare(case, seed)
    if case["op"] == "product":
        a, b = (q.double() * scales.double().repeat_interleave(BLOCK, 1)[:, :case["depth"]] for q, scales in (s["a"], s["b"]))
        return {"y": a @ b.t()}
    if case["op"] == "delta":
        return _exact_delta(case, s)
    out, x = {}, s["x"].double()
    if "residual" in s:
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
        out["total"] = x.clone()
    if case["op"] == "rows8":
        if case["norm"]:
            x = x * s["gamma"].double() / torch.sqrt((x ** 2).sum(1, keepdim=True) / case["width"] + EPS)
        scales = torch.empty(case["rows"], _blocks(case["width"]), device=DEV, dtype=torch.float64)
        for j in range(scales.shape[1]):
            block = x[:, j * BLOCK:(j + 1) * BLOCK]
            scale = torch.exp2(torch.ceil(torch.log2(block.abs().amax(1, keepdim=True) / 448.0)).clamp(-127, 127))
            scales[:, j:j + 1] = scale
            # the nearest multiple of the step that the value's size has: 3 bits after the first, from 2^-6 on
            block /= scale
            step = torch.exp2(torch.floor(torch.log2(block.abs().clamp_min(2.0 ** -6))) - 3)
            block.copy_(torch.round(block / step) * step)
        return dict(out, q=x, scales=scales)
    gamma = s["gamma"].double().requires_grad_(s["train"])
    x.requires_grad_(s["train"])
    y = x * gamma / torch.sqrt((x ** 2).sum(1, keepdim=True) / case["width"] + EPS)
    out["y"] = y.detach()
    if s["train"]:
        out["dx"], out["dgamma"] = torch.autograd.grad(y, (x, gamma), s["dy"].double())
        if "dtotal" in s:
            out["dx"] += s["dtotal"].double()
    return out


def _exact_delta(case, s):
    """S <- e^g S, e = v - S^T k, S <- S + beta k e^T, o = S^T q, for all sequences at once; back through it with the states of a
    stretch of tokens computed again."""
    seqs, heads_k, heads, dk, dv, T = (case[n] for n in ("seqs", "heads_k", "heads", "dk", "dv", "tokens"))
    N, group, train, scale = s["N"], case["heads"] // case["heads_k"], s["train"], case["dk"] ** -0.5
    at, held = _places(case, s, 1)
    q, k, v = _thirds(case, s["qkv"])
    wide = lambda rows, t, n, d: rows.reshape(N, n, d)[at[:, t]].double()                                   # noqa: E731   [seqs, n, d]
    some = lambda t: held[:, t].double()[:, None]                                                           # noqa: E731

    def token(t):
        on = some(t)
        qt, kt = (wide(r, t, heads_k, dk).repeat_interleave(group, 1) * on[:, :, None] for r in (q, k))
        g, b = s["g"][at[:, t]].double() * 1.0, s["beta"][at[:, t]].double() * on
        return qt * scale, kt, wide(v, t, heads, dv), torch.where(on > 0, torch.exp(g), 1.0), b

    def step(S, t):
        qt, kt, vt, a, b = token(t)
        S = S * a[:, :, None, None]
        e = vt - (S * kt[:, :, :, None]).sum(2)
        return S + kt[:, :, :, None] * (b[:, :, None] * e)[:, :, None, :], e

    S = s["s0"].double() if "s0" in s else torch.zeros(seqs, heads, dk, dv, device=DEV, dtype=torch.float64)
    o = torch.empty(N, heads, dv, device=DEV, dtype=torch.float64)
    stretch, marks = 64, []
    for t in range(T):
        if train and t % stretch == 0:
            marks.append(S)
        S, _ = step(S, t)
        on = held[:, t]
        o[at[on, t]] = (S * token(t)[0][:, :, :, None]).sum(2)[on]
    out = {"o": o.reshape(N, heads * dv)}
    if "s_last" in s:
        out["s_last"] = S
    if not train:
        return out
    f64 = dict(device=DEV, dtype=torch.float64)
    dq, dk_, dv_ = torch.empty(N, heads_k, dk, **f64), torch.empty(N, heads_k, dk, **f64), torch.empty(N, heads, dv, **f64)
    dg, dbeta = torch.empty(N, heads, **f64), torch.empty(N, heads, **f64)
    dS = s["ds_last"].double() if "ds_last" in s else torch.zeros(seqs, heads, dk, dv, **f64)
    for m in reversed(range(len(marks))):
        states = [marks[m]]
        for t in range(m * stretch, min(T, (m + 1) * stretch)):
            states.append(step(states[-1], t)[0])
        for t in reversed(range(m * stretch, min(T, (m + 1) * stretch))):
            qt, kt, vt, a, b = token(t)
            was, now = states[t - m * stretch], states[t - m * stretch + 1]
            faded = was * a[:, :, None, None]
            e = vt - (faded * kt[:, :, :, None]).sum(2)
            dot = wide(s["do"], t, heads, dv) * some(t)[:, :, None]
            on = held[:, t]
            rows = at[on, t]
            gq = (now * dot[:, :, None, :]).sum(3) * scale
            dS = dS + qt[:, :, :, None] * dot[:, :, None, :]
            du = (dS * kt[:, :, :, None]).sum(2)
            de = b[:, :, None] * du
            gk = (dS * (b[:, :, None] * e)[:, :, None, :]).sum(3) - (faded * de[:, :, None, :]).sum(3)
            dq[rows], dk_[rows] = (x.reshape(seqs, heads_k, group, dk).sum(2)[on] for x in (gq, gk))
            dv_[rows], dbeta[rows] = de[on], (du * e).sum(2)[on]
            dS = dS - kt[:, :, :, None] * de[:, :, None, :]
            dg[rows] = (dS * faded).sum((2, 3))[on]
            dS = dS * a[:, :, None, None]
            states[t - m * stretch + 1] = None
    grads = dq.reshape(N, heads_k * dk), dk_.reshape(N, heads_k * dk), dv_.reshape(N, heads * dv)
    out.update(dqkv=torch.cat(grads, 1) if case["joint"] else grads, dg=dg, dbeta=dbeta)
    if "ds0" in s:
        out["ds0"] = dS
    return out
