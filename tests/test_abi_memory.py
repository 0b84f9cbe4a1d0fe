"""What the entry points of the block with an associative memory refuse before they launch anything, and what they take with nothing to do.  Addresses are made up:
a call that is refused reads none."""
import pytest
import torch

from paper_2405_04416_amd import binding as B

P = 4096                    # an aligned address


def lib():
    return B.lib()


def error():
    return lib().dg_last_error().decode()


def norm(x=P, ldx=8, r=None, ldr=8, gamma=None, N=4, W=8, eps=1e-5, dtype=0, t=None, ldt=8, y=P, ldy=8):
    return lib().dg_rms_norm_fwd(x, ldx, r, ldr, gamma, N, W, eps, dtype, t, ldt, y, ldy, None)


def test_norm_refusals():
    assert norm(x=None, y=None, N=0) == 0
    for bad in (dict(x=None), dict(y=None), dict(W=0), dict(eps=-1.0), dict(eps=float("nan")), dict(dtype=3), dict(ldx=7), dict(ldy=7), dict(x=P + 2), dict(y=P + 2),
                dict(r=P + 2), dict(r=P, ldr=7), dict(t=P + 2), dict(t=P, ldt=7), dict(gamma=P + 2)):
        assert norm(**bad) == -1, bad
    assert norm(N=1 << 33) == -2
    assert norm(W=(1 << 20) + 1, N=1, ldx=1 << 21, ldy=1 << 21) == -2


def norm_bwd(t=P, ldt=8, gamma=None, dy=P, lddy=8, dt=None, lddt=8, N=4, W=8, eps=1e-5, dtype=0, dx=P, lddx=8, dgamma=None, ws=None, n=0):
    return lib().dg_rms_norm_bwd(t, ldt, gamma, dy, lddy, dt, lddt, N, W, eps, dtype, dx, lddx, dgamma, ws, n, None)


def test_norm_gradient_refusals():
    assert norm_bwd(t=None, dy=None, dx=None, N=0) == 0
    for bad in (dict(t=None), dict(dy=None), dict(W=0), dict(eps=-1.0), dict(dtype=9), dict(ldt=7), dict(lddy=7), dict(dt=P, lddt=7), dict(dt=P + 2), dict(lddx=7), dict(dx=P + 1),
                dict(dgamma=P + 2, ws=P, n=1 << 30)):
        assert norm_bwd(**bad) == -1, bad
    need = B.dg_rms_norm_bwd_workspace_bytes(4, 8)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=P, n=need - 1), dict(ws=P + 8, n=need)):
        assert norm_bwd(dgamma=P, **bad) == -3, bad
    assert B.dg_rms_norm_bwd_workspace_bytes(1 << 24, 32) <= 8 << 20


def rows8(x=P, ldx=8, N=4, W=8, dtype=0, q=P, ldq=16, s=P, lds=1):
    return lib().dg_e4m3_rows(x, ldx, N, W, dtype, q, ldq, s, lds, None)


def norm8(x=P, ldx=8, r=None, ldr=8, N=4, W=8, eps=1e-5, dtype=0, t=None, ldt=8, q=P, ldq=16, s=P, lds=1):
    return lib().dg_rms_norm_e4m3_fwd(x, ldx, r, ldr, None, N, W, eps, dtype, t, ldt, q, ldq, s, lds, None)


def test_rows_in_8_bits_refusals():
    for f in (rows8, norm8):
        assert f(x=None, q=None, s=None, N=0) == 0
        for bad in (dict(x=None), dict(q=None), dict(s=None), dict(q=P + 8), dict(ldq=24), dict(W=32, ldx=32, ldq=16), dict(W=129, ldx=129, ldq=144, lds=1), dict(dtype=3), dict(W=0)):
            assert f(**bad) == -1, bad
        assert f(N=1 << 33) == -2
    assert norm8(eps=-1.0) == -1 and norm8(r=P, ldr=7) == -1 and norm8(t=P, ldt=7) == -1


def product(a=P, lda=128, sa=P, ldsa=1, b=P, ldb=128, sb=P, ldsb=1, M=4, N=4, K=128, dtype=1, y=P, ldy=4, ws=None, n=0):
    return lib().dg_e4m3_product(a, lda, sa, ldsa, b, ldb, sb, ldsb, M, N, K, dtype, y, ldy, ws, n, None)


def test_product_refusals():
    assert product(a=None, sa=None, y=None, M=0) == 0 and product(b=None, sb=None, y=None, N=0) == 0
    for bad in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(y=None), dict(a=P + 8), dict(b=P + 8), dict(lda=136), dict(ldb=120), dict(K=129, lda=144, ldb=144),
                dict(K=0), dict(dtype=0), dict(dtype=3), dict(ldy=3), dict(y=P + 1)):
        assert product(**bad) == -1, bad
    for bad in (dict(M=(1 << 24) + 1), dict(N=(1 << 24) + 1, ldy=1 << 25), dict(M=1 << 20, N=(1 << 19) + 1, ldy=1 << 20), dict(lda=1 << 24), dict(ldb=1 << 24)):
        assert product(**bad) == -2, bad
    M, N, K = 100, 64, 8192                 # few results of long sums
    need = B.dg_e4m3_product_workspace_bytes(M, N, K)
    assert need > 0 and B.dg_e4m3_product_workspace_bytes(0, N, K) == 0 and B.dg_e4m3_product_workspace_bytes(4096, 4096, 128) == 0
    long = dict(M=M, N=N, K=K, lda=K, ldb=K, ldsa=64, ldsb=64, ldy=N)
    for bad in (dict(ws=None), dict(ws=P, n=need - 1), dict(ws=P + 8, n=need)):
        assert product(**long, **bad) == -3, bad


def delta(q=P, ldq=8, k=P, ldk=8, v=P, ldv=16, g=P, ldg=4, beta=P, ldb=4, N=6, n_seq=2, first=None, Hk=2, H=4, Dk=4, Dv=4, reverse=0, scale=1.0, dtype=0, s0=None, o=P, ldo=16,
          s_last=None, saved=None, saved_n=0, ws=P, n=1 << 40):
    return lib().dg_delta_rule_fwd(q, ldq, k, ldk, v, ldv, g, ldg, beta, ldb, N, n_seq, first, Hk, H, Dk, Dv, reverse, scale, dtype, s0, o, ldo, s_last, saved, saved_n, ws, n, None)


SHARED = (dict(q=None), dict(k=None), dict(v=None), dict(g=None), dict(beta=None), dict(ldq=7), dict(ldk=7), dict(ldv=15), dict(ldg=3), dict(ldb=3), dict(q=P + 2), dict(g=P + 2),
          dict(N=7), dict(n_seq=0), dict(Hk=3), dict(Hk=0), dict(H=0), dict(Dk=0), dict(Dv=0), dict(scale=float("inf")), dict(scale=float("nan")), dict(dtype=3), dict(first=P + 2))
BEYOND = (dict(Dk=129, ldq=1024, ldk=1024), dict(Dv=129, ldv=1024), dict(N=1 << 32), dict(n_seq=1 << 31), dict(H=(1 << 16) + 2, ldv=1 << 20, ldg=1 << 20, ldb=1 << 20), dict(ldq=1 << 24), dict(ldv=1 << 24),
          dict(N=1 << 31, n_seq=1, H=64, ldv=1 << 10, ldg=64, ldb=64), dict(N=0, n_seq=1 << 30, H=8))


def test_delta_rule_refusals():
    none = dict(q=None, k=None, v=None, g=None, beta=None, o=None, N=0, n_seq=0)
    assert delta(**none) == 0
    for bad in SHARED + (dict(o=None), dict(ldo=15), dict(o=P + 2), dict(s0=P + 2), dict(s_last=P + 1)):
        assert delta(**bad) == -1, bad
    for bad in BEYOND:
        assert delta(**bad) == -2, bad
    need = B.dg_delta_rule_saved_bytes(6, 2, 4, 4, 4)
    for bad in (dict(saved=P, saved_n=need - 1), dict(saved=P + 8, saved_n=need)):
        assert delta(**bad) == -3, bad
    long = dict(N=80, Dk=64, Dv=64, ldq=128, ldk=128, ldv=256, ldo=256)
    need = B.dg_delta_rule_fwd_workspace_bytes(80, 2, 4)
    for bad in (dict(ws=None, n=0), dict(n=need - 1), dict(ws=P + 8, n=need)):
        assert delta(**long, **bad) == -3, bad


def delta_bwd(q=P, ldq=8, k=P, ldk=8, v=P, ldv=16, g=P, ldg=4, beta=P, ldb=4, N=6, n_seq=2, first=None, Hk=2, H=4, Dk=4, Dv=4, reverse=0, scale=1.0, dtype=0, saved=P, saved_n=1 << 40,
              do=P, lddo=16, ds_last=None, dq=P, lddq=8, dk=P, lddk=8, dv=P, lddv=16, dg=P, lddg=4, dbeta=P, lddb=4, ds0=None, ws=P, n=1 << 40):
    return lib().dg_delta_rule_bwd(q, ldq, k, ldk, v, ldv, g, ldg, beta, ldb, N, n_seq, first, Hk, H, Dk, Dv, reverse, scale, dtype, saved, saved_n, do, lddo, ds_last, dq, lddq, dk, lddk,
                                   dv, lddv, dg, lddg, dbeta, lddb, ds0, ws, n, None)


def test_delta_rule_gradient_refusals():
    none = dict(q=None, k=None, v=None, g=None, beta=None, do=None, dq=None, dk=None, dv=None, dg=None, dbeta=None, saved=None, ws=None, N=0, n_seq=0)
    assert delta_bwd(**none) == 0
    for bad in SHARED + (dict(do=None), dict(lddo=15), dict(dq=None), dict(lddq=7), dict(dk=None), dict(lddk=7), dict(dv=None), dict(lddv=15), dict(dg=None), dict(lddg=3), dict(dbeta=None),
                         dict(lddb=3), dict(ds_last=P + 2), dict(ds0=P + 2)):
        assert delta_bwd(**bad) == -1, bad
    for bad in BEYOND:
        assert delta_bwd(**bad) == -2, bad
    held, need = B.dg_delta_rule_saved_bytes(6, 2, 4, 4, 4), B.dg_delta_rule_workspace_bytes(6, 2, 2, 4, 4, 4)
    for bad in (dict(saved=None), dict(saved_n=held - 1), dict(saved=P + 8), dict(ws=None), dict(n=need - 1), dict(ws=P + 4)):
        assert delta_bwd(**bad) == -3, bad


def test_sizes_of_what_is_kept():
    """What tokens write and a memory for each 64 of them and one more for each sequence; nothing grows with the square of the length."""
    marks, rows = (1000 // 64 + 3) * 4 * 32 * 16 * 4, 1000 * 4 * 16 * 4
    assert marks + rows <= B.dg_delta_rule_saved_bytes(1000, 3, 4, 32, 16) <= marks + rows + 64
    one, two = (B.dg_delta_rule_workspace_bytes(n, 1, 4, 4, 64, 64) for n in (1 << 20, 1 << 21))
    assert one < two < 2.1 * one


def test_the_most_rows():
    """Tokens are counted in steps of up to 64, in 32 bits.  (The last call lacks a workspace.)"""
    long = dict(n_seq=1, H=1, Hk=1)
    for N in ((1 << 32) - 1, (1 << 32) - 63):
        assert delta(N=N, **long) == -2 and delta_bwd(N=N, **long) == -2
    assert delta(N=(1 << 32) - 64, **long) == -3 and delta_bwd(N=(1 << 32) - 64, **long) == -3


def test_small_heads_need_no_room_for_chunks():
    """Heads that are taken token by token: what the gradient hands on (as much as is kept, and a number for each 64 tokens), and for the forward pass nothing."""
    for N, n_seq, Hk, H, D in ((65536 * 64, 65536, 2, 2, 16), ((1 << 20) * 64, 1 << 20, 2, 2, 16), (5000 * 30, 5000, 1, 3, 32), (3000, 1000, 2, 2, 8)):
        kept = B.dg_delta_rule_saved_bytes(N, n_seq, H, D, D)
        assert B.dg_delta_rule_workspace_bytes(N, n_seq, Hk, H, D, D) <= kept + (N // 64 + n_seq) * 4 + 64
        assert all(B.dg_delta_rule_fwd_least_workspace_bytes(N, n_seq, H, D, D, saves) == 0 for saves in (False, True))
        assert B.dg_delta_rule_fwd_workspace_bytes(N, n_seq, H) > 0                     # for any heads
    N, n_seq, H = 4000, 1000, 16                                                        # a few tokens
    assert B.dg_delta_rule_fwd_least_workspace_bytes(N, n_seq, H, 128, 128, False) == 0
    for shape in ((N, n_seq, H, 128, 128, True), (N + n_seq, n_seq, H, 128, 128, False), (64, 2, 2, 16, 16, False)):
        least = B.dg_delta_rule_fwd_least_workspace_bytes(*shape)
        assert 0 < least <= B.dg_delta_rule_fwd_workspace_bytes(*shape[:3]) and least < B.dg_delta_rule_workspace_bytes(*shape[:2], shape[2], *shape[2:5])


@pytest.mark.parametrize("call", [
    lambda x: B.dg_rms_norm_fwd(x, x[:, :4], None, 1e-5, None, x),
    lambda x: B.dg_rms_norm_fwd(x, None, None, 1e-5, None, x.half()),
    lambda x: B.dg_e4m3_rows(x, x.to(torch.float8_e4m3fn), torch.zeros(4, 2, dtype=torch.float8_e8m0fnu)),
    lambda x: B.dg_e4m3_product(x.to(torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.float8_e8m0fnu), x[:, :8].to(torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.float8_e8m0fnu), x),
    lambda x: B.dg_delta_rule_fwd(x, x, x, x[:, :3], x[:, :3], 3, 1, None, False, 1.0, None, x, None),
    lambda x: B.dg_delta_rule_fwd(x, x, x, x[:, :4].double(), x[:, :4], 4, 1, None, False, 1.0, None, x, None),
])
def test_binding_refuses_shapes_and_types(call):
    with pytest.raises(B.DistGridError):
        call(torch.zeros(4, 16))
