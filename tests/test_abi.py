"""Host-only checks of the C ABI: the library loads, exports every declared symbol, validates
arguments, and its grid descriptor agrees with the oracle's geometry (no GPU needed)."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import dg_inputs as di
import oracle
from paper_2405_04416_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _declared():
    text = open(os.path.join(ROOT, "include", "distgrid.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(dg_[a-z0-9_]+)\s*\(", text)))


def test_library_exports_every_declared_symbol():
    names = _declared()
    assert len(names) >= 18
    handle = C.CDLL(B.LIB_PATH)
    for n in names:
        assert hasattr(handle, n), n
    assert set(B.EXPORTS) == set(names)


def test_peaks_library_exports_its_symbols():
    from paper_2405_04416_amd import peaks
    handle = C.CDLL(peaks.LIB_PATH)
    for n in peaks.EXPORTS:
        assert hasattr(handle, n), n


def test_no_oracle_in_product_path():
    pkg = os.path.join(ROOT, "paper_2405_04416_amd")
    for dirpath, _, files in os.walk(pkg):
        for f in files:
            if f.endswith((".py", ".hip", ".h", ".cpp")):
                src = open(os.path.join(dirpath, f)).read()
                assert "import oracle" not in src and "from oracle" not in src and "dgo_" not in src, f


@pytest.mark.parametrize("name", list(di.CONFIGS))
def test_grid_descriptor_matches_oracle_geometry(name):
    cfg = di.config(name)
    g = cfg["grid"]
    ext = di.box_extent(cfg["parts"][0])
    b_lib = g.get("growth") or B.dg_growth_factor(g["n_min"], g["n_max"], g["L"])
    b_ora = g.get("growth") or oracle.growth_factor(g["n_min"], g["n_max"], g["L"])
    desc = B.dg_grid_desc_init(g["L"], g["F"], g["log2_T"], g["n_min"], b_lib, ext)
    ref = oracle.grid_init(g["L"], g["F"], g["log2_T"], g["n_min"], b_ora, ext)
    assert desc.n_levels == ref.L and desc.n_entries == ref.n_entries
    for l in range(ref.L):
        assert desc.n_voxels[l] == ref.N[l]
        assert tuple(desc.res[l]) == tuple(ref.shape[l])
        assert desc.dense[l] == ref.is_dense[l]
        assert desc.offset[l] == ref.first[l]
        assert tuple(desc.scale[l]) == tuple(ref.gain[l])          # bit-identical fp32
    assert desc.offset[ref.L] == ref.first[ref.L]


def test_argument_validation_on_host():
    with pytest.raises(B.DistGridError):
        B.dg_grid_desc_init(17, 2, 19, 16, 1.3, [1, 1, 1])
    with pytest.raises(B.DistGridError):
        B.dg_grid_desc_init(4, 4, 19, 16, 1.3, [1, 1, 1])
    with pytest.raises(B.DistGridError):
        B.dg_grid_desc_init(4, 2, 19, 16, 1.3, [1, 0, 1])
    assert b"extent" in B.lib().dg_last_error()
    m = B.dg_mlp_desc(32, 64, 16, 16, 64, 2)
    assert B.dg_mlp_weight_count(m) == 64 * 32 + 16 * 64 + 64 * 32 + 64 * 64 + 3 * 64
    assert B.dg_mlp_weight_count(m) == oracle.mlp_weight_count(oracle.mlp_desc(32, 64, 16, 16, 64, 2))
    assert B.dg_segments_workspace_bytes(1000, 4) >= 4 * 4 * 4
    # null pointers with N = 0 are accepted, unsupported shapes are refused before any launch
    desc = B.dg_grid_desc_init(4, 2, 12, 16, 1.5, [1, 1, 1])
    assert B.lib().dg_hashgrid_encode_fwd(C.byref(desc), None, None, 0, None, 0, None) == 0
    assert B.lib().dg_hashgrid_encode_fwd(C.byref(desc), None, None, 5, None, 0, None) == -1
    bad = B.dg_mlp_desc(24, 64, 16, 16, 64, 2)
    assert B.lib().dg_mlp_fwd(C.byref(bad), None, None, None, 4, 0, None, None, None) == -2


def test_occupancy_host_side():
    for N, ext in [(512, (2.0, 2.0, 0.25)), (8, (4.0, 2.0, 1.0)), (10, (1.0, 1.0, 0.25)), (33, (0.7, 3.1, 1.9))]:
        desc, ref = B.dg_occ_desc_init(N, ext), oracle.occ_init(N, ext)
        assert tuple(desc.res) == tuple(ref.shape) and desc.n_cells == ref.n_cells
        assert tuple(desc.scale) == tuple(ref.gain)                     # bit-identical fp32
    for it in list(range(0, 40)) + [4095, 4096, 9999, 10000, 10016, 299999]:
        assert B.dg_occ_schedule(it) == oracle.occ_schedule(it)
    with pytest.raises(B.DistGridError):
        B.dg_occ_desc_init(0, [1, 1, 1])
    with pytest.raises(B.DistGridError):
        B.dg_occ_desc_init(8, [1, -1, 1])
    with pytest.raises(B.DistGridError):
        B.dg_occ_desc_init(2048, [1, 1, 1])                             # 2^33 cells
    desc = B.dg_occ_desc_init(8, [1, 1, 1])
    lib = B.lib()
    assert lib.dg_occ_candidates(C.byref(desc), None, 0, 0, 0, 0, 0, 0, 32, None, None, None) == 0
    assert lib.dg_occ_candidates(C.byref(desc), None, 510, 5, 0, 1, 0, 0, 32, None, None, None) == -1    # warm-up: candidate i is cell i
    assert lib.dg_occ_candidates(C.byref(desc), None, 0, 5, 0, 0, 0, 0, 65, None, None, None) == -1
    assert lib.dg_march_workspace_bytes(0) >= 4 and lib.dg_march_workspace_bytes(1 << 20) >= 4 * 513
    box = (C.c_float * 6)(0, 0, 0, 1, 1, 1)
    assert lib.dg_march_segments(None, None, None, None, None, 0, 1, box, C.byref(desc), None, 0.0, 10, 0, 0, None, None, None, None,
                                 None, None, None, 0, None) == -1          # dt must be positive
    assert lib.dg_march_segments(None, None, None, None, None, 0, 1, box, C.byref(desc), None, 0.1, 70000, 0, 0, None, None, None,
                                 None, None, None, None, 0, None) == -1    # the jitter counter has 16 bits for the stratum
    assert lib.dg_composite_ragged_fwd(None, None, None, 0, None, None, None, 1, None, None, None) == 0
    assert lib.dg_composite_ragged_fwd(None, None, None, 3, None, None, None, 1, None, None, None) == -1


def test_optimiser_host_side():
    # the schedule is a host function: same values as the oracle's (fp32 result of a double computation)
    for it in (0, 1, 1234, 150000, 299999, 300000, 10 ** 6):
        assert B.dg_cosine_lr(0.05, 0.005, it, 300000) == pytest.approx(oracle.cosine_lr(0.05, 0.005, it, 300000), rel=2e-7)
    L = B.lib()
    f = C.c_float
    args = lambda n, step, b1=0.9, eps=1e-15: (None, None, None, None, C.c_uint64(n), f(0.01), f(b1), f(0.99), f(eps), step, f(0.0), 1, None, None)
    assert L.dg_adam_step(*args(0, 1)) == 0                 # nothing to do
    assert L.dg_adam_step(*args(8, 1)) == -1                # null pointers
    assert b"null" in L.dg_last_error()


def test_bench_refuses_more_than_one_gpu():
    import subprocess
    import sys
    res = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--gpus", "2"], capture_output=True, text=True)
    assert res.returncode != 0 and "ONE GPU" in res.stderr


def _field_arguments(degree, n_dir, short_dW):
    """Arguments of the two one-call bindings for 3 segments of 5 samples, on host tensors."""
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    i32, f16 = torch.int32, torch.float16
    grid, mlp = B.dg_grid_desc_init(4, 2, 12, 16, 1.5, [1.0] * 3), B.dg_mlp_desc(8, 32, 16, n_dir, 32, 1)
    n_seg, S = 3, 5
    N, n_w = n_seg * S, B.dg_mlp_weight_count(mlp)
    common = (grid, mlp, 0, n_seg, S, degree, 0, z(n_seg, dt=i32), z(n_seg, dt=i32), 1, z(n_w, dt=f16), z(N, 3), z(N), z(n_seg, degree * degree, dt=f16),
              z(N, 8, dt=f16), z(N), z(N, 3))
    table, Ck, Tk, dW = z(grid.n_entries, 2), z(n_seg, 1, 3), z(n_seg, 1), z(n_w - short_dW)
    return ((common, [0.0] * 6, 1, z(n_seg, 3), z(n_seg, 3), z(n_seg, 1, 2), table, Ck, Tk),
            (common, 1.0, Ck, Tk, z(N), z(N, 3), z(N, 8), table, dW, (table, dW), z(64), z(64)))


@pytest.mark.parametrize("degree,n_dir,short_dW,refused", [(2, 4, 0, ()), (2, 16, 0, ("fwd", "bwd")), (3, 16, 0, ("fwd", "bwd")), (2, 4, 1, ("bwd",))])
def test_one_call_bindings_refuse_what_the_single_ones_refuse(degree, n_dir, short_dW, refused, monkeypatch):
    """Rows of the direction table shorter than the networks read them, a weight gradient shorter than the networks write it: the
    bindings dg_mlp_fwd_app and dg_mlp_bwd_app refuse both.  The launching calls are replaced, nothing runs."""
    real, launched = B.lib(), []

    class Stub:
        def __getattr__(self, name):
            if name in ("dg_field_fwd", "dg_field_bwd"):
                return lambda *a: launched.append(name[-3:]) or 0
            return getattr(real, name)

    fwd, bwd = _field_arguments(degree, n_dir, short_dW)
    monkeypatch.setattr(B, "lib", lambda: Stub())
    monkeypatch.setattr(B, "_ptr", lambda t, dtype=None, optional=False: t.data_ptr())
    monkeypatch.setattr(B, "_stream", lambda: 0)
    for way, call, args in (("fwd", B.dg_field_fwd, fwd), ("bwd", B.dg_field_bwd, bwd)):
        launched.clear()
        if way in refused:
            with pytest.raises(AssertionError):
                call(*args)
            assert not launched
        else:
            call(*args)
            assert launched == [way]


@pytest.mark.parametrize("name", ["dg_field_fwd", "dg_field_bwd"])
def test_one_call_refuses_short_direction_rows(name):
    """The library looks at it before all else (every pointer of the call is NULL, nothing could be launched)."""
    grid, mlp = B.dg_grid_desc_init(16, 2, 14, 16, 1.4, [1.0] * 3), B.dg_mlp_desc(32, 64, 16, 16, 64, 2)
    call = B.FieldCall(grid=C.addressof(grid), mlp=C.addressof(mlp), n_seg=3, S=5, k_max=1, degree=2)
    assert getattr(B.lib(), name)(C.byref(call), None) != 0
    assert b"direction inputs" in B.lib().dg_last_error()


def test_fused_rendering_refuses_split_features():
    """No entry point passes them; the function behind dg_mlp_composite_fwd has no kernel for them and says so instead of returning
    success (n_seg = 0 and NULL pointers: nothing could be launched)."""
    render = getattr(B.lib(), "_ZN2dg15mlp_mfma_renderEPKcPKvS3_NS_13FeatureLayoutES3_S3_jjjjPKfS6_PKjS8_jPfS9_S9_P12ihipStream_t")
    p, u = C.c_void_p, C.c_uint32
    render.restype, render.argtypes = C.c_int, [C.c_char_p, p, p, C.c_int, p, p, u, u, u, u, p, p, p, p, u, p, p, p, p]
    kSplit = 2
    assert render(b"views", None, None, kSplit, None, None, 0, 64, 0, 1, None, None, None, None, 1, None, None, None, None) != 0
    assert b"split" in B.lib().dg_last_error()


def test_sequence_block_host_side():
    """What the library refuses before it launches anything, and what it takes with nothing to do (all pointers NULL)."""
    L = B.lib()
    assert L.dg_layer_norm_fwd(None, 8, None, None, 0, 8, 1e-5, 0, None, 8, None) == 0
    assert L.dg_layer_norm_fwd(None, 8, None, None, 4, 8, 1e-5, 0, None, 8, None) == -1           # null pointer
    assert L.dg_layer_norm_fwd(None, 8, None, None, 0, 0, 1e-5, 0, None, 8, None) == -1           # W
    assert L.dg_layer_norm_fwd(None, 8, None, None, 0, 8, -1.0, 0, None, 8, None) == -1           # eps
    assert L.dg_layer_norm_fwd(None, 8, None, None, 0, 8, 1e-5, 3, None, 8, None) == -1           # type
    assert L.dg_layer_norm_fwd(256, 7, None, None, 4, 8, 1e-5, 0, 256, 8, None) == -1             # rows that overlap
    assert L.dg_layer_norm_fwd(258, 8, None, None, 4, 8, 1e-5, 0, 256, 8, None) == -1             # misaligned fp32
    assert L.dg_layer_norm_fwd(None, 8, None, None, 1 << 33, 8, 1e-5, 0, None, 8, None) == -2
    assert L.dg_layer_norm_bwd(None, 8, None, None, 8, 0, 8, 1e-5, 0, None, 8, None, None, None, 0, None) == 0
    assert L.dg_layer_norm_bwd(256, 8, None, 256, 8, 4, 8, 1e-5, 0, 256, 8, 256, None, None, 0, None) == -3       # no workspace
    assert L.dg_layer_norm_bwd_workspace_bytes(0, 8) <= 64 and L.dg_layer_norm_bwd_workspace_bytes(1 << 24, 32) <= 8 << 20
    rec = lambda N, n_seq, W, p=None, dtype=0, ld=8, first=None: L.dg_recurrence_fwd(p, ld, p, ld, N, n_seq, first, W, 0, dtype, None, p, ld, None, None, None, 0, None)
    assert rec(0, 0, 8) == 0
    assert rec(12, 5, 8, 256) == -1 and b"one length" in L.dg_last_error()
    assert rec(12, 0, 8, 256) == -1
    assert rec(12, 3, 8) == -1 and rec(12, 3, 0, 256) == -1 and rec(12, 3, 9, 256) == -1 and rec(12, 3, 8, 256, 7) == -1
    assert rec(1 << 32, 1, 8, 256) == -2
    assert L.dg_recurrence_bwd(256, 8, 256, 8, 12, 3, None, 8, 0, 0, None, None, 256, 8, None, 256, 8, 256, 8, None, None, 0, None) == -1     # no states
    assert L.dg_recurrence_state_count(0, 8) == 0 and L.dg_recurrence_state_count(33, 8) == 24
    assert L.dg_dropout_fwd(None, None, 0, 0.5, 1, 0, 0, None, None) == 0
    assert L.dg_dropout_fwd(None, None, 4, 0.5, 1, 0, 0, None, None) == -1
    for p in (-0.1, 1.1, float("nan")):
        assert L.dg_dropout_fwd(256, None, 0, p, 1, 0, 0, 256, None) == -1
        assert L.dg_dropout_bwd(256, 0, p, 1, 0, 0, 256, None) == -1


def test_sequence_block_limits():
    """Sizes beyond the stated limits are refused before anything is launched."""
    L = B.lib()
    assert L.dg_dropout_fwd(256, None, (1 << 40) + 1, 0.5, 1, 0, 0, 256, None) == -2 and b"2^40" in L.dg_last_error()
    assert L.dg_dropout_bwd(256, (1 << 40) + 1, 0.5, 1, 0, 0, 256, None) == -2
    rec = lambda N, n_seq, W: L.dg_recurrence_fwd(256, W, 256, W, N, n_seq, None, W, 0, 0, None, 256, W, None, None, None, 0, None)
    assert rec(0, (1 << 32) - 1, 65) == -2 and b"2^38" in L.dg_last_error()
    assert rec(1 << 31, 1 << 31, 257) == -2 and rec(1 << 31, 1 << 20, (1 << 20) + 1) == -2
    assert L.dg_layer_norm_fwd(256, 1 << 20, None, None, (1 << 19) + 1, 1 << 20, 1e-5, 0, 256, 1 << 20, None) == -2
    assert L.dg_layer_norm_fwd(256, (1 << 20) + 1, None, None, 1, (1 << 20) + 1, 1e-5, 0, 256, (1 << 20) + 1, None) == -2
