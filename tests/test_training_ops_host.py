"""Refusals of the dropout, LayerNorm and relative-bias attention calls, on the host: nothing is launched (no GPU needed)."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2405_01248_amd as dp
    if not os.path.exists(dp.library_path()):
        from paper_2405_01248_amd import build
        build.build(verbose=False)
    return dp.load_library()


P, OFF, NAN = 0x10000, 0x10008, float("nan")
EINVAL, EUNSUPPORTED, EWORKSPACE, EALIGN = -1, -2, -3, -4


def _vp(v):
    return C.c_void_p(v) if v else None


def test_dropout_refusals(lib):
    def call(dtype=1, rows=4, cols=16, x=P, ldx=16, r=P, ldr=16, p=0.5, rng=P, y=P, ldy=16):
        return lib.dp_op_dropout(dtype, rows, cols, _vp(x), ldx, _vp(r), ldr, C.c_float(p), _vp(rng), 0, 0, _vp(y), ldy, None)
    assert call(rows=0) == 0
    assert call(dtype=2) == EINVAL and call(rows=-1) == EINVAL and call(cols=0) == EINVAL
    assert call(x=0) == EINVAL and call(y=0) == EINVAL
    assert call(ldx=15) == EINVAL and call(ldr=15) == EINVAL and call(ldy=15) == EINVAL
    assert call(x=OFF) == EALIGN and call(y=OFF) == EALIGN and call(r=OFF) == EALIGN and call(rng=P + 4) == EALIGN
    assert call(p=-0.1) == EINVAL and call(p=1.1) == EINVAL and call(p=NAN) == EINVAL
    assert call(rng=0) == EINVAL and b"generator" in lib.dp_last_error()
    assert call(rows=2 ** 31 - 1, cols=2 ** 31 - 1, ldx=2 ** 31 - 1, ldy=2 ** 31 - 1, ldr=2 ** 31 - 1) == EUNSUPPORTED


def test_layernorm_refusals(lib):
    def fwd(dtype=1, rows=4, d=16, eps=1e-5, x=P, ldx=16, r=P, ldr=16, p=0.5, rng=P, gamma=P, beta=P, s=P, lds=16, y=P, ldy=16, mean=P, rstd=P):
        return lib.dp_op_layernorm_fwd(dtype, 1, rows, d, C.c_float(eps), _vp(x), ldx, _vp(r), ldr, C.c_float(p), _vp(rng), 0, 0, _vp(gamma), _vp(beta),
                                       _vp(s), lds, _vp(y), ldy, _vp(mean), _vp(rstd), None)
    assert fwd(rows=0) == 0
    assert fwd(dtype=-1) == EINVAL and fwd(rows=-1) == EINVAL and fwd(d=0) == EINVAL and fwd(d=8193, ldx=9000) == EUNSUPPORTED
    assert fwd(eps=0.0) == EINVAL and fwd(eps=NAN) == EINVAL and fwd(eps=float("inf")) == EINVAL
    assert fwd(gamma=0) == EINVAL and fwd(beta=0) == EINVAL and fwd(x=0) == EINVAL and fwd(y=0) == EINVAL and fwd(rng=0) == EINVAL
    for n in ("ldx", "ldr", "lds", "ldy"):
        assert fwd(**{n: 15}) == EINVAL
    for n in ("x", "r", "s", "y", "gamma", "beta", "mean", "rstd"):
        assert fwd(**{n: OFF}) == EALIGN

    need = lib.dp_op_layernorm_bwd_workspace_bytes(4, 16)
    assert need > 0 and lib.dp_op_layernorm_bwd_workspace_bytes(0, 16) == 0 and lib.dp_op_layernorm_bwd_workspace_bytes(4, 8193) == 0

    def bwd(dtype=1, rows=4, d=16, dy=P, lddy=16, s=P, lds=16, mean=P, rstd=P, gamma=P, di=P, ldi=16, p=0.5, rng=P, ds=P, ldds=16, dx=P, lddx=16, dg=P, db=P,
            ws=P, wsb=need):
        return lib.dp_op_layernorm_bwd(dtype, 1, rows, d, _vp(dy), lddy, _vp(s), lds, _vp(mean), _vp(rstd), _vp(gamma), _vp(di), ldi, C.c_float(p), _vp(rng), 0, 0,
                                       _vp(ds), ldds, _vp(dx), lddx, _vp(dg), _vp(db), 0, _vp(ws), wsb, None)
    assert bwd(rows=0, dg=0, db=0) == 0
    assert bwd(dtype=7) == EINVAL and bwd(rows=-1) == EINVAL and bwd(d=-1) == EINVAL and bwd(d=8193, lddy=9000) == EUNSUPPORTED
    for n in ("dy", "s", "mean", "rstd", "rng", "ws"):
        assert bwd(**{n: 0}) == EINVAL
    assert bwd(ds=0, dx=0) == EINVAL
    for n in ("lddy", "lds", "ldi", "ldds", "lddx"):
        assert bwd(**{n: 15}) == EINVAL
    for n in ("dy", "s", "mean", "rstd", "gamma", "di", "ds", "dx", "dg", "db"):
        assert bwd(**{n: OFF}) == EALIGN
    assert bwd(ws=P + 128) == EALIGN and bwd(wsb=need - 1) == EWORKSPACE and b"too small" in lib.dp_last_error()


def test_layernorm_workspace_serves_fewer_rows(lib):
    for d in (1, 16, 640, 1001, 8192):
        sizes = [lib.dp_op_layernorm_bwd_workspace_bytes(n, d) for n in (1, 2, 17, 255, 1000, 4097, 100000)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))
