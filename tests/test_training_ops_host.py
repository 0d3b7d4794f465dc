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
    for d in (1, 16, 200, 640, 1001, 1280, 2048, 4096, 5000, 8192):
        sizes = [lib.dp_op_layernorm_bwd_workspace_bytes(n, d) for n in (1, 2, 17, 255, 1000, 1023, 1024, 1025, 2047, 2048, 4097, 100000)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_attention_refusals(lib):
    from paper_2405_01248_amd import binding as K

    def need(backward=1, B=2, H=2, nq=64, nk=64, d=64, nb=32):
        return lib.dp_op_attention_relbias_workspace_bytes(B, H, nq, nk, d, nb, backward)

    def args(a, bwd):
        bias = K.RelBias(a.pop("table", P), a.pop("nb", 32), a.pop("far", 128), a.pop("both", 1), a.pop("q0", 0))
        bias = None if a.pop("no_bias", False) else C.byref(bias)
        ld = a.pop("ld", 128)
        g = lambda n, default=P: _vp(a.pop(n, default))  # noqa: E731
        l = lambda n: a.pop("ld" + n, ld)  # noqa: E741, E731
        head = [a.pop("dtype", 1), a.pop("B", 2), a.pop("H", 2), a.pop("nq", 64), a.pop("nk", 64), a.pop("d", 64), 0, C.c_float(a.pop("scale", 0.125)),
                g("q"), l("q"), g("k"), l("k"), g("v"), l("v"), bias, g("lens", 0)]
        if bwd:
            out = head + [g("o"), l("o"), g("lse"), g("do"), l("do"), g("dq"), l("dq"), g("dk"), l("dk"), g("dv"), l("dv"), g("dt"), 0, g("ws"), a.pop("wsb", need()), None]
        else:
            out = head + [g("o"), l("o"), g("lse"), g("ws", 0), a.pop("wsb", 0), None]
        assert not a, a
        return out

    fwd = lambda **a: lib.dp_op_attention_relbias_fwd(*args(a, False))  # noqa: E731
    bwd = lambda **a: lib.dp_op_attention_relbias_bwd(*args(a, True))  # noqa: E731
    for call in (fwd, bwd):
        for n in ("B", "H", "nq", "nk", "d"):
            assert call(**{n: 0}) == EINVAL and call(**{n: -1}) == EINVAL
        assert call(dtype=2) == EINVAL and call(no_bias=True) == EINVAL and call(table=0) == EINVAL and call(table=OFF) == EALIGN
        assert call(scale=0.0) == EINVAL and call(scale=NAN) == EINVAL and call(scale=-1.0) == EINVAL and call(scale=1e-7) == EUNSUPPORTED and call(scale=1e7) == EUNSUPPORTED
        assert call(d=104, ld=208) == EUNSUPPORTED and call(d=60, ld=120) == EUNSUPPORTED and call(dtype=0, d=62) == EUNSUPPORTED
        assert call(ld=132) == EUNSUPPORTED and call(ld=120) == EINVAL and call(dtype=0, ld=130) == EUNSUPPORTED
        assert call(nb=1) == EINVAL and call(nb=33) == EINVAL and call(nb=2) == EINVAL and call(nb=514) == EUNSUPPORTED and call(far=1025) == EUNSUPPORTED
        assert call(far=8) == EINVAL and call(far=16, both=0) == EINVAL and call(far=0) == EINVAL
        assert call(q0=(1 << 29) + 1) == EUNSUPPORTED and call(q0=-(1 << 29) - 1) == EUNSUPPORTED
        assert call(nk=1 << 23) == EUNSUPPORTED and b"2 GiB" in lib.dp_last_error()
        assert call(B=256, H=256, ld=1 << 14) == EUNSUPPORTED
        assert call(lens=P + 2) == EALIGN and call(lse=OFF) == EALIGN
        for n in ("q", "k", "v", "o"):
            assert call(**{n: 0}) == EINVAL and call(**{n: OFF}) == EALIGN and call(**{"ld" + n: 120}) == EINVAL
    for n in ("do", "dq", "dk", "dv"):
        assert bwd(**{n: 0}) == EINVAL and bwd(**{n: OFF}) == EALIGN and bwd(**{"ld" + n: 120}) == EINVAL
    assert bwd(lse=0) == EINVAL and bwd(dt=OFF) == EALIGN and bwd(ws=0) == EINVAL and bwd(ws=P + 64) == EALIGN
    assert bwd(wsb=need() - 1) == EWORKSPACE
    assert need(B=0) == 0 and need(nb=0) == 0


def test_attention_workspace_serves_smaller_batches(lib):
    for backward in (0, 1):
        sizes = [lib.dp_op_attention_relbias_workspace_bytes(b, 12, 300, 300, 64, 32, backward) for b in range(1, 40)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_attention_workspace_serves_all_smaller_sizes(lib):
    import random
    r = random.Random(4)
    size = lambda n: r.choice([1, r.randrange(1, 64), r.randrange(1, 600), r.randrange(1, 5000)]) if n else r.randrange(1, 70)  # noqa: E731
    for _ in range(20000):
        h, d, nb = r.choice([1, 3, 8, 12, 16]), r.choice([8, 40, 64, 96]), r.choice([2, 32, 320])
        big = [size(0), size(1), size(1)]
        small = [r.randrange(1, n + 1) if r.random() < 0.5 else n for n in big]
        for backward in (0, 1):
            a, b = (lib.dp_op_attention_relbias_workspace_bytes(x[0], h, x[1], x[2], d, nb, backward) for x in (small, big))
            assert a <= b, (small, big, h, d, nb, backward)


def test_bucket_refusals(lib):
    from paper_2405_01248_amd import binding as K
    for bad in ((1, 128, 0), (0, 128, 0), (-4, 128, 0), (33, 128, 1), (2, 128, 1), (32, 16, 0), (32, 8, 1), (513, 1024, 0), (32, 1025, 1)):
        assert lib.dp_relative_bucket(*bad, 5) < 0
        with pytest.raises(K.DpipeError):
            K.relative_bucket(*bad, 5)
    assert lib.dp_relative_bucket(32, 128, 1, 0) == 0 and lib.dp_relative_bucket(32, 128, 1, -(2 ** 31)) == 15 and lib.dp_relative_bucket(32, 128, 0, 7) == 0


def test_buckets_agree_with_the_definition(lib):
    from oracle import training_ops as T
    for n, far, both in ((32, 128, True), (32, 128, False), (16, 64, True), (64, 256, True), (32, 100, False), (320, 800, True), (512, 1024, False), (4, 2, True), (2, 1024, False), (14, 27, True)):
        for dist in list(range(-1100, 1101)) + [-2 ** 31, 2 ** 31 - 1, -(2 ** 31) + 1]:
            assert lib.dp_relative_bucket(n, far, int(both), dist) == T.bucket(dist, n, far, both), (n, far, both, dist)
