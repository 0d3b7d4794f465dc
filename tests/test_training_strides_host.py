"""Row strides that the tile copies' 32-bit offsets do not hold are refused, on the host: nothing is launched (no GPU needed)."""
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


P, EUNSUPPORTED, EINVAL = 0x10000, -2, -1
NAMES = ("q", "k", "v", "o", "do", "dq", "dk", "dv")


def _call(lib, backward, dtype, n, ld):
    """One sample of one head, n rows; ld: row strides of some operands.  The workspace is left out (or too small), so that a call whose strides pass ends there."""
    from paper_2405_01248_amd import binding as K
    bias = K.RelBias(P, 32, 128, 1, 0)
    vp, f = C.c_void_p, C.c_float
    l = {name: ld.get(name, 64) for name in NAMES}  # noqa: E741
    head = [dtype, 1, 1, n, n, 64, 0, f(0.125), vp(P), l["q"], vp(P), l["k"], vp(P), l["v"], C.byref(bias), None, vp(P), l["o"]]
    if backward:
        return lib.dp_op_attention_relbias_bwd(*head, vp(P), vp(P), l["do"], vp(P), l["dq"], vp(P), l["dk"], vp(P), l["dv"], None, 0, None, 0, None)
    return lib.dp_op_attention_relbias_fwd(*head, vp(P + 4), None, 0, None)      # (lse off its alignment: the check behind those of the strides)


def test_strides_of_far_rows(lib):
    """A tile has up to 128 rows, whether they exist or not: the offset of the last, 127 strides of two bytes an element, must stay below 2^32, or rows that do
    not exist would be read from inside the sample."""
    far, ok = 1 << 24, (1 << 24) - 8
    assert 127 * 2 * ok + 2 * 64 < 1 << 32 < 127 * 2 * (far + (far >> 6)) + 2 * 64
    for n in (1, 2, 33, 60):
        for name in NAMES:
            assert _call(lib, True, 1, n, {name: far}) == EUNSUPPORTED, (n, name)
            assert name.replace("do", "d_o").encode() in lib.dp_last_error()
            assert _call(lib, True, 1, n, {name: ok}) == EINVAL and b"workspace" in lib.dp_last_error(), (n, name)
        for name in NAMES[:4]:
            assert _call(lib, False, 1, n, {name: far}) == EUNSUPPORTED, (n, name)
            assert _call(lib, False, 1, n, {name: ok}) == -4 and b"lse" in lib.dp_last_error(), (n, name)
    assert _call(lib, True, 0, 2, {"k": far}) == EINVAL and b"workspace" in lib.dp_last_error()      # fp32 rows go by 64-bit addresses
