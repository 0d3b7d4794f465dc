"""Attention with a relative position bias against its definition in 64 bits: lengths from one key up, ragged tiles, key lengths down to none, causal
masks that leave queries without a key, bias tables of few and of many buckets, entries of -infinity, NaN behind a sample's keys.

Bounds are elementwise.  U = 2^-24; h = 2^-8 where probabilities, dS and outputs are rounded to bf16, U where they stay fp32.
  logits      d_head products and the bias are added in fp32, scaled, and taken relative to a reference or to lse: off by at most
              e = (d_head + 32) U (scale |q| |k| + |bias| + |lse| + 1), which is the relative error of exp (the hardware's own 2 U are in the 32)
  o           sum over keys of P (h + 2 e + 2 average(e) + n U) |v|, and its own rounding
  lse         2 average(e) + (n + 64) U
  dS          P ((d_head + 8) U (|dO| |V| + |dO| |O|)) + 2 e |dS|
  dq, dk, dv  sums of (h |dS| or h P, the above, and n U for the additions), and their own rounding
  dtable      the sum of the errors of dS, and (2 (nq + nk) + 200) U of its magnitudes: at most nq + nk additions into one place, then the joining.
"""
import numpy as np
import pytest

from oracle import training_ops as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _make(dtype, B, H, nq, nk, d, seed, n_buckets, lens, gain=1.0, pad=0):
    """Device tensors (rows H * d + pad apart, NaN between them and behind the keys of a sample) and 64-bit values [B, H, n, d]."""
    import torch
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    g = np.random.default_rng(seed)
    dev, val = {}, {}
    for name, n, std in (("q", nq, gain), ("k", nk, 1.0), ("v", nk, 1.0), ("do", nq, 1.0)):
        x = torch.full((B, n, H * d + pad), float("nan"), dtype=t, device="cuda")
        x[:, :, :H * d] = torch.from_numpy(g.normal(0, std, size=(B, n, H * d))).to(t).cuda()
        w = x[:, :, :H * d].double().cpu().numpy().reshape(B, n, H, d).transpose(0, 2, 1, 3).copy()
        if name in "kv" and lens is not None:
            for b, m in enumerate(lens):
                x[b, max(m, 0):] = float("nan")
                w[b, :, max(m, 0):] = 0.0
        dev[name], val[name] = x, w
    table = torch.from_numpy(g.normal(0, 1.5, size=(n_buckets, H))).to(t).cuda()
    return t, dev, val, table, table.double().cpu().numpy()


def _close(got, want, bound, what):
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), (what, float((err / np.maximum(bound, 1e-300)).max()), np.unravel_index((err - bound).argmax(), err.shape))


def _check(dtype, B, H, nq, nk, d, causal, bidirectional, n_buckets, distance, query0, lens, gain=1.0, pad=0, forbid=(), garbage={}, workspace=True, seed=0, forbidden=-float("inf"), unseen=False):
    import torch
    from paper_2405_01248_amd import binding as K
    held = [query0 + nq] * B if unseen else lens      # (unseen: NaN in what the causal mask hides from all queries)
    t, dev, val, table, tv = _make(dtype, B, H, nq, nk, d, seed + nq * 31 + nk, n_buckets, held, gain, pad)
    for bk in forbid:
        table[bk] = forbidden
        tv[bk] = -np.inf
    for bk, x in garbage.items():      # buckets whose pairs are all masked
        table[bk] = x
        tv[bk] = 0.0
    dt, ld, scale = (K.DP_F32 if dtype == "f32" else K.DP_BF16), H * d + pad, 1.0 / np.sqrt(d)
    scale = float(np.float32(scale))
    key_len = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    bias = K.RelBias(table, n_buckets, distance, bidirectional, query0)
    out = lambda n: torch.full((B, n, ld), 7.0, dtype=t, device="cuda")  # noqa: E731
    o, dq, dk, dv = out(nq), out(nq), out(nk), out(nk)
    lse = torch.full((B, H, nq), 7.0, device="cuda")
    dtable = torch.full((n_buckets, H), 2.0, device="cuda")

    def ws(backward):
        n = K.op_attention_relbias_workspace_bytes(B, H, nq, nk, d, n_buckets, backward)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None

    def get(x):
        assert (x[:, :, H * d:].float() == 7.0).all()      # what lies between the rows is left as it was
        return x[:, :, :H * d].double().cpu().numpy().reshape(B, -1, H, d).transpose(0, 2, 1, 3)

    def fwd(oo, ll):
        K.op_attention_relbias_fwd(dt, B, H, nq, nk, d, causal, scale, dev["q"], ld, dev["k"], ld, dev["v"], ld, bias, key_len, oo, ld, ll, ws(False) if workspace else None)

    fwd(o, lse)
    torch.cuda.synchronize()
    bk = T.buckets(nq, nk, query0, n_buckets, distance, bidirectional)
    lens0 = None if lens is None else [min(max(m, 0), nk) for m in lens]
    args = (val["q"], val["k"], val["v"])
    wo, wlse = T.attention_relbias_fwd(*args, scale, tv, bk, causal, query0, lens0)
    n, h = nq + nk, (U if dtype == "f32" else 2.0 ** -8)
    with np.errstate(invalid="ignore"):
        s = T._logits(val["q"], val["k"], scale, tv, bk, causal, query0, lens0)
        P = np.exp(s - np.where(np.isneginf(wlse), 0.0, wlse)[..., None])
    mag = np.where(np.isneginf(s), 0.0, scale * (np.abs(val["q"]) @ np.abs(val["k"]).swapaxes(-1, -2)) + np.abs(np.where(np.isinf(tv), 0.0, tv)[bk]).transpose(2, 0, 1)[None])
    e = (d + 32) * U * (mag + np.where(np.isneginf(wlse), 0.0, np.abs(wlse))[..., None] + 1)
    avg = (P * e).sum(-1)
    _close(get(o), wo, h * np.abs(wo) + (P * (h + 2 * e + 2 * avg[..., None] + n * U)) @ np.abs(val["v"]) * (1 + h), "o")
    glse = lse.double().cpu().numpy()
    empty = np.isneginf(wlse)
    assert (np.isneginf(glse) == empty).all() and (get(o)[empty] == 0).all()
    _close(np.where(empty, 0, glse), np.where(empty, 0, wlse), 2 * avg + (n + 64) * U * (1 + np.where(empty, 0, np.abs(wlse))), "lse")
    o2 = out(nq)
    fwd(o2, None)
    assert torch.equal(o2, o)

    # backward, from o and lse as they were stored
    def bwd(q_, k_, v_, tab, accumulate):
        K.op_attention_relbias_bwd(dt, B, H, nq, nk, d, causal, scale, dev["q"], ld, dev["k"], ld, dev["v"], ld, bias, key_len, o, ld, lse, dev["do"], ld,
                                   q_, ld, k_, ld, v_, ld, tab, accumulate, ws(True))

    bwd(dq, dk, dv, dtable, False)
    torch.cuda.synchronize()
    ov, do = get(o), val["do"]
    wdq, wdk, wdv, wdt = T.attention_relbias_bwd(*args, ov, glse, do, scale, tv, bk, causal, query0, lens0)
    with np.errstate(invalid="ignore"):
        P = np.exp(s - np.where(empty, 0.0, glse)[..., None])
    dS = np.abs(P * (do @ val["v"].swapaxes(-1, -2) - (do * ov).sum(-1, keepdims=True)))
    E = P * ((d + 8) * U * (np.abs(do) @ np.abs(val["v"]).swapaxes(-1, -2) + (np.abs(do) * np.abs(ov)).sum(-1, keepdims=True))) + 2 * e * dS
    side = scale * ((h + n * U) * dS + (1 + h) * E)
    fin = (1 + h) if dtype == "bf16" else 1.0
    _close(get(dq), wdq, h * np.abs(wdq) + side @ np.abs(val["k"]) * fin, "dq")
    _close(get(dk), wdk, h * np.abs(wdk) + side.swapaxes(-1, -2) @ np.abs(val["q"]) * fin, "dk")
    _close(get(dv), wdv, h * np.abs(wdv) + (P * (h + 2 * e + n * U)).swapaxes(-1, -2) @ np.abs(do) * fin, "dv")
    per = (E + (2 * n + 200) * U * dS).sum(0)
    bound = np.stack([np.bincount(bk.ravel(), per[i].ravel(), n_buckets) for i in range(H)], 1)
    _close(dtable.double().cpu().numpy(), wdt, bound + U * np.abs(wdt), "dtable")
    if lens is not None:
        for b, m in enumerate(lens0):
            assert (get(dk)[b, :, m:] == 0).all() and (get(dv)[b, :, m:] == 0).all()
    # the same bits again, without the table and with its gradient added up
    q2, k2, v2, t2 = out(nq), out(nk), out(nk), dtable.clone()
    bwd(q2, k2, v2, t2, True)
    assert torch.equal(q2, dq) and torch.equal(k2, dk) and torch.equal(v2, dv) and torch.equal(t2, dtable + dtable)
    bwd(out(nq), out(nk), out(nk), None, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk,d,causal,bidirectional,n_buckets,distance,query0,lens", [
    (1, 1, 1, 1, 8, False, True, 4, 2, 0, None),
    (2, 3, 77, 77, 64, False, True, 32, 128, 0, [77, 13]),
    (2, 2, 130, 257, 40, False, True, 16, 64, 127, [257, 0]),        # a sample without keys
    (1, 2, 513, 513, 72, True, False, 32, 128, 0, None),
    (1, 1, 200, 64, 96, True, True, 4, 7, -70, None),                # 70 queries before the first key
    (3, 2, 1, 1000, 64, True, False, 32, 128, 999, [1000, 1, 517]),  # one new token each
    (2, 1, 5, 4097, 88, False, False, 32, 100, 4000, [4097, 2049]),
    (1, 2, 300, 300, 48, False, True, 320, 800, 0, None),            # more distances than a tile has
    (1, 1, 1100, 1100, 64, False, True, 64, 1024, 0, None),
    (1, 3, 700, 200, 80, True, False, 2, 2, 0, None),                # two buckets
    (2, 2, 63, 65, 24, True, False, 512, 1024, 5, [64, 66]),         # a length beyond the keys
    (1, 1, 128, 128, 64, True, True, 32, 128, 1000000, [100]),       # far behind all keys
    (1, 1, 640, 640, 64, False, True, 32, 128, -300, [-5]),          # a negative length: no keys
    (5, 7, 33, 31, 16, False, True, 8, 20, 0, [31, 30, 29, 1, 0]),
    (16, 20, 129, 130, 64, False, True, 32, 128, 0, None),
    (16, 12, 70, 300, 64, False, True, 32, 128, 100, [300] * 8 + [257] * 4 + [128, 129, 65, 0]),      # more key tiles than two a CU
    (16, 12, 66, 270, 40, False, False, 32, 128, 200, None),
    (2, 3, 90, 200, 96, False, True, 320, 800, 0, [200, 3]),         # few keys, more distances than LDS has room for beside them
    (2, 3, 520, 128, 88, False, True, 32, 128, 0, None),             # few keys, shares of the queries
    (3, 9, 384, 384, 64, True, True, 32, 128, 0, None),              # heads that do not go round the XCDs evenly
])
def test_against_the_definition(dtype, B, H, nq, nk, d, causal, bidirectional, n_buckets, distance, query0, lens):
    _check(dtype, B, H, nq, nk, d, causal, bidirectional, n_buckets, distance, query0, lens)


@pytest.mark.parametrize("d", [4, 12, 20, 36, 68, 92])
def test_fp32_head_widths(d):
    _check("f32", 2, 2, 45, 77, d, True, True, 16, 64, 40, [77, 50])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    """Keys and values of five samples, rows 2^17 elements apart, so that the last sample lies beyond 4 GiB: the same bits as from dense rows."""
    import torch
    from paper_2405_01248_amd import binding as K
    t, dt, n, ld = (torch.float32, K.DP_F32, 2100, 1 << 17) if dtype == "f32" else (torch.bfloat16, K.DP_BF16, 4096, 1 << 17)
    B, H, d, nq, nb = 5, 1, 64, 40, 32
    wide = torch.empty((B, n, ld), dtype=t, device="cuda")
    kv = torch.randn((B, n, 2 * d), device="cuda").to(t)
    wide[:, :, :2 * d] = kv
    q, do, table = torch.randn((B, nq, d), device="cuda").to(t), torch.randn((B, nq, d), device="cuda").to(t), torch.randn((nb, H), device="cuda").to(t)
    ws = torch.empty(K.op_attention_relbias_workspace_bytes(B, H, nq, n, d, nb, True), dtype=torch.uint8, device="cuda")
    wf = torch.empty(K.op_attention_relbias_workspace_bytes(B, H, nq, n, d, nb, False), dtype=torch.uint8, device="cuda")
    out = []
    for x, l in ((kv, 2 * d), (wide, ld)):
        g = torch.zeros_like(x)
        o, lse, dq, tab = torch.empty_like(q), torch.empty((B, H, nq), device="cuda"), torch.empty_like(q), torch.empty((nb, H), device="cuda")
        bias = K.RelBias(table, nb, 128, True, n - nq)
        K.op_attention_relbias_fwd(dt, B, H, nq, n, d, False, 0.125, q, d, x, l, x[:, :, d:], l, bias, None, o, d, lse, wf)
        K.op_attention_relbias_bwd(dt, B, H, nq, n, d, False, 0.125, q, d, x, l, x[:, :, d:], l, bias, None, o, d, lse, do, d, dq, d, g, l, g[:, :, d:], l, tab, False, ws)
        out.append([o, lse, dq, tab, g[:, :, :2 * d].clone()])
        del g
    for a, b in zip(*out):
        assert torch.equal(a, b)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_large_logits_and_forbidden_buckets(dtype):
    _check(dtype, 2, 3, 150, 190, 40, False, True, 32, 128, 20, [190, 77], pad=24)
    _check(dtype, 1, 2, 260, 260, 64, True, False, 32, 128, 0, None, gain=12.0)
    _check(dtype, 1, 2, 400, 400, 64, False, True, 32, 128, 0, None, gain=12.0)
    _check(dtype, 1, 2, 260, 300, 64, False, True, 32, 128, 0, None, forbid=(0, 3, 15, 31))      # -infinity: near, middle and both ends
    _check(dtype, 1, 2, 70, 70, 64, True, False, 8, 16, 0, [70], forbid=range(8))               # nothing is visible at all


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [-65536.0, -1e9, "lowest"])
def test_entries_that_mask_as_infinity_does(dtype, value):
    import torch
    lowest = torch.finfo(torch.float32 if dtype == "f32" else torch.bfloat16).min
    value = lowest if value == "lowest" else value
    _check(dtype, 1, 2, 260, 300, 64, False, True, 32, 128, 0, None, forbid=(0, 3, 15, 31), forbidden=value)
    _check(dtype, 2, 1, 150, 500, 40, False, True, 32, 128, 0, [500, 60], forbid=range(32), forbidden=value)      # nothing is visible at all


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,query0", [(1, 700, 331), (40, 1000, 500), (140, 200, 0), (300, 700, 77), (64, 256, -20), (5, 300, -5)])
def test_what_the_causal_mask_hides_from_all_queries_is_not_read(dtype, nq, nk, query0):
    _check(dtype, 2, 2, nq, nk, 64, True, False, 32, 128, query0, None, unseen=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [64, 300, 1000])
def test_anything_in_buckets_that_the_causal_mask_hides(dtype, n):
    # two directions of buckets under the causal mask: those of later keys hold infinities and NaN
    _check(dtype, 1, 2, n, n, 64, True, True, 32, 128, 0, [n - n // 3],
           garbage={k: v for k, v in zip(range(17, 32), [float("nan"), float("inf"), -float("inf")] * 5)})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(1, 3001), (32, 2500), (33, 700)])
def test_few_queries_without_a_workspace(dtype, nq, nk):
    _check(dtype, 2, 2, nq, nk, 64, True, False, 32, 128, nk - nq, [nk, nk // 3], workspace=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [
    (1, 3, 513, 513, 64, False, None), (1, 3, 513, 513, 64, True, None),                # shares of keys and of queries
    (1, 2, 70, 2100, 40, False, [1500]), (2, 1, 2050, 300, 96, True, [300, 7]),         # of one of them
    (1, 4, 1024, 1024, 80, True, [700]), (1, 5, 2048, 600, 48, False, [0]),             # shares that have nothing to do
    (1, 2, 600, 256, 64, False, None),                                                  # shares of the queries, all keys in a workgroup
    (1, 10, 900, 1000, 88, False, [777]), (2, 8, 1030, 1030, 72, True, [1030, 640]),    # the same with many rows to a workgroup
    (3, 6, 1100, 1100, 64, False, [1100, 1, 600]), (1, 40, 300, 290, 48, True, None),
    (1, 2, 30, 3000, 64, False, [2999]), (1, 2, 3000, 30, 40, False, None), (2, 12, 206, 206, 64, True, [206, 100]), (2, 3, 330, 300, 8, False, [0, 290])])
def test_gradients_in_shares(dtype, B, H, nq, nk, d, causal, lens):
    _check(dtype, B, H, nq, nk, d, causal, True, 32, 128, nk - nq if causal else 0, lens)


@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [
    (30, 12, 77, 77, 64, False, "some"), (7, 40, 130, 120, 96, True, None), (50, 8, 40, 33, 24, True, "some"), (9, 30, 64, 200, 72, False, "some"), (5, 60, 150, 256, 40, True, None),
    (1, 8, 1024, 77, 64, False, None), (2, 5, 2000, 128, 96, False, [128, 50]), (2, 6, 1500, 100, 40, True, None)])      # the last three: shares of the queries
def test_gradients_where_a_workgroup_has_all_keys(B, H, nq, nk, d, causal, lens):
    _check("bf16", B, H, nq, nk, d, causal, True, 32, 128, 0, [(nk * (i + 1)) // B for i in range(B)] if lens == "some" else lens)


@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [
    (1, 3, 1000, 2500, 64, True, None), (2, 2, 800, 2100, 88, False, [2100, 130]), (1, 1, 2200, 3000, 40, True, [2900]), (3, 4, 700, 2049, 64, True, [0, 1, 2049])])
def test_shares_of_the_keys(B, H, nq, nk, d, causal, lens):
    _check("bf16", B, H, nq, nk, d, causal, True, 32, 128, nk - nq if causal else 0, lens)
    _check("bf16", B, H, nq, nk, d, causal, True, 32, 128, -nq // 2 if causal else 50, lens, workspace=False, gain=6.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,d", [(300, 300, 96), (70, 500, 64), (500, 90, 72), (700, 260, 80), (33, 40, 96)])
@pytest.mark.parametrize("n_buckets,distance", [(320, 800), (512, 1024)])
def test_bias_of_many_distances(dtype, nq, nk, d, n_buckets, distance):
    _check(dtype, 1, 2, nq, nk, d, False, True, n_buckets, distance, 0, None)      # (sums by distance take most of LDS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk,d", [(1, 8, 1024, 1024, 64), (1, 2, 2048, 4096, 40), (3, 5, 520, 256, 96), (2, 4, 100, 3000, 64), (1, 16, 1, 4000, 64), (4, 12, 77, 77, 64)])
def test_nothing_is_written_behind_the_workspace(dtype, B, H, nq, nk, d):
    import torch
    from paper_2405_01248_amd import binding as K
    ld, nb, t = H * d, 32, torch.float32 if dtype == "f32" else torch.bfloat16
    q, do, o, dq = (torch.randn((B, nq, ld), device="cuda").to(t) for _ in range(4))
    k, v, dk, dv = (torch.randn((B, nk, ld), device="cuda").to(t) for _ in range(4))
    table, lse, dtable = torch.randn((nb, H), device="cuda").to(t), torch.empty((B, H, nq), device="cuda"), torch.empty((nb, H), device="cuda")
    bias = K.RelBias(table, nb, 128, True, 0)
    for backward in (False, True):
        n = K.op_attention_relbias_workspace_bytes(B, H, nq, nk, d, nb, backward)
        whole = torch.full((n + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        args = (K.DP_F32 if dtype == "f32" else K.DP_BF16, B, H, nq, nk, d, False, 0.125, q, ld, k, ld, v, ld, bias, None, o, ld, lse)
        if backward:
            K.op_attention_relbias_bwd(*args, do, ld, dq, ld, dk, ld, dv, ld, dtable, False, whole[:n])
        else:
            K.op_attention_relbias_fwd(*args, whole[:n] if n else None)
        assert (whole[n:] == 0x5A).all()


def test_captured_passes_and_another_stream():
    import torch
    from paper_2405_01248_amd import binding as K
    B, H, n, d, nb = 3, 4, 200, 64, 32
    qkv = torch.randn((B, n, 3 * H * d), device="cuda").bfloat16()
    q, k, v = (qkv[:, :, i * H * d:] for i in range(3))
    do, table = torch.randn((B, n, H * d), device="cuda").bfloat16(), torch.randn((nb, H), device="cuda").bfloat16()
    key_len = torch.tensor([200, 64, 0], dtype=torch.int32, device="cuda")

    def buffers():
        return {"o": torch.empty_like(do), "lse": torch.empty((B, H, n), device="cuda"), "dqkv": torch.empty_like(qkv), "dt": torch.empty((nb, H), device="cuda"),
                "ws": torch.empty(K.op_attention_relbias_workspace_bytes(B, H, n, n, d, nb, True), dtype=torch.uint8, device="cuda")}

    def step(b):
        bias, ld, hd = K.RelBias(table, nb, 128, True, 0), 3 * H * d, H * d
        K.op_attention_relbias_fwd(K.DP_BF16, B, H, n, n, d, False, 0.125, q, ld, k, ld, v, ld, bias, key_len, b["o"], hd, b["lse"], None)
        g = [b["dqkv"][:, :, i * hd:] for i in range(3)]
        K.op_attention_relbias_bwd(K.DP_BF16, B, H, n, n, d, False, 0.125, q, ld, k, ld, v, ld, bias, key_len, b["o"], hd, b["lse"], do, hd, g[0], ld, g[1], ld,
                                   g[2], ld, b["dt"], False, b["ws"])

    cap, eager, other = buffers(), buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cap)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cap)
    for i in range(3):
        qkv.normal_()
        key_len[1] = 64 + 50 * i
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):      # beside the others, with a workspace of its own
            step(other)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for name in ("o", "lse", "dqkv", "dt"):
            assert torch.equal(cap[name], eager[name]) and torch.equal(other[name], eager[name]), name
