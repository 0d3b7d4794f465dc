"""The dropout, LayerNorm and relative-bias attention operators together, as a trained sub-layer runs them: LayerNorm, projections, attention with a
relative position bias over padded samples, output projection, dropout onto the residual stream, LayerNorm; and all of its gradients.

Tolerances.  fp32: five operations in a row, each a sum of at most 200 products, 200 x 2^-24 of its magnitudes, which a result's largest element exceeds at
most eightfold: 5 x 200 x 2^-24 x 8 = 5e-4 of the largest element.  bf16: at most ten roundings of tensors between the inputs and a result, each at most 2^-8 of
the tensor, passed on with a gain of at most one by normalised tensors: a relative error in the mean square of at most 10 x 2^-8.
"""
import numpy as np
import pytest

from oracle import training_ops as T

pytestmark = pytest.mark.gpu

B, N, H, D = 3, 70, 4, 48
W = H * D
LENS, P, SEED, STEP, SITE, NB, FAR = [70, 33, 1], 0.2, 99, 5, 3, 16, 40


def _inputs(seed=0):
    g = np.random.default_rng(seed)
    n = lambda *s, std=1.0, mean=0.0: g.normal(mean, std, size=s)  # noqa: E731
    return {"x": n(B * N, W, std=1.5, mean=0.2), "g1": n(W, std=0.2, mean=1.0), "b1": n(W, std=0.2), "wqkv": n(3 * W, W, std=W ** -0.5), "table": n(NB, H),
            "wo": n(W, W, std=W ** -0.5), "bo": n(W, std=0.1), "g2": n(W, std=0.2, mean=1.0), "b2": n(W, std=0.2), "gy": n(B * N, W), "gs": n(B * N, W)}


def _heads(x):
    return x.reshape(-1, N, H, D).transpose(0, 2, 1, 3)


def _rows(x):
    return x.transpose(0, 2, 1, 3).reshape(-1, W)


def _oracle(v, lens=LENS, first_row=0):
    """Outputs and gradients of sum(y gy) + sum(s gs)."""
    scale, bk = float(np.float32(D ** -0.5)), T.buckets(N, N, 0, NB, FAR, True)
    n, m1, r1 = T.layernorm_fwd(v["x"], v["g1"], v["b1"], 1e-5)
    qkv = n @ v["wqkv"].T
    q, k, w = (_heads(qkv[:, i * W:(i + 1) * W]) for i in range(3))
    o, lse = T.attention_relbias_fwd(q, k, w, scale, v["table"], bk, False, 0, lens)
    a = _rows(o) @ v["wo"].T + v["bo"]
    keep = T.keep_mask(len(a), W, P, SEED, STEP, SITE, first_row)
    s = v["x"] + T.dropout(a, keep, P)
    y, m2, r2 = T.layernorm_fwd(s, v["g2"], v["b2"], 1e-5)
    ds, dg2, db2 = T.layernorm_bwd(v["gy"], s, m2, r2, v["g2"])
    ds = ds + v["gs"]
    da = T.dropout(ds, keep, P)
    do = da @ v["wo"]
    dq, dk, dv, dt = T.attention_relbias_bwd(q, k, w, o, lse, _heads(do), scale, v["table"], bk, False, 0, lens)
    dqkv = np.concatenate([_rows(dq), _rows(dk), _rows(dv)], 1)
    dx, dg1, db1 = T.layernorm_bwd(dqkv @ v["wqkv"], v["x"], m1, r1, v["g1"])
    return {"y": y, "s": s, "x": dx + ds, "g1": dg1, "b1": db1, "wqkv": dqkv.T @ n, "table": dt, "wo": da.T @ _rows(o), "g2": dg2, "b2": db2}


def _device(v, dtype, lens=LENS, first_row=0, grads=None):
    """The same on the GPU; grads: fp32 gradients of the parameters to add to."""
    import torch
    from paper_2405_01248_amd import binding as K
    t, dt = (torch.float32, K.DP_F32) if dtype == "f32" else (torch.bfloat16, K.DP_BF16)
    c = {n: torch.from_numpy(x).to(t).cuda() for n, x in v.items()}
    rows, batch, f32 = len(v["x"]), len(lens), torch.float32
    e = lambda *s, d=t: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
    acc = grads is not None
    grads = grads or {n: e(*v[n].shape, d=f32) for n in ("g1", "b1", "wqkv", "table", "wo", "g2", "b2")}
    rng, key_len = torch.tensor([SEED, STEP], dtype=torch.int64, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    n, m1, r1, qkv, o, lse, a = e(rows, W), e(rows, d=f32), e(rows, d=f32), e(rows, 3 * W), e(rows, W), e(batch, H, N, d=f32), e(rows, W)
    s, y, m2, r2 = e(rows, W, d=f32), e(rows, W), e(rows, d=f32), e(rows, d=f32)
    bias, scale = K.RelBias(c["table"], NB, FAR, True, 0), D ** -0.5
    parts = lambda x: [x[:, i * W:] for i in range(3)]  # noqa: E731
    x32 = c["x"].float()      # the residual stream
    K.op_layernorm_fwd(dt, False, rows, W, 1e-5, c["x"], W, None, 0, 0.0, None, 0, 0, c["g1"], c["b1"], None, 0, n, W, m1, r1)
    K.op_gemm(dt, n, W, 0, c["wqkv"], W, 0, rows, 3 * W, W, None, qkv, 3 * W)
    q, k, w = parts(qkv)
    K.op_attention_relbias_fwd(dt, batch, H, N, N, D, False, scale, q, 3 * W, k, 3 * W, w, 3 * W, bias, key_len, o, W, lse, None)
    K.op_gemm(dt, o, W, 0, c["wo"], W, 0, rows, W, W, c["bo"], a, W)
    K.op_layernorm_fwd(dt, True, rows, W, 1e-5, a, W, x32, W, P, rng, SITE, first_row, c["g2"], c["b2"], s, W, y, W, m2, r2)
    ws = e(max(K.op_layernorm_bwd_workspace_bytes(rows, W), K.op_attention_relbias_workspace_bytes(batch, H, N, N, D, NB, True)), d=torch.uint8)
    ds, da, do, dqkv, dn, dx = e(rows, W, d=f32), e(rows, W), e(rows, W), e(rows, 3 * W), e(rows, W), e(rows, W, d=f32)
    K.op_layernorm_bwd(dt, True, rows, W, c["gy"], W, s, W, m2, r2, c["g2"], c["gs"].float(), W, P, rng, SITE, first_row, ds, W, da, W, grads["g2"], grads["b2"], acc, ws)
    K.op_gemm(dt, da, W, 0, c["wo"], W, 1, rows, W, W, None, do, W)
    K.op_gemm(dt, da, W, 1, o, W, 1, W, W, rows, None, grads["wo"], W, True, acc)
    dq, dk, dv = parts(dqkv)
    K.op_attention_relbias_bwd(dt, batch, H, N, N, D, False, scale, q, 3 * W, k, 3 * W, w, 3 * W, bias, key_len, o, W, lse, do, W, dq, 3 * W, dk, 3 * W, dv, 3 * W,
                               grads["table"], acc, ws)
    K.op_gemm(dt, dqkv, 3 * W, 0, c["wqkv"], W, 1, rows, W, 3 * W, None, dn, W)
    K.op_gemm(dt, dqkv, 3 * W, 1, n, W, 1, 3 * W, W, rows, None, grads["wqkv"], W, True, acc)
    K.op_layernorm_bwd(dt, True, rows, W, dn, W, x32, W, m1, r1, c["g1"], ds, W, 0.0, None, 0, 0, dx, W, None, 0, grads["g1"], grads["b1"], acc, ws)
    torch.cuda.synchronize()
    return {"y": y, "s": s, "x": dx, **grads}


def _as_given(v, dtype):
    """The values that the device gets."""
    import torch
    return {n: torch.from_numpy(x).to(torch.float32 if dtype == "f32" else torch.bfloat16).double().numpy() for n, x in v.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_and_gradients(dtype):
    v = _as_given(_inputs(), dtype)
    want, got = _oracle(v), _device(v, dtype)
    for n, w in want.items():
        err = got[n].double().cpu().numpy() - w
        if dtype == "f32":
            assert np.abs(err).max() <= 5e-4 * np.abs(w).max(), (n, np.abs(err).max() / np.abs(w).max())
        else:
            assert np.linalg.norm(err) <= 10 * 2.0 ** -8 * np.linalg.norm(w), (n, np.linalg.norm(err) / np.linalg.norm(w))


def test_gradients_against_differences():
    """Along random directions of every input: differences of the loss in 64 bits (step 1e-4, relative error of its third order far below) and the device's fp32
    gradient, whose elements are off by at most 5e-4 of the largest."""
    v = _as_given(_inputs(1), "f32")
    got = _device(v, "f32")
    loss = lambda u: (lambda r: (r["y"] * v["gy"]).sum() + (r["s"] * v["gs"]).sum())(_oracle(u))  # noqa: E731
    g = np.random.default_rng(2)
    for n in ("x", "g1", "b1", "wqkv", "table", "wo", "g2", "b2"):
        d = g.normal(size=v[n].shape)
        grad = got[n].double().cpu().numpy()
        h = 1e-4
        slope = (loss({**v, n: v[n] + h * d}) - loss({**v, n: v[n] - h * d})) / (2 * h)
        assert abs(slope - (grad * d).sum()) <= 5e-4 * np.abs(grad).max() * np.abs(d).sum() / np.sqrt(d.size), n


def test_slices_of_the_batch_give_the_whole():
    """Samples one by one, with their own numbers of rows: they drop what the whole batch drops, and the parameters' gradients add up."""
    import torch
    v = _as_given(_inputs(3), "f32")
    whole, grads, ys, xs = _device(v, "f32"), None, [], []
    for b in range(B):
        part = {n: (x[b * N:(b + 1) * N] if n in ("x", "gy", "gs") else x) for n, x in v.items()}
        r = _device(part, "f32", LENS[b:b + 1], b * N, grads)
        grads = {n: r[n] for n in ("g1", "b1", "wqkv", "table", "wo", "g2", "b2")}
        ys.append(r["y"])
        xs.append(r["x"])
    assert torch.allclose(torch.cat(ys), whole["y"], rtol=0, atol=5e-4 * float(whole["y"].abs().max()))
    assert torch.allclose(torch.cat(xs), whole["x"], rtol=0, atol=5e-4 * float(whole["x"].abs().max()))
    for n, x in grads.items():
        assert torch.allclose(x, whole[n], rtol=0, atol=5e-4 * float(whole[n].abs().max())), n
