"""The backward of the attention with a relative position bias by the size of its table: the launches that it takes and records, and results against the definition."""
import pytest

from test_gpu_attention_relbias import _check

pytestmark = pytest.mark.gpu

DQ, DKV, REDUCE = "attn_bwd_dq", "attn_bwd_dkv", "reduce"


def _records(B, H, nq, nk, d, causal, n_buckets, distance, both, dtype="bf16"):
    """The records of a backward's launches."""
    import torch
    from paper_2405_01248_amd import binding as K
    ld = H * d
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    q, do, o, dq = (torch.randn((B, nq, ld), device="cuda").to(t) for _ in range(4))
    k, v, dk, dv = (torch.randn((B, nk, ld), device="cuda").to(t) for _ in range(4))
    table, lse, dtable = torch.randn((n_buckets, H), device="cuda").to(t), torch.zeros((B, H, nq), device="cuda"), torch.empty((n_buckets, H), device="cuda")
    ws = torch.empty(K.op_attention_relbias_workspace_bytes(B, H, nq, nk, d, n_buckets, True), dtype=torch.uint8, device="cuda")
    K.ktime_begin(64)
    K.op_attention_relbias_bwd(K.DP_F32 if dtype == "f32" else K.DP_BF16, B, H, nq, nk, d, causal, 0.125, q, ld, k, ld, v, ld, K.RelBias(table, n_buckets, distance, both, 0), None, o, ld, lse, do, ld,
                               dq, ld, dk, ld, dv, ld, dtable, False, ws)
    return K.ktime_end(64)


def _kinds(*args, **more):
    return [r["kind"] for r in _records(*args, **more)]


# One launch for all gradients where its workgroups all run at once: 512 with a table of 32 buckets to 128 distances (two a CU), 256 with one that leaves LDS for one.
@pytest.mark.parametrize("H,n,causal,small,large", [(16, 512, False, [DKV], [DQ, DKV]), (16, 512, True, [DKV], [DQ, DKV]), (8, 512, False, [DKV], [DKV]), (32, 512, False, [DQ, DKV], [DQ, DKV])])
def test_one_launch_where_its_workgroups_run_at_once(H, n, causal, small, large):
    for (n_buckets, distance), want in (((32, 128), small), ((64, 256), large)):
        kinds = _kinds(1, H, n, n, 64, causal, n_buckets, distance, not causal)
        assert [k for k in kinds if k in (DQ, DKV)] == want, (n_buckets, kinds)


# What is added up behind the kernels is a launch, and a record, of its own: parts of the table's gradient, shares of dQ, dK and dV (4 heads of 4096 are 512 workgroups of 32
# queries, two a CU, which leave none for shares; 6 are 192 of 128, in two shares).
@pytest.mark.parametrize("dtype,B,H,nq,nk,want", [("bf16", 1, 8, 512, 512, [DKV, REDUCE]), ("bf16", 1, 4, 4096, 4096, [DQ, DKV]), ("bf16", 1, 6, 4096, 4096, [DQ, DKV, REDUCE]), ("bf16", 8, 10, 300, 300, [DQ, DKV]),
                                                  ("bf16", 30, 10, 77, 77, [DKV, REDUCE]), ("bf16", 1, 8, 4096, 77, [DKV, REDUCE]), ("f32", 1, 8, 257, 257, ["attn_f32", REDUCE]),
                                                  ("f32", 2, 16, 512, 512, ["attn_f32"])])
def test_every_launch_is_recorded(dtype, B, H, nq, nk, want):
    assert _kinds(B, H, nq, nk, 64, False, 32, 128, True, dtype=dtype) == want


# Shares of the queries where a workgroup has all keys: no more workgroups than run at once, of which a CU holds two of up to 128 keys and width 64 with a table of 32 buckets to 128.
@pytest.mark.parametrize("H,nq,nk,d,n_buckets,distance,at_once", [(80, 2048, 77, 64, 32, 128, 512), (80, 2048, 77, 96, 32, 128, 256), (80, 2048, 77, 64, 64, 256, 256), (80, 1024, 200, 64, 32, 128, 256),
                                                                  (160, 1024, 250, 40, 32, 128, 256), (40, 4096, 77, 64, 32, 128, 512), (255, 1024, 77, 64, 32, 128, 512)])
def test_shares_of_the_queries_run_at_once(H, nq, nk, d, n_buckets, distance, at_once):
    main, join = _records(1, H, nq, nk, d, False, n_buckets, distance, True)
    assert main["kind"] == DKV and join["kind"] == REDUCE and join["n"] == 1
    shares, tiles = join["k"], (nq + 63) // 64
    each = -(-tiles // max(1, min(16, tiles // 2, at_once // H)))
    assert H * shares <= at_once and shares == -(-tiles // each), (shares, each)


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("B,H,nq,nk,d,causal", [(1, 16, 512, 512, 64, False), (1, 16, 512, 512, 64, True), (1, 12, 1000, 1000, 40, False), (1, 50, 300, 300, 64, False), (2, 10, 300, 250, 64, True), (4, 20, 700, 77, 64, False),
                                                (3, 8, 1024, 1024, 64, True), (1, 8, 2048, 2048, 64, False), (4, 18, 200, 200, 64, False), (3, 4, 520, 520, 88, False)])
def test_large_tables(B, H, nq, nk, d, causal, both):
    lens = [nk - i * nk // (B + 1) for i in range(B)]
    _check("bf16", B, H, nq, nk, d, causal, both, 64, 256, nk - nq, lens)


@pytest.mark.parametrize("both", [True, False])
@pytest.mark.parametrize("B,H,n", [(8, 10, 700), (9, 14, 300)])
def test_tables_that_leave_room_for_two_workgroups_a_cu(B, H, n, both):
    _check("bf16", B, H, n, n, 64, False, both, 512, 1024, 0, None)


# Every split of the backward and of the forward with tables whose end buckets, far sums and LDS differ from those of 32 buckets to 128 distances, queries without a key among them.
TABLES = [(64, 256, True), (64, 256, False), (512, 1024, False)]
TYPES = [("bf16", *table) for table in TABLES] + [("f32", 64, 256, False)]


def _offset(nq, nk, causal):
    return -(nq // 3) if causal else nk // 2 - 37      # (under the causal mask the first third sees nothing)


@pytest.mark.parametrize("dtype,n_buckets,distance,both", TYPES)
@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [
    (1, 3, 513, 513, 64, False, None), (1, 3, 513, 513, 64, True, None), (1, 2, 70, 2100, 40, False, [1500]), (2, 1, 2050, 300, 96, True, [300, 7]), (1, 4, 1024, 1024, 80, True, [700]),
    (1, 10, 900, 1000, 88, False, [777]), (2, 8, 1030, 1030, 72, True, [1030, 640]), (1, 6, 1500, 1500, 64, False, [1499]), (3, 6, 1100, 1100, 64, False, [1100, 1, 600]),
    (1, 2, 30, 3000, 64, False, [2999]), (1, 2, 3000, 30, 40, False, None), (2, 3, 330, 300, 8, True, [0, 290])])
def test_gradients_in_shares(dtype, n_buckets, distance, both, B, H, nq, nk, d, causal, lens):
    _check(dtype, B, H, nq, nk, d, causal, both, n_buckets, distance, _offset(nq, nk, causal), lens)


@pytest.mark.parametrize("n_buckets,distance,both", TABLES)
@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [
    (30, 12, 77, 77, 64, False, "some"), (7, 40, 130, 120, 96, True, None), (50, 8, 40, 33, 24, True, "some"), (9, 30, 64, 200, 72, False, "some"), (5, 60, 150, 256, 40, True, None),
    (2, 6, 1500, 100, 40, True, None), (2, 40, 1000, 250, 64, False, [250, 129])])
def test_gradients_where_a_workgroup_has_all_keys(n_buckets, distance, both, B, H, nq, nk, d, causal, lens):
    _check("bf16", B, H, nq, nk, d, causal, both, n_buckets, distance, _offset(nq, nk, causal), [(nk * (i + 1)) // B for i in range(B)] if lens == "some" else lens)


@pytest.mark.parametrize("n_buckets,distance,both", TABLES)
@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [(1, 3, 1000, 2500, 64, True, None), (2, 2, 800, 2100, 88, False, [2100, 130]), (3, 4, 700, 2049, 64, True, [0, 1, 2049]), (2, 8, 1, 4000, 64, False, [4000, 77])])
def test_shares_of_the_keys(n_buckets, distance, both, B, H, nq, nk, d, causal, lens):
    _check("bf16", B, H, nq, nk, d, causal, both, n_buckets, distance, _offset(nq, nk, causal), lens)


@pytest.mark.parametrize("dtype,n_buckets,distance,both", TYPES + [("bf16", 511, 1000, False)])
@pytest.mark.parametrize("B,H,nq,nk,d", [(1, 8, 1024, 1024, 64), (1, 2, 2048, 2500, 40), (3, 5, 520, 256, 96), (2, 40, 1000, 77, 64), (4, 12, 77, 77, 64)])
def test_nothing_is_written_behind_the_workspace(dtype, n_buckets, distance, both, B, H, nq, nk, d):
    import torch
    from paper_2405_01248_amd import binding as K
    ld, t = H * d, torch.float32 if dtype == "f32" else torch.bfloat16
    q, do, o, dq = (torch.randn((B, nq, ld), device="cuda").to(t) for _ in range(4))
    k, v, dk, dv = (torch.randn((B, nk, ld), device="cuda").to(t) for _ in range(4))
    table, lse, whole = torch.randn((n_buckets, H), device="cuda").to(t), torch.empty((B, H, nq), device="cuda"), torch.full((n_buckets * H + 4096,), 9.0, device="cuda")
    dtable = whole[:n_buckets * H].view(n_buckets, H)
    for backward in (False, True):
        n = K.op_attention_relbias_workspace_bytes(B, H, nq, nk, d, n_buckets, backward)
        ws = torch.full((n + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        args = (K.DP_F32 if dtype == "f32" else K.DP_BF16, B, H, nq, nk, d, False, 0.125, q, ld, k, ld, v, ld, K.RelBias(table, n_buckets, distance, both, 0), None, o, ld, lse)
        if backward:
            K.op_attention_relbias_bwd(*args, do, ld, dq, ld, dk, ld, dv, ld, dtable, False, ws[:n])
        else:
            K.op_attention_relbias_fwd(*args, ws[:n] if n else None)
        assert (ws[n:] == 0x5A).all() and (whole[n_buckets * H:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk", [(1, 6, 1500, 1500), (2, 20, 900, 77), (1, 4, 3, 3000)])
def test_captured_passes_and_another_stream(dtype, B, H, nq, nk):
    """Split passes with a table of one direction, replayed and beside the others on a second stream, each with buffers of its own."""
    import torch
    from paper_2405_01248_amd import binding as K
    d, nb, t, dt = 64, 64, torch.float32 if dtype == "f32" else torch.bfloat16, K.DP_F32 if dtype == "f32" else K.DP_BF16
    ld = H * d
    q, do = (torch.randn((B, nq, ld), device="cuda").to(t) for _ in range(2))
    kv, table = torch.randn((B, nk, 2 * ld), device="cuda").to(t), torch.randn((nb, H), device="cuda").to(t)
    key_len = torch.full((B,), nk, dtype=torch.int32, device="cuda")
    bias = K.RelBias(table, nb, 256, False, nk - nq - 20)

    def buffers():
        ws = [K.op_attention_relbias_workspace_bytes(B, H, nq, nk, d, nb, backward) for backward in (False, True)]
        return {"o": torch.empty_like(q), "lse": torch.empty((B, H, nq), device="cuda"), "dq": torch.empty_like(q), "dkv": torch.empty_like(kv), "dt": torch.empty((nb, H), device="cuda"),
                "ws": [torch.empty(n, dtype=torch.uint8, device="cuda") if n else None for n in ws]}

    def step(b):
        args = (dt, B, H, nq, nk, d, True, 0.125, q, ld, kv, 2 * ld, kv[:, :, ld:], 2 * ld, bias, key_len, b["o"], ld, b["lse"])
        K.op_attention_relbias_fwd(*args, b["ws"][0])
        K.op_attention_relbias_bwd(*args, do, ld, b["dq"], ld, b["dkv"], 2 * ld, b["dkv"][:, :, ld:], 2 * ld, b["dt"], False, b["ws"][1])

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
        kv.normal_()
        key_len[0] = nk - 500 * i if nk > 1000 else nk - 5 * i
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(other)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for name in ("o", "lse", "dq", "dkv", "dt"):
            assert torch.equal(cap[name], eager[name]) and torch.equal(other[name], eager[name]), name


# Buckets of distances that no query and key of the call have: rows of the last tile that do not exist meet them.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk,d,causal,both,query0,unused", [
    (1, 2, 33, 33, 64, False, True, 0, [13, 14, 15, 29, 30, 31]), (2, 3, 33, 33, 40, True, False, 0, range(23, 32)), (30, 12, 33, 33, 64, False, True, 0, [13, 14, 15, 29, 30, 31]),
    (1, 1, 1, 700, 64, False, False, 0, range(1, 32)), (1, 3, 70, 70, 96, True, True, 0, [15, *range(17, 32)]), (4, 12, 77, 300, 64, False, True, 0, [15]),
    (8, 10, 70, 70, 64, False, True, 0, [15, 31]), (4, 20, 70, 300, 64, False, True, 0, [15]), (1, 2, 40, 2000, 64, True, False, 0, range(24, 32)), (1, 8, 33, 300, 96, False, False, 0, range(23, 32)), (3, 40, 33, 520, 64, False, False, 0, range(23, 32))])
def test_anything_in_buckets_of_distances_that_do_not_occur(dtype, B, H, nq, nk, d, causal, both, query0, unused):
    from oracle import training_ops as T
    visible = [[not causal or k <= q + query0 for k in range(nk)] for q in range(nq)]
    assert not set(T.buckets(nq, nk, query0, 32, 128, both)[visible].tolist()) & set(unused)
    for x in (float("nan"), float("inf"), -float("inf")):
        _check(dtype, B, H, nq, nk, d, causal, both, 32, 128, query0, None, garbage={k: x for k in unused})


# Buckets that only keys behind a sample's length meet.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,nq,nk,d,query0,length", [(1, 2, 300, 300, 64, 0, 20), (1, 8, 70, 500, 40, -5, 15), (40, 10, 77, 77, 64, 0, 19), (3, 40, 130, 300, 64, 0, 17), (8, 12, 300, 400, 96, 0, 12),
                                                       (4, 3, 1, 2000, 64, 0, 20), (1, 3, 400, 2300, 64, 0, 18), (2, 40, 513, 90, 64, 0, 16)])
def test_anything_in_buckets_behind_the_key_lengths(dtype, B, H, nq, nk, d, query0, length):
    from oracle import training_ops as T
    bk = T.buckets(nq, nk, query0, 32, 128, True)
    hidden = sorted(set(bk[:, length:].ravel().tolist()) - set(bk[:, :length].ravel().tolist()))
    assert len(hidden) >= 4
    for x in (float("nan"), float("inf")):
        _check(dtype, B, H, nq, nk, d, False, True, 32, 128, query0, [length] * (B - 1) + [length - 1], garbage={k: x for k in hidden})


# Up to 32 queries of so many heads that each gets a workgroup of the kernel for many queries.
@pytest.mark.parametrize("B,H,nq,nk,d,causal,lens", [(75, 8, 1, 600, 64, True, None), (70, 10, 32, 77, 64, False, "some"), (40, 8, 17, 300, 96, True, "some"), (40, 16, 5, 700, 40, False, "some")])
def test_few_queries_of_many_heads(B, H, nq, nk, d, causal, lens):
    _check("bf16", B, H, nq, nk, d, causal, not causal, 32, 128, nk - nq, [(nk * (i + 1)) // B for i in range(B)] if lens else None)
