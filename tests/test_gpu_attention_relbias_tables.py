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
