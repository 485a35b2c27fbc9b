"""prq_linear_adapters on the GPU: many rows in windows, tall batches of high ranks, pools larger than what a batch uses, far rows and slots."""
import pytest

import beside_ref
from test_gpu_adapters import DT, _inputs, _normal, _rows

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _check(got, x, A, B, parts, rows, base, scale=None, ranks=None):
    want, bound = beside_ref.adapters_of_many(x, A, B, parts, rows, base, scale, ranks)
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), (off / bound).max()
    bare = (rows < 0) | (rows >= A.shape[0])
    assert torch.equal(got[bare], base[bare])


def _both_ways(prq, x, A, B, parts, rows, base, scale=None, ranks=None):
    pool = prq.Adapters(A, B, parts, scale=scale, ranks=ranks)
    out, y = (torch.full((base.shape[0], base.stride(0)), float("nan"), dtype=base.dtype, device="cuda")[:, : base.shape[1]] for _ in range(2))   # (base's stride)
    got = prq.linear_adapters(pool, x, rows, base, out=out)
    _check(got, x, A, B, parts, rows, base, scale, ranks)
    y.copy_(base)
    prq.linear_adapters(pool, x, rows, y)
    assert torch.equal(y, got) and prq.last_device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,R,S,pattern", [
    (4096, 16, 3, "some"), (4097, 16, 3, "mix"), (4097, 40, 5, "sorted"), (5000, 128, 7, "some"), (8191, 32, 60, "mix"), (8200, 72, 2, "runs"),
    (12289, 24, 1, "one"), (9000, 8, 2, "none"), (4500, 16, 300, "mix"), (4500, 48, 300, "some"), (4200, 16, 520, "mix"), (8400, 64, 513, "sorted")])
def test_windows_of_rows(prq, M, R, S, pattern, dtype):
    parts, K = [136, 72], 96
    g, x, A, B, base = _inputs(M + R, M, K, parts, R, S, dtype)
    _both_ways(prq, x, A, B, parts, _rows(pattern, M, S, g), base, scale=torch.rand(S, generator=g, device="cuda") * 2 - 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,R,parts,ranks", [
    (8192, 64, [2560, 2563], None), (8192, 40, [5120], None), (8100, 48, [2560, 2568], [48, 33, 7, 0]), (4096, 64, [9728, 1024, 1021], [64, 63, 1, 16]),
    (4096, 56, [10001], [8, 56, 40, 24])])
def test_tall_batches_of_high_ranks(prq, M, R, parts, ranks, dtype):
    """Sizes whose tiles go through tensor memory, 512 bytes of a row at a time; what lies behind a rank is NaN and infinities."""
    K, S = 64, 4
    g, x, A, B, base = _inputs(M + R, M, K, parts, R, S, dtype)
    if ranks:
        for s, r in enumerate(ranks):
            A[s, :, r:] = float("inf")
            B[s, :, r:] = float("nan")
        ranks = torch.tensor(ranks, dtype=torch.int32, device="cuda")
    for pattern in ("sorted", "some"):
        _both_ways(prq, x, A, B, parts, _rows(pattern, M, S, g), base, ranks=ranks)


@pytest.mark.parametrize("M,K,parts,R,S,used", [
    (129, 256, [264], 16, 64, 64), (500, 512, [96, 40], 16, 500, 3), (500, 512, [96, 40], 16, 500, 500), (900, 320, [64, 64, 33], 64, 64, 64), (900, 2560, [64], 32, 511, 20),
    (640, 1024, [520], 16, 40, 40), (639, 1024, [520], 16, 40, 40), (1000, 1024, [72, 72, 72], 64, 48, 48), (1000, 96, [200], 128, 62, 62), (1500, 96, [200], 128, 62, 62),
    (3000, 64, [64], 16, 150, 150), (1000, 256, [128], 8, 700, 700), (4000, 64, [1031], 48, 200, 6), (2000, 32, [8], 8, 100, 99)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_of_many_adapters(prq, M, K, parts, R, S, used, dtype):
    """More adapters than run at once, all of them in use or few; some of rank 0, some rows without one."""
    g, x, A, B, base = _inputs(M + S, M, K, parts, R, S, dtype)
    rows = torch.randint(0, used, (M,), generator=g, device="cuda", dtype=torch.int32)
    rows[3::11] = -1
    ranks = torch.randint(0, R + 1, (S,), generator=g, device="cuda", dtype=torch.int32)
    ranks[1] = 0
    _both_ways(prq, x, A, B, parts, rows, base, ranks=ranks)
    _both_ways(prq, x, A, B, parts, rows, base)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 6, 7, 12, 13, 16, 42, 43])
@pytest.mark.parametrize("R,parts", [(64, [128, 64, 64]), (128, [72, 33]), (40, [64, 64]), (24, [1040, 16, 8, 5])])
def test_few_rows_of_high_ranks(prq, M, R, parts):
    """On both sides of where a call changes from one launch to two."""
    K, S = 2560, 8
    g, x, A, B, base = _inputs(M + R, M, K, parts, R, S, "bf16")
    ranks = torch.tensor([R, R - 1, 0, 1, 17, R, 8, R], dtype=torch.int32, device="cuda")
    for pattern in ("mix", "some"):
        _both_ways(prq, x, A, B, parts, _rows(pattern, M, S, g), base, scale=torch.rand(S, generator=g, device="cuda") * 2 - 0.5, ranks=ranks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,S", [(511, 4), (512, 4), (513, 4), (1023, 64), (1024, 64), (31, 511), (33, 512)])
def test_where_the_form_changes(prq, M, S, dtype):
    parts, K, R = [200, 33], 1056, 16
    g, x, A, B, base = _inputs(M + S, M, K, parts, R, S, dtype)
    for pattern in ("mix", "some", "sorted"):
        _both_ways(prq, x, A, B, parts, _rows(pattern, M, S, g), base)


@pytest.mark.parametrize("M,S,R", [(300, 64, 16), (1000, 30, 64), (1100, 8, 128)])
def test_a_captured_call_finds_more_items_than_it_had(prq, M, S, R):
    """Captured with one adapter in use, replayed with all of them, and with none."""
    parts, K = [96, 72], 256
    g, x, A, B, base = _inputs(M, M, K, parts, R, S, "bf16")
    rows, pool, out = _rows("one", M, S, g), prq.Adapters(A, B, parts), torch.empty_like(base)
    ws, stream, graph = prq.adapters_workspace(pool, M), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        prq.linear_adapters(pool, x, rows, base, out=out, workspace=ws)
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        prq.linear_adapters(pool, x, rows, base, out=out, workspace=ws)
    for pattern in ("mix", "none", "some", "one"):
        rows.copy_(_rows(pattern, M, S, g))
        ws.fill_(255)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        _check(out, x, A, B, parts, rows, base)


@pytest.mark.parametrize("M,R,parts", [(5, 16, [64]), (300, 16, [64]), (300, 72, [64]), (8192, 64, [5120])])
def test_sums_beyond_the_range(prq, M, R, parts):
    """An infinite sum stays infinite, with the sign of its product; other rows and ranks are as ever."""
    K, S = 64, 2
    g, x, A, B, base = _inputs(M, M, K, parts, R, S, "f32")
    rows = torch.zeros(M, dtype=torch.int32, device="cuda")
    A[0, 0, 3] = 1.0
    B[0, :, 3] = B[0, :, 3].sign() * 0.5
    B[0, 7, 3] = 0.25
    x[2] = 2.0 ** 127
    A[0, 0, [r for r in range(R) if r != 3]] = 0
    got = prq.linear_adapters(prq.Adapters(A, B, parts), x, rows, base, out=torch.empty_like(base))
    some = B[0, :, 3] != 0
    assert torch.equal(got[2][some], (B[0, :, 3].float() * float("inf"))[some])
    ok = torch.arange(M, device="cuda") != 2
    _check(got[ok], x[ok], A, B, parts, rows[ok], base[ok])


@pytest.mark.parametrize("M,R", [(7, 16), (140, 16), (700, 24), (700, 128)])
def test_rows_and_slots_far_apart(prq, M, R):
    """Row strides and slots whose offsets pass 32 bits."""
    S, K, N, ld = 2 ** 31 // (8 * 2048 * R) * 8 + 9, 2048, 2048, 2 ** 31 // M // 8 * 8 + 4096
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    A, B = (torch.empty(S, *shape, dtype=torch.bfloat16, device="cuda") for shape in ((1, R, K), (N, R)))
    used = [0, 5, S - 2, S - 1]
    for s in used:
        A[s], B[s] = (_normal(g, 1, R, K) * 0.05).to(torch.bfloat16), (_normal(g, N, R) * 0.2).to(torch.bfloat16)
    x, y = (torch.empty(M, ld, dtype=torch.bfloat16, device="cuda")[:, :2048] for _ in range(2))
    x.copy_(_normal(g, M, K))
    y.copy_(_normal(g, M, N))
    pick = torch.randint(0, 4, (M,), generator=g, device="cuda")
    rows, base = torch.tensor(used, dtype=torch.int32, device="cuda")[pick].contiguous(), y.clone()
    prq.linear_adapters(prq.Adapters(A, B, [N]), x, rows, y)
    want, bound = beside_ref.adapters_of_many(x, A[used], B[used], [N], pick, base)
    assert ((y.double() - want).abs() <= bound).all()
    del A, B, x, y
    torch.cuda.empty_cache()


def test_a_row_table_that_begins_anywhere(prq):
    g, x, A, B, base = _inputs(3, 300, 64, [40], 16, 3, "bf16")
    table = _rows("mix", 304, 3, g)
    for at in (1, 2, 3):
        out = prq.linear_adapters(prq.Adapters(A, B, [40]), x, table[at: at + 300], base, out=torch.empty_like(base))
        _check(out, x, A, B, [40], table[at: at + 300], base)


def test_two_calls_at_once(prq):
    """Two streams, a workspace each, back to back without a wait in between: as one after another."""
    sides = []
    for seed, (M, R, S) in enumerate([(700, 72, 6), (1200, 16, 20)]):
        g, x, A, B, base = _inputs(seed, M, 512, [640, 256], R, S, "bf16")
        rows, pool = _rows("some", M, S, g), prq.Adapters(A, B, [640, 256])
        sides.append((pool, x, rows, base, [torch.empty_like(base) for _ in range(8)], prq.adapters_workspace(pool, M), torch.cuda.Stream(), A, B))
    torch.cuda.synchronize()
    for i in range(8):
        for pool, x, rows, base, outs, ws, stream, *_ in sides:
            prq.linear_adapters(pool, x, rows, base, out=outs[i], workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for pool, x, rows, base, outs, ws, stream, A, B in sides:
        _check(outs[0], x, A, B, [640, 256], rows, base)
        assert all(torch.equal(outs[0], o) for o in outs[1:])
    assert prq.last_device_status() == 0
