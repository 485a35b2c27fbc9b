"""prq_linear_adapters on the GPU against its 64-bit form."""
import numpy as np
import pytest

import beside_ref
from paper_2609_22106_b200 import synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _inputs(seed, M, K, parts, R, S, dtype, ldx=None, ldb=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    N = sum(parts)
    x = _normal(g, M, ldx or K).to(torch.bfloat16)[:, :K]
    A = (_normal(g, S, len(parts), R, K) * 0.05).to(torch.bfloat16)
    B = (_normal(g, S, N, R) * 0.2).to(torch.bfloat16)
    base = _normal(g, M, ldb or -(-N // 8) * 8).to(DT[dtype])[:, :N]
    return g, x, A, B, base


def _rows(pattern, M, S, g):
    r = torch.randint(0, S, (M,), generator=g, device="cuda", dtype=torch.int32)
    if pattern == "none":
        r[:] = -1
    elif pattern == "one":
        r[:] = S - 1
    elif pattern == "sorted":
        r = r.sort().values
    elif pattern == "some":       # a third without one, by every kind of entry that names none
        r[::3] = torch.tensor([-1, S, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda").repeat(M)[: len(r[::3])]
    elif pattern == "runs":       # a prompt, a gap, single rows
        r[: M // 2] = 0
        r[M // 2: M // 2 + M // 8] = -1
    return r.contiguous()


def _check(got, x, A, B, parts, rows, base, scale=None, ranks=None):
    want, bound = beside_ref.adapters(x, A, B, parts, rows, base, scale, ranks)
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), (off / bound).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,parts,R,S,pattern", [
    (1, 32, [1], 8, 1, "one"), (1, 2560, [512, 128, 128], 16, 3, "one"), (1, 64, [24], 8, 2, "none"), (2, 96, [8, 5], 8, 2, "mix"),
    (7, 256, [40], 16, 3, "some"), (8, 544, [264, 8], 24, 8, "mix"), (9, 2560, [1031], 64, 4, "one"), (16, 256, [128], 128, 2, "mix"),
    (17, 1056, [96, 8, 8, 31], 40, 5, "some"), (33, 4096, [320], 32, 33, "mix"), (64, 2560, [256, 64, 64], 16, 64, "mix"), (65, 320, [72], 8, 1, "one"),
    (97, 9728, [160], 32, 12, "some"), (127, 64, [33], 56, 200, "mix"), (128, 512, [640], 16, 4, "sorted"), (129, 512, [640], 16, 4, "sorted"),
    (200, 2560, [96, 96], 128, 3, "runs"), (255, 32, [1, ], 8, 300, "mix"), (256, 288, [1025], 16, 2, "one"), (300, 800, [520, 16], 48, 60, "some"),
    (387, 4096, [640], 32, 3, "sorted"), (513, 256, [256, 64, 64], 16, 513, "mix"), (700, 128, [64], 64, 2, "none"), (1025, 1024, [1160], 64, 5, "runs"),
    (2048, 320, [328], 120, 8, "sorted")])
def test_against_64_bits(prq, M, K, parts, R, S, pattern, dtype):
    g, x, A, B, base = _inputs(M + K, M, K, parts, R, S, dtype)
    rows = _rows(pattern, M, S, g)
    scale = torch.rand(S, generator=g, device="cuda") * 2 - 0.5
    before = base.clone()
    out = torch.full_like(base, float("nan")) if base.is_contiguous() else torch.full((M, base.stride(0)), float("nan"), dtype=base.dtype, device="cuda")[:, : sum(parts)]
    got = prq.linear_adapters(prq.Adapters(A, B, parts, scale=scale), x, rows, base, out=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(base, before)
    _check(got, x, A, B, parts, rows, base, scale)
    bare = (rows < 0) | (rows >= S)
    assert torch.equal(got[bare], base[bare])
    assert prq.linear_adapters(prq.Adapters(A, B, parts, scale=scale), x, rows, base) is base     # in place: the same
    assert torch.equal(base, got) and prq.last_device_status() == 0


@pytest.mark.parametrize("M", [1, 5, 40, 150, 600])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ranks_of_ones_own_and_what_lies_beyond_them(prq, M, dtype):
    """Ranks of every size, beyond the limits too; what A and B hold behind a rank is NaN and infinities, and not used."""
    parts, K, R = [104, 24], 352, 32
    ranks = torch.tensor([0, 1, 7, 8, 9, 16, 17, 31, 32, 33, -4], dtype=torch.int32, device="cuda")
    S = len(ranks)
    g, x, A, B, base = _inputs(M, M, K, parts, R, S, dtype)
    for s, r in enumerate(ranks.tolist()):
        A[s, :, min(max(r, 0), R):] = float("nan")
        B[s, :, min(max(r, 0), R):] = float("inf")
    rows = _rows("mix", M, S, g) if M > 1 else torch.tensor([6], dtype=torch.int32, device="cuda")
    got = prq.linear_adapters(prq.Adapters(A, B, parts, ranks=ranks), x, rows, base, out=torch.empty_like(base))
    _check(got, x, A, B, parts, rows, base, ranks=ranks)
    assert torch.equal(got[ranks[rows.long()] <= 0], base[ranks[rows.long()] <= 0])


@pytest.mark.parametrize("M", [3, 20, 140, 500])
def test_a_slice_of_a_wider_matrix_and_rows_behind_the_batch(prq, M):
    """x, base and y as slices of wider matrices: nothing outside of the call's rows and columns is written."""
    parts, K, R, S = [64, 41], 160, 16, 3
    N = sum(parts)
    g, x, A, B, _ = _inputs(M, M, K, parts, R, S, "bf16", ldx=K + 24)
    wide = _normal(g, M + 3, N + 31).to(torch.bfloat16)
    rows = _rows("some", M, S, g)
    before = wide.clone()
    y = wide[:M, 16: 16 + N]
    prq.linear_adapters(prq.Adapters(A, B, parts), x, rows, y)
    _check(y, x, A, B, parts, rows, before[:M, 16: 16 + N])
    wide[:M, 16: 16 + N] = before[:M, 16: 16 + N]
    assert torch.equal(wide, before)


@pytest.mark.parametrize("M", [6, 90, 300])
def test_what_is_not_finite_stays_with_its_rows(prq, M):
    parts, K, R, S = [72], 128, 16, 4
    g, x, A, B, base = _inputs(M, M, K, parts, R, S, "f32")
    rows = _rows("mix", M, S, g)
    rows[0], rows[1], rows[2], rows[3] = 0, 1, 2, -1
    x[0, 5], x[3, 7] = float("nan"), float("inf")       # row 3 has no adapter
    A[1, 0, 2, 3] = float("inf")
    got = prq.linear_adapters(prq.Adapters(A, B, parts), x, rows, base, out=torch.empty_like(base))
    bad = rows == 1
    bad[0] = True
    assert not torch.isfinite(got[bad]).any(dim=1).all() and torch.isnan(got[0]).all()
    ok = torch.nonzero(~bad).flatten()
    _check(got[ok], x[ok], A, B, parts, rows[ok], base[ok])


def test_nothing_to_do(prq):
    g, x, A, B, base = _inputs(1, 0, 64, [16], 8, 1, "f32")
    n = prq.kernel_launch_count()
    prq.linear_adapters(prq.Adapters(A, B, [16]), x, torch.empty(0, dtype=torch.int32, device="cuda"), base)
    assert prq.kernel_launch_count() == n


@pytest.mark.parametrize("M", [1, 64, 300])
def test_the_same_call_gives_the_same_bits(prq, M):
    g, x, A, B, base = _inputs(M, M, 2560, [512, 128], 16, 8, "f32")
    rows, pool = _rows("some", M, 8, g), prq.Adapters(A, B, [512, 128])
    first = prq.linear_adapters(pool, x, rows, base, out=torch.empty_like(base))
    for _ in range(5):
        assert torch.equal(first, prq.linear_adapters(pool, x, rows, base, out=torch.empty_like(base)))


@pytest.mark.parametrize("M", [2, 48, 260])
def test_a_captured_call_follows_its_inputs(prq, M):
    """Two graphs, a workspace each, replayed on two streams; between replays rows, adapters and activations change."""
    K, parts, R, S = 320, [96, 40], 16, 5
    sides = []
    for seed in (1, 2):
        g, x, A, B, base = _inputs(seed, M, K, parts, R, S, "bf16")
        rows, out, pool = _rows("mix", M, S, g), torch.empty_like(base), prq.Adapters(A, B, parts)
        ws = prq.adapters_workspace(pool, M)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            prq.linear_adapters(pool, x, rows, base, out=out, workspace=ws)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            prq.linear_adapters(pool, x, rows, base, out=out, workspace=ws)
        sides.append((g, x, A, B, base, rows, out, graph, stream))
    for turn in range(3):
        for g, x, A, B, base, rows, out, graph, stream in sides:
            rows.copy_(_rows(("some", "one", "mix")[turn], M, S, g))
            x.copy_(_normal(g, M, K))
            A.copy_(_normal(g, *A.shape) * 0.05)
        torch.cuda.synchronize()
        for *_, graph, stream in sides:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for g, x, A, B, base, rows, out, *_ in sides:
            _check(out, x, A, B, parts, rows, base)


def test_a_stream_that_is_not_the_current_one(prq):
    g, x, A, B, base = _inputs(9, 200, 512, [256], 16, 4, "bf16")
    rows, pool, out = _rows("mix", 200, 4, g), prq.Adapters(A, B, [256]), torch.empty_like(base)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    prq.linear_adapters(pool, x, rows, base, out=out, stream=side)
    side.synchronize()
    _check(out, x, A, B, [256], rows, base)


def test_tensors_refused(prq):
    g, x, A, B, base = _inputs(1, 4, 64, [16], 8, 2, "f32")
    rows, pool = _rows("mix", 4, 2, g), prq.Adapters(A, B, [16])
    for args in [(x.half(), rows, base), (x, rows.long(), base), (x, rows[:3], base), (x, rows, base.half()), (x[:, :32], rows, base), (x, rows, base[:, :8]),
                 (x.cpu(), rows, base), (x, rows.cpu(), base), (x, rows, base.t().contiguous().t())]:
        with pytest.raises(prq.PrqError):
            prq.linear_adapters(pool, *args)
    for args, more in [((A.half(), B, [16]), {}), ((A, B, [8]), {}), ((A, B, [8, 8]), {}), ((A, B[:1], [16]), {}), ((A, B, [16]), dict(scale=torch.ones(3, device="cuda"))),
                       ((A, B, [16]), dict(ranks=torch.ones(2, device="cuda"))), ((A, B.cpu(), [16]), {})]:
        with pytest.raises(prq.PrqError):
            prq.Adapters(*args, **more)


def test_an_attention_blocks_projections_as_they_are_used(prq, oracle):
    """q / k / v as one stacked layer with scale and permutation folded into its producer, folded adapters beside it, then the norms
    and rotations of its heads -- against 64 bits from the layer's own output on, and the folded adapters against unfolded ones."""
    heads, kv, D, K, R, S, M = 4, 2, 64, 512, 16, 3, 37
    parts = [heads * D, kv * D, kv * D]
    L = synth.layer(97, sum(parts), K, M, T_cal=64)
    w = prq.prepare_weights(L["W"], oracle.channel_amax(L["zcal"]), 0.5, 64)
    perm, s, inv_s = (w.get(f) for f in (prq.FIELD_PERM, prq.FIELD_S, prq.FIELD_INV_S))
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.from_numpy(L["x"].view(np.int16)).cuda().view(torch.bfloat16)
    folded_x = (x.float()[:, torch.from_numpy(perm).long().cuda()] * torch.from_numpy(inv_s[perm]).cuda()).to(torch.bfloat16)
    A = (_normal(g, S, 3, R, K) * 0.02).to(torch.bfloat16)
    B = (_normal(g, S, sum(parts), R) * 0.02).to(torch.bfloat16)
    fold = prq.fold_adapter(perm, s, A.view(torch.int16).cpu().numpy().view(np.uint16).reshape(-1, K))
    Af = torch.from_numpy(fold.view(np.int16)).cuda().view(torch.bfloat16).view(A.shape)
    rows = _rows("some", M, S, g)
    codes, _, sf = prq.quantize_act(w, folded_x, prq.ACT_IDENTITY)
    y = prq.linear(w, codes, sf, M, prq.BF16)
    base = y.clone()
    prq.linear_adapters(prq.Adapters(Af, B, parts), folded_x, rows, y)
    _check(y, folded_x, Af, B, parts, rows, base)
    # x / s and A * s are each rounded to bf16 once: 2^-8 of every product, twice
    want, bound = beside_ref.adapters(x, A, B, parts, rows, base)
    for m, a in enumerate(rows.tolist()):
        if 0 <= a < S:
            size = torch.stack([(x[m].double() * A[a, p].double()).abs().sum(1) for p in range(3)])
            part = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(parts, device="cuda"))
            bound[m] += 2.0 ** -7 * 1.01 * (B[a].double().abs() * size[part]).sum(1) * (1 + 2.0 ** -8)
    assert ((y.double() - want).abs() <= bound).all()

    before = y.clone()
    q, k = y[:, : parts[0]].view(M, heads, D), y[:, parts[0]: parts[0] + parts[1]].view(M, kv, D)
    positions = torch.randint(0, 40000, (M,), generator=g, device="cuda", dtype=torch.int32)
    wq, wk = (0.5 + torch.rand(D, generator=g, device="cuda") for _ in range(2))
    prq.norm_rotate_heads(prq.Rope(D, base=1e6), positions, q, k, wq, wk)
    f, factor = beside_ref.frequencies(D, base=1e6)
    for t, at, weight in ((q, slice(0, parts[0]), wq), (k, slice(parts[0], parts[0] + parts[1]), wk)):
        want, bound = beside_ref.heads(before[:, at].view(t.shape), positions, f, factor, D, "half", True, weight)
        assert ((t.double() - want).abs() <= bound).all()
    assert torch.equal(y[:, parts[0] + parts[1]:], before[:, parts[0] + parts[1]:])      # v is left alone
    assert prq.last_device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,R,parts", [(6, 128, 16, [72]), (90, 96, 24, [40, 33]), (700, 128, 16, [72]), (700, 128, 48, [72]), (700, 64, 128, [72, 19]), (8192, 64, 64, [5120])])
def test_an_adapter_that_is_not_finite_marks_its_own_rows(prq, M, K, R, parts, dtype):
    """An infinity in A: every column of its part, in every row of the adapter; in B: its column.  All other results are as ever."""
    S, N = 4, sum(parts)
    g, x, A, B, base = _inputs(M + R, M, K, parts, R, S, dtype)
    rows = _rows("mix", M, S, g)
    rows[:4] = torch.arange(4, dtype=torch.int32, device="cuda")
    A[1, -1, R - 1, 3] = float("inf")
    B[2, 7, 1], B[2, N - 1, R - 1] = float("inf"), -float("inf")
    out = torch.zeros(M, base.stride(0), dtype=base.dtype, device="cuda")[:, :N]
    got = prq.linear_adapters(prq.Adapters(A, B, parts), x, rows, base, out=out)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[rows == 1, N - parts[-1]:] = True
    bad[(rows == 2).nonzero(), torch.tensor([[7, N - 1]], device="cuda")] = True
    assert torch.equal(~torch.isfinite(got), bad)
    A[1, -1, R - 1, 3] = B[2, 7, 1] = B[2, N - 1, R - 1] = 0
    want, bound = beside_ref.adapters_of_many(x, A, B, parts, rows, base)
    assert ((got.double() - want).abs() <= bound)[~bad].all()
