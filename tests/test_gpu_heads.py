"""prq_rotate_heads and prq_norm_rotate_heads on the GPU against their 64-bit form."""
import pytest

import beside_ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _positions(g, M, far):
    return torch.randint(0, far, (M,), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)


def _check(got, t, positions, o, rot, layout, norm=False, weight=None, eps=1e-6):
    f, factor = beside_ref.frequencies(rot, **o)
    want, bound = beside_ref.heads(t, positions, f, factor, rot, layout, norm, weight, eps)
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), (off / bound).max()


PLAIN = dict(scaling="none")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("M,q,k,D,rot", [
    (1, 32, 8, 128, 128), (1, 1, 0, 64, 64), (3, 4, 1, 64, 32), (2, 3, 5, 80, 80), (5, 20, 20, 80, 32), (4, 7, 2, 96, 48), (7, 16, 2, 128, 64), (9, 5, 1, 256, 256),
    (2, 4, 2, 256, 64), (6, 2, 1, 192, 192), (3, 3, 3, 112, 112), (33, 8, 1, 576 - 64, 64), (2, 2, 1, 512, 256), (5, 2, 2, 18, 18), (4, 3, 1, 2, 2), (3, 2, 1, 20, 6),
    (2, 5, 3, 129, 34), (64, 32, 8, 128, 128), (130, 9, 3, 128, 128), (257, 6, 2, 64, 64), (1000, 3, 1, 128, 32), (513, 2, 2, 40, 40), (301, 40, 8, 128, 128),
    (150, 12, 1, 16, 16), (149, 4, 1, 48, 16), (700, 20, 20, 80, 32), (701, 7, 11, 96, 96), (702, 13, 1, 80, 80)])
def test_against_64_bits(prq, M, q, k, D, rot, norm, layout, dtype):
    g = _g(M + D + rot)
    y = _normal(g, M, (q + 2 * k) * D).to(DT[dtype])
    before = y.clone()
    tq, tk = y[:, : q * D].view(M, q, D), y[:, q * D: (q + k) * D].view(M, k, D)
    positions = _positions(g, M, 40960)
    weights = [0.5 + torch.rand(D, generator=g, device="cuda") for _ in range(2)] if norm and M != 7 else [None, None]
    rope = prq.Rope(D, rot, layout, base=1e6)
    call = (lambda *a, **o: prq.norm_rotate_heads(rope, positions, *a, *weights, **o)) if norm else (lambda *a, **o: prq.rotate_heads(rope, positions, *a, **o))
    out = [torch.full_like(t, float("nan")).contiguous() for t in (tq, tk)]
    got = call(tq, tk, out=out)
    assert got[0] is out[0] and got[1] is out[1] and torch.equal(y, before)
    for o, t, w in zip(out, (tq, tk), weights):
        _check(o, t, positions, dict(base=1e6), rot, layout, norm, w)
    call(tq, tk)        # in place: the same; the values behind the keys are left alone
    assert torch.equal(tq, out[0]) and torch.equal(tk, out[1]) and torch.equal(y[:, (q + k) * D:], before[:, (q + k) * D:])
    assert prq.last_device_status() == 0


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("o", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0, base=1e6), dict(scaling="yarn", factor=4.0, original_positions=32768, base=1e6),
                               dict(scaling="bands", factor=8.0, original_positions=8192, base=5e5)])
def test_far_positions_and_scalings(prq, o, dtype, norm):
    """Positions up to the last one, the first ones and negative ones: as exact everywhere."""
    g, D = _g(3), 128
    edge = [0, 1, 2, 7, 1023, 40959, 131071, 1048575, 2 ** 24 + 1, 2 ** 30 + 3, 2 ** 31 - 1, -1, -2, -4097, -2 ** 24 - 1, -2 ** 31 + 1]
    positions = torch.tensor(edge, dtype=torch.int32, device="cuda")
    q, k = (_normal(g, len(edge), h, D).to(DT[dtype]) for h in (4, 2))
    rope = prq.Rope(D, **o)
    got = (prq.norm_rotate_heads if norm else prq.rotate_heads)(rope, positions, q, k, out=(torch.empty_like(q), torch.empty_like(k)))
    # cosine and sine by the library's own frequencies, through exact integers: the fraction of a turn of every angle
    f, factor = rope.frequencies()
    want, _ = beside_ref.frequencies(D, **o)
    assert max(abs(a / b - 1) for a, b in zip(f, want)) < 2.0 ** -48
    import math
    from fractions import Fraction

    pi = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)
    for t, r in zip((q, k), got):
        z = t.double()
        rel = 0.0
        if norm:
            z, rel = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt(), (D / 2 + 8) * beside_ref.U
        for m, pos in enumerate(edge):
            turn = [Fraction(float(v)) / (2 * pi) * pos for v in f]
            angle = torch.tensor([float(2 * pi * (v - math.floor(v))) for v in turn], dtype=torch.float64, device="cuda")
            # (a frequency as a double is itself off by 2^-53)
            loose = torch.tensor([abs(pos) * float(v) * 2.0 ** -52 for v in f], dtype=torch.float64, device="cuda")
            a, b = z[m, :, : D // 2], z[m, :, D // 2:]
            c, s = angle.cos() * factor, angle.sin() * factor
            off = (a.abs() + b.abs()) * factor * (rel + 12 * beside_ref.U + loose)
            for res, at in ((a * c - b * s, slice(0, D // 2)), (b * c + a * s, slice(D // 2, D))):
                assert ((r[m, :, at].double() - res).abs() <= off + beside_ref.half_step(t.dtype) * (res.abs() + off)).all(), pos


@pytest.mark.parametrize("D,rot", [(128, 128), (80, 20)])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_left_out_and_rows_that_are_not_finite(prq, norm, D, rot):
    g, M = _g(8), 70
    q, k = (_normal(g, M, h, D).to(torch.bfloat16) for h in (8, 2))
    positions = _positions(g, M, 5000)
    left = torch.tensor([0, 3, 33, 69], device="cuda")
    positions[left] = prq.POSITION_NONE
    q[3], k[33] = float("nan"), float("inf")                    # rows left out
    q[5, 2, 7], k[6, 1, 1], q[7, 0] = float("nan"), float("inf"), 0.0   # (all zeros: the norm's eps)
    before = q.clone(), k.clone()
    call = prq.norm_rotate_heads if norm else prq.rotate_heads
    out = torch.full_like(q, 3.0), torch.full_like(k, 5.0)
    rope = prq.Rope(D, rot)
    call(rope, positions, q, k, out=out)
    assert (out[0][left] == 3).all() and (out[1][left] == 5).all()
    call(rope, positions, q, k)
    for t, b, o in zip((q, k), before, out):
        assert torch.equal(t[left].view(torch.int16), b[left].view(torch.int16))
        ok = torch.isfinite(b.float()).all(-1)
        ok[left] = False
        f, factor = beside_ref.frequencies(rot)
        want, bound = beside_ref.heads(b, positions, f, factor, rot, "half", norm)
        assert ((o.double() - want).abs() <= bound)[ok].all() and torch.equal(o[ok], t[ok])
    assert torch.isnan(q[5, 2].float()).any() and (q[7, 0] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignments(prq, D, dtype):
    """Heads by rows and rows by heads, pointers that are only aligned to an element, one head read for all, guards around everything."""
    g, M, H, dt = _g(D), 21, 6, DT[dtype]
    positions = _positions(g, M, 3000)
    rope = prq.Rope(D)
    for kind in ("heads first", "odd", "odd rows", "broadcast", "gaps"):
        x = _normal(g, M, H, D).to(dt)
        if kind == "heads first":
            store = torch.full((H, M, D), 9.0, dtype=dt, device="cuda")
            out, x = store.transpose(0, 1), x.transpose(0, 1).contiguous().transpose(0, 1)
        elif kind == "odd":
            store = torch.full((M * H * D + 3,), 9.0, dtype=dt, device="cuda")
            out = store[1: 1 + M * H * D].view(M, H, D)
        elif kind == "odd rows":
            store = torch.full((M, H * D + 1), 9.0, dtype=dt, device="cuda")
            out = store[:, : H * D].view(M, H, D)
        elif kind == "broadcast":
            x = x[:1, :1].expand(M, H, D)
            store = out = torch.full((M, H, D), 9.0, dtype=dt, device="cuda")
        else:
            store = torch.full((M, H, D + 16), 9.0, dtype=dt, device="cuda")
            out = store[..., 8: 8 + D]
        guard = store.clone()
        out.copy_(torch.full_like(out, 7.0))
        inside = store != guard
        prq.rotate_heads(rope, positions, x, out=out)
        _check(out, x, positions, PLAIN, D, "half")
        assert (store[~inside] == 9).all(), kind


def test_turning_back(prq):
    """A negative position is the rotation's transpose: <R x, y> = <x, R' y>, and R' R x = x."""
    g, M, D = _g(4), 50, 128
    x, y = (_normal(g, M, 4, D) for _ in range(2))
    positions = _positions(g, M, 100000)
    for layout in ("half", "pairs"):
        rope = prq.Rope(D, 96, layout)
        rx = prq.rotate_heads(rope, positions, x, out=torch.empty_like(x))
        ty = prq.rotate_heads(rope, -positions, y, out=torch.empty_like(y))
        a, b = (rx.double() * y.double()).sum(-1), (x.double() * ty.double()).sum(-1)
        # each element is off by (|a| + |b|) 12 u and a rounding: 2^-19 of the lengths' product is above that for both sums
        assert ((a - b).abs() <= 2.0 ** -19 * x.double().norm(dim=-1) * y.double().norm(dim=-1)).all()
        back = prq.rotate_heads(rope, -positions, rx, out=torch.empty_like(rx))
        assert ((back - x).norm(dim=-1) <= 2.0 ** -19 * x.norm(dim=-1)).all()
        # differences of the rotation along y are the transposed rotation of y
        step = prq.rotate_heads(rope, positions, x + y, out=torch.empty_like(x)).double() - rx.double()
        assert ((step * y.double()).sum(-1) - (y.double() * prq.rotate_heads(rope, positions, y, out=torch.empty_like(y)).double()).sum(-1)).abs().max() <= 2.0 ** -17 * D * 16


def test_captured_and_on_another_stream(prq):
    g, M, D = _g(6), 40, 128
    q, k = (_normal(g, M, h, D).to(torch.bfloat16) for h in (8, 2))
    positions, rope = _positions(g, M, 9000), prq.Rope(D)
    out = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    prq.norm_rotate_heads(rope, positions, q, k, out=out, stream=side)
    side.synchronize()
    _check(out[0], q, positions, PLAIN, D, "half", True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prq.norm_rotate_heads(rope, positions, q, k, out=out)
    del rope                                        # a captured call holds what it needs
    for seed in (1, 2):
        q.copy_(_normal(_g(seed), M, 8, D))
        positions.copy_(_positions(_g(seed), M, 100000))
        graph.replay()
        _check(out[0], q, positions, PLAIN, D, "half", True)
        _check(out[1], k, positions, PLAIN, D, "half", True)


def test_no_rows_and_no_heads(prq):
    rope, n = prq.Rope(64), prq.kernel_launch_count()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    prq.rotate_heads(rope, none, torch.empty(0, 4, 64, device="cuda"))
    prq.rotate_heads(rope, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.empty(3, 0, 64, device="cuda"))
    assert prq.kernel_launch_count() == n


def test_offsets_beyond_32_bits(prq):
    """Heads that stand 2^31 elements and more from the first one."""
    M, D = 3, 64
    far = torch.zeros((1 << 31) + (1 << 30) + 4 * D, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(far, (M, 2, D), ((1 << 30) + (1 << 29), D, 1))
    x.copy_(_normal(_g(1), M, 2, D))
    before, positions = x.clone(), torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    prq.rotate_heads(prq.Rope(D), positions, x)
    _check(x, before, positions, PLAIN, D, "half")


def test_tensors_refused(prq):
    rope = prq.Rope(64)
    q, pos = torch.zeros(3, 2, 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [(pos.long(), q, None), (pos[:2], q, None), (pos.cpu(), q, None), (pos, q.cpu(), None), (pos, q.half(), None), (pos, q, q.bfloat16()), (pos, q[..., :32], None),
           (pos, q[0], None), (pos, q.transpose(1, 2).contiguous().transpose(1, 2), None)]
    for p, a, b in bad:
        with pytest.raises(prq.PrqError):
            prq.rotate_heads(rope, p, a, b)
    with pytest.raises(prq.PrqError):
        prq.rotate_heads(rope, pos, q, out=torch.zeros(3, 2, 32, device="cuda"))
    for w in (torch.ones(32, device="cuda"), torch.ones(64, device="cuda").bfloat16(), torch.ones(64), torch.ones(128, device="cuda")[::2]):
        with pytest.raises(prq.PrqError):
            prq.norm_rotate_heads(rope, pos, q, q_weight=w)
