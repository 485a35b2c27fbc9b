"""Adapters and position rotation, what needs no GPU: refusals, frequencies, the fold, what a call launches."""
import ctypes
import importlib.util
import math
import sys

import numpy as np
import pytest

import beside_ref
from paper_2609_22106_b200 import synth
from test_lib_fake_runtime import _aligned, fake  # noqa: F401  (fixture)

SCALINGS = [dict(scaling="none"), dict(scaling="none", base=1e6), dict(scaling="linear", factor=3.5), dict(scaling="ntk", factor=8.0, base=5e5),
            dict(scaling="yarn", factor=4.0, original_positions=32768, base=1e6), dict(scaling="yarn", factor=16.0, original_positions=4096, beta_fast=24.0, beta_slow=2.0),
            dict(scaling="yarn", factor=1.0, original_positions=2048), dict(scaling="bands", factor=8.0, original_positions=8192, base=5e5),
            dict(scaling="bands", factor=32.0, original_positions=4096, low_factor=2.0, high_factor=16.0)]


@pytest.mark.parametrize("o", SCALINGS)
@pytest.mark.parametrize("rot", [4, 32, 128, 256])
def test_frequencies(prq, o, rot):
    f, factor = prq.Rope(rot, **o).frequencies()
    want, want_factor = beside_ref.frequencies(rot, **o)
    # the reference's own powers and products in 64 bits are off by some 2^-50
    assert np.allclose(f, want, rtol=2.0 ** -48, atol=0) and math.isclose(factor, want_factor, rel_tol=1e-14)


def test_frequencies_of_a_single_pair_and_a_factor_of_ones_own(prq):
    f, factor = prq.Rope(64, rot_dim=2, attention_factor=0.75).frequencies()
    assert f.tolist() == [1.0] and factor == 0.75


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=514), dict(head_dim=128, rot_dim=3), dict(head_dim=128, rot_dim=130), dict(head_dim=512), dict(head_dim=512, rot_dim=258),
    dict(head_dim=65), dict(head_dim=64, base=1.0), dict(head_dim=64, base=-2.0), dict(head_dim=64, base=math.inf), dict(head_dim=64, factor=0.5),
    dict(head_dim=64, factor=math.nan), dict(head_dim=64, rot_dim=2, scaling="ntk", factor=2.0), dict(head_dim=64, scaling="yarn", factor=2.0),
    dict(head_dim=64, scaling="yarn", factor=2.0, original_positions=4096, beta_fast=1.0, beta_slow=2.0), dict(head_dim=64, scaling="bands", factor=2.0),
    dict(head_dim=64, scaling="bands", factor=2.0, original_positions=4096, low_factor=4.0, high_factor=4.0), dict(head_dim=64, attention_factor=-1.0),
    dict(head_dim=64, layout="other"), dict(head_dim=64, scaling="other")])
def test_frequencies_refused(prq, bad):
    with pytest.raises(prq.PrqError):
        prq.Rope(**bad)


def test_options_of_a_smaller_struct_are_refused(prq):
    o, h = prq.RopeOpts(8, 64), ctypes.c_void_p()
    assert prq.lib().prq_rope_create(ctypes.addressof(o), ctypes.byref(h)) == 1
    assert prq.lib().prq_rope_create(None, ctypes.byref(h)) == 1
    assert prq.lib().prq_rope_frequencies(None, None, None) == 1
    prq.lib().prq_rope_free(None)


def test_fold_adapter_is_the_rounded_product(prq):
    rng = np.random.default_rng(3)
    K, rows = 96, 5
    perm = rng.permutation(K).astype(np.int32)
    s = np.exp(rng.standard_normal(K)).astype(np.float32)
    A = synth.weights(4, rows, K)
    want = synth.f32_to_bf16(synth.bf16_to_f32(A)[:, perm] * s[perm])
    assert np.array_equal(prq.fold_adapter(perm, s, A), want)
    for i, (p, f) in enumerate([(np.r_[perm[:-1], K], s), (np.r_[perm[:-1], -1], s), (perm, np.r_[s[:-1], np.inf])]):
        with pytest.raises(prq.PrqError):
            prq.fold_adapter(p, f, A)
    with pytest.raises(prq.PrqError):
        prq.fold_adapter(perm[:-1], s[:-1], A)


def _pool(fake, S=4, R=16, K=64, parts=(32, 16), **other):  # noqa: F811
    some = _aligned(16)
    f = dict(struct_size=ctypes.sizeof(fake.AdapterPool), n_slots=S, max_rank=R, K=K, n_parts=len(parts), part_N=(ctypes.c_int * 4)(*parts[:4]), A=some.ctypes.data,
             B=some.ctypes.data, scale=None, ranks=None)
    return fake.AdapterPool(**{**f, **other})


def _call(fake, pool, M=3, ldx=64, ldb=48, ldy=48, dtype=0, **other):  # noqa: F811
    some, ws = _aligned(16), _aligned(1 << 20)
    a = dict(rows=some.ctypes.data, x=some.ctypes.data, base=some.ctypes.data, y=some.ctypes.data, ws=ws.ctypes.data, bytes=1 << 20)
    a.update(other)
    before = fake.kernel_launch_count()
    rc = fake.lib().prq_linear_adapters(ctypes.addressof(pool) if pool is not None else None, a["rows"], a["x"], M, ldx, a["base"], ldb, a["y"], ldy, dtype,
                                        a["ws"], a["bytes"], None)
    launched = fake.kernel_launch_count() - before
    assert (launched > 0) == (rc == 0 and M > 0)
    return rc


def test_adapters_taken(fake):  # noqa: F811
    assert _call(fake, _pool(fake)) == 0
    assert _call(fake, _pool(fake), M=0, rows=None, x=None) == 0
    assert _call(fake, _pool(fake, parts=(32, 13)), ldb=48) == 0
    assert _call(fake, _pool(fake), dtype=1, ldb=56, ldy=48, base=_aligned(16).ctypes.data) == 0


@pytest.mark.parametrize("status,pool,call", [
    (1, dict(struct_size=8), {}), (1, dict(S=0), {}), (1, dict(R=0), {}), (1, dict(R=12), {}), (1, dict(R=136), {}), (1, dict(K=48), {}), (1, dict(K=0), {}),
    (1, dict(n_parts=0), {}), (1, dict(n_parts=5), {}), (1, dict(parts=(20, 16)), {}), (1, dict(parts=(32, 0)), {}), (1, dict(parts=(1 << 30, 1 << 30)), {}),
    (1, dict(A=None), {}), (1, dict(B=None), {}), (2, dict(A=8), {}), (2, dict(B=8), {}), (2, dict(scale=2), {}), (2, dict(ranks=2), {}),
    (1, {}, dict(M=-1)), (1, {}, dict(dtype=2)), (1, {}, dict(ldx=56)), (1, {}, dict(ldb=40, ldy=40)), (1, {}, dict(ldb=56)), (2, {}, dict(ldx=68)),
    (2, {}, dict(ldb=50, ldy=50)), (2, {}, dict(ldb=52, ldy=52, dtype=1)), (1, {}, dict(rows=None)), (1, {}, dict(x=None)), (1, {}, dict(base=None)),
    (1, {}, dict(y=None)), (2, {}, dict(rows=2)), (2, {}, dict(x=8)), (2, {}, dict(base=8)), (2, {}, dict(y=8))])
def test_adapters_refused(fake, status, pool, call):  # noqa: F811
    assert _call(fake, _pool(fake, **pool), **call) == status


def test_adapters_refused_without_a_workspace_or_a_pool(fake):  # noqa: F811
    assert _call(fake, None) == 1
    p = _pool(fake)
    need = fake.lib().prq_adapters_workspace_bytes(ctypes.addressof(p), 3)
    if need:
        assert _call(fake, p, ws=None) == 8 and _call(fake, p, bytes=need - 1) == 8 and _call(fake, p, ws=8) == 2
    assert _call(fake, p, bytes=max(need, 1)) == 0
    assert fake.lib().prq_adapters_workspace_bytes(ctypes.addressof(p), 0) == 0 and fake.lib().prq_adapters_workspace_bytes(None, 3) == 0


def test_adapters_workspace_by_rows_and_slots(fake):  # noqa: F811
    def need(M, **f):
        pool = _pool(fake, **f)
        return fake.lib().prq_adapters_workspace_bytes(ctypes.addressof(pool), M)

    assert need(512) == 0 and need(513) > 513 * 2 * 16 * 4 and need(513, S=64) == 0 and need(1024, S=64) > 0 and need(1 << 20, S=600) == 0
    assert need(1, R=64) > 2 * 64 * 4 and all(need(M + 1, R=R, S=S) >= need(M, R=R, S=S) for R in (40, 64, 128) for S in (1, 2, 8, 64) for M in range(1, 600))   # up to M rows
    assert need(5000) > need(4096) and need((1 << 23) - 1) > (1 << 23) * 2 * 16 * 4 - 1024 and need(1 << 23) == 0
    big = _pool(fake)
    assert _call(fake, big, M=1 << 23) == 1 and _call(fake, big, M=513, bytes=need(513) - 1) == 8 and _call(fake, big, M=513, ws=None) == 8
    assert _call(fake, big, M=513, ws=_aligned(1 << 20).ctypes.data + 8) == 2 and _call(fake, big, M=513) == 0 and _call(fake, _pool(fake, S=64), M=513, ws=None, bytes=0) == 0


def _heads(fake, x=1, out=1, ldx=256, hsx=64, ldout=256, hsout=64, heads=4, weight=0):  # noqa: F811
    some = _aligned(16).ctypes.data
    at = lambda v: some if v == 1 else v
    return fake._HEADS.pack(at(x), at(out), ldx, hsx, ldout, hsout, heads, at(weight))


def _rotate(fake, q, k=None, M=3, dtype=1, eps=None, positions=1, rope=True):  # noqa: F811
    r = fake.Rope(64)
    pos = _aligned(16).ctypes.data if positions == 1 else positions
    before = fake.kernel_launch_count()
    handle = r._h if rope else None
    rc = fake.lib().prq_rotate_heads(handle, pos, M, q, k, dtype, None) if eps is None else fake.lib().prq_norm_rotate_heads(handle, pos, M, q, k, eps, dtype, None)
    launched = fake.kernel_launch_count() - before
    assert launched <= (rc == 0)
    return rc, launched


def test_heads_taken(fake):  # noqa: F811
    h = _heads(fake)
    assert _rotate(fake, h) == (0, 1) and _rotate(fake, h, h) == (0, 1) and _rotate(fake, h, h, eps=1e-6) == (0, 1)   # one launch for both
    assert _rotate(fake, h, M=0) == (0, 0) and _rotate(fake, _heads(fake, 0, 0, heads=0)) == (0, 0)
    assert _rotate(fake, _heads(fake, heads=0), h) == (0, 1)
    assert _rotate(fake, _heads(fake, ldx=64, ldout=64, hsx=192, hsout=192)) == (0, 1)      # heads by heads
    assert _rotate(fake, _heads(fake, ldx=0, hsx=0, out=1 << 20)) == (0, 1)                   # one head read for all


@pytest.mark.parametrize("status,q,call", [
    (1, dict(x=0), {}), (1, dict(out=0), {}), (1, dict(heads=-1), {}), (1, dict(hsout=32, out=1 << 20), {}), (1, dict(ldout=32, out=1 << 20), {}),
    (1, dict(ldx=512), {}), (1, dict(hsx=128), {}), (2, dict(x=3), {}), (2, dict(out=3), {}), (2, dict(x=6), dict(dtype=0)), (2, dict(weight=2), dict(eps=1e-6)),
    (1, {}, dict(M=-1)), (1, {}, dict(dtype=2)), (1, {}, dict(eps=0.0)), (1, {}, dict(eps=-1.0)), (1, {}, dict(eps=math.nan)), (1, {}, dict(eps=math.inf)),
    (1, {}, dict(positions=None)), (2, {}, dict(positions=2)), (1, {}, dict(rope=False))])
def test_heads_refused(fake, status, q, call):  # noqa: F811
    assert _rotate(fake, _heads(fake, **q), **call) == (status, 0)
    if "x" not in q and not call:
        assert _rotate(fake, _heads(fake), _heads(fake, **q), **call) == (status, 0)
    assert _rotate(fake, None) == (1, 0)


def test_more_heads_than_a_row_can_have(fake):  # noqa: F811
    assert _rotate(fake, _heads(fake, heads=65536, ldx=1 << 23, ldout=1 << 23)) == (0, 1)
    assert _rotate(fake, _heads(fake, heads=65537, ldx=1 << 23, ldout=1 << 23)) == (1, 0)


def test_a_thread_that_finds_torch_loaded_finds_all_of_its_names(prq):
    """Two threads' first calls may meet: at no line of the load is torch set and another name not."""
    pytest.importorskip("torch")
    spec = importlib.util.spec_from_file_location("prq_binding_loaded_anew", prq.__file__)
    anew = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(anew)
    bad, lines = [], []

    def step(frame, event, arg):
        if frame.f_code is anew._load_torch.__code__:
            lines.append(frame.f_lineno)
            if anew._torch is not None and None in (anew._f32, anew._bf16, anew._i32, anew._current_device):
                bad.append(frame.f_lineno)
            return step

    before = sys.gettrace()
    sys.settrace(step)
    try:
        anew._load_torch()
    finally:
        sys.settrace(before)
    assert anew._torch is not None and len(set(lines)) > 3 and not bad


class _Tensor:
    """What the binding asks of a CUDA tensor, over host bytes (device memory to the stand-in)."""

    def __init__(self, torch, shape, stride, dtype, device=0):
        self.shape, self._stride, self.dtype, self._device, self._bytes = torch.Size(shape), tuple(stride), dtype, device, _aligned(1 << 16)

    stride = lambda self: self._stride
    dim = lambda self: len(self.shape)
    get_device = lambda self: self._device
    data_ptr = lambda self: self._bytes.ctypes.data
    is_contiguous = lambda self: True


@pytest.fixture
def tensors(fake, monkeypatch):  # noqa: F811
    """The binding over the stand-in with such tensors on its device 0, and a stream to pass."""
    torch = pytest.importorskip("torch")
    fake._load_torch()
    monkeypatch.setattr(fake, "_current_device", lambda: 0)
    return torch, lambda *a, **o: _Tensor(torch, *a, **o), type("Stream", (), {"cuda_stream": 0})


def test_a_norm_without_its_eps_is_refused(fake, tensors):  # noqa: F811
    """... and not taken for a rotation without a norm."""
    torch, tensor, stream = tensors
    rope, positions, q = fake.Rope(64), tensor((3,), (1,), torch.int32), tensor((3, 2, 64), (128, 64, 1), torch.bfloat16)
    n = fake.kernel_launch_count()
    for eps in (None, 0.0, -1.0, math.nan):
        with pytest.raises(fake.PrqError):
            fake.norm_rotate_heads(rope, positions, q, eps=eps, stream=stream)
    assert fake.kernel_launch_count() == n
    assert fake.norm_rotate_heads(rope, positions, q, eps=1e-5, stream=stream) is q and fake.kernel_launch_count() == n + 1


def test_a_launch_that_fails_is_not_counted(fake):  # noqa: F811
    L, h = fake.lib(), _heads(fake)
    for eps in (None, 1e-6):
        L.fake_fail_launch(1)
        assert _rotate(fake, h, h, eps=eps) == (4, 0) and _rotate(fake, h, h, eps=eps) == (0, 1)
    for M, nth in ((3, 1), (513, 1), (513, 2)):           # one launch, the first and the second one of two
        before = fake.kernel_launch_count()
        L.fake_fail_launch(nth)
        pool, some, ws = _pool(fake), _aligned(16).ctypes.data, _aligned(1 << 20).ctypes.data
        call = lambda: L.prq_linear_adapters(ctypes.addressof(pool), some, some, M, 64, some, 48, some, 48, 0, ws, 1 << 20, None)
        assert call() == 4 and fake.kernel_launch_count() == before + nth - 1
        assert call() == 0


def test_a_factor_that_is_no_fp32_number_is_refused(prq):
    """Kernels multiply by it in fp32: one beyond that range would turn every element into infinities or zeros."""
    for bad in (1e39, 1.7e308, 1e-46, 5e-324):
        with pytest.raises(prq.PrqError):
            prq.Rope(64, attention_factor=bad)
    for good in (3.4e38, 1e-45, 0.5):
        assert prq.Rope(64, attention_factor=good).frequencies()[1] == good


def test_row_strides_beyond_an_int_are_refused(fake, tensors):  # noqa: F811
    """... and not cut to 32 bits on their way to the C call, which would read and write other rows."""
    torch, tensor, stream = tensors
    K, N, far = 64, 48, 2 ** 32 + 64
    pool = fake.Adapters.__new__(fake.Adapters)
    pool._pool = _pool(fake, K=K, parts=(N,))
    pool.K, pool.N, pool.device, pool._free_rows, pool._p = K, N, 0, 512, ctypes.addressof(pool._pool)
    rows = lambda M: tensor((M,), (1,), torch.int32)
    matrix = lambda M, n, ld, dtype=torch.bfloat16: tensor((M, n), (ld, 1), dtype)
    n = fake.kernel_launch_count()
    for ldx, ldb, ldy in ((far, 48, 48), (64, far, far), (64, far, 48), (64, 48, far)):
        with pytest.raises(fake.PrqError):
            fake.linear_adapters(pool, matrix(2, K, ldx), rows(2), matrix(2, N, ldb), out=matrix(2, N, ldy), stream=stream)
    assert fake.kernel_launch_count() == n
    for M, ld in ((2, 2 ** 31 - 8), (1, far)):           # the largest one; a single row has none
        fake.linear_adapters(pool, matrix(M, K, ld), rows(M), matrix(M, N, ld), out=matrix(M, N, ld), stream=stream)
    assert fake.kernel_launch_count() == n + 2


@pytest.mark.parametrize("answer", [None, 64])
def test_whether_a_call_needs_a_workspace_is_what_the_library_says(fake, tensors, monkeypatch, answer):  # noqa: F811
    """None: as it is; 64: a library that wants one of every call."""
    torch, tensor, _ = tensors
    ask = fake.lib().prq_adapters_workspace_bytes
    if answer:
        monkeypatch.setattr(fake.lib(), "prq_adapters_workspace_bytes", lambda p, M: answer)
    for S, parts, R in ((4, [64], 8), (4, [64, 32], 16), (4, [32, 32, 32], 16), (4, [32, 32, 32, 32], 24), (2, [64], 64), (2, [64], 72), (2, [64, 64], 40), (600, [64], 128)):
        A, B = tensor((S, len(parts), R, 64), (1, 1, 1, 1), torch.bfloat16), tensor((S, sum(parts), R), (1, 1, 1), torch.bfloat16)
        A.is_cuda = True
        pool = fake.Adapters(A, B, parts)
        assert all((answer or ask(pool._p, M)) == 0 for M in range(1, pool._free_rows + 1))
        if not answer and len(parts) * R <= 64 and R % 16 == 0:
            assert pool._free_rows == 512
