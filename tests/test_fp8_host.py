"""The 8-bit float linears and the optimizer step on the host (no GPU): sizes, refusals before any HIP call, the wrappers'
checks, and the tests' own reference against torch's conversion and closed forms."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import _fp8_ref as ref

OK, INVALID, UNSUPPORTED, OVERFLOW = 0, 1, 2, 3
F16, BF16, I8, F32 = 1, 2, 3, 5


@pytest.fixture(scope="module")
def spl():
    from paper_2405_03594_amd import LIB_PATH, build

    if not os.path.exists(LIB_PATH):
        build.build()
    import paper_2405_03594_amd as spl

    return spl


@pytest.fixture(scope="module")
def L(spl):
    return spl.lib()


# ------------------------------------------------------------------------------------------------ the reference


def test_reference_codes():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.values(np.arange(256)), v, equal_nan=True)
    x = torch.linspace(-448, 448, 40001, dtype=torch.float64)
    x = torch.cat((x, x * 2.0 ** -10, torch.from_numpy((ref.values(np.arange(126)) + ref.values(np.arange(1, 127))) / 2)))
    assert np.array_equal(ref.nearest(x.float().double().numpy()), x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_reference_scale():
    for e in (-127, -50, 0, 60):
        assert ref.exponent(448.0 * 2.0 ** e) == e
        assert ref.exponent(448.0 * 2.0 ** e * (1 + 2.0 ** -23)) == e + 1
    assert ref.exponent(0.0) == -127 and ref.exponent(2.0 ** -149) == -127
    x = np.random.default_rng(0).standard_normal((200, 300))
    for block in (1, 128):
        back = ref.round_trip(x, block)
        top = np.abs(x).max()
        assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * 2 * top / 448)).all()


def test_reference_stochastic():
    """Between two codes the mean over all random bits is the value, to a step of 2^-20."""
    u = np.arange(2 ** 20) / 2 ** 20
    for x in (1.03, 5.3e-3, -200.7, 0.0):
        got = ref.stochastic(np.full(2 ** 20, x), 0, u, False)
        assert abs(got.mean() - x) <= 2.0 ** -19 * max(abs(x), 2.0 ** -6)
    assert (ref.stochastic(np.full(4, 1e-9), 0, np.zeros(4), True) == 2.0 ** -9).all()


# ------------------------------------------------------------------------------------------------ sizes


def test_sizes(L):
    assert L.spl_fp8_codes_bytes(3, 129, 2) == 2 * 3 * 256 and L.spl_fp8_codes_bytes(1, 1, 1) == 128
    assert L.spl_fp8_scales_bytes(3, 129, 2, 1) == 2 * 3 * 4 and L.spl_fp8_scales_bytes(129, 640, 1, 128) == 2 * 8
    for rows, cols, count in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1, (1 << 22) + 1, 1), (1, 1, 65536),
                              (1 << 30, 1 << 22, 1)):
        assert L.spl_fp8_codes_bytes(rows, cols, count) == -1 and L.spl_fp8_scales_bytes(rows, cols, count, 1) == -1
    assert L.spl_fp8_scales_bytes(1, 1, 1, 2) == -1
    assert L.spl_fp8_grouped_cols(0, 4) == 128 and L.spl_fp8_grouped_cols(1, 4) == 128
    assert L.spl_fp8_grouped_cols(1 << 22, 60000) == -1 and L.spl_fp8_grouped_cols(-1, 1) == -1
    assert L.spl_linear_fp8_workspace_bytes(0, 1, 1) == -1 and L.spl_linear_fp8_rows_workspace_bytes(0, 1, 1) == 0
    assert L.spl_linear_fp8_grouped_rows_workspace_bytes(1, 1, 1, 0) == -1
    assert L.spl_linear_fp8_rows_workspace_bytes(500, 64, 100) >= 500 * 132


@pytest.mark.parametrize("rows,groups", [(1, 1), (5, 3), (300, 5), (1000, 64), (128, 200), (129, 1)])
def test_grouped_cols_holds_any_split(L, rows, groups):
    """The bound holds the worst split: as many groups as there are rows of one row past a multiple of 128 each."""
    rng = np.random.default_rng(rows)
    cols = L.spl_fp8_grouped_cols(rows, groups)
    for k in range(200):
        cuts = np.sort(rng.integers(0, rows + 1, groups - 1))
        n = np.diff(np.concatenate([[0], cuts, [rows]]))
        assert 128 * int(np.sum(-(-n // 128))) <= cols
    n = [1] * min(groups, rows)
    n[0] += rows - sum(n)
    assert 128 * sum(-(-v // 128) for v in n) <= cols


# ------------------------------------------------------------------------------------------------ refusals of the ABI


def _m(**kw):
    from paper_2405_03594_amd import _Fp8

    d = dict(codes=0x10000, scales=0x20000, rows=64, cols=256, count=1, codes_bytes=1 << 30, scales_bytes=1 << 30, block=1)
    d.update(kw)
    return _Fp8(**d)


P = ctypes.c_void_p
BAD = [dict(codes=0), dict(codes=0x10008), dict(scales=0), dict(scales=0x20002), dict(rows=0), dict(rows=1 << 31), dict(cols=0),
       dict(cols=1 << 23), dict(count=0), dict(count=70000), dict(block=0), dict(block=64), dict(codes_bytes=64 * 256 - 1),
       dict(scales_bytes=64 * 4 - 1)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_matrices(L, kw):
    Y, ok, bad = P(0x40000), _m(), _m(**kw)
    assert L.spl_linear_fp8(bad, ok, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8(ok, bad, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(P(0x50000), BF16, 4, 256, bad, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_grouped(ok, bad, P(0x60000), BF16, Y, None) == INVALID
    assert L.spl_linear_fp8_grouped_weight_grad(bad, ok, P(0x60000), 2, 100, F32, Y, None) == INVALID
    assert L.spl_dequantize_fp8(bad, F32, Y, None) == INVALID
    if "rows" not in kw and "cols" not in kw and "count" not in kw:
        assert L.spl_quantize_fp8(P(0x50000), BF16, 64, 256, 256, 1, None, 0, bad, None, None) == INVALID


def test_refused_products(L):
    Y, x, w = P(0x40000), _m(), _m(rows=100)
    assert L.spl_linear_fp8(None, w, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8(x, w, I8, Y, None, None) == UNSUPPORTED
    assert L.spl_linear_fp8(x, w, BF16, None, None, None) == INVALID
    assert L.spl_linear_fp8(x, w, BF16, P(0x40008), None, None) == INVALID
    assert L.spl_linear_fp8(x, _m(cols=257), BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8(x, _m(count=2), BF16, Y, None, None) == INVALID
    X = P(0x50000)
    assert L.spl_linear_fp8_rows(X, F32, 4, 256, w, BF16, Y, None, None) == UNSUPPORTED
    assert L.spl_linear_fp8_rows(X, BF16, 4, 255, w, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(X, BF16, -1, 256, w, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(X, BF16, 4, 256, _m(count=2), BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(None, BF16, 4, 256, w, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(P(0x50001), BF16, 4, 256, w, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_rows(X, BF16, 4000, 256, w, BF16, Y, None, None) == INVALID          # needs a workspace
    assert L.spl_linear_fp8_rows(X, BF16, 4000, 256, w, BF16, Y, P(0x70010), None) == INVALID
    assert L.spl_linear_fp8_rows(None, BF16, 0, 256, w, BF16, None, None, None) == OK            # no rows: nothing to do
    assert L.spl_linear_fp8_grouped_rows(X, BF16, 4, 256, w, None, BF16, Y, None, None) == INVALID
    assert L.spl_linear_fp8_grouped(x, w, P(0x60002), BF16, Y, None) == INVALID
    assert L.spl_linear_fp8_grouped(x, w, None, BF16, Y, None) == INVALID
    assert L.spl_linear_fp8_grouped_weight_grad(x, _m(cols=384), P(0x60000), 2, 100, F32, Y, None) == INVALID
    assert L.spl_linear_fp8_grouped_weight_grad(x, w, P(0x60000), 3, 300, F32, Y, None) == INVALID   # 256 columns are too few
    assert L.spl_linear_fp8_grouped_weight_grad(x, w, P(0x60000), 0, 100, F32, Y, None) == INVALID


def test_products_past_the_grids(L):
    """W of 2^28 rows, which the streaming kernels' grids do not hold; one row less is a size like others."""
    huge = dict(rows=1 << 28, codes_bytes=1 << 36, scales_bytes=1 << 36, cols=128)
    Y, x, starts, ws = P(0x7000000000000), _m(cols=128, rows=4, codes=P(0x6000000000000)), P(0x50000), P(0x5000000000000)
    w = _m(codes=P(0x1000000000000), scales=P(0x2000000000000), **huge)
    assert L.spl_linear_fp8(x, w, BF16, Y, ws, None) == UNSUPPORTED
    assert L.spl_linear_fp8_rows(P(0x50000), BF16, 4, 128, w, BF16, Y, ws, None) == UNSUPPORTED
    assert L.spl_linear_fp8_grouped(x, w, starts, BF16, Y, None) == UNSUPPORTED
    assert L.spl_linear_fp8_grouped_weight_grad(x, w, starts, 1, 100, BF16, Y, None) == UNSUPPORTED
    assert L.spl_linear_fp8_kernel(0, 4, 1 << 28, 128, 0, 0, BF16) == -1
    assert L.spl_linear_fp8_kernel(0, 4, (1 << 28) - 1, 128, 0, 0, BF16) == 1


def test_refused_shared_memory(L):
    """Results in the memory of what the same call reads or writes: refused before anything runs (64 x 256 codes at 0x10000
    are 0x4000 bytes, 64 x 4 scales at 0x20000 are 0x100)."""
    x, w = _m(codes=P(0x100000), scales=P(0x110000)), _m()
    starts = P(0x600000)
    for y in (0x100000, 0x103ff0, 0x110000, 0x10000, 0x13ff0, 0x20000, 0xff010, 0x10010):
        assert L.spl_linear_fp8(x, w, BF16, P(y), None, None) == INVALID, hex(y)
        assert L.spl_linear_fp8_grouped(x, w, starts, BF16, P(y), None) == INVALID, hex(y)
    X = P(0x50000)                                            # 4 rows of 256, 300 apart: 3 * 600 + 512 bytes
    for y in (0x50000, 0x50900, 0x4fe10, 0x10000, 0x20000):
        assert L.spl_linear_fp8_rows(X, BF16, 4, 300, w, BF16, P(y), None, None) == INVALID, hex(y)
        assert L.spl_linear_fp8_grouped_rows(X, BF16, 4, 300, w, starts, BF16, P(y), None, None) == INVALID, hex(y)
    q = L.spl_quantize_fp8
    t = _m(rows=256, cols=64, codes=P(0x200000), scales=P(0x300000))
    assert q(P(0x10000), BF16, 64, 256, 256, 1, None, 0, w, None, None) == INVALID
    assert q(P(0x1fe00), BF16, 64, 256, 256, 1, None, 0, w, None, None) == INVALID           # its scales
    assert q(P(0x200000), BF16, 64, 256, 256, 1, None, 0, w, t, None) == INVALID
    assert q(P(0x700000), BF16, 64, 256, 256, 1, None, 0, w, _m(rows=256, cols=64), None) == INVALID   # both at one place
    g = L.spl_linear_fp8_grad                                 # M 64, N 256, K 64: dX 0x2000 bytes, dW 0x10000
    a = (P(0x700000), 256, P(0x800000), 64, BF16, 64, _m())
    ws = P(0x900000)
    for dx, dw in ((0x400000, 0x401000), (0x10000, 0x400000), (0x400000, 0x20000), (0x900000, 0x400000)):
        assert g(*a, None, F32, P(dx), P(dw), ws, None) == INVALID, (hex(dx), hex(dw))
    assert L.spl_linear_fp8_grouped_weight_grad(x, w, starts, 1, 100, F32, P(0x10000), None) == INVALID
    assert L.spl_dequantize_fp8(w, F32, P(0x13ff0), None) == INVALID


def test_refused_quantize(L):
    X, o, t = P(0x50000), _m(), _m(rows=256, cols=64)
    q = L.spl_quantize_fp8
    assert q(X, I8, 64, 256, 256, 1, None, 0, o, None, None) == UNSUPPORTED
    assert q(X, BF16, 64, 256, 256, 1, None, 0, None, None, None) == INVALID
    assert q(X, BF16, 64, 256, 255, 1, None, 0, o, None, None) == INVALID
    assert q(None, BF16, 64, 256, 256, 1, None, 0, o, None, None) == INVALID
    assert q(P(0x50002), F32, 64, 256, 256, 1, None, 0, o, None, None) == INVALID
    assert q(X, BF16, 65, 256, 256, 1, None, 0, o, None, None) == INVALID
    assert q(X, BF16, 64, 256, 256, 2, None, 0, o, None, None) == INVALID
    assert q(X, BF16, 64, 256, 256, 1, None, 0, o, o, None) == INVALID
    assert q(X, BF16, 64, 256, 256, 1, None, 0, o, _m(rows=256, cols=64, block=128), None) == INVALID
    assert q(X, BF16, 64, 256, 256, 1, P(0x60000), 2, o, t, None) == INVALID                   # too few columns for 2 groups
    assert q(X, BF16, 64, 256, 256, 1, P(0x60000), 0, o, None, None) == INVALID
    assert q(X, BF16, (1 << 22) + 1, 1, 1, 1, None, 0, _m(rows=(1 << 22) + 1, cols=1), None, None) == UNSUPPORTED
    assert q(None, BF16, 0, 256, 256, 1, None, 0, o, None, None) == OK


def test_refused_adamw(spl, L):
    T, Y = spl._AdamwTensor, spl._AdamwTypes
    good = dict(param=0x1000, grad=0x2000, m=0x3000, v=0x4000, n=16, decay=0.1)
    types = Y(F32, F32, 0, 32)

    def refused(ty=types, **kw):
        rows = (T * 1)(T(**dict(good, **kw)))
        return L.spl_adamw_plan_bytes(rows, 1, ty)

    assert refused() > 0
    for kw in (dict(param=None), dict(param=0x1002), dict(grad=None), dict(m=None), dict(v=0x4001), dict(n=-1), dict(n=1 << 41),
               dict(decay=math.inf), dict(decay=math.nan), dict(n=1 << 39)):
        assert refused(**kw) == -1, kw
    assert refused(Y(I8, F32, 0, 32)) == refused(Y(F32, F32, 0, 16)) == refused(Y(F32, F32, F32, 32)) == -1
    assert refused(Y(F32, F32, BF16, 32)) == -1                               # no copy given
    assert refused(Y(F32, F32, 0, 8)) == -1                                   # no scales given
    rows = (T * 2)(T(**good), T(**dict(good, param=0x1010, grad=0x2000, m=0x5000, v=0x6000)))
    host = (ctypes.c_uint8 * int(L.spl_adamw_plan_bytes(rows, 2, types)))()
    assert L.spl_adamw_plan(rows, 2, types, host) == INVALID                  # the params overlap
    rows[1].param = 0x1040
    assert L.spl_adamw_plan(rows, 2, types, host) == OK                       # gradients may be shared
    rows[1].m = 0x2020
    assert L.spl_adamw_plan(rows, 2, types, host) == INVALID                  # a state inside the gradient
    step = lambda **kw: L.spl_adamw_step(*[dict(dict(plan=P(0x1000), chunks=1, ty=types, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1,  # noqa: E731
                                                     dev=None, scale=None, seed=0, stream=None), **kw)[k]
                                           for k in ("plan", "chunks", "ty", "lr", "b1", "b2", "eps", "step", "dev", "scale",
                                                     "seed", "stream")])
    for kw in (dict(plan=None), dict(plan=P(0x1008)), dict(chunks=-1), dict(chunks=1 << 24), dict(lr=math.nan), dict(b1=1.0),
               dict(b1=-0.1), dict(b2=1.0), dict(eps=-1.0), dict(eps=math.inf), dict(step=0), dict(step=1 << 31),
               dict(dev=P(0x1002)), dict(scale=P(0x1001)), dict(ty=Y(F32, F32, 0, 7)), dict(ty=None)):
        assert step(**kw) == INVALID, kw
    assert step(plan=None, chunks=0) == OK


# ------------------------------------------------------------------------------------------------ the wrappers


def _cpu_matrix(spl, rows=64, cols=256, block=1, count=None):
    lead = () if count is None else (count,)
    pitch = -(-cols // 128) * 128
    codes = torch.zeros((*lead, rows, pitch), dtype=torch.uint8)
    scales = torch.zeros((*lead, -(-rows // block), -(-(pitch // 128) // 4) * 4), dtype=torch.uint8)
    return spl.Fp8Matrix(codes, scales, cols, block)


def test_matrix_checks(spl):
    m = _cpu_matrix(spl, 130, 300, 128)
    assert (m.rows, m.cols, m.count, m.block) == (130, 300, 1, 128) and m.block_scales().shape == (2, 3)
    assert _cpu_matrix(spl, 4, 300, 1, 3).count == 3
    c, s = m.codes, m.scales
    for args in ((c[:, :256], s, 300, 128), (c.float(), s, 300, 128), (c, s[:, :3], 300, 128), (c, s.int(), 300, 128),
                 (c, s, 300, 1), (c, s, 300, 64), (c, s, 0, 128), (c, s, 400, 128), (c[0], s, 300, 128), (c[:, ::2], s, 150, 128)):
        with pytest.raises(ValueError):
            spl.Fp8Matrix(*args)
    m.codes = m.codes[:100]                            # a call sees what the matrix is now
    with pytest.raises(ValueError):
        m.view()
    with pytest.raises(ValueError):
        spl.Fp8Matrix.empty(0, 5, device="cpu")


def test_matrix_of(spl):
    codes = torch.randint(0, 126, (2, 10, 300), dtype=torch.uint8)
    scales = torch.randint(0, 255, (2, 10, 3), dtype=torch.uint8)
    m = spl.Fp8Matrix.of(codes, scales, 300, 1)
    assert torch.equal(m.codes[..., :300], codes) and (m.codes[..., 300:] == 0).all()
    assert torch.equal(m.block_scales(), scales) and m.codes.shape == (2, 10, 384) and m.scales.shape == (2, 10, 4)
    whole = torch.zeros((4, 512), dtype=torch.float8_e4m3fn)
    same = spl.Fp8Matrix.of(whole, torch.zeros((1, 4), dtype=torch.uint8), 512, 128)
    assert same.codes.data_ptr() == whole.data_ptr()
    for args in ((codes, scales, 301, 1), (codes, scales, 250, 1), (codes, scales[:, :9], 300, 1), (codes.int(), scales, 300, 1),
                 (codes, scales, 300, 2)):
        with pytest.raises(ValueError):
            spl.Fp8Matrix.of(*args)


def test_matrix_of_clears_the_padding(spl):
    """Codes wider than the matrix may hold anything behind its columns; a product reads whole blocks."""
    codes = torch.full((3, 256), 0x7f, dtype=torch.uint8)      # NaN codes
    codes[:, :200] = 0x38
    scales = torch.full((3, 2), 127, dtype=torch.uint8)
    for given in (codes, torch.cat([codes, codes], 1)):
        m = spl.Fp8Matrix.of(given, scales, 200, 1)
        assert m.codes.shape == (3, 256) and (m.codes[:, 200:] == 0).all() and (m.codes[:, :200] == 0x38).all()
    assert (codes[:, 200:] == 0x7f).all()


def test_wrappers_refuse(spl):
    x, w = torch.zeros((4, 256), dtype=torch.bfloat16), _cpu_matrix(spl)
    starts = torch.zeros(4, dtype=torch.int32)
    many = _cpu_matrix(spl, count=3)
    calls = [
        lambda: spl.quantize_fp8(x), lambda: spl.quantize_fp8(x.double()), lambda: spl.quantize_fp8(x[0]),
        lambda: spl.quantize_fp8(x, block=2), lambda: spl.quantize_fp8(x.t()), lambda: spl.quantize_fp8(x[:0]),
        lambda: spl.quantize_fp8(x, starts=starts), lambda: spl.quantize_fp8_both(x, block=128, starts=starts),
        lambda: spl.quantize_fp8_both(x[None], starts=starts), lambda: spl.quantize_fp8_both(x, starts=starts.long()),
        lambda: spl.quantize_fp8_both(x, starts=starts[:1]), lambda: spl.quantize_fp8(x[:, :0]),
        lambda: spl.quantize_fp8(torch.zeros((1, 4)).expand(3, 4)),
        lambda: spl.dequantize_fp8(w), lambda: spl.dequantize_fp8(w, torch.int8),
        lambda: spl.linear_fp8(x, w), lambda: spl.linear_fp8(x[:, :255], w), lambda: spl.linear_fp8(x.float(), w),
        lambda: spl.linear_fp8(x, many), lambda: spl.linear_fp8(_cpu_matrix(spl, cols=384), w), lambda: spl.linear_fp8(w, w),
        lambda: spl.linear_fp8_grouped(x, many, starts[:3]), lambda: spl.linear_fp8_grouped(x, many, starts),
        lambda: spl.linear_fp8_grouped(x, many, starts.float()), lambda: spl.linear_fp8_grouped(many, many, starts),
        lambda: spl.linear_fp8_grad(x, x, w), lambda: spl.linear_fp8_grad(x[:2], x, w),
        lambda: spl.linear_fp8_grad(x[:, :64].float(), x, _cpu_matrix(spl, 256, 64)),
        lambda: spl.linear_fp8_grad(x[:, :64], x, _cpu_matrix(spl, 256, 64), grad_dtype=torch.int8),
        lambda: spl.linear_fp8_grad(x[:, :64], x, _cpu_matrix(spl, 256, 64)),
        lambda: spl.linear_fp8_grouped_grad(x[:, :64], x, _cpu_matrix(spl, 256, 64, count=3), starts),
        lambda: spl.linear_fp8_grouped_grad(x[:, :64], x, _cpu_matrix(spl, 256, 64, count=3), starts[:2]),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i}")


def test_adamw_wrappers_refuse(spl):
    t = lambda n=8, dt=torch.float32: torch.zeros(n, dtype=dt)  # noqa: E731
    eight = spl.Fp8Vector.zeros(8, device="cpu")
    calls = [
        lambda: spl.adamw_plan([t()], [t()], [t()], [t()]),                       # host tensors
        lambda: spl.adamw_plan([t()], [t(), t()], [t()], [t()]), lambda: spl.adamw_plan([t()], [t(9)], [t()], [t()]),
        lambda: spl.adamw_plan([t()], [t()], [t(dt=torch.bfloat16)], [t()]), lambda: spl.adamw_plan([t(dt=torch.int32)], [t()], [t()], [t()]),
        lambda: spl.adamw_plan([t(), t(dt=torch.bfloat16)], [t(), t()], [t(), t()], [t(), t()]),
        lambda: spl.adamw_plan([t()], [t()], [eight], [t()]), lambda: spl.adamw_plan([t(9)], [t(9)], [eight], [eight]),
        lambda: spl.adamw_plan([t()], [t()], [t()], [t()], weight_decay=[0.1, 0.2]),
        lambda: spl.adamw_plan([t()], [t()], [t()], [t()], copies=[t()]), lambda: spl.adamw_plan([t(16)[::2]], [t()], [t()], [t()]),
        lambda: spl.Fp8Vector(torch.zeros(100, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8), 100),
        lambda: spl.Fp8Vector(torch.zeros(128, dtype=torch.uint8), torch.zeros(2, dtype=torch.uint8), 100),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i}")
    empty = spl.adamw_plan([], [], [], [])
    spl.adamw_step(empty, 1e-3)                                                    # nothing to do
    with pytest.raises(ValueError):
        spl.adamw_step(empty, 1e-3, step=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        spl.adamw_step(empty, 1e-3, grad_scale=torch.zeros(1, dtype=torch.float64))
