"""Every kernel of the 8-bit float products on the GPU, at ragged sizes that reach it (which sizes reach which kernel is held
by test_fp8_kernels_host.py): small integers, whose sums are exact in every type; random values against 64 bits; a NaN.

Tolerances are those of test_gpu_fp8.py: half a unit of the result's last place, 2^-9 of the largest product of each block
for the sums of 16-bit results, (K + 2) 2^-24 of the sum of magnitudes for fp32 ones."""
import numpy as np
import pytest
import torch

import _fp8_cases as cases
import _fp8_ref as ref

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
CODE = {torch.float16: 1, torch.bfloat16: 2, torch.float32: 5}
FLOATS = [torch.bfloat16, torch.float16, torch.float32]


def _spl():
    import paper_2405_03594_amd as spl

    return spl


def _np(t):
    return t.detach().cpu().double().numpy()


def _held(q):
    """What a quantized matrix stands for, from its codes and scales."""
    codes, scale = q.codes.cpu().numpy(), q.block_scales().cpu().numpy()
    if codes.ndim == 2:
        return ref.held(codes, scale, q.block, q.cols)
    return [ref.held(c, s, q.block, q.cols) for c, s in zip(codes, scale)]


def _random(shape, seed):
    """Values over several powers of two, rows and columns of unequal size, so small that no product's sum leaves fp16."""
    g = torch.Generator().manual_seed(seed)
    return 2.0 ** -5 * torch.randn(shape, generator=g) * torch.exp(torch.randn((*shape[:-1], 1), generator=g)) * torch.exp(
        0.5 * torch.randn((shape[-1],), generator=g))


def _small(M, N, K, seed):
    """Integers whose products' sums stay within 256, which every type holds."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-2, 3, (M, K), generator=g).float()
    w = torch.randint(-1, 2, (N, K), generator=g).float() * (torch.rand((N, K), generator=g) < 0.1)
    return x, w


def _tops(x):
    """The largest magnitude of each row's blocks of 128 columns."""
    x = np.abs(np.pad(x, ((0, 0), (0, -x.shape[1] % 128))))
    return x.reshape(len(x), -1, 128).max(2)


def _check(got, x, w, what):
    """got is x w^T of the held values, rounded once."""
    dtype, K = got.dtype, x.shape[1]
    want, sizes = x @ w.T, np.abs(x) @ np.abs(w).T
    if dtype == torch.float32:
        bound = EPS[dtype] * ((K + 2) * sizes) + 1e-38
    else:
        tiny = 2.0 ** -24 if dtype == torch.float16 else 1e-38
        bound = EPS[dtype] * np.abs(want) * (1 + 2.0 ** -7) + 2.0 ** -9 * (_tops(x) @ _tops(w).T) + K / 128 * 2.0 ** -24 * sizes + tiny
    off = np.abs(_np(got) - want)
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, first {np.argwhere(bad)[0]}, worst {np.nanmax(off / bound):.2f}"


def _reaches(form, M, N, K, groups, x, dtype, want):
    spl = _spl()
    got = spl.lib().spl_linear_fp8_kernel(form, M, N, K, groups, x, CODE[dtype])
    assert got == want, f"this device takes kernel {got}, not {want}"


def _id(case):
    return "-".join(str(len(v) - 1) + "groups" if isinstance(v, list) else str(v) for v in case)


@pytest.mark.parametrize("case", cases.CODES, ids=_id)
def test_codes(case):
    spl = _spl()
    M, N, K, k16, k32 = case
    x, w = _small(M, N, K, M + N)
    whole = x @ w.T                                    # exact: whole numbers far below 2^24
    assert whole.abs().max() <= 256
    q, qw = spl.quantize_fp8(x.cuda()), spl.quantize_fp8(w.cuda(), 128)
    r, rw = spl.quantize_fp8(_random((M, K), 1).cuda()), spl.quantize_fp8(_random((N, K), 2).cuda(), 1)
    hr, hrw = _held(r), _held(rw)
    for dtype in FLOATS:
        _reaches(0, M, N, K, 0, 0, dtype, k32 if dtype == torch.float32 else k16)
        assert torch.equal(spl.linear_fp8(q, qw, dtype=dtype).cpu(), whole.to(dtype)), dtype
        out = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
        y = spl.linear_fp8(r, rw, out=out)
        _check(y, hr, hrw, f"{dtype}")
        assert torch.equal(spl.linear_fp8(r, rw, dtype=dtype), y), dtype      # the same bits again
    # a NaN in one row of X and one of W is in that row and that column, nowhere else
    at, to = M - 1, N // 2
    x[at, K - 1], w[to, K // 2] = float("nan"), float("inf")
    q, qw = spl.quantize_fp8(x.cuda()), spl.quantize_fp8(w.cuda(), 1)
    for dtype in FLOATS:
        y = spl.linear_fp8(q, qw, dtype=dtype).cpu()
        assert torch.isnan(y[at]).all() and torch.isnan(y[:, to]).all(), dtype
        y[at], y[:, to] = 0, 0
        clean = whole.to(dtype)
        clean[at], clean[:, to] = 0, 0
        assert torch.equal(y, clean), dtype


@pytest.mark.parametrize("xtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", cases.ROWS, ids=_id)
def test_rows(case, xtype):
    spl = _spl()
    M, N, K, k16, k32 = case
    x, w = _small(M, N, K, M + N)
    whole = x @ w.T
    assert whole.abs().max() <= 256
    qw, rw = spl.quantize_fp8(w.cuda(), 128), spl.quantize_fp8(_random((N, K), 2).cuda(), 1)
    wide = torch.zeros((M, K + 13), dtype=xtype)
    wide[:, 5:5 + K] = _random((M, K), 1).to(xtype)
    r = wide.cuda()[:, 5:5 + K]
    hr, hrw = _held(spl.quantize_fp8(r)), _held(rw)
    for dtype in FLOATS:
        _reaches(0, M, N, K, 0, CODE[xtype], dtype, k32 if dtype == torch.float32 else k16)
        assert torch.equal(spl.linear_fp8(x.to(xtype).cuda(), qw, dtype=dtype).cpu(), whole.to(dtype)), dtype
        _check(spl.linear_fp8(r, rw, dtype=dtype), hr, hrw, f"{dtype}, slice")
        _check(spl.linear_fp8(r.contiguous(), rw, dtype=dtype), hr, hrw, f"{dtype}")


@pytest.mark.parametrize("case", range(len(cases.GROUPED)))
def test_grouped(case):
    spl = _spl()
    starts, M, N, K, c16, c32, r16, r32 = cases.GROUPED[case]
    E = len(starts) - 1
    at = torch.tensor(starts, dtype=torch.int32).cuda()
    x, w = _small(M, E * N, K, M + N)
    w = w.view(E, N, K)
    r = _random((M, K), 1).to(torch.bfloat16)
    qw = spl.quantize_fp8(w.cuda(), 1)
    rw = spl.quantize_fp8(_random((E * N, K), 2).view(E, N, K).cuda(), 128)
    q, qr = spl.quantize_fp8(x.cuda()), spl.quantize_fp8(r.cuda())
    hr, hrw = _held(qr), _held(rw)
    owned = torch.zeros(M, dtype=torch.bool)
    owned[starts[0]:starts[-1]] = True
    for dtype in FLOATS:
        f32 = dtype == torch.float32
        for xt, given, values, kernel in ((0, q, qr, c32 if f32 else c16),
                                          (2, x.to(torch.bfloat16).cuda(), r.cuda(), r32 if f32 else r16)):
            _reaches(1, M, N, K, E, xt, dtype, kernel)
            out, y = (torch.full((M, N), 7.0, dtype=dtype, device="cuda") for _ in range(2))
            spl.linear_fp8_grouped(given, qw, at, out=out)
            spl.linear_fp8_grouped(values, rw, at, out=y)
            assert (out.cpu()[~owned] == 7.0).all() and (y.cpu()[~owned] == 7.0).all()
            for e, (a, b) in enumerate(zip(starts, starts[1:])):
                if b > a:
                    whole = x[a:b] @ w[e].T
                    assert whole.abs().max() <= 256 and torch.equal(out[a:b].cpu(), whole.to(dtype)), (dtype, e)
                    _check(y[a:b], hr[a:b], hrw[e], f"{dtype}, expert {e}")


@pytest.mark.parametrize("case", range(len(cases.SUMS)))
def test_weight_grad(case):
    """The sums over an expert's tokens; integers whose sums over the tokens stay within 256 (a twentieth of dY is not zero)."""
    spl = _spl()
    starts, N, K, T, k16, k32 = cases.SUMS[case]       # dY [T][N], X [T][K]
    E = len(starts) - 1
    at = torch.tensor(starts, dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(case)
    dy = torch.randint(-1, 2, (T, N), generator=g).float() * (torch.rand((T, N), generator=g) < 0.05)
    x = torch.randint(-2, 3, (T, K), generator=g).float()
    rdy, rx = _random((T, N), 1), _random((T, K), 2)
    trans = lambda t: spl.quantize_fp8(t.cuda(), transposed=True, starts=at)  # noqa: E731
    a, b, ra, rb = trans(dy), trans(x), trans(rdy), trans(rx)
    ha, hb = _held(ra), _held(rb)
    for dtype in FLOATS:
        _reaches(2, N, K, T, E, 0, dtype, k32 if dtype == torch.float32 else k16)
        dw, rw = (spl.linear_fp8_grouped_weight_grad(p, q, at, T, dtype=dtype) for p, q in ((a, b), (ra, rb)))
        assert dw.shape == (E, N, K) and dw.dtype == dtype
        block = 0
        for e, (s, t) in enumerate(zip(starts, starts[1:])):
            whole = dy[s:t].T @ x[s:t]
            assert torch.equal(dw[e].cpu(), whole.to(dtype)), (dtype, e)
            cols = slice(128 * block, 128 * block + t - s)
            if t > s:
                assert whole.abs().max() <= 256
                _check(rw[e], ha[:, cols], hb[:, cols], f"{dtype}, expert {e}")
            else:
                assert (rw[e] == 0).all()
            block += -(-(t - s) // 128)


def test_gradients_take_them_too():
    """Both gradients at a size whose dX and dW take the large kernels, and at one whose sums are split, are those of the
    calls that they stand for, bit for bit."""
    spl = _spl()
    for M, N, K in ((2051, 2306, 1302), (66, 4100, 300), (4100, 70, 66)):
        x, dy = _random((M, K), 1).to(torch.bfloat16).cuda(), _random((M, N), 2).to(torch.bfloat16).cuda()
        _, wt = spl.quantize_fp8_both(_random((N, K), 3).cuda(), 128)
        q, qt = spl.quantize_fp8_both(dy)
        xt = spl.quantize_fp8(x, transposed=True)
        for dt in FLOATS:
            dx, dw = spl.linear_fp8_grad(dy, x, wt, grad_dtype=dt)
            assert torch.equal(dx, spl.linear_fp8(q, wt)) and torch.equal(dw, spl.linear_fp8(qt, xt, dtype=dt)), (M, dt)
        _check(dx, _held(q), _held(wt), "dX")
        _check(dw, _held(qt), _held(xt), "dW")


def test_split_sums_and_tiles_in_graphs():
    """Calls with a workspace and of the large tiles in two captured graphs, replayed in turn with eager calls of the same
    sizes between: each has the eager result's bits every time."""
    spl = _spl()
    sizes = [(100, 257, 4096), (2051, 2306, 1302)]
    ws = [spl.quantize_fp8(_random((N, K), 1).cuda(), 128) for _, N, K in sizes]
    xs = [[_random((M, K), 5 + s).to(torch.bfloat16).cuda() for s in range(3)] for M, _, K in sizes]
    eager = [[spl.linear_fp8(x, w) for x in some] for some, w in zip(xs, ws)]
    held = [x[0].clone() for x in xs]
    torch.cuda.synchronize()
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append([spl.linear_fp8(x, w) for x, w in zip(held, ws)])
        graphs.append(g)
    for r in (1, 2, 0, 1):
        for h, x in zip(held, xs):
            h.copy_(x[r])
        for g, out in zip(graphs, got):
            g.replay()
            assert torch.equal(spl.linear_fp8(xs[0][2], ws[0]), eager[0][2])
            torch.cuda.synchronize()
            assert all(torch.equal(a, e[r]) for a, e in zip(out, eager)), r


@pytest.mark.parametrize("M,N,K,k16,k32", [c for c in cases.CODES if c[3] in (1, 9, 3, 16, 17, 18, 19, 20, 22)][::2], ids=str)
def test_sums_that_cancel(M, N, K, k16, k32):
    """What the documents say of sums whose products cancel: those of fp32 results keep what is left, those of 16-bit
    results are off by up to 2^-9 of each block's largest product.  In each whole block of 128 two products of 2^16 cancel
    and the other 126 are 2^-2 each, 31.5 in all: exact in fp32 (the sums on the way are multiples of 2^-2 below 2^18)."""
    spl = _spl()
    K = K // 128 * 128
    x, w = torch.full((M, K), 2.0 ** -2), torch.ones((N, K))
    for k in range(0, K, 128):
        x[:, k + 3], x[:, k + 77] = 256.0, -256.0
        w[:, k + 3] = w[:, k + 77] = 256.0
    q, qw = spl.quantize_fp8(x.cuda()), spl.quantize_fp8(w.cuda(), 128)
    assert np.array_equal(_held(q), _np(x)) and np.array_equal(_held(qw), _np(w))      # codes hold the values
    want = 31.5 * (K // 128)
    assert (spl.linear_fp8(q, qw, dtype=torch.float32) == want).all()
    for dtype in (torch.bfloat16, torch.float16):
        y = _np(spl.linear_fp8(q, qw, dtype=dtype))
        bound = 2.0 ** -9 * 2.0 ** 16 * (K // 128) * (1 + EPS[dtype]) + EPS[dtype] * want
        assert (np.abs(y - want) <= bound).all(), (dtype, np.abs(y - want).max(), bound)


@pytest.mark.parametrize("case", [c for c in cases.CODES if c[3] in (1, 10, 3, 16, 17, 18, 19, 20, 22)][1::2], ids=_id)
def test_both_operands_in_wide_blocks(case):
    """X with a scale for 128 x 128 entries too, and a matrix times its own transpose."""
    spl = _spl()
    M, N, K, k16, k32 = case
    q, qw = spl.quantize_fp8(_random((M, K), 1).cuda(), 128), spl.quantize_fp8(_random((N, K), 2).cuda(), 128)
    h, hw = _held(q), _held(qw)
    for dtype in FLOATS:
        _check(spl.linear_fp8(q, qw, dtype=dtype), h, hw, f"{dtype}")
    _check(spl.linear_fp8(qw, qw, dtype=torch.float32), hw, hw, "W W^T")
