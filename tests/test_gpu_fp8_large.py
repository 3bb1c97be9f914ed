"""8-bit float products past what one launch holds: 2^22 tiles, 65535 tiles of rows along a grid's second axis, 2^32 threads.
The inputs repeat themselves, so that the results are those of a small call over and over."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

PERIOD = 4099                                         # rows after which the inputs repeat; prime to every tile


@pytest.fixture(autouse=True)
def _memory():
    """Tens of GB for a moment; other tests get them back."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def _spl():
    import paper_2405_03594_amd as spl

    return spl


def _repeat(small, rows):
    """small [PERIOD, ...] over and over, `rows` rows, without a temporary of that size."""
    out = torch.empty((rows, *small.shape[1:]), dtype=small.dtype, device="cuda")
    whole = rows // PERIOD
    out[:whole * PERIOD].view(whole, *small.shape).copy_(small.expand(whole, *small.shape))
    out[whole * PERIOD:] = small[:rows - whole * PERIOD]
    return out


def _repeats(big, small):
    rows = big.shape[0]
    whole = rows // PERIOD
    step = 4096
    for a in range(0, whole, step):
        b = min(whole, a + step)
        part = big[a * PERIOD:b * PERIOD].view(b - a, *small.shape)
        if not (part == small).all():
            return False
    return bool((big[whole * PERIOD:] == small[:rows - whole * PERIOD]).all())


@pytest.mark.parametrize("M,kernel", [((1 << 28) + 777, 16)])
def test_more_tiles_than_a_launch(M, kernel):
    """2^22 tiles of 64 rows and 13 more."""
    spl = _spl()
    assert spl.lib().spl_linear_fp8_kernel(0, M, 2, 100, 0, 0, 2) == kernel and M // 64 > 1 << 22
    g = torch.Generator(device="cuda").manual_seed(1)
    small = spl.quantize_fp8(torch.randn((PERIOD, 100), generator=g, device="cuda"))
    w = spl.quantize_fp8(torch.randn((2, 100), generator=g, device="cuda"))
    want = spl.linear_fp8(small, w, dtype=torch.bfloat16)
    x = spl.Fp8Matrix(_repeat(small.codes, M), _repeat(small.scales, M), 100, 1)
    assert _repeats(spl.linear_fp8(x, w, dtype=torch.bfloat16), want)


@pytest.mark.parametrize("rows16", [False, True])
def test_more_experts_than_a_grid(rows16):
    """50000 experts of six rows: the streaming kernels may need 65625 tiles of 16 rows."""
    spl = _spl()
    E, N, K = 50000, 20, 1136
    M = 6 * E
    kernel = spl.lib().spl_linear_fp8_kernel(1, M, N, K, E, 2 if rows16 else 0, 5)
    assert kernel in (1, 5) and (M + 15 * E) // 16 > 65535
    g = torch.Generator(device="cuda").manual_seed(2)
    w = spl.quantize_fp8(torch.randn((1, N, K), generator=g, device="cuda").expand(E, N, K).contiguous())
    w.codes[1::2] ^= 128                               # every other expert's weights with the other sign
    x = torch.randn((PERIOD, K), generator=g, device="cuda").to(torch.bfloat16)
    one = spl.Fp8Matrix(w.codes[0].contiguous(), w.scales[0].contiguous(), K, 1)
    qx = spl.quantize_fp8(x)
    want = spl.linear_fp8(qx, one, dtype=torch.float32)
    given = _repeat(x, M)
    out = torch.full((M, N), 7.0, dtype=torch.float32, device="cuda")
    at = torch.arange(0, M + 1, 6, dtype=torch.int32, device="cuda")
    spl.linear_fp8_grouped(given if rows16 else spl.quantize_fp8(given), w, at, out=out)
    out.view(E, 6, N)[1::2] *= -1
    # two fp32 sums of K products in different orders
    sizes = spl.dequantize_fp8(qx).abs() @ spl.dequantize_fp8(one).abs().T
    assert ((out - _repeat(want, M)).abs() <= _repeat(2 * (K + 2) * 2.0 ** -24 * sizes * (1 + 2.0 ** -10), M)).all()


def test_more_values_than_a_launch():
    """dequantize_fp8 of 2^35 values and some."""
    spl = _spl()
    rows, cols = (1 << 28) + 55, 127
    assert rows * 16 > ((1 << 24) - 1) * 256          # pieces of 8 values, threads of a launch
    g = torch.Generator(device="cuda").manual_seed(3)
    small = spl.quantize_fp8(torch.randn((PERIOD, cols), generator=g, device="cuda"))
    x = spl.Fp8Matrix(_repeat(small.codes, rows), _repeat(small.scales, rows), cols, 1)
    got = spl.dequantize_fp8(x, torch.bfloat16)
    assert _repeats(got, spl.dequantize_fp8(small, torch.bfloat16))
