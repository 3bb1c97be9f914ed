"""AdamW bit for bit: the formula of spl_adamw_step in numpy's float32, whose every product, sum, quotient and root is
rounded to nearest by itself; the factors in 64 bits, rounded once.  No tolerance: the same operations in the same order
have one result.  Plans of few elements and of many, which cut their tensors into chunks of 2048 and of 8192."""
import math

import numpy as np
import pytest
import torch

import _fp8_ref as ref

pytestmark = pytest.mark.gpu

F = np.float32
LR, B1, B2, EPS, DECAY, SEED = 1e-2, 0.9, 0.99, 1e-6, 0.1, 99


def _spl():
    import paper_2405_03594_amd as spl

    return spl


def update(p, g, m, v, step, scale, decay=DECAY):
    """(p, m, v, sqrt(v)) in float32."""
    assert all(t.dtype == F for t in (p, g, m, v))
    keep, rate = F(1.0 - LR * decay), F(LR / (1.0 - B1 ** step))
    root = F(1.0 / math.sqrt(1.0 - B2 ** step))
    b1, c1, b2, c2, eps = F(B1), F(1.0 - B1), F(B2), F(1.0 - B2), F(EPS)
    with np.errstate(all="ignore"):
        if scale is not None:
            g = g * F(scale)
        m = m * b1 + g * c1
        v = v * b2 + (g * g) * c2
        r = np.sqrt(v)
        return p * keep - rate * (m / (r * root + eps)), m, v, r


def encode(x, rnd, keep):
    """(codes' values [n], bytes) of an 8-bit state, the rounding with 20 random bits each."""
    n, x = len(x), ref.blocks(x)
    rnd = ref.blocks(rnd.astype(np.uint32))
    top = np.abs(x).max(1).view(np.uint32)
    e = (top >> 23).astype(np.int64)
    byte = np.maximum(e - 8 + ((top & 0x7FFFFF) > 0x600000), 0)
    s = x * np.ldexp(F(1), 127 - byte).astype(F)[:, None]
    a = np.abs(s)
    large = ((a.view(np.uint32) + rnd) & np.uint32(0xFFF00000)).view(F)
    small = np.floor(a * F(512) + rnd.astype(F) * F(2.0 ** -20)) * F(2.0 ** -9)
    a = np.where(a < F(2.0 ** -6), small, large)
    if keep:
        a = np.where(x > 0, np.maximum(a, F(2.0 ** -9)), a)
    return np.copysign(a, x).reshape(-1)[:n], byte


def decode(codes, byte, n):
    return (ref.values(codes).astype(F).reshape(-1, 128) * np.ldexp(F(1), byte.astype(np.int64) - 127).astype(F)[:, None]).reshape(-1)[:n]


def _values(n, seed):
    g = torch.Generator().manual_seed(seed)
    wide = torch.exp(2 * torch.randn(n, generator=g))
    return [torch.randn(n, generator=g), torch.randn(n, generator=g) * 0.1 * wide, torch.randn(n, generator=g) * 0.1 * wide,
            torch.rand(n, generator=g) * 0.01 * wide * wide]


SMALL = [1, 5, 127, 128, 129, 2047, 2048, 2049, 20000]
# past 2048 x 2048 elements in all chunks hold 8192, in four turns; tensors that end in each turn and on both sides of a chunk
LARGE = [1, 127, 128, 2047, 2048, 2049, 4095, 4097, 6143, 6145, 8191, 8192, 8193, 8192 + 2049, 20000, 0, 4_190_003]


def _check(spl, sizes, pd, gd, bits, shift, scale):
    place = lambda t: torch.nn.functional.pad(t, (shift, 0)).cuda()[shift:] if shift else t.cuda()  # noqa: E731
    host = [_values(n, 10 + i) for i, n in enumerate(sizes)]
    host = [[h[0].to(pd), h[1].to(gd), h[2], h[3]] for h in host]
    p, g = ([place(h[k]) for h in host] for k in (0, 1))
    copies = [torch.full((n,), 3.0, dtype=torch.bfloat16, device="cuda") for n in sizes]
    if bits == 32:
        m, v = ([place(h[k]) for h in host] for k in (2, 3))
    else:
        start = []
        for h in host:
            if not len(h[0]):
                start.append([(np.zeros(0, np.uint8), np.zeros(0, np.uint8))] * 2)
                continue
            zero = np.zeros(len(h[0]), np.uint32)
            got = [encode(x.numpy(), zero, False) for x in (h[2], h[3].sqrt())]
            start.append([(ref.nearest(ref.blocks(a)).reshape(-1), b.astype(np.uint8)) for a, b in got])
        m, v = ([spl.Fp8Vector(torch.from_numpy(s[k][0]).cuda(), torch.from_numpy(s[k][1]).cuda(), n) for s, n in zip(start, sizes)]
                for k in (0, 1))
    plan = spl.adamw_plan(p, g, m, v, weight_decay=DECAY, copies=copies)
    step = 7
    spl.adamw_step(plan, LR, (B1, B2), EPS, step=step, seed=SEED, grad_scale=None if scale is None else torch.tensor([scale], device="cuda"))
    wrong = []

    def same(what, i, got, want):
        if not np.array_equal(got, want):
            wrong.append((what, sizes[i], int((got != want).sum())))

    for i, (h, n) in enumerate(zip(host, sizes)):
        if not n:
            continue
        p0, g0 = h[0].float().numpy(), h[1].float().numpy()
        if bits == 32:
            m0, v0 = h[2].numpy(), h[3].numpy()
        else:
            m0, r0 = (decode(c, b, n) for c, b in start[i])
            v0 = r0 * r0
        wp, wm, wv, wr = update(p0, g0, m0, v0, step, scale)
        wide = torch.from_numpy(wp)
        same("p", i, p[i].cpu().float().numpy(), wide.to(pd).float().numpy())
        same("copy", i, copies[i].cpu().float().numpy(), wide.to(torch.bfloat16).float().numpy())
        if bits == 32:
            same("m", i, m[i].cpu().numpy(), wm)
            same("v", i, v[i].cpu().numpy(), wv)
        else:
            for what, vec, x, rnd, keep in zip("mr", (m[i], v[i]), (wm, wr), ref.random20(n, SEED, step, i), (False, True)):
                a, b = encode(x, rnd, keep)
                same(what + " scales", i, vec.scales.cpu().numpy(), b)
                codes = vec.codes.cpu().numpy()
                same(what, i, ref.values(codes[:n]).astype(F), a)
                same(what + " past the end", i, codes[n:] & 127, np.zeros(len(codes) - n, np.uint8))
    assert not wrong, wrong


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pd,gd,shift,scale", [(torch.float32, torch.float32, 0, 0.37), (torch.float32, torch.bfloat16, 0, None),
                                               (torch.bfloat16, torch.float32, 1, 0.37), (torch.float16, torch.float16, 3, 3.0)])
def test_every_operation_is_rounded_by_itself(pd, gd, shift, scale, bits):
    _check(_spl(), SMALL, pd, gd, bits, shift, scale)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pd,gd,shift,scale", [(torch.float32, torch.bfloat16, 0, 0.37), (torch.bfloat16, torch.float32, 1, None)])
def test_many_elements(pd, gd, shift, scale, bits):
    """Chunks of 8192: later turns of a chunk's loop, ends in each of them, scales of blocks in them, bits of far elements."""
    spl = _spl()
    assert sum(LARGE) > 2048 * 2048
    _check(spl, LARGE, pd, gd, bits, shift, scale)


def test_chunks_of_a_plan():
    """Where the chunks change their length: 2048 x 2048 elements in all are still cut into 2048 each, one more into 8192."""
    spl = _spl()
    for n, chunks in ((2048 * 2048, 2048), (2048 * 2048 + 1, 513)):
        t = [torch.zeros(n, device="cuda") for _ in range(4)]
        t[1].fill_(1.0)
        plan = spl.adamw_plan(*[[x] for x in t])
        assert plan.chunks == chunks
        spl.adamw_step(plan, LR, (B1, B2), EPS, step=1)
        want = [torch.from_numpy(np.broadcast_to(x, n).copy()) for x in
                update(np.zeros(1, F), np.ones(1, F), np.zeros(1, F), np.zeros(1, F), 1, None, 0.01)[:3]]
        assert all(torch.equal(t[i].cpu(), w) for i, w in ((0, want[0]), (2, want[1]), (3, want[2]))), n
