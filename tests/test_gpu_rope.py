"""Norms of query and key heads with the rotation, the gradients, and what the 4-bit cache stores, on the GPU.

Tolerances.  A result is rounded once to the 16-bit type: half a unit in its last place, u |y|.  Before that each
element is a few fp32 operations: x r w (r from a sum of up to 256 squares, a root and a division: at most 16 roundings
of 2^-24), then two products and a sum: 24 roundings of the terms' size, 2^-19 of |a| + |b|, is more than they can do."""
import math

import pytest
import torch

import _attn_ref as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]


def _spl():
    import paper_2405_03594_amd as spl

    return spl


def _angles(rows, rot, seed=0):
    a = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.stack((a.cos(), a.sin()), -1).float()


def _make(T, H, Hk, D, rot, dt, seed, fused=False, weights=True, rows=50):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(T, H + 2 * Hk, D, generator=g) * torch.exp(torch.randn(1, H + 2 * Hk, 1, generator=g))
    qkv = qkv.to(dt)
    q, k, v = qkv.split([H, Hk, Hk], 1)
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dt) if weights else None for _ in range(2)]
    pos = torch.randint(0, rows, (T,), generator=g).int()
    rope = _angles(rows, rot) if rot else None
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    if fused:
        dev = qkv.cuda().split([H, Hk, Hk], 1)
    else:
        dev = [t.contiguous().cuda() for t in (q, k, v)]
    return (q, k, v), w, pos, rope, dev, [cuda(t) for t in w], pos.cuda(), cuda(rope)


def _near(got, want, mag, dt, what):
    bad = (got.cpu().double() - want).abs() > ref.UNIT[dt] * want.abs() + ref.STEP[dt] + 2.0 ** -19 * mag
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}"


def _mag(x, w, eps, rot):
    """|a| + |b| bound of what the rotation mixes: the largest normalised entry of the head, twice."""
    n = ref.norm_rope(x.double(), None if w is None else w.double(), eps, None, False)
    return (2 * n.abs().amax(-1, keepdim=True)).expand_as(n)


CASES = [
    # T, H, Hk, D, rot, interleaved, fused, weights
    (1, 1, 1, 8, 0, False, False, True), (1, 32, 32, 128, 128, False, False, True), (3, 5, 1, 16, 16, True, True, True),
    (7, 4, 2, 40, 32, False, False, True), (5, 6, 3, 64, 64, False, True, True), (5, 6, 3, 64, 32, True, False, True),
    (9, 24, 8, 96, 48, True, True, True), (9, 24, 8, 96, 96, False, True, True), (4, 3, 2, 72, 16, False, False, True),
    (33, 8, 8, 128, 64, False, True, True), (33, 9, 2, 128, 128, True, False, False), (2, 7, 7, 256, 256, False, True, True),
    (2, 7, 3, 256, 128, True, False, True), (6, 2, 2, 200, 112, False, False, True), (700, 32, 32, 128, 128, False, False, True),
    (17, 40, 4, 128, 0, False, False, True), (17, 40, 4, 128, 128, False, False, False)]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("case", CASES)
def test_forward(case, dt):
    T, H, Hk, D, rot, inter, fused, weights = case
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(T, H, Hk, D, rot, dt, 1, fused, weights)
    qo, ko = _spl().qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1], eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    cs = rope.double()[pos.long()] if rot else None
    for got, x, wt, nm in ((qo, q, w[0], "q"), (ko, k, w[1], "k")):
        assert got.is_contiguous() and got.dtype == dt
        want = ref.norm_rope(x.double(), None if wt is None else wt.double(), 1e-5, cs, inter)
        _near(got, want, _mag(x, wt, 1e-5, rot), dt, nm)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("case", CASES)
def test_gradient(case, dt):
    """dx by the formula; the extra terms (g w and xh mean(g w xh)) are bounded by r times the head's largest |g w|
    (|xh| mean |g w xh| <= sqrt(D) max |g w|).  dw is a sum of T heads fp32 terms: 2^-22 of the sum of their sizes for a
    handful of them in a row, growing with the root of their number at worst."""
    T, H, Hk, D, rot, inter, fused, weights = case
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(T, H, Hk, D, rot, dt, 2, fused, weights)
    g = torch.Generator().manual_seed(9)
    up = [torch.randn(x.shape, generator=g).to(dt) for x in (q, k)]
    spl = _spl()
    out = spl.qk_norm_rope_grad(up[0].cuda(), up[1].cuda(), dq, dk, dpos, drope, dw[0], dw[1], eps=1e-5,
                                interleaved=inter)
    again = spl.qk_norm_rope_grad(up[0].cuda(), up[1].cuda(), dq, dk, dpos, drope, dw[0], dw[1], eps=1e-5,
                                  interleaved=inter)
    torch.cuda.synchronize()
    cs = rope.double()[pos.long()] if rot else None
    for i, (x, wt) in enumerate(((q, w[0]), (k, w[1]))):
        want, want_w = ref.norm_rope_grad(up[i].double(), x.double(), None if wt is None else wt.double(), 1e-5, cs, inter)
        size = up[i].double().abs().amax(-1, keepdim=True) * 2
        if wt is not None:
            r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-5)
            size = size * r * wt.double().abs().max() * math.sqrt(D)
        _near(out[i], want, size.expand_as(want), dt, "dq dk"[3 * i:3 * i + 2])
        assert torch.equal(out[i], again[i])
        if wt is None:
            assert out[2 + i] is None
            continue
        xh = x.double() * r
        back = ref.norm_rope(up[i].double(), None, 0, None if cs is None else torch.stack((cs[..., 0], -cs[..., 1]), -1),
                             inter)
        total = (back * xh).abs().sum((0, 1)) + 2 * (xh.abs() * up[i].double().abs().amax(-1, keepdim=True)).sum((0, 1))
        n = x.shape[0] * x.shape[1]
        assert out[2 + i].dtype == torch.float32
        assert ((out[2 + i].cpu().double() - want_w).abs() <= 2.0 ** -22 * math.sqrt(8 + n) * total).all()
        assert torch.equal(out[2 + i], again[2 + i])


@pytest.mark.parametrize("dt", DTYPES)
def test_a_head_does_not_depend_on_its_company(dt):
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(300, 8, 2, 128, 128, dt, 3)
    spl = _spl()
    qo, ko = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    for t in (0, 17, 299):
        q1, k1 = spl.qk_norm_rope(dq[t:t + 1, 3:4].contiguous(), dk[t:t + 1, 1:].contiguous(), dpos[t:t + 1], drope, dw[0],
                                  dw[1])
        assert torch.equal(q1[0, 0], qo[t, 3]) and torch.equal(k1[0, 0], ko[t, 1])


def test_in_place_and_other_strides():
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(20, 6, 2, 64, 64, torch.bfloat16, 4)
    spl = _spl()
    qo, ko = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    # heads first in memory, and a row of padding between tokens
    hq = dq.transpose(0, 1).contiguous().transpose(0, 1)
    pad = torch.zeros(20, 2, 72, dtype=dk.dtype, device="cuda")
    pad[..., :64] = dk
    q2, k2 = spl.qk_norm_rope(hq, pad[..., :64], dpos, drope, dw[0], dw[1])
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    a, b = dq.clone(), dk.clone()
    spl.qk_norm_rope(a, b, dpos, drope, dw[0], dw[1], q_out=a, k_out=b)
    assert torch.equal(a, qo) and torch.equal(b, ko)


def test_positions_without_an_angle_give_nan_there_only():
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(6, 2, 2, 64, 32, torch.float16, 5)
    spl = _spl()
    good, _ = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    dpos = dpos.clone()
    dpos[1], dpos[4] = -1, 50
    qo, _ = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    for t in range(6):
        if t in (1, 4):
            assert torch.isnan(qo[t, :, :32]).all() and torch.equal(qo[t, :, 32:], good[t, :, 32:])
        else:
            assert torch.equal(qo[t], good[t])


def test_no_tokens():
    spl = _spl()
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(2, 2, 2, 64, 64, torch.float16, 6)
    qo, ko = spl.qk_norm_rope(dq[:0], dk[:0], dpos[:0], drope, dw[0], dw[1])
    assert qo.shape == (0, 2, 64)
    out = spl.qk_norm_rope_grad(dq[:0], dk[:0], dq[:0], dk[:0], dpos[:0], drope, dw[0], dw[1])
    torch.cuda.synchronize()
    assert (out[2] == 0).all() and (out[3] == 0).all()


# ---------------------------------------------------------------------------------------------- the cache


def _bits(t):
    return t.contiguous().view(torch.int16)


def _same(got, want):
    """Equal values, NaN where NaN."""
    got, want = got.cpu().double(), want
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 128])
def test_append_stores_the_rotated_keys_and_the_values(D, page, dt):
    spl = _spl()
    T, H, Hk = 77, 6, 3
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(T, H, Hk, D, D // 2, dt, 7, fused=True)
    pages = 12
    cache = spl.KVCache.empty(pages, Hk, D, page, dt)
    cache.data.fill_(0xA5)
    g = torch.Generator().manual_seed(1)
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    slots[5], slots[6] = -1, pages * page                        # not stored
    before = cache.data.clone()
    ko = torch.empty_like(dk, memory_format=torch.contiguous_format)
    qo = spl.qk_norm_rope_append(dq, dk, dv, dpos, drope, slots.cuda(), cache, dw[0], dw[1], k_out=ko)
    q1, k1 = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    assert torch.equal(_bits(qo), _bits(q1)) and torch.equal(_bits(ko), _bits(k1))
    keys, values = spl.cache_read(cache, slots.cuda())
    torch.cuda.synchronize()
    kept = torch.tensor([i for i in range(T) if i not in (5, 6)])
    _same(keys[kept.cuda()], ref.stored(ko.cpu()[kept]))
    _same(values[kept.cuda()], ref.stored(v[kept]))
    assert (keys[5:7] == 0).all() and (values[5:7] == 0).all()
    # only the slots' own bytes changed: what the others hold is what they held
    rest = torch.tensor(sorted(set(range(pages * page)) - set(slots.tolist()))).int().cuda()
    old = spl.KVCache(before, page, D, dt)
    for a, b in zip(spl.cache_read(cache, rest), spl.cache_read(old, rest)):
        assert torch.equal(_bits(a), _bits(b))


@pytest.mark.parametrize("dt", DTYPES)
def test_every_payload_is_stored_as_the_format_says(dt):
    """All 65536 payloads as values, each in a group with zeros and with random company, and groups on the halves between
    the format's values."""
    spl = _spl()
    g = torch.Generator().manual_seed(2)
    every = torch.arange(-32768, 32768).to(torch.int16).view(dt)
    a = torch.zeros(65536, 32, dtype=dt)
    a[torch.arange(65536), torch.arange(65536) % 32] = every
    b = every[torch.randperm(65536, generator=g)].view(2048, 32)                 # wild groups
    finite = every[torch.isfinite(every)]
    scale = finite[torch.randint(0, len(finite), (4096,), generator=g)].float()[:, None]
    halves = torch.tensor([0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7])
    c = (scale * halves[torch.randint(0, 16, (4096, 32), generator=g)] / 8).to(dt)
    groups = torch.cat((a, b, c))
    n = len(groups) // 4
    v = groups[: 4 * n].view(n, 1, 128)
    cache = spl.KVCache.empty(-(-n // 64), 1, 128, 64, dt)
    slots = torch.arange(n).int().cuda()
    spl.qk_norm_rope_append(v.cuda(), v.cuda(), v.cuda(), None, None, slots, cache)
    keys, values = spl.cache_read(cache, slots)
    torch.cuda.synchronize()
    sample = torch.randperm(4 * n, generator=g)[:6000]
    want = ref.stored(groups[sample])
    _same(keys.view(-1, 32)[sample.cuda()], want)
    _same(values.view(-1, 32)[sample.cuda()], want)


FEW = [(1500, 1, 1, 96, 96, False, True, True), (2500, 4, 1, 128, 64, True, False, True),
       (4001, 3, 1, 64, 32, True, True, True), (600, 1, 1, 256, 256, False, False, False),
       (9000, 2, 1, 40, 32, False, False, True)]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("case", FEW)
def test_few_heads_of_many_tokens(case, dt):
    """A wave's slots run on over the tokens: the forward pass and the gradient, and the bits of a call of many heads."""
    test_forward(case, dt)
    test_gradient(case, dt)
    T, _, _, D, rot, inter, _, _ = case
    _, _, _, _, (q, k, v), w, pos, rope = _make(T, 24, 24, D, rot, dt, 3)
    spl = _spl()
    args = dict(eps=1e-5, interleaved=inter)
    many = spl.qk_norm_rope(q, k, pos, rope, w[0], w[1], **args)
    few = spl.qk_norm_rope(q[:, 5:6], k[:, 7:8], pos, rope, w[0], w[1], **args)
    torch.cuda.synchronize()
    assert torch.equal(few[0], many[0][:, 5:6]) and torch.equal(few[1], many[1][:, 7:8])


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_few_heads_stored(D):
    """Slots of their own for each token of a wave, some of them none."""
    T, page, dt = 1500, 32, torch.bfloat16
    (q, k, v), w, pos, rope, (dq, dk, dv), dw, dpos, drope = _make(T, 3, 1, D, D, dt, 4)
    spl = _spl()
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(5))[:T].int()
    slots[::7] = -1
    slots[3::70] = pages * page + 5
    cache = spl.KVCache.empty(pages, 1, D, page, dt)
    ko = torch.empty_like(dk)
    qo = spl.qk_norm_rope_append(dq, dk, dv, dpos, drope, slots.cuda(), cache, dw[0], dw[1], k_out=ko)
    want = spl.qk_norm_rope(dq, dk, dpos, drope, dw[0], dw[1])
    keys, values = spl.cache_read(cache, slots.cuda())
    torch.cuda.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    held = (slots >= 0) & (slots < pages * page)
    _same(keys[held.cuda()], ref.stored(ko.cpu()[held]))
    _same(values[held.cuda()], ref.stored(v[held]))
    assert not keys[~held.cuda()].any() and not values[~held.cuda()].any()


def test_a_cache_past_four_gigabytes():
    spl = _spl()
    D, page, Hk = 128, 256, 8
    pages = (9 << 29) // (Hk * spl.kv_page_bytes(D, page)) + 3                   # 4.5 GiB
    data = torch.zeros(pages, Hk, spl.kv_page_bytes(D, page), dtype=torch.uint8, device="cuda")
    cache = spl.KVCache(data, page, D, torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(4, Hk, D, generator=g).bfloat16()
    slots = torch.tensor([0, 5, pages * page - 1, (pages - 2) * page + 100]).int().cuda()
    spl.qk_norm_rope_append(x.cuda(), x.cuda(), x.cuda(), None, None, slots, cache)
    keys, values = spl.cache_read(cache, slots)
    q = torch.randn(1, Hk, D, generator=g).bfloat16()
    table = torch.tensor([[pages - 1]]).int().cuda()
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    data[pages - 1, :, :] = 0
    spl.qk_norm_rope_append(x[:1].cuda(), x[:1].cuda(), x[:1].cuda(), None, None,
                            torch.tensor([(pages - 1) * page]).int().cuda(), cache)
    out = spl.attention_fp4(q.cuda(), cache, table, one, torch.tensor([0, 1]).int().cuda(), max_new=1)
    torch.cuda.synchronize()
    _same(keys, ref.stored(x))
    _same(values, ref.stored(x))
    _same(out, ref.stored(x[:1]))                                # one token: its value
