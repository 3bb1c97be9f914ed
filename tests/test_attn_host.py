"""The attention half of a layer on the host (no GPU): the references' own pins, the entry points' refusals, the page
layout's coverage, size functions."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import _attn_ref as ref
import paper_2405_03594_amd as spl

INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def L():
    import os

    from paper_2405_03594_amd import build

    if not os.path.exists(spl.LIB_PATH):
        build.build()
    return spl.lib()


# ---------------------------------------------------------------------------------------------- the references


def test_stored_values_are_the_nearest_of_the_format():
    # a group whose largest is 6 has scale 1: the format's values read back as themselves, halfway ones go to even codes
    x = torch.zeros(1, 32, dtype=torch.float16)
    x[0, :8] = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6.0])
    x[0, 8:15] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x[0, 15:22] = -x[0, 8:15]
    y = ref.stored(x)[0]
    assert torch.equal(y[:8], x[0, :8].double())
    assert y[8:15].tolist() == [0, 1, 1, 2, 2, 4, 4]
    assert (-y[15:22]).tolist() == [0, 1, 1, 2, 2, 4, 4]


def test_stored_scale_is_the_least_that_holds_seven():
    for top, want in ((7.0, 6.0), (7.01, 8.0), (3.5, 3.0), (3.52, 4.0), (13.9, 12.0), (14.1, 16.0)):
        x = torch.zeros(32, dtype=torch.float16)
        x[5] = top
        assert ref.stored(x)[5] == want, top


def test_stored_error_on_gaussians():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(2000, 32, generator=g).half()
    err = (ref.stored(x) - x.double()).square().mean().sqrt().item()
    assert 0.108 < err < 0.116                       # 0.112 of the standard deviation


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("with_weight", [False, True])
def test_gradient_formula_against_differences(interleaved, with_weight):
    g = torch.Generator().manual_seed(4)
    T, H, D, rot = 3, 2, 24, 16
    x = torch.randn(T, H, D, generator=g, dtype=torch.float64)
    w = 1 + 0.3 * torch.randn(D, generator=g, dtype=torch.float64) if with_weight else None
    a = torch.rand(T, rot // 2, generator=g, dtype=torch.float64) * 6
    cs = torch.stack((a.cos(), a.sin()), -1)
    dy = torch.randn(T, H, D, generator=g, dtype=torch.float64)
    dx, dw = ref.norm_rope_grad(dy, x, w, 1e-5, cs, interleaved)
    f = lambda x, w: float((ref.norm_rope(x, w, 1e-5, cs, interleaved) * dy).sum())  # noqa: E731
    h = 1e-6
    for i in itertools.product((0, T - 1), (0, H - 1), range(D)):
        d = torch.zeros_like(x)
        d[i] = h
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * h) - dx[i]) < 1e-7
    if with_weight:
        for c in range(D):
            d = torch.zeros_like(w)
            d[c] = h
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * h) - dw[c]) < 1e-7


# ---------------------------------------------------------------------------------------------- the page layout


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_page_layout_covers_the_region_once(L, dim, page):
    """Every nibble of the code areas and every scale byte belongs to one entry of the format."""
    G = dim // 32
    S = max(2, 1 << (G - 1).bit_length())
    U = {64: 4, 96: 8, 128: 8, 256: 16}[dim]
    size = L.spl_kv_page_bytes(dim, page)
    assert size == page * (dim + 2 * S)
    nibbles = np.zeros(2 * page * dim, dtype=np.int32)
    scales = np.zeros(size, dtype=np.int32)
    for b in range(page):
        for c in range(dim):
            g, j, e = c // 32, c % 32 // 8, c % 8
            nibbles[2 * (b * dim // 2 + 4 * (j * G + g)) + e] += 1
            u, e = c // U, c % U
            nibbles[2 * (page * dim // 2 + U // 2 * (8 * (b // 8 * (dim // U) + u) + b % 8)) + e] += 1
        for g in range(G):
            scales[page * dim + b * S + g] += 1
            scales[page * (dim + S) + 8 * (b // 8 * S + g) + b % 8] += 1
    assert (nibbles == 1).all()
    assert scales.max() == 1 and scales.sum() == 2 * page * G and (scales[: page * dim] == 0).all()


def test_page_sizes_without_a_cache(L):
    for dim, page in ((32, 16), (80, 16), (512, 16), (128, 8), (128, 24), (128, 512), (0, 0), (-128, 16), (128, -16)):
        assert L.spl_kv_page_bytes(dim, page) == 0
    with pytest.raises(ValueError):
        spl.kv_page_bytes(80, 16)


# ---------------------------------------------------------------------------------------------- refusals (C)


def _h(heads=4, data=0x10000, ts=512, hs=128):
    return spl._Heads(data, ts, hs, heads)


def _c(**kw):
    d = dict(data=0x100000, pages=8, data_bytes=1 << 30, page=16, heads=4, head_dim=128, dtype=2)
    d.update(kw)
    return spl._KVCache(*[d[n] for n, _ in spl._KVCache._fields_])


def test_block_tables_checks(L):
    ok = dict(cached=0x1000, fresh=0x2000, requests=2, tokens=2, page=16, table=0x3000, width=4, free=0x4000, count=9,
              head=0x5000, row=0x6000, lens=0x7000, pos=0x8000, slots=0x9000, state=0xA000)

    def call(**kw):
        d = dict(ok, **kw)
        return L.spl_block_tables(*d.values(), None)

    for kw in (dict(cached=0), dict(fresh=0), dict(table=0), dict(free=0), dict(head=0), dict(row=0), dict(lens=0),
               dict(pos=0), dict(slots=0), dict(state=0), dict(requests=0), dict(requests=-1), dict(tokens=-1),
               dict(tokens=1 << 31), dict(width=0), dict(width=1 << 40), dict(count=-1), dict(table=0x3002),
               dict(head=0xA000)):
        assert call(**kw) == INVALID, kw
    for page in (0, 8, 24, 512, -16):
        assert call(page=page) == UNSUPPORTED


def test_norm_rope_checks(L):
    def call(q=_h(), k=_h(), tokens=2, dim=128, dtype=2, wq=0x1000, wk=0x1000, eps=1e-5, pos=0x2000, rope=0x3000, rows=9,
             rot=128, qo=0x20000, ko=0x30000):
        return L.spl_qk_norm_rope(q, k, tokens, dim, dtype, wq, wk, eps, pos, rope, rows, rot, 0, qo, ko, None)

    for kw in (dict(q=None), dict(k=None), dict(q=_h(0)), dict(q=_h(-1)), dict(q=_h(data=0)), dict(q=_h(data=0x10008)),
               dict(q=_h(ts=4)), dict(k=_h(hs=3)), dict(q=_h(ts=-8)), dict(tokens=-1), dict(tokens=1 << 31),
               dict(wq=0x1008), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(pos=0),
               dict(rope=0), dict(rows=0), dict(qo=0), dict(ko=0x30008)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(dim=0), dict(dim=12), dict(dim=264), dict(dtype=3), dict(dtype=0), dict(rot=8), dict(rot=24),
               dict(rot=144), dict(rot=-16)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(tokens=0, qo=0, ko=0) == 0


def test_norm_rope_grad_checks(L):
    def call(dq=_h(), dk=_h(), q=_h(), k=_h(), tokens=2, wq=0x1000, wk=0x1000, do=0x20000, dko=0x30000, dwq=0x4000,
             dwk=0x5000, ws=0x60000, dim=128, rot=128):
        return L.spl_qk_norm_rope_grad(dq, dk, q, k, tokens, dim, 2, wq, wk, 1e-5, 0x2000, 0x3000, 9, rot, 0, do, dko,
                                       dwq, dwk, ws, None)

    for kw in (dict(dq=None), dict(q=None), dict(dq=_h(3)), dict(dk=_h(5)), dict(wq=0), dict(wk=0), dict(do=0),
               dict(dko=0), dict(ws=0), dict(ws=0x60008), dict(dwq=0x4002), dict(q=_h(data=0))):
        assert call(**kw) == INVALID, kw
    assert call(rot=8) == UNSUPPORTED
    size = L.spl_qk_norm_rope_grad_workspace_bytes
    assert size(0, 4, 4, 128) == 0
    assert size(5, 4, 4, 128) > 0
    for a in ((-1, 4, 4, 128), (5, 0, 4, 128), (5, 4, -4, 128), (5, 4, 4, 12), (1 << 31, 4, 4, 128),
              (1 << 30, 4096, 4096, 256)):
        assert size(*a) == -1, a


def test_append_and_read_checks(L):
    def call(q=_h(), k=_h(), v=_h(), tokens=2, slots=0x7000, cache=_c(), qo=0x20000, ko=0):
        return L.spl_qk_norm_rope_append(q, k, v, tokens, 0x1000, 0x1000, 1e-5, 0x2000, 0x3000, 9, 128, 0, slots, cache,
                                         qo, ko, None)

    bytes_ = 8 * 4 * L.spl_kv_page_bytes(128, 16)
    for kw in (dict(k=_h(5)), dict(v=_h(3)), dict(v=None), dict(v=_h(data=0)), dict(slots=0), dict(qo=0), dict(ko=8),
               dict(cache=None), dict(cache=_c(data=0)), dict(cache=_c(data=0x100008)), dict(cache=_c(pages=0)),
               dict(cache=_c(heads=0)), dict(cache=_c(data_bytes=bytes_ - 1)), dict(cache=_c(pages=1 << 27)),
               dict(cache=_c(pages=1 << 62))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(page=8), dict(page=48), dict(head_dim=80), dict(dtype=3)):
        assert call(cache=_c(**kw)) == UNSUPPORTED, kw
    read = L.spl_cache_read
    assert read(_c(), 0, 2, 0x1000, 0x2000, None) == INVALID
    assert read(_c(), 0x100, -1, 0x1000, 0x2000, None) == INVALID
    assert read(_c(), 0x100, 2, 0x1008, 0x2000, None) == INVALID
    assert read(_c(page=8), 0x100, 2, 0x1000, 0x2000, None) == UNSUPPORTED
    assert read(_c(), 0, 0, 0, 0, None) == 0


def test_attention_checks(L):
    def call(q=_h(8), tokens=2, cache=_c(), table=0x1000, requests=2, width=4, lens=0x2000, row=0x3000, max_new=1,
             max_len=64, scale=0.1, window=0, out=0x4000, lse=0, ws=0x10000):
        return L.spl_attention_fp4(q, tokens, cache, table, requests, width, lens, row, max_new, max_len, scale, window,
                                   out, lse, ws, None)

    for kw in (dict(q=None), dict(q=_h(6)), dict(q=_h(8, data=0)), dict(q=_h(8, ts=12)), dict(cache=None), dict(table=0),
               dict(lens=0), dict(row=0), dict(out=0), dict(out=0x4008), dict(lse=2), dict(requests=0), dict(width=0),
               dict(width=1 << 40), dict(max_new=-1), dict(max_len=-1), dict(window=-1), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(tokens=-1), dict(tokens=1 << 31), dict(lens=0x2001),
               dict(max_len=65536, width=5000, ws=0), dict(max_len=65536, width=5000, ws=0x10080)):
        assert call(**kw) == INVALID, kw
    assert call(cache=_c(head_dim=80)) == UNSUPPORTED
    assert call(tokens=0, out=0) == 0
    size = L.spl_attention_fp4_workspace_bytes
    assert size(_c(), 2, 8, 2, 4, 1, 64) == 0                    # one chunk: no workspace
    assert size(_c(), 1, 8, 1, 5000, 1, 65536) > 0
    for a in ((_c(), -1, 8, 2, 4, 1, 64), (_c(), 2, 6, 2, 4, 1, 64), (_c(), 2, 8, 0, 4, 1, 64), (None, 2, 8, 2, 4, 1, 64),
              (_c(page=8), 2, 8, 2, 4, 1, 64), (_c(), 1 << 30, 4096, 2, 4, 1, 64)):
        assert size(*a) == -1


def test_the_workspace_holds_any_window(L):
    """The size is asked without the window, which only takes tokens away: fewer tokens never need more."""
    size = L.spl_attention_fp4_workspace_bytes
    for requests, heads in ((1, 1), (3, 2), (26, 2), (7, 5), (40, 8), (1, 8)):
        for dim in (64, 256):
            last = 0
            for steps in range(1, 420):
                now = size(_c(heads=heads, head_dim=dim), requests, 4 * heads, requests, 5000, 1, 32 * steps)
                assert now >= last, (requests, heads, dim, steps)
                last = now


# ---------------------------------------------------------------------------------------------- refusals (Python)


def _qkv(T=2, H=4, Hk=2, D=128, dt=torch.bfloat16):
    return [torch.zeros(T, h, D, dtype=dt) for h in (H, Hk, Hk)]


def test_wrappers_refuse_mismatched_tensors_before_any_launch():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = spl.KVCache(torch.zeros(3, 2, spl.kv_page_bytes(128, 16), dtype=torch.uint8), 16, 128, torch.bfloat16)
    q, k, v = _qkv()
    rope = torch.zeros(9, 64, 2)
    bad = [
        lambda: spl.KVCache(torch.zeros(3, 2, 100, dtype=torch.uint8), 16, 128, torch.bfloat16),
        lambda: spl.KVCache(torch.zeros(3, 2, spl.kv_page_bytes(128, 16)), 16, 128, torch.bfloat16),
        lambda: spl.KVCache(cache.data, 16, 128, torch.float32),
        lambda: spl.KVCache(cache.data[:, ::2], 16, 128, torch.bfloat16),
        lambda: spl.block_tables(i32(2), i32(3), i32(2, 4), i32(9), i32(1), 16, 2),
        lambda: spl.block_tables(i32(2).long(), i32(2), i32(2, 4), i32(9), i32(1), 16, 2),
        lambda: spl.block_tables(i32(2), i32(2), i32(4, 2).T, i32(9), i32(1), 16, 2),
        lambda: spl.block_tables(i32(2), i32(2), i32(2, 4), i32(9, 1), i32(1), 16, 2),
        lambda: spl.block_tables(i32(2), i32(2), i32(2, 4), i32(9), i32(2), 16, 2),
        lambda: spl.block_tables(i32(2), i32(2), i32(2, 4), i32(9), i32(1), 16, -1),
        lambda: spl.qk_norm_rope(q[0], k, i32(2), rope),
        lambda: spl.qk_norm_rope(q.float(), k.float(), i32(2), rope),
        lambda: spl.qk_norm_rope(q, k.half(), i32(2), rope),
        lambda: spl.qk_norm_rope(q, k[:1], i32(2), rope),
        lambda: spl.qk_norm_rope(q, k[..., :64], i32(2), rope),
        lambda: spl.qk_norm_rope(q, k, i32(3), rope),
        lambda: spl.qk_norm_rope(q, k, i32(2).long(), rope),
        lambda: spl.qk_norm_rope(q, k, i32(2), rope.half()),
        lambda: spl.qk_norm_rope(q, k, i32(2), rope[..., 0]),
        lambda: spl.qk_norm_rope(q, k, i32(2), rope, q_weight=torch.ones(64, dtype=q.dtype)),
        lambda: spl.qk_norm_rope(q, k, i32(2), rope, k_weight=torch.ones(128)),
        lambda: spl.qk_norm_rope(torch.zeros(2, 4, 132, dtype=q.dtype)[..., 4:], k, i32(2), rope),
        lambda: spl.qk_norm_rope(torch.zeros(2, 128, 4, dtype=q.dtype).transpose(1, 2), k, i32(2), rope),
        lambda: spl.qk_norm_rope_grad(q[:, :3], k, q, k, i32(2), rope),
        lambda: spl.qk_norm_rope_grad(q, k.half(), q, k, i32(2), rope),
        lambda: spl.qk_norm_rope_append(q, k, v, i32(2), rope, i32(3), cache),
        lambda: spl.qk_norm_rope_append(q, k, q, i32(2), rope, i32(2), cache),
        lambda: spl.qk_norm_rope_append(*_qkv(D=64), i32(2), rope, i32(2), cache),
        lambda: spl.qk_norm_rope_append(*_qkv(dt=torch.float16), i32(2), rope, i32(2), cache),
        lambda: spl.cache_read(cache, i32(2, 1)),
        lambda: spl.cache_read(cache, i32(2).long()),
        lambda: spl.attention_fp4(q[:, :3], cache, i32(2, 4), i32(2), i32(3)),
        lambda: spl.attention_fp4(q, cache, i32(2), i32(2), i32(3)),
        lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(3), i32(3)),
        lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(2)),
        lambda: spl.attention_fp4(q, cache, i32(2, 4).long(), i32(2), i32(3)),
        lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(3), lse=torch.zeros(2, 2)),
        # everything right but the device
        lambda: spl.block_tables(i32(2), i32(2), i32(2, 4), i32(9), i32(1), 16, 2),
        lambda: spl.qk_norm_rope(q, k, i32(2), rope),
        lambda: spl.qk_norm_rope_append(q, k, v, i32(2), rope, i32(2), cache),
        lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(3)),
        lambda: spl.cache_read(cache, i32(2)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")


class _Recorder:
    """Stands for the library: keeps the arguments of each call, accepts them all.  Sizes are the library's."""

    def __init__(self):
        self.calls, self.spl_kv_page_bytes = [], spl.lib().spl_kv_page_bytes

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


def _calls(monkeypatch):
    """The wrappers on CPU tensors, their calls recorded instead of made."""
    rec = _Recorder()
    monkeypatch.setattr(spl, "lib", lambda: rec)
    monkeypatch.setattr(spl, "_on_device", lambda *a: None)
    monkeypatch.setattr(spl, "_on", lambda stream: 0)
    monkeypatch.setattr(spl, "_attention_workspace", lambda *a: 0)
    return rec.calls


def test_a_cache_whose_data_are_replaced_is_called_with_the_new_ones(monkeypatch):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    data = lambda pages, dim: torch.zeros(pages, 2, spl.kv_page_bytes(dim, 16), dtype=torch.uint8)  # noqa: E731
    cache = spl.KVCache(data(3, 128), 16, 128, torch.bfloat16)
    calls = _calls(monkeypatch)

    def step(D):
        q, k, v = _qkv(D=D)
        spl.qk_norm_rope_append(q, k, v, None, None, i32(2), cache)
        spl.cache_read(cache, i32(2))
        spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(3))
        views = [next(a for a in args if isinstance(a, spl._KVCache)) for _, args in calls]
        calls.clear()
        assert len(views) == 3
        for v in views:
            assert (v.data, v.pages, v.data_bytes) == (cache.data.data_ptr(), len(cache.data), cache.data.numel())
            assert (v.page, v.heads, v.head_dim) == (16, 2, D) and (cache.pages, cache.heads) == (len(cache.data), 2)

    step(128)
    cache.data = data(7, 128)                                    # grown
    step(128)
    cache.data, cache.head_dim = data(5, 64), 64
    step(64)
    for name, value in (("data", data(5, 128)), ("data", data(5, 64)[:, ::2]), ("data", data(5, 64).float()),
                        ("data", None), ("page", 32), ("head_dim", 128), ("dtype", torch.float32)):
        q, k, v = _qkv(D=64)
        was = getattr(cache, name)
        setattr(cache, name, value)
        for call in (lambda: spl.qk_norm_rope_append(q, k, v, None, None, i32(2), cache),
                     lambda: spl.cache_read(cache, i32(2)),
                     lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(3))):
            with pytest.raises(ValueError):
                call()
        assert not calls
        setattr(cache, name, was)
    step(64)


def test_block_tables_refuses_results_that_share_memory_with_another_array(L):
    """Workgroups read the lengths and the free list while others write the results."""
    size = dict(cached=8, fresh=8, table=32, free=36, head=4, row=12, lens=8, pos=16, slots=16, state=8)
    at = {n: 0x1000 * (i + 1) for i, n in enumerate(size)}

    def call(at):
        return L.spl_block_tables(at["cached"], at["fresh"], 2, 4, 16, at["table"], 4, at["free"], 9, at["head"],
                                  at["row"], at["lens"], at["pos"], at["slots"], at["state"], None)

    for a in ("table", "row", "lens", "pos", "slots", "state"):
        for b in size:
            if a == b:
                continue
            for offset in (0, size[b] - 4, 4 - size[a]):         # the same start, one entry in common at either end
                assert call(dict(at, **{a: at[b] + offset})) == INVALID, (a, b, offset)


def test_sizes_past_one_launch_are_refused(L):
    """A launch has fewer than 2^32 threads in x: past them a refusal before any launch, and no workspace."""
    read = lambda heads, dim, tokens: L.spl_cache_read(_c(heads=heads, head_dim=dim, page=256), 0x7000, tokens, 0x10000,  # noqa: E731
                                                       0, None)
    assert read(8, 128, 1 << 25) == read(1, 64, 1 << 29) == read(4, 256, (1 << 25) - 1) == UNSUPPORTED
    assert read(64, 128, 1 << 30) == INVALID         # past what the call takes at all

    def call(cache, tokens, heads, requests, max_new):
        sizes = (requests, 1, max_new, 16)
        size = L.spl_attention_fp4_workspace_bytes(cache, tokens, heads, *sizes)
        if size >= 0:
            return size
        assert size == -1
        for window in (0, 5):
            assert L.spl_attention_fp4(_h(heads), tokens, cache, 0x1000, requests, 1, 0x2000, 0x3000, max_new, 16, 0.1,
                                       window, 0x4000, 0, 0x10000, None) == UNSUPPORTED
        return -1

    # single rows: requests * key heads workgroups of 256 threads
    assert call(_c(), 1 << 22, 4, (1 << 22) - 1, 1) == 0 and call(_c(), 1 << 22, 4, 1 << 22, 1) == -1
    assert call(_c(), 5, 4, (1 << 22) - 1, 1) == 0 and call(_c(), 5, 4, 1 << 22, 1) == -1
    # many rows: workgroups of 512 threads for 128 rows and for each request
    assert call(_c(), 1 << 21, 4, (1 << 21) - (1 << 14) - 1, 0) == 0
    assert call(_c(), 1 << 21, 4, (1 << 21) - (1 << 14), 0) == -1
    # 256 channels: workgroups of 256 threads for 16 rows and for each request
    assert call(_c(head_dim=256), 1 << 22, 4, (1 << 22) - (1 << 18) - 1, 0) == 0
    assert call(_c(head_dim=256), 1 << 22, 4, (1 << 22) - (1 << 18), 0) == -1


def test_numbers_past_32_bits_are_refused_and_not_cut(monkeypatch):
    """A window of 2^32 is not no window, and 2^32 + 64 is not a page of 64 tokens."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = spl.KVCache(torch.zeros(3, 2, spl.kv_page_bytes(128, 16), dtype=torch.uint8), 16, 128, torch.bfloat16)
    q, k, v = _qkv()
    for n in (1 << 32, (1 << 32) + 64, (1 << 31), -(1 << 32) + 16, 1 << 64):
        for call in (lambda: spl.kv_page_bytes(128, n + 16), lambda: spl.kv_page_bytes(n + 128, 16),
                     lambda: spl._attention_workspace(16, 2, 128, 2, 4, 2, 4, n, 0),
                     lambda: spl._attention_workspace(16, 2, 128, 2, 4, 2, 4, 0, n)):
            with pytest.raises(ValueError):
                call()
    calls = _calls(monkeypatch)
    for n in (1 << 32, (1 << 32) + 64, (1 << 31), -(1 << 32) + 16):
        for call in (lambda: spl.block_tables(i32(2), i32(2), i32(2, 4), i32(9), i32(1), n + 64, 2),
                     lambda: spl.attention_fp4(q, cache, i32(2, 4), i32(2), i32(3), window=n)):
            with pytest.raises(ValueError):
                call()
    assert not calls
