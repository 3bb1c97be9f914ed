"""attention_fp4 on the GPU against the definition in 64 bits, over what the cache holds.

Tolerance, element by element: a softmax weight is rounded once to the 16-bit type (u of it), and so is the result (u,
or half the type's smallest step); where the sum of weights is taken before their rounding the same u enters once more: 3 u of sum p |v|.  A score is a sum
of D fp32 products, off by at most 2^-20 of the sum of their sizes (its partial sums' roundings) for D <= 256, and an
exponent's error is the weight's relative error, twice with the normalisation: 2^-18 (1 + that sum) more."""
import pytest
import torch

import _attn_ref as ref

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _spl():
    import paper_2405_03594_amd as spl

    return spl


class Batch:
    """A filled cache and a batch over it; keys and values as the cache reads them back."""

    def __init__(self, new, lens, H, Hk, D, page, dt, seed=0, fill=0xFF, scale_keys=1.0, extra=0):
        spl = _spl()
        g = torch.Generator().manual_seed(seed)
        self.new, self.lens, self.dt = new, lens, dt
        held = [-(-n // page) for n in lens]
        pages = sum(held) + 2
        self.cache = spl.KVCache.empty(pages, Hk, D, page, dt)
        self.cache.data.fill_(fill)                              # what no token was stored in
        ids = torch.randperm(pages, generator=g)
        width = max(held + [1]) + extra
        self.table = torch.full((len(lens), width), -1)
        self.keys, self.values = [], []
        n = 0
        for r, m in enumerate(held):
            self.table[r, :m] = ids[n:n + m]
            n += m
            L = lens[r]
            k = (torch.randn(L, Hk, D, generator=g) * torch.exp(0.5 * torch.randn(1, Hk, D, generator=g)) * scale_keys)
            v = torch.randn(L, Hk, D, generator=g) * torch.exp(torch.randn(L, Hk, 1, generator=g))
            k, v = k.to(dt), v.to(dt)
            if L:
                at = torch.arange(L)
                slots = (self.table[r, at // page] * page + at % page).int().cuda()
                k, v = k.cuda(), v.cuda()
                spl.qk_norm_rope_append(k, k, v, None, None, slots, self.cache)
                k, v = (x.cpu().double() for x in spl.cache_read(self.cache, slots))
            self.keys.append(k.double())
            self.values.append(v.double())
        self.table = self.table.int().cuda()
        self.row_start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)])
        self.q = torch.randn(sum(new), H, D, generator=g).to(dt)
        self.D = D

    def run(self, **kw):
        args = dict(max_new=max(self.new), max_len=max(self.lens))
        args.update(kw)
        q = args.pop("q", None)
        q = self.q.cuda() if q is None else q
        lse = torch.full(q.shape[:2], 7.0, device="cuda")
        out = torch.full(q.shape, 9.0, dtype=self.dt, device="cuda")
        _spl().attention_fp4(q, self.cache, self.table, torch.tensor(self.lens).int().cuda(),
                             self.row_start.int().cuda(), lse=lse, out=out, **args)
        torch.cuda.synchronize()
        return out.cpu().double(), lse.cpu().double()

    def check(self, scale=None, window=0, **kw):
        got, lse = self.run(scale=scale, window=window, **kw)
        s = self.D ** -0.5 if scale is None else scale
        want, want_lse, mag, top = ref.attention(self.q.double(), self.keys, self.values, self.row_start, self.lens, s,
                                                 window)
        loose = 2.0 ** -18 * (1 + top)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        bad = (got - want).abs().nan_to_num() > ((3 * ref.UNIT[self.dt] + loose) * mag).nan_to_num() + ref.STEP[self.dt]
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float((got - want).abs().nan_to_num().max())}"
        seen = torch.isfinite(want_lse)
        assert torch.equal(torch.isneginf(lse), torch.isneginf(want_lse))
        assert ((lse - want_lse)[seen].abs() <= 3 * ref.UNIT[self.dt] + loose).all()
        return got


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_decode(D, page, dt):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300]
    Batch([1] * len(lens), lens, 6, 2, D, page, dt).check()


@pytest.mark.parametrize("H,Hk", [(1, 1), (8, 8), (8, 1), (16, 1), (15, 3), (32, 2), (17, 1), (40, 1), (64, 2)])
def test_head_layouts(H, Hk):
    Batch([1, 1, 1], [40, 7, 129], H, Hk, 64, 16, BF, seed=1).check()


@pytest.mark.parametrize("dt", [BF, HF])
def test_requests_that_see_nothing(dt):
    """No tokens yet, no rows, fewer tokens than rows (the first rows stand before the request): zeros and -inf."""
    b = Batch([1, 0, 3, 1, 5, 2], [0, 40, 3, 1, 2, 50], 4, 2, 64, 16, dt, seed=2)
    got = b.check()
    assert (got[0] == 0).all() and (got[5:8] == 0).all()          # 5 rows of a request of 2 tokens: the first 3
    Batch([1], [0], 4, 2, 128, 16, dt).check()


@pytest.mark.parametrize("window", [1, 5, 16, 33, 64, 100, 1000])
@pytest.mark.parametrize("new", [[1, 1, 1], [9, 1, 40]])
def test_windows(new, window):
    Batch(new, [200, 70, 90], 4, 2, 64, 16, BF, seed=3).check(window=window)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("dt", [BF, HF])
def test_chunks_of_prompts(D, dt):
    Batch([5, 1, 17, 33, 1, 2], [5, 40, 100, 33, 1, 260], 6, 2, D, 32, dt, seed=4).check()


@pytest.mark.parametrize("D,dt,H,Hk", [(64, HF, 8, 8), (96, BF, 24, 8), (128, BF, 16, 16), (128, HF, 12, 3)])
@pytest.mark.parametrize("window", [0, 150])
def test_the_kernel_for_many_rows(D, dt, H, Hk, window):
    """Enough rows for a workgroup on every CU; prompts of odd lengths, one after other tokens, beside single rows."""
    rows = 128 * torch.cuda.get_device_properties(0).multi_processor_count // H + 40
    b = Batch([rows - 70, 1, 67, 1, 0, 2], [rows + 61, 300, 67, 1, 5, 2], H, Hk, D, 64, dt, seed=5)
    big = b.run(window=window)
    few = [r for r in range(6) if r != 0]
    # the long prompt's rows are checked at places, the others all
    pick = sorted({0, 1, 31, 32, 127, 128, rows - 72, rows - 71, *range(0, rows - 70, 97)})
    at = torch.tensor(pick)
    first = b.row_start[1]
    want, want_lse, mag, top = ref.attention(b.q.double()[first:], [b.keys[r] for r in few], [b.values[r] for r in few],
                                             b.row_start[1:] - first, [b.lens[r] for r in few], D ** -0.5, window)
    loose = 2.0 ** -18 * (1 + top)
    assert ((big[0][first:] - want).abs() <= (3 * ref.UNIT[dt] + loose) * mag + ref.STEP[dt]).all()
    fin = torch.isfinite(want_lse)
    assert ((big[1][first:] - want_lse)[fin].abs() <= 3 * ref.UNIT[dt] + loose).all()
    for t in pick:
        p = b.lens[0] - b.new[0] + t
        w, l, m, top = ref.attention(b.q.double()[t:t + 1], b.keys[:1], b.values[:1], [0, 1], [p + 1], D ** -0.5, window)
        tol = (3 * ref.UNIT[dt] + 2.0 ** -18 * (1 + top))
        assert ((big[0][t] - w[0]).abs() <= tol * m[0] + ref.STEP[dt]).all(), t
        assert ((big[1][t] - l[0]).abs() <= tol).all(), t


def test_long_requests_are_split_and_joined():
    b = Batch([1, 1, 1], [9000, 1, 700], 4, 2, 128, 128, BF, seed=6)
    b.check()
    b.check(max_len=0)                                           # not known: by the table's width
    b.check(max_len=100)                                         # far too low a hint
    b = Batch([3, 2], [5000, 2500], 8, 2, 64, 64, HF, seed=7, extra=30)
    b.check()
    b.check(max_new=0)                                           # not known: tiles are looked up
    b.check(max_new=0, window=3000)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("window", [0, 37])
def test_tiles_of_twice_the_rows(D, dt, window):
    """Many rows over a wide table: two tiles of 16 rows a workgroup; ends of 1 to 31 rows, some without any key."""
    H = 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    new = [70, 1, 145, 31, 33, 17]                               # 297 rows of each head: tiles for every workgroup
    b = Batch(new, [150, 60, 145, 33, 20, 0], H, H, D, 64, dt, seed=16, extra=40)
    got = b.check(max_len=0, window=window)
    assert (got[70 + 1 + 145 + 31:][:13] == 0).all() and (got[-17:] == 0).all()
    _poison(b, 2, 100, 3, False, True)                           # seen by the last 45 rows of 145
    _poison(b, 3, 32, 5, True, False)                            # by the last of 31
    first = 70 + 1
    got = b.check(max_len=0, window=window)
    assert torch.isfinite(got[first:first + 100]).all() and torch.isnan(got[first + 100, 3, :32]).all()
    assert torch.isnan(got[first + 145 + 30, 5]).all()


@pytest.mark.parametrize("requests", [33, 63, 64, 65])
def test_many_requests_of_different_lengths(requests):
    """Served in the order of their lengths up to 64 of them: each once, equal lengths among them, and none at all."""
    heads = torch.cuda.get_device_properties(0).multi_processor_count // 16
    lens = [(37 * i) % 90 if i % 5 else 40 for i in range(requests)]
    lens[3] = lens[requests - 1] = 0
    lens[7] = 530
    b = Batch([1 + (i % 3 == 0) for i in range(requests)], lens, heads, heads, 64, 64, BF, seed=19)
    b.check()


def test_tiles_are_found_among_many_requests():
    """More than a wave's lanes of requests, of no row to 90, the last ones empty."""
    new = [(7 * i) % 4 for i in range(130)] + [90, 0, 0]
    lens = [n + (13 * i) % 50 for i, n in enumerate(new)]
    b = Batch(new, lens, 4, 2, 64, 16, HF, seed=20)
    b.check()
    b.check(max_new=0)


def test_tiles_of_twice_the_rows_under_a_window():
    H = 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch([290], [2200], H, H, 64, 32, HF, seed=18)
    got, lse = b.run(window=2040)
    for t in (0, 1, 15, 16, 31, 32, 129, 130, 161, 288, 289):    # the window's start passes 0 at row 129
        p = 2200 - 290 + t
        w, l, m, top = ref.attention(b.q.double()[t:t + 1], b.keys, b.values, [0, 1], [p + 1], 64 ** -0.5, 2040)
        tol = 3 * ref.UNIT[HF] + 2.0 ** -18 * (1 + top)
        assert ((got[t] - w[0]).abs() <= tol * m[0] + ref.STEP[HF]).all(), t
        assert ((lse[t] - l[0]).abs() <= tol).all(), t


@pytest.mark.parametrize("new,lens,extra", [([1, 3], [700, 90], 0), ([297], [310], 40), ([1040, 1], [1040, 70], 0)])
def test_pages_past_four_gigabytes(new, lens, extra):
    """The same bits where the pages lie past 4 GiB: single rows, two tiles a workgroup, many rows."""
    H = 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch(new, lens, H, H, 64, 64, BF, seed=21, extra=extra)
    hint = 0 if extra else max(lens)
    want = b.run(max_len=hint)
    small = b.cache
    more = (9 << 29) // (small.data.numel() // small.pages)      # 4.5 GiB before them
    data = torch.zeros(more + small.pages, *small.data.shape[1:], dtype=torch.uint8, device="cuda")
    data[more:] = small.data
    b.cache = _spl().KVCache(data, 64, 64, BF)
    b.table = torch.where(b.table >= 0, b.table + more, b.table).int()
    got = b.run(max_len=hint)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_split_requests_beside_prompts():
    """Single rows over many tokens are split and joined in a call whose prompts are not."""
    H = 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch([1, 520, 3, 1, 16, 0], [1500, 520, 2100, 40, 1900, 700], H, H, 64, 64, BF, seed=17)
    got, lse = b.run()
    for r in (0, 2, 3, 4):
        s, e = int(b.row_start[r]), int(b.row_start[r + 1])
        w, l, m, top = ref.attention(b.q.double()[s:e], b.keys[r:r + 1], b.values[r:r + 1], [0, e - s], [b.lens[r]],
                                     64 ** -0.5, 0)
        tol = 3 * ref.UNIT[BF] + 2.0 ** -18 * (1 + top)
        assert ((got[s:e] - w).abs() <= tol * m + ref.STEP[BF]).all(), r
        assert ((lse[s:e] - l).abs() <= tol).all(), r


def test_a_window_that_is_split_further_than_its_requests():
    """5440 tokens are split into 9, a window of 5100 of them into 10: the workspace has room."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    R = 26 * cus // 256
    lens = [5440] + [50] * (R - 2) + [5300]
    b = Batch([1] * R, lens, 2, 2, 64, 64, BF, seed=22)
    got, lse = b.run(window=5100)
    for r in (0, 1, R - 1):
        w, l, m, top = ref.attention(b.q.double()[r:r + 1], b.keys[r:r + 1], b.values[r:r + 1], [0, 1], [lens[r]],
                                     64 ** -0.5, 5100)
        tol = 3 * ref.UNIT[BF] + 2.0 ** -18 * (1 + top)
        assert ((got[r] - w[0]).abs() <= tol * m[0] + ref.STEP[BF]).all(), r
        assert ((lse[r] - l[0]).abs() <= tol).all(), r


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 3e-3])
def test_scales(scale):
    Batch([1, 20], [70, 45], 4, 4, 64, 16, BF, seed=8).check(scale=scale)


def test_peaked_scores():
    """Scores of some hundred: weights of 0 and 1, the reference moving at every step."""
    Batch([1, 12], [400, 300], 4, 2, 128, 16, BF, seed=9, scale_keys=25.0).check()
    Batch([1, 12], [400, 300], 4, 2, 128, 16, HF, seed=10, scale_keys=25.0).check()


def _poison(b, r, t, head, keys, values):
    """Stores NaN keys and/or infinite values for one token and head of request r (first 32 channels only)."""
    spl = _spl()
    page = b.cache.page
    slot = (b.table[r, t // page].cpu() * page + t % page).int().view(1).cuda()
    k, v = b.keys[r][t:t + 1].to(b.dt), b.values[r][t:t + 1].to(b.dt)
    if keys:
        k[0, head, 3] = float("nan")
        b.keys[r][t, head, :32] = float("nan")
    if values:
        v[0, head, 5] = float("inf")
        b.values[r][t, head, :32] = float("nan")
    spl.qk_norm_rope_append(k.cuda(), k.cuda(), v.cuda(), None, None, slot, b.cache)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("keys,values", [(True, False), (False, True), (True, True)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(D, keys, values):
    b = Batch([1, 1, 8], [50, 60, 70], 4, 2, D, 16, BF, seed=11)
    _poison(b, 1, 13, 1, keys, values)                           # seen by the one row, by the second pair of heads
    _poison(b, 2, 66, 0, keys, values)                           # seen by the last 4 of 8 rows, by the first pair
    got = b.check()
    assert torch.isfinite(got[0]).all() and torch.isnan(got[1, 2:]).any() and torch.isfinite(got[1, :2]).all()
    assert torch.isfinite(got[2:6]).all() and torch.isnan(got[6:, :2]).any() and torch.isfinite(got[6:, 2:]).all()
    b.check(window=4)                                            # outside the window of the first


@pytest.mark.parametrize("keys,values", [(True, False), (False, True)])
def test_values_that_are_not_finite_among_many_rows(keys, values):
    H, D = 16, 128
    rows = 128 * torch.cuda.get_device_properties(0).multi_processor_count // H + 5
    b = Batch([rows], [rows], H, H, D, 64, HF, seed=12)
    clean = b.run()[0]
    bad = rows - 150
    _poison(b, 0, bad, 3, keys, values)
    got = b.run()[0]
    assert torch.equal(got[:bad], clean[:bad])                   # earlier rows and other heads do not change by a bit
    others = [h for h in range(H) if h != 3]
    assert torch.equal(got[:, others], clean[:, others])
    part = got[bad:, 3]
    assert torch.isnan(part[:, :32]).all()
    assert torch.isnan(part[:, 32:]).all() if keys else torch.equal(part[:, 32:], clean[bad:, 3, 32:])


@pytest.mark.parametrize("fill", [0x00, 0x7F, 0x8E, 0xFD, 0xFE])
@pytest.mark.parametrize("dt", [BF, HF])
def test_what_no_token_was_stored_in_does_not_matter(dt, fill):
    Batch([1, 1, 9], [33, 17, 45], 4, 2, 128, 32, dt, seed=13, fill=fill).check()


def test_pages_that_are_not_there_hold_no_keys():
    b = Batch([1, 6, 1], [70, 90, 64], 4, 2, 64, 16, BF, seed=14)
    b.table[0, 1], b.table[1, 2], b.table[1, 5], b.table[2, :] = -1, 10 ** 6, -5, -1
    for r, gone in ((0, [1]), (1, [2, 5]), (2, [0, 1, 2, 3])):
        for p in gone:
            b.keys[r][16 * p:16 * p + 16] = float("nan")
    got, lse = b.run()
    for r in range(3):
        for t in range(int(b.row_start[r]), int(b.row_start[r + 1])):
            p = b.lens[r] - int(b.row_start[r + 1]) + t
            seen = torch.isfinite(b.keys[r][:p + 1, 0, 0])
            if not seen.any():
                assert (got[t] == 0).all() and torch.isneginf(lse[t]).all()
                continue
            w, l, m, top = ref.attention(b.q.double()[t:t + 1], [b.keys[r][:p + 1][seen]], [b.values[r][:p + 1][seen]],
                                         [0, 1], [int(seen.sum())], 0.125, 0)
            assert ((got[t] - w[0]).abs() <= (3 * ref.UNIT[BF] + 2.0 ** -18 * (1 + top)) * m[0]).all()


def test_strided_queries_and_rows_of_no_request():
    b = Batch([2, 3], [40, 50], 4, 2, 64, 16, BF, seed=15)
    want = b.run()[0]
    wide = torch.zeros(5, 4 + 3, 64 + 8, dtype=BF, device="cuda")
    wide[:, :4, :64] = b.q.cuda()
    assert torch.equal(b.run(q=wide[:, :4, :64])[0], want)
    flip = b.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(b.run(q=flip)[0], want)
    padded = torch.cat((b.q, torch.zeros(9, 4, 64, dtype=BF))).cuda()
    got, lse = b.run(q=padded)
    assert torch.equal(got[:5], want) and (got[5:] == 9).all() and (lse[5:] == 7).all()
    long = Batch([1, 1], [9000, 4], 4, 2, 64, 64, BF, seed=16)    # the same where the tokens are split
    one = long.run()[0]
    got, lse = long.run(q=torch.cat((long.q, torch.zeros(7, 4, 64, dtype=BF))).cuda())
    assert torch.equal(got[:2], one) and (got[2:] == 9).all() and (lse[2:] == 7).all()


def test_no_tokens():
    spl = _spl()
    cache = spl.KVCache.empty(1, 2, 64, 16, BF)
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = spl.attention_fp4(torch.zeros(0, 4, 64, dtype=BF, device="cuda"), cache, z.view(1, 1), z, torch.cat((z, z)))
    assert out.shape == (0, 4, 64)


def test_the_same_call_gives_the_same_bits_on_any_stream():
    b = Batch([1] * 9, [4000, 10, 999, 2500, 1, 64, 3000, 2000, 77], 8, 8, 128, 64, HF, seed=17)
    first = b.run()
    side = torch.cuda.Stream()
    q, lens, rows = b.q.cuda(), torch.tensor(b.lens).int().cuda(), b.row_start.int().cuda()
    torch.cuda.synchronize()
    for stream in (None, side, side):
        out = _spl().attention_fp4(q, b.cache, b.table, lens, rows, max_new=1, max_len=4000, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().double(), first[0])


def test_a_serving_step_in_a_graph():
    """Tables, append and attention of one token step captured once and replayed as the requests grow: every replay
    against the eager calls, with other work between."""
    spl = _spl()
    R, H, Hk, D, page, dt = 5, 8, 2, 128, 16, BF
    g = torch.Generator().manual_seed(18)
    lens0 = [30, 1, 16, 47, 0]
    width, pages = 8, 40
    free = torch.randperm(pages, generator=g).int().cuda()
    a = torch.arange(256, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    rope = torch.stack((a.cos(), a.sin()), -1).float().cuda()
    q = torch.randn(R, H, D, generator=g).to(dt).cuda()
    kv = torch.randn(2, R, Hk, D, generator=g).to(dt).cuda()
    w = torch.ones(D, dtype=dt, device="cuda")

    def fresh():
        cached, head = torch.tensor(lens0).int().cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
        table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
        cache = spl.KVCache.empty(pages, Hk, D, page, dt)
        # the tokens before: zeros in pages of their own
        p = spl.block_tables(torch.zeros_like(cached), cached, table, free, head, page, sum(lens0))
        z = torch.zeros(sum(lens0), Hk, D, dtype=dt, device="cuda")
        spl.qk_norm_rope_append(z, z, z, None, None, p.slots, cache)
        return cached, p.free_head.clone(), table, cache

    def step(cached, head, table, cache, new):
        plan = spl.block_tables(cached, new, table, free, head, page, R)
        qo = spl.qk_norm_rope_append(q, kv[0], kv[1], plan.positions, rope, plan.slots, cache, w, w)
        out = spl.attention_fp4(qo, cache, table, plan.lens, plan.row_start, max_new=1, max_len=width * page)
        cached.copy_(plan.lens)
        head.copy_(plan.free_head)
        return out, plan.missing

    new = torch.ones(R, dtype=torch.int32, device="cuda")
    state = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*fresh(), new)
    torch.cuda.current_stream().wait_stream(side)
    eager = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, missing = step(*state, new)
    for i in range(6):
        q.normal_()
        kv.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want, lost = step(*eager, new)
        torch.cuda.synchronize()
        assert int(missing) == 0 and int(lost) == 0
        assert torch.equal(got, want), i
        assert torch.equal(state[2], eager[2]) and torch.equal(state[3].data, eager[3].data)
    assert eager[0].tolist() == [n + 6 for n in lens0]


# (rows, lengths) of requests and their heads: 18, 6 and 1 splits of the longest
LOW = [([2, 1, 3], [9000, 300, 2000], 4, 4), ([3, 1], [3000, 40], 8, 2), ([40, 2], [9000, 70], 4, 4),
       ([2, 1, 5], [300, 40, 5], 4, 4)]


@pytest.mark.parametrize("max_new", [1, 2])
@pytest.mark.parametrize("new,lens,H,Hk", LOW)
def test_the_first_rows_of_a_request_of_more_than_max_new(new, lens, H, Hk, max_new):
    """Only rows past max_new may be left out, whether the request is split or not."""
    b = Batch(new, lens, H, Hk, 128, 64, BF, seed=23)
    got, lse = b.run(max_new=max_new)
    want, want_lse, mag, top = ref.attention(b.q.double(), b.keys, b.values, b.row_start, lens, 128 ** -0.5, 0)
    first = [int(b.row_start[r]) + t for r in range(len(new)) for t in range(min(new[r], max_new))]
    tol = 3 * ref.UNIT[BF] + 2.0 ** -18 * (1 + top)
    assert ((got[first] - want[first]).abs() <= tol * mag[first] + ref.STEP[BF]).all()
    assert ((lse[first] - want_lse[first]).abs() <= tol).all()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("length", [300, 3000, 9000])
def test_an_infinite_value_of_no_weight_reaches_its_row_however_it_is_split(length, D, dt):
    """Weights below 2^-300 of the row's largest are 0, and 0 times an infinity is NaN: in one split, in 6, in 18."""
    b = Batch([1], [length], 4, 2, D, 64, dt, seed=24)
    spl = _spl()
    k = torch.full((length, 2, D), 4.0, dtype=dt)                # scores of 16 sqrt(D), and their negatives before the middle
    k[:length // 2] = -4.0
    v = b.values[0].to(dt)
    v[10, 1, 5] = float("inf")
    at = torch.arange(length)
    slots = (b.table[0].cpu()[at // 64] * 64 + at % 64).int().cuda()
    spl.qk_norm_rope_append(k.cuda(), k.cuda(), v.cuda(), None, None, slots, b.cache)
    b.q = torch.full((1, 4, D), 4.0, dtype=dt)
    b.keys[0] = k.double()
    b.values[0] = spl.cache_read(b.cache, slots)[1].cpu().double()
    got = b.check()
    assert torch.isnan(got[0, 2:, :32]).all() and torch.isfinite(got[0, :2]).all()
    assert torch.isfinite(got[0, 2:, 32:]).all()


def test_results_belong_to_the_stream_that_writes_them():
    """Not to blocks that the current stream freed and may still use, and kept while the current stream reads them."""
    spl = _spl()
    b = Batch([300, 9], [300, 40], 16, 4, 128, 16, BF, seed=27)
    lens, rows, q = torch.tensor(b.lens).int().cuda(), b.row_start.int().cuda(), b.q.cuda()
    k = torch.randn(309, 4, 128, device="cuda").to(BF)
    w = torch.ones(128, dtype=BF, device="cuda")
    slots = torch.arange(309, device="cuda").int() % (b.cache.pages * 16)
    fresh = spl.KVCache.empty(40, 4, 128, 16, BF)
    table, free = torch.zeros(2, 40, dtype=torch.int32, device="cuda"), torch.arange(60, device="cuda").int()
    head = torch.zeros(1, dtype=torch.int32, device="cuda")
    new = torch.tensor([300, 9], device="cuda").int()
    calls = {
        "block_tables": lambda s: spl.block_tables(new, new, table, free, head, 16, 309, stream=s).row_start,
        "qk_norm_rope": lambda s: spl.qk_norm_rope(q, k, None, None, w, w, stream=s),
        "qk_norm_rope_grad": lambda s: spl.qk_norm_rope_grad(q, k, q, k, None, None, w, w, stream=s),
        "qk_norm_rope_append": lambda s: spl.qk_norm_rope_append(q, k, k, None, None, slots, fresh, stream=s),
        "cache_read": lambda s: spl.cache_read(b.cache, slots, stream=s),
        "attention_fp4": lambda s: spl.attention_fp4(q, b.cache, b.table, lens, rows, stream=s),
    }
    side = torch.cuda.Stream()
    for name, call in calls.items():
        as_list = lambda x: list(x) if isinstance(x, (tuple, list)) else [x]  # noqa: E731
        want = [x.clone() for x in as_list(call(None))]
        for stream in (side, torch.cuda.ExternalStream(side.cuda_stream)):
            torch.cuda.synchronize()
            freed = [torch.empty_like(x) for x in want]          # blocks of these sizes, back in the current stream's pool
            places = {x.untyped_storage().data_ptr() for x in freed}
            del freed
            got = as_list(call(stream))
            torch.cuda.current_stream().wait_stream(side)
            at = [x.untyped_storage().data_ptr() for x in got]
            assert not places & set(at), name
            torch.cuda._sleep(20_000_000)                        # the current stream reads them late
            copies = [x.clone() for x in got]
            del got
            again = as_list(call(stream))
            assert not set(at) & {x.untyped_storage().data_ptr() for x in again}, name
            torch.cuda.synchronize()
            bits = lambda x: x.contiguous().view(torch.uint8)  # noqa: E731  (places without a token read back as NaN)
            for x, y, z in zip(want, copies, again):
                assert torch.equal(bits(x), bits(y)) and torch.equal(bits(x), bits(z)), name


@pytest.mark.parametrize("max_new", [0, 1100])
def test_prompts_among_more_requests_than_a_wave_has_lanes(max_new):
    """The kernel for many rows finds its tiles past the first 64 requests, and none at all in a batch of single rows."""
    H = 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    new, lens = [1] * 150, [(37 * i) % 90 + 1 for i in range(150)]
    new[70], lens[70] = 1100, 1130                               # the prompts in the second and third 64 requests
    new[131], lens[131] = 17, 17
    new[3] = lens[5] = 0
    b = Batch(new, lens, H, H, 64, 64, BF, seed=25)
    got, lse = b.run(max_new=max_new)
    for r in range(150):
        s, e = int(b.row_start[r]), int(b.row_start[r + 1])
        for t in range(s, e) if r != 70 else (s, s + 1, s + 127, s + 128, s + 700, e - 1):
            p = lens[r] - e + t
            if p < 0:
                assert (got[t] == 0).all() and torch.isneginf(lse[t]).all()
                continue
            w, l, m, top = ref.attention(b.q.double()[t:t + 1], b.keys[r:r + 1], b.values[r:r + 1], [0, 1], [p + 1],
                                         64 ** -0.5, 0)
            tol = 3 * ref.UNIT[BF] + 2.0 ** -18 * (1 + top)
            assert ((got[t] - w[0]).abs() <= tol * m[0] + ref.STEP[BF]).all(), (r, t)
            assert ((lse[t] - l[0]).abs() <= tol).all(), (r, t)
    rows = 128 * torch.cuda.get_device_properties(0).multi_processor_count // H
    one = Batch([1] * rows, [1 + i % 3 for i in range(rows)], H, H, 64, 16, BF, seed=26)      # no prompt, and max_new not known
    want, known = one.run(max_new=0), one.run()
    assert torch.equal(want[0], known[0]) and torch.equal(want[1], known[1])


# requests for each of the kernels: single rows, their splits, tiles of 16 rows, of 32, many rows of one request and of two
GIVEN = {"rows": ([1, 1, 4], [30, 70, 90], 4, {}), "splits": ([1, 3], [9000, 8000], 4, {}),
         "tiles": ([1, 20, 9], [30, 70, 60], 4, dict(max_new=0)), "wide": ([290], [2200], 64, dict(max_len=0)),
         "prompt": ([700], [760], 64, {}), "prompts": ([600, 50], [640, 90], 64, {})}


def _check_given(b, rows, tokens, window, **kw):
    """The first `rows` rows, at the positions that lens and row_start give them, over the first `tokens` tokens."""
    got, lse = b.run(q=b.q[:rows].cuda(), window=window, **kw)
    for r in range(len(b.lens)):
        s, e = int(b.row_start[r]), min(int(b.row_start[r + 1]), rows)
        pick = range(s, e) if e - s < 40 else sorted({s, s + 1, s + 31, min(s + 128, e - 1), (s + e) // 2, *range(e - 12, e)})
        for t in pick:
            p = b.lens[r] - int(b.row_start[r + 1]) + t
            lo, hi = max(0, p - window + 1) if window else 0, min(p + 1, tokens)
            if hi <= lo:
                assert (got[t] == 0).all() and torch.isneginf(lse[t]).all(), (r, t)
                continue
            w, l, m, top = ref.attention(b.q.double()[t:t + 1], [b.keys[r][lo:hi]], [b.values[r][lo:hi]], [0, 1], [hi - lo],
                                         b.D ** -0.5, 0)
            tol = 3 * ref.UNIT[b.dt] + 2.0 ** -18 * (1 + top)
            assert ((got[t] - w[0]).abs() <= tol * m[0] + ref.STEP[b.dt]).all(), (r, t)
            assert ((lse[t] - l[0]).abs() <= tol).all(), (r, t)


@pytest.mark.parametrize("window", [0, 25])
@pytest.mark.parametrize("kind", GIVEN)
def test_rows_of_a_request_that_the_call_does_not_have(kind, window):
    """A step with fewer rows than new tokens has the first rows of its last requests, not their last ones."""
    new, lens, H, kw = GIVEN[kind]
    H = H if H < 64 else 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch(new, lens, H, H, 64, 32, BF, seed=28, extra=40 if kind == "wide" else 0)
    _check_given(b, sum(new) - (1 if max(new) < 9 else 7), max(lens), window, **kw)


@pytest.mark.parametrize("window", [0, 25])
@pytest.mark.parametrize("kind", GIVEN)
def test_tokens_past_the_table(kind, window):
    """Requests longer than the table's pages: rows keep their positions and see the tokens that have pages."""
    new, lens, H, kw = GIVEN[kind]
    H = H if H < 64 else 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch(new, lens, H, H, 64, 32, BF, seed=29)
    width = max(2, b.table.shape[1] - 1)
    if kind == "wide":                               # pages that no token has, so that the launch counts on many
        kw = dict(max_len=2200)
    b.table = b.table[:, :width].contiguous()
    _check_given(b, sum(new), 32 * width, window, **kw)
    if kind not in ("wide", "splits"):
        b.table = b.table[:, :1].contiguous()
        _check_given(b, sum(new), 32, window, **kw)


@pytest.mark.parametrize("new,length,H", [([1], 50, 4), ([1], 9000, 4), ([20], 50, 4), ([600], 600, 64)])
def test_rows_whose_scores_are_all_minus_infinity(new, length, H):
    """As rows that see no key: 0 and -inf; beside them a head whose scores are finite."""
    H = H if H < 64 else 64 * torch.cuda.get_device_properties(0).multi_processor_count // 256
    b = Batch(new, [length], H, H, 64, 64, BF, seed=30)
    k = torch.full((length, H, 64), -2.0, dtype=BF)
    at = torch.arange(length)
    slots = (b.table[0].cpu()[at // 64] * 64 + at % 64).int().cuda()
    _spl().qk_norm_rope_append(k.cuda(), k.cuda(), b.values[0].to(BF).cuda(), None, None, slots, b.cache)
    clean = b.run()[0]
    assert torch.isfinite(clean).all()
    b.q[:, 1, 7] = float("inf")
    got, lse = b.run()
    assert (got[:, 1] == 0).all() and torch.isneginf(lse[:, 1]).all()
    others = [h for h in range(H) if h != 1]
    assert torch.equal(got[:, others], clean[:, others])
