"""block_tables on the GPU against its definition, token by token; every number exact."""
import numpy as np
import pytest

import _attn_ref as ref

pytestmark = pytest.mark.gpu


def _run(cached, new, table, free, head, page, tokens):
    import torch

    import paper_2405_03594_amd as spl

    dev = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    t = dev(table)
    plan = spl.block_tables(dev(cached), dev(new), t, dev(free), dev([head]), page, tokens)
    again = t.clone()
    plan2 = spl.block_tables(dev(cached), dev(new), again, dev(free), dev([head]), page, tokens)
    torch.cuda.synchronize()
    got = {n: getattr(plan, n).cpu().numpy() for n in ("row_start", "lens", "positions", "slots")}
    got.update(table=t.cpu().numpy(), free_head=int(plan.free_head), missing=int(plan.missing))
    assert torch.equal(t, again) and torch.equal(plan.slots, plan2.slots)          # the call can be repeated
    return got


def _check(cached, new, table, free, head, page, tokens):
    got = _run(cached, new, table, free, head, page, tokens)
    want = ref.tables(cached, new, table, free, head, page, tokens)
    for n in ("table", "row_start", "lens", "positions", "slots"):
        assert np.array_equal(got[n], np.asarray(want[n])), n
    assert got["free_head"] == want["free_head"]
    assert (got["missing"] == 0) == (want["missing"] == 0)
    if sum(max(int(n), 0) for n in new) <= tokens:
        assert got["missing"] == want["missing"]


def _case(seed, R, page, most_cached, most_new, zero=0.2):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, most_cached + 1, R)
    new = np.where(rng.random(R) < zero, 0, rng.integers(1, most_new + 1, R))
    width = -(-(most_cached + most_new) // page) + 1
    held = -(-cached // page)
    total = int(held.sum() + (-(-(cached + new) // page) - held).sum()) + 5
    ids = rng.permutation(total)
    table = np.full((R, width), -1)
    n = 0
    for r in range(R):
        table[r, :held[r]] = ids[n:n + held[r]]
        n += held[r]
    return cached, new, table, ids, n


@pytest.mark.parametrize("R,page,most_cached,most_new", [
    (1, 16, 0, 1), (1, 16, 15, 1), (1, 16, 16, 1), (1, 64, 100, 700), (3, 16, 40, 1), (64, 32, 300, 5), (65, 128, 1000, 40),
    (255, 256, 600, 3), (1023, 16, 50, 2), (1024, 16, 50, 2), (1025, 16, 50, 2), (2500, 16, 33, 4), (7, 16, 900, 6000)])
def test_tables(R, page, most_cached, most_new):
    cached, new, table, free, head = _case(R * 7 + page, R, page, most_cached, most_new)
    _check(cached, new, table, free, head, page, int(new.sum()))


def test_rows_past_the_last_request_and_tokens_past_the_rows():
    cached, new, table, free, head = _case(5, 20, 16, 90, 30)
    _check(cached, new, table, free, head, 16, int(new.sum()) + 300)
    _check(cached, new, table, free, head, 16, int(new.sum()) - 17)
    _check(cached, np.zeros_like(new), table, free, head, 16, 0)
    _check(cached, np.zeros_like(new), table, free, head, 16, 12)


@pytest.mark.parametrize("short", [1, 5, 1000])
def test_a_free_list_that_runs_out(short):
    cached, new, table, free, head = _case(6, 40, 16, 90, 60)
    _check(cached, new, table, free[:max(head, len(free) - 5 - short)], head, 16, int(new.sum()))
    _check(cached, new, table, free[:0], 0, 16, int(new.sum()))


def test_a_table_that_is_too_narrow():
    cached, new, table, free, head = _case(8, 30, 16, 200, 90)
    for width in (1, 4, table.shape[1] - 3):
        _check(cached, new, table[:, :width], free, head, 16, int(new.sum()))


def test_negative_lengths_missing_pages_and_odd_heads():
    cached, new, table, free, head = _case(9, 12, 32, 100, 50)
    cached, new, table = cached.copy(), new.copy(), table.copy()
    cached[3] = -7
    new[4] = -2
    cached[5], table[5] = 40, -1                     # a request whose pages are gone
    _check(cached, new, table, free, head, 32, int(np.maximum(new, 0).sum()))
    _check(cached, new, table, free, -5, 32, int(np.maximum(new, 0).sum()))
    _check(cached, new, table, free, len(free) + 9, 32, int(np.maximum(new, 0).sum()))


@pytest.mark.parametrize("short", [0, 1, 4, 1000])
@pytest.mark.parametrize("rows", [0, 1, 50, 300, 10 ** 6])
def test_a_token_without_a_row_and_a_slot_is_missing_once(rows, short):
    """Too few rows and a free list that runs out: what is missing is the tokens that lack one or both, token by token."""
    cached, new, table, free, head = _case(11, 30, 16, 90, 40)
    total = int(new.sum())
    rows = min(rows, total + 20)
    free = free[:max(head, len(free) - 5 - short)]
    slots = ref.tables(cached, new, table, free, head, 16, total)["slots"]
    want = sum(t >= rows or slots[t] < 0 for t in range(total))
    assert _run(cached, new, table, free, head, 16, rows)["missing"] == want
    gone = table.copy()
    gone[::3] = -1                                   # requests whose pages are gone
    slots = ref.tables(cached, new, gone, free, head, 16, total)["slots"]
    want = sum(t >= rows or slots[t] < 0 for t in range(total))
    assert _run(cached, new, gone, free, head, 16, rows)["missing"] == want
