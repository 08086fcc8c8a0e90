"""The paged cache at lengths of many millions of rows.  All entries of a table name a few pages (pages may be shared),
so the pools stay small."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE, PAGES = 1024, 64


def _far(kv, n_new, group):
    """One sequence of kv rows, row t in page (t / 1024) % 64, one kv head; queries and keys of zeros."""
    from paper_2508_17892_b200 import PagedCache
    eng = PagedCache(n_kv_heads=1, n_q_heads=group, page_size=PAGE, max_seqs=1)
    blocks = -(-kv // PAGE)
    table = (torch.arange(blocks, dtype=torch.int32, device="cuda") % PAGES)[None].contiguous()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = eng.batch(i32(0, n_new), i32(kv), table, n_new, n_new)
    q = torch.zeros(n_new, group, 128, dtype=torch.bfloat16, device="cuda")
    k_pool = torch.zeros(PAGES, PAGE, 1, 128, dtype=torch.bfloat16, device="cuda")
    return eng, batch, q, k_pool


def _rows_per_slot(kv):
    """How many of the rows 0 .. kv - 1 lie in each (page, row of the page)."""
    full, rest = divmod(kv, PAGE * PAGES)
    count = torch.full((PAGES * PAGE,), full, dtype=torch.int64)
    count[:rest] += 1
    return count


# 32 heads share tiles of two tokens, 16 of four; the last tile is not full, so every key tile is masked.  Head and
# token distance multiplied pass 2^31 behind 67 and 134 million rows.  One token: the kernel of few rows.
@pytest.mark.parametrize("group,n_new,kv", [(32, 3, 68_000_001), (16, 5, 135_000_003), (16, 1, 135_000_003)])
def test_weights_of_far_rows(group, n_new, kv):
    """Logits and lse are 0, so a visible (head, token, row) gives exactly 1: the weights are counts (below 2^24, exact in
    any order of addition)."""
    eng, batch, q, k_pool = _far(kv, n_new, group)
    w = torch.zeros(PAGES, 1, PAGE, device="cuda")
    eng.accumulate(batch, q, torch.zeros(n_new, group, device="cuda"), k_pool, w)
    eng.check_status()
    want = sum(_rows_per_slot(kv - n_new + 1 + j) for j in range(n_new)) * group
    assert int(want.max()) < 1 << 24
    assert torch.equal(w.flatten().long().cpu(), want)
    eng.close()


@pytest.mark.parametrize("group,n_new,kv", [(32, 3, 68_000_001), (16, 1, 135_000_003)])
def test_attention_over_far_rows(group, n_new, kv):
    """Equal logits: the output is the mean of the values (1 in even rows of a page, 0 in odd ones), lse the logarithm of
    the rows that a token sees."""
    eng, batch, q, k_pool = _far(kv, n_new, group)
    v_pool = torch.zeros_like(k_pool)
    v_pool[:, ::2] = 1.0
    out, lse = eng.attention(batch, q, k_pool, v_pool, want_lse=True)
    eng.check_status()
    for j in range(n_new):
        rows = kv - n_new + 1 + j
        want = ((rows + 1) // 2) / rows
        # A CTA's sums are whole numbers below 2^24 (under 10^6 rows each), so exact; adding up at most 300 of them is off
        # by 300 * 2^-24 < 2^-15.7 of the total, in numerator and denominator; the division and the logarithm (of about 27,
        # in ln units 18) by 2^-22 of themselves; the output is rounded to bf16 (2^-8).
        assert float((out[j].double() - want).abs().max()) <= (2.0 ** -8 + 2.0 ** -14) * want
        assert float((lse[j].double() - math.log(rows)).abs().max()) <= 2.0 ** -15
    eng.close()
