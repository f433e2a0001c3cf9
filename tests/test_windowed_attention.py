"""Sliding-window attention with sinks: the planner's lists on a host-only pool, and the kernels against a plain
64-bit implementation.  Hidden keys are made unusable wherever the contract allows it: table entries of pages that
no new token sees are -1, hidden tokens of the pages that remain hold NaN in K and V."""
import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import operator_reference as R

BIG = 2 ** 31 - 1
WINDOWS = [(1, 0), (1, 1), (7, 3), (16, 0), (16, 16), (33, 17), (100, 4), (128, 0), (129, 130), (500, 20), (4000, 0), (BIG, 0),
           (5, BIG), (BIG, BIG)]


def _hide(batch, window, sinks, rows_per_block=1 << 30):
    """-1 for table entries of pages that no new token of the sequence sees; the pages' number."""
    cut = 0
    for s in range(batch.batch):
        n, ctx = int(batch.q_lens[s]), int(batch.ctx_lens[s])
        if n == 0:
            continue
        seen = R.visible(n, ctx, window, sinks).any(0)
        for lp in range((ctx + 15) // 16):
            part = seen[lp * 16:(lp + 1) * 16]
            if not part.any():
                batch.block_tables[s, lp] = -1
                cut += 1
            elif batch.k_pool is not None:
                slots = np.nonzero(~part)[0]
                batch.k_pool[batch.block_tables[s, lp], :, slots] = W.CANARY
                batch.v_pool[batch.block_tables[s, lp], :, slots] = W.CANARY
    return cut


def _batch(shape, seed, q_lens, ctx_lens, with_pool=True):
    return W._assemble(f"window_{seed}", shape, W.make_rng(seed), np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32),
                       1.3, with_pool=with_pool)


RAGGED = ([1] * 12 + [0, 2, 5, 100, 129, 300, 128],
          [1, 2, 15, 16, 17, 33, 64, 100, 129, 700, 1300, 2049, 50, 2, 700, 133, 600, 300, 1025])


@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_windowed_plan_lists(window, sinks):
    """Every visible (row, key) pair is covered exactly once by the lists under the kernels' mask rule, every table
    entry in them is that of the right page, and no hidden page is listed more than the page's granularity asks for."""
    b = _batch((8, 2, 64), 3, *RAGGED, with_pool=False)
    true_table = b.block_tables.copy()
    _hide(b, window, sinks)
    pool = ap.kv_pool_create(b.num_pages, 2, 64, device=-1)
    plan = ap.plan_create_windowed(pool, b.q_lens, b.ctx_lens, b.block_tables, 8, window, sinks)
    ex = ap.plan_export(plan)
    info, hb, bt = ex["info"], ex["info"]["decode_head_block"], ex["bt_flat"]
    rows = b.q_indptr
    total_seen = pairs = 0
    for s in range(b.batch):
        n, ctx = int(b.q_lens[s]), int(b.ctx_lens[s])
        if n:
            see = R.visible(n, ctx, window, sinks)
            total_seen += int(see.any(0).sum())
            pairs += int(see.sum()) if n > 1 else 0
    assert info["kv_tokens"] == total_seen and info["prefill_pairs"] == pairs

    def keys_of(row, pages, vpos, vlen):
        """(page, slot) of the keys the row at compacted position vpos sees, by the kernels' rule."""
        v = np.arange(min(vlen, 16 * len(pages)))
        v = v[(v <= vpos) & ((v > vpos - window) | (v < sinks))]
        return [(int(pages[i // 16]), int(i % 16)) for i in v]

    for s in range(b.batch):
        n, ctx = int(b.q_lens[s]), int(b.ctx_lens[s])
        want = [[(int(true_table[s, j // 16]), int(j % 16)) for j in np.nonzero(r)[0]] for r in R.visible(n, ctx, window, sinks)]
        if n == 1:
            items = ex["decode_items"][ex["decode_items"][:, 0] == rows[s]]
            for head in range(0, 2, hb):
                its = sorted((it for it in items.tolist() if it[1] == head), key=lambda it: it[3])
                kv_len = its[0][5]
                covered = [p for it in its for p in range(it[3], it[3] + it[4])]
                assert covered == list(range((kv_len + 15) // 16))
                pages = bt[its[0][2]:its[0][2] + len(covered)]
                assert all(it[2] == its[0][2] and it[5] == kv_len for it in its)
                assert keys_of(0, pages, kv_len - 1, kv_len) == want[0]
                lo = max(0, kv_len - window)             # a kept page shows at least one key
                for i in range(len(covered)):
                    assert 16 * i < sinks or 16 * i + 16 > lo
        for r0, nr, qh, kvh, off, pos0, vctx, qb in ex["prefill_tiles"].tolist():
            if rows[s] <= r0 < rows[s + 1] and qh == 0:
                pages = bt[off:off + (vctx + 15) // 16]
                assert vctx == pos0 + nr
                for r in range(nr):
                    assert keys_of(r, pages, pos0 + r, vctx) == want[r0 - rows[s] + r]
    covered_rows = sorted(r for t in ex["prefill_tiles"].tolist() if t[2] == 0 for r in range(t[0], t[0] + t[1]))
    assert covered_rows == [r for s in range(b.batch) if b.q_lens[s] > 1 for r in range(rows[s], rows[s + 1])]
    assert (bt >= 0).all()
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


def test_windowed_plan_refusals_and_predictions():
    pool = ap.kv_pool_create(64, 2, 64, device=-1)
    bt = np.arange(40, dtype=np.int32)[None]
    for window, sinks in ((0, 0), (-1, 4), (4, -1), (-2 ** 32 + 9, 0), (4, -2 ** 40)):
        with pytest.raises(ap.ApError) as e:
            ap.plan_create_windowed(pool, [1], [600], bt, 8, window, sinks)
        assert e.value.status == B.AP_ERR_INVALID_ARG
    # an entry of a visible page is validated, one of a hidden page is not
    bad = bt.copy()
    bad[0, 3] = -7
    ap.plan_destroy(ap.plan_create_windowed(pool, [1], [600], bad, 8, 100, 4))
    for window, sinks in ((600, 0), (1, 49), (552, 0)):
        with pytest.raises(ap.ApError) as e:
            ap.plan_create_windowed(pool, [1], [600], bad, 8, window, sinks)
        assert e.value.status == B.AP_ERR_BAD_BLOCK_TABLE
    # what ap_plan_create refuses is refused here too
    for args, status in ((([2], [1], bt, 8), B.AP_ERR_INVALID_ARG), (([1], [641], bt, 8), B.AP_ERR_INVALID_ARG),
                         (([1], [33], bt, 7), B.AP_ERR_INVALID_ARG), (([1], [33], bt, 32), B.AP_ERR_UNSUPPORTED)):
        with pytest.raises(ap.ApError) as e:
            ap.plan_create_windowed(pool, *args, 16, 0)
        assert e.value.status == status
    # the work figures count visible keys: 100 + 4 of a decode row
    plan = ap.plan_create_windowed(pool, [1], [600], bt, 8, 100, 4)
    full = ap.plan_create(pool, [1], [600], bt, 8)
    wide = ap.plan_create_windowed(pool, [1], [600], bt, 8, 2 ** 32 + 5, 2 ** 33)        # (not 5 and 0)
    pw, pf = ap.plan_predict(plan), ap.plan_predict(full)
    assert pw["decode_flops"] == 4 * 8 * 64 * 104 and pf["decode_flops"] == 4 * 8 * 64 * 600
    assert pw["decode_bytes"] < pf["decode_bytes"] and ap.plan_predict(wide) == pf
    for p in (plan, full, wide):
        ap.plan_destroy(p)
    ap.kv_pool_destroy(pool)


def _check(batch, window, sinks, **kw):
    _hide(batch, window, sinks)
    dev = R.Device(batch, lambda pool: ap.plan_create_windowed(pool, batch.q_lens, batch.ctx_lens, batch.block_tables,
                                                               batch.num_q_heads, window, sinks), **kw)
    try:
        ap.kv_append(dev.pool, dev.plan, dev.k_new, dev.v_new)
        dev.attend()
        out, lse = dev.results()
        k, v = (W.bf16_bits_to_f64(R.to_bits(p)) for p in (dev.k_pool, dev.v_pool))
        ref = R.attention(lambda s: R.table_rows(batch, k, s), lambda s: R.table_rows(batch, v, s), batch, window, sinks)
        R.check(out, lse, ref, f"window {window} sinks {sinks}")
        return dev.info
    finally:
        dev.close()


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_windowed_decode(window, sinks):
    for shape in ((32, 8, 128), (8, 2, 64)):
        _check(_batch(shape, 11, [1] * 13 + [0], [1, 2, 15, 16, 17, 31, 33, 64, 100, 129, 700, 1300, 9001, 77]), window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_windowed_prefill(window, sinks):
    for shape in ((6, 2, 128), (8, 4, 64)):
        _check(_batch(shape, 12, [2, 5, 100, 129, 300, 128, 200], [2, 700, 133, 600, 300, 1025, 201]), window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 8, 64), (5, 1, 128), (64, 8, 128)], ids=str)
@pytest.mark.parametrize("mode,single", [(0, True), (3, True), (3, False)], ids=["sequential", "one_launch", "two_streams"])
def test_windowed_mixed_iterations(shape, mode, single):
    info = _check(_batch(shape, 13, [150, 1, 1, 1, 40], [400, 90, 1300, 17, 1000]), 200, 4, side_by_side=mode, single_launch=single)
    assert info["side_by_side"] == (1 if mode else 0)


@pytest.mark.gpu
def test_a_window_that_covers_the_context_gives_the_plain_result():
    """Decode rows: same pages, same arithmetic, same order of summation, so bit for bit what the plan without a window
    gives.  Prefill rows use a finer polynomial for one weight in eight (2.7e-6 of it instead of 7.7e-5), so their bits
    may differ; both are held against the 64-bit result."""
    b = _batch((32, 8, 128), 14, [1, 1, 1, 70], [40, 3000, 129, 500])
    got = []
    for make in (None, lambda pool: ap.plan_create_windowed(pool, b.q_lens, b.ctx_lens, b.block_tables, 32, BIG, 7)):
        dev = R.Device(b, make, side_by_side=0)
        ap.kv_append(dev.pool, dev.plan, dev.k_new, dev.v_new)
        dev.attend()
        got.append(dev.results())
        k, v = (W.bf16_bits_to_f64(R.to_bits(p)) for p in (dev.k_pool, dev.v_pool))
        dev.close()
    ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b)
    for out, lse in got:
        R.check(out, lse, ref)
    assert np.array_equal(got[0][0][:3], got[1][0][:3]) and np.array_equal(got[0][1][:3], got[1][1][:3])


@pytest.mark.gpu
@pytest.mark.parametrize("window", [None, BIG], ids=["plain", "windowed"])
@pytest.mark.parametrize("mode,q_lens,ctx_lens", [
    (6, [1, 1, 1, 1, 8, 1, 1, 1], [935, 877, 16, 1242, 706, 669, 865, 596]),
    (3, [1, 1, 1, 1, 1, 1, 1, 44], [10, 158, 59, 13, 79, 161, 31, 86])])
def test_items_of_a_page_or_two_read_their_own_queries(window, mode, q_lens, ctx_lens):
    """Decode rows of a page or two between long ones, 32 query heads per item, a few SMs: the producer runs two items
    ahead, and the query buffer of an item must not be refilled while a warp's loads from it are in flight.  The lists
    and the order of every sum are fixed, so all runs have to agree bit for bit with one that the reference has passed."""
    b = _batch((64, 8, 128), 15, q_lens, ctx_lens)
    make = None if window is None else (
        lambda pool: ap.plan_create_windowed(pool, b.q_lens, b.ctx_lens, b.block_tables, 64, window, 0))
    for single in (True, False):
        dev = R.Device(b, make, side_by_side=mode, single_launch=single)
        ap.kv_append(dev.pool, dev.plan, dev.k_new, dev.v_new)
        k, v = (W.bf16_bits_to_f64(R.to_bits(p)) for p in (dev.k_pool, dev.v_pool))
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b)
        dev.attend()
        first = dev.results()
        for run in range(500):
            dev.attend()
            if run % 4 == 3:
                out, lse = dev.results()
                assert np.array_equal(out, first[0]) and np.array_equal(lse, first[1]), f"run {run}, single launch {single}"
        dev.close()
        R.check(*first, ref)
