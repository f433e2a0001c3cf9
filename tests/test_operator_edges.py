"""Edges of the operators on paged pools: values of every size, what masked keys may hold, what a NaN does."""
import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import kv4_reference as Q
import operator_reference as R
from harness import to_bits, to_dev


def _batch(shape, seed, q_lens, ctx_lens, with_pool=True):
    return W._assemble(f"edges_{seed}", shape, W.make_rng(seed), np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32),
                       1.3, with_pool=with_pool)


def _times(bits, factor):
    """bf16 bits of the values times a power of two; slots without a token stay as they are."""
    scaled = W.f32_to_bf16_bits((W.bf16_bits_to_f64(bits) * factor).astype(np.float32))
    return np.where(bits == W.CANARY, bits, scaled)


def _put_row(plane, page, slot, bits, four_bit):
    if four_bit:
        Q.put(plane, np.array([page]), np.array([slot]), bits[None])
    else:
        plane[page, :, slot] = bits


def _planes(batch, four_bit):
    """(K, V) planes as numpy, with the batch's new tokens in place."""
    planes = list(Q.planes_of(batch)) if four_bit else [batch.k_pool.copy(), batch.v_pool.copy()]
    page, slot = Q.new_slots(batch)
    for plane, new in zip(planes, (batch.k_new, batch.v_new)):
        for i in range(batch.n_new):
            _put_row(plane, page[i], slot[i], new[i], four_bit)
    return planes


def _attend(batch, planes, four_bit, window=None, sinks=0):
    """(out bits, lse, k, v): the library's attention over the planes, and the values they stand for in float64."""
    make = None if window is None else (lambda pool: ap.plan_create_windowed(
        pool, batch.q_lens, batch.ctx_lens, batch.block_tables, batch.num_q_heads, window, sinks))
    dev = R.Device(batch, make, k_plane=planes[0], v_plane=planes[1], four_bit=four_bit)
    try:
        dev.attend()
        out, lse = dev.results()
    finally:
        dev.close()
    k, v = (Q.values(p, batch.head_dim) if four_bit else W.bf16_bits_to_f64(p) for p in planes)
    return out, lse, k, v


def _check_of_any_size(out_bits, lse, ref, longest, what):
    """operator_reference.check without its absolute slack: the value that is rounded to bf16 at the end is within
    s = (2^-8 + 2e-4) A of ref, plus longest 2^-149 for sums of at most `longest` products that may round to fp32's
    subnormals, each addition and each product by 2^-150.  The rounding adds half an ulp of bf16 at up to |ref| + s (s may
    cross into the next binade), which is never below half a subnormal's, 2^-134."""
    ref_out, ref_lse, absw = ref
    got = W.bf16_bits_to_f64(out_bits)
    assert np.isfinite(got).all() and np.isfinite(lse).all(), f"{what}: non-finite output"
    s = absw * (2.0 ** -8 + 2e-4) + longest * 2.0 ** -149
    half_ulp = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(ref_out) + s, 1e-300))) - 8), 2.0 ** -134)
    excess = np.abs(got - ref_out) - (s + half_ulp)
    i = np.unravel_index(np.argmax(excess), excess.shape)
    assert excess[i] <= 0, f"{what}: {got[i]} against {ref_out[i]} at {i} (A {absw[i]})"
    lerr = np.abs(lse - ref_lse)
    assert (lerr <= 2e-4 + 1e-5 * np.abs(ref_lse)).all(), f"{what}: lse off by {lerr.max()}"


# ------------------------------------------------------------- every size --

SIZES = [(0, 0, 100), (0, 0, -100), (0, 0, 117), (0, 0, -118), (0, 0, -127), (100, -100, 0), (-100, 100, 0), (117, -117, 117),
         (-117, 113, -117)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 2, 64), (6, 2, 128)], ids=str)
@pytest.mark.parametrize("k_log2,q_log2,v_log2", SIZES)
def test_4bit_attention_over_values_of_one_size(shape, k_log2, q_log2, v_log2):
    """Every value of a plane, new tokens included, near one power of two, so that steps are near 2^-130 .. 2^117 and nothing
    larger hides them; q by the inverse of K's size, so that scores stay those of N(0, 1) rows.  Decode and prefill
    rows, with and without a window."""
    b = _batch(shape, 61, [1, 1, 1, 20, 150], [200, 37, 2100, 64, 300])
    b.k_pool, b.v_pool, b.q = _times(b.k_pool, 2.0 ** k_log2), _times(b.v_pool, 2.0 ** v_log2), _times(b.q, 2.0 ** q_log2)
    b.k_new, b.v_new = _times(b.k_new, 2.0 ** k_log2), _times(b.v_new, 2.0 ** v_log2)
    planes = _planes(b, True)
    for window, sinks in ((None, 0), (90, 4)):
        out, lse, k, v = _attend(b, planes, True, window, sinks)
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b, window, sinks)
        _check_of_any_size(out, lse, ref, 2100, f"window {window}")


@pytest.mark.gpu
@pytest.mark.parametrize("value", [2.0 ** 114, 2.0 ** 116, 2.0 ** 118, 2.0 ** 121 * (1 - 2.0 ** -8)], ids=lambda v: f"{v:.3g}")
def test_4bit_queries_up_to_the_stated_limit(value):
    """All elements of a query equal, just below the 2^121 from which a head's result is NaN; K as much smaller.  Scores: at most
    d products of 8 |k'| (k' ~ N(0, 1) / 8), as for N(0, 1) rows."""
    for shape in ((8, 2, 64), (6, 2, 128)):
        b = _batch(shape, 62, [1, 1, 1, 40], [200, 33, 1500, 90])
        b.q[:] = W.f32_to_bf16_bits(np.array([value], np.float32))[0]
        b.k_pool, b.k_new = (_times(x, 2.0 ** -np.ceil(np.log2(value))) for x in (b.k_pool, b.k_new))
        planes = _planes(b, True)
        out, lse, k, v = _attend(b, planes, True)
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b)
        _check_of_any_size(out, lse, ref, 1500, f"q {value}")


# ----------------------------------------------------------- masked places --

@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
@pytest.mark.parametrize("window,sinks", [(None, 0), (24, 3)])
def test_a_masked_key_weighs_nothing_however_large_its_v(four_bit, window, sinks):
    """Rows of a block that do not see a key, which other rows of the same block see, get none of its V of 2^119."""
    for shape in ((6, 2, 128), (8, 2, 64)):
        b = _batch(shape, 63, [128, 200], [128, 500])
        planes = _planes(b, four_bit)
        big = np.full((shape[1], shape[2]), W.f32_to_bf16_bits(np.array([2.0 ** 119], np.float32))[0], np.uint16)
        large = {0: range(64, 128), 1: range(400, 432)}
        for s, keys in large.items():
            for j in keys:
                _put_row(planes[1], b.block_tables[s, j // 16], j % 16, big, four_bit)
        out, lse, k, v = _attend(b, planes, four_bit, window, sinks)
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b, window, sinks)
        _check_of_any_size(out, lse, ref, 500, f"window {window}")


@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
@pytest.mark.parametrize("window", [None, 40])
def test_a_visible_nan_key_makes_its_rows_nan_and_no_others(four_bit, window):
    """K of one token is NaN: every row that sees the token is NaN in out and lse, every other row is as if it were not there.
    The token in turn at each place of a 16-token page (the softmax treats keys differently by their place)."""
    shape = (6, 2, 128)
    b = _batch(shape, 64, [1, 70, 1, 150], [100, 90, 700, 400])
    nan = np.full((2, 128), 0x7FC0, np.uint16)
    clean = _planes(b, four_bit)
    for place in range(16):
        planes = [p.copy() for p in clean]
        bad = {0: 80 + place, 1: 32 + place, 2: 672 + place, 3: 320 + place}
        for s, j in bad.items():
            _put_row(planes[0], b.block_tables[s, j // 16], j % 16, nan, four_bit)
        out, lse, _, v = _attend(b, planes, four_bit, window)
        got, row = W.bf16_bits_to_f64(out), 0
        k = Q.values(clean[0], 128) if four_bit else W.bf16_bits_to_f64(clean[0])
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b, window)
        for s in range(4):
            n, ctx = int(b.q_lens[s]), int(b.ctx_lens[s])
            sees = R.visible(n, ctx, window)[:, bad[s]]
            o, l = got[row:row + n], lse[row:row + n]
            assert np.isnan(o[sees]).all() and np.isnan(l[sees]).all(), f"place {place}, sequence {s}"
            part = [x[row:row + n][~sees] for x in ref]
            if not sees.all():
                R.check(out[row:row + n][~sees], l[~sees], part, f"place {place}, sequence {s}")
            row += n


# --------------------------------------------------------- overlapped launches --

def test_only_plan_lists_are_read_through_the_read_only_path():
    """A kernel may be resident while the one before still writes its inputs, and the read-only path may then hand out
    stale lines: __ldg is for lists that were uploaded before any kernel of the step."""
    import os
    import re
    from paper_2604_07144_b200 import build
    lists = ("append_dst", "positions", "pages", "pairs", "cta_begin", "cur_bt", "bt", "bt_flat", "src", "&merges")
    found = 0
    for name in sorted(os.listdir(build.CSRC)):
        text = re.sub(r"//.*", "", open(os.path.join(build.CSRC, name)).read())
        for arg in re.findall(r"__ldg\(\s*(&?\w+)", text):
            assert arg in lists, f"{name}: __ldg({arg} ...)"
            found += 1
    assert found >= 10


@pytest.mark.gpu
@pytest.mark.parametrize("shape,n", [((8, 2, 64), 3), ((32, 8, 128), 40), ((32, 8, 128), 900)], ids=str)
def test_rows_read_back_from_one_pool_and_appended_to_another_at_once(shape, n):
    """append to a 4-bit pool -> read back -> append to a bf16 pool -> read back, 24 steps with new data through the same
    buffers, captured without a gap: the rows in the bf16 pool are those that the 4-bit pool stands for."""
    import torch
    hq, hkv, d = shape
    b = _batch(shape, 65, [1] * n, [1 + (7 * i) % 60 for i in range(n)], with_pool=False)
    gen = torch.Generator(device="cuda:0").manual_seed(7)
    k, v = (torch.randn((24, n, hkv, d), generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(2))
    pools = [ap.kv_pool_create_4bit(b.num_pages, hkv, d), ap.kv_pool_create(b.num_pages, hkv, d)]
    plans = [ap.plan_create(p, b.q_lens, b.ctx_lens, b.block_tables, hq) for p in pools]
    mid = [torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]

    def steps(sync):
        res = [torch.zeros((24, n, hkv, d), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]

        def run():
            for i in range(24):
                ap.kv_append(pools[0], plans[0], k[i], v[i])
                sync()
                ap.kv_read_new(pools[0], plans[0], mid[0], mid[1])
                sync()
                ap.kv_append(pools[1], plans[1], mid[0], mid[1])
                sync()
                ap.kv_read_new(pools[1], plans[1], res[0][i], res[1][i])
                sync()
        return run, res
    run, alone = steps(torch.cuda.synchronize)
    run()
    assert not torch.equal(alone[0][0], alone[0][1])
    run, chained = steps(lambda: None)
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=st):
        run()
    for _ in range(20):
        for x in chained + mid:
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(ap.last_device_status(p) == 0 for p in pools)
        assert all(torch.equal(x, y) for x, y in zip(chained, alone))
    del g
    for p in plans:
        ap.plan_destroy(p)
    for p in pools:
        ap.kv_pool_destroy(p)


# -------------------------------------------------------------------- refusals --

def _host_plan(shape=(8, 2, 64), rows=4):
    hq, hkv, d = shape
    pool = ap.kv_pool_create(64, hkv, d, device=-1)
    return pool, ap.plan_create(pool, [1] * rows, [20] * rows, np.arange(2 * rows, dtype=np.int32).reshape(rows, 2), hq)


def test_strided_tensors_are_refused_where_the_library_reads_or_writes_rows_in_a_row():
    """Slices of one projection, expanded and transposed tensors, every second row: the rotated append takes row strides,
    nothing else does."""
    import torch
    pool, plan = _host_plan()
    fused = torch.zeros((4, 12, 64), dtype=torch.bfloat16)
    q, k = torch.zeros((4, 8, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    lse, ws = torch.zeros((4, 8)), torch.zeros(1 << 16, dtype=torch.uint8)
    bad_k = [fused[:, 8:10], k[:1].expand(4, 2, 64), torch.zeros((2, 4, 64), dtype=torch.bfloat16).transpose(0, 1),
             torch.zeros((8, 2, 64), dtype=torch.bfloat16)[::2], torch.zeros((4, 2, 128), dtype=torch.bfloat16)[:, :, ::2]]
    bad_q = [fused[:, :8], q[:1].expand(4, 8, 64), torch.zeros((8, 8, 64), dtype=torch.bfloat16)[::2]]
    for bad in bad_k:
        for call in (ap.kv_append, ap.kv_read_new):
            for args in ((bad, k), (k, bad)):
                with pytest.raises(ValueError):
                    call(pool, plan, *args)
    for bad in bad_q:
        for call, more in ((ap.attention_iteration, (lse, ws)), (ap.attention_iteration_static, (lse,))):
            for args in ((bad, q), (q, bad)):
                with pytest.raises(ValueError):
                    call(pool, plan, *args, *more)
    for more in ((torch.zeros((8, 4)).t(), ws), (lse, torch.zeros(1 << 17, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            ap.attention_iteration(pool, plan, q, q, *more)
    with pytest.raises(ValueError):
        ap.attention_iteration_static(pool, plan, q, q, torch.zeros((8, 4)).t())
    rows = [np.zeros((4, h, 64), np.uint16) for h in (8, 2, 2, 8)]
    for i in range(4):
        args = list(rows)
        args[i] = np.zeros((4, 2 * args[i].shape[1], 64), np.uint16)[:, ::2]
        with pytest.raises(ValueError):
            ap.serving_iteration_host(pool, [1] * 4, [20] * 4, np.arange(8, dtype=np.int32).reshape(4, 2), 8, *args)
    # what is contiguous, or an address, gets as far as the library, which launches nothing for a host-only pool
    for call in (lambda: ap.kv_append(pool, plan, k, k), lambda: ap.kv_append(pool, plan, 4096, 8192),
                 lambda: ap.kv_read_new(pool, plan, fused[:1, 8:10].repeat(4, 1, 1), k),
                 lambda: ap.attention_iteration(pool, plan, q, q, None, ws),
                 lambda: ap.attention_iteration_static(pool, plan, q, q, lse)):
        with pytest.raises(ap.ApError) as e:
            call()
        assert e.value.status == B.AP_ERR_CUDA
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


def test_tensors_that_are_too_small_or_of_another_type_are_refused():
    """The library gets addresses: rows that are not there would be read past the tensor's end, and fp16 or fp32 as bf16."""
    import torch
    pool, plan = _host_plan()
    bf = torch.bfloat16
    q, k, lse, ws = torch.zeros((4, 8, 64), dtype=bf), torch.zeros((4, 2, 64), dtype=bf), torch.zeros((4, 8)), torch.zeros(1 << 16, dtype=torch.uint8)
    rope = lambda k_new, v_new, **more: ap.kv_append_rope(pool, plan, k_new, v_new, **more)
    for bad in (k[:3], torch.zeros((4, 1, 64), dtype=bf), k.half(), k.float(), k.double(), torch.zeros((4, 2, 64), dtype=torch.int32),
                torch.zeros(4 * 2 * 64 - 1, dtype=bf)):
        for call in (lambda a, b: ap.kv_append(pool, plan, a, b), lambda a, b: ap.kv_read_new(pool, plan, a, b), rope):
            for args in ((bad, k), (k, bad)):
                with pytest.raises(ValueError):
                    call(*args)
    wide = torch.zeros((5, 16, 64), dtype=bf)
    for bad in (wide[:3, :2], wide[:, :3], wide[:, :2].half(), torch.zeros((4, 2, 128), dtype=bf)[:, :, :32]):
        with pytest.raises(ValueError):
            rope(bad, k)
    for bad in (q[:3], q.float(), q.half(), torch.zeros(10, dtype=bf)):
        for args in ((bad, q), (q, bad)):
            with pytest.raises(ValueError):
                ap.attention_iteration(pool, plan, *args, lse, ws)
            with pytest.raises(ValueError):
                ap.attention_iteration_static(pool, plan, *args, lse)
            with pytest.raises(ValueError):
                rope(k, k, q=args[0], q_rot=args[1])
    for bad in (lse[:3], lse.half(), lse.double(), q):
        with pytest.raises(ValueError):
            ap.attention_iteration(pool, plan, q, q, bad, ws)
        with pytest.raises(ValueError):
            ap.attention_iteration_static(pool, plan, q, q, bad)
    with pytest.raises(ValueError):
        ap.attention_iteration(pool, plan, q, q, lse, ws, (1 << 16) + 1)
    rows = [np.zeros((4, h, 64), np.uint16) for h in (8, 2, 2, 8)]
    for i in range(4):
        args = list(rows)
        args[i] = args[i][:3]
        with pytest.raises(ValueError):
            ap.serving_iteration_host(pool, [1] * 4, [20] * 4, np.arange(8, dtype=np.int32).reshape(4, 2), 8, *args)
    with pytest.raises(ValueError):
        ap.serving_iteration_host(pool, [1] * 4, [20] * 4, np.arange(8, dtype=np.int32).reshape(4, 2), 8, *rows, np.zeros((3, 8), np.float32))
    table = np.arange(8, dtype=np.int32).reshape(4, 2)
    for i, bad in ((0, np.float32), (1, np.float16), (2, np.float64), (3, np.int32), (4, np.float64), (4, np.float16), (4, np.uint16)):
        args = rows + [np.zeros((4, 8), np.float32)]
        args[i] = args[i].astype(bad)
        with pytest.raises(ValueError):
            ap.serving_iteration_host(pool, [1] * 4, [20] * 4, table, 8, *args)
    for cast in (lambda x: x, lambda x: x.view(np.int16), lambda x: x.view(np.uint8), lambda x: torch.from_numpy(x.view(np.int16))):
        with pytest.raises(ap.ApError) as e:
            ap.serving_iteration_host(pool, [1] * 4, [20] * 4, table, 8, *(cast(x) for x in rows), np.zeros((4, 8), np.float32))
        assert e.value.status == B.AP_ERR_CUDA
    for create, size in ((ap.kv_pool_create, ap.kv_pool_bytes(8, 2, 64)), (ap.kv_pool_create_4bit, ap.kv_pool_bytes_4bit(8, 2, 64))):
        planes = torch.zeros(size, dtype=torch.uint8), torch.zeros(size - 1, dtype=torch.uint8)
        for args in (planes, planes[::-1]):
            with pytest.raises(ValueError):
                create(8, 2, 64, *args, device=-1)
    # more rows than the plan's, other shapes of the same memory, and bit patterns are fine: the library answers
    for call in (lambda: ap.kv_append(pool, plan, torch.zeros((9, 2, 64), dtype=bf), k.view(4, 128)),
                 lambda: ap.kv_append(pool, plan, k.view(torch.int16), k.view(torch.uint8)),
                 lambda: rope(wide[:, :2], wide[:4, 2:4], q=wide[:, :8], q_rot=torch.zeros((9, 8, 64), dtype=bf)),
                 lambda: ap.attention_iteration(pool, plan, q.view(1, 4, 512), q, lse.view(torch.int32), ws, 1 << 16)):
        with pytest.raises(ap.ApError) as e:
            call()
        assert e.value.status == B.AP_ERR_CUDA
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
def test_a_plan_without_new_tokens_takes_any_tensors_and_touches_none():
    import torch
    b = _batch((8, 2, 64), 70, [0, 0], [40, 20])
    dev = R.Device(b)
    before = dev.k_pool.clone()
    nothing = torch.empty(0, dtype=torch.bfloat16)
    ap.kv_append(dev.pool, dev.plan, nothing, nothing)
    ap.kv_append_rope(dev.pool, dev.plan, nothing, nothing, q=nothing, q_rot=nothing)
    ap.kv_append_rope(dev.pool, dev.plan, dev.k_pool[:, :, 0], None)
    ap.kv_read_new(dev.pool, dev.plan, nothing, nothing)
    ap.attention_iteration(dev.pool, dev.plan, nothing, nothing, nothing, None)
    ap.attention_iteration_static(dev.pool, dev.plan, None, None)
    ap.serving_iteration_host(dev.pool, b.q_lens, b.ctx_lens, b.block_tables, 8, None, None, None, None)
    assert ap.last_device_status(dev.pool) == 0
    assert np.array_equal(to_bits(dev.k_pool), to_bits(before)) and torch.isnan(dev.out.float()).all() and torch.isnan(dev.lse).all()
    dev.close()


@pytest.mark.gpu
def test_host_arrays_are_refused_where_a_kernel_would_read_or_write_them():
    b = _batch((8, 2, 64), 66, [1, 20], [40, 20])
    dev = R.Device(b)
    rows = np.zeros((21, 2, 64), np.uint16)
    for call in (lambda: ap.kv_append(dev.pool, dev.plan, rows, dev.v_new), lambda: ap.kv_read_new(dev.pool, dev.plan, rows, rows),
                 lambda: ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, rows),
                 lambda: ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, q=b.q, q_rot=dev.q),
                 lambda: ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, q=dev.q, q_rot=b.q),
                 lambda: ap.attention_iteration(dev.pool, dev.plan, b.q, dev.out, dev.lse, dev.workspace),
                 lambda: ap.attention_iteration(dev.pool, dev.plan, dev.q, dev.out, np.zeros((21, 8), np.float32), dev.workspace),
                 lambda: ap.attention_iteration(dev.pool, dev.plan, dev.q, dev.out, dev.lse, np.zeros(1 << 16, np.uint8)),
                 lambda: ap.attention_iteration_static(dev.pool, dev.plan, dev.q, b.q),
                 lambda: ap.kv_pool_create(b.num_pages, 2, 64, b.k_pool, b.v_pool)):
        with pytest.raises(ValueError):
            call()
    dev.close()


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused_and_pinned_ones_are_read():
    import torch
    b = _batch((8, 2, 64), 66, [1, 20], [40, 20])
    dev = R.Device(b)
    host = [t.cpu() for t in (dev.k_new, dev.v_new, dev.q)]
    with pytest.raises(ValueError):
        ap.kv_append(dev.pool, dev.plan, host[0], dev.v_new)
    with pytest.raises(ValueError):
        ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, host[1])
    with pytest.raises(ValueError):
        ap.attention_iteration(dev.pool, dev.plan, host[2], dev.out, dev.lse, dev.workspace)
    with pytest.raises(ValueError):
        ap.attention_iteration(dev.pool, dev.plan, dev.q, dev.out, dev.lse.cpu(), dev.workspace)
    with pytest.raises(ValueError):
        ap.attention_iteration(dev.pool, dev.plan, dev.q, dev.out, dev.lse, dev.workspace.cpu())
    with pytest.raises(ValueError):
        ap.kv_pool_create(b.num_pages, 2, 64, dev.k_pool.cpu(), dev.v_pool)
    pinned = [t.pin_memory() for t in host[:2]]
    ap.kv_append(dev.pool, dev.plan, *pinned)
    assert ap.last_device_status(dev.pool) == 0
    page, slot = Q.new_slots(b)
    assert np.array_equal(to_bits(dev.k_pool)[page, :, slot], b.k_new) and np.array_equal(to_bits(dev.v_pool)[page, :, slot], b.v_new)
    dev.close()


# ------------------------------------------------------------------ plan lists --

@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
def test_windowed_table_entries_grow_with_the_prompt_and_not_with_its_square(four_bit):
    """Blocks of query rows share their sequence's entries unless pages between the sinks and their window are left out;
    those that do leave pages out have no more entries than sinks and window ask for."""
    ctx, hkv = 1 << 17, 2
    table = np.random.default_rng(1).permutation(ctx // 16).astype(np.int32)[None]
    pool = (ap.kv_pool_create_4bit if four_bit else ap.kv_pool_create)(ctx // 16, hkv, 64, device=-1)
    blocks = ctx // 128
    for window, sinks, most in ((2 ** 31 - 1, 0, ctx // 16), (ctx, 4, ctx // 16), (4096, 0, ctx // 16), (1, 0, ctx // 16),
                                (5, 2 ** 31 - 1, ctx // 16), (1000, ctx // 2, ctx // 16 + blocks // 2 * (ctx // 32 + 72)),
                                (1024, 4, ctx // 16 + blocks * 74)):
        plan = ap.plan_create_windowed(pool, [ctx], [ctx], table, 2, window, sinks)
        ex = ap.plan_export(plan)
        assert len(ex["bt_flat"]) <= most, (window, sinks)
        # every block's entries are still those of the pages it sees
        number = np.arange(ctx // 16) if four_bit else table[0]
        for r0, nr, qh, _, off, pos0, vctx, _ in ex["prefill_tiles"].tolist()[:: 97]:
            page = np.arange((r0 + nr + 15) // 16)
            first = max(0, r0 - window + 1) // 16
            want = number[page[(page >= first) | (16 * page < sinks)]]
            assert vctx == pos0 + nr and np.array_equal(ex["bt_flat"][off:off + (vctx + 15) // 16], want), (window, sinks, r0)
        ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


# ------------------------------------------------------------------- rotation --

def test_rotation_frequencies_by_repeated_products_are_as_good_as_stated():
    """The rotated append forms base^(-2 i / R) / 2 pi by i products in extended precision and rounds it to 64 bits; the angle
    at position 2^31 is then off by at most 1.04 2^-52 2^31 f_i: two roundings of 2^-53 each, one its product with the
    position, and 64 of 2^-63.  Against 60 digits;
    with 64-bit products base 2 missed it (1.9e-6)."""
    from decimal import Decimal, getcontext
    if np.finfo(np.longdouble).nmant < 63:
        pytest.skip("no extended precision here")
    getcontext().prec = 60
    two_pi = Decimal("6.28318530717958647692528676655900576839433879875021164194989")
    inv_2pi = np.longdouble("0.159154943091895335768883763372514362")
    far = 2 ** 31
    for base in (0.5, 1.0001, 2.0, 10000.0, 500000.0, 1e6, 1e9):
        for rotary in (16, 48, 64, 128):
            ratio, f = np.power(np.longdouble(base), np.longdouble(-2) / np.longdouble(rotary)), np.longdouble(1)
            for i in range(rotary // 2):
                exact = Decimal(base) ** (Decimal(-2 * i) / Decimal(rotary))
                turn = float(f * inv_2pi)
                off = abs(Decimal(far * turn) * two_pi - far * exact)          # far * turn: one rounding, as in the kernel
                assert off <= Decimal(1.04 * 2.0 ** -52 * far) * exact, (base, rotary, i, float(off))
                f = f * ratio


# -------------------------------------------------------------- 32-bit numbers --

def test_slots_and_positions_that_pass_32_bits_are_refused():
    """A plan names a slot as page * 16 + slot and adds up to two steps of 128 keys to a position, in 32 bits."""
    for create in (ap.kv_pool_create, ap.kv_pool_create_4bit):
        with pytest.raises(ap.ApError) as e:
            create((1 << 27) + 1, 1, 64, device=-1)
        assert e.value.status == B.AP_ERR_UNSUPPORTED
        pool = create(16, 1, 64, device=-1)
        table = np.zeros((1, 1 << 27), np.int32)                             # (never touched: no memory of its own)
        for q_len, window in ((1, None), (2, None), (1, 100), (300, 100)):
            for ctx in (2 ** 31 - 1, 2 ** 31 - 255):
                with pytest.raises(ap.ApError) as e:
                    if window is None:
                        ap.plan_create(pool, [q_len], [ctx], table, 1)
                    else:
                        ap.plan_create_windowed(pool, [q_len], [ctx], table, 1, window)
                assert e.value.status == B.AP_ERR_UNSUPPORTED
        # the longest one, of a window that shows only its end
        far = 2 ** 31 - 256
        plan = ap.plan_create_windowed(pool, [1], [far], table, 1, 40)
        assert ap.plan_export(plan)["append_dst"].tolist() == [(far - 1) % 16]
        ap.plan_destroy(plan)
        # a sequence without new tokens may be described in any way
        ap.plan_destroy(ap.plan_create(pool, [0, 1], [2 ** 31 - 1, 5], np.zeros((2, 1), np.int32), 1))
        ap.kv_pool_destroy(pool)


# ------------------------------------------------------------------- host call --

@pytest.mark.gpu
def test_the_host_call_validates_a_batch_before_it_sizes_its_staging_by_it():
    """On a 4-bit pool the staging grows with the contexts of prefill chunks; a context that the table does not hold is
    INVALID_ARG, whatever memory it would take, and the pool goes on as before."""
    shape = (6, 2, 128)
    b = _batch(shape, 67, [1, 30], [100, 60])
    planes = _planes(b, True)
    dev = R.Device(b, k_plane=planes[0], v_plane=planes[1], four_bit=True)

    def call(q_lens, ctx_lens, table, q=b.q, k=b.k_new, v=b.v_new):
        out, lse = np.zeros((len(q), 6, 128), np.uint16), np.zeros((len(q), 6), np.float32)
        ap.serving_iteration_host(dev.pool, q_lens, ctx_lens, table, 6, q, k, v, out, lse)
        return out, lse
    first = call(b.q_lens, b.ctx_lens, b.block_tables)
    for ctx, status in ((2 ** 31 - 257, B.AP_ERR_INVALID_ARG), (2 ** 31 - 1, B.AP_ERR_UNSUPPORTED), (1 << 24, B.AP_ERR_INVALID_ARG)):
        with pytest.raises(ap.ApError) as e:
            call([1, 30], [100, ctx], b.block_tables)
        assert e.value.status == status, ctx
    again = call(b.q_lens, b.ctx_lens, b.block_tables)
    assert all(np.array_equal(x, y) for x, y in zip(first, again))
    k, v = (Q.values(p, 128) for p in planes)
    ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b)
    R.check(*first, ref)
    dev.close()


# ----------------------------------------------------------- out of host memory --

def test_a_page_copy_without_host_memory_returns_a_status():
    """In a child process whose address space may not grow: the list of destinations does not fit, and the call says so instead
    of ending the process with an exception at a C entry."""
    import os
    import subprocess
    import sys
    child = """
import ctypes, resource
import numpy as np
from paper_2604_07144_b200 import binding as B
lib = B.load()
desc = B.PoolDesc(1 << 26, 16, 1, 64, None, None, -1)
pool = ctypes.c_void_p()
assert lib.ap_kv_pool_create_4bit(ctypes.byref(pool), ctypes.byref(desc)) == 0
ids = np.arange(4, dtype=np.int32)
assert lib.ap_kv_copy_pages(pool, pool, 2, ids.ctypes.data, ids[2:].ctypes.data, None) == 0
size = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (size + (8 << 20), resource.RLIM_INFINITY))
print("status", lib.ap_kv_copy_pages(pool, pool, 2, ids.ctypes.data, ids[2:].ctypes.data, None))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", child], cwd=root, capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and done.stdout.split() == ["status", str(B.AP_ERR_CUDA)], done.stdout + done.stderr


# ------------------------------------------------------------- more of the forms --

def test_struct_sizes_of_the_operators_match_the_header(tmp_path):
    import ctypes
    import os
    import subprocess
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    fields = ("rotary_dim", "interleaved", "base", "inv_freq", "amplitude", "q_row_stride", "k_row_stride", "v_row_stride")
    src.write_text('#include "ap_serving.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {\n'
                   '  printf("%zu %zu", sizeof(ap_rope_desc), sizeof(ap_window_desc));\n'
                   + "".join(f'  printf(" %zu", offsetof(ap_rope_desc, {f}));\n' for f in fields)
                   + '  printf(" %zu", offsetof(ap_window_desc, sinks));\n  return 0;\n}\n')
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", inc, str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [ctypes.sizeof(B.RopeDesc), ctypes.sizeof(B.WindowDesc), *(getattr(B.RopeDesc, f).offset for f in fields),
                   B.WindowDesc.sinks.offset]
    # the packed form that the binding passes
    packed = B._ROPE_DESC.pack(64, 1, 2.5, 4096, 0.5, 8, 16, 24)
    desc = B.RopeDesc.from_buffer_copy(packed)
    assert len(packed) == got[0] and tuple(getattr(desc, f) for f in fields) == (64, 1, 2.5, 4096, 0.5, 8, 16, 24)


def test_amplitudes_and_bases_that_are_no_numbers_are_refused():
    import torch
    pool, plan = _host_plan()
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for kw in (dict(amplitude=float("inf")), dict(amplitude=float("nan")), dict(amplitude=1e39), dict(amplitude=-1e300), dict(base=float("inf")),
               dict(base=-2), dict(base=0)):
        with pytest.raises(ap.ApError) as e:
            ap.kv_append_rope(pool, plan, k, k, **kw)
        assert e.value.status == B.AP_ERR_INVALID_ARG, kw
    for kw in (dict(amplitude=np.float32(1.5), base=10000), dict(amplitude=-2, base=np.float64(7), rotary_dim=np.int64(32), interleaved=np.bool_(True))):
        with pytest.raises(ap.ApError) as e:
            ap.kv_append_rope(pool, plan, k, k, **kw)
        assert e.value.status == B.AP_ERR_CUDA, kw
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 2, 64), (6, 2, 128), (40, 40, 64)], ids=str)
def test_rotated_append_to_a_4bit_pool_in_place_without_q_and_with_given_frequencies(shape):
    """q in place, q left out, given frequencies and an amplitude: what the pool stores is the quantised form of what a bf16 pool
    stores, and q is rotated alike."""
    b = _batch(shape, 68, [1, 20, 1], [77, 300, 5000])
    page, slot = Q.new_slots(b)
    freq = np.array([0.9 ** i / (1 + i % 3) for i in range(shape[2] // 2)])
    for kw in (dict(inv_freq=freq), dict(inv_freq=freq[:16], rotary_dim=32, interleaved=True, amplitude=1.25), dict(base=2.0)):
        for with_q in (True, False):
            rows, q_out = [], []
            for four_bit in (False, True):
                planes = [Q.empty_plane(b.num_pages, shape[1], shape[2], s) for s in (1, 2)] if four_bit else (None, None)
                dev = R.Device(b, k_plane=planes[0], v_plane=planes[1], four_bit=four_bit)
                ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, **(dict(q=dev.q, q_rot=dev.q) if with_q else {}), **kw)
                assert ap.last_device_status(dev.pool) == 0
                q_out.append(to_bits(dev.q))
                if four_bit:
                    for plane, r, got in zip(planes, rows, (dev.k_pool, dev.v_pool)):
                        Q.put(plane, page, slot, r)
                        assert np.array_equal(got.cpu().numpy(), plane)
                else:
                    rows = [to_bits(p)[page, :, slot] for p in (dev.k_pool, dev.v_pool)]
                dev.close()
            assert np.array_equal(*q_out) and np.array_equal(q_out[0], b.q) == (not with_q)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(None, 0), (3000, 20), (700, 1000)])
def test_4bit_prefill_of_long_contexts(window, sinks):
    """Chunks on prefixes of thousands of tokens, alone and beside decode rows, with sinks that reach past a block's window."""
    for shape in ((8, 2, 64), (5, 1, 128)):
        b = _batch(shape, 69, [300, 2, 1, 130], [9000, 5001, 7000, 2500])
        out, lse, k, v = _attend(b, _planes(b, True), True, window, sinks)
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b, window, sinks)
        R.check(out, lse, ref, f"window {window}")
