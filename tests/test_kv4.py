"""4-bit pools: quantising append, read-back, page copy, and attention against a plain 64-bit implementation over
the values the planes stand for.  Slots without a token hold arbitrary codes and NaN steps."""
import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import kv4_reference as Q
import operator_reference as R
from harness import to_bits, to_dev
from test_windowed_attention import _hide as hide

SHAPES = [(8, 2, 64), (6, 2, 128), (5, 1, 128), (8, 8, 64), (32, 8, 128), (64, 8, 128), (3, 3, 128)]


def _batch(shape, seed, q_lens, ctx_lens, with_pool=True):
    return W._assemble(f"kv4_{seed}", shape, W.make_rng(seed), np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32),
                       1.3, with_pool=with_pool)


# ------------------------------------------------------------------ CPU --

def test_reference_format_round_trip_and_error_bound():
    rng = np.random.default_rng(0)
    for d in (64, 128):
        codes = rng.integers(0, 16, (5, 3, d), dtype=np.uint8)
        assert np.array_equal(Q.unpack(Q.pack(codes)), codes)
        x = W.f32_to_bf16_bits((rng.standard_normal((40, 2, d)) * 2.0 ** rng.integers(-30, 30, (40, 2, 1))).astype(np.float32))
        codes, steps = Q.quantise(x)
        s = np.repeat(W.bf16_bits_to_f64(steps), 32, -1)
        v = (codes.astype(float) - 8) * s
        assert codes.min() >= 1 and codes.max() <= 15
        assert (np.abs(v - W.bf16_bits_to_f64(x)) <= s / 2).all()
        assert np.array_equal(W.bf16_bits_to_f64(W.f32_to_bf16_bits(v)), v)      # a bf16 number
        assert (np.ceil(np.abs(W.bf16_bits_to_f64(x)).reshape(40, 2, -1, 32).max(-1) / 7 / (s[..., ::32] * 17 / 16)) <= 1).all()


def test_quantiser_without_divisions_is_exact():
    """The append forms the step from a product with (1 - 2^-16) / 7 and rint(x / s) from one with an approximate 1 / s (see
    kv4.cuh).  Every 8-bit x, every 5-bit s and every scale between them, in fp32 as the kernel does it, against
    exact fractions; 1 / s with up to two ulps of error either way."""
    from fractions import Fraction
    f = np.float32
    # steps: five significant bits at or above m / 7
    m = np.arange(128, 256).astype(f)
    t = m * f(0.14285496)
    step = ((t.view(np.uint32) + np.uint32(0x7FFFF)) & ~np.uint32(0x7FFFF)).view(f)
    for mi, si in zip(m, step):
        grid = [Fraction(S) * Fraction(2) ** e for e in range(-3, 3) for S in range(16, 32)]
        assert Fraction(float(si)) == min(g for g in grid if g >= Fraction(int(mi), 7))
    # codes
    for S in range(16, 32):
        exact = f(1) / f(S)
        for inv in (exact, *(np.nextafter(exact, f(d), dtype=f) for d in (0, 1)),
                    *(np.nextafter(np.nextafter(exact, f(d), dtype=f), f(d), dtype=f) for d in (0, 1))):
            for n in range(-12, 4):
                x = (np.arange(128, 256) * 2.0 ** n).astype(f)
                x = x[x <= 7 * S]
                want = [round(Fraction(float(v)) / S) for v in x]                 # Python rounds ties to even
                for sign in (1, -1):
                    y = (sign * x.astype(np.float64) * np.float64(inv) + 1536.0).astype(f)       # one rounding: an FMA
                    code = (y + f(12581384)).view(np.uint32) & 15
                    assert code.tolist() == [8 + sign * w for w in want]


def test_4bit_pool_descriptions_and_refusals():
    assert ap.kv_pool_bytes_4bit(10, 8, 128) == 10 * 8 * 1152 and ap.kv_pool_bytes_4bit(10, 2, 64) == 10 * 2 * 576
    assert ap.kv_pool_bytes_4bit(0, 8, 128) == 0 and ap.kv_pool_bytes_4bit(4, 2, 96) == 0
    for kw, status in ((dict(num_pages=0, num_kv_heads=2, head_dim=64), B.AP_ERR_INVALID_ARG),
                       (dict(num_pages=4, num_kv_heads=2, head_dim=96), B.AP_ERR_UNSUPPORTED),
                       (dict(num_pages=4, num_kv_heads=2, head_dim=64, page_size=32), B.AP_ERR_UNSUPPORTED)):
        with pytest.raises(ap.ApError) as e:
            ap.kv_pool_create_4bit(device=-1, **kw)
        assert e.value.status == status
    pool, plain = ap.kv_pool_create_4bit(64, 2, 64, device=-1), ap.kv_pool_create(64, 2, 64, device=-1)
    with pytest.raises(ap.ApError) as e:                       # pages do not move between formats
        ap.kv_copy_pages(pool, plain, [0], [0])
    assert e.value.status == B.AP_ERR_INVALID_ARG
    ap.kv_copy_pages(pool, pool, [3], [0])
    bt = np.arange(40, dtype=np.int32)[None]
    plan = ap.plan_create(pool, [1], [600], bt, 8)
    for call in (ap.kv_append, ap.kv_read_new):
        with pytest.raises(ap.ApError) as e:
            call(pool, plan, 0, 0)
        assert e.value.status == B.AP_ERR_CUDA                 # a host-only pool launches nothing
        with pytest.raises(ap.ApError) as e:
            call(plain, plan, 0, 0)
        assert e.value.status == B.AP_ERR_INVALID_ARG          # another pool's plan
    ap.plan_destroy(plan)
    for p in (pool, plain):
        ap.kv_pool_destroy(p)


def test_4bit_plan_lists():
    """Decode items cover every (row, kv head block, page) once, on a list per two warps' SM share; prefill units read numbered
    copies of the pages, whose list names the right pages; workspace and work figures follow."""
    b = _batch((32, 8, 128), 3, [1, 300, 1, 0, 5, 1], [700, 1000, 9000, 20, 40, 17], with_pool=False)
    for window, sinks in ((None, 0), (200, 20), (64, 0)):
        pool = ap.kv_pool_create_4bit(b.num_pages, 8, 128, device=-1)
        ap.kv_pool_set_side_by_side(pool, 40)                  # no difference to the default on a 4-bit pool
        plan = (ap.plan_create(pool, b.q_lens, b.ctx_lens, b.block_tables, 32) if window is None else
                ap.plan_create_windowed(pool, b.q_lens, b.ctx_lens, b.block_tables, 32, window, sinks))
        ex, rows = ap.plan_export(plan), b.q_indptr
        info = ex["info"]
        assert info["side_by_side"] == 0 and info["decode_head_block"] == 8 and info["launches_attention"] == (4 if info["merge_entries"] else 3)
        assert info["decode_ctas"] <= 296
        for s in (0, 2, 5):
            for head in (0,):
                its = ex["decode_items"][(ex["decode_items"][:, 0] == rows[s]) & (ex["decode_items"][:, 1] == head)]
                covered = sorted(p for it in its.tolist() for p in range(it[3], it[3] + it[4]))
                assert covered == list(range((its[0][5] + 15) // 16))
                got = ex["bt_flat"][its[0][2]:its[0][2] + len(covered)]
                see = R.visible(1, int(b.ctx_lens[s]), window, sinks).any(0)
                want = [p for i, p in enumerate(b.block_tables[s, :len(see) // 16 + 1]) if see[16 * i:16 * i + 16].any()]
                assert list(got) == want
        # every unit's entries number copies; a copy's number says which visible page of which sequence it is
        numbers, base = {}, 0
        for s in (1, 4):
            see = R.visible(int(b.q_lens[s]), int(b.ctx_lens[s]), window, sinks)
            kept = [i for i in range((see.shape[1] + 15) // 16) if see[:, 16 * i:16 * i + 16].any()]
            numbers[s] = {lp: base + i for i, lp in enumerate(kept)}
            base += len(kept)
        for r0, nr, qh, _, off, pos0, vctx, _ in ex["prefill_tiles"].tolist():
            s = 1 if r0 < rows[2] else 4
            see = R.visible(int(b.q_lens[s]), int(b.ctx_lens[s]), window, sinks)[r0 - rows[s]:r0 - rows[s] + nr]
            if window is None:
                want = [numbers[s][i] for i in range((int(b.ctx_lens[s]) + 15) // 16)]
            else:
                want = [numbers[s][i] for i in range((see.shape[1] + 15) // 16) if see[:, 16 * i:16 * i + 16].any()]
            assert list(ex["bt_flat"][off:off + len(want)]) == want
        wide = 2 * base * 8 * 16 * 128 * 2
        parts = ap.plan_workspace_bytes(plan) - wide
        slots = int((ex["decode_items"][:, 6] >= 0).sum())
        assert 0 <= parts - slots * 8 * 4 * 129 * 4 < 512
        if window is None:
            pred = ap.plan_predict(plan)
            per_token = 2 * 8 * 72
            assert pred["decode_bytes"] == 9717 * per_token + 3 * (2 * 32 * 128 * 2 + 32 * 4) + (44 + 563 + 2) * 4
            assert pred["append_bytes"] == 308 * (2 * 8 * 256 + per_token)
        ap.plan_destroy(plan)
        ap.kv_pool_destroy(pool)


# ------------------------------------------------------------------ GPU --

def _check_attention(batch, window=None, sinks=0, append=True, planes=None):
    if window is not None:
        hide(batch, window, sinks)       # table entries of unseen pages -1, unseen tokens of the others NaN
    kp, vp = planes or Q.planes_of(batch)
    make = None if window is None else (lambda pool: ap.plan_create_windowed(
        pool, batch.q_lens, batch.ctx_lens, batch.block_tables, batch.num_q_heads, window, sinks))
    dev = R.Device(batch, make, k_plane=kp, v_plane=vp, four_bit=True)
    try:
        if append:
            ap.kv_append(dev.pool, dev.plan, dev.k_new, dev.v_new)
            page, slot = Q.new_slots(batch)
            Q.put(kp, page, slot, batch.k_new)
            Q.put(vp, page, slot, batch.v_new)
        dev.attend()
        out, lse = dev.results()
        assert np.array_equal(dev.k_pool.cpu().numpy(), kp) and np.array_equal(dev.v_pool.cpu().numpy(), vp)
        k, v = (Q.values(p, batch.head_dim) for p in (kp, vp))
        ref = R.attention(lambda s: R.table_rows(batch, k, s), lambda s: R.table_rows(batch, v, s), batch, window, sinks)
        R.check(out, lse, ref, batch.name)
        return dev.info
    finally:
        dev.close()


def _awkward_rows(n, hkv, d, seed):
    """bf16 rows with groups of every kind: zero, one value, powers of two, ties, tiny, huge, inf, NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, hkv, d)).astype(np.float32)
    x[0::9] = 0.0
    x[1::9, :, :32] = 3.5
    x[2::9] *= np.float32(2.0 ** -125)
    x[3::9] *= np.float32(2.0 ** 100)
    x[4::9] = rng.integers(-7, 8, x[4::9].shape) * np.float32(0.5)             # multiples and halves of a step
    bits = W.f32_to_bf16_bits(x)
    bits[5::9, :, 7] = 0x7F80                                                # inf
    bits[6::9, 0, d - 1] = 0xFFC1                                            # NaN in one group
    bits[7::9, :, 40] = 0x7BC0                                               # not below 2^120
    bits[8::9, :, :] = rng.integers(0, 128, bits[8::9].shape)                 # bf16 denormals
    return bits


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_quantising_append_and_read_back_bit_for_bit(shape):
    b = _batch(shape, 21, [1, 1, 0, 37, 1, 16, 3], [1, 16, 9, 50, 300, 16, 35], with_pool=False)
    n, hkv, d = b.n_new, b.num_kv_heads, b.head_dim
    for k, v in ((b.k_new, b.v_new), (_awkward_rows(n, hkv, d, 1), _awkward_rows(n, hkv, d, 2))):
        kp, vp = (Q.empty_plane(b.num_pages, hkv, d, s) for s in (1, 2))
        dev = R.Device(b, k_plane=kp, v_plane=vp, four_bit=True)
        ap.kv_append(dev.pool, dev.plan, to_dev(k), to_dev(v))
        k_back, v_back = (to_dev(np.full((n + 1, hkv, d), 0x1234, np.uint16)) for _ in range(2))
        ap.kv_read_new(dev.pool, dev.plan, k_back, v_back)
        assert ap.last_device_status(dev.pool) == 0
        page, slot = Q.new_slots(b)
        Q.put(kp, page, slot, k)
        Q.put(vp, page, slot, v)
        assert np.array_equal(dev.k_pool.cpu().numpy(), kp) and np.array_equal(dev.v_pool.cpu().numpy(), vp)
        for back, plane in ((k_back, kp), (v_back, vp)):
            want, got = Q.values(plane, d)[page, :, slot], W.bf16_bits_to_f64(to_bits(back))
            assert np.array_equal(got[:n], want, equal_nan=True) and (to_bits(back)[n] == 0x1234).all()
        dev.close()


@pytest.mark.gpu
def test_read_back_of_a_bf16_pool():
    b = _batch((8, 2, 64), 22, [1, 40, 1], [5, 100, 300])
    dev = R.Device(b)
    ap.kv_append(dev.pool, dev.plan, dev.k_new, dev.v_new)
    import torch
    k, v = torch.zeros_like(dev.k_new), torch.zeros_like(dev.v_new)
    ap.kv_read_new(dev.pool, dev.plan, k, v)
    assert ap.last_device_status(dev.pool) == 0
    assert np.array_equal(to_bits(k), b.k_new) and np.array_equal(to_bits(v), b.v_new)
    with pytest.raises(ap.ApError) as e:
        ap.kv_read_new(dev.pool, dev.plan, k.data_ptr() + 2, v)
    assert e.value.status == B.AP_ERR_INVALID_ARG
    dev.close()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_4bit_decode(shape):
    _check_attention(_batch(shape, 23, [1] * 14 + [0], [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 129, 700, 1000, 5]))


@pytest.mark.gpu
def test_4bit_decode_long_contexts_are_cut_and_merged():
    info = _check_attention(_batch((32, 8, 128), 24, [1, 1, 1], [20000, 9001, 333]))
    assert info["merge_entries"] > 0 and info["decode_ctas"] > 148
    info = _check_attention(_batch((8, 2, 64), 25, [1], [30011]))
    assert info["merge_entries"] > 0
    # many short rows: more items than a block keeps descriptions of
    info = _check_attention(_batch((5, 1, 128), 26, [1] * 2000, np.random.default_rng(1).integers(1, 40, 2000)))
    assert info["decode_items"] >= 2000


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (16, 16), (33, 17), (100, 4), (500, 20), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
def test_4bit_windowed(window, sinks):
    for shape in ((6, 2, 128), (8, 4, 64)):
        b = _batch(shape, 27, [1] * 9 + [2, 5, 129, 300], [1, 15, 17, 33, 64, 129, 700, 1300, 9001, 2, 600, 133, 1024])
        _check_attention(b, window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 2, 64), (6, 2, 128), (5, 1, 128), (32, 8, 128)], ids=str)
def test_4bit_prefill_and_mixed(shape):
    _check_attention(_batch(shape, 28, [2, 16, 100, 129, 300], [2, 16, 600, 129, 1000]))
    _check_attention(_batch(shape, 29, [150, 1, 1, 1, 40, 0], [400, 90, 1300, 17, 1000, 3]))


@pytest.mark.gpu
def test_4bit_values_of_every_size():
    """Steps from 2^-130 to 2^100 in one cache: values that differ by orders of magnitude do not disturb one another."""
    b = _batch((8, 2, 64), 30, [1, 1, 20], [200, 37, 64])
    rng = np.random.default_rng(3)
    scale = 2.0 ** rng.integers(-125, -20, (b.num_pages, 1, 16, 1))
    for name in ("k_pool", "v_pool"):
        pool = getattr(b, name)
        held = pool != W.CANARY
        setattr(b, name, np.where(held, W.f32_to_bf16_bits((W.bf16_bits_to_f64(pool) * scale).astype(np.float32)), W.CANARY))
    _check_attention(b)


@pytest.mark.gpu
def test_4bit_page_offsets_past_32_bits():
    """Planes of 5 GB: the pages in use lie at both ends."""
    import torch
    b = _batch((32, 8, 128), 31, [1, 1, 30], [700, 33, 200])
    pages = (5 << 30) // (8 * 1152)
    small = [Q.planes_of(b)][0]
    page, slot = Q.new_slots(b)
    where = np.concatenate([np.arange(b.num_pages // 2), pages - 1 - np.arange(b.num_pages - b.num_pages // 2)]).astype(np.int32)
    k, v = (torch.zeros((pages, 8, 1152), dtype=torch.uint8, device="cuda:0") for _ in range(2))
    at = torch.from_numpy(where.astype(np.int64)).cuda()
    for big, plane in ((k, small[0]), (v, small[1])):
        big[at] = torch.from_numpy(plane).cuda()
    pool = ap.kv_pool_create_4bit(pages, 8, 128, k, v)
    plan = ap.plan_create(pool, b.q_lens, b.ctx_lens, np.where(b.block_tables >= 0, where[b.block_tables], -1), 32)
    ws = torch.empty(max(256, ap.plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda:0")
    out = torch.empty((b.n_new, 32, 128), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.empty((b.n_new, 32), device="cuda:0")
    ap.kv_append(pool, plan, to_dev(b.k_new), to_dev(b.v_new))
    ap.attention_iteration(pool, plan, to_dev(b.q), out, lse, ws)
    assert ap.last_device_status(pool) == 0
    for plane, new in zip(small, (b.k_new, b.v_new)):
        Q.put(plane, page, slot, new)
    assert np.array_equal(k[at].cpu().numpy(), small[0]) and np.array_equal(v[at].cpu().numpy(), small[1])
    kv, vv = (Q.values(p, 128) for p in small)
    R.check(to_bits(out), lse.cpu().numpy(), R.attention(lambda s: R.table_rows(b, kv, s), lambda s: R.table_rows(b, vv, s), b))
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
def test_4bit_page_copy():
    b = _batch((6, 2, 128), 32, [1, 20], [300, 100])
    kp, vp = Q.planes_of(b)
    dev = R.Device(b, k_plane=kp, v_plane=vp, four_bit=True)
    import torch
    k2, v2 = (torch.from_numpy(Q.empty_plane(40, 2, 128, 9 + i)).cuda() for i in range(2))
    before = k2.cpu().numpy().copy()
    other = ap.kv_pool_create_4bit(40, 2, 128, k2, v2)
    ap.kv_copy_pages(other, dev.pool, [39, 0, 7], [1, 5, 5])
    assert ap.last_device_status(other) == 0
    before[[39, 0, 7]] = kp[[1, 5, 5]]
    assert np.array_equal(k2.cpu().numpy(), before) and np.array_equal(v2.cpu().numpy()[[39, 0, 7]], vp[[1, 5, 5]])
    ap.kv_pool_destroy(other)
    dev.close()


@pytest.mark.gpu
def test_4bit_library_planes_host_call_and_static_workspace():
    """Planes owned by the library start as zeros; the host-buffer call and the no-allocation call take a 4-bit pool."""
    rng = W.make_rng(33)
    hq, hkv, d, chunk = 6, 2, 128, 70
    pool = ap.kv_pool_create_4bit(32, hkv, d)
    table = np.arange(32, dtype=np.int32).reshape(2, 16)[:, ::-1].copy()
    b1 = W.Batch("a", hq, hkv, d, 32, np.array([chunk, 130], np.int32), np.array([chunk, 130], np.int32), table,
                 *(rng.normal_bf16((chunk + 130, h, d)) for h in (hq, hkv, hkv)))
    b2 = W.Batch("b", hq, hkv, d, 32, np.array([1, 1], np.int32), np.array([chunk + 1, 131], np.int32), table,
                 *(rng.normal_bf16((2, h, d)) for h in (hq, hkv, hkv)))
    kp, vp = (np.zeros((32, hkv, Q.tile_bytes(d)), np.uint8) for _ in range(2))
    for b in (b1, b2):
        out, lse = np.zeros((b.n_new, hq, d), np.uint16), np.zeros((b.n_new, hq), np.float32)
        ap.serving_iteration_host(pool, b.q_lens, b.ctx_lens, b.block_tables, hq, b.q, b.k_new, b.v_new, out, lse)
        page, slot = Q.new_slots(b)
        Q.put(kp, page, slot, b.k_new)
        Q.put(vp, page, slot, b.v_new)
        k, v = (Q.values(p, d) for p in (kp, vp))
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b)
        R.check(out, lse, ref, "host call")
    import torch
    plan = ap.plan_create(pool, b2.q_lens, b2.ctx_lens, table, hq)
    o = torch.full((2, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    l = torch.full((2, hq), float("nan"), device="cuda:0")
    ap.attention_iteration_static(pool, plan, to_dev(b2.q), o, l)
    assert ap.last_device_status(pool) == 0
    R.check(to_bits(o), l.cpu().numpy(), ref, "static")
    ap.plan_destroy(plan)
    # pages of a long prefill chunk do not fit into the static array: refused, nothing launched
    big = ap.kv_pool_create_4bit(600, hkv, d)
    plan = ap.plan_create(big, [2], [9600], np.arange(600, dtype=np.int32)[None], hq)
    assert ap.plan_workspace_bytes(plan) > ap.static_workspace_bytes()
    with pytest.raises(ap.ApError) as e:
        ap.attention_iteration_static(big, plan, o, o, l)
    assert e.value.status == B.AP_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(ap.ApError) as e:
        ap.attention_iteration(big, plan, o, o, l, torch.empty(4096, dtype=torch.uint8, device="cuda:0"))
    assert e.value.status == B.AP_ERR_WORKSPACE_TOO_SMALL
    ap.plan_destroy(plan)
    for p in (big, pool):
        ap.kv_pool_destroy(p)


@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
def test_without_lse_and_with_one_workspace_for_all_layers(four_bit):
    """lse may be NULL; a workspace that is large enough serves plans of different layers in turn (what it holds before
    a call does not matter), and pools on two streams do not disturb one another."""
    import torch
    shape, n = (6, 2, 128), 4
    batches = [_batch(shape, 50 + i, [1, 1, 60, 1], [700 + 100 * i, 33, 300, 5000]) for i in range(n)]
    devs = []
    for i, b in enumerate(batches):
        make = None if i % 2 else (lambda pool, b=b: ap.plan_create_windowed(pool, b.q_lens, b.ctx_lens, b.block_tables, 6, 100, 4))
        planes = Q.planes_of(b) if four_bit else (None, None)
        devs.append(R.Device(b, make, k_plane=planes[0], v_plane=planes[1], four_bit=four_bit))
    size = max(256, *(d.workspace_bytes for d in devs))
    ws = [torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for d in devs:
        ap.kv_append(d.pool, d.plan, d.k_new, d.v_new)
    torch.cuda.synchronize()
    for _ in range(3):
        for i, d in enumerate(devs):
            with torch.cuda.stream(streams[i // 2]):
                d.out.fill_(float("nan"))
                ap.attention_iteration(d.pool, d.plan, d.q, d.out, None, ws[i // 2], size)
    torch.cuda.synchronize()
    for i, (b, d) in enumerate(zip(batches, devs)):
        assert ap.last_device_status(d.pool) == 0 and np.isnan(d.lse.cpu().numpy()).all()
        k, v = ((Q.values(p.cpu().numpy(), 128) if four_bit else W.bf16_bits_to_f64(to_bits(p))) for p in (d.k_pool, d.v_pool))
        window, sinks = (None, 0) if i % 2 else (100, 4)
        ref = R.attention(lambda s: R.table_rows(b, k, s), lambda s: R.table_rows(b, v, s), b, window, sinks)
        R.check(to_bits(d.out)[:b.n_new], ref[1], ref, f"layer {i}")
        d.close()


@pytest.mark.gpu
@pytest.mark.parametrize("window", [None, 40])
def test_4bit_mixed_dispatches_agree_and_replay(window):
    """Prefill on the second stream behind decode, or on the caller's: the same lists, so the same bits; eager from a stream of the
    caller's, and captured.  The out rows are poisoned and read right behind the call, which has to cover both parts."""
    import torch
    b = _batch((16, 4, 128), 41, [1, 130, 1, 1, 64, 1] + [1] * 20, [700, 600, 33, 5000, 64, 1] + [90 + 41 * i for i in range(20)])
    make = (lambda p: ap.plan_create(p, b.q_lens, b.ctx_lens, b.block_tables, 16)) if window is None else (
        lambda p: ap.plan_create_windowed(p, b.q_lens, b.ctx_lens, b.block_tables, 16, window, 3))
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    rows = torch.randn((int(b.ctx_lens.sum()), 4, 128), generator=gen, device="cuda:0").to(torch.bfloat16)
    q = torch.randn((b.n_new, 16, 128), generator=gen, device="cuda:0").to(torch.bfloat16)
    results = []
    for mode in (0, 1):
        pool = ap.kv_pool_create_4bit(b.num_pages, 4, 128)
        ap.kv_pool_set_side_by_side(pool, mode)
        fill = ap.plan_create(pool, b.ctx_lens, b.ctx_lens, b.block_tables, 16)
        ap.kv_append(pool, fill, rows, -rows)
        plan = make(pool)
        info = ap.plan_get_info(plan)
        assert info["side_by_side"] == 0 and info["decode_rows"] == 24 and info["prefill_tiles"] > 0
        ws = torch.empty(max(256, ap.plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda:0")
        out, lse = torch.empty_like(q), torch.empty((b.n_new, 16), device="cuda:0")
        seen = [torch.empty_like(out), torch.empty_like(lse)]
        st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()

        def step():
            ws.fill_(0xFF)
            out.fill_(float("nan"))
            lse.fill_(float("nan"))
            ap.attention_iteration(pool, plan, q, out, lse, ws)
            seen[0].copy_(out)
            seen[1].copy_(lse)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            step()
        st.synchronize()
        results.append([x.clone() for x in seen])
        with torch.cuda.graph(g, stream=st):
            step()
        for _ in range(10):
            seen[0].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert ap.last_device_status(pool) == 0 and torch.equal(seen[0], results[-1][0]) and torch.equal(seen[1], results[-1][1])
        del g
        for p in (plan, fill):
            ap.plan_destroy(p)
        ap.kv_pool_destroy(pool)
    assert torch.isfinite(results[0][0].float()).all() and torch.isfinite(results[0][1]).all()
    assert all(torch.equal(x, y) for x, y in zip(*results))
