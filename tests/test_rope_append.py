"""Append with the rotary embedding against the definition in 64 bits, and whole layers made of the operators that
belong together: rotated append, windowed attention, 4-bit cache."""
import math

import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import kv4_reference as Q
import operator_reference as R
from harness import to_bits, to_dev

ROTATIONS = [dict(rotary_dim=64), dict(rotary_dim=64, interleaved=True, base=500000.0), dict(rotary_dim=16, base=1e6),
             dict(rotary_dim=48, interleaved=True), dict(rotary_dim=32, amplitude=1.25)]


def _batch(shape, seed, q_lens, ctx_lens, with_pool=True):
    return W._assemble(f"rope_{seed}", shape, W.make_rng(seed), np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32),
                       1.3, with_pool=with_pool)


def positions(batch):
    return np.concatenate([np.arange(int(c) - int(n), int(c)) for n, c in zip(batch.q_lens, batch.ctx_lens)])


def rotated(bits, pos, rotary_dim, base=10000.0, interleaved=False, inv_freq=None, amplitude=1.0):
    """(float64 result, bound of the error before the rounding to bf16) for bf16 rows [n, heads, d]."""
    x = W.bf16_bits_to_f64(bits)
    h = rotary_dim // 2
    f = np.array([base ** (-2.0 * i / rotary_dim) for i in range(h)]) if inv_freq is None else np.asarray(inv_freq)
    # p f exactly enough: whole turns taken off in long double
    turns = np.asarray(pos, np.longdouble)[:, None] * (np.asarray(f, np.longdouble) / (2 * np.longdouble(math.pi) + np.longdouble(1.2246467991473532e-16) * 2))
    ang = np.asarray((turns - np.rint(turns)) * 2 * np.longdouble(math.pi), np.float64)[:, None]
    c, s = amplitude * np.cos(ang), amplitude * np.sin(ang)
    y, slack = x.copy(), np.zeros_like(x)
    ia, ib = (np.arange(0, rotary_dim, 2), np.arange(1, rotary_dim, 2)) if interleaved else (np.arange(h), np.arange(h, rotary_dim))
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    # fp32: two products and a sum (2^-24 each), cosine and sine to 2 ulp, an angle to 2^-24 turns of pi
    slack[..., ia] = slack[..., ib] = (np.abs(a) + np.abs(b)) * amplitude * 1e-6
    return y, slack


def check_rows(got_bits, ref, slack, what):
    got = W.bf16_bits_to_f64(got_bits)
    a = np.abs(ref)
    half_ulp = np.where(a > 0, 2.0 ** (np.floor(np.log2(np.maximum(a, 1e-300))) - 8), 0.0)
    excess = np.abs(got - ref) - (half_ulp + slack)
    i = np.unravel_index(np.argmax(excess), excess.shape)
    assert excess[i] <= 0, f"{what}: {got[i]} against {ref[i]} at {i}"


def fused(batch):
    """q, k, v as slices of one device tensor of projections, and that tensor's bits."""
    rows = np.concatenate([batch.q, batch.k_new, batch.v_new], axis=1)
    t = to_dev(rows)
    hq, hkv = batch.num_q_heads, batch.num_kv_heads
    return t, t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:]


# ------------------------------------------------------------------ CPU --

def test_rope_refusals():
    pool = ap.kv_pool_create(64, 2, 64, device=-1)
    plan = ap.plan_create(pool, [1], [600], np.arange(40, dtype=np.int32)[None], 8)
    import ctypes

    def status(rope=None, pool_=pool, q=None, q_rot=None, **fields):
        d = B.RopeDesc(64, 0, 10000.0, None, 1.0, 0, 0, 0)
        for k, v in fields.items():
            setattr(d, k, v)
        return B.load().ap_kv_append_rope(pool_.handle, plan.handle, ctypes.byref(d) if rope is None else None, q, 4096, 8192,
                                          q_rot, None)
    assert status() == B.AP_ERR_CUDA                                     # valid, but the pool is host-only
    for bad in (dict(rotary_dim=0), dict(rotary_dim=-16), dict(rotary_dim=80), dict(rotary_dim=17), dict(base=0.0), dict(base=-1.0),
                dict(base=float("inf")), dict(base=float("nan")), dict(amplitude=float("nan")), dict(interleaved=2),
                dict(q_row_stride=8 * 64 - 8), dict(k_row_stride=64), dict(v_row_stride=2 * 64 + 4), dict(q=4096), dict(q_rot=4096),
                dict(k_row_stride=-128), dict(q_row_stride=1 << 40), dict(v_row_stride=2 ** 63 - 8)):
        assert status(**bad) == B.AP_ERR_INVALID_ARG, bad
    assert status(rope=0) == B.AP_ERR_INVALID_ARG
    assert status(rotary_dim=24) == B.AP_ERR_UNSUPPORTED
    freq = np.array([1.0] * 31 + [np.inf])
    assert status(inv_freq=freq.ctypes.data) == B.AP_ERR_INVALID_ARG
    assert status(inv_freq=freq.ctypes.data, rotary_dim=32, base=0.0) == B.AP_ERR_CUDA       # base is not looked at
    with pytest.raises(ValueError):
        ap.kv_append_rope(pool, plan, 0, 0, inv_freq=np.ones(3))
    for far in (2 ** 32 + 64, -2 ** 32 + 64):                            # would wrap to 64
        with pytest.raises(ap.ApError) as e:
            ap.kv_append_rope(pool, plan, 4096, 8192, rotary_dim=far)
        assert e.value.status == B.AP_ERR_INVALID_ARG
    import torch
    row = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    rows = torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    for bad in (row.expand(4, 2, 64), rows.transpose(0, 1), rows[:, :, ::2], rows[:, ::2]):  # overlapping rows, strided heads
        with pytest.raises(ValueError):
            ap.kv_append_rope(pool, plan, bad, rows)
        with pytest.raises(ValueError):
            ap.kv_append_rope(pool, plan, rows, rows, q=bad, q_rot=rows)
        with pytest.raises(ValueError):
            ap.kv_read_new(pool, plan, rows, bad)
    for strided in (rows[:, :2], rows[::2]):                             # fine as inputs, not as results
        with pytest.raises(ValueError):
            ap.kv_append_rope(pool, plan, rows, rows, q=rows, q_rot=strided)
        with pytest.raises(ValueError):
            ap.kv_read_new(pool, plan, strided, rows)
    other = ap.kv_pool_create(64, 2, 64, device=-1)
    assert status(pool_=other) == B.AP_ERR_INVALID_ARG
    ap.plan_destroy(plan)
    for p in (pool, other):
        ap.kv_pool_destroy(p)


def test_reference_rotation_keeps_norms_and_relative_positions():
    rng = np.random.default_rng(1)
    x, y = (W.f32_to_bf16_bits(rng.standard_normal((1, 1, 64)).astype(np.float32)) for _ in range(2))
    for kw in ROTATIONS[:4]:
        a, _ = rotated(x, [1000003], **kw)
        assert np.isclose((a ** 2).sum(), (W.bf16_bits_to_f64(x) ** 2).sum(), rtol=1e-12)
        dots = [(rotated(x, [p], **kw)[0] * rotated(y, [p - 7], **kw)[0]).sum() for p in (7, 5000, 900001)]
        assert np.allclose(dots, dots[0], rtol=0, atol=1e-8)


# ------------------------------------------------------------------ GPU --

@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 2, 64), (32, 8, 128), (5, 1, 128), (64, 8, 128), (3, 3, 64), (1, 1, 64)], ids=str)
def test_rotated_append(shape):
    """q, K and V, strided and contiguous, both pairings, partial rotation; every other byte of the pool stays."""
    b = _batch(shape, 41, [1, 1, 0, 37, 1, 16, 1], [1, 2, 9, 50, 300, 16, 4097])
    pos, (page, slot) = positions(b), Q.new_slots(b)
    full = [dict(rotary_dim=shape[2], base=500000.0)] if shape[2] > 64 else []
    for i, kw in enumerate(ROTATIONS + full):
        dev = R.Device(b)
        q_rot = to_dev(np.full((b.n_new + 1,) + b.q.shape[1:], 0x1234, np.uint16))
        if i % 2:
            _, q, k, v = fused(b)
        else:
            q, k, v = dev.q, dev.k_new, dev.v_new
        ap.kv_append_rope(dev.pool, dev.plan, k, v, q=q, q_rot=q_rot, **kw)
        assert ap.last_device_status(dev.pool) == 0
        got_k, got_v = to_bits(dev.k_pool), to_bits(dev.v_pool)
        check_rows(to_bits(q_rot)[:b.n_new], *rotated(b.q, pos, **kw), f"q {kw}")
        assert (to_bits(q_rot)[b.n_new] == 0x1234).all()
        check_rows(got_k[page, :, slot], *rotated(b.k_new, pos, **kw), f"k {kw}")
        want_k, want_v = b.k_pool.copy(), b.v_pool.copy()
        want_k[page, :, slot], want_v[page, :, slot] = got_k[page, :, slot], b.v_new
        assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v)
        dev.close()


@pytest.mark.gpu
def test_rotation_in_place_without_q_and_with_given_frequencies():
    b = _batch((8, 2, 64), 42, [1, 20], [77, 300])
    pos, (page, slot) = positions(b), Q.new_slots(b)
    dev = R.Device(b)
    freq = np.array([0.9 ** i / (1 + i % 3) for i in range(32)])
    ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, q=dev.q, q_rot=dev.q, inv_freq=freq)
    check_rows(to_bits(dev.q), *rotated(b.q, pos, 64, inv_freq=freq), "q in place")
    check_rows(to_bits(dev.k_pool)[page, :, slot], *rotated(b.k_new, pos, 64, inv_freq=freq), "k")
    with_q = to_bits(dev.k_pool)
    ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, inv_freq=freq)
    assert ap.last_device_status(dev.pool) == 0 and np.array_equal(to_bits(dev.k_pool), with_q)
    # position 0 and a zero frequency change nothing
    ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, inv_freq=np.zeros(32))
    assert np.array_equal(to_bits(dev.k_pool)[page, :, slot], b.k_new)
    # overlaps are refused
    _, q, k, v = fused(b)
    for out in (q, k, v):
        with pytest.raises((ap.ApError, ValueError)):
            ap.kv_append_rope(dev.pool, dev.plan, k, v, q=q, q_rot=out)
    with pytest.raises(ap.ApError) as e:
        ap.kv_append_rope(dev.pool, dev.plan, k, v, q=q, q_rot=q.data_ptr())
    assert e.value.status == B.AP_ERR_INVALID_ARG
    with pytest.raises(ap.ApError) as e:
        ap.kv_append_rope(dev.pool, dev.plan, dev.k_new, dev.v_new, q=dev.q, q_rot=dev.q.data_ptr() + 128)
    assert e.value.status == B.AP_ERR_INVALID_ARG
    with pytest.raises(ap.ApError) as e:
        ap.kv_append_rope(dev.pool, dev.plan, dev.k_new.data_ptr() + 2, dev.v_new)
    assert e.value.status == B.AP_ERR_INVALID_ARG
    dev.close()


@pytest.mark.gpu
def test_far_positions():
    """Angles of positions up to 2^27: pages may be shared for reading, so one sequence's table can name few pages."""
    import torch
    ctx = np.array([65536, 1 << 20, (1 << 27) - 3], np.int64)
    table = np.zeros((3, (1 << 27) // 16), np.int32)
    for s in range(3):
        table[s] = 3
        table[s, (ctx[s] - 1) // 16] = s
    k_pool, v_pool = (torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    pool = ap.kv_pool_create(4, 2, 64, k_pool, v_pool)
    plan = ap.plan_create(pool, [1, 1, 1], ctx, table, 8)
    rng = W.make_rng(43)
    q, k, v = (rng.normal_bf16((3, h, 64)) for h in (8, 2, 2))
    q_rot = to_dev(np.zeros_like(q))
    ap.kv_append_rope(pool, plan, to_dev(k), to_dev(v), q=to_dev(q), q_rot=q_rot, base=1e6)
    assert ap.last_device_status(pool) == 0
    check_rows(to_bits(q_rot), *rotated(q, ctx - 1, 64, base=1e6), "q")
    got = to_bits(k_pool)[np.arange(3), :, (ctx - 1) % 16]
    check_rows(got, *rotated(k, ctx - 1, 64, base=1e6), "k")
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 2, 64), (6, 2, 128), (40, 40, 64)], ids=str)
@pytest.mark.parametrize("kw", ROTATIONS[:4], ids=str)
def test_rotated_append_to_a_4bit_pool(shape, kw):
    """What a 4-bit pool stores is the quantised form of exactly the rows a bf16 pool stores."""
    b = _batch(shape, 44, [1, 1, 37, 16], [1, 300, 50, 16])
    page, slot = Q.new_slots(b)
    _, q, k, v = fused(b)
    rows = []
    dev = R.Device(b)
    q1 = to_dev(np.zeros_like(b.q))
    ap.kv_append_rope(dev.pool, dev.plan, k, v, q=q, q_rot=q1, **kw)
    assert ap.last_device_status(dev.pool) == 0
    rows = [to_bits(p)[page, :, slot] for p in (dev.k_pool, dev.v_pool)]
    dev.close()
    planes = [Q.empty_plane(b.num_pages, shape[1], shape[2], s) for s in (1, 2)]
    dev = R.Device(b, k_plane=planes[0], v_plane=planes[1], four_bit=True)
    q4 = to_dev(np.zeros_like(b.q))
    ap.kv_append_rope(dev.pool, dev.plan, k, v, q=q, q_rot=q4, **kw)
    assert ap.last_device_status(dev.pool) == 0
    for plane, r, got in zip(planes, rows, (dev.k_pool, dev.v_pool)):
        Q.put(plane, page, slot, r)
        assert np.array_equal(got.cpu().numpy(), plane)
    assert np.array_equal(to_bits(q4), to_bits(q1))
    dev.close()


@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
def test_layers_of_an_iteration_captured_in_a_graph(four_bit):
    """As a serving loop uses them: two iterations (a prompt, then a mixed one), each with a windowed and a full layer of
    rotated append + attention on pools of their own, captured into one CUDA graph per iteration, both graphs alive
    and replayed in turn with new inputs; against the 64-bit reference of the same layers."""
    import torch
    hq, hkv, d = 6, 2, 128
    window, sinks, base = 40, 4, 10000.0
    rng = W.make_rng(45)
    its = [([70, 33], [70, 33]), ([1, 45], [71, 78])]
    table = np.arange(16, dtype=np.int32).reshape(2, 8)
    make = ap.kv_pool_create_4bit if four_bit else ap.kv_pool_create
    pools = [make(16, hkv, d) for _ in range(2)]
    plans, ws, ins, outs, graphs = [], [], [], [], []
    stream = torch.cuda.Stream()
    for q_lens, ctx in its:
        n = sum(q_lens)
        pl = [ap.plan_create_windowed(pools[0], q_lens, ctx, table, hq, window, sinks), ap.plan_create(pools[1], q_lens, ctx, table, hq)]
        plans.append(pl)
        ws.append([torch.empty(max(256, ap.plan_workspace_bytes(p)), dtype=torch.uint8, device="cuda:0") for p in pl])
        ins.append(torch.zeros((n, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda:0"))
        outs.append([[torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda:0"),
                      torch.zeros((n, hq), device="cuda:0")] for _ in pl])
    torch.cuda.synchronize()

    def layers(i):
        x = ins[i]
        for layer in range(2):
            q_rot, out, lse = outs[i][layer]
            ap.kv_append_rope(pools[layer], plans[i][layer], x[:, hq:hq + hkv], x[:, hq + hkv:], q=x[:, :hq], q_rot=q_rot, base=base)
            ap.attention_iteration(pools[layer], plans[i][layer], q_rot, out, lse, ws[i][layer])

    for i in range(2):
        with torch.cuda.stream(stream):
            layers(i)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            layers(i)
        graphs.append(g)
    for trial in range(2):
        cached = [np.zeros((2, 128, hkv, d)) for _ in range(2)]                # K, V rows by (sequence, position)
        for i, (q_lens, ctx) in enumerate(its):
            n = sum(q_lens)
            bits = rng.normal_bf16((n, hq + 2 * hkv, d))
            with torch.cuda.stream(stream):
                ins[i].copy_(to_dev(bits))
                for layer in outs[i]:
                    for t in layer:
                        t.fill_(float("nan"))
                graphs[i].replay()
            stream.synchronize()
            b = W.Batch("it", hq, hkv, d, 16, np.array(q_lens, np.int32), np.array(ctx, np.int32), table, bits[:, :hq],
                        bits[:, hq:hq + hkv], bits[:, hq + hkv:])
            pos = positions(b)
            k_read, v_read = (torch.zeros((n, hkv, d), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
            for layer in range(2):
                assert ap.last_device_status(pools[layer], stream) == 0
                q_rot, out, lse = outs[i][layer]
                check_rows(to_bits(q_rot), *rotated(b.q, pos, d, base=base), "q")
                ap.kv_read_new(pools[layer], plans[i][layer], k_read, v_read)
                kb, vb = W.bf16_bits_to_f64(to_bits(k_read)), W.bf16_bits_to_f64(to_bits(v_read))
                if four_bit:                         # half a step of the rotated row's groups
                    ref, slack = rotated(b.k_new, pos, d, base=base)
                    step = np.repeat(np.abs(ref).reshape(n, hkv, -1, 32).max(-1) / 7 * (1 + 2.0 ** -4) * (1 + 2.0 ** -7), 32, -1)
                    assert (np.abs(kb - ref) <= step / 2 + np.abs(ref) * 2.0 ** -8 + slack).all()
                else:
                    check_rows(to_bits(k_read), *rotated(b.k_new, pos, d, base=base), "k")
                    assert np.array_equal(to_bits(v_read), b.v_new)
                for s in range(2):
                    rows = slice(int(b.q_indptr[s]), int(b.q_indptr[s + 1]))
                    cached[0][s, ctx[s] - q_lens[s]:ctx[s]], cached[1][s, ctx[s] - q_lens[s]:ctx[s]] = kb[rows], vb[rows]
                b.q = to_bits(q_rot)
                ref = R.attention(lambda s: cached[0][s, :ctx[s]], lambda s: cached[1][s, :ctx[s]], b,
                                  window if layer == 0 else None, sinks if layer == 0 else 0)
                R.check(to_bits(out), lse.cpu().numpy(), ref, f"iteration {i} layer {layer}")
                b.q = bits[:, :hq]
    del graphs
    torch.cuda.synchronize()
    for pl in plans:
        for p in pl:
            ap.plan_destroy(p)
    for p in pools:
        ap.kv_pool_destroy(p)


@pytest.mark.gpu
@pytest.mark.parametrize("four_bit", [False, True], ids=["bf16", "4bit"])
@pytest.mark.parametrize("shape,n", [((8, 2, 64), 3), ((32, 8, 128), 40)], ids=["small", "larger"])
def test_back_to_back_launches_see_what_the_one_before_wrote(shape, n, four_bit):
    """Kernels overlap the end of the one before them.  32 steps with data of their own through the same pages and the same
    rotated queries, captured without a gap: append with rotation, read back, attention.  Each has to give what it
    gives alone, bit for bit (the order of every sum is fixed)."""
    import torch
    hq, hkv, d = shape
    b = _batch(shape, 31, [1] * n, [37 + 5 * i for i in range(n)])
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    draw = lambda heads: torch.randn((32, n, heads, d), generator=gen, device="cuda:0").to(torch.bfloat16)
    q, k, v = draw(hq), draw(hkv), draw(hkv)
    if four_bit:
        pool = ap.kv_pool_create_4bit(b.num_pages, hkv, d)
        fill = ap.plan_create(pool, b.ctx_lens, b.ctx_lens, b.block_tables, hq)
        rows = torch.randn((int(b.ctx_lens.sum()), hkv, d), generator=gen, device="cuda:0").to(torch.bfloat16)
        ap.kv_append(pool, fill, rows, rows)
    else:
        planes = [to_dev(x) for x in (b.k_pool, b.v_pool)]
        pool = ap.kv_pool_create(b.num_pages, hkv, d, *planes)
    plan = ap.plan_create(pool, b.q_lens, b.ctx_lens, b.block_tables, hq)
    ws = torch.empty(max(256, ap.plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda:0")
    q_rot = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda:0")

    def steps(sync):
        res = [torch.empty((32, n, h, d), dtype=torch.bfloat16, device="cuda:0") for h in (hkv, hkv, hq)]
        lse = torch.empty((32, n, hq), dtype=torch.float32, device="cuda:0")

        def run():
            for i in range(32):
                ap.kv_append_rope(pool, plan, k[i], v[i], q[i], q_rot)
                sync()
                ap.kv_read_new(pool, plan, res[0][i], res[1][i])
                sync()
                ap.attention_iteration(pool, plan, q_rot, res[2][i], lse[i], ws)
                sync()
        return run, res + [lse]
    run, alone = steps(torch.cuda.synchronize)
    run()
    run, chained = steps(lambda: None)
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=st):
        run()
    for _ in range(20):
        for x in chained:
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert ap.last_device_status(pool) == 0
        for x, y in zip(chained, alone):
            assert torch.equal(x, y)
    del g
    if four_bit:
        ap.plan_destroy(fill)
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)
