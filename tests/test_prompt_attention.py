"""Attention of whole packed prompts against its definition in 64 bits."""
import ctypes

import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import layer_reference as R
from test_state_layers import NAN, Case, bits, dev, f64, host

SHAPES = [(8, 2, 64), (8, 8, 64), (6, 2, 128), (5, 1, 128), (16, 2, 128), (4, 4, 128)]
LENS = [[1], [5, 1, 0, 16, 17], [64], [65], [63, 64, 65, 1, 128, 2], [129, 300], [0, 257, 7, 33, 511], [640], [*range(1, 61), 200],
        [64, 33, 1, 20] * 50]


def inputs(seed, lens, hq, hkv, d, extra=2, scale=1.0):
    rng = np.random.default_rng(seed)
    n = int(sum(lens))
    q, k, v = bits(rng, n + extra, hq, d, scale=scale), bits(rng, n + extra, hkv, d), bits(rng, n + extra, hkv, d)
    for t in (q, k, v):
        t[n:] = NAN
    return n, q, k, v


def run(lens, hq, hkv, d, q, k, v, scale=0.0, want_lse=True, stream=None, pool=None):
    import torch
    own = pool is None
    pool = pool or ap.kv_pool_create(1, hkv, d)
    plan = ap.prompt_plan_create(pool, lens, hq, softmax_scale=scale)
    out = dev(np.full((q.shape[0], hq, d), NAN, np.uint16))
    lse = torch.full((q.shape[0], hq), 7.0, device="cuda") if want_lse else None
    ap.prompt_attention(pool, plan, q, k, v, out, lse, stream=stream)
    assert ap.last_device_status(pool) == 0
    ap.prompt_plan_destroy(plan)
    if own:
        ap.kv_pool_destroy(pool)
    return out, lse


def check(out, lse, n, q, k, v, lens, scale=None):
    with np.errstate(invalid="ignore"):
        ref, slack, ref_lse, lse_slack = R.prompt(f64(q[:n]), f64(k[:n]), f64(v[:n]), lens, scale)
    got = host(out)
    R.bf16_close(f64(got[:n]), ref, slack, "out")
    assert (got[n:] == NAN).all()
    if lse is not None:
        R.fp32_close(host(lse)[:n].astype(np.float64), ref_lse, lse_slack, "lse")
        assert (host(lse)[n:] == 7.0).all()


# ------------------------------------------------------------------ CPU --

def test_refusals():
    pool = ap.kv_pool_create(1, 2, 64, device=-1)
    lib = B.load()

    def refused(lens, hq, status):
        with pytest.raises(ap.ApError) as e:
            ap.prompt_plan_create(pool, lens, hq)
        assert e.value.status == status
    refused([1, -1], 8, B.AP_ERR_INVALID_ARG)
    refused([1], 7, B.AP_ERR_INVALID_ARG)
    refused([1], 0, B.AP_ERR_INVALID_ARG)
    refused([1], 18, B.AP_ERR_UNSUPPORTED)
    refused([1 << 30, 1 << 30], 8, B.AP_ERR_UNSUPPORTED)
    for bad in ([2 ** 32 + 1], [1.5], [[1]]):
        with pytest.raises(ValueError):
            ap.prompt_plan_create(pool, bad, 8)
    plan = ap.prompt_plan_create(pool, [3, 0, 200, 64, 65], 6)
    info = ap.prompt_plan_get_info(plan)
    assert info["n_rows"] == 332 and info["pairs"] == sum(n * (n + 1) // 2 for n in (3, 200, 64, 65)) and info["launches"] == 2
    assert info["tiles"] == 5 * 2 * 2 and info["short_units"] == 0         # (heads 0-2: two units; two kv heads)
    for lens, tiles, short, launches in (([3, 0, 64], 0, 5 * 2, 1), ([200] + [17] * 46, 48 * 4, 0, 2), ([200] + [17] * 47, 2 * 4, 94 * 2, 3)):
        p = ap.prompt_plan_create(pool, lens, 6)                           # (blocks of 16 rows; up to 185 units of short prompts)
        info = ap.prompt_plan_get_info(p)
        assert (info["tiles"], info["short_units"], info["launches"]) == (tiles, short, launches), lens
        ap.prompt_plan_destroy(p)

    def status(pool_=pool, strides=True, **kw):
        st = B.PromptStrides(0, 0, 0)
        for k, v in kw.items():
            setattr(st, k + "_row_stride", v)
        return lib.ap_prompt_attention(pool_.handle, plan.prompt_handle, 4096, 8192, 12288, 1 << 30, None, ctypes.byref(st) if strides else None, None)
    assert status() == B.AP_ERR_CUDA                                   # valid, but the pool is host-only
    assert status(strides=False) == B.AP_ERR_INVALID_ARG
    other = ap.kv_pool_create(1, 2, 64, device=-1)
    assert status(pool_=other) == B.AP_ERR_INVALID_ARG
    for bad in (dict(q=6 * 64 - 8), dict(k=64), dict(v=132), dict(q=-384), dict(k=2 ** 32 + 8), dict(v=2 ** 63 - 8)):
        assert status(**bad) == B.AP_ERR_INVALID_ARG, bad
    import torch

    def bf(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)
    good = dict(q=bf(332, 6, 64), k=bf(332, 2, 64), v=bf(332, 2, 64), out=bf(332, 6, 64))
    for name, bad in dict(q=bf(331, 6, 64), k=bf(332, 4, 64), v=bf(332, 2, 32), out=bf(332, 12, 64)[:, ::2]).items():
        with pytest.raises((ValueError, ap.ApError)):
            ap.prompt_attention(pool, plan, **{**good, name: bad})
    with pytest.raises(ValueError):
        ap.prompt_attention(pool, plan, **good, lse=bf(332, 6))
    empty = ap.prompt_plan_create(pool, [0, 0], 8)
    assert ap.prompt_plan_get_info(empty)["launches"] == 0
    for p in (plan, empty):
        ap.prompt_plan_destroy(p)
    for p in (pool, other):
        ap.kv_pool_destroy(p)


def test_reference_is_the_textbook_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 1, 8)), rng.standard_normal((7, 1, 8))
    out, _, lse, _ = R.prompt(q, k, v, [3, 4])
    assert np.allclose(out[0], v[0]) and np.allclose(out[3], v[3])      # a first token sees itself
    x = q[5, 1] @ k[3:6, 0].T / np.sqrt(8)
    assert np.allclose(out[5, 1], np.exp(x) @ v[3:6, 0] / np.exp(x).sum()) and np.isclose(lse[5, 1], np.log(np.exp(x).sum()))


# ------------------------------------------------------------------ GPU --

@pytest.mark.gpu
@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:8])))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}")
def test_prompts(shape, lens):
    n, q, k, v = inputs(len(lens) + shape[0], lens, *shape)
    out, lse = run(lens, *shape, dev(q), dev(k), dev(v))
    check(out, lse, n, q, k, v, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.5, 2.0])
def test_explicit_scale_and_growing_keys(scale):
    """Scores far apart, maxima that move along the prompt: the reference maximum has to follow."""
    lens = [700, 40]
    n, q, k, v = inputs(11, lens, 8, 2, 128)
    k[:n] = W.f32_to_bf16_bits((f64(k[:n]) * np.linspace(0.2, 4, n)[:, None, None]).astype(np.float32))
    out, lse = run(lens, 8, 2, 128, dev(q), dev(k), dev(v), scale=scale)
    check(out, lse, n, q, k, v, lens, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_strided_rows(d):
    lens, hq, hkv = [130, 3, 90], 8, 2
    n, q, k, v = inputs(21, lens, hq, hkv, d)
    t = dev(np.concatenate([q, k, v], 1))
    out, lse = run(lens, hq, hkv, d, t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:], want_lse=False)
    check(out, lse, n, q, k, v, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_what_no_row_of_a_prompt_sees_does_not_reach_it(d):
    """NaN and infinities in one prompt's K and V leave its neighbours alone; a NaN key makes the rows from it on NaN."""
    lens, shape = [200, 50, 333, 20, 30], (4, 2, d)
    n, q, k, v = inputs(31, lens, *shape)
    k[200:250], v[200:250] = NAN, NAN
    v[583:603] = 0x7F80
    k[200 + 50 + 300, 0] = NAN
    out, lse = run(lens, *shape, dev(q), dev(k), dev(v))
    got, kl = f64(host(out)[:n]), host(lse)[:n]
    clean = [(0, 200), (250, 550), (603, 633)]
    with np.errstate(invalid="ignore", over="ignore"):
        ref, slack, ref_lse, lse_slack = R.prompt(f64(q[:n]), f64(k[:n]), f64(v[:n]), lens)
    for a, b in clean:
        heads = slice(2, 4) if (a, b) == (250, 550) else slice(0, 4)
        R.bf16_close(got[a:b, heads], ref[a:b, heads], slack[a:b, heads], "out")
        R.fp32_close(kl[a:b, heads].astype(np.float64), ref_lse[a:b, heads], lse_slack[a:b, heads], "lse")
    assert np.isnan(got[550:583, :2]).all() and np.isfinite(got[250:583, 2:]).all() and np.isfinite(got[250:550, :2]).all()
    assert np.isnan(got[200:250]).all()


@pytest.mark.gpu
def test_prompts_are_the_paged_kernels_prompts():
    """The same prompts through the cache: append, attention_iteration; then a decode step over what was appended."""
    import torch
    hq, hkv, d, lens = 8, 2, 128, [300, 1, 64, 130]
    n, q, k, v = inputs(41, lens, hq, hkv, d, extra=0)
    need = [-(-(m + 1) // 16) for m in lens]
    table = np.full((len(lens), max(need)), -1, np.int32)
    ids = np.random.default_rng(5).permutation(sum(need)).astype(np.int32)
    for s, m in enumerate(need):
        table[s, :m] = ids[sum(need[:s]):sum(need[:s]) + m]
    pool = ap.kv_pool_create(sum(need), hkv, d)
    plan = ap.plan_create(pool, lens, lens, table, hq)
    ws = torch.empty(max(256, ap.plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda")
    tq, tk, tv = dev(q), dev(k), dev(v)
    paged, paged_lse = torch.empty_like(tq), torch.empty((n, hq), device="cuda")
    direct, lse = run(lens, hq, hkv, d, tq, tk, tv, pool=pool)
    ap.kv_append(pool, plan, tk, tv)
    ap.attention_iteration(pool, plan, tq, paged, paged_lse, ws)
    check(direct, lse, n, q, k, v, lens)
    check(paged, None, n, q, k, v, lens)
    assert (paged_lse - lse).abs().max().item() < 1e-3
    assert ap.last_device_status(pool) == 0
    ap.plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
def test_a_hybrid_iteration_run_together_and_captured():
    """Prompt attention, append, convolution and scan of one iteration, one after the other, eager and as a graph."""
    import torch
    lens, hq, hkv, d = [150, 20, 1], 8, 2, 64
    n, q, k, v = inputs(51, lens, hq, hkv, d, extra=0)
    c = Case(52, 64, 16, 4, lens, [150, 25, 3], extra_rows=0).open()
    pool = ap.kv_pool_create(32, hkv, d)
    prompts = ap.prompt_plan_create(pool, lens, hq)
    tq, tk, tv = dev(q), dev(k), dev(v)
    out, lse = torch.empty_like(tq), torch.empty((n, hq), device="cuda")
    x, dt, a, b, cc, w, z = (dev(t) for t in (c.x, c.dt, c.a, c.b, c.c, c.weight, c.z))
    mid, y, ws = c.blank(), c.blank(), c.workspace()

    def iteration():
        ap.prompt_attention(pool, prompts, tq, tk, tv, out, lse)
        ap.conv_iteration(c.pool, c.plan, x, w, mid)
        ap.scan_iteration(c.pool, c.plan, mid, dt, a, b, cc, y, z=z, d_skip=None, workspace=ws)
    iteration()
    torch.cuda.synchronize()
    check(out, None, n, q, k, v, lens)
    first = host(out), host(y), host(c.d_state)
    c.x = host(mid)                                                       # the scan's input
    c.check_scan(y, piece=64, z=c.z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iteration()
    c.d_conv.copy_(dev(c.conv))
    c.d_state.copy_(dev(c.state))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(host(out), first[0]) and np.array_equal(host(y), first[1])
    assert np.array_equal(host(c.d_state).view(np.int32), first[2].view(np.int32))
    ap.prompt_plan_destroy(prompts)
    ap.kv_pool_destroy(pool)
    c.close()


@pytest.mark.gpu
def test_two_streams_overlaps_and_the_profile():
    """One plan on two streams at once; results over results or inputs are refused; every kernel is in the profile."""
    import torch
    lens, hq, hkv, d = [200, 20, 65, 1, 300], 6, 2, 64
    sets = [inputs(seed, lens, hq, hkv, d, extra=0) for seed in (61, 62)]
    n = sets[0][0]
    pool = ap.kv_pool_create(1, hkv, d)
    plan = ap.prompt_plan_create(pool, lens, hq)
    tensors = [[dev(t) for t in s[1:]] for s in sets]
    results = [(torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, hq, device="cuda")) for _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for t, r, st in zip(tensors, results, streams):
        with torch.cuda.stream(st):
            ap.prompt_attention(pool, plan, *t, *r)
    torch.cuda.synchronize()
    for s, (out, lse) in zip(sets, results):
        check(out, lse, *s, lens)
    q, k, v = tensors[0]
    out, lse = results[0]
    both = torch.empty(n * hq * (d // 2 + 1), device="cuda")
    shared = both[:n * hq * d // 2].view(torch.bfloat16).view(n, hq, d), both[n * hq * d // 2 - 4:n * hq * d // 2 - 4 + n * hq].view(n, hq)
    for a in ((q, k, v, q, lse), (q, k, v, out, k.view(-1)[:2 * n * hq].view(torch.float32).view(n, hq)), (q, k, v, *shared)):
        with pytest.raises(ap.ApError) as e:
            ap.prompt_attention(pool, plan, *a)
        assert e.value.status == B.AP_ERR_INVALID_ARG
    ap.profile_enable(pool)
    ap.prompt_attention(pool, plan, q, k, v, out, lse)
    times = ap.profile_collect(pool)
    assert sum(launches for _, launches in times.values()) == ap.prompt_plan_get_info(plan)["launches"] == 2
    assert sum(ms for ms, _ in times.values()) > 0
    ap.profile_enable(pool, False)
    assert ap.last_device_status(pool) == 0
    ap.prompt_plan_destroy(plan)
    ap.kv_pool_destroy(pool)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """q, k and v in rows 2^26 elements apart, for both kernels."""
    import torch
    lens, hq, hkv, d = [5, 66], 2, 1, 64
    n, q, k, v = inputs(71, lens, hq, hkv, d, extra=0)
    wide = torch.empty((n, 1 << 26), dtype=torch.bfloat16, device="cuda")
    at, views = (1 << 26) - 256, []
    for t, heads in ((q, hq), (k, hkv), (v, hkv)):
        view = wide[:, at:at + heads * d].unflatten(1, (heads, d))
        view.copy_(dev(t))
        views.append(view)
        at += heads * d
    out, lse = run(lens, hq, hkv, d, *views)
    check(out, lse, n, q, k, v, lens)
