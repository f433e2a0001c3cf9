"""Edges of the operators over state slots: states and decays at the ends of fp32, what a call may not depend on, refusals."""
import os
import re
from unittest import mock

import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import layer_reference as R
from test_state_layers import NAN, Case, dev, f64, host

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def reference(c, piece=0, z=False, softplus=False):
    """R.scan of a case where a row's decay by itself may leave fp32 (its product with the state does not)."""
    with mock.patch.object(R, "LARGEST", 1e300):
        return R.scan(f64(c.x[:c.n]), f64(c.dt[:c.n]), c.a.astype(np.float64), f64(c.b[:c.n]), f64(c.c[:c.n]),
                      np.where(c.live[:, None, None], c.state, 0), c.q_lens, c.ctx_lens, c.slots, piece=piece,
                      z=f64(c.z[:c.n]) if z else None, softplus=softplus)


def check(c, out, ref, slack, state, off):
    assert np.isfinite(slack).all() and np.isfinite(off[c.touched]).all()             # (every element is compared)
    assert max(np.abs(ref).max(), np.abs(state[c.touched]).max()) < 1e37
    R.bf16_close(f64(host(out)[:c.n]), ref, slack, "out")
    assert (host(out)[c.n:] == NAN).all()
    R.fp32_close(host(c.d_state)[c.touched].astype(np.float64), state[c.touched], off[c.touched], "state")


def bf16(v):
    return W.f32_to_bf16_bits(np.asarray(v, np.float32))


# ------------------------------------------------------------------ CPU --

def test_strided_tensors_of_another_element_size_are_refused():
    """The library takes row strides in elements of two bytes: a view of bytes has strides twice too long for its memory."""
    import torch
    pool = ap.state_pool_create(4, 64, 16, 4, device=-1)
    plan = ap.state_plan_create(pool, [2], [2], [0])
    kv = ap.kv_pool_create(4, 2, 64, device=-1)
    prompts = ap.prompt_plan_create(kv, [2], 2)
    append = ap.plan_create(kv, [2], [2], np.array([[0]], np.int32), 2)

    def rows(dtype, *shape):                                   # every other part of a wider tensor's rows
        return torch.zeros((shape[0], 2, *shape[1:]), dtype=dtype)[:, 0]
    good = {t: rows(t, 2, 64) for t in (torch.bfloat16, torch.int16, torch.uint8)}
    heads = {t: rows(t, 2, 2, 64) for t in good}
    w, bc, a = torch.zeros(64, 4, dtype=torch.bfloat16), rows(torch.bfloat16, 2, 16), torch.zeros(64, 16)
    calls = [lambda t: ap.conv_iteration(pool, plan, good[t], w, good[torch.bfloat16]),
             lambda t: ap.conv_iteration(pool, plan, good[torch.bfloat16], w, good[t]),
             lambda t: ap.scan_iteration(pool, plan, good[t], good[torch.bfloat16], a, bc, bc, good[torch.bfloat16].clone()),
             lambda t: ap.scan_iteration(pool, plan, good[torch.bfloat16], good[torch.bfloat16], a, rows(t, 2, 16), bc, good[torch.bfloat16].clone()),
             lambda t: ap.prompt_attention(kv, prompts, heads[t], heads[torch.bfloat16], heads[torch.bfloat16], torch.zeros(2, 2, 64, dtype=torch.bfloat16)),
             lambda t: ap.kv_append_rope(kv, append, heads[t], heads[torch.bfloat16])]
    for call in calls:
        for t in (torch.bfloat16, torch.int16):
            with pytest.raises(ap.ApError) as e:
                call(t)
            assert e.value.status == B.AP_ERR_CUDA             # (taken, but the pool is host-only)
        with pytest.raises(ValueError):
            call(torch.uint8)
    for destroy, x in ((ap.state_plan_destroy, plan), (ap.prompt_plan_destroy, prompts), (ap.plan_destroy, append),
                       (ap.state_pool_destroy, pool), (ap.kv_pool_destroy, kv)):
        destroy(x)


def test_expanded_planes_are_refused():
    """A plane that is one page many times over has fewer bytes than it says."""
    import torch
    one = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    whole = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    for k, v in ((one.expand(4, 2, 16, 64), whole), (whole, one.expand(4, 2, 16, 64))):
        with pytest.raises(ValueError):
            ap.kv_pool_create(4, 2, 64, k, v, device=-1)
        with pytest.raises(ValueError):
            ap.kv_pool_create_4bit(4, 2, 64, k, v, device=-1)


def test_negative_workspaces_are_refused():
    """A size below zero would wrap to a huge one."""
    import torch
    kv = ap.kv_pool_create(4, 2, 64, device=-1)
    plan = ap.plan_create(kv, [1], [1], np.array([[0]], np.int32), 2)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    pool = ap.state_pool_create(4, 64, 16, 4, device=-1)
    rows = ap.state_plan_create(pool, [2], [2], [0])
    x, bc, a = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 16, dtype=torch.bfloat16), torch.zeros(64, 16)
    space = torch.zeros(256, dtype=torch.uint8)
    for workspace in (space, 4096, None):
        with pytest.raises(ValueError):
            ap.attention_iteration(kv, plan, q, q.clone(), workspace=workspace, workspace_bytes=-1)
        if workspace is not None:
            with pytest.raises(ValueError):
                ap.scan_iteration(pool, rows, x, x, a, bc, bc, x.clone(), workspace=workspace, workspace_bytes=-1)
    for destroy, h in ((ap.plan_destroy, plan), (ap.state_plan_destroy, rows), (ap.state_pool_destroy, pool), (ap.kv_pool_destroy, kv)):
        destroy(h)


def test_larger_tensors_of_other_heads_are_refused():
    """Rows to spare are fine; rows of another width would be read as if they were the plan's."""
    import torch
    kv = ap.kv_pool_create(4, 2, 64, device=-1)
    prompts = ap.prompt_plan_create(kv, [3], 4)

    def bf(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)
    good = dict(q=bf(3, 4, 64), k=bf(3, 2, 64), v=bf(3, 2, 64), out=bf(3, 4, 64))
    for name, ok in dict(q=bf(5, 4, 64), k=bf(4, 128), v=bf(1000), out=bf(9, 256)).items():
        with pytest.raises(ap.ApError) as e:
            ap.prompt_attention(kv, prompts, **{**good, name: ok})
        assert e.value.status == B.AP_ERR_CUDA                  # (taken, but the pool is host-only)
    for name, bad in dict(q=bf(3, 8, 64), k=bf(3, 4, 64), v=bf(3, 3, 64), out=bf(3, 8, 64)).items():
        with pytest.raises(ValueError):
            ap.prompt_attention(kv, prompts, **{**good, name: bad})
    empty = ap.prompt_plan_create(kv, [0], 4)
    with pytest.raises(ap.ApError) as e:
        ap.prompt_attention(kv, empty, bf(3, 5), bf(3, 7), bf(2, 9), bf(3, 5))
    assert e.value.status == B.AP_ERR_CUDA                      # (a plan without tokens takes any tensors)
    ap.prompt_plan_destroy(empty)
    ap.prompt_plan_destroy(prompts)
    ap.kv_pool_destroy(kv)


def test_polynomials_are_as_good_as_stated():
    """The coefficients of the scan's softplus and 2^x, as the source has them: the errors that its comments state."""
    source = open(os.path.join(ROOT, "paper_2604_07144_b200", "csrc", "scan.cu")).read()

    def part(begin, end):
        return source[source.index(begin):source.index(end, source.index(begin))]

    def poly(body, x, first):
        p = np.zeros_like(x)
        for c in re.findall(first, body):
            p = p * x + float(np.float32(c))
        return p

    one, two = part("float softplus(float x)", "return"), part("float2 softplus2(float2 x)", "float max_nan(")
    u = np.linspace(1e-9, 1, 400001)
    want = np.log1p(u) / u
    for body, pattern in ((one, r"(?:p = |u, )(-?\d+\.\d*)f"), (two, r"two\((-?\d+\.\d*)f\)")):
        assert len(re.findall(pattern, body)) == 10
        assert np.abs(poly(body, u, pattern) / want - 1).max() < 3.5e-8
    exp2 = part("// 2^x for two values", "// 2^x, to be multiplied")
    f = np.concatenate([np.linspace(-0.5, -1e-6, 200001), np.linspace(1e-6, 0.5, 200001)])
    pattern = r"make_float2\((0\.\d+)f, "
    assert len(re.findall(pattern, exp2)) == 5
    assert np.abs(f * poly(exp2, f, pattern) / np.expm1(f * np.log(2)) - 1).max() < 4.7e-7


# ------------------------------------------------------------------ GPU --

@pytest.mark.gpu
@pytest.mark.parametrize("fresh", [True, False], ids=["from_zeros", "from_its_slot"])
@pytest.mark.parametrize("states", [8, 16, 32, 64])
def test_growth_over_whole_pieces_of_a_cut(states, fresh):
    """A sequence cut along time whose layer grows by e^96 and more over one piece and decays by as much over the next: the
    state stays in range, a piece's factor does not.  Without inputs until row 448, so from zeros it stays zero until there."""
    n, ch = 700, 64
    c = Case(900 + states, ch, states, 4, [n], [n if fresh else n + 5])
    rng = np.random.default_rng(states)
    t = np.arange(n)
    step = np.where(t < 448, np.where(t // 64 % 2 == 0, -1.5, 1.5), -0.02)
    c.dt[:n] = bf16(np.broadcast_to(step[:, None], (n, ch)))
    c.x[:448] = 0
    c.a = rng.uniform(1.0, 1.4, (ch, states)).astype(np.float32)                       # (a row: e^(1.5 a))
    c.a[::2] *= -1                                                                      # (these begin with growth, the others with decay)
    c.state[c.live] = (1e-2 * rng.uniform(0.5, 1, c.state[c.live].shape)).astype(np.float32)
    c.state[c.live, ::2] *= 1e-28
    c.state[c.live, 1::2] *= 1e28
    c.open()
    assert ap.state_plan_get_info(c.plan)["segments"] == n // 64
    ref = reference(c, piece=64)
    out = c.run_scan(softplus=False)
    check(c, out, *ref)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [8, 16, 32, 64])
def test_a_row_whose_decay_alone_leaves_fp32(states):
    """Decays of a single row from e^-150 to e^150 on states that stay in range: zeros stay zeros, small states grow to large
    ones and large ones shrink, in chunks as in single tokens."""
    lens, ctx = [40, 1, 1, 3, 1, 17], [40, 1, 9, 3, 7, 30]
    ch = 72
    c = Case(920 + states, ch, states, 4, lens, ctx)
    rng = np.random.default_rng(states)
    row = 0
    for s, m in enumerate(lens):
        # growth and decay in turn, so that a state comes back to where it was; inputs, as small, with a decay only
        step = np.where(np.arange(m) % 2 == 0, 1.25, -1.25) * (1 if s != 4 else -1)
        c.dt[row:row + m] = bf16(np.broadcast_to(step[:, None], (m, ch)))
        c.x[row:row + m][step > 0] = 0
        c.x[row:row + m][step < 0] = bf16(1e-31 * f64(c.x[row:row + m][step < 0]))
        row += m
    c.a = rng.uniform(75, 120, (ch, states)).astype(np.float32)
    state = rng.uniform(0.5, 1, c.state.shape) * np.where(rng.random(c.state.shape) < 0.3, 0, 1e-31)
    state[c.slots[4]] = np.where(state[c.slots[4]] == 0, 0, state[c.slots[4]] * 1e62)   # (this one only decays)
    c.state[c.live] = state[c.live]
    c.open()
    ref = reference(c)
    out = c.run_scan(softplus=False)
    check(c, out, *ref)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states,channels", [(16, 72), (16, 8), (8, 40), (8, 72), (32, 8), (64, 200)])
def test_what_ran_before_does_not_change_a_bit(states, channels):
    """Channels that do not fill a warp: identical calls give identical bits, whatever another call left in shared memory."""
    import torch
    c = Case(940 + states, channels, states, 4, [200, 1, 37], [200, 4, 45])
    c.a /= states
    c.open()
    wide = 8192
    pool = ap.state_pool_create(8, wide, states, 4)
    plan = ap.state_plan_create(pool, [16] * 8, [16] * 8, range(8))
    assert ap.state_plan_get_info(plan)["split_seqs"] == 0
    rows = [torch.empty(128, wide, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    a, bc = torch.zeros(wide, states, device="cuda"), torch.ones(128, states, dtype=torch.bfloat16, device="cuda")
    seen = []
    for left in (0.0, float("nan"), 1e30, -0.25):
        rows[0].fill_(left)
        rows[1].fill_(left)
        ap.scan_iteration(pool, plan, rows[0], rows[1], a, bc, bc, rows[2], z=rows[0], softplus=False)
        c.d_state.copy_(dev(c.state))
        out = c.run_scan(**c.all_scan())
        seen.append((host(out)[:c.n], host(c.d_state)[c.touched].view(np.int32)))
    c.check_scan(out, piece=64, **c.all_scan())
    for got in seen[1:]:
        assert np.array_equal(got[0], seen[0][0]) and np.array_equal(got[1], seen[0][1])
    ap.state_plan_destroy(plan)
    ap.state_pool_destroy(pool)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [8, 16, 32, 64])
def test_raw_steps_of_either_sign_over_three_tiles(states):
    """Growth that stays in range, so that every row of every tile is compared."""
    c = Case(960 + states, 72, states, 4, [9, 1, 40], [9, 6, 50])
    c.a /= 4 * states
    c.open()
    out = c.run_scan(softplus=False)
    check(c, out, *reference(c))
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states,channels,lens", [(16, 64, [700]), (64, 40, [513]), (8, 128, [1025])])
def test_cut_along_time_within_a_pieces_roundings(states, channels, lens):
    """A sum of a piece's steps rounds as often as the piece has rows, not the sequence."""
    c = Case(980 + states, channels, states, 4, lens, [n + 3 for n in lens]).open()
    pieces = ap.state_plan_get_info(c.plan)["segments"]
    assert pieces >= 5
    c.check_scan(c.run_scan(**c.all_scan()), piece=lens[0] // pieces, **c.all_scan())
    c.close()
