"""Short causal convolution and selective scan over state slots against their definitions in 64 bits."""
import ctypes

import numpy as np
import pytest

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import binding as B
from paper_2604_07144_b200 import workloads as W

import layer_reference as R

NAN = 0x7FC1


def bits(rng, *shape, scale=1.0):
    return W.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


f64 = W.bf16_bits_to_f64


def dev(a):
    """numpy (uint16: bf16 bits) -> device tensor"""
    import torch
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(a).cuda()


def host(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.cpu().numpy()


class Case:
    """A batch over a layer's slots; every slot and every row that no call may read is NaN."""

    def __init__(self, seed, channels, states, width, q_lens, ctx_lens, extra_rows=3, slots=None):
        rng = np.random.default_rng(seed)
        self.channels, self.states, self.width = channels, states, width
        self.q_lens, self.ctx_lens = np.asarray(q_lens, np.int32), np.asarray(ctx_lens, np.int32)
        self.n, self.rows = int(self.q_lens.sum()), int(self.q_lens.sum()) + extra_rows
        self.num_slots = len(q_lens) + 3
        self.slots = rng.permutation(self.num_slots)[:len(q_lens)].astype(np.int32) if slots is None else np.asarray(slots, np.int32)
        self.x, self.dt, self.z = bits(rng, self.rows, channels), bits(rng, self.rows, channels, scale=0.7), bits(rng, self.rows, channels)
        self.b, self.c = bits(rng, self.rows, states), bits(rng, self.rows, states)
        for t in (self.x, self.dt, self.z, self.b, self.c):
            t[self.n:] = NAN
        self.weight, self.bias = bits(rng, channels, width, scale=0.5), bits(rng, channels)
        self.dt_bias = rng.uniform(-6, -1, channels).astype(np.float32)
        self.a = -(np.arange(1, states + 1) * np.exp(0.3 * rng.standard_normal((channels, states)))).astype(np.float32)
        self.skip = rng.standard_normal(channels).astype(np.float32)
        self.conv = bits(rng, self.num_slots, width - 1, channels)
        self.state = rng.standard_normal((self.num_slots, channels, states)).astype(np.float32)
        self.live = np.zeros(self.num_slots, bool)              # slots that the batch goes on from
        for s, (q, c) in enumerate(zip(self.q_lens, self.ctx_lens)):
            self.live[self.slots[s]] = c > q > 0
        self.conv[~self.live] = NAN
        self.state[~self.live] = np.nan
        self.touched = np.zeros(self.num_slots, bool)
        self.touched[self.slots[self.q_lens > 0]] = True

    def open(self):
        self.d_conv, self.d_state = dev(self.conv), dev(self.state)
        self.pool = ap.state_pool_create(self.num_slots, self.channels, self.states, self.width, self.d_conv, self.d_state)
        self.plan = ap.state_plan_create(self.pool, self.q_lens, self.ctx_lens, self.slots)
        return self

    def close(self):
        import torch
        torch.cuda.synchronize()
        ap.state_plan_destroy(self.plan)
        ap.state_pool_destroy(self.pool)

    def workspace(self):
        import torch
        return torch.full((max(256, ap.state_plan_workspace_bytes(self.plan)),), 0xFF, dtype=torch.uint8, device="cuda")

    def check_conv(self, out, bias=True, silu=True):
        ref, slack, state = R.conv(f64(self.x[:self.n]), f64(self.weight), f64(self.bias) if bias else None,
                                   np.where(self.live[:, None, None], f64(self.conv), 0), self.q_lens, self.ctx_lens, self.slots, silu)
        got = host(out)
        R.bf16_close(f64(got[:self.n]), ref, slack, "out")
        assert (got[self.n:] == NAN).all()
        now = host(self.d_conv)
        assert np.array_equal(now[~self.touched], self.conv[~self.touched])
        assert np.array_equal(f64(now[self.touched]), state[self.touched])

    def check_scan(self, out, piece=0, **kw):
        args = {k: v[:self.n] if k == "z" else v for k, v in kw.items() if v is not None}
        if "z" in args:
            args["z"] = f64(args["z"])
        ref, slack, state, off = R.scan(f64(self.x[:self.n]), f64(self.dt[:self.n]), self.a.astype(np.float64), f64(self.b[:self.n]),
                                        f64(self.c[:self.n]), np.where(self.live[:, None, None], self.state, 0), self.q_lens, self.ctx_lens,
                                        self.slots, piece=piece, **args)
        got = host(out)
        R.bf16_close(f64(got[:self.n]), ref, slack, "out")
        assert (got[self.n:] == NAN).all()
        now = host(self.d_state)
        assert np.array_equal(now[~self.touched].view(np.int32), self.state[~self.touched].view(np.int32))
        R.fp32_close(now[self.touched].astype(np.float64), state[self.touched], off[self.touched], "state")

    def blank(self):
        return dev(np.full((self.rows, self.channels), NAN, np.uint16))

    def all_scan(self):
        return dict(z=self.z, d_skip=self.skip, dt_bias=self.dt_bias)

    def run_scan(self, out=None, z=None, d_skip=None, dt_bias=None, softplus=True, stream=None):
        out = self.blank() if out is None else out
        ap.scan_iteration(self.pool, self.plan, dev(self.x), dev(self.dt), dev(self.a), dev(self.b), dev(self.c), out,
                          z=None if z is None else dev(z), d_skip=None if d_skip is None else dev(d_skip),
                          dt_bias=None if dt_bias is None else dev(dt_bias), softplus=softplus, workspace=self.workspace(), stream=stream)
        return out


BATCHES = [
    ([1], [1]), ([1], [9]), ([2], [2]), ([3], [7]), ([16], [16]), ([17], [18]), ([33, 1, 2], [33, 5, 9]),
    ([0, 1, 40, 0, 1, 2, 1, 97], [4, 1, 900, 0, 77, 2, 5, 97]), ([1] * 19, list(range(1, 20))), ([65, 64, 31, 32], [65, 65, 31, 40]),
]


# ------------------------------------------------------------------ CPU --

def test_plan_and_pool_refusals():
    lib = B.load()

    def pool_status(**kw):
        d = B.StateDesc(4, 64, 16, 4, None, None, -1)
        for k, v in kw.items():
            setattr(d, k, v)
        h = ctypes.c_void_p()
        st = lib.ap_state_pool_create(ctypes.byref(h), ctypes.byref(d))
        if st == 0:
            lib.ap_state_pool_destroy(h)
        else:
            assert not h.value and lib.ap_state_pool_scan_bytes(ctypes.byref(d)) == 0 or "base" in str(kw)
        return st
    assert pool_status() == 0
    for bad in (dict(num_slots=0), dict(channels=0), dict(channels=-8), dict(state_dim=0), dict(conv_width=0), dict(num_slots=-1),
                dict(conv_base=4096), dict(scan_base=4096), dict(conv_base=8, device=0), dict(scan_base=24, device=0),
                dict(conv_base=1 << 20, scan_base=(1 << 20) + 4 * 3 * 64 * 2 - 16, device=0),                 # planes that share 16 bytes
                dict(conv_base=(1 << 20) + 4 * 64 * 16 * 4 - 16, scan_base=1 << 20, device=0)):
        assert pool_status(**bad) == B.AP_ERR_INVALID_ARG, bad
    for bad in (dict(channels=12), dict(channels=(1 << 20) + 8), dict(state_dim=4), dict(state_dim=24), dict(state_dim=128),
                dict(conv_width=1), dict(conv_width=5)):
        assert pool_status(**bad) == B.AP_ERR_UNSUPPORTED, bad
    assert ap.state_pool_conv_bytes(3, 64, 16, 4) == 3 * 3 * 64 * 2 and ap.state_pool_scan_bytes(3, 64, 16, 4) == 3 * 64 * 16 * 4

    pool = ap.state_pool_create(4, 64, 16, 4, device=-1)

    def refused(q, c, s, status=B.AP_ERR_INVALID_ARG):
        with pytest.raises(ap.ApError) as e:
            ap.state_plan_create(pool, q, c, s)
        assert e.value.status == status
    refused([1, 1], [1, 2], [2, 2])                                   # a slot twice
    refused([1], [1], [4])
    refused([1], [1], [-1])
    refused([2], [1], [0])
    refused([-1], [1], [0])
    refused([1 << 30, 1 << 30], [1 << 30, 1 << 30], [0, 1], B.AP_ERR_UNSUPPORTED)
    with pytest.raises(ValueError):
        ap.state_plan_create(pool, [1], [1], [2 ** 32])
    with pytest.raises(ValueError):
        ap.state_plan_create(pool, [1, 1], [1], [0])
    with pytest.raises(ValueError):
        ap.state_plan_create(pool, [1.5], [2], [0])
    plan = ap.state_plan_create(pool, [0, 1, 0], [5, 1, 0], [2, 2, 9])     # (without new tokens a slot is not looked at)
    assert ap.state_plan_get_info(plan) == dict(n_new=1, single_rows=1, chunk_seqs=0, split_seqs=0, segments=0, launches_scan=1)
    for q, launches in (([1, 1], 1), ([1, 2], 1), ([2, 2], 1), ([1 << 16], 2), ([1 << 16, 1, 70], 2)):    # (single tokens go with the walks)
        p = ap.state_plan_create(pool, q, q, list(range(len(q))))
        assert ap.state_plan_get_info(p)["launches_scan"] == launches
        ap.state_plan_destroy(p)
    empty = ap.state_plan_create(pool, [], [], [])
    assert ap.state_plan_get_info(empty)["n_new"] == 0 and ap.state_plan_workspace_bytes(empty) == 0
    for p in (plan, empty):
        ap.state_plan_destroy(p)
    ap.state_pool_destroy(pool)


def test_call_refusals():
    import torch
    pool, other = ap.state_pool_create(4, 64, 16, 4, device=-1), ap.state_pool_create(4, 64, 32, 4, device=-1)
    plan = ap.state_plan_create(pool, [2], [2], [0])
    lib = B.load()

    def conv(pool_=pool, desc=True, **kw):
        d = B.ConvDesc(1, 0, 0, 4096, 8192, None, 1 << 20)
        for k, v in kw.items():
            setattr(d, k, v)
        return lib.ap_conv_iteration(pool_.state_handle, plan.state_plan_handle, ctypes.byref(d) if desc else None, None)

    def scan(pool_=pool, desc=True, **kw):
        d = B.ScanDesc(1, 0, 0, 0, 0, 0, 0, *[4096] * 5, 1 << 20, *[4096] * 3)
        for k, v in kw.items():
            setattr(d, k, v)
        return lib.ap_scan_iteration(pool_.state_handle, plan.state_plan_handle, ctypes.byref(d) if desc else None, None, 0, None)
    assert conv() == scan() == B.AP_ERR_CUDA                            # valid, but the pool is host-only
    assert conv(pool_=other) == scan(pool_=other) == B.AP_ERR_INVALID_ARG
    assert conv(desc=False) == scan(desc=False) == B.AP_ERR_INVALID_ARG
    for far in (56, 68, -64, 2 ** 32 + 8, 2 ** 63 - 8):
        for name in ("x", "out"):
            assert conv(**{name + "_row_stride": far}) == B.AP_ERR_INVALID_ARG, (name, far)
        for name in ("x", "dt", "z", "out"):
            assert scan(**{name + "_row_stride": far}) == B.AP_ERR_INVALID_ARG, (name, far)
    for name in ("b", "c"):
        assert scan(**{name + "_row_stride": 8}) == scan(**{name + "_row_stride": 20}) == B.AP_ERR_INVALID_ARG
    assert conv(silu=2) == scan(softplus=-1) == B.AP_ERR_INVALID_ARG

    def bf(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)
    good = dict(x=bf(2, 64), dt=bf(2, 64), a=torch.zeros(64, 16), b=bf(2, 16), c=bf(2, 16), out=bf(2, 64))
    for name, bad in dict(x=bf(1, 64), dt=bf(2, 32), a=torch.zeros(64, 8), b=bf(2, 32), c=bf(2, 32)[:, ::2], out=torch.zeros(2, 64)).items():
        with pytest.raises(ValueError):
            ap.scan_iteration(pool, plan, **{**good, name: bad})
    for bad in (bf(1, 64).expand(2, 64), bf(64, 2).T, bf(2, 64).double(), np.zeros((2, 64), np.float32)):
        with pytest.raises(ValueError):
            ap.conv_iteration(pool, plan, bad, bf(64, 4), bf(2, 64))
        with pytest.raises(ValueError):
            ap.scan_iteration(pool, plan, **{**good, "z": bad})
    with pytest.raises(ValueError):
        ap.conv_iteration(pool, plan, bf(2, 64), bf(64, 3), bf(2, 64))
    with pytest.raises(ValueError):
        ap.scan_iteration(pool, plan, **good, d_skip=bf(64))
    with pytest.raises(ValueError):
        ap.scan_iteration(pool, plan, **good, dt_bias=torch.zeros(63))
    with pytest.raises(ValueError):
        ap.state_pool_create(4, 64, 16, 4, bf(4, 3, 63), device=-1)
    ap.state_plan_destroy(plan)
    for p in (pool, other):
        ap.state_pool_destroy(p)


def test_reference_steps_and_chunks_agree():
    """The reference itself: a prompt is its tokens one by one; without decay and gate a scan is a running sum."""
    c = Case(1, 8, 8, 4, [12], [12])
    x, w = f64(c.x[:12]), f64(c.weight)
    whole, _, st = R.conv(x, w, None, np.zeros_like(f64(c.conv)), [12], [12], [0], True)
    st2 = np.zeros_like(st)
    for t in range(12):
        y, _, st2 = R.conv(x[t:t + 1], w, None, st2, [1], [t + 1], [0], True)
        assert np.allclose(y[0], whole[t], rtol=1e-12)
    assert np.array_equal(st, st2)
    one = np.ones((12, 8))
    y, _, s, _ = R.scan(x, one, np.zeros((8, 8)), one, one / 8, np.zeros(c.state.shape), [12], [12], [0], softplus=False)
    assert np.allclose(y, np.cumsum(x, 0)) and np.allclose(s[0], x.sum(0)[:, None] * np.ones(8))


# ------------------------------------------------------------------ GPU --

@pytest.mark.gpu
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_conv(width, batch):
    c = Case(100 + batch, [8, 64, 200, 1032][batch % 4], 8, width, *BATCHES[batch]).open()
    bias, silu = batch % 3 != 1, batch % 2 == 0
    out = c.blank()
    ap.conv_iteration(c.pool, c.plan, dev(c.x), dev(c.weight), out, bias=dev(c.bias) if bias else None, silu=silu)
    c.check_conv(out, bias, silu)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [8, 16, 32, 64])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_scan(states, batch):
    c = Case(200 + batch, [8, 64, 200, 136][(batch + states // 16) % 4], states, 4, *BATCHES[batch]).open()
    kw = {k: v for i, (k, v) in enumerate(c.all_scan().items()) if (batch + states // 8) % 4 != i}
    c.check_scan(c.run_scan(**kw), piece=ap.state_plan_get_info(c.plan)["segments"] and 64, **kw)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states,channels,lens,fresh", [(16, 64, [700], True), (16, 136, [333, 1, 640, 5], False), (64, 40, [513, 128], False),
                                                         (8, 128, [1025], False), (32, 72, [300, 129, 257], True)])
def test_scan_cut_along_time(states, channels, lens, fresh):
    c = Case(300 + states, channels, states, 4, lens, lens if fresh else [n + 3 for n in lens]).open()
    info = ap.state_plan_get_info(c.plan)
    assert info["split_seqs"] >= 1 and info["segments"] > info["split_seqs"] and ap.state_plan_workspace_bytes(c.plan) > 0
    c.check_scan(c.run_scan(**c.all_scan()), piece=max(lens), **c.all_scan())
    with pytest.raises(ap.ApError) as e:
        ap.scan_iteration(c.pool, c.plan, dev(c.x), dev(c.dt), dev(c.a), dev(c.b), dev(c.c), c.blank())
    assert e.value.status == B.AP_ERR_WORKSPACE_TOO_SMALL
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [8, 16, 64])
def test_scan_without_softplus_and_with_far_values(states):
    """Raw steps of either sign (growth as well as decay), decays that underflow, steps of 0, large negative steps."""
    c = Case(400 + states, 72, states, 4, [9, 1, 40], [9, 6, 50]).open()
    c.check_scan(c.run_scan(softplus=False), softplus=False)
    c.close()
    c = Case(410 + states, 72, states, 4, [9, 1, 40], [9, 6, 50])
    v = c.dt[:c.n].reshape(-1)
    for i, far in enumerate((-30.0, 60.0, -100.0, 1000.0, 0.0, 5.0)):
        v[i::97] = W.f32_to_bf16_bits(np.full(len(v[i::97]), far, np.float32))
    c.open()
    c.check_scan(c.run_scan(z=c.z), z=c.z)
    c.close()


@pytest.mark.gpu
def test_nan_stays_in_its_channel_and_sequence():
    c = Case(500, 64, 16, 4, [40, 1, 33], [41, 5, 33])
    c.x[5, 7] = c.dt[20, 11] = c.z[30, 3] = NAN
    c.dt[40, 2] = W.f32_to_bf16_bits(np.array([np.inf], np.float32))[0]
    c.open()
    with np.errstate(invalid="ignore"):
        c.check_scan(c.run_scan(**c.all_scan()), piece=64, **c.all_scan())
    out = c.blank()
    ap.conv_iteration(c.pool, c.plan, dev(c.x), dev(c.weight), out)
    with np.errstate(invalid="ignore"):
        got = f64(host(out)[:c.n])
    seen = np.isnan(got)
    assert seen[5:9, 7].all() and seen.sum() == 4
    c.close()


@pytest.mark.gpu
def test_strided_rows_and_larger_tensors():
    c = Case(600, 136, 16, 4, [50, 1, 1, 21], [50, 9, 1, 40]).open()
    import torch
    xz = dev(np.concatenate([c.x, c.z], 1))
    proj = dev(np.concatenate([np.full((c.rows, 24), NAN, np.uint16), c.b, c.c], 1))
    both = dev(np.full((c.rows, 2 * c.channels), NAN, np.uint16))
    ap.conv_iteration(c.pool, c.plan, xz[:, :c.channels], dev(c.weight), both[:, :c.channels], bias=dev(c.bias))
    c.check_conv(both[:, :c.channels].contiguous())
    assert (host(both[:, c.channels:]) == NAN).all()
    ap.scan_iteration(c.pool, c.plan, xz[:, :136], dev(c.dt), dev(c.a), proj[:, 24:40], proj[:, 40:], both[:, 136:], z=xz[:, 136:],
                      d_skip=dev(c.skip), dt_bias=dev(c.dt_bias), workspace=c.workspace())
    c.check_scan(both[:, 136:].contiguous(), piece=64, **c.all_scan())
    # what would overwrite an input or a slot is refused; slices that lie between one another are not
    for bad in (dict(x=xz[:, :136], out=xz[:, 136:], z=xz[:, 136:]), dict(x=xz[:, :136], out=xz[:, 8:144]),
                dict(x=xz[:, 136:], out=xz[1:, 136:])):
        kw = dict(dt=dev(c.dt), a=dev(c.a), b=proj[:, 24:40], c=proj[:, 40:], workspace=c.workspace())
        with pytest.raises(ap.ApError) as e:
            ap.scan_iteration(c.pool, c.plan, **kw, **bad)
        assert e.value.status == B.AP_ERR_INVALID_ARG
    ap.scan_iteration(c.pool, c.plan, xz[:, :136], dev(c.dt), dev(c.a), proj[:, 24:40], proj[:, 40:], xz[:, 136:], workspace=c.workspace())
    with pytest.raises(ap.ApError):
        ap.conv_iteration(c.pool, c.plan, dev(c.x), dev(c.weight), ap.state_pool_conv_base(c.pool))
    with pytest.raises(ap.ApError):
        ap.conv_iteration(c.pool, c.plan, ap.state_pool_conv_base(c.pool), dev(c.weight), c.blank())
    for name in ("x", "dt", "b"):
        kw = dict(x=dev(c.x), dt=dev(c.dt), b=proj[:, 24:40])
        kw[name] = ap.state_pool_scan_base(c.pool)
        with pytest.raises(ap.ApError):
            ap.scan_iteration(c.pool, c.plan, a=dev(c.a), c=proj[:, 40:], out=c.blank(), workspace=c.workspace(), **kw)
    torch.cuda.synchronize()
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("states", [16, 64])
def test_iterations_that_follow_one_another(states):
    """A prompt in one piece, and as chunks and single tokens over several iterations of two layers that share plans: the
    same states and rows within the bounds, whatever the cuts."""
    n, ch = 421, 72
    whole = Case(700 + states, ch, states, 4, [n], [n], extra_rows=0, slots=[1]).open()
    ref, slack, state, off = R.scan(f64(whole.x), f64(whole.dt), whole.a.astype(np.float64), f64(whole.b), f64(whole.c),
                                    np.zeros(whole.state.shape), [n], [n], [1], piece=n)
    y, y_slack, conv = R.conv(f64(whole.x), f64(whole.weight), None, np.zeros(whole.conv.shape), [n], [n], [1], False)
    second = ap.state_pool_create(whole.num_slots, ch, states, 4)
    out, out2, conv_out = whole.blank(), whole.blank(), whole.blank()
    x, dt, a, b, c = (dev(t) for t in (whole.x, whole.dt, whole.a, whole.b, whole.c))
    at = 0
    for m in (1, 2, 150, 1, 3, 200, 64):
        plan = ap.state_plan_create(whole.pool, [m, 0], [at + m, 0], [1, 0])
        rows = slice(at, at + m)
        import torch
        ws = torch.empty(max(256, ap.state_plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda")
        for pool, o in ((whole.pool, out), (second, out2)):
            ap.scan_iteration(pool, plan, x[rows], dt[rows], a, b[rows], c[rows], o[rows], workspace=ws)
        ap.conv_iteration(whole.pool, plan, x[rows], dev(whole.weight), conv_out[rows], silu=False)
        torch.cuda.synchronize()
        ap.state_plan_destroy(plan)
        at += m
    assert at == n
    for o in (out, out2):
        R.bf16_close(f64(host(o)), ref, slack, "out")
    R.bf16_close(f64(host(conv_out)), y, y_slack, "conv")
    R.fp32_close(host(whole.d_state)[1].astype(np.float64), state[1], off[1], "state")
    assert np.array_equal(f64(host(whole.d_conv)[1]), conv[1])
    ap.state_pool_destroy(second)
    whole.close()


@pytest.mark.gpu
def test_a_layer_with_one_plane():
    import torch
    x = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda")
    w, a, b = (torch.zeros(64, 4, dtype=torch.bfloat16, device="cuda"), torch.zeros(64, 8, device="cuda"),
               torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda"))
    for planes, works in ((dict(conv_base=torch.zeros(3, 3, 64, dtype=torch.bfloat16, device="cuda")), "conv"),
                          (dict(scan_base=torch.zeros(3, 64, 8, device="cuda")), "scan")):
        pool = ap.state_pool_create(3, 64, 8, 4, **planes)
        plan = ap.state_plan_create(pool, [2], [2], [1])
        for name, call in (("conv", lambda: ap.conv_iteration(pool, plan, x, w, torch.empty_like(x))),
                           ("scan", lambda: ap.scan_iteration(pool, plan, x, x, a, b, b, torch.empty_like(x)))):
            if name == works:
                call()
            else:
                with pytest.raises(ap.ApError) as e:
                    call()
                assert e.value.status == B.AP_ERR_INVALID_ARG
        torch.cuda.synchronize()
        ap.state_plan_destroy(plan)
        ap.state_pool_destroy(pool)


@pytest.mark.gpu
def test_captured_replayed_and_on_another_stream():
    import torch
    c = Case(800, 64, 16, 4, [300, 1, 40], [300, 4, 40]).open()
    x, dt, a, b, cc, w = (dev(t) for t in (c.x, c.dt, c.a, c.b, c.c, c.weight))
    ws, out, mid = c.workspace(), c.blank(), c.blank()

    def layer():
        ap.conv_iteration(c.pool, c.plan, x, w, mid)
        ap.scan_iteration(c.pool, c.plan, mid, dt, a, b, cc, out, workspace=ws)
    layer()
    torch.cuda.synchronize()
    first = host(out), host(c.d_state), host(c.d_conv)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        layer()
    for _ in range(2):
        c.d_conv.copy_(dev(c.conv))
        c.d_state.copy_(dev(c.state))
        out.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        # (the scan's sums have one order: the same bits)
        assert np.array_equal(host(out)[:c.n], first[0][:c.n])
        assert np.array_equal(host(c.d_state).view(np.int32), first[1].view(np.int32)) and np.array_equal(host(c.d_conv), first[2])
    c.d_conv.copy_(dev(c.conv))
    c.d_state.copy_(dev(c.state))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        layer()
    side.synchronize()
    assert np.array_equal(host(out)[:c.n], first[0][:c.n])
    c.close()


@pytest.mark.gpu
def test_what_overlaps_is_refused_and_nothing_written():
    import torch
    c = Case(810, 64, 16, 4, [400], [400]).open()
    need = ap.state_plan_workspace_bytes(c.plan)
    assert need > 0
    x, dt, a, b, cc, out = dev(c.x), dev(c.dt), dev(c.a), dev(c.b), dev(c.c), c.blank()
    big = torch.full((need + c.state.nbytes + x.nbytes + 512,), 0x7F, dtype=torch.uint8, device="cuda")
    base = -big.data_ptr() % 256
    inside = big[base:base + c.state.nbytes].view(torch.float32).view(c.state.shape)
    pool = ap.state_pool_create(c.num_slots, 64, 16, 4, scan_base=inside)
    start = (c.num_slots - 1) * 64 * 16 * 4 // 256 * 256                                   # (the workspace begins in the last slot)
    good = dict(x=x, dt=dt, a=a, b=b, c=cc, out=out, workspace=c.workspace())

    def refused(pool, **kw):
        with pytest.raises(ap.ApError) as e:
            ap.scan_iteration(pool, c.plan, **{**good, **kw})
        assert e.value.status == B.AP_ERR_INVALID_ARG, list(kw)
    refused(pool, workspace=big[base + start:base + start + need])
    refused(c.pool, out=x)
    over = big[base:base + x.nbytes].view(torch.bfloat16).view(c.rows, 64)                # (its first rows lie in the slots)
    refused(pool, x=over)
    refused(pool, out=over)
    refused(c.pool, b=good["workspace"].view(torch.bfloat16)[:16 * c.rows].view(c.rows, 16))
    with pytest.raises(ap.ApError):
        ap.conv_iteration(c.pool, c.plan, x, dev(c.weight), x)
    torch.cuda.synchronize()
    assert (big == 0x7F).all() and (host(out) == NAN).all()
    assert np.array_equal(host(c.d_state).view(np.int32), c.state.view(np.int32)) and np.array_equal(host(c.d_conv), c.conv)
    ap.state_pool_destroy(pool)
    c.close()


@pytest.mark.gpu
def test_one_plan_for_two_layers_at_once():
    """Two layers' calls on two streams, one plan: each its slots, its workspace, its result; then as two graphs."""
    import torch
    lens, ctx = [500, 1, 33, 200], [500, 7, 40, 200]
    one, two = Case(820, 64, 16, 4, lens, ctx).open(), Case(821, 64, 16, 4, lens, ctx)
    two.slots = one.slots
    rng = np.random.default_rng(822)
    two.conv, two.state, two.live, two.touched = bits(rng, *one.conv.shape), one.state[::-1].copy(), one.live, one.touched
    two.conv[~two.live], two.state[~two.live] = NAN, np.nan
    two.state[two.live] = rng.standard_normal(two.state[two.live].shape).astype(np.float32)
    two.d_conv, two.d_state = dev(two.conv), dev(two.state)
    two.pool = ap.state_pool_create(two.num_slots, 64, 16, 4, two.d_conv, two.d_state)
    two.plan = one.plan
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = [[dev(t) for t in (c.x, c.dt, c.a, c.b, c.c)] for c in (one, two)]
    space, outs = [c.workspace() for c in (one, two)], [c.blank() for c in (one, two)]
    torch.cuda.synchronize()

    def call(i):
        c = (one, two)[i]
        ap.scan_iteration(c.pool, c.plan, *args[i], outs[i], workspace=space[i])
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            call(i)
    torch.cuda.synchronize()
    for c, out in zip((one, two), outs):
        c.check_scan(out, piece=64)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i in range(2):
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            call(i)
    first = [host(o) for o in outs]
    for c, out in zip((one, two), outs):
        c.d_state.copy_(dev(c.state))
        out.fill_(0)
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert np.array_equal(host(outs[i])[:one.n], first[i][:one.n])
    ap.state_pool_destroy(two.pool)
    one.close()


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Rows 2^26 elements apart, and slots whose states begin past 2^31 elements."""
    import torch
    c = Case(830, 64, 64, 4, [37, 1], [37, 5], extra_rows=0)
    wide = torch.empty((c.rows, 1 << 26), dtype=torch.bfloat16, device="cuda")
    cols = {}
    for i, name in enumerate(("x", "dt", "z", "b", "c")):
        cols[name] = wide[:, (1 << 26) - 512 + 64 * i:(1 << 26) - 512 + 64 * (i + 1)]
        cols[name].copy_(dev(getattr(c, name)))
    slots, far = (1 << 19) + 8, 1 << 19
    small_state, small_conv = dev(c.state), dev(c.conv)
    big_state = torch.empty((slots, 64, 64), device="cuda")
    big_conv = torch.empty((slots, 3, 64), dtype=torch.bfloat16, device="cuda")
    assert c.num_slots <= 8
    big_state[far:far + c.num_slots].copy_(small_state)
    big_conv[far:far + c.num_slots].copy_(small_conv)
    c.d_state, c.d_conv = big_state[far:far + c.num_slots], big_conv[far:far + c.num_slots]
    pool = ap.state_pool_create(slots, 64, 64, 4, big_conv, big_state)
    plan = ap.state_plan_create(pool, c.q_lens, c.ctx_lens, c.slots + far)
    ws = torch.empty(max(256, ap.state_plan_workspace_bytes(plan)), dtype=torch.uint8, device="cuda")
    for run, check in ((lambda o: ap.conv_iteration(pool, plan, cols["x"], dev(c.weight), o), lambda o: c.check_conv(o, bias=False)),
                       (lambda o: ap.scan_iteration(pool, plan, cols["x"], cols["dt"], dev(c.a), cols["b"], cols["c"], o, z=cols["z"],
                                                    workspace=ws), lambda o: c.check_scan(o, z=c.z))):
        out = wide[:, (1 << 26) - 128:(1 << 26) - 64]
        run(out)
        torch.cuda.synchronize()
        check(out)
    ap.state_plan_destroy(plan)
    ap.state_pool_destroy(pool)


@pytest.mark.gpu
def test_the_librarys_own_planes_begin_as_zeros_on_any_stream():
    import torch
    side = torch.cuda.Stream()
    x, w = torch.ones(1, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, 4, dtype=torch.bfloat16, device="cuda")
    a, b = torch.zeros(64, 16, device="cuda"), torch.ones(1, 16, dtype=torch.bfloat16, device="cuda")
    out, y = torch.empty_like(x), torch.empty_like(x)
    torch.cuda.synchronize()
    pool = ap.state_pool_create(20000, 64, 16, 4)
    with torch.cuda.stream(side):
        plan = ap.state_plan_create(pool, [1], [2], [19999])
        ap.conv_iteration(pool, plan, x, w, out, silu=False)
        ap.scan_iteration(pool, plan, x, x, a, b, b, y, softplus=False)
    side.synchronize()
    assert (out == 1).all() and (y == 16).all()                     # 0 0 0 1 convolved with ones; 16 states of 1 * 1
    ap.state_plan_destroy(plan)
    ap.state_pool_destroy(pool)
