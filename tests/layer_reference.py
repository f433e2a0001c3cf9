"""The operators of hybrid layers by their definitions in 64 bits, each with a bound on what fp32 arithmetic may add before
the last rounding.  Sequence by sequence and token by token; nothing here is shared with the library."""
import math

import numpy as np

U = 2.0 ** -24                      # half a step of fp32, relative
EX2 = 2.0 ** -22                    # ex2.approx, relative (two steps of fp32)


def half_step(x, eps):
    """Half a step of a floating type with machine epsilon `eps` at x, for results that may round up a binade."""
    a = np.abs(x)
    return np.where(a > 0, 2.0 ** np.floor(np.log2(np.maximum(a * (1 + eps), 1e-300))) * eps / 2, 0.0)


LARGEST = 3.38e38                   # below the largest number of bf16 and of fp32


def _close(got, ref, slack, eps, what):
    """Results beyond LARGEST have no number to be compared with: fp32 and bf16 end there, and infinity is what they round to.
    (slack is infinite where something on the way was.)"""
    with np.errstate(invalid="ignore", over="ignore"):
        in_range = ~np.isposinf(slack) & ~(np.abs(ref) + slack > LARGEST)
        assert np.array_equal(np.isnan(got) & in_range, np.isnan(ref) & in_range), f"{what}: NaN in other places"
        skip = ~in_range | np.isnan(ref) | (got == ref)
        excess = np.where(skip, 0, np.abs(got - ref) - slack - half_step(np.where(skip, 0, np.abs(ref) + slack), eps))
    at = np.unravel_index(np.argmax(excess), excess.shape) if excess.size else ()
    assert not excess.size or excess[at] <= 0, f"{what}: {got[at]} against {ref[at]} (slack {slack[at]}) at {at}"


def bf16_close(got, ref, slack, what=""):
    """|got - ref| within half a step of bf16 and `slack`, element by element; NaN where ref is NaN."""
    _close(got, ref, slack, 2.0 ** -7, what)


def fp32_close(got, ref, slack, what=""):
    _close(got, ref, slack, 2.0 ** -23, what)


def gated(y, slack, z):
    """y z / (1 + e^-z), and its bound: e^-z is off by EX2 and by the rounding of its argument, then three roundings and a
    division good to two steps."""
    s = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
    g = z * s
    with np.errstate(invalid="ignore", over="ignore"):
        return y * g, np.where(np.isposinf(slack), np.inf, np.abs(g) * slack) + np.abs(y * g) * (EX2 + 2 * np.abs(z) * 1.4427 * U + 8 * U)


def conv(x, weight, bias, state, q_lens, ctx_lens, slots, silu):
    """(out, slack, state): x [n, c], weight [c, w], state [slots, w - 1, c] in float64."""
    n, c = x.shape
    w = weight.shape[1]
    out, slack, state = np.zeros((n, c)), np.zeros((n, c)), state.copy()
    row = 0
    for ql, cl, slot in zip(q_lens, ctx_lens, slots):
        if ql == 0:
            continue
        seen = np.concatenate([state[slot] if cl > ql else np.zeros((w - 1, c)), x[row:row + ql]])
        for t in range(ql):
            terms = weight.T * seen[t:t + w]
            y = terms.sum(0) + (0 if bias is None else bias)
            big = np.abs(terms).sum(0) + (0 if bias is None else np.abs(bias))
            e = (w + 1) * U * big                                   # a product and a sum a tap
            if silu:
                s = 1 / (1 + np.exp(-y))
                # |d/dy (y s)| <= 1.1; the rest as in gated()
                y, e = y * s, 1.1 * e + np.abs(y * s) * (EX2 + 2 * np.abs(y) * 1.4427 * U + 8 * U)
            out[row + t], slack[row + t] = y, e
        state[slot] = seen[ql:]
        row += ql
    return out, slack, state


def scan(x, dt, a, b, c, state, q_lens, ctx_lens, slots, z=None, d_skip=None, dt_bias=None, softplus=True, piece=0):
    """(out, slack, state, state's slack).  `piece`: rows that a sequence cut along time may have in a piece (their steps are
    added up in fp32 there)."""
    n, ch = x.shape
    out, slack = np.zeros((n, ch)), np.zeros((n, ch))
    state, off = state.astype(np.float64).copy(), np.zeros(state.shape)
    row = 0
    for ql, cl, slot in zip(q_lens, ctx_lens, slots):
        if ql == 0:
            continue
        h = state[slot].copy() if cl > ql else np.zeros(state.shape[1:])
        size, err = np.abs(h), np.zeros_like(h)
        for t in range(row, row + ql):
            raw = dt[t] + (0 if dt_bias is None else dt_bias)
            if softplus:
                d = np.maximum(raw, 0) + np.log1p(np.exp(-np.abs(raw)))
                # the sum rounds once; u = e^-|raw| is off by EX2 and its argument's rounding; the polynomial by 2^-22.5
                e_d = 2 * U * np.abs(raw) + d * (EX2 + 2.0 ** -22 + 2 * U) + 3 * np.abs(raw) * U * d
            else:
                d = raw
                e_d = U * np.abs(raw)
            arg = d[:, None] * a
            decay = np.exp(arg)
            dx, e_dx = d * x[t], (e_d + U * np.abs(d)) * np.abs(x[t])
            new = dx[:, None] * b[t][None]
            # the decay: its argument is off by e_d a, by two roundings (three with log2 e's own) and, in a piece, by the
            # roundings of the sum; then EX2
            e_arg = e_d[:, None] * np.abs(a) + np.abs(arg) * (4 + piece) * U
            lost = np.isposinf(err) | (decay > LARGEST)          # fp32 ends there, and what comes after says nothing
            with np.errstate(over="ignore", invalid="ignore"):
                err = decay * err + decay * size * (e_arg + EX2) + e_dx[:, None] * np.abs(b[t])[None] + U * np.abs(new)
                size = decay * size + np.abs(new)
                h = decay * h + new
                err = np.where(lost | (size > LARGEST), np.inf, err + U * size)
                y = (h * c[t][None]).sum(1)
                e = (err * np.abs(c[t])[None]).sum(1) + (len(c[t]) + 2) * U * (size * np.abs(c[t])[None]).sum(1)
            e = np.where(np.isposinf(err).any(1), np.inf, e)
            if d_skip is not None:
                y, e = y + d_skip * x[t], e + 3 * U * np.abs(d_skip * x[t])
            if z is not None:
                y, e = gated(y, e, z[t])
            out[t], slack[t] = y, e
        # (a state that came through a piece's sum of decays: the same bound)
        state[slot], off[slot] = h, err
        row += ql
    return out, slack, state, off


def prompt(q, k, v, lens, scale=None):
    """(out, slack, lse, lse's slack): q [n, hq, d], k, v [n, hkv, d] in float64."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, slack = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, lse_slack = np.zeros((n, hq)), np.zeros((n, hq))
    row = 0
    for m in lens:
        at = slice(row, row + m)
        for h in range(hq if m else 0):
            qq, kk, vv = q[at, h], k[at, h // g], v[at, h // g]
            x = scale * (qq @ kk.T)
            size = scale * (np.abs(qq) @ np.abs(kk).T)
            hidden = np.arange(m)[None] > np.arange(m)[:, None]
            x[hidden] = -math.inf
            top = x.max(1, keepdims=True)
            p = np.exp(x - top)
            total = p.sum(1, keepdims=True)
            p /= total
            # a score: d products and sums in fp32, and its place relative to the maximum, in fp32; a weight's exponential:
            # 2^-18 covers the quartic's 2.7e-6; the weight itself goes into P V in bf16 (2^-8), sums in fp32
            e_x = np.where(hidden, 0, (d + 4) * U * size + 4 * U * (np.abs(np.where(hidden, 0, x)) + np.abs(top)))
            e_p = p * (2 * e_x + 2 * (p * e_x).sum(1, keepdims=True) + 2.0 ** -17)
            out[at, h] = p @ vv
            slack[at, h] = (p * 2.0 ** -8 + e_p) @ np.abs(vv) + m * U * (p @ np.abs(vv)) + 1e-30
            lse[at, h] = (top + np.log(total))[:, 0]
            lse_slack[at, h] = (p * e_x).sum(1) + 2.0 ** -17 + m * U + 4 * U * np.abs(lse[at, h])
        row += m
    return out, slack, lse, lse_slack
