"""Plain 64-bit references and a device harness for windowed attention, the rotated append and the 4-bit cache.
Test infrastructure only; shares no code with the library."""
import numpy as np

import paper_2604_07144_b200 as ap
from paper_2604_07144_b200 import workloads as W

from harness import to_bits, to_dev

PAGE = 16


def visible(n_new, ctx, window=None, sinks=0):
    """[n_new, ctx] truth table: which keys the new tokens (the last n_new of ctx) see."""
    p = np.arange(ctx - n_new, ctx)[:, None]
    j = np.arange(ctx)[None]
    if window is None:
        return j <= p
    return (j <= p) & ((j > p - window) | (j < sinks))


def attention(k_rows, v_rows, batch, window=None, sinks=0, scale=None):
    """(out, lse, abs_weighted) in float64.  k_rows(s), v_rows(s): [ctx, Hkv, d] of sequence s; rows that no
    new token sees may hold anything.  abs_weighted = sum_j p_j |v_j|, for the rounding bound of the weights."""
    hq, hkv, d = batch.num_q_heads, batch.num_kv_heads, batch.head_dim
    scale = scale or 1.0 / np.sqrt(d)
    q = W.bf16_bits_to_f64(batch.q)
    out, lse = np.zeros((batch.n_new, hq, d)), np.zeros((batch.n_new, hq))
    absw = np.zeros_like(out)
    row = 0
    for s in range(batch.batch):
        n, ctx = int(batch.q_lens[s]), int(batch.ctx_lens[s])
        if n == 0:
            continue
        see = visible(n, ctx, window, sinks)
        kept = see.any(0)
        see, k, v = see[:, kept], k_rows(s)[kept], v_rows(s)[kept]
        for h in range(hq):
            x = scale * (q[row:row + n, h] @ k[:, h // (hq // hkv)].T)
            x = np.where(see, x, -np.inf)
            m = x.max(1, keepdims=True)
            e = np.exp(x - m)
            l = e.sum(1, keepdims=True)
            vh = v[:, h // (hq // hkv)]
            out[row:row + n, h] = (e / l) @ vh
            absw[row:row + n, h] = (e / l) @ np.abs(vh)
            lse[row:row + n, h] = (m + np.log(l))[:, 0]
        row += n
    return out, lse, absw


def table_rows(batch, plane_f64, s):
    """[ctx, Hkv, d] of sequence s gathered from a [pages, Hkv, 16, d] plane (entries of -1 give NaN rows)."""
    ctx = int(batch.ctx_lens[s])
    pages = batch.block_tables[s, :(ctx + PAGE - 1) // PAGE]
    rows = plane_f64[np.maximum(pages, 0)]                       # [n, Hkv, 16, d]
    rows = np.where((pages < 0)[:, None, None, None], np.nan, rows)
    return rows.transpose(0, 2, 1, 3).reshape(-1, batch.num_kv_heads, batch.head_dim)[:ctx]


def check(out_bits, lse, ref, what=""):
    """Per element: |out - ref| <= 2^-8 A + half an ulp of bf16 at ref + 2e-4 A + 1e-6, A = sum_j p_j |v_j|: a weight is
    rounded to bf16 once (2^-8 of it), the result once, and 2e-4 covers the exponential (the cubic on the FMA pipe is
    off by at most 7.7e-5 of a weight, and by as much again through the sum), ex2.approx (2^-22), scores and sums in
    fp32.  lse: 7.7e-5 of the sum, scores with d products of at most 2^-24 each relative to sum |q k| scale (below
    1e-4 for N(0,1) rows at d <= 128)."""
    ref_out, ref_lse, absw = ref
    got = W.bf16_bits_to_f64(out_bits)
    assert np.isfinite(got).all() and np.isfinite(lse).all(), f"{what}: non-finite output"
    a = np.abs(ref_out)
    half_ulp = np.where(a > 0, 2.0 ** (np.floor(np.log2(np.maximum(a, 1e-300))) - 8), 0.0)
    excess = np.abs(got - ref_out) - (absw * (2.0 ** -8 + 2e-4) + half_ulp + 1e-6)
    i = np.unravel_index(np.argmax(excess), excess.shape)
    assert excess[i] <= 0, f"{what}: {got[i]} against {ref_out[i]} at {i} (A {absw[i]})"
    lerr = np.abs(lse - ref_lse)
    assert (lerr <= 2e-4 + 1e-5 * np.abs(ref_lse)).all(), f"{what}: lse off by {lerr.max()}"


class Device:
    """Pool, plan and tensors of a batch on the GPU; `plan` (a function of the pool) may make a plan of its own."""

    def __init__(self, batch, make_plan=None, side_by_side=None, single_launch=None, k_plane=None, v_plane=None,
                 four_bit=False):
        import torch
        self.batch, dev = batch, "cuda:0"
        if four_bit:
            self.k_pool, self.v_pool = torch.from_numpy(k_plane).to(dev), torch.from_numpy(v_plane).to(dev)
            self.pool = ap.kv_pool_create_4bit(batch.num_pages, batch.num_kv_heads, batch.head_dim, self.k_pool, self.v_pool)
        else:
            self.k_pool = to_dev(batch.k_pool if k_plane is None else k_plane)
            self.v_pool = to_dev(batch.v_pool if v_plane is None else v_plane)
            self.pool = ap.kv_pool_create(batch.num_pages, batch.num_kv_heads, batch.head_dim, self.k_pool, self.v_pool)
        self.q, self.k_new, self.v_new = to_dev(batch.q), to_dev(batch.k_new), to_dev(batch.v_new)
        n = batch.n_new
        # one row more than the call writes: it has to stay as it is
        self.out = torch.full((n + 1, batch.num_q_heads, batch.head_dim), float("nan"), dtype=torch.bfloat16, device=dev)
        self.lse = torch.full((n + 1, batch.num_q_heads), float("nan"), dtype=torch.float32, device=dev)
        if side_by_side is not None:
            ap.kv_pool_set_side_by_side(self.pool, side_by_side)
        if single_launch is not None:
            ap.kv_pool_set_single_launch(self.pool, single_launch)
        make_plan = make_plan or (lambda pool: ap.plan_create(pool, batch.q_lens, batch.ctx_lens, batch.block_tables,
                                                              batch.num_q_heads))
        self.plan = make_plan(self.pool)
        self.info = ap.plan_get_info(self.plan)
        nbytes = ap.plan_workspace_bytes(self.plan)
        # poisoned, and with a guard behind the size the plan asks for
        self.workspace = torch.full((max(nbytes, 256) + 256,), 0xFF, dtype=torch.uint8, device=dev)
        self.workspace_bytes = nbytes

    def attend(self):
        ap.attention_iteration(self.pool, self.plan, self.q, self.out, self.lse, self.workspace, self.workspace_bytes)

    def results(self):
        """(out bits, lse) of the batch's rows, after checking the status, the row behind them and the workspace's guard."""
        assert ap.last_device_status(self.pool) == 0
        n = self.batch.n_new
        assert np.isnan(self.lse[n].cpu().numpy()).all() and (to_bits(self.out[n]) == to_bits(self.out[n])[0, 0]).all()
        assert (self.workspace[max(self.workspace_bytes, 256):] == 0xFF).all()
        return to_bits(self.out)[:n], self.lse.cpu().numpy()[:n]

    def close(self):
        import torch
        torch.cuda.synchronize()
        ap.plan_destroy(self.plan)
        ap.kv_pool_destroy(self.pool)
