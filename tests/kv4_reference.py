"""The 4-bit page format in numpy, written from its description in ap_serving.h (float64; shares no code with the
library).  bf16 tensors are uint16 bit patterns.  Test infrastructure only."""
import numpy as np

from paper_2604_07144_b200 import workloads as W

PAGE, GROUP = 16, 32


def tile_bytes(d):
    return PAGE * (d // 2 + d // 16)


def quantise(bits):
    """bf16 bits [..., d] -> (codes uint8 [..., d], steps bf16 bits [..., d / 32])."""
    x = W.bf16_bits_to_f64(bits).reshape(*bits.shape[:-1], bits.shape[-1] // GROUP, GROUP)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(-1)
        bad = ~(top < 2.0 ** 120)
        top = np.where(bad, 0.0, top)
        q = top / 7.0
        # five significant bits, but no finer than fp32's 2^-149 allows at bit 19: 2^-130
        unit = np.where(q > 0, 2.0 ** np.maximum(np.floor(np.log2(np.where(q > 0, q, 1.0))) - 4, -130.0), 1.0)
        step = np.ceil(q / unit) * unit
        codes = np.where(step[..., None] > 0, np.rint(x / np.where(step > 0, step, 1.0)[..., None]), 0.0)
    codes = np.where(bad[..., None], 0.0, codes) + 8
    step = np.where(bad, np.nan, step)
    return codes.astype(np.uint8).reshape(bits.shape), np.where(bad, np.uint16(0x7FC0), W.f32_to_bf16_bits(step))


def pack(codes):
    """codes [..., d] -> the d / 2 bytes of a stored row."""
    d = codes.shape[-1]
    out = np.zeros((*codes.shape[:-1], d // 2), np.uint8)
    for g in range(d // GROUP):
        for t in range(4):
            word = t * (d // GROUP) + g
            for e in range(8):
                out[..., 4 * word + e // 2] |= (codes[..., 32 * g + 8 * t + e] << (4 * (e % 2))).astype(np.uint8)
    return out


def unpack(rows):
    d = rows.shape[-1] * 2
    codes = np.zeros((*rows.shape[:-1], d), np.uint8)
    for g in range(d // GROUP):
        for t in range(4):
            word = t * (d // GROUP) + g
            for e in range(8):
                codes[..., 32 * g + 8 * t + e] = (rows[..., 4 * word + e // 2] >> (4 * (e % 2))) & 15
    return codes


def put(plane, page, slot, bits):
    """Writes rows bits [n, Hkv, d] to (page[i], slot[i]) of a 4-bit plane [pages, Hkv, tile bytes]."""
    d = bits.shape[-1]
    codes, steps = quantise(bits)
    rows, steps = pack(codes), np.ascontiguousarray(steps).view(np.uint8)
    for i in range(len(page)):
        plane[page[i], :, slot[i] * (d // 2):(slot[i] + 1) * (d // 2)] = rows[i]
        at = PAGE * d // 2 + slot[i] * (d // 16)
        plane[page[i], :, at:at + d // 16] = steps[i]


def values(plane, d):
    """float64 [pages, Hkv, 16, d]: what the plane stands for."""
    codes = unpack(plane[..., :PAGE * d // 2].reshape(*plane.shape[:2], PAGE, d // 2))
    steps = np.ascontiguousarray(plane[..., PAGE * d // 2:]).view(np.uint16).reshape(*plane.shape[:2], PAGE, d // GROUP)
    steps = W.bf16_bits_to_f64(steps)
    return ((codes.astype(np.float64) - 8).reshape(*codes.shape[:-1], -1, GROUP) * steps[..., None]).reshape(codes.shape)


def empty_plane(num_pages, hkv, d, seed):
    """A plane that holds no token: arbitrary codes, NaN steps."""
    plane = np.random.default_rng(seed).integers(0, 256, (num_pages, hkv, tile_bytes(d)), dtype=np.uint8)
    steps = np.full((num_pages, hkv, PAGE * d // GROUP), W.CANARY, np.uint16)
    plane[..., PAGE * d // 2:] = steps.view(np.uint8).reshape(num_pages, hkv, -1)
    return plane


def new_slots(batch):
    """(page, slot) of every new token row."""
    page, slot = [], []
    for s in range(batch.batch):
        for p in range(int(batch.ctx_lens[s]) - int(batch.q_lens[s]), int(batch.ctx_lens[s])):
            page.append(int(batch.block_tables[s, p // PAGE]))
            slot.append(p % PAGE)
    return np.array(page, np.int64), np.array(slot, np.int64)


def planes_of(batch, seed=5):
    """4-bit planes holding a batch's cached tokens (the bf16 pool's, quantised), NaN steps everywhere else."""
    out = []
    for i, pool in enumerate((batch.k_pool, batch.v_pool)):
        plane = empty_plane(batch.num_pages, batch.num_kv_heads, batch.head_dim, seed + i)
        held = (pool != W.CANARY).any(-1).all(1)                       # [pages, 16]
        page, slot = np.nonzero(held)
        put(plane, page, slot, pool[page, :, slot])
        out.append(plane)
    return out
