"""Helpers of the quantised-cache tests: rows with the values that a format treats differently, layouts, tolerances."""
import numpy as np
import torch

import oracle as O
import paper_2606_00144_amd as bd
import synth
from gpu_utils import bf16_host64


def bits_of(x):
    """bf16 bits of a float array whose values are exact or to be rounded (NaN and infinities allowed)."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.view(torch.int16).numpy().view(np.uint16)


def rows(shape, seed, scale=1.0):
    g = np.random.default_rng(seed)
    ch = np.exp(0.5 * g.standard_normal(shape[-1]))
    return synth.f32_to_bf16_bits((scale * ch * g.standard_normal(shape)).astype(np.float32))


def special_rows(n, seed):
    """Rows [n][128] whose blocks hold the borders: zeros, ties of the grid, maxima around the exponent's step,
    subnormals, the largest bf16, infinities and NaN."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((n, 4, 32)).astype(np.float32)
    tie = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 3.0], np.float32)
    for r in range(n):
        for b in range(4):
            kind = int(g.integers(0, 10))
            if kind == 0:
                x[r, b] = 0.0
            elif kind == 1:
                x[r, b] = np.float32(2.0) ** int(g.integers(-20, 20)) * g.choice(tie, 32) * g.choice([-1, 1], 32)
            elif kind == 2:                                  # the maximum on, just below and just above a step
                top = g.choice([1.75, 1.765625, 1.7421875, 1.8125, 1.8203125, 1.8046875, 1.0, 1.9921875])
                x[r, b] = np.clip(x[r, b], -1, 1)
                x[r, b, g.integers(0, 32)] = top * 2.0 ** int(g.integers(-10, 10))
            elif kind == 3:
                x[r, b] *= np.float32(2.0) ** -125
            elif kind == 4:
                x[r, b] = g.choice([-1, 1], 32) * 2.0 ** g.integers(-133, -120, 32)
            elif kind == 5:
                x[r, b, 0] = 3.3895314e38 * g.choice([-1, 1])
                x[r, b, 1:] *= 1e37
            elif kind == 6:
                x[r, b, g.integers(0, 32)] = g.choice([np.inf, -np.inf, np.nan])
            elif kind == 7:
                x[r, b] = g.choice([-0.0, 0.0, 1.0], 32)
    return bits_of(x.reshape(n, 128))


def values_as_bits(codes, scales, bits):
    """bf16 bits of finite cache values (exact)."""
    return synth.f32_to_bf16_bits(O.mx_values(codes, scales, bits).astype(np.float32))


def to_dev(cache):
    return bd.QuantKV(*[torch.from_numpy(np.ascontiguousarray(b)).cuda() for b in cache])


def to_host(cache):
    return tuple(b.cpu().numpy() for b in cache)


def garbage(shape, seed):
    """Bytes of memory never written: any code, any scale, not-a-numbers among them."""
    g = np.random.default_rng(seed)
    b = g.integers(0, 256, size=shape, dtype=np.uint8)
    b[..., ::3] = 255
    return b


def make_cache(S, Hkv, cap, bits, lens, seed, k_scale=1.0):
    """A cache [S][Hkv][cap] of quantised rows below lens and garbage above, and its values as bf16 bits (K, V)."""
    cache = [garbage((S, Hkv, cap, w), seed + i) for i, w in enumerate((16 * bits, 16 * bits, 4, 4))]
    vals = []
    for which, sc in ((0, k_scale), (1, 1.0)):
        c, s = O.mx_quantise(rows((S, Hkv, cap, 128), seed + 10 + which, sc), bits)
        for i, L in enumerate(lens):
            cache[which][i, :, :L], cache[which + 2][i, :, :L] = c[i, :, :L], s[i, :, :L]
        vals.append(values_as_bits(c, s, bits))
    return tuple(cache), vals[0], vals[1]


def to_pages(cache, lens, page, seed, extra=3):
    """The cache's rows in a pool of pages under a random table (unused entries -1): (pool, table)."""
    S, Hkv, cap = cache[0].shape[:3]
    width = (cap + page - 1) // page
    need = [(int(L) + page - 1) // page for L in lens]
    total = sum(need) + extra
    perm = np.random.default_rng(seed).permutation(total).astype(np.int32)
    table, at = np.full((S, width), -1, np.int32), 0
    pool = [garbage((total, Hkv, page, b.shape[3]), seed + 1 + i) for i, b in enumerate(cache)]
    for s, m in enumerate(need):
        table[s, :m] = perm[at:at + m]
        at += m
        for j in range(m):
            n = min(page, int(lens[s]) - j * page)
            for b, src in zip(pool, cache):
                b[table[s, j], :, :n] = src[s, :, j * page:j * page + n]
    return tuple(pool), table


def check_out(out, lse, ro, rl, k, v, q, attend, n, what):
    """Outputs against the oracle's, by arithmetic.

    The weights are rounded to bf16 (2^-8 at most, torch's eps / 2) and normalised by their own sum, so an output
    moves by at most 2^-8 (A + |o|) with A = sum p |v|; its own rounding adds 2^-8 |o|.  fp32 rounding of the scores
    (128 products: 130 * 2^-24 of X = max sum |q k| scale) moves a weight by that much, relatively.  The
    log-sum-exp moves by the scores' error, by the sum of n weights (at most n / 16 additions in a row) and by its
    own few roundings.  `attend(q, k, v)`: the oracle with these tensors (for A).
    """
    A = attend(q, k, v & np.uint16(0x7FFF))[0]
    absq, absk = O.bf16_to_f64(q), O.bf16_to_f64(k)
    X = np.abs(absq).max() * np.abs(absk).sum(-1).max() / np.sqrt(128.0)       # an upper bound of every row's
    fp32 = 130 * 2.0 ** -24 * X
    got = bf16_host64(out)
    tol = 2.0 ** -8 * (A + 2 * np.abs(ro)) + 2 * fp32 * A + 1e-30
    err = np.abs(got - ro)
    assert got.shape == ro.shape, what
    assert (err <= tol).all(), f"{what}: worst {np.nanmax(err - tol)} past its bound, {int((~(err <= tol)).sum())} of {err.size}"
    if lse is not None:
        gl = lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isneginf(gl), np.isneginf(rl)) and not np.isnan(gl).any(), what
        fin = ~np.isneginf(rl)
        tl = fp32 + (n / 16 + 64) * 2.0 ** -24 + 8 * 2.0 ** -24 * np.abs(rl[fin])
        d = np.abs(gl[fin] - rl[fin])
        assert (d <= tl).all(), f"{what}: log-sum-exp off by {d.max()}"
