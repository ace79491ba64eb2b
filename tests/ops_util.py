"""Plain 64-bit forms of the operators around the attention (numpy and torch on
the CPU, from the definitions in include/vdattn.h; no code of the library), and
the bounds their outputs are held to."""
from __future__ import annotations

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
G = 128  # values per scale
P = 16   # tokens per page
TINY = np.float32(2.0 ** -117)
PER_448 = np.float32(1.0) / np.float32(448.0)


def cpu64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bits(t):
    """The bit patterns of a tensor of 8-, 16-, 32- or 64-bit values."""
    w = {1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[t.element_size()]
    return t.detach().cpu().contiguous().view(w).numpy()


def same_bits(a, b, what=""):
    assert a.shape == b.shape, what
    assert np.array_equal(bits(a), bits(b)), what


# ---------------------------------------------------------------------------
# 8 bits
# ---------------------------------------------------------------------------
def codes_of(y32):
    """(codes, scales) of fp32 rows by the definition, operation for operation: each is one
    correctly rounded fp32 operation, so an equal y gives equal bits."""
    y32 = np.asarray(y32, np.float32)
    m, k = y32.shape
    kb = -(-k // G)
    z = np.zeros((m, kb * G), np.float32)
    z[:, :k] = y32
    z = z.reshape(m, kb, G)
    s = np.maximum(np.abs(z).max(-1), TINY) * PER_448  # (np.maximum carries a NaN)
    with np.errstate(all="ignore"):
        q = z * (np.float32(1.0) / s)[..., None]
    q = torch.from_numpy(q.reshape(m, kb * G)[:, :k].copy()).to(E4M3)
    return q, torch.from_numpy(s)


def values_of(codes, scales):
    """What 8-bit rows stand for, in 64 bits."""
    k = codes.shape[1]
    with np.errstate(invalid="ignore"):
        return cpu64(codes) * np.repeat(cpu64(scales), G, axis=1)[:, :k]


def check_codes(codes, scales, y, rel):
    """Codes and scales of rows y (64 bits) whose fp32 values are within ``rel`` of them.

    The scale is max |y| / 448 within rel + 2 2^-24 (the constant and the product), the
    ratio y / scale within 2 rel + 4 2^-24, its code half a step of e4m3 from it: 2^-4 of
    its magnitude, 2^-10 below the normal numbers (the least of which is 2^-6)."""
    m, k = y.shape
    kb = -(-k // G)
    z = np.zeros((m, kb * G))
    z[:, :k] = np.abs(y)
    top = np.maximum(z.reshape(m, kb, G).max(-1), float(TINY))
    s = cpu64(scales)
    assert s.shape == top.shape
    assert (np.abs(s * 448.0 - top) <= (rel + 4 * 2.0 ** -24) * top).all()
    err = np.abs(values_of(codes, scales) - y)
    far = 4 * rel + 8 * 2.0 ** -24
    bound = (2.0 ** -4 + far) * np.abs(y) + 2.0 ** -10 * np.repeat(s, G, axis=1)[:, :k] * (1 + far)
    assert (err <= bound).all(), "max excess %g" % float((err - bound).max())


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------
# y against 64 bits: at most 32 squares of a lane, 4 + 2 exchanges and 16 wavefronts are
# summed one after another, 54 roundings of 2^-24 on a sum of positive terms; with the mean
# and eps 56, halved by the root: 28; the root, the reciprocal and two products: 32 2^-24.
NORM_REL = 32 * 2.0 ** -24


def norm(x, w, eps, residual=None):
    """(h, y): the normed rows h as bf16 and y in 64 bits."""
    h = x.cpu()
    if residual is not None:
        h = (h.double() + residual.cpu().double()).to(torch.bfloat16)
    d = h.double().numpy()
    y = d / np.sqrt((d * d).mean(1, keepdims=True) + eps) * cpu64(w)
    return h, y


def check_bf16(got, ref, rel):
    """bf16 rows against 64 bits: half a step, 2^-8 of the magnitude (2^-134 below the
    normal numbers), after an fp32 value within rel of it."""
    err = np.abs(cpu64(got) - ref)
    bound = (2.0 ** -8 + 2 * rel) * np.abs(ref) + 2.0 ** -134
    assert (err <= bound).all(), "max excess %g" % float((err - bound).max())


# ---------------------------------------------------------------------------
# Gate: exp within 2 2^-23 (two units in the last place), the sum, the quotient and
# the product one rounding each: 4 + 3 roundings of 2^-24, doubled.
# ---------------------------------------------------------------------------
GATE_REL = 16 * 2.0 ** -24


def gated(x, gate):
    g, u = cpu64(gate), cpu64(x)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u


# ---------------------------------------------------------------------------
# Linear
#
# The matrix core adds a block's products in fp32, 8 neighbours of K at a time: of the 8,
# each is first cut (towards zero) to a multiple of 2^(E - 13), E the largest sum of the
# operands' exponents among the products that are not zero (an exponent is at least -6, that
# of e4m3's subnormal numbers).  Found by probing single products beside cancelling large
# ones; test_gpu_linear_fp8.py holds the probes.
# ---------------------------------------------------------------------------
def linear(a, a_scales, b, b_scales):
    """(c, magnitudes): the product in 64 bits, and of the absolute values."""
    n = b.shape[0]
    av = values_of(a, a_scales)
    bv = values_of(b, torch.from_numpy(np.repeat(cpu64(b_scales), G, axis=0)[:n]))
    return av @ bv.T, np.abs(av) @ np.abs(bv).T


def _exponents(v):
    e = np.frexp(v)[1] - 1
    return np.where(v == 0, -100, np.maximum(e, -6)).astype(np.int32)


def linear_cut(a, a_scales, b, b_scales):
    """The product with each 8 neighbours' products cut as the matrix core cuts them, the
    rest in 64 bits."""
    n, k = b.shape
    sa, sb = cpu64(a_scales), np.repeat(cpu64(b_scales), G, axis=0)[:n]
    av, bv = cpu64(a), cpu64(b)
    ea, eb = _exponents(av), _exponents(bv)
    out = np.zeros((a.shape[0], n))
    for i in range(a.shape[0]):
        p = (av[i] * bv).reshape(n, k // 8, 8)
        e = (ea[i] + eb).reshape(n, k // 8, 8).max(-1, keepdims=True)
        p = np.ldexp(np.trunc(np.ldexp(p, 13 - e)), e - 13).sum(-1)
        out[i] = (p * np.repeat(sa[i] * sb, G // 8, axis=1)[:, :k // 8]).sum(1)
    return out


def check_linear(got, x, rows=None):
    """Every output (of the given rows) within
      2^-8 |c| + 7 2^-13 mag + (32 + K / 128 + 4) 2^-24 mag + 2^-134 of 64 bits,
    and up to 24 rows and 160 columns within the same without the second term of the
    product with cut terms.  The output's rounding is half a bf16 step; of 8 products the
    largest is whole and the other 7 lose less than 2^(E - 13) each, the largest being at
    least 2^E unless subnormal (then the whole group is cut at 2^(E - 13) too, which the
    second check holds exactly); the 16 groups of a block are added in fp32 with at most
    2^-23 lost at each addition, the scales' product and the fused multiply-adds round once
    each."""
    a, a_s, b, b_s = (t.cpu() for t in x)
    rows = np.arange(a.shape[0]) if rows is None else np.asarray(rows)
    K, n = a.shape[1], b.shape[0]
    c, mag = linear(a[rows], a_s[rows], b, b_s)
    g = cpu64(got)[rows]
    assert np.isfinite(g).all()
    far = (32 + K // G + 5) * 2.0 ** -24 * mag + 2.0 ** -134
    r = np.unique(np.linspace(0, len(rows) - 1, 24).astype(int))
    q = np.unique(np.linspace(0, n - 1, 160).astype(int))
    bs = b_s[torch.from_numpy(q // G)].numpy()
    cut = np.stack([linear_cut(a[rows[r]], a_s[rows[r]], b[j:j + 1], torch.from_numpy(bs[i:i + 1]))[:, 0]
                    for i, j in enumerate(q)], 1)
    at = np.ix_(r, q)
    err = np.abs(g[at] - cut)
    bound = 2.0 ** -8 * np.abs(cut) + far[at]
    assert (err <= bound).all(), "max excess over the cut sums %g" % float((err - bound).max())
    normal = 7 * 2.0 ** -13 * mag + cut_of_subnormals(a[rows], a_s[rows], b, b_s)
    err = np.abs(g - c)
    bound = 2.0 ** -8 * np.abs(c) + (1 + 2.0 ** -8) * (far + normal)
    assert (err <= bound).all(), "max excess %g" % float((err - bound).max())


def cut_of_subnormals(a, a_scales, b, b_scales):
    """What groups whose largest product has a subnormal factor may lose besides: at most 8
    times 2^-13 of a product with that factor taken as 2^-6."""
    def lifted(t):
        v = np.abs(cpu64(t))
        return torch.from_numpy(np.where((v > 0) & (v < 2.0 ** -6), 2.0 ** -6, 0.0)), torch.from_numpy(np.maximum(v, 2.0 ** -6) * (v > 0))
    la, ua = lifted(a)
    lb, ub = lifted(b)
    return 8 * 2.0 ** -13 * (linear(la, a_scales, ub, b_scales)[0] + linear(ua, a_scales, lb, b_scales)[0])


# ---------------------------------------------------------------------------
# Page map
# ---------------------------------------------------------------------------
def page_map(q_lens, cached, free, table, num_pages, rows):
    """The outputs of vd_map_pages, one request and token after another."""
    q, c, free = [int(v) for v in q_lens], [int(v) for v in cached], [int(v) for v in free]
    table = np.array(table, np.int64)
    stride = table.shape[1] if table.ndim == 2 else 0
    cu, ctx, status, slots, used, dry = [0], [], [], np.full(rows, -1, np.int64), 0, False
    for r in range(len(q)):
        s, n = max(q[r], 0), c[r] + max(q[r], 0)
        start, end = cu[-1], cu[-1] + s
        cu.append(end)
        have, total = -(-c[r] // P), -(-n // P)
        st = (1 if q[r] < 0 or c[r] < 0 or n > 2 ** 31 - 1 else 0) | (2 if total > stride else 0)
        st |= 8 if end > rows else 0
        if st == 0 and total > have and (dry or used + total - have > len(free)):
            st, dry = 4, True
        status.append(st)
        ctx.append(n if st == 0 else 0)
        if st:
            continue
        for i in range(have, total):
            table[r, i] = free[used]
            used += 1
        for t in range(start, end):
            p = c[r] + t - start
            page = table[r, p // P]
            if 0 <= page < num_pages:
                slots[t] = page * P + p % P
    cu = np.minimum(np.array(cu, np.int64), 2 ** 31 - 1)
    return dict(cu_q_lens=cu.astype(np.int32), context_lens=np.array(ctx, np.int32),
                status=np.array(status, np.int32), slot_mapping=slots,
                pages_used=np.array([used], np.int32), page_table=table.astype(np.int32))
