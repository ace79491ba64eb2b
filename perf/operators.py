"""Cases of the operators that surround the paged attention in a serving step:
the page map made from request lengths, the RMS norm with the residual's
addition, the quantization of rows to 8 bits, and the 8-bit linear layer.

A case is a dict of plain values.  ``prepare`` makes what a serving program has
in hand before the call, ``run`` is one call (the plain form in 32 bits, or the
library's entry point where ``own`` is true), ``work`` the bytes and operations
it cannot do without, and ``exact`` the same outputs in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

P = 16       # tokens per page
G = 128      # values per scale
E4M3 = torch.float8_e4m3fn
TINY = 2.0 ** -117            # the least largest magnitude of a group
PER_448 = float(np.float32(1.0 / 448.0))
EPS = 1e-5


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
def _pages(name, *, dec=0, dec_hi=1, pre=0, chunk_lo=1, chunk_hi=1, off_hi=0, pad=0, short=False, lens=0):
    """``pre`` requests that add a chunk of chunk_lo .. chunk_hi tokens behind 0 ..
    off_hi cached ones, and ``dec`` that add one token to 1 .. dec_hi cached ones;
    ``pad`` unused rows at the end; ``short``: the free list ends too early."""
    c = dict(kind="pages", dec=dec, dec_hi=dec_hi, pre=pre, chunk_lo=chunk_lo, chunk_hi=chunk_hi,
             off_hi=off_hi, pad=pad, short=short, lens=lens)
    return dict(c, name=name) if name else c


def _norm(name, m, k, *, fp8, residual=True, pad=0):
    c = dict(kind="norm", m=m, k=k, fp8=fp8, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _quant(name, m, k, *, gate, pad=0):
    c = dict(kind="quant", m=m, k=k, gate=gate, pad=pad)
    return dict(c, name=name) if name else c


def _linear(name, m, n, k, pad=0, by_row=False):
    """``by_row``: the activations' scales lie row by row, and not as the library's
    own quantization leaves them (the scales of a block of K side by side)."""
    c = dict(kind="linear", m=m, n=n, k=k, pad=pad, by_row=by_row)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a serving batch's decode step: 64 requests, a token each
        _pages("pages_decode", dec=64, dec_hi=4096, lens=1),
        # continuous batching: long prompt chunks beside many decodes, rows padded
        # to a captured size
        _pages("pages_mixed", dec=600, dec_hi=32768, pre=24, chunk_lo=300, chunk_hi=8192,
               off_hi=16384, pad=333, lens=2),
        # one user's token: the norm in front of a bf16 projection
        _norm("norm_decode", 1, 4096, fp8=False),
        # a decode batch of a wide model, in front of an 8-bit projection
        _norm("norm_fp8_decode", 77, 8192, fp8=True),
        # a prefill's tokens
        _norm("norm_fp8_prefill", 8192, 4096, fp8=True),
        # a decode batch's attention output, in front of the output projection
        _quant("quant_decode", 64, 4096, gate=False),
        # a prefill's MLP: SiLU(gate) * up out of one product's two halves
        _quant("quant_gate_prefill", 4096, 14336, gate=True),
        # one user's token through the output projection
        _linear("linear_m1", 1, 4096, 4096),
        # a decode batch through the query, key and value projection
        _linear("linear_decode", 48, 6144, 4096),
        # a verify batch of odd size into a width off every tile, K in half blocks
        _linear("linear_ragged", 333, 5000, 2112, by_row=True),
        # prefill: the query, key and value projection, and a wide model's MLP
        _linear("linear_prefill", 4096, 6144, 4096),
        _linear("linear_wide", 4096, 28672, 8192),
    ]


def _log_int(rng, lo, hi):
    """An integer of lo .. hi, uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["pages", "norm", "quant", "linear"], [2, 3, 2, 5])[0]
    if kind == "pages":
        pre = rng.choice([0, 0, 1, _log_int(rng, 2, 32)])
        c = _pages(None, dec=_log_int(rng, 1, 3000), dec_hi=_log_int(rng, 16, 32768), pre=pre,
                   pad=rng.choice([0, 0, 1, 100]), short=rng.random() < 0.15,
                   lens=rng.randrange(1 << 20))
        if pre:
            c["chunk_hi"] = _log_int(rng, 20, 8192)
            c["chunk_lo"] = max(1, c["chunk_hi"] // rng.choice([1, 3, 20]))
            c["off_hi"] = rng.choice([0, _log_int(rng, 16, 32768)])
        return c
    if kind == "norm":
        while True:
            m, k = _log_int(rng, 1, 8192), 8 * _log_int(rng, 8, 2048)
            if rng.random() < 0.7:
                k = max(128, k // 128 * 128)
            if m * k <= 8192 * 4096:
                return _norm(None, m, k, fp8=rng.random() < 0.6, residual=rng.random() < 0.8,
                             pad=rng.choice([0, 0, 8, 128]))
    if kind == "quant":
        while True:
            m, k = _log_int(rng, 1, 8192), 8 * _log_int(rng, 16, 3584)
            if rng.random() < 0.7:
                k = max(128, k // 128 * 128)
            if m * k <= 4096 * 14336:
                return _quant(None, m, k, gate=rng.random() < 0.5, pad=rng.choice([0, 0, 8, 64]))
    while True:
        m, n, k = _log_int(rng, 1, 8192), _log_int(rng, 100, 28672), 64 * _log_int(rng, 2, 224)
        if rng.random() < 0.6:
            n = max(128, n // 128 * 128)
        if rng.random() < 0.8:
            k = max(128, k // 128 * 128)
        if 2.0 * m * n * k <= 1.9e12:
            return _linear(None, m, n, k, rng.choice([0, 0, 16, 64]), rng.random() < 0.25)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, scale=1.0):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    return x.normal_(0.0, scale, generator=gen)


def _lengths(case):
    """(new tokens, cached tokens) of every request, chunks first."""
    rng = np.random.default_rng([81, case["lens"]])
    s = rng.integers(case["chunk_lo"], case["chunk_hi"] + 1, case["pre"])
    off = rng.integers(0, case["off_hi"] + 1, case["pre"])
    dec = rng.integers(1, case["dec_hi"] + 1, case["dec"])
    return (np.concatenate([s, np.ones(case["dec"], np.int64)]).astype(np.int64),
            np.concatenate([off, dec]).astype(np.int64))


def _page_inputs(case, seed):
    """Lengths, a table with the cached tokens' pages, and the free pages, of a
    shuffled pool."""
    s, c = _lengths(case)
    have, total = -(-c // P), -(-(c + s) // P)
    new = int((total - have).sum())
    pages = int(total.sum()) + new // 4 + 8
    perm = torch.randperm(pages, generator=_gen(seed), device="cuda").int()
    stride = int(total.max()) + 3
    table = torch.full((len(s), stride), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(stride, device="cuda")[None] < torch.from_numpy(have).cuda()[:, None]] = \
        perm[:int(have.sum())]
    free = perm[int(have.sum()):]
    if case["short"]:
        free = free[:new * 2 // 3]
    return dict(q_lens=torch.from_numpy(s.astype(np.int32)).cuda(),
                cached=torch.from_numpy(c.astype(np.int32)).cuda(), table=table,
                free=free.contiguous(), pages=pages, rows=int(s.sum()) + case["pad"])


def _norm_inputs(case, seed):
    """Hidden rows with a few channels far larger than the others, as a model's
    residual stream has them."""
    gen, m, k = _gen(seed), case["m"], case["k"]
    big = 1.0 + 30.0 * (torch.rand(k, generator=gen, device="cuda") < 0.01)
    x = dict(x=_normal(gen, (m, k + case["pad"]))[:, :k], w=(1.0 + 0.2 * _normal(gen, (k,))))
    if case["residual"]:
        x["res"] = _normal(gen, (m, k + case["pad"]), 3.0)[:, :k]
        x["res"] *= big.bfloat16()
    return x


def _quant_inputs(case, seed):
    gen, m, k = _gen(seed), case["m"], case["k"]
    if not case["gate"]:
        return dict(x=_normal(gen, (m, k + case["pad"]))[:, :k], gate=None)
    both = _normal(gen, (m, 2 * k + case["pad"]), 2.0)
    return dict(x=both[:, k:2 * k], gate=both[:, :k])


def _to_blocks(w):
    """Weights as e4m3 with a scale for each block of 128 x 128."""
    n, k = w.shape
    nb, kb = -(-n // G), -(-k // G)
    full = torch.zeros((nb * G, kb * G), dtype=torch.float32, device=w.device)
    full[:n, :k] = w
    full = full.view(nb, G, kb, G)
    s = full.abs().amax((1, 3)).clamp_(min=TINY) / 448.0
    full /= s[:, None, :, None]
    return full.view(nb * G, kb * G)[:n, :k].to(E4M3).contiguous(), s


def _linear_inputs(case, seed):
    """A checkpoint's weights in 8 bits, and activations as a quantization
    leaves them (rows padded by ``pad`` bytes)."""
    gen, m, n, k = _gen(seed), case["m"], case["n"], case["k"]
    kb = -(-k // G)
    b, bs = _to_blocks(_normal(gen, (n, k), 0.02).float())
    a = torch.empty((m, k + case["pad"]), dtype=E4M3, device="cuda")
    a.copy_((_normal(gen, (m, k + case["pad"])) * 120.0).clamp_(-448.0, 448.0))
    s = torch.empty((m, kb) if case["by_row"] else (kb, m), dtype=torch.float32, device="cuda")
    s.uniform_(0.002, 0.02, generator=gen)
    s = s if case["by_row"] else s.t()
    return dict(a=a[:, :k], a_s=s, b=b, b_s=bs)


_INPUTS = {"pages": _page_inputs, "norm": _norm_inputs, "quant": _quant_inputs,
           "linear": _linear_inputs}


def prepare(case, seed):
    return dict(_INPUTS[case["kind"]](case, seed), kind=case["kind"], fp8=case.get("fp8"))


# ---------------------------------------------------------------------------
# One call
# ---------------------------------------------------------------------------
def run(state):
    if own:
        return _call(state)
    return _PLAIN[state["kind"]](state)


def _call(s):
    from paper_2609_38981_amd import vdattn as V

    if s["kind"] == "linear":
        return V.linear_fp8(s["a"], s["a_s"], s["b"], s["b_s"])
    if s["kind"] == "quant":
        return V.quantize_fp8(s["x"], gate=s["gate"])
    if s["kind"] == "norm":
        f = V.rmsnorm_fp8 if s["fp8"] else V.rmsnorm
        return f(s["x"], s["w"], EPS, residual=s.get("res"))
    m = V.map_pages(s["q_lens"], s["cached"], s["free"], s["table"], s["pages"], s["rows"])
    return {"cu_q_lens": m.cu_q_lens, "context_lens": m.context_lens, "table": s["table"],
            "slots": m.slot_mapping, "status": m.status, "used": m.pages_used}


def _codes(y):
    """Rows as e4m3, and a scale for each 128 values of a row (the last group of a
    row may be shorter)."""
    m, k = y.shape
    kb = -(-k // G)
    z = torch.nn.functional.pad(y, (0, kb * G - k)).view(m, kb, G)
    s = z.abs().amax(-1).clamp(min=TINY) * PER_448
    q = (z * (1.0 / s)[..., None]).view(m, kb * G)[:, :k].to(E4M3)
    return q.contiguous(), s


def _plain_norm(s):
    h = s["x"]
    if s.get("res") is not None:
        h = (h.float() + s["res"].float()).bfloat16()
    f = h.float()
    y = f * (1.0 / (f.square().sum(-1, keepdim=True) / f.shape[1] + EPS).sqrt()) * s["w"].float()
    out = _codes(y) if s["fp8"] else (y.bfloat16(),)
    if s.get("res") is not None:
        out = (*out, h)
    return out if len(out) > 1 else out[0]


def _plain_quant(s):
    y = s["x"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        y = g / (1.0 + torch.exp(-g)) * y
    return _codes(y)


def _plain_linear(s):
    k, n = s["a"].shape[1], s["b"].shape[0]
    a = s["a"].float() * s["a_s"].repeat_interleave(G, 1)[:, :k]
    b = s["b"].float() * s["b_s"].repeat_interleave(G, 0)[:n].repeat_interleave(G, 1)[:, :k]
    return torch.matmul(a, b.t()).bfloat16()


def _plain_pages(x):
    q, c, table, free = x["q_lens"].long(), x["cached"].long(), x["table"], x["free"]
    rows, stride = x["rows"], table.shape[1]
    s = q.clamp(min=0)
    n = c + s
    end = s.cumsum(0)
    cu = torch.cat([end.new_zeros(1), end])
    have, total = (c + P - 1) // P, (n + P - 1) // P
    status = ((q < 0) | (c < 0) | (n > 2 ** 31 - 1)).int() + 2 * (total > stride).int() + \
        8 * (end > rows).int()
    need = torch.where(status == 0, total - have, 0)
    taken = need.cumsum(0)
    status = status + 4 * ((need > 0) & (taken > free.shape[0])).int()
    ok = status == 0
    first = taken - need  # of the request's new pages in the free list
    last = max(free.shape[0] - 1, 0)
    some = free if free.shape[0] else free.new_full((1,), -1)
    at = torch.arange(stride, device=q.device)[None]
    new = ok[:, None] & (at >= have[:, None]) & (at < total[:, None])
    table = torch.where(new, some[(first[:, None] + at - have[:, None]).clamp(0, last)], table)
    t = torch.arange(rows, device=q.device)
    r = torch.searchsorted(end, t, right=True).clamp(max=q.shape[0] - 1)
    pos = c[r] + t - cu[r]
    page = table[r, (pos // P).clamp(0, stride - 1)].long()
    fine = (t < end[-1]) & ok[r] & (page >= 0) & (page < x["pages"])
    return {"cu_q_lens": cu.int(), "context_lens": torch.where(ok, n, 0).int(), "table": table,
            "slots": torch.where(fine, page * P + pos % P, -1), "status": status,
            "used": torch.where(ok & (need > 0), taken, 0).amax().int().view(1)}


_PLAIN = {"pages": _plain_pages, "norm": _plain_norm, "quant": _plain_quant,
          "linear": _plain_linear}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "pages":
        s, c = _lengths(case)
        new = int((-(-(c + s) // P) + -c // P).sum())
        old = int(((c % P) > 0).sum())  # a request's last cached page, read for its slots
        return {"bytes": 20.0 * len(s) + 8.0 * (int(s.sum()) + case["pad"]) + 8.0 * new + 4.0 * old,
                "flops": 0.0}
    m, k = case["m"], case["k"]
    kb = -(-k // G)
    codes = m * k + 4.0 * m * kb
    if case["kind"] == "norm":
        rows = 2.0 * m * k
        return {"bytes": rows * (3 if case["residual"] else 1) + 2.0 * k + (codes if case["fp8"] else rows),
                "flops": 5.0 * m * k}
    if case["kind"] == "quant":
        return {"bytes": 2.0 * m * k * (2 if case["gate"] else 1) + codes,
                "flops": (8.0 if case["gate"] else 3.0) * m * k}
    n = case["n"]
    return {"bytes": codes + n * k + 4.0 * -(-n // G) * kb + 2.0 * m * n, "flops": 2.0 * m * n * k}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits
# ---------------------------------------------------------------------------
def _exact_codes(y):
    q, s = torch.empty_like(y), []
    for i in range(0, y.shape[1], G):
        g = y[:, i:i + G]
        top = g.abs().max(1).values.clamp(min=TINY) / 448.0
        q[:, i:i + G] = (g / top[:, None]).to(E4M3).double()
        s.append(top)
    return q, torch.stack(s, 1)


def exact(case, seed):
    if case["kind"] == "pages":
        return None  # whole numbers
    x = _INPUTS[case["kind"]](case, seed)
    if case["kind"] == "linear":
        a, b = x["a"].double(), x["b"].double()
        for i in range(0, a.shape[1], G):
            a[:, i:i + G] *= x["a_s"][:, i // G, None].double()
            for j in range(0, b.shape[0], G):
                b[j:j + G, i:i + G] *= x["b_s"][j // G, i // G].double()
        return a @ b.t()
    if case["kind"] == "quant":
        y = x["x"].double()
        if case["gate"]:
            g = x["gate"].double()
            y = y * g * torch.sigmoid(g)
        return _exact_codes(y)
    h = x["x"].double()
    if case["residual"]:
        h = (h + x["res"].double()).bfloat16().double()
    y = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + EPS) * x["w"].double()
    out = list(_exact_codes(y)) if case["fp8"] else [y]
    if case["residual"]:
        out.append(h)
    return tuple(out) if len(out) > 1 else out[0]
