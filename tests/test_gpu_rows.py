"""GPU tests of the row operators (vd_rmsnorm, vd_rmsnorm_fp8, vd_quantize_fp8)
against their plain 64-bit forms, and of a row's bits: they depend on the row
alone, not on M, the row's place, strides or how the call is made."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_38981_amd import vdattn as V
from tests import gpu_util as U
from tests import ops_util as O

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    U.require_gpu()


def _rows(seed, m, k, pad=0, scale=1.0):
    """bf16 rows, row i larger by 2^(i mod 5); NaN in the padding (never read)."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((m, k + pad), float("nan"), dtype=torch.bfloat16)
    x[:, :k] = (torch.randn((m, k), generator=g) * scale * 2.0 ** (torch.arange(m)[:, None] % 5)).bfloat16()
    return x.cuda()[:, :k]


def _weight(seed, k):
    return (1.0 + 0.2 * torch.randn(k, generator=torch.Generator().manual_seed(seed))).bfloat16().cuda()


# one vector, one wavefront, its last lanes idle, two and several wavefronts, ragged groups
# of 8 .. 120 values, the largest row
SIZES = [(1, 8), (3, 64), (5, 136), (2, 512), (7, 520), (4, 1024), (3, 1032), (130, 2880), (1, 4096),
         (9, 5120), (2, 8200), (3, 16384), (2, 16392), (2, 32768)]


@pytest.mark.parametrize("m,k", SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(m, k, residual):
    x, w = _rows(k + m, m, k, pad=8 * (m % 3)), _weight(k, k)
    r = _rows(k + m + 1, m, k, pad=16, scale=3.0) if residual else None
    h, y = O.norm(x, w, EPS, r)
    got = V.rmsnorm(x, w, EPS, residual=r)
    codes = V.rmsnorm_fp8(x, w, EPS, residual=r)
    torch.cuda.synchronize()
    if residual:
        O.same_bits(got[1], h)
        O.same_bits(codes[2], h)
        got = got[0]
    O.check_bf16(got, y, O.NORM_REL)
    O.check_codes(codes[0], codes[1], y, O.NORM_REL)
    assert codes[1].shape == (m, -(-k // 128))


@pytest.mark.parametrize("m,k", [(1, 8), (3, 128), (5, 136), (2, 1000), (17, 2880), (65, 4096), (3, 14336),
                                 (1, 40000), (70000, 8)])
@pytest.mark.parametrize("gate", [False, True])
def test_quantize(m, k, gate):
    both = _rows(3 * k + m, m, 2 * k, pad=8, scale=2.0)
    x = both[:, k:]
    if gate:
        codes, scales = V.quantize_fp8(x, gate=both[:, :k])
        torch.cuda.synchronize()
        O.check_codes(codes, scales, O.gated(x, both[:, :k]), O.GATE_REL)
    else:
        codes, scales = V.quantize_fp8(x)
        torch.cuda.synchronize()
        q, s = O.codes_of(x.float().cpu().numpy())
        O.same_bits(scales, s)
        O.same_bits(codes, q)


@pytest.mark.parametrize("k", [520, 4096, 16392])
def test_rows_do_not_depend_on_the_call(k):
    """Rows of a 300-row call, one by one, as a suffix, with padded strides, in place, and
    normed after their addition instead of with it: the same bits."""
    m = 300
    x, w, r = _rows(k, m, k), _weight(k, k), _rows(k + 9, m, k, scale=3.0)
    out, h = V.rmsnorm(x, w, EPS, residual=r)
    q, s, _ = V.rmsnorm_fp8(x, w, EPS, residual=r)
    gq, gs = V.quantize_fp8(x, gate=r)
    for lo, hi in [(0, 1), (1, 2), (299, 300), (100, 117), (7, 300)]:
        o2, h2 = V.rmsnorm(x[lo:hi], w, EPS, residual=r[lo:hi])
        q2, s2, _ = V.rmsnorm_fp8(x[lo:hi], w, EPS, residual=r[lo:hi])
        O.same_bits(o2, out[lo:hi])
        O.same_bits(h2, h[lo:hi])
        O.same_bits(q2, q[lo:hi])
        O.same_bits(s2, s[lo:hi])
        q3, s3 = V.quantize_fp8(x[lo:hi], gate=r[lo:hi])
        O.same_bits(q3, gq[lo:hi])
        O.same_bits(s3, gs[lo:hi])
    O.same_bits(V.rmsnorm(h, w, EPS), out)
    q4, s4 = V.rmsnorm_fp8(h, w, EPS)
    O.same_bits(q4, q)
    O.same_bits(s4, s)
    # in place: the sum over the residual, the norm over x
    xi, ri = x.clone(), r.clone()
    o5, h5 = V.rmsnorm(xi, w, EPS, residual=ri, residual_out=ri, out=xi)
    assert o5 is xi and h5 is ri
    O.same_bits(xi, out)
    O.same_bits(ri, h)
    xi, ri = x.clone(), r.clone()
    V.rmsnorm(xi, w, EPS, residual=ri, residual_out=xi, out=ri)
    O.same_bits(ri, out)
    O.same_bits(xi, h)
    xi, ri = x.clone(), r.clone()
    q5, s5, h5 = V.rmsnorm_fp8(xi, w, EPS, residual=ri, residual_out=ri)
    O.same_bits(q5, q)
    O.same_bits(s5, s)
    O.same_bits(ri, h)
    # strided rows in and out, scales row by row
    big = torch.zeros((m, k + 64), dtype=torch.bfloat16, device="cuda")
    big[:, 8:8 + k] = x
    codes = torch.full((m, k + 24), 1.0, device="cuda").to(V.E4M3)
    sc = torch.zeros((m, -(-k // 128) + 3), device="cuda")
    V.rmsnorm_fp8(big[:, 8:8 + k], w, EPS, residual=r, out=codes[:, 8:8 + k],
                  scales=sc[:, 1:1 - (-k // 128)])
    O.same_bits(codes[:, 8:8 + k], q)
    O.same_bits(sc[:, 1:1 - (-k // 128)], s)
    assert (codes[:, :8].float() == 1).all() and (codes[:, 8 + k:].float() == 1).all()
    assert (sc[:, 0] == 0).all() and (sc[:, 1 - (-k // 128):] == 0).all()


@pytest.mark.parametrize("m,k", [(1024, 4104), (2077, 4104), (1025, 128), (70000, 200)])
def test_many_rows(m, k):
    """Calls whose rows go to the dies in runs and whose groups in tiles: every row has the bits
    of calls of 100 rows, and nothing behind the last row or group is written."""
    x, r, w = _rows(k, m, k), _rows(k + 1, m, k, scale=3.0), _weight(1, k)
    kb = -(-k // 128)
    for f in (lambda a, b, **o: V.rmsnorm_fp8(a, w, EPS, residual=b, **o), lambda a, b, **o: V.quantize_fp8(a, **o),
              lambda a, b, **o: V.quantize_fp8(a, gate=b, **o)):
        codes = torch.full((m + 40, k + 8), 1.0, device="cuda").to(V.E4M3)
        scales = torch.full((kb + 1, m + 40), -1.0, device="cuda").t()
        got = f(x, r, out=codes[:m, :k], scales=scales[:m, :kb])
        for lo in sorted({0, 31, m // 2, m - 100}):
            part = f(x[lo:lo + 100], r[lo:lo + 100])
            for p, whole in zip(part, got):
                O.same_bits(p, whole[lo:lo + 100], lo)
        all_rows = torch.cat([f(x[i:i + 500], r[i:i + 500])[1] for i in range(0, m, 500)])
        O.same_bits(all_rows, got[1])
        assert (codes[m:].float() == 1).all() and (codes[:, k:].float() == 1).all()
        assert (scales[m:] == -1).all() and (scales[:, kb:] == -1).all()


def test_not_finite_and_extreme_values():
    k = 264
    w = torch.ones(k, dtype=torch.bfloat16, device="cuda")
    x = _rows(1, 8, k)
    x[1, 3], x[2, 200], x[3, 263] = float("nan"), float("inf"), -float("inf")
    x[4] = 0
    x[5] = 3e38                # the sum of squares is past fp32: the norm is 0 where 64 bits have 1
    x[6] = 2.0 ** -133         # the least bf16
    x[7, :] = 0
    x[7, 130] = 2.0 ** -133
    q, s = V.quantize_fp8(x)
    rq, rs = O.codes_of(x.float().cpu().numpy())
    fine = torch.isfinite(rs)
    assert torch.equal(fine, torch.isfinite(s.cpu()))
    O.same_bits(s.cpu()[fine], rs[fine])
    got, want = O.values_of(q, s), O.values_of(rq, rs)
    assert np.array_equal(got, want, equal_nan=True)
    # the groups of the three rows are NaN throughout, and only they
    bad = np.isnan(got)
    assert bad[1, :128].all() and bad[2, 128:256].all() and bad[3, 256:].all()
    assert bad.sum() == 128 + 128 + 8
    # the norm: a row that holds one is NaN (an infinity: 0 at the finite values), the others not
    out = V.rmsnorm(x, w, EPS).float().cpu()
    assert out[1].isnan().all() and out[2, 200].isnan() and out[3, 263].isnan()
    assert (out[4] == 0).all() and (out[5] == 0).all() and torch.isfinite(out[[0, 6, 7]]).all()
    # a zero row without eps has no norm, as by the formula
    assert V.rmsnorm(x[4:5], w, 0.0).isnan().all()
    # SiLU at both ends
    g = torch.tensor([[-3e38, -100.0, -0.0, 100.0, 3e38, 1.0, 2.0, 4.0]], dtype=torch.bfloat16).cuda()
    q, s = V.quantize_fp8(torch.ones_like(g), gate=g)
    assert torch.isfinite(s).all() and O.values_of(q, s)[0, 0] == 0


def test_offsets_past_32_bits():
    """Rows that lie past 2^32 bytes: the last ones equal themselves alone."""
    m, k = 560000, 4096  # 4.6 GB a matrix
    x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(-20000, 20000, generator=torch.Generator(device="cuda").manual_seed(1))
    x.clamp_(-100, 100)
    w = _weight(1, k)
    out = V.rmsnorm(x, w, EPS)
    O.same_bits(V.rmsnorm(x[m - 3:].clone(), w, EPS), out[m - 3:])
    del out
    q, s = V.quantize_fp8(x)
    q2, s2 = V.quantize_fp8(x[m - 3:].clone())
    O.same_bits(q2, q[m - 3:])
    O.same_bits(s2, s[m - 3:])


def test_wrappers_refuse():
    x, w = _rows(1, 4, 128), _weight(1, 128)
    for f, e in [(lambda: V.rmsnorm(x.float(), w), TypeError),
                 (lambda: V.rmsnorm(x, w[:64]), ValueError),
                 (lambda: V.rmsnorm(x, w, residual=x[:2]), ValueError),
                 (lambda: V.rmsnorm(x, w, residual_out=x), ValueError),
                 (lambda: V.rmsnorm(x, w, residual=x, residual_out=x, out=x), V.VdError),
                 (lambda: V.rmsnorm(x.t(), w), ValueError),
                 (lambda: V.rmsnorm(x, w, eps=-1.0), V.VdError),
                 (lambda: V.rmsnorm(x[:, 4:68], w[:64]), V.VdError),
                 (lambda: V.rmsnorm(x[:, :100], w[:100]), V.VdError),
                 (lambda: V.rmsnorm(x[:1].expand(4, 128), w), V.VdError),
                 (lambda: V.rmsnorm_fp8(x, w, out=torch.empty_like(x)), TypeError),
                 (lambda: V.quantize_fp8(x, gate=x[:, :64]), ValueError),
                 (lambda: V.quantize_fp8(x, scales=torch.empty((4, 2), device="cuda")), ValueError),
                 (lambda: V.quantize_fp8(x, scales=torch.empty((1, 1), device="cuda").expand(4, 1)),
                  V.VdError)]:
        with pytest.raises(e):
            f()
    assert V.rmsnorm(x[:0], w).shape == (0, 128)
    q, s = V.quantize_fp8(x[:0])
    assert q.shape == (0, 128) and s.shape == (0, 1)


def test_wrappers_refuse_rows_past_31_bits():
    """2^32 + 128 columns would be 128 to a 32-bit argument."""
    x = torch.empty((0, 2**32 + 128), dtype=torch.bfloat16, device="cuda")
    w = torch.empty(2**32 + 128, dtype=torch.bfloat16, device="cuda")  # 8.6 GB
    for f in (lambda: V.quantize_fp8(x), lambda: V.rmsnorm(x, w), lambda: V.rmsnorm_fp8(x, w)):
        with pytest.raises(ValueError):
            f()
