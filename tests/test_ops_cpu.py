"""CPU checks of the operators around the attention: the host checks of
vd_map_pages, vd_rmsnorm, vd_rmsnorm_fp8, vd_quantize_fp8 and vd_linear_fp8
(every case returns before a kernel is launched), the Python wrappers'
refusals, and the tests' own plain forms against worked values."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

from paper_2609_38981_amd import vdattn as V
from tests import ops_util as O

FAKE = 0x10000  # 16-byte aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    return V.load_library()


def _caller(fn, names, ok):
    def call(**kw):
        d = dict(ok, **kw)
        return fn(*[d[n] for n in names], None)
    return call


def test_every_operator_is_declared(lib):
    names = V.declared_functions()
    for name in ("vd_map_pages", "vd_rmsnorm", "vd_rmsnorm_fp8", "vd_quantize_fp8", "vd_linear_fp8"):
        assert name in names and hasattr(lib, name), name


NORM = "x ldx res ldr w eps sum lds out ldo M K".split()
NORM_OK = dict(x=FAKE, ldx=128, res=FAKE, ldr=128, w=FAKE, eps=1e-5, sum=FAKE, lds=128, out=FAKE + 4096,
               ldo=128, M=4, K=128)
NORM8 = "x ldx res ldr w eps sum lds out ldo s s_row s_blk M K".split()
NORM8_OK = dict(NORM_OK, s=FAKE, s_row=1, s_blk=4)


@pytest.mark.parametrize("fp8", [False, True])
def test_norm_rejects_before_launch(lib, fp8):
    call = _caller(lib.vd_rmsnorm_fp8 if fp8 else lib.vd_rmsnorm, NORM8 if fp8 else NORM,
                   NORM8_OK if fp8 else NORM_OK)
    assert call(M=0) == 0 and call(K=0) == 0 and call(M=0, x=None, out=None, w=None) == 0
    bad = [dict(M=-1), dict(K=-8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
           dict(x=None), dict(x=FAKE + 8), dict(ldx=120), dict(ldx=132), dict(w=None),
           dict(w=FAKE + 2), dict(res=None), dict(sum=None), dict(ldr=64), dict(lds=64),
           dict(res=FAKE + 4), dict(sum=FAKE + 8), dict(out=None), dict(ldo=64), dict(ldo=130),
           dict(out=FAKE + 4), dict(out=FAKE)]
    if fp8:
        bad += [dict(s=None), dict(s=FAKE + 2), dict(s_row=0), dict(s_row=-1),
                dict(K=256, ldx=256, ldr=256, lds=256, ldo=256, s_blk=0)]
    else:
        bad += [dict(out=FAKE + 8)]
    for kw in bad:
        assert call(**kw) == -1, kw
    big = dict(ldx=65536, ldr=65536, lds=65536, ldo=65536)
    for k in (1, 100, 124, 32776):
        assert call(K=k, **big) == -2, k


def test_quantize_rejects_before_launch(lib):
    names = "x ldx gate ldg out ldo s s_row s_blk M K".split()
    ok = dict(x=FAKE, ldx=256, gate=FAKE, ldg=256, out=FAKE, ldo=256, s=FAKE, s_row=1, s_blk=4, M=4,
              K=256)
    call = _caller(lib.vd_quantize_fp8, names, ok)
    assert call(M=0) == 0 and call(K=0) == 0
    for kw in (dict(M=-1), dict(K=-8), dict(x=None), dict(x=FAKE + 2), dict(ldx=248), dict(ldx=260),
               dict(gate=FAKE + 8), dict(ldg=8), dict(ldg=257), dict(out=None), dict(out=FAKE + 4),
               dict(ldo=255), dict(ldo=260), dict(s=None), dict(s=FAKE + 1), dict(s_row=0),
               dict(s_blk=0), dict(s_blk=-4), dict(M=2**62), dict(M=2**26 + 1)):
        assert call(**kw) == -1, kw
    assert call(K=252) == -2


def test_linear_fp8_rejects_before_launch(lib):
    names = "a lda as as_row as_blk b ldb bs bs_row bs_blk c ldc M N K".split()
    ok = dict(a=FAKE, lda=128, b=FAKE, ldb=128, c=FAKE, ldc=16, M=4, N=16, K=128, as_row=1, as_blk=4,
              bs=FAKE, bs_row=1, bs_blk=1)
    ok["as"] = FAKE
    call = _caller(lib.vd_linear_fp8, names, ok)
    assert call(M=0) == 0 and call(N=0) == 0
    bad = [dict(M=-1), dict(N=-1), dict(K=-1), dict(c=None), dict(ldc=8), dict(c=FAKE + 1),
           dict(a=None), dict(b=None), dict(bs=None), {"as": None}, dict(lda=64), dict(ldb=64),
           dict(lda=136), dict(ldb=132), dict(lda=2**29 + 16), dict(ldb=2**30), dict(a=FAKE + 8), dict(b=FAKE + 4), {"as": FAKE + 2},
           dict(bs=FAKE + 1), dict(as_row=-1), dict(as_blk=-1), dict(bs_row=-1), dict(bs_blk=-1)]
    for kw in bad:
        assert call(**kw) == -1, kw
    # more outputs than any launch covers
    assert call(M=2**62, N=2**30, ldc=2**30, K=0) == -1
    for k in (32, 96, 160):
        assert call(K=k, lda=256, ldb=256) == -2, k


@pytest.mark.skipif(torch.cuda.is_available(), reason="its pointers are not memory: without a "
                    "device only the launches fail")
@pytest.mark.parametrize("m,n,k,ld,want", [
    (1, 1, 64, 64, -4), (1, 4096, 4096, 4096, -4), (48, 6144, 4096, 4096, -4),
    (4096, 28672, 8192, 8192, -4), (4096, 6144, 4096, 2**24, -4), (2**22, 2**16, 0, 0, -4),
    (2**30, 1, 0, 0, -4), (1, 2**30, 0, 0, -4), (2**26, 2**12, 64, 64, -4), (2**33, 1, 0, 0, -1),
    (2**28, 2**16, 64, 2**24, -1), (2**40, 1, 0, 0, -1), (2**62, 2**31 - 1, 0, 0, -1),
    (1, 1, 2**31 - 64, 2**29, -1)])
def test_linear_fp8_launches_or_refuses_every_size(lib, m, n, k, ld, want):
    """A call of any size launches a kernel or is refused: without a device a launch is
    reported as failed, never VD_OK."""
    got = lib.vd_linear_fp8(FAKE, ld, FAKE, 1, 2**40, FAKE, ld, FAKE, 1, 2**40, FAKE, n, m, n, k, None)
    assert got == want


@pytest.mark.skipif(torch.cuda.is_available(), reason="its pointers are not memory")
@pytest.mark.parametrize("m,k", [(1, 8), (1, 32768), (2**20, 520), (2**27, 8), (2**40, 16)])
def test_row_operators_launch(lib, m, k):
    """As above: the norm of any number of rows, the 8-bit rows up to 2^27 groups."""
    assert lib.vd_rmsnorm(FAKE, k, FAKE, k, FAKE, 1e-5, FAKE, k, FAKE + 16, k, m, k, None) == -4
    assert lib.vd_rmsnorm_fp8(FAKE, k, None, 0, FAKE, 1e-5, None, 0, FAKE, k, FAKE, 1, m, m, k, None) == -4
    want = -4 if m * -(-k // 128) <= 2**27 else -1
    assert lib.vd_quantize_fp8(FAKE, k, FAKE, k, FAKE, k, FAKE, 1, m, m, k, None) == want


def test_map_pages_rejects_before_launch(lib):
    fields = dict(num_seqs=2, total_q_tokens=4, q_lens=FAKE, cached_lens=FAKE + 64,
                  free_pages=FAKE + 128, num_free=3, num_pages=8, page_table=FAKE + 256, pt_stride=4,
                  cu_q_lens=FAKE + 512, context_lens=FAKE + 576, slot_mapping=FAKE + 640,
                  status=FAKE + 704, pages_used=FAKE + 768)

    def call(**kw):
        return lib.vd_map_pages(ctypes.byref(V._PageMap(**dict(fields, **kw))), None)

    assert lib.vd_map_pages(None, None) == -1
    for name in ("q_lens", "cached_lens", "free_pages", "page_table", "cu_q_lens", "context_lens",
                 "slot_mapping", "status", "pages_used"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: FAKE + 2}) == -1, name
    assert call(slot_mapping=FAKE + 644) == -1
    for kw in (dict(num_seqs=-1), dict(num_seqs=2**31 - 1), dict(total_q_tokens=-1), dict(total_q_tokens=2**31),
               dict(num_free=-1), dict(num_pages=-1), dict(pt_stride=0), dict(context_lens=FAKE),
               dict(context_lens=FAKE + 64), dict(status=FAKE), dict(status=FAKE + 64)):
        assert call(**kw) == -1, kw


def test_wrappers_refuse_host_tensors():
    x = torch.zeros((2, 128), dtype=torch.bfloat16)
    q = x.to(V.E4M3)
    s = torch.ones((2, 1))
    i = torch.zeros(2, dtype=torch.int32)
    for f in (lambda: V.rmsnorm(x, x[0]), lambda: V.rmsnorm_fp8(x, x[0]), lambda: V.quantize_fp8(x),
              lambda: V.linear_fp8(q, s, q, s), lambda: V.map_pages(i, i, i, i.view(2, 1), 4, 2)):
        with pytest.raises((TypeError, ValueError)):
            f()


def test_plain_codes_on_worked_values():
    y = np.zeros((3, 200), np.float32)
    y[0, 0], y[0, 5] = 448.0, -1.0     # scale 1 (one unit off at most): codes as they are
    y[0, 130] = 7.0                    # the short group: scale 7 / 448
    y[2, 3] = np.nan
    q, s = O.codes_of(y)
    assert abs(float(s[0, 0]) - 1.0) <= 2.0 ** -23 and abs(float(s[0, 1]) * 64.0 - 1.0) <= 2.0 ** -23
    v = q.double().numpy()
    assert v[0, 0] == 448.0 and v[0, 5] == -1.0 and v[0, 130] == 448.0
    assert (v[1] == 0).all() and (s[1] > 0).all() and torch.isfinite(s[1]).all()
    assert np.isnan(O.values_of(q, s)[2, :128]).all() and (v[2, 128:] == 0).all()


def test_plain_page_map_on_worked_values():
    # 2 requests: 20 cached + 1 new (the page is there), 16 cached + 18 new (two new pages)
    table = np.full((2, 4), -1)
    table[0, :2], table[1, 0] = (7, 3), 5
    m = O.page_map([1, 18], [20, 16], [9, 2, 4], table, 10, 21)
    assert m["cu_q_lens"].tolist() == [0, 1, 19] and m["context_lens"].tolist() == [21, 34]
    assert m["page_table"].tolist() == [[7, 3, -1, -1], [5, 9, 2, -1]] and m["pages_used"] == [2]
    assert m["slot_mapping"].tolist() == [3 * 16 + 4] + [9 * 16 + i for i in range(16)] + [32, 33, -1, -1]
    m = O.page_map([1, 18, 1], [20, 16, 32], [9], np.full((3, 4), 1), 10, 20)
    assert m["status"].tolist() == [0, 4, 4] and m["pages_used"] == [0]
