"""GPU tests of the page map (vd_map_pages) against the plain form that goes
request by request and token by token: every value is equal."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_38981_amd import vdattn as V
from tests import gpu_util as U
from tests import ops_util as O

pytestmark = pytest.mark.gpu
FILL = -77


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    U.require_gpu()


def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(np.array(v, dtype=np.int64).astype(np.int32))).cuda()


def _run(q, c, free, table, num_pages, rows):
    t = _i32(table)
    B = len(q)
    i32 = lambda n: torch.full((n,), FILL, dtype=torch.int32, device="cuda")  # noqa: E731
    out = V.PageMap(i32(B + 1), i32(B), torch.full((rows,), FILL, dtype=torch.int64, device="cuda"),
                    i32(B), i32(1))
    V.map_pages(_i32(q), _i32(c), _i32(free), t, num_pages, rows, out=out)
    torch.cuda.synchronize()
    return dict(cu_q_lens=out.cu_q_lens, context_lens=out.context_lens, status=out.status,
                slot_mapping=out.slot_mapping, pages_used=out.pages_used, page_table=t)


def _check(q, c, free, table, num_pages, rows):
    want = O.page_map(q, c, free, table, num_pages, rows)
    got = _run(q, c, free, table, num_pages, rows)
    for name, w in want.items():
        g = got[name].cpu().numpy()
        assert g.dtype == w.dtype and g.shape == w.shape, name
        assert np.array_equal(g, w), (name, np.flatnonzero((g != w).ravel())[:5])
    return want


def _batch(seed, B, s_hi, c_hi, extra=5, short=0):
    rng = np.random.default_rng(seed)
    q, c = rng.integers(0, s_hi + 1, B), rng.integers(0, c_hi + 1, B)
    q[rng.random(B) < 0.4] = 1
    have, total = -(-c // 16), -(-(c + q) // 16)
    new = int((total - have).sum())
    pages = int(total.sum()) + extra
    perm = rng.permutation(pages)
    table = np.full((B, max(1, int(total.max(initial=0)) + 2)), FILL)
    at = 0
    for r in range(B):
        table[r, :have[r]] = perm[at:at + have[r]]
        at += have[r]
    return q, c, perm[at:at + max(new - short, 0) + (0 if short else extra)], table, pages, int(q.sum())


@pytest.mark.parametrize("B,s_hi,c_hi", [(1, 1, 0), (1, 1, 15), (1, 1, 16), (1, 5000, 100), (3, 17, 40),
                                         (64, 1, 4096), (255, 40, 300), (1024, 3, 64), (1025, 9, 100),
                                         (4096, 2, 33), (4097, 5, 20), (9000, 3, 50), (7, 3000, 0)])
@pytest.mark.parametrize("pad", [0, 1, 2000])
def test_map(B, s_hi, c_hi, pad):
    q, c, free, table, pages, rows = _batch(B * 7 + s_hi, B, s_hi, c_hi)
    _check(q, c, free, table, pages, rows + pad)


@pytest.mark.parametrize("seed", range(4))
def test_short_free_list_and_short_rows(seed):
    """The free list ends inside the batch: the first request that does not fit and the later
    ones that need a page are refused, those that need none are not; likewise the rows."""
    q, c, free, table, pages, rows = _batch(seed, 300, 60, 200, short=100)
    want = _check(q, c, free, table, pages, rows)
    assert (want["status"] == 4).any() and (want["status"] == 0).any()
    want = _check(q, c, free, table, pages, rows // 2)
    assert (want["status"] & 8).any()
    _check(q, c, free[:0], table, pages, rows)
    _check(q, c, free, table[:, :4], pages, rows)  # a narrow table refuses the long ones


def test_lengths_that_no_call_can_hold():
    """Negative and huge lengths refuse their requests and harm no other."""
    big = 2**31 - 1
    table = np.arange(48).reshape(8, 6)
    q = [3, -1, 1, big, 2, 5, big, 4]
    c = [20, 16, -5, 1, 32, big, big, 0]
    want = _check(q, c, [100, 101, 102, 103], table, 200, 64)
    assert want["status"].tolist()[:3] == [0, 1, 1] and want["status"][3] & 1
    # the same without the ones whose rows take up the call
    q = [3, -1, 1, 0, 2, 5, 0, 4]
    want = _check(q, c, [100, 101, 102, 103], table, 200, 64)
    assert want["status"].tolist() == [0, 1, 1, 0, 0, 3, 2, 0]
    # many huge ones: the sums saturate
    _check([big] * 2000 + [1], [0] * 2000 + [5], [1], np.zeros((2001, 2)), 10, 100)


def test_page_ids_outside_the_pool_have_no_slots():
    table = np.array([[5, 900], [-3, 7]])
    want = _check([4, 20], [18, 10], [2, 40, 1], table, 40, 24)
    assert (want["slot_mapping"][:4] == -1).all() and (want["slot_mapping"][4:10] == -1).all()


def test_empty_calls():
    _check([], [], [], np.zeros((0, 1)), 4, 0)
    _check([], [], [1], np.zeros((0, 1)), 4, 70)
    _check([0, 0], [0, 33], [], np.zeros((2, 3)), 4, 0)
    _check([0], [0], [1], np.zeros((1, 1)), 4, 3)
    # by the wrapper's own allocation
    m = V.map_pages(_i32([2]), _i32([15]), _i32([3]), _i32([[1, 9]]), 4, 2)
    assert m.slot_mapping.tolist() == [31, 48] and m.context_lens.tolist() == [17]
    assert m.cu_q_lens.tolist() == [0, 2] and m.status.tolist() == [0] and m.pages_used.tolist() == [1]


def test_slots_past_32_bits():
    pages = 2**31 - 1
    want = _check([2, 1], [15, 8], [pages - 1], np.array([[pages - 2, 0], [2**28 + 3, 0]]), pages, 3)
    assert want["slot_mapping"].tolist() == [(pages - 2) * 16 + 15, (pages - 1) * 16, (2**28 + 3) * 16 + 8]


def test_table_past_32_bits():
    """A table of 2.4e9 entries: the last requests' pages are where they belong."""
    B, stride = 9200, 2**18
    table = torch.full((B, stride), FILL, dtype=torch.int32, device="cuda")
    c = torch.zeros(B, dtype=torch.int32, device="cuda")
    c[B - 1] = 16 * (stride - 2)
    table[B - 1, stride - 3] = 5
    q = torch.ones(B, dtype=torch.int32, device="cuda")
    q[B - 1] = 20
    free = torch.arange(10, B + 20, dtype=torch.int32, device="cuda")
    m = V.map_pages(q, c, free, table, B + 30, B + 19)
    assert (m.status == 0).all() and int(m.pages_used) == B + 1
    assert table[B - 1, stride - 2:].tolist() == [10 + B - 1, 10 + B]
    assert torch.equal(table[:B - 1, 0], free[:B - 1]) and (table[B - 2, 1:] == FILL).all()
    assert m.slot_mapping[B - 1:].tolist() == [(10 + B - 1) * 16 + i for i in range(16)] + [
        (10 + B) * 16 + i for i in range(4)]


def test_wrapper_refuses():
    i = _i32([1, 2])
    t = _i32([[0], [1]])
    for f, e in [(lambda: V.map_pages(i.long(), i, i, t, 4, 3), TypeError),
                 (lambda: V.map_pages(i, i[:1], i, t, 4, 3), ValueError),
                 (lambda: V.map_pages(i, i, i, t[:1], 4, 3), ValueError),
                 (lambda: V.map_pages(i, i, i, t.t(), 4, 3), ValueError),
                 (lambda: V.map_pages(i, i, i, t, -1, 3), V.VdError),
                 (lambda: V.map_pages(i, i, i, t, 4, -3), V.VdError),
                 (lambda: V.map_pages(i, i, i, t, 4, 3, out=V.PageMap(i, i, i, i, i)), (TypeError, ValueError))]:
        with pytest.raises(e):
            f()


def test_wrapper_refuses_a_table_past_31_bits():
    """A row of 2^32 + 1 entries would be 1 to a 32-bit argument."""
    i = _i32([1])
    table = torch.empty((1, 2**32 + 1), dtype=torch.int32, device="cuda")  # 17 GB
    with pytest.raises(ValueError):
        V.map_pages(i, i, i, table, 4, 1)
