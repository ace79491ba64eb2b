"""GPU: the operators run together as a serving step runs them -- page map, norm in
8 bits, projection, attention that appends its keys, 8-bit rows, projection, the
second norm with the residual, the gated MLP -- over two layers of a small model.

* Every operator's outputs are held to its plain 64-bit form on the step's own inputs.
* Requests in one call have the bits of each alone and of a prompt in two chunks.
* The step captured in a HIP graph replays bit for bit with other lengths and tokens in
  its buffers, and with the program's own eager work between the replays."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2609_38981_amd import vdattn as V
from tests import gpu_util as U
from tests import ops_util as O

pytestmark = pytest.mark.gpu
H, HQ, HKV, D, F = 512, 8, 2, 64, 1408
QKV = (HQ + 2 * HKV) * D
EPS = 1e-5
LAYERS = 2


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    U.require_gpu()


class Model:
    """Weights in 8 bits (blocks of 128 x 128), page pools and a free list."""

    def __init__(self, seed, pages):
        g = torch.Generator().manual_seed(seed)
        self.attn = V.VdAttn(HQ, HKV, D)
        self.pages = pages
        self.layers = []
        for _ in range(LAYERS):
            p = {n: self._weights(g, *s) for n, s in dict(qkv=(QKV, H), o=(H, HQ * D), up=(2 * F, H),
                                                          down=(H, F)).items()}
            p["n1"], p["n2"] = ((1 + 0.1 * torch.randn(H, generator=g)).bfloat16().cuda() for _ in range(2))
            self.layers.append(p)

    @staticmethod
    def _weights(g, n, k):
        w = torch.randn((n, k), generator=g) * k ** -0.5
        nb, kb = -(-n // 128), -(-k // 128)
        full = torch.zeros((nb * 128, kb * 128))
        full[:n, :k] = w
        full = full.view(nb, 128, kb, 128)
        s = full.abs().amax((1, 3)) / 448.0
        q = (full / s[:, None, :, None]).view(nb * 128, kb * 128)[:n, :k]
        return q.to(V.E4M3).cuda(), s.cuda()

    def pools(self):
        return [(self.attn.new_pool(self.pages).zero_(), self.attn.new_pool(self.pages).zero_())
                for _ in range(LAYERS)]

    def step(self, x, q_lens, cached, free, table, pools, max_q, max_ctx, seen=None):
        """One call: new rows x [T, H] of all requests -> their last hidden rows."""
        T = x.shape[0]
        m = V.map_pages(q_lens, cached, free, table, self.pages, T)
        res, h = x, None
        for w, (kp, vp) in zip(self.layers, pools):
            if h is None:
                q, s = V.rmsnorm_fp8(res, w["n1"], EPS)
                first = (res, None)
            else:
                first = (h, res)
                q, s, res = V.rmsnorm_fp8(h, w["n1"], EPS, residual=res)
            qkv = V.linear_fp8(q, s, *w["qkv"]).view(T, HQ + 2 * HKV, D)
            k, v = (qkv[:, HQ + i * HKV:HQ + (i + 1) * HKV].contiguous() for i in (0, 1))
            self.attn.kv_write(k, v, m.slot_mapping, kp, vp, self.pages)
            b = V.Batch(qkv[:, :HQ].contiguous(), m.cu_q_lens, m.context_lens, table, kp, vp, self.pages,
                        max_q, max_ctx)
            o = self.attn.forward(b, out=torch.zeros_like(b.q)).view(T, HQ * D)
            oq, os = V.quantize_fp8(o)
            ao = V.linear_fp8(oq, os, *w["o"])
            nq, ns, res2 = V.rmsnorm_fp8(ao, w["n2"], EPS, residual=res)
            up = V.linear_fp8(nq, ns, *w["up"])
            gq, gs = V.quantize_fp8(up[:, F:], gate=up[:, :F])
            h = V.linear_fp8(gq, gs, *w["down"])
            if seen is not None:
                seen.append(dict(w=w, first=first, q=(q, s), qkv=qkv.view(T, QKV), o=o, oq=(oq, os), ao=ao,
                                 res=res, nq=(nq, ns), res2=res2, up=up, gq=(gq, gs), h=h))
            res = res2
        return V.rmsnorm(h, self.layers[0]["n1"], EPS, residual=res)[0], m


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _x(seed, T):
    return torch.randn((T, H), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def _free(seed, pages):
    return torch.from_numpy(np.random.default_rng(seed).permutation(pages).astype(np.int32)).cuda()


PROMPTS = [37, 1, 16, 130, 64]


def _rows(m, x):
    return {i: x[int(m.cu_q_lens[i]):int(m.cu_q_lens[i + 1])] for i in range(m.context_lens.numel())}


def _serve(model, xs, plan, seed, together=True):
    """Runs the prompts' rows in the given chunks; returns every request's rows."""
    pools = model.pools()
    free = _free(seed, model.pages)
    table = torch.full((len(xs), 12), -1, dtype=torch.int32, device="cuda")
    done, outs = [0] * len(xs), [[] for _ in xs]
    for take in plan:
        groups = [list(range(len(xs)))] if together else [[i] for i in range(len(xs))]
        for ids in groups:
            new = [take[i] for i in ids]
            if not sum(new):
                continue
            x = torch.cat([xs[i][done[i]:done[i] + take[i]] for i in ids])
            t = table[ids].contiguous()
            out, m = model.step(x, _i32(new), _i32([done[i] for i in ids]), free, t, pools, max(new),
                                max(done[i] + take[i] for i in ids))
            assert (m.status == 0).all()
            table[ids] = t
            free = free[int(m.pages_used):].contiguous()
            for j, rows in _rows(m, out).items():
                outs[ids[j]].append(rows)
                done[ids[j]] += take[ids[j]]
    return [torch.cat(o) for o in outs]


def test_bits_do_not_depend_on_batch_and_chunks():
    model = Model(1, 64)
    xs = [_x(10 + i, n) for i, n in enumerate(PROMPTS)]
    whole = _serve(model, xs, [PROMPTS], 1)
    alone = _serve(model, xs, [PROMPTS], 2, together=False)
    first = [0, 1, 15, 50, 63]
    chunks = _serve(model, xs, [first, [n - f for n, f in zip(PROMPTS, first)]], 3)
    tail = _serve(model, xs, [[max(n - 3, 0) for n in PROMPTS]] + [
        [1 if n > 3 or j < n else 0 for n in PROMPTS] for j in range(3)], 4)
    for i in range(len(xs)):
        assert torch.isfinite(whole[i].float()).all() and whole[i].shape == (PROMPTS[i], H)
        O.same_bits(alone[i], whole[i], i)
        O.same_bits(chunks[i], whole[i], i)
        O.same_bits(tail[i], whole[i], i)


def test_every_operator_of_the_step():
    model = Model(2, 64)
    T = sum(PROMPTS)
    seen = []
    table = torch.full((5, 12), -1, dtype=torch.int32, device="cuda")
    free = _free(7, 64)
    out, m = model.step(_x(3, T), _i32(PROMPTS), _i32([0] * 5), free, table, model.pools(), 130, 130, seen)
    want = O.page_map(PROMPTS, [0] * 5, free.tolist(), np.full((5, 12), -1), 64, T)
    assert m.slot_mapping.tolist() == want["slot_mapping"].tolist()
    assert table.tolist() == want["page_table"].tolist()
    for L in seen:
        w = L["w"]
        x, r = L["first"]
        O.check_codes(*L["q"], O.norm(x, w["n1"], EPS, r)[1], O.NORM_REL)
        O.check_linear(L["qkv"], (*L["q"], *w["qkv"]))
        q, s = O.codes_of(L["o"].float().cpu().numpy())
        O.same_bits(L["oq"][0], q)
        O.same_bits(L["oq"][1], s)
        O.check_linear(L["ao"], (*L["oq"], *w["o"]))
        h, y = O.norm(L["ao"], w["n2"], EPS, L["res"])
        O.same_bits(L["res2"], h)
        O.check_codes(*L["nq"], y, O.NORM_REL)
        O.check_linear(L["up"], (*L["nq"], *w["up"]))
        O.check_codes(*L["gq"], O.gated(L["up"][:, F:], L["up"][:, :F]), O.GATE_REL)
        O.check_linear(L["h"], (*L["gq"], *w["down"]))
    assert torch.isfinite(out.float()).all()


def test_padded_rows_and_refused_requests_leave_the_others():
    """Rows behind the last request, and a request that the free list cannot hold, change no
    other request's rows."""
    model = Model(3, 64)
    T = sum(PROMPTS)
    x = torch.cat([_x(30, T), _x(31, 21)])
    def run(free, rows, q, xx):
        table = torch.full((len(q), 12), -1, dtype=torch.int32, device="cuda")
        return model.step(xx[:rows], _i32(q), _i32([0] * len(q)), free, table, model.pools(), 130, 130)
    ref, _ = run(_free(1, 64), T, PROMPTS, x)
    out, m = run(_free(2, 64), T + 21, PROMPTS, x)
    assert (m.slot_mapping[T:] == -1).all()
    O.same_bits(out[:T], ref)
    # 37, 1 and 16 tokens take 5 pages; the 130 do not fit in the 4 left, nor do the 64 after them
    out, m = run(_free(3, 64)[:9], T, PROMPTS, x)
    assert m.status.tolist() == [0, 0, 0, 4, 4] and m.context_lens.tolist() == [37, 1, 16, 0, 0]
    O.same_bits(out[:54], ref[:54])


def test_graph_replays_equal_eager():
    model = Model(4, 96)
    B, steps = 5, 4
    lens = [30, 7, 64, 1, 100]
    pools, eager_pools = model.pools(), model.pools()
    free = _free(5, 96)
    table = torch.full((B, 12), -1, dtype=torch.int32, device="cuda")
    T = sum(lens)
    x0 = _x(50, T)
    for p in (pools, eager_pools):
        t = table.clone()
        _, m = model.step(x0, _i32(lens), _i32([0] * B), free, t, p, 100, 100)
    table, used = t, int(m.pages_used)
    # buffers of the captured decode step: lengths, tokens, free pages, table
    q_lens, cached = _i32([1] * B), _i32(lens)
    x = _x(60, B + 3)  # (three padding rows)
    pool_free = free[used:].contiguous()
    run = lambda t, p: model.step(x, q_lens, cached, pool_free, t, p, 1, 160)  # noqa: E731
    warm = [(a.clone(), b.clone()) for a, b in pools]
    run(table.clone(), warm)
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    graph_table = table.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            out, m = run(graph_table, pools)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for i in range(steps):
        x.copy_(_x(70 + i, B + 3))
        want, wm = run(table, eager_pools)
        want, wm = want.clone(), wm.context_lens.clone()
        torch.cuda.synchronize()
        out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        O.same_bits(out[:B], want[:B], i)
        O.same_bits(graph_table, table, i)
        for (a, b), (c, d) in zip(pools, eager_pools):
            O.same_bits(a, c, i)
            O.same_bits(b, d, i)
        taken = int(m.pages_used)
        assert wm.tolist() == m.context_lens.tolist()
        cached.copy_(wm)
        pool_free[:pool_free.numel() - taken].copy_(pool_free[taken:].clone())


def test_another_stream():
    """Calls on a stream that is not the current one, by the stream argument and as the
    current stream, give the same bits."""
    model = Model(6, 64)
    x = _x(1, 100)
    w = model.layers[0]
    ref = V.linear_fp8(*V.rmsnorm_fp8(x, w["n1"], EPS), *w["qkv"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q, s = V.rmsnorm_fp8(x, w["n1"], EPS, stream=side)
    a = V.linear_fp8(q, s, *w["qkv"], stream=side)
    with torch.cuda.stream(side):
        b = V.linear_fp8(*V.rmsnorm_fp8(x, w["n1"], EPS), *w["qkv"])
    side.synchronize()
    O.same_bits(a, ref)
    O.same_bits(b, ref)
