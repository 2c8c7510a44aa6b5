"""The calls of one attention layer together, as a program makes them: a training step (norm and rotation, attention, its gradients, the gradients of
norm and rotation) and a server (a prompt through slimattn_fwd and into the 4-bit cache, later slices and single tokens over the cache).

Training, tolerances, in the 2-norm of 32 rows of a head relative to the result's (gradient_bounds).  fp32: a rotated row is off by 2^-19 of its largest pair,
which is at most sqrt(d) = 8 of its root mean square: 1.6e-5; a score by sqrt(2) of that, a probability (over the sum) by twice a score: 4.5e-5; the
backward rotation's terms by 2^-18 of the row's largest: 3e-5; attention itself 4e-6: together below 1e-4.  bf16: attention 4 * 2^-9; q and k rounded to half a
step, 2^-8 each, move a score (64 products, independent roundings) by sqrt(2) * 2^-8 of sqrt(64) / 8 = 1 and a probability by at most twice that; dq, dk rounded
before and after the backward rotation, 2^-8 each: 2^-7 + 2 sqrt(2) * 2^-8 + 2 * 2^-8 < 7 * 2^-8.  A weight's gradient: the same fraction of the sum of its terms' sizes."""
import numpy as np
import pytest
import torch

import cache_reference as C
import gradient_bounds as G
import paper_2509_26246_amd as S
import rope_reference as R
from paper_2509_26246_amd import harness as H
from test_gpu_cache import _cache, _check_attend, _ptr, _same

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HQ, HKV, D = 4, 2, 64


def _freq(d=D):
    return torch.tensor([1e4 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float32)


def _attention(q, k, v, cu, scale):
    """Packed causal attention in 64 bits, differentiable."""
    out = []
    for a, b in zip(cu[:-1], cu[1:]):
        kk, vv = (x[a:b].repeat_interleave(HQ // HKV, 1).transpose(0, 1) for x in (k, v))
        s = scale * (q[a:b].transpose(0, 1) @ kk.transpose(1, 2).contiguous())
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), -torch.inf)
        out.append((s.softmax(-1) @ vv).transpose(0, 1))
    return torch.cat(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_step(dtype):
    dt, scale, eps = DT[dtype], D ** -0.5, 1e-6
    L = [200, 1, 131, 64, 37]
    T, cu0 = sum(L), [0] + list(np.cumsum(L))
    g = torch.Generator().manual_seed(5)
    x = torch.randn(T, HQ + 2 * HKV, D, generator=g).to(dt)
    do = (0.1 * torch.randn(T, HQ, D, generator=g)).to(dt)
    wq, wk = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in L])

    # on the device: columns of one projection, gradients into columns of one buffer
    cu, sl = S.build_slices(L, 64)
    units = [S.build_units(cu, sl, "TOKEN_CAP", cap=128, backward=b) for b in (False, True)]
    z = [np.zeros((T, h, D), np.float32) for h in (HQ, HKV, HKV, HQ)]
    prob = H.make_problem(*z, cu, sl, *units, bf16=dtype == "bf16", scale=scale)
    proj, dproj = x.cuda(), torch.full((T, HQ + 2 * HKV, D), float("nan"), dtype=dt, device="cuda")
    rot = H.Rotary(HQ, HKV, D, dt, _freq().cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True, eps=eps)
    dpos = pos.cuda()

    def step():
        rot.forward(proj[:, :HQ], proj[:, HQ:HQ + HKV], dpos, prob.q, prob.k)
        prob.v.copy_(proj[:, HQ + HKV:])
        prob.forward()
        prob.backward()
        rot.backward(proj[:, :HQ], proj[:, HQ:HQ + HKV], dpos, prob.dQ, prob.dK, dproj[:, :HQ], dproj[:, HQ:HQ + HKV])
        dproj[:, HQ + HKV:].copy_(prob.dV)

    prob.dO.copy_(do)
    step()
    torch.cuda.synchronize()
    got = [t.clone() for t in (prob.o, dproj, rot.dq_weight, rot.dk_weight)]

    # in 64 bits, by automatic differentiation
    xr, wqr, wkr = (t.double().requires_grad_() for t in (x, wq, wk))
    M = R.rotation(pos, _freq(), [D // 2], False, D, D, False)
    turned = []
    for a, w in ((xr[:, :HQ], wqr), (xr[:, HQ:HQ + HKV], wkr)):
        n = a / torch.sqrt((a * a).mean(-1, keepdim=True) + eps)
        turned.append((M[:, None] @ (n * w)[..., None])[..., 0])
    o = _attention(*turned, xr[:, HQ + HKV:], cu0, scale)
    loss = (o * do.double()).sum()
    loss.backward()
    tol = 7 * 2.0 ** -8 if dtype == "bf16" else 1e-4
    assert G.worst_block(got[0].float().cpu().numpy(), o.detach().numpy()) <= tol
    dx = got[1].float().cpu().numpy()
    for name, a, b in (("dQ", 0, HQ), ("dK", HQ, HQ + HKV), ("dV", HQ + HKV, HQ + 2 * HKV)):
        e = G.relative_error(name, dx[:, a:b], xr.grad[:, a:b].numpy())
        assert e <= tol, f"{name}: {e:.2e}"
    for name, dw, ref, a, b, w in (("q", got[2], wqr.grad, 0, HQ, wqr), ("k", got[3], wkr.grad, HQ, HQ + HKV, wkr)):
        h = x[:, a:b].double()
        gy = torch.einsum("tji,thj->thi", M, torch.from_numpy(dx[:, a:b]).double().abs())     # sizes only
        terms = (gy.abs().amax(-1, keepdim=True) * h.abs()).sum((0, 1)) + 1e-30
        assert ((dw.double().cpu() - ref).abs() <= 4 * tol * terms).all(), name

    # and against differences: the loss along a direction, both sides of the point, in 64 bits
    u = torch.randn(x.shape, generator=g).double()

    def value(t):
        y = x.double() + t * u
        rows = [R.forward(y[:, :HQ], wq, M, True, eps), R.forward(y[:, HQ:HQ + HKV], wk, M, True, eps)]
        return float((_attention(*rows, y[:, HQ + HKV:], cu0, scale) * do.double()).sum())

    slope = (value(1e-4) - value(-1e-4)) / 2e-4
    along = float((torch.from_numpy(dx).double() * u).sum())
    size = float(np.linalg.norm(dx.astype(np.float64)) * u.norm() / u.numel() ** 0.5)         # a random direction sees 1 / sqrt(n) of the norms' product
    assert abs(slope - along) <= (6 * tol + 1e-6) * size, (slope, along, size)

    # recorded once and replayed, with eager work between: the same bits
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        for t in (prob.o, dproj, rot.dq_weight, rot.dk_weight):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (prob.o, dproj, rot.dq_weight, rot.dk_weight)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_server(dtype):
    dt, scale, page = DT[dtype], D ** -0.5, 16
    u8 = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    first, later, steps = [130, 1, 47], [70, 0, 3], 4                 # prompts, a later slice of some, then single tokens
    n = len(first)
    total = [a + b + steps for a, b in zip(first, later)]
    g = torch.Generator().manual_seed(6)
    x = [torch.randn(t, HQ + 2 * HKV, D, generator=g).to(dt) for t in total]
    wq, wk = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
    rot = H.Rotary(HQ, HKV, D, dt, _freq().cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True)
    c = _cache(total, HKV, D, dt, page, max_rows=sum(later), hq=HQ)
    c.lens.zero_()
    keys = [torch.zeros(0, HKV, D) for _ in range(n)]                 # what the cache has to hold
    values = [torch.zeros(0, HKV, D) for _ in range(n)]

    def rotated(rows, q, k, rows_pos):
        """q, k of the call against 64 bits: half a step and 2^-19 of the row's largest pair."""
        M = R.rotation(rows_pos, _freq(), [D // 2], False, D, D, False)
        for got, a, b, w in ((q, 0, HQ, wq), (k, HQ, HQ + HKV, wk)):
            ref = R.forward(rows[:, a:b], w, M, True, 1e-6)
            err = (got.double().cpu() - ref).abs()
            assert (err <= u8 * ref.abs() + 2.0 ** -19 * ref.abs().amax(-1, keepdim=True) * 2 ** 0.5).all()

    def held(rows, k, counts):
        at = 0
        for b, m in enumerate(counts):
            keys[b] = torch.cat([keys[b], C.held(k[at:at + m].cpu())])
            values[b] = torch.cat([values[b], C.held(rows[at:at + m, HQ + HKV:])])
            at += m

    # the prompts: rotation, attention over the rows themselves, keys and values into the cache
    rows = torch.cat([a[:m] for a, m in zip(x, first)])
    pos = torch.cat([torch.arange(m, dtype=torch.int32) for m in first])
    proj = rows.cuda()
    q, k = torch.empty(len(rows), HQ, D, dtype=dt, device="cuda"), torch.empty(len(rows), HKV, D, dtype=dt, device="cuda")
    c.lens.copy_(torch.tensor(first))
    rot.forward(proj[:, :HQ], proj[:, HQ:HQ + HKV], pos.cuda(), q, k)
    c.write(k, proj[:, HQ + HKV:], _ptr(first))
    torch.cuda.synchronize()
    rotated(rows, q, k, pos)
    held(rows, k, first)
    # read back, what slimattn_fwd then gives is what attention over the cache gives: each within its roundings (of P, the output, in fp32 the scores) of 64 bits
    kk, vv = torch.empty_like(k), torch.empty_like(k)
    c.read(kk, vv, _ptr(first))
    _same(kk, torch.cat(keys))
    _same(vv, torch.cat(values))
    cu, sl = S.build_slices(first, 64)
    units = [S.build_units(cu, sl, "TOKEN_CAP", cap=128, backward=b) for b in (False, True)]
    prob = H.make_problem(*[np.zeros((len(rows), h, D), np.float32) for h in (HQ, HKV, HKV, HQ)], cu, sl, *units, bf16=dtype == "bf16", scale=scale)
    prob.q.copy_(q), prob.k.copy_(kk), prob.v.copy_(vv)
    prob.forward()
    want, at = [], 0
    for b, m in enumerate(first):
        want.append(C.attend(q[at:at + m].cpu(), keys[b], values[b], HQ // HKV, scale, 0)[0])
        at += m
    assert G.worst_block(prob.o.float().cpu().numpy(), torch.cat(want).numpy()) <= (G.REL_BF16 if dtype == "bf16" else G.REL_F32)

    # later slices: several rows of a sequence at once, none of another
    rows = torch.cat([a[m:m + w] for a, m, w in zip(x, first, later)])
    pos = torch.cat([torch.arange(m, m + w, dtype=torch.int32) for m, w in zip(first, later)])
    proj = rows.cuda()
    q, k = torch.empty(len(rows), HQ, D, dtype=dt, device="cuda"), torch.empty(len(rows), HKV, D, dtype=dt, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(HQ, len(rows), device="cuda")
    c.lens += torch.tensor(later, dtype=torch.int32).cuda()
    rot.forward(proj[:, :HQ], proj[:, HQ:HQ + HKV], pos.cuda(), q, k)
    c.write(k, proj[:, HQ + HKV:], _ptr(later))
    c.attend(q, o, lse, scale, _ptr(later))
    torch.cuda.synchronize()
    rotated(rows, q, k, pos)
    held(rows, k, later)
    lens = [a + b for a, b in zip(first, later)]
    _check_attend(o, lse, q.cpu(), torch.cat(keys), torch.cat(values), lens, later, HQ // HKV, scale, dt)

    # single tokens: one step recorded, replayed for each; lengths, positions and rows change in place
    proj = torch.zeros(n, HQ + 2 * HKV, D, dtype=dt, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    q, k = torch.empty(n, HQ, D, dtype=dt, device="cuda"), torch.empty(n, HKV, D, dtype=dt, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(HQ, n, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        pos.copy_(c.lens)
        c.lens += 1
        rot.forward(proj[:, :HQ], proj[:, HQ:HQ + HKV], pos, q, k)
        c.write(k, proj[:, HQ + HKV:])
        c.attend(q, o, lse, scale)
    for i in range(steps):
        rows = torch.stack([a[m + i] for a, m in zip(x, lens)])
        proj.copy_(rows)
        graph.replay()
        torch.cuda.synchronize()
        at = torch.tensor([m + i for m in lens], dtype=torch.int32)
        assert torch.equal(c.lens.cpu(), at + 1) and torch.equal(pos.cpu(), at)
        rotated(rows, q, k, at)
        held(rows, k, [1] * n)
        _check_attend(o, lse, q.cpu(), torch.cat(keys), torch.cat(values), [m + i + 1 for m in lens], [1] * n, HQ // HKV, scale, dt)
