"""slimattn_rope_fwd / slimattn_rope_bwd against the plain 64-bit forms of rope_reference.py.

Tolerances.  An output is rounded once to its type: half a step, eps / 2 of the value.  Before that, in 32 bits (u = 2^-24): the mean square is
8 fused steps, up to 4 exchanges and the factor, each u, halved by the root: 7 u, the root and its step 2 u, the two products 2 u; sine and
cosine: angle u * pi / 4, sum 2 u, remainder 2e-9; the rotation 2 u of either product: together below 20 u (|a| + |b|) <= 29 u * length of the pair,
taken as 32 u = 2^-19 of the row's largest pair.  Backward the same for each of its two terms, and the second has two sums: 2^-18 of the terms.
Weight gradients: 32 u for a term and one u for every addition it goes through: up to 48 heads, 6 exchanges, 4 waves, 64 partial sums of a
column and 16 of them: below 2^-16 of the sum of the terms' absolute values."""
import pytest
import torch

import paper_2509_26246_amd as S
import rope_reference as R
from paper_2509_26246_amd import harness as H

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _data(T, hq, hkv, d, dt, seed, fused):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, hq + 2 * hkv, d, generator=g).to(dt)
    gq, gk = ((0.1 * torch.randn(T, h, d, generator=g)).to(dt) for h in (hq, hkv))
    wq, wk = 1 + 0.3 * torch.randn(d, generator=g), 1 + 0.3 * torch.randn(d, generator=g)
    dev = x.cuda()
    q, k = dev[:, :hq], dev[:, hq:hq + hkv]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    return q, k, gq, gk, wq, wk


def _half_step(ref, dt):
    return torch.finfo(dt).eps / 2 * ref.abs()


def _check(name, got, ref, tol):
    err = (got.double().cpu() - ref).abs()
    bad = err > tol
    assert not bad.any(), f"{name}: {int(bad.sum())} values, worst {float((err / tol.clamp_min(1e-300)).max()):.2f} of the tolerance"


def _pair_scale(y):
    """Largest pair length (or value) of each row."""
    return y.abs().amax(-1, keepdim=True) * 2 ** 0.5


def _run(T, hq, hkv, d, dtype, *, norm=True, weights=True, rotary=None, sections=None, dealt=False, adjacent=False, fused=True, positions=None,
         eps=1e-6, seed=0):
    dt, rotary = DT[dtype], d if rotary is None else rotary
    sections = sections or [rotary // 2]
    q, k, gq, gk, wq, wk = _data(T, hq, hkv, d, dt, seed, fused)
    if not (norm and weights):
        wq = wk = None
    if positions is None:
        positions = torch.randint(0, 1 << 20, (len(sections), T), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int32)
    freq = torch.tensor([1e4 ** (-2 * i / max(rotary, 1)) for i in range(rotary // 2)], dtype=torch.float32)
    rot = H.Rotary(hq, hkv, d, dt, freq.cuda() if rotary else None, q_weight=None if wq is None else wq.cuda(),
                   k_weight=None if wk is None else wk.cuda(), norm=norm, eps=eps, rotary_dim=rotary, sections=sections, dealt=dealt,
                   adjacent=adjacent)
    pos = positions.cuda() if rotary else None
    guard = 3                                              # rows behind the last token stay as they were
    outs = [torch.full((T + guard, h, d), 7.0, dtype=dt, device="cuda") for h in (hq, hkv)]
    rot.forward(q, k, pos, *outs)
    dx = torch.full((T, hq + 2 * hkv, d), 7.0, dtype=dt, device="cuda")
    grads = [dx[:, :hq], dx[:, hq:hq + hkv]] if fused else [torch.empty(T, h, d, dtype=dt, device="cuda") for h in (hq, hkv)]
    if norm:
        rot.workspace.fill_(0xFF)
    rot.backward(q, k, pos, gq.cuda(), gk.cuda(), *grads)
    torch.cuda.synchronize()
    assert all((o[T:] == 7).all() for o in outs)
    if fused and hkv:
        assert (dx[:, hq + hkv:] == 7).all()               # the value columns of the projection's gradient
    M = R.rotation(positions, freq, sections, dealt, rotary, d, adjacent)
    for name, x, w, out, gy, dgot, dwgot in (("q", q, wq, outs[0], gq, grads[0], rot.dq_weight), ("k", k, wk, outs[1], gk, grads[1], rot.dk_weight)):
        if x.shape[1] == 0:
            continue
        x = x.cpu()
        ref = R.forward(x, w, M, norm, eps)
        _check(name, out[:T], ref, _half_step(ref, dt) + 2.0 ** -19 * _pair_scale(ref))
        dref, dwref = R.backward(x, w, M, norm, eps, gy)
        if norm:
            xd, g = x.double(), torch.einsum("tji,thj->thi", M, gy.double())
            r = 1 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + eps)
            h = (g * (w.double() if w is not None else 1)).abs()
            terms = r * (h.amax(-1, keepdim=True) + (xd * r).abs().amax(-1, keepdim=True) * (h * (xd * r).abs()).mean(-1, keepdim=True)) * 2 ** 0.5
            _check("d" + name, dgot, dref, _half_step(dref, dt) + 2.0 ** -18 * terms)
            _check(f"d{name}_weight", dwgot, dwref, _half_step(dwref, torch.float32) + 2.0 ** -16 * (g * xd * r).abs().sum((0, 1)))
        else:
            _check("d" + name, dgot, dref, _half_step(dref, dt) + 2.0 ** -19 * _pair_scale(dref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,hq,hkv,d", [(1, 32, 8, 128), (1, 1, 1, 16), (2, 5, 1, 64), (7, 3, 3, 32), (129, 8, 2, 128), (1000, 2, 1, 64), (333, 40, 8, 32)])
def test_sizes(dtype, T, hq, hkv, d):
    _run(T, hq, hkv, d, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm,weights", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rotary,sections,dealt", [(128, 128, [64], False), (128, 96, [16, 16, 16], True), (128, 64, [5, 20, 7], False), (64, 8, [1, 1, 1, 1], True),
                                                     (64, 64, [0, 31, 1, 0], True), (32, 24, [12], False), (16, 16, [3, 5], True), (16, 8, [4], False)])
def test_kinds(dtype, norm, weights, adjacent, d, rotary, sections, dealt):
    _run(37, 4, 2, d, dtype, norm=norm, weights=weights, rotary=rotary, sections=sections, dealt=dealt, adjacent=adjacent)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_alone_queries_alone_keys_alone(dtype):
    _run(19, 4, 2, 64, dtype, rotary=0, sections=[0])
    _run(19, 0, 3, 64, dtype, fused=False)
    _run(19, 3, 0, 64, dtype, fused=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_over_the_whole_range(dtype):
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 1 << 24, (1 << 24) + 1, 123456789], dtype=torch.int32)
    # a turn count of 2^31 / 2 pi in 64 bits is off by 2^-24 of a turn's radians at the most: inside the angle's part of the tolerance
    _run(9, 2, 1, 128, dtype, positions=pos[None])


@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("f32", 16)])
def test_more_tokens_than_the_backward_has_groups(dtype, d):
    _run(70001 if d == 32 else 140001, 1, 1, d, dtype, fused=False)


def test_zero_rows_and_small_and_large_values():
    dt, d = torch.float32, 64
    x = torch.randn(6, 1, d, generator=torch.Generator().manual_seed(1))
    x[0] = 0
    x[1] *= 1e-18
    x[2] *= 1e15
    x[3, 0, 5] = float("nan")
    freq, pos, w = torch.rand(32), torch.arange(6, dtype=torch.int32), torch.rand(d)
    rot = H.Rotary(1, 1, d, dt, freq.cuda(), q_weight=w.cuda(), k_weight=w.cuda(), norm=True, eps=1e-6)
    q, k = x.cuda(), x.cuda().clone()
    out = [torch.empty_like(q), torch.empty_like(k)]
    rot.forward(q, k, pos.cuda(), *out)
    ref = R.forward(x, w, R.rotation(pos, freq, [32], False, d, d, False), True, 1e-6)
    rows = [0, 1, 2, 4, 5]                                  # the row with a NaN is its own affair
    _check("q", out[0][rows], ref[rows], _half_step(ref[rows], dt) + 2.0 ** -19 * _pair_scale(ref[rows]) + 1e-300)
    assert torch.isnan(out[0][3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_gives_the_same_bits(dtype):
    dt, T, hq, hkv, d = DT[dtype], 65, 4, 2, 128
    q, k, gq, gk, wq, wk = _data(T, hq, hkv, d, dt, 5, False)
    gq, gk = gq.cuda(), gk.cuda()
    rot = H.Rotary(hq, hkv, d, dt, torch.rand(64).cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    out, grads = [torch.empty_like(q), torch.empty_like(k)], [torch.empty_like(q), torch.empty_like(k)]
    rot.forward(q, k, pos, *out)
    rot.backward(q, k, pos, gq, gk, *grads)
    dw = rot.dq_weight.clone()
    hq2, hk2 = gq.clone(), gk.clone()
    rot.backward(q, k, pos, hq2, hk2, hq2, hk2)            # over the incoming gradient
    assert torch.equal(hq2, grads[0]) and torch.equal(hk2, grads[1]) and torch.equal(dw, rot.dq_weight)
    q2, k2 = q.clone(), k.clone()
    rot.backward(q2, k2, pos, gq, gk, q2, k2)              # over the inputs
    assert torch.equal(q2, grads[0]) and torch.equal(k2, grads[1])
    q2, k2 = q.clone(), k.clone()
    rot.forward(q2, k2, pos, q2, k2)
    assert torch.equal(q2, out[0]) and torch.equal(k2, out[1])


def test_one_weight_gradient_alone_and_no_tokens():
    d, T = 64, 11
    q, k, gq, gk, wq, wk = _data(T, 2, 1, d, torch.float32, 6, False)
    rot = H.Rotary(2, 1, d, torch.float32, torch.rand(32).cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    grads = [torch.empty_like(q), torch.empty_like(k)]
    rot.backward(q, k, pos, gq.cuda(), gk.cuda(), *grads)
    both = rot.dk_weight.clone()
    rot.dq_weight, keep = None, rot.dq_weight
    rot.dk_weight.fill_(5)
    rot.backward(q, k, pos, gq.cuda(), gk.cuda(), *grads)
    assert torch.equal(both, rot.dk_weight)
    rot.dq_weight = keep
    none = [t[:0] for t in (q, k, pos)]
    rot.backward(*none, gq[:0].cuda(), gk[:0].cuda(), grads[0][:0], grads[1][:0])      # sums over nothing
    assert (rot.dq_weight == 0).all() and (rot.dk_weight == 0).all()


def test_recorded_into_a_graph_and_on_another_stream():
    T, hq, hkv, d, dt = 300, 8, 2, 128, torch.bfloat16
    q, k, gq, gk, wq, wk = _data(T, hq, hkv, d, dt, 7, True)
    gq, gk = gq.cuda(), gk.cuda()
    rot = H.Rotary(hq, hkv, d, dt, torch.rand(64).cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    new = lambda: [torch.zeros(T, h, d, dtype=dt, device="cuda") for h in (hq, hkv, hq, hkv)]

    def step(b):
        rot.forward(q, k, pos, b[0], b[1])
        rot.backward(q, k, pos, gq, gk, b[2], b[3])
    eager, graphed = new(), new()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        step(graphed)
    for i in range(3):
        q.mul_(1.25)
        pos.add_(1000 * i)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(eager)
        torch.cuda.current_stream().wait_stream(side)
        want = [t.clone() for t in eager] + [rot.dq_weight.clone(), rot.dk_weight.clone()]
        rot.dq_weight.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, graphed + [rot.dq_weight, rot.dk_weight]))


def test_binding_refuses_what_is_not_a_matching_tensor():
    d, T = 64, 4
    rot = H.Rotary(2, 1, d, torch.float32, torch.rand(32).cuda(), norm=True)
    q, k, pos = torch.zeros(T, 2, d, device="cuda"), torch.zeros(T, 1, d, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    o = lambda t: torch.empty_like(t)
    for bad in ((q.cpu(), k, pos, o(q), o(k)), (q.half(), k, pos, o(q), o(k)), (q, k[:, :, :32], pos, o(q), o(k)), (q, k, pos.long(), o(q), o(k)),
                (q, k, pos[:2], o(q), o(k)), (q, k, pos, o(q)[:2], o(k)), (q.transpose(0, 1).contiguous().transpose(0, 1), k, pos, o(q), o(k)),
                (q, k, pos, o(q), o(k).cpu())):
        with pytest.raises(ValueError):
            rot.forward(*bad)
    with pytest.raises(S.SlimAttnError):
        rot.forward(q, k, pos, torch.empty(T * 2 * d + 1, device="cuda")[1:], o(k))   # not 16-byte aligned


def test_elements_behind_two_to_the_31():
    T, hq, hkv, d, dt = (1 << 18) + 5, 64, 2, 128, torch.bfloat16
    freq = torch.tensor([1e4 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float32).cuda()
    rot = H.Rotary(hq, hkv, d, dt, freq, norm=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn(T, h, d, generator=g, device="cuda", dtype=dt) for h in (hq, hkv))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    assert q.numel() > 1 << 31
    n = 300
    last = [t[-n:].clone() for t in (q, k)]
    want, outs = [torch.empty_like(t) for t in last], [torch.empty_like(q), torch.empty_like(k)]
    rot.forward(*last, pos[-n:].contiguous(), *want)
    rot.forward(q, k, pos, *outs)
    assert all(torch.equal(a[-n:], b) for a, b in zip(outs, want))
    rot.backward(*last, pos[-n:].contiguous(), *[t[-n:].contiguous() for t in outs], *want)
    rot.backward(q, k, pos, *outs, q, k)                     # (in place of the inputs)
    assert torch.equal(q[-n:], want[0]) and torch.equal(k[-n:], want[1])
