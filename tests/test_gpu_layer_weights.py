"""Gradients of the norm weights behind a training step of one attention layer, with a bound that a wrong gradient does not pass.

dw_c = sum over tokens and heads of g_tc y_tc, with y = x r the normed rows (mean square 1) and g the gradient of the weighted rows.  g is off by `tol` of its 2-norm in
every 32 rows of a head (test_gpu_layer derives 7 * 2^-8 in bf16 and 1e-4 in fp32).  These errors are of either sign, so the vector dw is off by about
sqrt(sum (tol g y)^2) = tol |g|; twice that is allowed.  A sum of terms of either sign is about as long as they are: |dw| is near |g|, the bound 5% of it in
bf16.  The first tests plant mistakes in the oracle and need no GPU."""
from functools import lru_cache

import numpy as np
import pytest
import torch

import paper_2509_26246_amd as S
import rope_reference as R
from paper_2509_26246_amd import harness as H
from test_gpu_layer import D, DT, HKV, HQ, _attention, _freq

TOL = {"bf16": 7 * 2.0 ** -8, "f32": 1e-4}
L = [200, 1, 131, 64, 37]
EPS, SCALE = 1e-6, D ** -0.5


def _inputs(dtype):
    g = torch.Generator().manual_seed(11)
    T = sum(L)
    x = torch.randn(T, HQ + 2 * HKV, D, generator=g).to(DT[dtype])
    do = (0.1 * torch.randn(T, HQ, D, generator=g)).to(DT[dtype])
    return x, do, 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g), torch.cat([torch.arange(n, dtype=torch.int32) for n in L])


@lru_cache(maxsize=None)
def _reference(dtype):
    """For q and k: dw, g and y in 64 bits, by automatic differentiation; and the gradient of the turned rows."""
    x, do, wq, wk, pos = _inputs(dtype)
    M = R.rotation(pos, _freq(), [D // 2], False, D, D, False)
    parts, turned = [], []
    for rows, w in ((x[:, :HQ], wq), (x[:, HQ:HQ + HKV], wk)):
        a, w = rows.double(), w.double().requires_grad_()
        y = a / torch.sqrt((a * a).mean(-1, keepdim=True) + EPS)
        weighted = (y * w).requires_grad_()
        weighted.retain_grad()
        turned.append((M[:, None] @ weighted[..., None])[..., 0])
        turned[-1].retain_grad()
        parts.append((a, w, y, weighted))
    (_attention(*turned, x[:, HQ + HKV:].double(), [0] + list(np.cumsum(L)), SCALE) * do.double()).sum().backward()
    return [dict(dw=w.grad, g=n.grad, y=y.detach(), x=a, turned=t.grad) for (a, w, y, n), t in zip(parts, turned)]


def _bound(ref, dtype):
    return 2 * TOL[dtype] * float(ref["g"].norm())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_bound_is_passed_by_no_wrong_gradient(dtype):
    refs = _reference(dtype)
    for ref, other in zip(refs, refs[::-1]):
        dw, g, y, bound = ref["dw"], ref["g"], ref["y"], _bound(ref, dtype)
        assert torch.allclose(dw, (g * y).sum((0, 1)))
        assert dw.norm() > 8 * bound
        wrong = {"nothing": 0 * dw, "the other sign": -dw, "the other weight's": other["dw"], "rows without their norm": (g * ref["x"]).sum((0, 1)),
                 "not turned back": (ref["turned"] * y).sum((0, 1)), "a head less": (g * y)[:, 1:].sum((0, 1)), "32 tokens less": (g * y)[:-32].sum((0, 1)),
                 "twice a token": dw + (g * y)[g.norm(dim=(1, 2)).argmax()].sum(0), "halves swapped": dw.roll(D // 2)}
        for name, w in wrong.items():
            if name == "rows without their norm":          # (random rows have a norm near 1 of their own: told apart in full precision only)
                if dtype == "bf16":
                    continue
            assert (w - dw).norm() > bound, name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradients_of_a_training_step(dtype):
    x, do, wq, wk, pos = _inputs(dtype)
    cu, sl = S.build_slices(L, 64)
    units = [S.build_units(cu, sl, "TOKEN_CAP", cap=128, backward=b) for b in (False, True)]
    z = [np.zeros((sum(L), h, D), np.float32) for h in (HQ, HKV, HKV, HQ)]
    prob = H.make_problem(*z, cu, sl, *units, bf16=dtype == "bf16", scale=SCALE)
    rot = H.Rotary(HQ, HKV, D, DT[dtype], _freq().cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), norm=True, eps=EPS)
    x, pos = x.cuda(), pos.cuda()
    dx = torch.empty_like(x)
    rot.forward(x[:, :HQ], x[:, HQ:HQ + HKV], pos, prob.q, prob.k)
    prob.v.copy_(x[:, HQ + HKV:])
    prob.dO.copy_(do)
    prob.forward()
    prob.backward()
    rot.backward(x[:, :HQ], x[:, HQ:HQ + HKV], pos, prob.dQ, prob.dK, dx[:, :HQ], dx[:, HQ:HQ + HKV])
    for got, ref in zip((rot.dq_weight, rot.dk_weight), _reference(dtype)):
        err = float((got.double().cpu() - ref["dw"]).norm())
        assert err <= _bound(ref, dtype), f"{err / _bound(ref, dtype):.2f} of the bound"
