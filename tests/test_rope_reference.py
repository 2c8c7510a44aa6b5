"""The plain 64-bit forms the GPU tests of slimattn_rope_* compare with, pinned on the CPU: a hand-worked rotation, lengths kept, gradients
against differences; and the entry points' refusals, which are decided on the host before anything is launched."""
import math

import numpy as np
import pytest
import torch

import paper_2509_26246_amd as S
import rope_reference as R


def test_pairs_are_dealt_in_turn_or_in_blocks():
    assert R.axis_of_pair([2, 1, 3], False) == [0, 0, 1, 2, 2, 2]
    assert R.axis_of_pair([2, 1, 3], True) == [0, 1, 2, 0, 2, 2]


def test_hand_worked_rotation():
    # one quarter turn of pair 0, none of the others: (a, b) -> (-b, a)
    f = torch.tensor([math.pi / 2, 0.0, 0.0, 0.0])
    x = torch.arange(1.0, 17.0).view(1, 1, 16)
    y = R.forward(x, None, R.rotation(torch.ones(1, 1), f, [4], False, 8, 16, False), False, 0.0)
    assert np.allclose(y[0, 0].numpy(), [-5, 2, 3, 4, 1, 6, 7, 8] + list(range(9, 17)), atol=1e-6)
    y = R.forward(x, None, R.rotation(torch.ones(1, 1), f, [4], False, 8, 16, True), False, 0.0)
    assert np.allclose(y[0, 0].numpy(), [-2, 1] + list(range(3, 17)), atol=1e-6)


@pytest.mark.parametrize("norm,weight", [(True, True), (True, False), (False, False)])
def test_gradients_against_differences(norm, weight):
    g = torch.Generator().manual_seed(3)
    x, dy = torch.randn(3, 2, 16, generator=g, dtype=torch.float64), torch.randn(3, 2, 16, generator=g, dtype=torch.float64)
    w = torch.randn(16, generator=g, dtype=torch.float64) if weight else None
    rot = R.rotation(torch.tensor([[0, 5, 1000], [7, 8, 9]]), torch.rand(4, generator=g), [3, 1], True, 8, 16, False)
    loss = lambda x, w: (R.forward(x, w, rot, norm, 1e-3) * dy).sum()
    dx, dw = R.backward(x, w, rot, norm, 1e-3, dy)
    h = 1e-6
    for _ in range(20):
        i = tuple(int(torch.randint(n, (), generator=g)) for n in x.shape)
        e = torch.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-7
    if weight:
        for c in range(16):
            e = torch.zeros_like(w)
            e[c] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[c]) < 1e-6


# Addresses are never looked at: every call is refused before a launch.
GOOD = dict(total_tokens=8, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=S.BF16, rotary_dim=64, sections=[32], eps=1e-6, flags=S.ROPE_NORM)
A = 1 << 20


def _refused(call, **over):
    ptr = {"q": A, "k": 2 * A, "positions": 3 * A, "inv_freq": 4 * A, "q_out": 5 * A, "k_out": 6 * A, "dq": 7 * A, "dk": 8 * A,
           "dq_weight": 9 * A, "dk_weight": 10 * A, "workspace": 11 * A}
    kw = dict(GOOD)
    for name, v in over.items():
        (ptr if name in ptr else kw)[name] = v
    first = [ptr[n] for n in ("q", "k", "positions", "inv_freq", "q_out", "k_out")]
    with pytest.raises(S.SlimAttnError) as e:
        S.rope_fwd(*first, **kw) if call == "fwd" else S.rope_bwd(*first, *[ptr[n] for n in ("dq", "dk", "dq_weight", "dk_weight", "workspace")], **kw)
    assert e.value.code == -1


BAD = [dict(head_dim=48), dict(head_dim=256), dict(dtype=2), dict(rotary_dim=4, sections=[2]), dict(rotary_dim=72, sections=[36]),
       dict(rotary_dim=-8, sections=[-4]), dict(rotary_dim=0, sections=[0], flags=0), dict(sections=[31]), dict(sections=[33, -1]),
       dict(sections=[8, 8, 8, 4, 4]), dict(sections=[]), dict(eps=0.0), dict(eps=float("nan")), dict(eps=-1.0), dict(eps=float("inf")),
       dict(flags=8), dict(total_tokens=-1), dict(n_q_heads=0, n_kv_heads=0), dict(n_q_heads=-1), dict(n_kv_heads=70000),
       dict(q_stride=4 * 64 - 8), dict(q_stride=4 * 64 + 4), dict(k_stride=-8), dict(q=A + 8), dict(k=0), dict(positions=0), dict(positions=2),
       dict(inv_freq=0), dict(q_out=0), dict(k_out=6 * A + 2), dict(q_weight=1)]


@pytest.mark.parametrize("bad", BAD + [dict(q_out=A + 512), dict(q_out=2 * A), dict(k_out=A), dict(k_out=5 * A + 16),
                                       dict(q_out=A, q_stride=512), dict(q_out=3 * A - 512, k=3 * A - 256)], ids=str)
def test_forward_refuses(bad):
    _refused("fwd", **bad)


@pytest.mark.parametrize("bad", BAD + [dict(dq_stride=4 * 64 + 4), dict(dk_stride=64), dict(workspace=0), dict(workspace=11 * A + 4), dict(dq=7 * A + 8),
                                       dict(dq_weight=2), dict(dq=6 * A), dict(dk=5 * A), dict(dq=A + 512), dict(dq=A, q_stride=512), dict(dk=7 * A + 16),
                                       dict(dq=5 * A, dq_stride=512), dict(dk=7 * A + 512, dq_stride=384, dk_stride=256)], ids=str)
def test_backward_refuses(bad):
    _refused("bwd", **bad)


def test_no_tokens_is_accepted_without_looking_at_tensors():
    S.rope_fwd(0, 0, 0, 0, 0, 0, **dict(GOOD, total_tokens=0))


def test_workspace_is_the_same_for_any_number_of_tokens():
    shape = {k: v for k, v in GOOD.items() if k != "total_tokens"}
    need = {S.rope_bwd_workspace_bytes(t, **shape) for t in (0, 1, 7, 4096, 1 << 20)}
    assert len(need) == 1 and need.pop() > 0
    assert S.rope_bwd_workspace_bytes(64, **dict(shape, flags=0)) == 0 and S.rope_bwd_workspace_bytes(64, **dict(shape, head_dim=48)) == 0


@pytest.mark.parametrize("n", [5, 400])
def test_axes_are_not_looked_at_without_a_rotation(n):
    shape = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=S.BF16, rotary_dim=0, sections=[0] * n, flags=S.ROPE_NORM)
    S.rope_bwd(None, None, None, None, None, None, None, None, None, None, None, total_tokens=0, **shape)


def test_expanded_and_overlapping_rows_are_refused(monkeypatch):
    from paper_2509_26246_amd import binding as B
    monkeypatch.setattr(B, "_current_device", lambda: -1)      # (tensors of the CPU pass for the GPU's: every call is refused before a launch)
    q, k = torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    pos, freq, outs = torch.zeros(8, dtype=torch.int32), torch.ones(32), [torch.zeros_like(q), torch.zeros_like(k)]
    for bad in (q[:1].expand(8, 4, 64), q.flatten().as_strided((8, 4, 64), (64, 64, 1)), q[:, :1].expand(8, 4, 64)):
        with pytest.raises(ValueError):
            S.rope_fwd(bad, k, pos, freq, *outs, **GOOD)
        with pytest.raises(ValueError):
            S.rope_bwd(q, k, pos, freq, *outs, bad, k, None, None, None, **GOOD)


def test_more_tokens_than_a_launch_has_threads_for_are_refused():
    far = dict(total_tokens=(1 << 27) + 1, n_q_heads=1, n_kv_heads=0)
    _refused("fwd", **far, k=0, k_out=0, q=1 << 40, q_out=1 << 42)
    _refused("bwd", **far, k=0, k_out=0, q=1 << 40, q_out=1 << 42, dq=1 << 44)
