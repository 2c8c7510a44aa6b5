"""Tensors whose memory does not lie as the operators would read it are refused by their shapes, before a launch; those that lie so by another shape are
taken; outputs that lie over anything else of the call are refused.  Tensors of the CPU stand for the GPU's, and addresses are never looked at: no call here
reaches a kernel."""
import pytest
import torch

import paper_2509_26246_amd as S
from paper_2509_26246_amd import binding as B
from paper_2509_26246_amd import harness as H

T, HQ, HKV, D = 8, 4, 2, 64
ROPE = dict(total_tokens=T, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, dtype=S.F32, rotary_dim=D, sections=[16, 8, 8], flags=S.ROPE_NORM)
CACHE = dict(n_rows=4, n_pages=8, page_size=16, n_kv_heads=HKV, head_dim=D, dtype=S.F32, n_seqs=4, max_pages=4)


@pytest.fixture(autouse=True)
def _cpu_for_gpu(monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: -1)


def _f(*shape):
    return torch.zeros(*shape)


def _i(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _rope(call, over):
    t = dict(q=_f(T, HQ, D), k=_f(T, HKV, D), positions=_i(3, T), inv_freq=_f(D // 2), q_out=_f(T, HQ, D), k_out=_f(T, HKV, D), q_weight=_f(D), k_weight=_f(D),
             dq=_f(T, HQ, D), dk=_f(T, HKV, D), dq_weight=_f(D), dk_weight=_f(D), workspace=torch.zeros(1 << 21, dtype=torch.uint8))
    t.update(over)
    first = [t[n] for n in ("q", "k", "positions", "inv_freq", "q_out", "k_out")]
    weights = dict(q_weight=t["q_weight"], k_weight=t["k_weight"])
    if call == "fwd":
        S.rope_fwd(*first, **weights, **ROPE)
    else:
        S.rope_bwd(*first, *[t[n] for n in ("dq", "dk", "dq_weight", "dk_weight", "workspace")], **weights, **ROPE)


def _cache(call, over):
    t = dict(k=_f(4, HKV, D), v=_f(4, HKV, D), cache=torch.zeros(8 * 16 * HKV * 72, dtype=torch.uint8), page_table=_i(4, 4), lens=_i(4), q=_f(4, HQ, D), o=_f(4, HQ, D),
             lse=_f(HQ, 4), workspace=torch.zeros(1 << 25, dtype=torch.uint8))
    t.update(over)
    if call == "write":
        S.cache_write(t["k"], t["v"], t["cache"], t["page_table"], t["lens"], **CACHE)
    elif call == "read":
        S.cache_read(t["cache"], t["page_table"], t["lens"], t["k"], t["v"], **CACHE)
    else:
        S.cache_attn(t["q"], t["cache"], t["page_table"], t["lens"], t["o"], t["lse"], t["workspace"], n_q_heads=HQ, scale=0.1, **CACHE)


FORWARD = [dict(positions=_i(3, T + 1)), dict(positions=_i(T, 3)), dict(positions=_i(3 * T + 1)), dict(positions=_i(3, 1, T + 2)), dict(inv_freq=_f(D)), dict(q_weight=_f(HQ, D)),
           dict(k_weight=_f(2 * D)), dict(q_out=_f(T, 2 * HQ, D)), dict(q_out=_f(T, HQ, 2 * D)), dict(k_out=_f(2, T, HKV, D)), dict(k_out=_f(T, D, HKV)), dict(q_out=_f(T, 2 * HQ * D))]


@pytest.mark.parametrize("call,bad", [("fwd", b) for b in FORWARD] + [("bwd", b) for b in FORWARD + [dict(dq_weight=_f(HQ, D)), dict(dk_weight=_f(D + 1))]],
                         ids=lambda x: x if isinstance(x, str) else "-".join(f"{k}{tuple(v.shape)}" for k, v in x.items()))
def test_rotation_refuses(call, bad):
    with pytest.raises(ValueError):
        _rope(call, bad)


TABLES = [dict(page_table=_i(4, 5)), dict(page_table=_i(8, 3))]


@pytest.mark.parametrize("call,bad", [("write", b) for b in TABLES] + [("read", b) for b in TABLES + [dict(k=_f(4, 2 * HKV, D)), dict(v=_f(4, HKV, 2 * D)), dict(v=_f(3, 4, HKV, D))]]
                         + [("attn", b) for b in TABLES + [dict(lse=_f(HQ, 6)), dict(lse=_f(4 * HQ + 1)), dict(lse=_f(2 * HQ, 4)), dict(q=_f(4, 2 * HQ, D)),
                                                           dict(o=_f(4, 2 * HQ, D)), dict(q=_f(4, HQ, 2 * D)), dict(q=_f(4, D, HQ))]],
                         ids=lambda x: x if isinstance(x, str) else "-".join(f"{k}{tuple(v.shape)}" for k, v in x.items()))
def test_cache_refuses(call, bad):
    with pytest.raises(ValueError):
        _cache(call, bad)


@pytest.mark.parametrize("shape", [(T, HQ, D), (T + 3, HQ, D), (T, HQ * D), (T + 3, HQ * D), (T * HQ * D,), (T * HQ * D + 5,), (2, T // 2, HQ, D), (T, 2, HQ // 2, D)], ids=str)
def test_packed_rows_by_another_shape_are_taken(shape):
    x = _f(*shape)
    assert B._packed_ptr(x, T, HQ, D, torch.float32, "x", -1) == x.data_ptr()


@pytest.mark.parametrize("lines,n,shape,more", [(3, T, (3, T), False), (3, T, (3 * T,), False), (1, T, (T,), False), (1, T, (T + 4,), False), (1, T, (1, T + 4), False),
                                                (HQ, T, (2, HQ // 2, T), False), (3, 5, (4, 5), True), (3, 5, (20,), True), (3, 0, (3, 0), False)], ids=str)
def test_lines_by_another_shape_are_taken(lines, n, shape, more):
    x = _f(*shape)
    assert B._lines_ptr(x, torch.float32, lines, n, "x", -1, more) == x.data_ptr()


def test_ambiguous_heads_are_not_guessed():
    for shape in ((T, 2, D), (2, T, D), (T // 2, D), (T, 2 * D)):
        with pytest.raises(ValueError):
            B._packed_ptr(_f(*shape), T, 1, D, torch.float32, "x", -1)


@pytest.mark.parametrize("weights", [dict(q_weight=_f(D)), dict(k_weight=_f(D)), dict(q_weight=_f(D), k_weight=_f(D))], ids=lambda w: "-".join(w))
def test_weights_without_a_norm_are_refused(weights):
    with pytest.raises(ValueError):
        H.Rotary(HQ, HKV, D, torch.float32, _f(D // 2), device="cpu", **weights)
    H.Rotary(HQ, HKV, D, torch.float32, _f(D // 2), norm=True, device="cpu", **weights)
    H.Rotary(HQ, HKV, D, torch.float32, _f(D // 2), device="cpu")


A = 1 << 32


def _overlaps_rope(call, over, **shape):
    ptr = {n: (i + 1) * A for i, n in enumerate(("q", "k", "positions", "inv_freq", "q_out", "k_out", "dq", "dk", "dq_weight", "dk_weight", "workspace", "q_weight", "k_weight"))}
    ptr.update({n: (ptr[v[0]] + v[1]) for n, v in over.items()})
    kw = dict(ROPE, q_weight=ptr["q_weight"], k_weight=ptr["k_weight"], **shape)
    first = [ptr[n] for n in ("q", "k", "positions", "inv_freq", "q_out", "k_out")]
    with pytest.raises(S.SlimAttnError) as e:
        S.rope_fwd(*first, **kw) if call == "fwd" else S.rope_bwd(*first, *[ptr[n] for n in ("dq", "dk", "dq_weight", "dk_weight", "workspace")], **kw)
    assert e.value.code == -1


ROW = HQ * D * 4                                           # bytes of a token's queries


@pytest.mark.parametrize("over", [dict(positions=("q_out", 0)), dict(positions=("q_out", T * ROW - 4)), dict(positions=("q_out", -4)), dict(inv_freq=("k_out", 64)),
                                  dict(q_weight=("q_out", 256)), dict(k_weight=("q_out", 4)), dict(k_weight=("k_out", -D * 4 + 4))], ids=str)
def test_forward_refuses_outputs_over_its_other_inputs(over):
    _overlaps_rope("fwd", over)


@pytest.mark.parametrize("over", [dict(dk_weight=("dq_weight", 0)), dict(dk_weight=("dq_weight", D * 4 - 4)), dict(dq_weight=("dk_weight", 4)), dict(dq_weight=("workspace", 64)),
                                  dict(workspace=("dk_weight", -1024)), dict(workspace=("dq", 0)), dict(workspace=("dk_out_", 0)), dict(workspace=("q", -4096)),
                                  dict(dq_weight=("dq", ROW)), dict(dk_weight=("k", 0)), dict(dq_weight=("q_weight", 0)), dict(positions=("dq", 0)), dict(inv_freq=("dk", 8)),
                                  dict(q_weight=("dq", 0)), dict(positions=("workspace", 0)), dict(dk_weight=("inv_freq", 0))], ids=str)
def test_backward_refuses_outputs_over_anything(over):
    _overlaps_rope("bwd", {n: ((v[0] if v[0] != "dk_out_" else "k_out"), v[1]) for n, v in over.items()})


def test_rows_with_room_between_them():
    # the gradients of a fused projection: what lies over a row is refused, also over the last one and over two at once
    for at in (0, ROW - 4, 3 * ROW - 4, 3 * ROW, 7 * 3 * ROW + ROW - 4, ROW - D * 4 + 4, 3 * ROW - D * 4 + 4):
        _overlaps_rope("bwd", dict(dq_weight=("dq", at)), dq_stride=3 * HQ * D)


def _overlaps_cache(call, over):
    ptr = {n: (i + 1) * A for i, n in enumerate(("k", "v", "cache", "page_table", "lens", "row_ptr", "q", "o", "lse", "workspace"))}
    ptr.update({n: ptr[v[0]] + v[1] for n, v in over.items()})
    with pytest.raises(S.SlimAttnError) as e:
        if call == "write":
            S.cache_write(ptr["k"], ptr["v"], ptr["cache"], ptr["page_table"], ptr["lens"], ptr["row_ptr"], **CACHE)
        elif call == "read":
            S.cache_read(ptr["cache"], ptr["page_table"], ptr["lens"], ptr["k"], ptr["v"], ptr["row_ptr"], **CACHE)
        else:
            S.cache_attn(*[ptr[n] for n in ("q", "cache", "page_table", "lens", "o", "lse", "workspace", "row_ptr")], n_q_heads=HQ, scale=0.1, **CACHE)
    assert e.value.code == -1


ARRAYS = [("lens", 0), ("lens", 12), ("page_table", 60), ("row_ptr", 16)]


@pytest.mark.parametrize("call,over", [(call, {n: (out, 16 - at)}) for call, outs in (("write", ("cache",)), ("read", ("k", "v")), ("attn", ("o", "lse", "workspace"))) for out in outs for n, at in ARRAYS]
                         + [("attn", o) for o in (dict(lse=("o", 4)), dict(lse=("q", 0)), dict(workspace=("o", 16)), dict(o=("workspace", 1024)), dict(lse=("workspace", 0)),
                                                  dict(workspace=("q", 0)), dict(workspace=("cache", 0)), dict(o=("cache", 64)), dict(lse=("cache", 0)), dict(o=("q", 16)))], ids=str)
def test_cache_calls_refuse_outputs_over_anything(call, over):
    _overlaps_cache(call, over)


@pytest.mark.parametrize("scale", [3.4e38, -3.0e38, 1.8e38, float("inf"), float("nan")])
def test_scales_beyond_the_exponentials_units_are_refused(scale):
    # the kernels work in units of log 2: a finite scale whose product with log2 e is not made every row NaN; the limit is 2^127 = 1.7e38
    ptr = {n: (i + 1) * A for i, n in enumerate(("q", "cache", "page_table", "lens", "o", "lse", "workspace"))}
    with pytest.raises(S.SlimAttnError) as e:
        S.cache_attn(*ptr.values(), n_q_heads=HQ, scale=scale, **CACHE)
    assert e.value.code == -1
