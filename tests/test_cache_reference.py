"""The plain 64-bit cache of cache_reference.py, pinned on the CPU to values worked by hand; and the entry points' refusals, decided on the host."""
import math

import pytest
import torch

import cache_reference as R
import paper_2509_26246_amd as S


def test_hand_worked_groups():
    # a = 6 -> s = 1: every border of the eight levels goes to the even code
    x = torch.tensor([6, -6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.75, 2.5, 2.6, 3.5, 5.0, 5.1, 0, -0.3, -5.0] + [0] * 16, dtype=torch.float64)
    want = [6, -6, 0, 0.5, 1, 0.5, 1, 2, 2, 3, 4, 4, 6, 0, -0.5, -4] + [0] * 16
    assert R.held(x).tolist() == want
    # a = 1 -> 1/6 = 0.101010|1010..b to six bits: 43/256; 1 / s = 5.95 -> 6 s
    x = torch.zeros(32, dtype=torch.float64)
    x[3], x[5] = 1.0, -0.1
    y = R.held(x)
    assert y[3] == 6 * 43 / 256 and y[5] == -0.5 * 43 / 256
    x[0] = math.inf
    assert torch.isnan(R.held(x)).all()
    assert (R.held(torch.full((32,), 2.0 ** -101)) == 0).all()
    big = torch.full((32,), 3.4e38)
    assert (R.held(big) == 6 * 1.3125 * 2.0 ** 125).all() and torch.isfinite(R.held(big).to(torch.bfloat16)).all()


def test_every_value_is_a_bf16_number():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2000, 32, generator=g) * torch.exp(20 * torch.randn(2000, 1, generator=g))
    y = R.held(x)
    assert torch.equal(y.nan_to_num(1), y.to(torch.bfloat16).double().nan_to_num(1))
    a = x.double().abs().amax(-1)
    kept = (a >= 2.0 ** -100) & (a < 2.0 ** 127)           # below a group is zero, above its scale is held back
    err = ((y - x.double()).abs().amax(-1) / a)[kept]
    assert kept.sum() > 1900 and err.max() <= (1 + 2.0 ** -6) / 6 + 2.0 ** -6    # half the largest step, and what a rounded scale leaves above six


def test_attention_sees_up_to_its_row():
    q, k, v = torch.ones(2, 1, 4), torch.zeros(3, 1, 4), torch.arange(12.0).view(3, 1, 4)
    o, lse, _ = R.attend(q, k, v, 1, 1.0, 1)
    assert torch.allclose(o[0, 0], v[:2, 0].double().mean(0)) and torch.allclose(o[1, 0], v[:, 0].double().mean(0))
    assert torch.allclose(lse[0], torch.tensor([2.0, 3.0], dtype=torch.float64).log())
    o, lse, _ = R.attend(q, k[:1], v[:1], 1, 1.0, -1)
    assert (o[0] == 0).all() and lse[0, 0] == -math.inf and lse[0, 1] == 0


A = 1 << 32
GOOD = dict(n_rows=4, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, dtype=S.BF16, n_seqs=4, max_pages=4)
PTR = dict(k=A, v=2 * A, cache=3 * A, page_table=4 * A, lens=5 * A, q=6 * A, o=7 * A, lse=8 * A, workspace=9 * A, row_ptr=None)


def _call(call, over):
    ptr, kw = dict(PTR), dict(GOOD)
    strides = {}
    for name, x in over.items():
        if name in ("k_stride", "v_stride"):
            strides[name] = x
        elif name in ("n_q_heads", "scale"):
            kw[name] = x
        else:
            (ptr if name in ptr else kw)[name] = x
    if call == "write":
        return S.cache_write(ptr["k"], ptr["v"], ptr["cache"], ptr["page_table"], ptr["lens"], ptr["row_ptr"], **strides, **kw)
    if call == "read":
        return S.cache_read(ptr["cache"], ptr["page_table"], ptr["lens"], ptr["k"], ptr["v"], ptr["row_ptr"], **kw)
    kw.setdefault("n_q_heads", 8)
    kw.setdefault("scale", 0.1)
    return S.cache_attn(ptr["q"], ptr["cache"], ptr["page_table"], ptr["lens"], ptr["o"], ptr["lse"], ptr["workspace"], ptr["row_ptr"], **kw)


BAD = [dict(n_pages=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(n_kv_heads=0), dict(head_dim=32), dict(head_dim=96),
       dict(dtype=7), dict(n_seqs=-1), dict(n_seqs=65537, n_rows=65537), dict(max_pages=0), dict(max_pages=1 << 27), dict(n_rows=-1), dict(n_rows=5),
       dict(row_ptr=2), dict(lens=0), dict(lens=5 * A + 1), dict(page_table=0), dict(cache=0), dict(cache=3 * A + 8)]


@pytest.mark.parametrize("call,bad", [("write", b) for b in BAD + [dict(k=0), dict(v=2 * A + 2), dict(k_stride=64), dict(v_stride=132), dict(k_stride=-128),
                                                                   dict(k=3 * A + 16), dict(v=3 * A - 16)]]
                         + [("read", b) for b in BAD + [dict(k=0), dict(v=2 * A + 8), dict(v=A), dict(k=2 * A - 16), dict(k=3 * A), dict(v=3 * A + 16)]]
                         + [("attn", b) for b in BAD + [dict(n_q_heads=0), dict(n_q_heads=7), dict(n_q_heads=-2), dict(scale=float("nan")), dict(scale=float("inf")),
                                                        dict(q=0), dict(o=7 * A + 8), dict(lse=8 * A + 2), dict(workspace=0), dict(workspace=9 * A + 4),
                                                        dict(o=6 * A), dict(o=6 * A + 16)]], ids=str)
def test_refuses(call, bad):
    with pytest.raises(S.SlimAttnError) as e:
        _call(call, bad)
    assert e.value.code == -1


@pytest.mark.parametrize("call", ["write", "read", "attn"])
def test_nothing_to_do_is_accepted(call):
    _call(call, dict(n_rows=0, n_seqs=0, k=0, v=0, q=0, o=0, lens=0, page_table=0, cache=3 * A))
    _call(call, dict(n_rows=0, row_ptr=16))


def test_sizes():
    assert S.cache_bytes(8, 16, 2, 64) == 8 * 16 * 2 * 72 and S.cache_bytes(1, 256, 8, 128) == 256 * 8 * 144
    assert S.cache_bytes(0, 16, 2, 64) == 0 and S.cache_bytes(8, 24, 2, 64) == 0 and S.cache_bytes(1 << 20, 256, 8, 128) == (1 << 20) * 256 * 8 * 144
    assert S.cache_attn_workspace_bytes(8, **GOOD) > 0
    assert S.cache_attn_workspace_bytes(7, **GOOD) == 0 and S.cache_attn_workspace_bytes(8, **dict(GOOD, head_dim=32)) == 0


def test_expanded_rows_are_refused(monkeypatch):
    from paper_2509_26246_amd import binding as B
    monkeypatch.setattr(B, "_current_device", lambda: -1)      # (tensors of the CPU pass for the GPU's: every call is refused before a launch)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    lens, table, cache = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4, dtype=torch.int32), torch.zeros(8 * 16 * 2 * 72, dtype=torch.uint8)
    for bad in (k[:1].expand(4, 2, 64), k[:, :1].expand(4, 2, 64)):
        for pair in ((bad, k), (k, bad)):
            with pytest.raises(ValueError):
                S.cache_write(*pair, cache, table, lens, **GOOD)


@pytest.mark.parametrize("call", ["write", "read", "attn"])
@pytest.mark.parametrize("bad", [dict(n_rows=(1 << 25) + 1, row_ptr=16), dict(max_pages=(1 << 26) + 1)], ids=str)
def test_sizes_beyond_a_launch_and_beyond_positions_are_refused(call, bad):
    far = dict(k=1 << 44, v=1 << 45, q=1 << 46, o=1 << 47)
    with pytest.raises(S.SlimAttnError) as e:
        _call(call, dict(far, **bad))
    assert e.value.code == -1


def test_workspaces_grow_with_rows():
    for dtype in (S.BF16, S.F32):
        for hq, hkv, n_seqs, max_pages in ((8, 1, 1, 4), (8, 8, 64, 16), (64, 1, 3, 1000), (32, 8, 256, 64)):
            shape = dict(n_pages=8, page_size=64, n_kv_heads=hkv, head_dim=128, dtype=dtype, n_seqs=n_seqs, max_pages=max_pages)
            sizes = [S.cache_attn_workspace_bytes(hq, n_rows=n, **shape) for n in (0, 1, 2, 3, 16, 17, 100, 129, 1000, 5000, 100000)]
            assert sizes == sorted(sizes) and sizes[0] > 0
