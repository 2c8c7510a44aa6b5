"""slimattn_cache_write / _read / _attn against the plain 64-bit forms of cache_reference.py.

What the cache holds is compared for equality: its roundings are those of real quotients, and reading back rounds nothing.

Attention, tolerances (u = 2^-24, L keys, C = 2 for a sum's growth over lane groups, waves and parts).  Codes are exact; scores are fp32 sums of at most 128
products per scale, added up over four groups: below 2^-18 of scale * sum |q_c k_c|, called E.  lse: E, plus rounding it and the sum of L terms, each term's
exponential u * |S| (its argument's rounding): E + 2^-20 (1 + |lse|).  o in bf16: P * scale rounded to bf16 (2^-8 each, half a step) and the output (2^-8):
2^-8 sum p |v| + 2^-8 |o|, plus E as a factor on every term: 2 E sum p |v|.  In f32 three bf16 terms hold 24 bits, so both 2^-8 become 2^-20."""
import numpy as np
import pytest
import torch

import cache_reference as R
import paper_2509_26246_amd as S
from paper_2509_26246_amd import harness as H

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _values(shape, seed, dt, offset=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g)
    if offset:
        x = 0.5 * x + torch.randn(shape[-1], generator=g)
    return x.to(dt)


def _cache(lens, hkv, d, dt, page, seed=0, max_rows=0, hq=0, extra=3, more_columns=1):
    """A cache whose pages are in no order, filled with bytes that decode to NaN scales, and its table (entries past a length: nonsense)."""
    need = [-(-n // page) for n in lens]
    n_pages = max(sum(need) + extra, 1)
    order = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max(max(need, default=0), 1) + more_columns), 0x7fffffff, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    c = H.KVCache(n_pages, page, hkv, d, dt, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), max_rows=max_rows, n_q_heads=hq)
    c.cache.fill_(0xFF)
    if c.workspace is not None:
        c.workspace.fill_(0xFF)
    return c


def _ptr(rows):
    return torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32).cuda()


def _same(got, want):
    got, want = got.double().cpu(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0), want.nan_to_num(0)), f"{int((got.nan_to_num(0) != want.nan_to_num(0)).sum())} values differ"


# ---- writing and reading back ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,hkv,page", [([1], 1, 16), ([17, 0, 5, 300], 2, 16), ([33, 64, 1], 8, 32), ([100] * 70, 1, 64), ([1000], 5, 256), ([129, 127], 3, 128)])
def test_whole_sequences(dtype, d, lens, hkv, page):
    dt = DT[dtype]
    c = _cache(lens, hkv, d, dt, page)
    n = sum(lens)
    k, v = _values((n, hkv, d), 1, dt), _values((n, hkv, d), 2, dt, False)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    out = [torch.full((n + 2, hkv, d), 7.0, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out, _ptr(lens))
    _same(out[0][:n], R.held(k))
    _same(out[1][:n], R.held(v))
    assert all((o[n:] == 7).all() for o in out)            # rows behind the last sequence


def test_growing_token_by_token_and_by_slices():
    lens, hkv, d, dt, page = [40, 23, 64], 2, 128, torch.bfloat16, 16
    c = _cache(lens, hkv, d, dt, page)
    k, v = _values((64, 3, hkv, d), 3, dt), _values((64, 3, hkv, d), 4, dt)
    starts = [30, 16, 60]                                  # written as one slice each, the rest token by token
    flat = lambda x, a, b: torch.cat([x[a[s]:b[s], s] for s in range(3)]).cuda()
    c.lens.copy_(torch.tensor(starts))
    c.write(flat(k, [0] * 3, starts), flat(v, [0] * 3, starts), _ptr(starts))
    done = list(starts)
    while done != lens:
        new = [min(a + 1, b) for a, b in zip(done, lens)]
        c.lens.copy_(torch.tensor(new))
        rows = [b - a for a, b in zip(done, new)]
        c.write(flat(k, done, new), flat(v, done, new), _ptr(rows))
        done = new
    out = [torch.empty(sum(lens), hkv, d, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out, _ptr(lens))
    _same(out[0], R.held(flat(k, [0] * 3, lens).cpu()))
    _same(out[1], R.held(flat(v, [0] * 3, lens).cpu()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_borders_extremes_infinities(dtype):
    dt, d = DT[dtype], 128
    rows = []
    for s in (1.0, 43 / 256, 63 / 64, 2.0 ** -99, 2.0 ** 120, 33 / 1024):
        mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=torch.float64) * s
        near = torch.cat([mids, mids * (1 + 2.0 ** -7), mids * (1 - 2.0 ** -8), -mids])
        if dt == torch.float32:
            m32 = mids.float()
            near = torch.cat([mids, torch.nextafter(m32, m32 * 2).double(), torch.nextafter(m32, m32 * 0).double(), -mids])
        near[-1] = 6 * s
        rows.append(near)
    tiny, inf, nan, big, low = (torch.zeros(32, dtype=torch.float64) for _ in range(5))
    tiny[4], inf[7], nan[9], low[3] = 2.0 ** -100, float("inf"), float("nan"), 2.0 ** -101
    inf[1] = nan[2] = 1.0
    big[:] = 3.38e38
    big[5] = -3.38e38
    rows += [tiny, inf, nan, big, low, torch.zeros(32, dtype=torch.float64)]
    x = torch.stack(rows).reshape(3, 1, 4 * 32).to(dt)
    c = _cache([3], 1, d, dt, 16)
    c.write(x.cuda(), x.cuda(), _ptr([3]))
    out = [torch.empty(3, 1, d, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out, _ptr([3]))
    _same(out[0], R.held(x))
    _same(out[1], R.held(x))


def test_columns_of_a_projection_and_one_row_per_sequence():
    B, hkv, d, dt = 9, 2, 64, torch.bfloat16
    x = _values((B, 4 + 2 * hkv, d), 5, dt).cuda()
    k, v = x[:, 4:4 + hkv], x[:, 4 + hkv:]
    c = _cache([5 * b + 1 for b in range(B)], hkv, d, dt, 32)
    c.write(k, v)
    out = [torch.empty(B, hkv, d, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out)
    _same(out[0], R.held(k.cpu()))
    _same(out[1], R.held(v.cpu()))


def test_pages_that_are_not_there_and_rows_before_the_start():
    hkv, d, dt, page = 1, 64, torch.bfloat16, 16
    c = _cache([40, 3], hkv, d, dt, page, extra=0)
    c.page_table[0, 1] = c._shape["n_pages"]               # one past the last
    c.page_table[1, 0] = -1
    k, v = _values((50, hkv, d), 6, dt), _values((50, hkv, d), 7, dt)
    ptr = torch.tensor([0, 40, 45], dtype=torch.int32).cuda()   # five rows for a sequence of three; rows 45.. are nobody's
    before = c.cache.clone()
    c.write(k.cuda(), v.cuda(), ptr)
    out = [torch.full((50, hkv, d), 7.0, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out, ptr)
    for o, x in zip(out, (k, v)):
        want = R.held(x)
        want[16:32] = 0
        want[40:45] = 0
        want[45:] = 7
        _same(o, want)
    assert int((c.cache != before).sum()) > 0
    c.lens.copy_(torch.tensor([-5, 1 << 30]))              # taken as 0 and as the table's end
    c.write(k.cuda(), v.cuda(), ptr)
    c.read(*out, ptr)
    assert (out[0][:45] == 0).all() and (out[0][45:] == 7).all()


# ---- attention ---------------------------------------------------------------------------------------------------

def _attend(lens, rows, hq, hkv, d, dtype, page, *, scale=None, seed=0, ptr=True, want_lse=True, qf=1.0):
    dt = DT[dtype]
    scale = d ** -0.5 if scale is None else scale
    c = _cache(lens, hkv, d, dt, page, seed, max_rows=sum(rows), hq=hq)
    k, v = _values((sum(lens), hkv, d), seed + 1, dt), _values((sum(lens), hkv, d), seed + 2, dt)
    if sum(lens):
        c.write(k.cuda(), v.cuda(), _ptr(lens))
    n = sum(rows)
    q = (_values((n, hq, d), seed + 3, dt, False).float() * qf).to(dt)
    o = torch.full((n + 2, hq, d), 7.0, dtype=dt, device="cuda")
    lse = torch.full((hq, n), 7.0, device="cuda") if want_lse else None
    c.attend(q.cuda(), o[:n], lse, scale, _ptr(rows) if ptr else None)
    torch.cuda.synchronize()
    assert (o[n:] == 7).all()
    _check_attend(o[:n], lse, q, R.held(k), R.held(v), lens, rows, hq // hkv, scale, dt)
    return c, q, o[:n], lse


def _check_attend(o, lse, q, k, v, lens, rows, group, scale, dt):
    u8 = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -20
    o, lse = o.double().cpu(), None if lse is None else lse.double().cpu()
    ends, at = np.cumsum(lens), 0
    for end, n, r in zip(ends, lens, rows):
        kb, vb, qb = k[end - n:end], v[end - n:end], q[at:at + r].double()
        ro, rl, size = R.attend(qb, kb, vb, group, scale, n - r)
        kg = kb.abs().repeat_interleave(group, 1)
        E = 2.0 ** -18 * abs(scale) * torch.einsum("nhd,lhd->nhl", qb.abs(), kg).amax(-1) if n else torch.zeros(r, qb.shape[1], dtype=torch.float64)
        E = E[..., None]
        err = (o[at:at + r] - ro).abs()
        tol = u8 * size + u8 * ro.abs() + 2 * E * size
        assert (err <= tol).all(), f"o: {float((err / tol.clamp_min(1e-300)).max()):.2f} of the tolerance, length {n}"
        if lse is not None:
            gl, seen = lse[:, at:at + r], torch.isfinite(rl)
            assert torch.equal(torch.isneginf(gl), ~seen)
            le = (gl - rl).abs()[seen]
            lt = (E[..., 0].T + 2.0 ** -20 * (1 + rl.abs()))[seen]
            assert (le <= lt).all(), f"lse: {float((le / lt).max()):.2f} of the tolerance, length {n}"
        at += r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (8, 2), (3, 3), (5, 1), (12, 2), (20, 1)])
def test_single_tokens(dtype, d, hq, hkv):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 700]
    _attend(lens, [1] * len(lens), hq, hkv, d, dtype, 16, ptr=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages(dtype, page):
    _attend([300, 31, 513], [1, 1, 1], 4, 2, 128, dtype, page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_causal_and_rows_that_see_nothing(dtype, d):
    # whole prompts, drafted tokens, none at all, and more rows than the sequence has tokens
    _attend([65, 300, 40, 7, 0, 130], [65, 5, 0, 10, 2, 33], 6, 2, d, dtype, 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_keys_divided_among_blocks(dtype):
    _attend([9000, 1, 3000], [1, 1, 2], 8, 1, 128, dtype, 64)
    _attend([20011], [1], 2, 2, 64, dtype, 256)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_slice(dtype):
    _attend([700], [150], 8, 1, 128, dtype, 64)
    _attend([333, 210], [200, 210], 4, 4, 64, dtype, 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (6, 2), (5, 5), (20, 1), (64, 1)])
def test_many_query_columns(d, hq, hkv):
    # tiles of 128 columns that end inside a row's heads, keys that end inside a tile, prompts with and without keys before them
    _attend([200, 64, 65, 0, 77], [90, 64, 65, 30, 100], hq, hkv, d, "bf16", 16)
    _attend([1200], [100], hq, hkv, d, "bf16", 256)


def test_many_query_columns_over_long_keys():
    _attend([9000], [37], 8, 1, 128, "bf16", 64)           # few items, their keys divided among blocks
    _attend([5000, 33, 2500], [40, 33, 1], 8, 2, 64, "bf16", 32, qf=8.0)
    _attend([70, 3000], [1, 60], 64, 1, 64, "bf16", 64)    # 64 columns of one row


def test_prompts_beside_single_tokens():
    lens = [130, 500, 64, 1, 300, 9]
    _attend(lens, [130, 1, 20, 1, 2, 0], 8, 2, 128, "bf16", 16)
    _attend([300] * 5, [1] * 5, 64, 1, 128, "bf16", 16, ptr=False)


def test_many_sequences():
    r = np.random.default_rng(3)
    lens = [int(x) for x in r.integers(0, 90, 700)]        # more than the blocks' scan takes at once
    rows = [int(min(x, 2)) for x in r.integers(0, 3, 700)]
    _attend(lens, rows, 4, 2, 64, "bf16", 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0, 1e-30])
def test_scales(dtype, scale):
    _attend([300, 20], [1, 3], 4, 2, 64, dtype, 16, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_scores_and_no_lse(dtype):
    _attend([600, 90], [1, 4], 4, 2, 128, dtype, 16, qf=30.0, want_lse=False)


@pytest.mark.parametrize("dtype,hq,rows", [("bf16", 2, 3), ("f32", 2, 3), ("bf16", 8, 30), ("bf16", 16, 70)])
def test_infinities_behind_a_rows_position_are_not_seen(dtype, hq, rows):
    # the keys or values of the second last token are NaN: earlier rows must not notice, the two that see it must
    hkv, d, dt, n = 1, 64, DT[dtype], 100
    for spoil in ("k", "v"):
        c = _cache([n], hkv, d, dt, 16, max_rows=rows, hq=hq)
        k, v = _values((n, hkv, d), 1, dt), _values((n, hkv, d), 2, dt)
        (k if spoil == "k" else v)[-2, :, :32] = float("nan")
        c.write(k.cuda(), v.cuda(), _ptr([n]))
        q = _values((rows, hq, d), 3, dt, False)
        o = torch.empty(rows, hq, d, dtype=dt, device="cuda")
        lse = torch.empty(hq, rows, device="cuda")
        c.attend(q.cuda(), o, lse, 0.125, _ptr([rows]))
        _check_attend(o[:-2], lse[:, :-2].contiguous(), q[:-2], R.held(k)[:-2], R.held(v)[:-2], [n - 2], [rows - 2], hq, 0.125, dt)
        assert torch.isnan(o[-2:] if spoil == "k" else o[-2:, :, :32]).all()
        if spoil == "v":                                   # the other scale group's channels are not spoilt
            clean = R.held(v)
            clean[-2, :, :32] = 0
            want, _, size = R.attend(q[-2:], R.held(k), clean, hq, 0.125, n - 2)
            err = (o[-2:, :, 32:].double().cpu() - want[..., 32:]).abs()
            assert (err <= 2.0 ** -6 * (size[..., 32:] + want[..., 32:].abs())).all()


@pytest.mark.parametrize("hq", [4, 128])
def test_pages_that_are_not_there_are_not_seen(hq):
    hkv, d, dt, n = 2, 128, torch.bfloat16, 200
    c = _cache([n, n], hkv, d, dt, 32, max_rows=2, hq=hq, extra=0)
    k, v = _values((2 * n, hkv, d), 1, dt), _values((2 * n, hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr([n, n]))
    c.page_table[0, 2], c.page_table[1, 0], c.page_table[1, 6] = -1, c._shape["n_pages"], 1 << 30
    q = _values((2, hq, d), 3, dt, False)
    o, lse = torch.empty(2, hq, d, dtype=dt, device="cuda"), torch.empty(hq, 2, device="cuda")
    c.attend(q.cuda(), o, lse, 0.1)
    keep0 = [j for j in range(n) if j // 32 != 2]
    keep1 = [n + j for j in range(n) if j // 32 not in (0, 6)]
    kh, vh = R.held(k), R.held(v)
    for b, keep in enumerate((keep0, keep1)):
        _check_attend(o[b:b + 1], lse[:, b:b + 1], q[b:b + 1], kh[keep], vh[keep], [len(keep)], [1], hq // 2, 0.1, dt)
    c.page_table.fill_(-1)
    c.attend(q.cuda(), o, lse, 0.1)
    assert (o == 0).all() and torch.isneginf(lse).all()


def test_the_same_bits_each_time_and_in_a_graph():
    lens, rows, hq, hkv, d = [5000, 300, 17], [1, 2, 1], 8, 2, 128
    c, q, o, lse = _attend(lens, rows, hq, hkv, d, "bf16", 64)
    q, ptr = q.cuda(), _ptr(rows)
    want_o, want_l = o.clone(), lse.clone()
    for _ in range(3):
        c.workspace.fill_(0xFF)
        c.attend(q, o, lse, d ** -0.5, ptr)
        assert torch.equal(o, want_o) and torch.equal(lse, want_l)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        c.attend(q, o2, lse2, d ** -0.5, ptr)
    for n in ([5000, 300, 17], [4000, 299, 2], [1, 2, 17]):   # lengths are read when the graph runs
        c.lens.copy_(torch.tensor(n))
        c.attend(q, o, lse, d ** -0.5, ptr)
        o2.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_two_streams_with_a_workspace_each():
    lens = [3000, 800]
    a = _attend(lens, [1, 1], 8, 1, 128, "bf16", 64, seed=1)
    b = _attend(lens, [1, 1], 8, 1, 128, "bf16", 64, seed=9)
    wants = [x[2].clone() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs = [x[1].cuda() for x in (a, b)]
    torch.cuda.synchronize()
    for _ in range(4):
        for x, q, s in zip((a, b), qs, streams):
            with torch.cuda.stream(s):
                x[0].attend(q, x[2], x[3], 128 ** -0.5)
    torch.cuda.synchronize()
    assert all(torch.equal(x[2], w) for x, w in zip((a, b), wants))


def test_binding_refuses_what_is_not_a_matching_tensor():
    c = _cache([20, 30], 2, 64, torch.bfloat16, 16, max_rows=2, hq=4)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(4, 2, device="cuda")
    for bad in ((k.float(), k), (k, k.cpu()), (k, k[:, :1]), (k[:, :, :32], k), (k, k[:1])):
        with pytest.raises(ValueError):
            c.write(*bad)
        with pytest.raises(ValueError):
            c.read(*bad)
    with pytest.raises(ValueError):
        c.write(k, k, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        c.write(k, k, torch.zeros(3, dtype=torch.int64, device="cuda"))
    for bad in ((q.float(), q, lse), (q, q.cpu(), lse), (q, torch.empty_like(q), lse[:2]), (q, torch.empty_like(q), lse.half())):
        with pytest.raises(ValueError):
            c.attend(*bad, 0.1)
    with pytest.raises(S.SlimAttnError):
        c.write(k[:1], k[:1])                              # two sequences, one row, no row_ptr
    c.workspace = c.workspace[:64]
    with pytest.raises(ValueError):
        c.attend(q, torch.empty_like(q), lse, 0.1)


def test_pages_that_are_not_there_for_many_query_columns():
    hq, hkv, d, dt, n, rows = 16, 2, 128, torch.bfloat16, 200, 40            # 320 columns of a sequence
    c = _cache([n, n], hkv, d, dt, 32, max_rows=2 * rows, hq=hq, extra=0)
    k, v = _values((2 * n, hkv, d), 1, dt), _values((2 * n, hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr([n, n]))
    c.page_table[0, 2], c.page_table[1, 0], c.page_table[1, 6] = -1, c._shape["n_pages"], 1 << 30
    q = _values((2 * rows, hq, d), 3, dt, False)
    o, lse = torch.empty(2 * rows, hq, d, dtype=dt, device="cuda"), torch.empty(hq, 2 * rows, device="cuda")
    c.attend(q.cuda(), o, lse, 0.1, _ptr([rows, rows]))
    kh, vh = R.held(k), R.held(v)
    for b, gone in enumerate(((2,), (0, 6))):
        for i in (0, 7, 30, 39):
            keep = [b * n + j for j in range(n - rows + i + 1) if j // 32 not in gone]
            at = b * rows + i
            _check_attend(o[at:at + 1], lse[:, at:at + 1], q[at:at + 1], kh[keep], vh[keep], [len(keep)], [1], hq // 2, 0.1, dt)
    c.page_table.fill_(-1)
    c.attend(q.cuda(), o, lse, 0.1, _ptr([rows, rows]))
    assert (o == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("scale,qf", [(0.0, 1.0), (-0.3, 1.0), (1e-30, 1.0), (0.1, 30.0)])
def test_scales_for_many_query_columns(scale, qf):
    _attend([300, 20, 257], [40, 20, 33], 16, 2, 64, "bf16", 16, scale=scale, qf=qf)


def test_the_same_bits_for_many_query_columns_beside_few_and_in_a_graph():
    lens, rows, hq, hkv, d = [5000, 300, 700], [200, 2, 90], 8, 2, 128
    c, q, o, lse = _attend(lens, rows, hq, hkv, d, "bf16", 64)
    q, ptr = q.cuda(), _ptr(rows)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        c.attend(q, o2, lse2, d ** -0.5, ptr)
    for n in ([5000, 300, 700], [4000, 299, 60], [150, 1, 700], [5000, 300, 700]):
        c.lens.copy_(torch.tensor(n))
        c.workspace.fill_(0xFF)
        c.attend(q, o, lse, d ** -0.5, ptr)
        o2.zero_()
        c.workspace.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # the rows dealt out otherwise; the later sequences now reach positions never written, whose NaN are equal only as bits
    ptr.copy_(torch.tensor([0, 2, 202, 292]))
    c.lens.copy_(torch.tensor([300, 700, 5000]))
    c.attend(q, o, lse, d ** -0.5, ptr)
    g.replay()
    torch.cuda.synchronize()
    assert torch.isfinite(o[:2].float()).all()
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))


def test_a_handle_for_single_tokens_needs_no_row_count():
    lens, d = [900, 3, 40], 64
    c = _cache(lens, 2, d, torch.bfloat16, 16, hq=8)       # (max_rows = 0)
    k, v = _values((sum(lens), 2, d), 1, torch.bfloat16), _values((sum(lens), 2, d), 2, torch.bfloat16)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    q = _values((3, 8, d), 3, torch.bfloat16, False)
    o = torch.empty(3, 8, d, dtype=torch.bfloat16, device="cuda")
    c.attend(q.cuda(), o, None, 0.125)
    _check_attend(o, None, q, R.held(k), R.held(v), lens, [1, 1, 1], 4, 0.125, torch.bfloat16)


@pytest.mark.parametrize("rows", [1, 40])
def test_pages_behind_four_gigabytes(rows):
    hq, hkv, d, page, lens, dt = 32, 8, 128, 64, [200, 131], torch.bfloat16
    n_pages = (9 << 29) // (page * hkv * 144)                # 4.8 GB
    c = _cache(lens, hkv, d, dt, page, max_rows=2 * rows, hq=hq, extra=n_pages)
    n_pages = c._shape["n_pages"]
    assert n_pages * page * hkv * 144 > 1 << 32
    table = torch.full_like(c.page_table, 0x7fffffff)
    table[0, :4] = torch.tensor([n_pages - 1, 3, n_pages // 2, n_pages - 2])
    table[1, :3] = torch.tensor([n_pages - 4, 0, n_pages - 3])
    c.page_table.copy_(table)
    k, v = _values((sum(lens), hkv, d), 1, dt), _values((sum(lens), hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    kk, vv = torch.empty_like(k, device="cuda"), torch.empty_like(k, device="cuda")
    c.read(kk, vv, _ptr(lens))
    _same(kk, R.held(k))
    _same(vv, R.held(v))
    q = _values((2 * rows, hq, d), 3, dt, False)
    o, lse = torch.empty(2 * rows, hq, d, dtype=dt, device="cuda"), torch.empty(hq, 2 * rows, device="cuda")
    c.attend(q.cuda(), o, lse, d ** -0.5, _ptr([rows, rows]))
    _check_attend(o, lse, q, R.held(k), R.held(v), lens, [rows, rows], hq // hkv, d ** -0.5, dt)
