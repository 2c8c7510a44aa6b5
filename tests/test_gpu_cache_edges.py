"""slimattn_cache_attn where its parts meet: values that are not finite under weights of zero, in every kind of step and in both kernels.

A spoilt value's group of 32 channels has to be NaN in each row that sees its key, however small the key's weight is, and in no other row; tolerances of
what is not spoilt are those of test_gpu_cache."""
import pytest
import torch

import cache_reference as R
from test_gpu_cache import DT, _cache, _check_attend, _ptr, _values

pytestmark = pytest.mark.gpu


# single tokens, few rows (one and two tiles of 16 columns), and bf16 sequences of more than 112 columns
@pytest.mark.parametrize("dtype,hq,rows", [("bf16", 1, 1), ("bf16", 2, 3), ("f32", 2, 3), ("bf16", 8, 4), ("f32", 8, 4), ("bf16", 8, 30), ("bf16", 16, 70)])
# among the last keys, in a step that only some rows see whole, and in one that all do
@pytest.mark.parametrize("key", [299, 298, 290, 257, 256, 231, 200, 10])
def test_a_nan_under_a_weight_of_zero_is_seen(dtype, hq, rows, key):
    hkv, d, dt, n, scale = 1, 128, DT[dtype], 300, 0.125
    # the cache holds 1.008 for 1: every score is 60 * 0.125 * 128 * 1.008 = 967, the spoilt key's -967: its weight is 0 in any type, e^-1935
    k, v = torch.ones(n, hkv, d), _values((n, hkv, d), 2, dt).float()
    k[key] = -1
    v[key, 0, 5], v[key, 0, 100] = float("nan"), float("inf")                # groups 0 and 3
    k, v = k.to(dt), v.to(dt)
    c = _cache([n], hkv, d, dt, 16, max_rows=rows, hq=hq)
    c.write(k.cuda(), v.cuda(), _ptr([n]))
    q = torch.full((rows, hq, d), 60.0, dtype=dt)
    o, lse = torch.empty(rows, hq, d, dtype=dt, device="cuda"), torch.empty(hq, rows, device="cuda")
    c.attend(q.cuda(), o, lse, scale, _ptr([rows]))
    sees = torch.arange(n - rows, n) >= key
    nan = torch.isnan(o.float()).cpu()
    spoilt = torch.zeros(d, dtype=torch.bool)
    spoilt[:32] = spoilt[96:] = True
    assert torch.equal(nan, (sees[:, None, None] & spoilt).expand(rows, hq, d))
    clean = R.held(v)
    clean[key] = 0                                         # what the other channels of the key add: 0 times a finite value
    want, lse_want, size = R.attend(q, R.held(k), clean, hq, scale, n - rows)
    u, E = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20, 2.0 ** -18 * 970
    err = (o.double().cpu() - want).abs()
    assert (err <= u * size + u * want.abs() + 2 * E * size)[~nan].all()
    assert ((lse.double().cpu() - lse_want).abs() <= E + 2.0 ** -20 * 1000).all()


@pytest.mark.parametrize("dtype,hq,lens,rows", [("bf16", 8, [700, 1, 2000], [1, 1, 1]), ("f32", 4, [300] * 9, [1] * 9), ("bf16", 8, [500, 130], [40, 30]),
                                                ("bf16", 4, [260] * 40, [1] * 40), ("bf16", 16, [3000], [100]), ("bf16", 8, [64], [1])])
def test_tables_with_room_to_grow(dtype, hq, lens, rows):
    # many more blocks are launched than have work: which of them work, and on what, goes by the lengths
    hkv, d, dt, page, scale = 1, 128, DT[dtype], 16, 0.09
    c = _cache(lens, hkv, d, dt, page, max_rows=sum(rows), hq=hq, more_columns=4096)
    k, v = _values((sum(lens), hkv, d), 1, dt), _values((sum(lens), hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    q = _values((sum(rows), hq, d), 3, dt, False)
    o, lse = torch.empty(sum(rows), hq, d, dtype=dt, device="cuda"), torch.empty(hq, sum(rows), device="cuda")
    for _ in range(2):
        c.attend(q.cuda(), o, lse, scale, _ptr(rows))
        _check_attend(o, lse, q, R.held(k), R.held(v), lens, rows, hq, scale, dt)


@pytest.mark.parametrize("dtype,hq,more", [("bf16", 4, 5), ("f32", 4, 5), ("bf16", 16, 40), ("bf16", 4, 1 << 20)])
def test_rows_beyond_the_tensors_are_no_rows(dtype, hq, more):
    # row_ptr ends behind the tensors' last row: the last sequence has the rows up to there, at the positions before its end, for every call alike
    hkv, d, dt, rows, lens, scale = 2, 64, DT[dtype], [3, 50], [40, 90], 0.125
    n = sum(rows)
    c = _cache(lens, hkv, d, dt, 16, max_rows=n, hq=hq)
    k, v = _values((sum(lens), hkv, d), 1, dt), _values((sum(lens), hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    beyond = torch.tensor([0, 3, n + more], dtype=torch.int32).cuda()
    last = torch.cat([torch.arange(37, 40), torch.arange(40 + 40, 40 + 90)])
    out = [torch.empty(n, hkv, d, dtype=dt, device="cuda") for _ in range(2)]
    c.read(*out, beyond)
    for got, x in zip(out, (k, v)):
        assert torch.equal(got.double().cpu(), R.held(x)[last])
    q = _values((n, hq, d), 3, dt, False)
    o, lse = torch.empty(n, hq, d, dtype=dt, device="cuda"), torch.empty(hq, n, device="cuda")
    c.attend(q.cuda(), o, lse, scale, beyond)
    _check_attend(o, lse, q, R.held(k), R.held(v), lens, rows, hq // hkv, scale, dt)
    new = [_values((n, hkv, d), s, dt) for s in (7, 8)]
    c.write(*[x.cuda() for x in new], beyond)
    c.read(*out, _ptr(rows))
    for got, x in zip(out, new):
        assert torch.equal(got.double().cpu(), R.held(x))


@pytest.mark.parametrize("dtype,hq,hkv,d,lens", [("bf16", 8, 1, 128, [40000]), ("bf16", 5, 1, 64, [34000]), ("f32", 8, 1, 128, [36000]), ("f32", 2, 2, 64, [70001]),
                                                 ("bf16", 8, 1, 128, [70000, 33000])])
def test_hundreds_of_parts(dtype, hq, hkv, d, lens):
    # one item's keys over 130 to 280 blocks, whose parts a block of 1024 threads adds up: lists filled with ones before, the same bits each time
    dt, n, scale = DT[dtype], len(lens), d ** -0.5
    c = _cache(lens, hkv, d, dt, 64, max_rows=n, hq=hq)
    k, v = _values((sum(lens), hkv, d), 1, dt), _values((sum(lens), hkv, d), 2, dt)
    c.write(k.cuda(), v.cuda(), _ptr(lens))
    q = _values((n, hq, d), 3, dt, False)
    o, lse = torch.empty(n, hq, d, dtype=dt, device="cuda"), torch.empty(hq, n, device="cuda")
    c.attend(q.cuda(), o, lse, scale)
    _check_attend(o, lse, q, R.held(k), R.held(v), lens, [1] * n, hq // hkv, scale, dt)
    again, lse2 = torch.empty_like(o), torch.empty_like(lse)
    c.workspace.fill_(0xFF)
    c.attend(q.cuda(), again, lse2, scale)
    assert torch.equal(o, again) and torch.equal(lse, lse2)
