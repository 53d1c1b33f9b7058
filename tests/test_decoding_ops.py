"""The decoding operators (paper_1802_07170_amd/decoding.py) against plain implementations in 64 bits on the CPU.

Bounds: a sum of n fp32 numbers in any order is within n * 2^-23 of the sum of their absolute values (2^-24 for a rounded
addition, twice that for one that is cut off); storing a result adds half a step, 2^-24 of it in fp32 and 2^-8 in bf16.
"""
import math

import numpy as np
import pytest
import torch

from paper_1802_07170_amd import binding

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
CUT = 2.0 ** -23
MAGNITUDES = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6])


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def dev(t, dtype=None):
    return t.to(device="cuda", dtype=dtype if dtype is not None else t.dtype)


@pytest.fixture
def D():
    from paper_1802_07170_amd import decoding
    return decoding


# ---- 4-bit weights ---------------------------------------------------------------------------------------------
def plain_pack(w, group):
    """Codes and scales by the definition, from fp32 numbers."""
    n, k = w.shape
    groups = -(-k // group)
    x = np.zeros((n, groups * group), np.float32)
    x[:, :k] = w
    x = x.reshape(n, groups, group)
    scale = torch.from_numpy(np.abs(x).max(2) / np.float32(6)).to(BF).float().numpy()
    size = np.abs(x) / np.where(scale > 0, scale, 1)[:, :, None]
    code = np.abs(size[..., None] - MAGNITUDES[:8].astype(np.float32)).argmin(-1)
    for low, odd in ((.25, 0), (.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5., 6)):     # of two as near the even code
        code = np.where(size == low, odd, code)
    code = np.where(scale[:, :, None] > 0, code + 8 * (x < 0), 0)
    return code.reshape(n, -1)[:, :k], scale


@pytest.mark.parametrize("n,k,group,dtype", [(1, 1, 32, FP), (3, 33, 32, FP), (16, 128, 64, BF), (17, 200, 128, FP), (50, 336, 32, BF), (33, 1000, 64, FP)])
def test_pack_takes_the_nearest_codes(D, n, k, group, dtype):
    w = (0.05 * randn(n * k, n, k)).to(dtype)
    w[0, : min(k, 32)] = 0                                   # a group of zeros, at least in part
    got = D.QuantWeight.pack(dev(w), group)
    code, scale = plain_pack(w.float().numpy(), group)
    want = MAGNITUDES[code] * np.repeat(scale, group, 1)[:, :k]
    assert np.array_equal(got.values().cpu().numpy(), want.astype(np.float32))


def test_pack_takes_strided_weights_borders_and_values_that_are_no_numbers(D):
    wide = randn(1, 20, 300)
    got = D.QuantWeight.pack(dev(wide)[:, 5:205], 64).values().cpu()
    assert torch.equal(got, D.QuantWeight.pack(dev(wide[:, 5:205].contiguous()), 64).values().cpu())
    w = torch.zeros(3, 96)
    w[0, :16] = torch.tensor([6, -6, .25, .26, .75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -.25, -.75, .2, -5, .74])   # scale 1: the borders themselves
    w[1, 40], w[1, 70], w[2, 0] = math.inf, 1.0, math.nan
    got = D.QuantWeight.pack(dev(w), 32).values().cpu()
    assert torch.equal(got[0, :16], torch.tensor([6, -6, 0, .5, 1, 1, 2, 2, 4, 4, 6, -0., -1, 0, -4, .5]))
    assert got[1, 32:64].isnan().all() and not got[1, :32].isnan().any() and abs(got[1, 70] - 1) < 2 ** -8 and got[2, :32].isnan().all()


@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (16, 16, 128), (19, 130, 64), (40, 96, 32)])
def test_codes_come_back_as_what_they_stand_for(D, n, k, group):
    codes = (torch.arange(n * k).reshape(n, k) * 7 % 256).to(torch.uint8)
    scales = (randn(n, n, -(-k // group)) + 3).to(BF)
    got = D.QuantWeight.from_codes(dev(codes), dev(scales), group).values().cpu().numpy()
    want = MAGNITUDES[codes.numpy() & 15] * np.repeat(scales.float().numpy(), group, 1)[:, :k]
    assert np.array_equal(got, want.astype(np.float32))


def product_bound(x, w, bias, want, dtype, out_dtype):
    parts = 3 if dtype == FP else 1
    total = x.abs().double() @ w.abs().double().T + (0 if bias is None else bias.abs().double())
    return (parts * x.shape[1] + 16) * CUT * total + 2.0 ** -22 + half_step(out_dtype) * want.abs()


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 128), (2, 15, 7), (3, 17, 31), (16, 40, 33), (17, 100, 129), (1, 4096, 300), (5, 8200, 260), (33, 8200, 130),
                                   (70, 100, 1100), (130, 48, 64), (40, 8208, 2050),
                                   (390, 8208, 133), (640, 8208, 130), (450, 8200, 264), (1000, 4100, 72)])     # (these fill the chip with 64 rows to a workgroup, or more)
@pytest.mark.parametrize("dtype,out_dtype,group,bias,tanh", [(BF, FP, 64, True, False), (BF, BF, 32, False, True), (FP, FP, 128, True, False), (FP, FP, 32, False, True),
                                                             (FP, BF, 64, True, False)])
def test_product(D, m, n, k, dtype, out_dtype, group, bias, tanh):
    x, b = randn(m + k, m, k).to(dtype), randn(n, n)
    weight = D.QuantWeight.pack(dev(0.1 * randn(n + k, n, k)), group)
    w = weight.values().cpu()
    y = D.quant_product(dev(x), weight, bias=dev(b) if bias else None, tanh=tanh, out_dtype=out_dtype).cpu()
    assert y.dtype == out_dtype
    want = x.double() @ w.double().T + (b.double() if bias else 0)
    want = want.tanh() if tanh else want
    off = (y.double() - want).abs() - product_bound(x.float(), w, b if bias else None, want, dtype, out_dtype)
    assert off.max() <= 0, off.max()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_product_of_strided_rows_leaves_its_neighbours_alone(D, dtype):
    big = randn(3, 20, 401).to(dtype)
    weight = D.QuantWeight.pack(dev(randn(4, 50, 200)), 32)
    whole = D.quant_product(dev(big[:, 7:207].contiguous()), weight)
    for x in (dev(big)[:, 7:207], dev(big.repeat(1, 2))[:, 7:207]):      # rows that begin anywhere
        assert torch.equal(D.quant_product(x, weight), whole)
    out = torch.full((22, 61), 7.0, dtype=dtype, device="cuda")
    D.quant_product(dev(big)[:, 7:207], weight, out=out[1:21, 3:53])
    assert torch.equal(out[1:21, 3:53], whole)
    out[1:21, 3:53] = 7.0
    assert (out == 7.0).all()
    assert D.quant_product(dev(big)[:0, 7:207], weight).shape == (0, 50)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_product_does_not_see_what_is_beside_its_rows(D, dtype):
    for m, n, k in ((5, 100, 72), (20, 9000, 40), (390, 8208, 136), (650, 8208, 200), (390, 8208, 131)):
        wide = torch.full((m + 3, k + 24), math.nan, dtype=dtype, device="cuda")
        weight = D.QuantWeight.pack(dev(0.1 * randn(n, n, k)), 128)
        for at in (8, 3):                                    # rows that begin at whole 16 bytes, and elsewhere
            wide.fill_(math.nan)
            x = wide[1:m + 1, at:at + k]
            x.copy_(dev(randn(m, m, k), dtype))
            out = torch.full((m + 2, n + 8), 7.0, device="cuda")
            D.quant_product(x, weight, out=out[1:-1, 4:-4])
            assert torch.equal(out[1:-1, 4:-4], D.quant_product(x.contiguous(), weight, out_dtype=FP))
            out[1:-1, 4:-4] = 7.0
            assert (out == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_product_keeps_rows_apart_and_infinities_where_they_are(D, dtype):
    x = randn(5, 9, 160).to(dtype)
    codes = torch.full((40, 160), 2, dtype=torch.uint8)                  # weights of one
    codes[:, 3] = 10
    weight = D.QuantWeight.from_codes(dev(codes), torch.ones(40, 5, dtype=BF, device="cuda"), 32)
    clean = D.quant_product(dev(x), weight, out_dtype=FP)
    x[2, 5], x[4, 3], x[6, 100] = math.inf, math.inf, math.nan
    got = D.quant_product(dev(x), weight, out_dtype=FP)
    rest = [0, 1, 3, 5, 7, 8]
    assert torch.equal(got[rest], clean[rest])
    assert (got[2] == math.inf).all() and (got[4] == -math.inf).all() and got[6].isnan().all()
    big = torch.full((1, 160), 3.4028e38 if dtype == FP else 3.38e38)    # the largest numbers have their parts, too
    big[0, 80:] *= -1
    weight = D.QuantWeight.from_codes(dev(torch.full((1, 160), 1, dtype=torch.uint8)), torch.full((1, 5), 2.0 ** -40, dtype=BF, device="cuda"), 32)
    assert torch.isfinite(D.quant_product(dev(big, dtype)[:, 64:96], D.QuantWeight.from_codes(
        dev(torch.tensor([[1] + [0] * 31], dtype=torch.uint8)), torch.ones(1, 1, dtype=BF, device="cuda"), 32), out_dtype=FP)).all()


# ---- source rows in 8 bits -------------------------------------------------------------------------------------
def plain_cache(x, lengths):
    """What the codes of x [b, s, h, d] stand for, by the definition."""
    out = np.zeros(x.shape, np.float32)
    for b, n in enumerate(lengths):
        for h in range(x.shape[2]):
            for t in range(0, n, 32):
                part = x[b, t:min(n, t + 32), h].astype(np.float64)
                scale = np.float32(np.abs(part).max() / 127)
                if scale > 0:
                    out[b, t:min(n, t + 32), h] = np.clip(np.rint(part / np.float64(scale)), -127, 127).astype(np.float32) * scale
    return out


@pytest.mark.parametrize("b,s,h,d", [(1, 1, 1, 1), (3, 33, 1, 16), (4, 64, 2, 40), (2, 70, 3, 64), (5, 31, 1, 336), (2, 100, 1, 1024),
                                     (3, 300, 2, 8), (2, 200, 1, 96), (4, 129, 2, 120), (2, 65, 2, 33), (2, 40, 1, 520)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_cache_holds_the_nearest_codes(D, b, s, h, d, dtype):
    k, v = randn(b + s, b, s, h, d).to(dtype), (3 * randn(b + s + 1, b, s, h, d)).to(dtype)
    lengths = [0 if i == 3 else max(1, s - 13 * i) for i in range(b)]
    for i, n in enumerate(lengths):                          # what is behind a length is not looked at
        k[i, n:], v[i, n:] = math.nan, math.inf
    cache = D.SourceCache(b, h, d, s + 5)
    cache.fill(dev(k), dev(v), torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    for got, x in zip(cache.read(), (k, v)):
        assert np.array_equal(got.cpu().numpy(), plain_cache(x.float().numpy(), lengths))
    # the same rows from other layouts: time-major, and heads in front
    tm = [dev(x.transpose(0, 1).contiguous()).transpose(0, 1) for x in (k, v)]
    hm = [dev(x.transpose(1, 2).contiguous()).transpose(1, 2) for x in (k, v)]
    for other in (tm, hm):
        again = D.SourceCache(b, h, d, s + 5).fill(*other, torch.tensor(lengths, dtype=torch.int32, device="cuda"))
        assert all(torch.equal(x, y) for x, y in zip(again.read(), cache.read()))


def test_cache_codes_on_borders_and_blocks_that_hold_no_numbers(D):
    x = torch.zeros(1, 70, 1, 8)
    x[0, 0, 0] = torch.tensor([127, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -127])     # scale 1: of two codes the even one
    x[0, 40, 0, 2] = math.inf
    x[0, 66, 0, 1] = 1e-44                                                       # less than 127 of the smallest numbers
    keys, values = D.SourceCache(1, 1, 8, 70).fill(dev(x), dev(-x), torch.tensor([70], dtype=torch.int32, device="cuda")).read()
    assert keys[0, 0, 0].tolist() == [127, 0, 2, 2, 0, -2, 126, -127] and values[0, 0, 0].tolist() == [-127, 0, -2, -2, 0, 2, -126, 127]
    assert keys[0, 32:64].isnan().all() and torch.isfinite(keys[0, :32]).all() and torch.isfinite(keys[0, 64:]).all()
    long = D.SourceCache(2, 1, 8, 70)
    long.fill(dev(x.repeat(2, 1, 1, 1))[:, :32], dev(x.repeat(2, 1, 1, 1))[:, :32], torch.tensor([99, -4], dtype=torch.int32, device="cuda"))
    assert torch.equal(long.read()[0][0], keys[0, :32]) and (long.read()[0][1] == 0).all()      # lengths are clamped


def attend_plain(q, k, v, lengths, scale):
    """In 64 bits, and a bound of what the kernel may be off."""
    rows, heads, d = q.shape
    per, share = rows // k.shape[0], heads // k.shape[2]
    out, bound = torch.zeros(rows, heads, d, dtype=torch.float64), torch.zeros(rows, heads, d, dtype=torch.float64)
    fp = q.dtype == FP
    for r in range(rows):
        n = lengths[r // per]
        for h in range(heads):
            if n == 0:
                continue
            kk, vv, x = k[r // per, :n, h // share].double(), v[r // per, :n, h // share].double(), q[r, h].double()
            s = kk @ x * scale
            a = torch.softmax(s, 0)
            out[r, h] = a @ vv
            # scores: sums of d products (3 d in fp32), three multiplications; exponentials: 2^-22 of their argument and 2^-21 of the value
            off = ((3 if fp else 1) * d + 16) * CUT * (kk.abs() @ x.abs() * abs(scale)).max() + (s.max() - s.min() + 4) * 2.0 ** -21
            # weights in parts: 2^-16 of them left out with 16-bit operands, 2^-24 in fp32; sums of n; the quotient
            rel = 2 * off + (3 * n + 64) * CUT + (2.0 ** -24 if fp else 2.0 ** -16)
            bound[r, h] = rel * (a @ vv.abs()) + half_step(q.dtype) * out[r, h].abs() + 1e-30
    return out, bound


@pytest.mark.parametrize("b,per,kv,share,d,lengths", [
    (1, 1, 1, 1, 16, [1]), (2, 3, 1, 1, 64, [0, 31]), (3, 10, 1, 1, 1024, [50, 1, 33]), (2, 16, 1, 1, 336, [32, 37]), (2, 17, 1, 1, 100, [129, 127]),
    (1, 1, 4, 4, 128, [700]), (2, 5, 2, 3, 64, [130, 400]), (1, 2, 1, 1, 512, [1500]), (3, 1, 2, 8, 192, [0, 128, 300]), (1, 40, 1, 1, 256, [260]), (1, 2, 3, 1, 1, [40]),
    (2, 20, 2, 2, 32, [257, 600]), (1, 3, 1, 8, 80, [513]), (2, 33, 1, 1, 96, [65, 256]), (3, 18, 1, 1, 500, [129, 0, 40]), (1, 5, 2, 1, 48, [70]), (1, 17, 1, 2, 768, [200])])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention(D, b, per, kv, share, d, lengths, dtype):
    s = max(lengths)
    k, v, q = randn(d, b, s, kv, d), randn(d + 1, b, s, kv, d), randn(d + 2, b * per, kv * share, d).to(dtype)
    for i, n in enumerate(lengths):
        k[i, n:], v[i, n:] = math.nan, math.nan
    cache = D.SourceCache(b, kv, d, s + 40)
    cache.fill(dev(k, dtype), dev(v, dtype), torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    hk, hv = (x.cpu() for x in cache.read())
    for scale in (1 / math.sqrt(d), 3.0):
        got = cache.attend(dev(q), scale=scale)
        want, bound = attend_plain(q, hk, hv, lengths, scale)
        off = (got.cpu().double() - want).abs() - bound
        assert off.max() <= 0, (scale, off.max())
        assert torch.equal(cache.attend(dev(q), scale=scale), got)
    # queries and results in the rows of wider tensors, at any offset
    wide = torch.full((b * per, kv * share * d + 3), 5.0, dtype=dtype, device="cuda")
    wq = wide.clone()
    wq[:, 1:-2] = dev(q).reshape(b * per, -1)
    out = wide[:, 2:-1].unflatten(1, (kv * share, d))
    cache.attend(wq[:, 1:-2].unflatten(1, (kv * share, d)), scale=3.0, out=out)
    assert torch.equal(out, got)
    assert (wide[:, :2] == 5.0).all() and (wide[:, -1:] == 5.0).all()


def test_attention_with_scores_far_apart_and_blocks_that_hold_no_numbers(D):
    k = torch.zeros(2, 200, 1, 32)
    k[:, :, 0, 0] = torch.linspace(-90, 90, 200)
    v = torch.arange(200.).reshape(1, 200, 1, 1).expand(2, 200, 1, 32).contiguous()
    k[1, 150, 0, 3] = math.nan
    q = torch.zeros(2, 1, 32)
    q[:, 0, 0] = 50.0
    cache = D.SourceCache(2, 1, 32, 200).fill(dev(k), dev(v), torch.tensor([200, 140], dtype=torch.int32, device="cuda"))
    hk, hv = (x.cpu() for x in cache.read())
    got = cache.attend(dev(q)).cpu()
    want, bound = attend_plain(q, hk, hv, [200, 140], 1.0)
    assert ((got.double() - want).abs() <= bound).all()      # (the NaN lies behind the second sequence's length)
    cache.fill(dev(k), dev(v), torch.tensor([200, 151], dtype=torch.int32, device="cuda"))
    got = cache.attend(dev(q)).cpu()
    assert torch.isfinite(got[0]).all() and got[1].isnan().all()


# ---- a search's choice -----------------------------------------------------------------------------------------
def plain_select(logits, scores, n):
    b, beam = scores.shape
    z = logits.double().reshape(b, beam, -1)
    total = scores.double()[:, :, None] + torch.log_softmax(z, 2)
    bad = ~(torch.isfinite(scores)[:, :, None] & ((z < math.inf).all(2, keepdim=True)) & (z > -math.inf).any(2, keepdim=True))
    total = torch.where(bad | (z == -math.inf), -math.inf, total).reshape(b, -1)
    if total.shape[1] < n:
        total = torch.cat([total, torch.full((b, n - total.shape[1]), -math.inf, dtype=total.dtype)], 1)
    # of equal logits of a row the first; of equal rows, too: the order is by (score, row, token)
    best, at = torch.sort(total, dim=1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    found = best > -math.inf
    v = z.shape[2]
    rows = torch.where(found, at // v + beam * torch.arange(b)[:, None], -1)
    return best, rows.int(), torch.where(found, at % v, -1).int()


def check_select(D, logits, scores, n=None):
    got = [t.cpu() for t in D.beam_select(dev(logits) if not logits.is_cuda else logits, dev(scores), n)]
    want = plain_select(logits.cpu(), scores, scores.shape[1] if n is None else n)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    live = want[0] > -math.inf
    assert (got[0][~live] == -math.inf).all()
    # the log of a sum of at most 32 + vocab / 32768 additions, exponentials within 2^-21 each; stored in fp32
    off = (got[0].double() - want[0]).abs()[live]
    assert off.numel() == 0 or (off <= (40 + logits.shape[1] / 32768) * CUT + 2.0 ** -21 + 2.0 ** -24 * want[0][live].abs()).all(), off.max()
    return got


@pytest.mark.parametrize("b,beam,vocab,n", [(1, 1, 1, None), (2, 3, 5, None), (1, 10, 511, None), (3, 4, 512, None), (2, 16, 513, 5), (5, 4, 9064, None), (1, 32, 3001, 32),
                                            (1, 2, 3, 32), (2, 10, 40001, 20), (70, 2, 1000, 3)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_selection(D, b, beam, vocab, n, dtype):
    logits = (3 * randn(vocab, b * beam, vocab)).to(dtype)
    scores = -5 + randn(b, b, beam)
    check_select(D, logits, scores, n)
    scores[:, beam // 2:] = -math.inf                        # places without a hypothesis: what stands there is not looked at
    logits[beam // 2] = math.nan
    check_select(D, logits, scores, n)
    scores[0] = -math.inf
    check_select(D, logits, scores, n)


def test_selection_of_equal_and_of_impossible_extensions(D):
    same = torch.zeros(6, 5000)
    check_select(D, same, torch.zeros(2, 3))                 # every extension as good as the next
    check_select(D, same, torch.tensor([[-1.0, -1.0, 0.0], [0.0, -math.inf, 0.0]]), 32)
    few = torch.full((6, 5000), -math.inf)
    few[0, 4999], few[1, 17], few[1, 18], few[4, 3] = 1.0, 2.0, 2.0, -4.0
    check_select(D, few, torch.zeros(2, 3), 4)               # fewer than asked for, a row without any
    odd = randn(7, 8, 700)
    odd[1, 5], odd[2, 6], odd[4] = math.nan, math.inf, -math.inf
    scores = torch.zeros(2, 4)
    scores[1, 1], scores[1, 2] = math.nan, math.inf
    check_select(D, odd, scores)
    steps = (torch.arange(20000) % 7 * 0.25).repeat(4, 1)    # 2857 best ones in each row
    check_select(D, steps.to(BF), torch.zeros(1, 4), 32)
    late = torch.zeros(1, 70000)
    late[0, 65536:65568] = torch.arange(32.)
    check_select(D, late, torch.zeros(1, 1), 32)


def test_selection_of_rows_that_begin_anywhere(D):
    wide = randn(8, 6, 2051)
    for dtype in (BF, FP):
        logits = dev(wide, dtype)[:, 2:2049]
        check_select(D, logits, -randn(9, 2, 3).abs(), 7)


@pytest.mark.parametrize("dtype,shape", [(FP, (64,)), (BF, (40,)), (BF, (3, 5)), (torch.uint8, (7,)), (torch.int64, ()), (FP, (1024,))])
def test_reorder(D, dtype, shape):
    rows = torch.tensor([[3, 0, 0], [-1, 5, 2], [6, 1, -7]], dtype=torch.int32)
    src = [(10 * randn(i, 6, *shape)).to(dtype) for i in range(40)]
    dst = [(10 * randn(i + 50, 9, *shape)).to(dtype) for i in range(40)]
    out = [dev(t) for t in dst]
    D.beam_reorder(dev(rows), [dev(t) for t in src], out)
    for s, d, o in zip(src, dst, out):
        flat = rows.reshape(-1)
        want = torch.stack([s[int(r)] if 0 <= r < 6 else d[i] for i, r in enumerate(flat)])
        assert torch.equal(o.cpu(), want)


def test_reorder_of_strided_rows(D):
    src, dst = dev(randn(1, 5, 30)), torch.zeros(5, 41, device="cuda")
    rows = torch.tensor([4, 3, 2, 1, 0], dtype=torch.int32, device="cuda")
    D.beam_reorder(rows, [src[:, 3:20], src[:, 20:]], [dst[:, 1:18], dst[:, 18:28]])
    assert torch.equal(dst[:, 1:18], src[:, 3:20].flip(0)) and torch.equal(dst[:, 18:28], src[:, 20:].flip(0))
    assert (dst[:, 0] == 0).all() and (dst[:, 28:] == 0).all()
    with pytest.raises(binding.CmtError, match="overlaps"):
        D.beam_reorder(rows, [src], [src])
    with pytest.raises(binding.CmtError, match="overlap"):
        D.beam_reorder(rows, [src, src], [dst[:, :30], dst[:, 5:35]])
    both = torch.cat([src, torch.zeros(5, 30, device="cuda")], 1)
    D.beam_reorder(rows, [both[:, :30]], [both[:, 30:]])     # columns of one matrix
    assert torch.equal(both[:, 30:], src.flip(0)) and torch.equal(both[:, :30], src)
    with pytest.raises(binding.CmtError, match="overlaps"):
        D.beam_reorder(rows, [both[:, :30]], [both[:, 29:59]])
    D.beam_reorder(rows[:0], [src], [dst[:0, :30]])          # nothing to move
    D.beam_reorder(rows, [], [])


# ---- together ----------------------------------------------------------------------------------------------------
def position(D, s):
    """One position as a search makes it: gates, attention, logits, choice, states."""
    gates = D.quant_product(s["x"], s["w_gates"], bias=s["b"], out_dtype=BF)
    query = D.quant_product(gates, s["w_query"], tanh=True)
    context = s["cache"].attend(query.unflatten(1, (1, -1)), scale=0.1)
    logits = D.quant_product(context.flatten(1), s["w_out"], out_dtype=FP)
    scores, rows, tokens = D.beam_select(logits, s["scores"])
    D.beam_reorder(rows, [gates, context], s["moved"])
    return [gates, query, context, logits, scores, rows, tokens, *s["moved"]]


def test_a_position_on_streams_of_its_own_and_replayed_from_a_graph(D):
    b, beam, h = 3, 4, 96
    mk = lambda seed: dict(x=dev(randn(seed, b * beam, h), BF), scores=dev(-randn(seed + 1, b, beam).abs()))
    keep = dict(w_gates=D.QuantWeight.pack(dev(0.1 * randn(1, 4 * h, h)), 32), w_query=D.QuantWeight.pack(dev(0.1 * randn(2, h, 4 * h)), 64),
                w_out=D.QuantWeight.pack(dev(0.3 * randn(3, 1000, h)), 64), b=dev(randn(4, 4 * h)), cache=D.SourceCache(b, 1, h, 300))
    keep["cache"].fill(dev(randn(5, b, 300, 1, h), BF), dev(randn(6, b, 300, 1, h), BF), torch.tensor([300, 7, 150], dtype=torch.int32, device="cuda"))
    moved = lambda: [torch.zeros(b * beam, 4 * h, dtype=BF, device="cuda"), torch.zeros(b * beam, 1, h, dtype=BF, device="cuda")]
    inputs = [mk(10 * i) for i in range(3)]
    want = [[t.clone() for t in position(D, dict(keep, **i, moved=moved()))] for i in inputs]
    side = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for st, i in zip(side, inputs):                          # three at once
        with torch.cuda.stream(st):
            got.append(position(D, dict(keep, **i, moved=moved())))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(g, w))
    state = dict(keep, x=inputs[0]["x"].clone(), scores=inputs[0]["scores"].clone(), moved=moved())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = position(D, state)
    for k in (1, 2, 0, 1):
        state["x"].copy_(inputs[k]["x"])
        state["scores"].copy_(inputs[k]["scores"])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want[k])), k
        position(D, dict(keep, **inputs[2], moved=moved()))  # the program's own work in between
        torch.cuda.synchronize()


def test_refusals_on_the_device(D):
    w = D.QuantWeight.pack(dev(randn(1, 20, 64)), 32)
    x = dev(randn(2, 3, 64))
    for call in (lambda: D.quant_product(x[:, :63], w), lambda: D.quant_product(x.half(), w), lambda: D.quant_product(x, w, bias=x[0]),
                 lambda: D.quant_product(x.t()[:3].t(), w), lambda: D.quant_product(x, w, out_dtype=torch.float16), lambda: D.quant_product(x.cpu(), w),
                 lambda: D.quant_product(x, w, out=torch.empty(3, 21, device="cuda")), lambda: D.quant_product(x.clone().requires_grad_(), w),
                 lambda: D.quant_product(x, w, out=x[:, :20]), lambda: D.beam_select(x, torch.zeros(2, 2, device="cuda")),
                 lambda: D.QuantWeight.from_codes(torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, 3, dtype=BF, device="cuda"), 32),
                 lambda: D.SourceCache(2, 1, 64, 9).read(), lambda: D.SourceCache(2, 1, 64, 9).attend(x[:2, None]),
                 lambda: D.beam_reorder(torch.zeros(3, dtype=torch.int32, device="cuda"), [x], [x[:2]])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: D.QuantWeight.pack(x, 48), lambda: D.beam_select(x, torch.zeros(3, 1, device="cuda"), 33), lambda: D.SourceCache(2, 1, 1025, 9),
                 lambda: D.quant_product(x[:1].expand(3, 64), w), lambda: D.SourceCache(70000, 1, 16, 9)):
        with pytest.raises(binding.CmtError):
            call()
    cache = D.SourceCache(3, 1, 64, 9).fill(x[:, None, None].expand(3, 9, 1, 64), x[:, None, None].expand(3, 9, 1, 64),
                                            torch.full((3,), 9, dtype=torch.int32, device="cuda"))
    with pytest.raises(binding.CmtError, match="finite"):
        cache.attend(x[:, None], scale=math.inf)
    for bad in (x[:2, None], x[:, None, :32], x[:, None].half()):
        with pytest.raises(ValueError):
            cache.attend(bad)


# ---- offsets that 32 bits do not hold: exact cases whose answer lies behind the 2^32nd byte ------------------------
def test_a_weight_of_more_than_4_gib_of_codes(D):
    n, k = (1 << 17) + 16, 1 << 16
    w = torch.zeros(n, k, dtype=BF, device="cuda")
    w[-1] = torch.tensor([6.0, -4.0, 0.5, 3.0], device="cuda").repeat(k // 4)       # the scale is 1: the codes are exact
    weight = D.QuantWeight.pack(w, 128)
    assert weight.packed.numel() > 1 << 32
    del w
    x = (torch.arange(2 * k, device="cuda").view(2, k) % 3).to(BF)                # sums below 2^24
    want = (x.double() * torch.tensor([6.0, -4.0, 0.5, 3.0], device="cuda").repeat(k // 4).double()).sum(1)
    y = D.quant_product(x, weight, out_dtype=FP)
    assert torch.equal(y[:, -1].double(), want) and not y[:, :-1].any()


def test_a_cache_of_more_than_4_gib(D):
    tokens = (1 << 22) + 40
    x = torch.zeros(1, tokens, 1, 1024, dtype=BF, device="cuda")
    row = (torch.arange(1024, device="cuda") % 255 - 127).to(BF)                  # the scale is 1: the codes are exact
    x[0, tokens - 3, 0] = row
    cache = D.SourceCache(1, 1, 1024, tokens).fill(x, x, torch.tensor([tokens], dtype=torch.int32, device="cuda"))
    assert cache.data.numel() > 1 << 33
    q = torch.sign(row)[None, None].contiguous()                                  # its score is far above the others', which are 0
    assert torch.equal(cache.attend(q)[0, 0], row)
    assert not cache.attend(-q).isnan().any()


def test_logits_of_more_than_2_to_the_32(D):
    sentences, beam, vocab = 4112, 2, 1 << 19
    logits = torch.empty(sentences * beam, vocab, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(7))
    scores = -torch.rand(sentences, beam, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    assert logits.numel() > 1 << 32
    new, rows, tokens = D.beam_select(logits, scores)
    last = 3
    few = D.beam_select(logits[-last * beam:], scores[-last:])
    assert torch.equal(new[-last:], few[0]) and torch.equal(rows[-last:], few[1] + (sentences - last) * beam) and torch.equal(tokens[-last:], few[2])


def test_rows_of_a_gib(D):
    source = torch.zeros(5, 1 << 30, dtype=torch.uint8, device="cuda")
    source[:, -1] = torch.arange(1, 6, device="cuda")
    target = torch.full((6, 1 << 30), 9, dtype=torch.uint8, device="cuda")
    D.beam_reorder(torch.tensor([4, 0, -1, 5, 4, 3], dtype=torch.int32, device="cuda"), [source], [target])
    assert target[:, -1].tolist() == [5, 1, 9, 9, 5, 4] and target[:, 0].tolist() == [0, 0, 9, 9, 0, 0]
