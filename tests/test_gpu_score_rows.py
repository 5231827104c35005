"""Products with a packed table (hs_score_packed), score adjustments
(hs_adjust_scores), top-k of rows (hs_topk_rows) against 64-bit references, and the
operators together."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_22578_amd as hs
import rows_reference as ref
from gpu_harness import device

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF32 = 2.0 ** -24


def packed_table(rng, rows, dim, group, scale_dtype):
    codes = torch.from_numpy(rng.integers(0, 256, (rows, dim // 2)).astype(np.uint8))
    sc = torch.from_numpy((rng.standard_normal((rows, dim // group)) * 0.1).astype(np.float32)
                          ).to(scale_dtype)
    return (hs.RowTable(codes.to(device()), sc.to(device()), group=group),
            ref.unpack(codes, sc, group))


@pytest.mark.parametrize("group,dim", [(32, 32), (32, 96), (32, 160), (32, 1024), (64, 64),
                                       (64, 192), (64, 768), (128, 128), (128, 640), (128, 4096)])
@pytest.mark.parametrize("xt", [F32, BF16])
def test_score_packed_sizes(group, dim, xt):
    rng = np.random.default_rng(dim + group)
    for m, rows, sdt, out in [(1, 1, BF16, F32), (1, 500, F32, BF16), (2, 65, BF16, F32),
                              (5, 1000, BF16, BF16), (16, 130, F32, F32), (17, 63, BF16, F32),
                              (33, 257, BF16, F32), (65, 40, F32, F32), (130, 100, BF16, BF16)]:
        table, values = packed_table(rng, rows, dim, group, sdt)
        x = torch.from_numpy(rng.standard_normal((m, dim)).astype(np.float32)).to(xt)
        got = hs.score_packed(table, x.to(device()), out_dtype=out)
        want, bound = ref.score_packed(values, ref.f64(x), group)
        ref.check(got, want, bound, out, f"m={m} rows={rows} dim={dim} group={group}")


@pytest.mark.parametrize("m,rows,dim,group,xt,sdt", [
    # x staged whole by 16 or 8 waves: four, two and one of them share the columns
    (5, 66_001, 3712, 64, F32, BF16), (12, 1000, 3200, 32, BF16, F32), (13, 9001, 3328, 128, BF16, BF16),
    (30, 33_333, 1280, 64, BF16, BF16), (7, 9001, 1472, 32, F32, BF16), (40, 20_001, 1056, 32, BF16, F32), (16, 70_001, 2048, 64, BF16, BF16),
    # in parts: for many rows, few, rows of x in several blocks, the widest
    (16, 40_001, 2080, 32, F32, BF16), (22, 30_001, 1184, 32, F32, F32), (35, 1573, 2048, 128, BF16, F32),
    (48, 40_001, 2176, 128, BF16, BF16), (16, 300, 4096, 32, F32, BF16), (70, 600, 2304, 64, BF16, BF16),
    (37, 1001, 2304, 32, F32, BF16), (3, 97, 16_384, 128, F32, BF16), (64, 97, 16_384, 64, BF16, F32)])
def test_score_packed_staging(m, rows, dim, group, xt, sdt):
    g = torch.Generator().manual_seed(m + rows)
    codes = torch.randint(0, 256, (rows, dim // 2), dtype=torch.uint8, generator=g)
    scales = (torch.randn(rows, dim // group, generator=g) * 0.1).to(sdt)
    table = hs.RowTable(codes.to(device()), scales.to(device()), group=group)
    x = torch.randn(m, dim, generator=g).to(xt)
    got = hs.score_packed(table, x.to(device()))
    # (a part of the rows: the ends and some between)
    some = torch.unique(torch.cat([torch.arange(min(rows, 300)),
                                   torch.randint(0, rows, (300,), generator=g),
                                   torch.arange(max(rows - 300, 0), rows)]))
    values = ref.unpack(codes[some], scales[some], group)
    want, bound = ref.score_packed(values, ref.f64(x), group)
    ref.check(got[:, some.to(device())], want, bound, F32)
    assert torch.isfinite(got).all()
    assert torch.equal(got, hs.score_packed(table, x.to(device())))


def test_score_packed_places_every_column():
    """One-hot rows pick single table columns: exact, so any mixed-up column shows."""
    rng = np.random.default_rng(3)
    for group, dim in [(32, 288), (64, 320), (128, 384)]:
        table, values = packed_table(rng, 70, dim, group, F32)
        for xt in (F32, BF16):
            x = torch.eye(dim, dtype=xt, device=device())
            got = hs.score_packed(table, x).cpu().double().numpy()
            np.testing.assert_array_equal(got, values.astype(np.float32).astype(np.float64).T)


def test_score_packed_fp32_rows_keep_their_bits():
    """A single column: the product of an fp32 value and a code needs all three parts."""
    rng = np.random.default_rng(4)
    codes = torch.full((16, 16), 0x22, dtype=torch.uint8)         # all codes 1.0
    table = hs.RowTable(codes.to(device()), torch.ones(16, 1, device=device()), group=32)
    x = torch.zeros(40, 32)
    v = rng.standard_normal(40).astype(np.float32) * np.exp(rng.standard_normal(40) * 20)
    v[:3] = 3.4e38, -1.1754944e-38, 1.0000001
    x[torch.arange(40), torch.arange(40) % 32] = torch.from_numpy(v.astype(np.float32))
    got = hs.score_packed(table, x.to(device())).cpu()
    assert torch.equal(got, x.sum(1, keepdim=True).expand(40, 16))


def test_score_packed_fp32_rows_near_the_least_values():
    """The three parts end at bf16's least value, 2^-133: fp32 values from 2^-110 on keep
    their 24 bits, smaller ones lose what lies below it; bf16 rows lose nothing."""
    rng = np.random.default_rng(5)
    v = ((1 + rng.random(400)) * 2.0 ** rng.integers(-149, -90, 400)).astype(np.float32)
    v[::2] *= -1
    x = torch.zeros(400, 32)
    x[torch.arange(400), torch.arange(400) % 32] = torch.from_numpy(v)
    codes = torch.full((16, 16), 0x22, dtype=torch.uint8, device=device())      # all codes 1.0
    for scale in (1.0, 2.0 ** 100):
        table = hs.RowTable(codes, torch.full((16, 1), scale, device=device()), group=32)
        got = ref.f64(hs.score_packed(table, x.to(device())))[:, 0]
        want = v.astype(np.float64) * scale
        whole = np.abs(v) >= 2.0 ** -110
        np.testing.assert_array_equal(got[whole], want[whole])
        assert (np.abs(got - want) < 2.0 ** -133 * scale).all()
        b = x.to(BF16)
        got = ref.f64(hs.score_packed(table, b.to(device())))[:, 0]
        np.testing.assert_array_equal(got, ref.f64(b).sum(axis=1) * scale)


def test_score_packed_strided_out_and_equal_rows():
    rng = np.random.default_rng(6)
    table, values = packed_table(rng, 333, 256, 64, BF16)
    same = table.data[7].clone()
    table.data[300] = same
    table.scales[300] = table.scales[7]
    x = torch.randn(9, 256, device=device())
    buf = torch.full((9, 400), 7.0, device=device())
    got = hs.score_packed(table, x, out=buf[:, :333])
    assert torch.all(buf[:, 333:] == 7.0)
    assert torch.equal(got[:, 7], got[:, 300])
    assert torch.equal(got, hs.score_packed(table, x))
    # a NaN in one row of x stays in that row
    x[4, 100] = float("nan")
    bad = hs.score_packed(table, x)
    assert torch.isnan(bad[4]).all() and torch.equal(bad[:4], got[:4]) and \
        torch.equal(bad[5:], got[5:])


def test_score_packed_large_table_offsets():
    """More than 4 GiB of codes: rows at the end score as in a table of their own."""
    rows, dim = 2_200_000, 4096
    codes = torch.zeros((rows, dim // 2), dtype=torch.uint8, device=device())
    scales = torch.ones((rows, dim // 128), dtype=BF16, device=device())
    codes[-100:] = torch.randint(0, 256, (100, dim // 2), device=device(), dtype=torch.uint8)
    x = torch.randn(2, dim, device=device()).to(BF16)
    got = hs.score_packed(hs.RowTable(codes, scales, group=128), x)
    tail = hs.score_packed(hs.RowTable(codes[-100:].clone(), scales[-100:].clone(), group=128), x)
    want, bound = ref.score_packed(ref.unpack(codes[-100:], scales[-100:], 128), ref.f64(x), 128)
    ref.check(got[:, -100:], want, bound, F32)
    ref.check(tail, want, bound, F32)
    assert torch.all(got[:, :-100] == 0)


# ------------------------------------------------------------------ adjustments

def ragged(rng, rows, each, cols, outside=True):
    n = rng.integers(0, each + 1, rows)
    n[rng.integers(0, rows)] = each
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    ids = np.minimum(np.exp(rng.random(off[-1]) * np.log(cols + 1)).astype(np.int64) - 1, cols - 1)
    if outside and len(ids) > 4:
        ids[rng.random(len(ids)) < 0.03] = -5
        ids[rng.random(len(ids)) < 0.03] = cols
    return ids.astype(np.int32), off


def run_adjust(rng, rows, cols, dtype, seen=True, bias=True, allow="rows", scores=None, each=200):
    dev = device()
    if scores is None:
        scores = torch.from_numpy((4 * rng.standard_normal((rows, cols))).astype(np.float32))
    scores = scores.to(dtype)
    kw, rk = {}, {}
    if seen:
        ids, off = ragged(rng, rows, each, cols)
        rk.update(seen=ids, seen_off=off, prompt_len=rng.integers(0, each, rows).astype(np.int32),
                  repetition=(0.5 + rng.random(rows)).astype(np.float32),
                  frequency=rng.standard_normal(rows).astype(np.float32),
                  presence=rng.standard_normal(rows).astype(np.float32))
    if bias:
        ids, off = ragged(rng, rows, 30, cols)
        rk.update(bias_id=ids, bias_off=off,
                  bias=(5 * rng.standard_normal(len(ids))).astype(np.float32))
    kw = {n: torch.from_numpy(v).to(dev) for n, v in rk.items()}
    if allow:
        ok = rng.random((rows if allow == "rows" else 1, cols)) < 0.6
        ok[rng.integers(0, len(ok))] = False            # a row whose mask leaves nothing
        words = ref.mask_words(ok).to(dev)
        kw["allow"] = words if allow == "rows" else words[0]
        rk["allow"] = np.broadcast_to(ok, (rows, cols))
    want, mag = ref.adjust(ref.f64(scores), **rk)
    bound = 8 * 2.0 ** -24 * np.where(np.isfinite(mag), mag, 0.0)
    dev_scores = scores.to(dev)
    got = hs.adjust_scores(dev_scores, **kw)
    ref.check(got, want, bound, dtype, f"{rows} x {cols}")
    assert torch.equal(dev_scores.cpu().view(-1).view(torch.uint8),
                       scores.reshape(-1).view(torch.uint8))     # the input stays
    hs.adjust_scores(dev_scores, out=dev_scores, **kw)           # in place: the same bits
    assert torch.equal(dev_scores.view(-1).view(torch.uint8), got.view(-1).view(torch.uint8))
    return kw, got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (1, 2047), (2, 2049),
                                       (5, 8192), (1, 32_000), (3, 50_257), (130, 8200),
                                       (300, 40_001)])
def test_adjust_sizes(dtype, rows, cols):
    rng = np.random.default_rng(rows * 7 + cols)
    run_adjust(rng, rows, cols, dtype)


@pytest.mark.parametrize("seen,bias,allow", [(True, False, None), (False, True, None),
                                             (False, False, "rows"), (False, False, "one"),
                                             (False, False, None), (True, True, "one")])
def test_adjust_parts(seen, bias, allow):
    rng = np.random.default_rng(11)
    run_adjust(rng, 4, 5000, F32, seen, bias, allow)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_adjust_infinities_nan_and_lowest(dtype):
    """Infinities, NaN and the type's lowest value: kept where allowed, -inf where not."""
    rng = np.random.default_rng(12)
    s = 4 * rng.standard_normal((6, 3000)).astype(np.float32)
    low = torch.finfo(dtype).min
    for v in (np.inf, -np.inf, np.nan, low, 0.0, -0.0):
        s[rng.integers(0, 6, 400), rng.integers(0, 3000, 400)] = v
    run_adjust(rng, 6, 3000, dtype, scores=torch.from_numpy(s), seen=False)
    run_adjust(rng, 6, 3000, dtype, scores=torch.from_numpy(s), seen=False, bias=False,
               allow="rows")


def test_adjust_long_history_counts_and_last_bias():
    """One token seen 100,000 times; the same bias column given many times."""
    dev = device()
    n = 100_000
    seen = torch.full((n + 3,), 5, dtype=torch.int32, device=dev)
    seen[-3:] = torch.tensor([9, 9, 6], dtype=torch.int32)
    off = torch.tensor([0, n + 3], dtype=torch.int64, device=dev)
    bid = torch.tensor([3, 3, 4, 3, 4], dtype=torch.int32, device=dev)
    b = torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0], device=dev)
    boff = torch.tensor([0, 5], dtype=torch.int64, device=dev)
    s = torch.ones(1, 10, device=dev)
    got = hs.adjust_scores(s, seen=seen, seen_off=off,
                           prompt_len=torch.tensor([n - 1000], dtype=torch.int32, device=dev),
                           repetition=torch.tensor([2.0], device=dev),
                           frequency=torch.tensor([0.5], device=dev),
                           presence=torch.tensor([0.25], device=dev), bias_id=bid, bias=b,
                           bias_off=boff).cpu()[0]
    want = torch.ones(10)
    want[5] = 0.5 - 0.5 * 1000 - 0.25
    want[9] = 0.5 - 0.5 * 2 - 0.25
    want[6] = 0.5 - 0.5 - 0.25
    want[3], want[4] = 9.0, 17.0
    assert torch.equal(got, want)


def test_adjust_strides_and_alignment():
    """Rows inside wider buffers, odd strides and starts; what lies around stays."""
    rng = np.random.default_rng(13)
    kw, want = run_adjust(rng, 7, 3001, BF16)
    dev = device()
    src = torch.full((7, 3017), 3.0, dtype=BF16, device=dev)
    # (undo: the scores of run_adjust come from the same generator)
    rng = np.random.default_rng(13)
    s = torch.from_numpy((4 * rng.standard_normal((7, 3001))).astype(np.float32)).to(BF16)
    for a in (0, 1, 8):
        view = src[:, a:a + 3001]
        view.copy_(s)
        dst = torch.full((7, 3024), 4.0, dtype=BF16, device=dev)
        out = dst[:, 5:5 + 3001]
        hs.adjust_scores(view, out=out, **kw)
        assert torch.equal(out, want)
        assert torch.all(dst[:, :5] == 4.0) and torch.all(dst[:, 5 + 3001:] == 4.0)


def test_adjust_offsets_are_clamped():
    """Row offsets outside their list, and a decreasing pair, read nothing outside."""
    dev = device()
    s = torch.zeros(4, 64, device=dev)
    seen = torch.tensor([1, 2, 3], dtype=torch.int32, device=dev)
    off = torch.tensor([-7, 1, 0, 2, 99], dtype=torch.int64, device=dev)   # row 1 is reversed
    got = hs.adjust_scores(s, seen=seen, seen_off=off,
                           presence=torch.ones(4, device=dev)).cpu()
    want = torch.zeros(4, 64)
    want[0, 1] = want[2, 1] = want[2, 2] = want[3, 3] = -1.0
    assert torch.equal(got, want)
    # the ends of int64, for both lists: the second row has all of them
    lo, hi = -2 ** 63, 2 ** 63 - 1
    off = torch.tensor([hi, lo, hi, hi, lo], dtype=torch.int64, device=dev)
    got = hs.adjust_scores(s, seen=seen, seen_off=off, presence=torch.ones(4, device=dev),
                           bias_id=seen, bias=torch.full((3,), 0.25, device=dev),
                           bias_off=off).cpu()
    want = torch.zeros(4, 64)
    want[1, 1:4] = -0.75
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(300, 40_001), (130, 40_007), (2, 3001)])
def test_adjust_more_marked_columns_than_the_table_holds(dtype, rows, cols):
    """Ranges of columns with more than 1,536 seen or biased ones are taken in pieces:
    marks over the whole row, in the second half of its first range, at its end, in one list
    and in both, entries in any order, some of them again and again."""
    rng = np.random.default_rng(cols)
    dev = device()
    width = min(10_240, cols)
    regions = [(0, cols, 0.9), (width // 2, width, 1.0), (0, width, 0.25), (cols - 4000, cols, 0.8),
               (0, cols, 0.05)]

    def entries():
        off, ids = [0], []
        for r in range(rows):
            if r < 2 * len(regions):
                lo, hi, p = regions[r % len(regions)]
                lo = max(lo, 0)
                c = rng.permutation(np.flatnonzero(rng.random(hi - lo) < p) + lo)
                c = np.concatenate([c, rng.choice(c, len(c) // 3), [-1, cols]])
            else:
                c = rng.integers(0, cols, rng.integers(0, 40))
            ids.append(c)
            off.append(off[-1] + len(c))
        return np.concatenate(ids).astype(np.int32), np.array(off, dtype=np.int64)

    seen, seen_off = entries()
    bias_id, bias_off = entries()
    ok = rng.random((rows, cols)) < 0.8
    rk = dict(seen=seen, seen_off=seen_off, bias_id=bias_id, bias_off=bias_off,
              bias=(5 * rng.standard_normal(len(bias_id))).astype(np.float32),
              prompt_len=(rng.random(rows) * np.diff(seen_off)).astype(np.int32),
              repetition=(0.5 + rng.random(rows)).astype(np.float32),
              frequency=rng.standard_normal(rows).astype(np.float32),
              presence=rng.standard_normal(rows).astype(np.float32))
    kw = {n: torch.from_numpy(v).to(dev) for n, v in rk.items()}
    scores = torch.from_numpy((4 * rng.standard_normal((rows, cols))).astype(np.float32)).to(dtype)
    want, mag = ref.adjust(ref.f64(scores), allow=ok, **rk)
    dev_scores = scores.to(dev)
    got = hs.adjust_scores(dev_scores, allow=ref.mask_words(ok).to(dev), **kw)
    # (at most six roundings of values that the magnitudes bound)
    ref.check(got, want, 8 * 2.0 ** -24 * np.where(np.isfinite(mag), mag, 0.0), dtype)
    hs.adjust_scores(dev_scores, allow=ref.mask_words(ok).to(dev), out=dev_scores, **kw)
    assert torch.equal(dev_scores, got)


# ------------------------------------------------------------------ top-k

def check_topk(scores, k):
    got_s, got_i = hs.topk_rows(scores, k)
    want_s, want_i = ref.topk(scores.float().cpu().numpy(), k)
    np.testing.assert_array_equal(got_i.cpu().numpy(), want_i)
    np.testing.assert_array_equal(got_s.cpu().numpy(), want_s)


@pytest.mark.parametrize("rows,cols,k", [
    (1, 1, 1), (1, 1, 5), (3, 7, 7), (2, 100, 1024), (1, 4095, 3), (1, 4096, 512), (2, 4097, 513),
    (1, 32_000, 50), (5, 50_257, 1), (700, 333, 20), (70, 9001, 100), (2, 100_003, 1024),
    (24, 250_000, 100), (1, 1_000_003, 64),
    (5, 72_232, 9), (2, 3_000_001, 300), (1, 6_000_000, 5), (1, 40_000, 1024), (3, 33_001, 256)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_topk_sizes(rows, cols, k, dtype):
    rng = np.random.default_rng(rows + cols + k)
    s = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).to(dtype)
    check_topk(s.to(device()), k)


@pytest.mark.parametrize("k", [1, 10, 300, 1024])
def test_topk_hard_orders(k):
    """Equal scores, ascending, descending, a few distinct values, masked rows, NaN."""
    rng = np.random.default_rng(k)
    cols = 40_000
    s = np.zeros((9, cols), dtype=np.float32)
    s[1] = np.arange(cols)
    s[2] = -np.arange(cols)
    s[3] = rng.integers(0, 3, cols)
    s[4] = -np.inf
    s[5, :] = -np.inf
    s[5, [17, 39_999]] = -3.4e38
    s[6] = np.where(rng.random(cols) < 0.5, np.nan, rng.standard_normal(cols))
    s[7] = np.where(rng.random(cols) < 0.5, 0.0, -0.0)
    s[8, 12_345:12_400] = np.inf
    check_topk(torch.from_numpy(s).to(device()), k)


@pytest.mark.parametrize("cols,k", [(300_000, 20), (9_000_000, 20), (2_000_000, 700)])
def test_topk_long_rows_of_equal_scores(cols, k):
    """More strips, and groups of them, with the k-th best score than their lists hold."""
    s = torch.zeros(2, cols, device=device())
    s[1, ::3] = 1.0
    s[1, cols - 5] = 2.0
    s[0, 1000:] = -1.0
    got_s, got_i = hs.topk_rows(s, k)
    assert got_i[0].tolist() == list(range(k)) and torch.all(got_s[0] == 0)
    first = [cols - 5] + [3 * i for i in range(k)]
    assert got_i[1].tolist() == first[:k]
    assert got_s[1].tolist() == [2.0] + [1.0] * (k - 1)


def test_long_rows_past_32_bits():
    """A row of more than 4 GiB, and rows that start past it."""
    dev = device()
    cols = 2 ** 31 - 1
    s = torch.full((1, cols), -2.0, dtype=BF16, device=dev)
    at = [3, 2 ** 30 + 11, 2 ** 31 - 2]
    s[0, at[0]], s[0, at[1]], s[0, at[2]] = 1.0, 3.0, 2.0
    got_s, got_i = hs.topk_rows(s, 3)
    assert got_i[0].tolist() == [at[1], at[2], at[0]] and got_s[0].tolist() == [3.0, 2.0, 1.0]
    ids = torch.tensor([at[2], 5], dtype=torch.int32, device=dev)
    off = torch.tensor([0, 2], dtype=torch.int64, device=dev)
    one = torch.ones(1, device=dev)
    hs.adjust_scores(s, seen=ids, seen_off=off, presence=one, out=s)
    assert s[0, at[2]].item() == 1.0 and s[0, 5].item() == -3.0 and s[0, 6].item() == -2.0
    s = s.view(-1)[:2 ** 31 - 32768].view(-1, 32768)     # 65,535 rows
    rows = s.shape[0]
    s.fill_(0.5)
    s[rows - 1, 77] = 9.0
    off = torch.zeros(rows + 1, dtype=torch.int64, device=dev)
    off[-1] = 1
    hs.adjust_scores(s, bias_id=torch.tensor([4], dtype=torch.int32, device=dev), bias=one,
                     bias_off=off, out=s)
    assert s[rows - 1, 4].item() == 1.5 and s[rows - 2, 4].item() == 0.5
    got_s, got_i = hs.topk_rows(s, 2)
    assert got_i[rows - 1].tolist() == [77, 4] and got_i[rows - 2].tolist() == [0, 1]


def test_topk_strides_and_many_rows():
    rng = np.random.default_rng(2)
    buf = torch.from_numpy(rng.standard_normal((40, 5003)).astype(np.float32)).to(device())
    check_topk(buf[:, 1:5000], 33)
    check_topk(buf.to(BF16)[:, 3:4999], 33)
    check_topk(torch.from_numpy(rng.standard_normal((3000, 700)).astype(np.float32)).to(device()),
               9)


# ------------------------------------------------------------------ together

def test_decoding_step_chain_in_a_graph():
    """Token rows -> (states) -> logits of the packed head -> penalties and masks ->
    candidates, captured and replayed, each replay against the eager call and the
    64-bit reference."""
    dev = device()
    rng = np.random.default_rng(21)
    vocab, dim, batch, k = 5000, 256, 6, 20
    weights = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32))
    table = hs.pack_rows(weights.to(dev), group=32)
    ids = torch.zeros(batch, dtype=torch.int32, device=dev)
    seen = torch.zeros(batch * 8, dtype=torch.int32, device=dev)
    off = torch.arange(batch + 1, device=dev) * 8
    ok = rng.random((batch, vocab)) < 0.5
    ok[2] = False
    ok[3] = False
    ok[3, 77] = True
    words = ref.mask_words(ok).to(dev)
    rep = torch.full((batch,), 1.5, device=dev)
    h = torch.empty(batch, dim, dtype=BF16, device=dev)
    logits = torch.empty(batch, vocab, device=dev)
    out = (torch.empty(batch, k, device=dev), torch.empty(batch, k, dtype=torch.int32, device=dev))
    ws = torch.empty(hs.hs_topk_rows_bytes(batch, vocab, k), dtype=torch.uint8, device=dev)

    def step():
        hs.embed(table, ids, scale=dim ** -0.5, out=h)
        hs.score_packed(table, h, out=logits)
        hs.adjust_scores(logits, allow=words, seen=seen, seen_off=off, repetition=rep, out=logits)
        hs.topk_rows(logits, k, out=out, ws=ws)

    s = torch.cuda.Stream(dev)
    step()                                # (warm-up)
    torch.cuda.synchronize(dev)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    values = ref.unpack(table.data, table.scales, 32)
    for rep_no in range(3):
        ids.copy_(torch.from_numpy(rng.integers(0, vocab, batch)))
        seen.copy_(torch.from_numpy(rng.integers(0, vocab, batch * 8)))
        step()
        eager = [t.clone() for t in (h, logits, out[0], out[1])]
        for t in (logits, out[0], out[1]):
            t.fill_(-5)
        torch.cuda.synchronize(dev)
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize(dev)
        for a, b in zip(eager, (h, logits, out[0], out[1])):
            assert torch.equal(a, b)
        x, bound = ref.score_packed(values, ref.f64(h), 32)
        want, mag = ref.adjust(x, seen=seen.cpu().numpy(), seen_off=off.cpu().numpy(),
                               repetition=rep.cpu().numpy(), allow=ok)
        ref.check(logits, want, 2 * bound + 8 * 2.0 ** -24 * mag, F32)
        ts, ti = ref.topk(logits.cpu().numpy(), k)
        np.testing.assert_array_equal(out[1].cpu().numpy(), ti)
        np.testing.assert_array_equal(out[0].cpu().numpy(), ts)
        assert (ti[2] == -1).all() and ti[3][0] == 77 and (ti[3][1:] == -1).all()


@pytest.mark.parametrize("per_request", [False, True])
@pytest.mark.parametrize("qt", [F32, BF16])
def test_run_packed_window(per_request, qt):
    """The window over a packed corpus with filters: every request gets the best allowed
    chunks of its own query row (in batches smaller than the distinct queries)."""
    dev = device()
    rng = np.random.default_rng(31)
    R, d, N, k, group = 300, 128, 4099, 12, 64
    keys = rng.integers(0, 90, R).astype(np.int64) * 1_000_003 - 40
    rows = rng.standard_normal((90, d)).astype(np.float32)
    q = torch.from_numpy(rows[(keys + 40) // 1_000_003]).to(qt)
    corpus = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32))
    table = hs.pack_rows(corpus.to(dev), group=group)
    values = ref.unpack(table.data, table.scales, group)
    if per_request:      # equal requests have equal filters
        ok = (rng.random((90, N)) < 0.3)[(keys + 40) // 1_000_003]
    else:
        ok = np.broadcast_to(rng.random(N) < 0.3, (R, N))
    words = ref.mask_words(ok if per_request else ok[0]).to(dev)
    dt = hs.HS_F32 if qt == F32 else hs.HS_BF16
    m = hs.MergedRetrieval(R, d, N, k, dt, dt, device=dev)
    m.enable_packed(batch=32)
    m.run_packed(torch.from_numpy(keys).to(dev), q.to(dev), table, allow=words,
                 stream=torch.cuda.current_stream(dev))
    torch.cuda.synchronize(dev)
    dd = oracle.dedup(keys)
    nu = dd["n_unique"]
    assert int(m.n_unique.item()) == nu
    exact, bound = ref.score_packed(values, ref.f64(q), group)
    exact = np.where(ok, exact, -np.inf)
    gi, gs = m.out_index.cpu().numpy(), m.out_score.cpu().numpy().astype(np.float64)
    for r in range(R):
        mine = exact[r, gi[r]]
        tol = bound[r, gi[r]] + HALF32 * np.abs(mine)
        assert len(set(gi[r])) == k and np.isfinite(mine).all()
        assert (np.abs(gs[r] - mine) <= tol).all()
        kth = np.sort(exact[r])[-k]
        assert (mine >= kth - 2 * bound[r].max()).all()
        assert (np.diff(gs[r]) <= 0).all()


def test_streams_and_two_calls_at_once():
    """Calls on two streams with workspaces of their own, while the default stream is
    current: results as alone."""
    dev = device()
    rng = np.random.default_rng(41)
    s = [torch.from_numpy(rng.standard_normal((8, 60_000)).astype(np.float32)).to(dev)
         for _ in range(2)]
    want = [hs.topk_rows(x, 40) for x in s]
    torch.cuda.synchronize(dev)
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    for _ in range(3):
        got = [hs.topk_rows(x, 40, stream=st) for x, st in zip(s, streams)]
        torch.cuda.synchronize(dev)
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_each_operator_twice_at_once():
    """The other operators on two streams at once, each call with tensors (and a workspace)
    of its own: results as alone."""
    dev = device()
    rng = np.random.default_rng(43)
    calls = []
    for i in range(2):
        table, _ = packed_table(rng, 20_000, 512, 64, BF16)
        x = torch.from_numpy(rng.standard_normal((7 + 20 * i, 512)).astype(np.float32)).to(dev)
        ids = torch.from_numpy(rng.integers(-1, 20_000, 9000 + 9000 * i)).to(dev)
        d = torch.from_numpy(rng.standard_normal((len(ids), 130)).astype(np.float32)).to(dev)
        s = torch.from_numpy(rng.standard_normal((9, 30_000)).astype(np.float32)).to(dev)
        seen = torch.from_numpy(rng.integers(0, 30_000, 9 * 50).astype(np.int32)).to(dev)
        off = torch.arange(10, device=dev) * 50
        pen = torch.ones(9, device=dev)
        w = torch.from_numpy(rng.standard_normal((3000, 256)).astype(np.float32)).to(dev)
        calls.append([
            lambda st, t=table, i=ids: hs.embed(t, i, scale=3.0, stream=st),
            lambda st, i=ids, d=d: hs.embed_grad(d, i, 20_000, stream=st),
            lambda st, t=table, x=x: hs.score_packed(t, x, stream=st),
            lambda st, s=s, i=seen, o=off, p=pen: hs.adjust_scores(
                s, seen=i, seen_off=o, frequency=p, stream=st),
            lambda st, w=w: hs.pack_rows(w, group=64, stream=st).data])
    want = [[call(None) for call in side] for side in calls]
    torch.cuda.synchronize(dev)
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    for _ in range(3):
        got = [[], []]
        for pair in zip(*calls):
            for call, st, to in zip(pair, streams, got):
                to.append(call(st))
        torch.cuda.synchronize(dev)
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
