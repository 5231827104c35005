"""Embedding lookup (hs_embed), packing (hs_pack_rows) and the lookup's gradient
(hs_embed_grad) against 64-bit references."""
import numpy as np
import pytest
import torch

import paper_2607_22578_amd as hs
import rows_reference as ref
from gpu_harness import device

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def make_table(rng, kind, rows, dim, group=32, scale_dtype=BF16):
    """(RowTable, its fp64 values, roundings per value in fp32)."""
    dev = device()
    x = torch.from_numpy(rng.standard_normal((rows, dim)).astype(np.float32))
    if kind == "fp4":
        codes = torch.from_numpy(rng.integers(0, 256, (rows, dim // 2)).astype(np.uint8))
        sc = torch.from_numpy((0.01 + rng.random((rows, dim // group))).astype(np.float32)
                              ).to(scale_dtype)
        t = hs.RowTable(codes.to(dev), sc.to(dev), group=group)
        return t, ref.unpack(codes, sc, group), 2
    if kind == "fp8":
        codes = x.to(torch.float8_e4m3fn)
        sc = torch.from_numpy((0.01 + rng.random(rows)).astype(np.float32))
        v = codes.float().double().numpy() * ref.f64(sc)[:, None]
        return hs.RowTable(codes.to(dev), sc.to(dev)), v, 2
    x = x.to(F32 if kind == "f32" else BF16)
    return hs.RowTable(x.to(dev)), ref.f64(x), 1


@pytest.mark.parametrize("kind,dim,group", [
    ("f32", 1, 0), ("f32", 12, 0), ("f32", 771, 0), ("f32", 1024, 0), ("bf16", 3, 0),
    ("bf16", 8, 0), ("bf16", 12, 0), ("bf16", 4096, 0), ("bf16", 16384, 0), ("fp8", 16, 0),
    ("fp8", 7, 0), ("fp8", 1032, 0), ("fp4", 32, 32), ("fp4", 96, 32), ("fp4", 4160, 64),
    ("fp4", 1152, 128)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_embed_types_and_sizes(kind, dim, group, out):
    rng = np.random.default_rng(dim * 31 + len(kind))
    rows = 301
    sdt = F32 if dim % 64 == 32 else BF16
    table, values, ops = make_table(rng, kind, rows, dim, group, sdt)
    for n, idt in [(0, torch.int32), (1, torch.int64), (5, torch.int32), (777, torch.int64)]:
        ids = rng.integers(-3, rows + 3, n)
        if n > 4:
            ids[:3] = rows - 1, 0, 2 ** 31 - 1
        got = hs.embed(table, torch.from_numpy(ids).to(idt).to(device()), scale=1.7, pad_id=7,
                       out_dtype=out)
        assert got.dtype == out and got.shape == (n, dim)
        want = ref.embed(values, ids, 1.7, 7)
        ref.check(got, want, ops * 2.0 ** -24 * np.abs(want), out, f"{kind} {dim} {n}")


def test_embed_shapes_out_and_unaligned_out():
    rng = np.random.default_rng(1)
    table, values, _ = make_table(rng, "bf16", 50, 64)
    ids = rng.integers(0, 50, (3, 4, 5))
    dev_ids = torch.from_numpy(ids).to(device())
    got = hs.embed(table, dev_ids, scale=2.0)
    assert got.shape == (3, 4, 5, 64) and got.dtype == BF16
    ref.check(got, ref.embed(values, ids, 2.0), 0.0, BF16)
    # rows that start 2 bytes past 16: the narrow accesses; what lies around stays
    buf = torch.full((60 * 64 + 9,), 5.0, dtype=BF16, device=device())
    out = buf[1:1 + 60 * 64].view(3, 4, 5, 64)
    hs.embed(table, dev_ids, scale=2.0, out=out)
    assert torch.equal(out, got)
    assert buf[0].item() == 5.0 and torch.all(buf[1 + 60 * 64:] == 5.0)


def test_embed_offsets_past_32_bits():
    """A table of more than 4 GiB: its last rows."""
    rows, dim = 300_000, 8192
    data = torch.zeros((rows, dim), dtype=BF16, device=device())
    at = torch.tensor([0, 131_072, 262_144, rows - 1], device=device())
    data[at] = torch.randn(4, dim, device=device()).to(BF16)
    got = hs.embed(hs.RowTable(data), at)
    assert torch.equal(got, data[at])


@pytest.mark.parametrize("src", [F32, BF16])
@pytest.mark.parametrize("scale_dtype", [F32, BF16])
@pytest.mark.parametrize("group,dim,rows", [(32, 32, 1), (32, 96, 700), (64, 320, 37),
                                            (128, 128, 65), (128, 1024, 129)])
def test_pack_rows_bit_exact(src, scale_dtype, group, dim, rows):
    rng = np.random.default_rng(group + dim)
    x = rng.standard_normal((rows, dim)).astype(np.float32)
    x *= np.exp(rng.standard_normal((rows, 1)) * 8)     # scales far apart
    x[0, :group] = 0.0                                  # a group of zeros
    if rows > 3:
        # a group whose scale is 1: every midpoint, tie and end of the E2M1 range
        x[1, :group] = np.resize([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -5, .2, 5.5], group)
        x[2, :group] = np.float32(1e-42)                # subnormal magnitudes
        x[3, :group] = np.float32(3.0e38)               # near the top
    t = torch.from_numpy(x).to(src)
    packed = hs.pack_rows(t.to(device()), group=group, scale_dtype=scale_dtype)
    codes, scales = ref.pack(t, group, scale_dtype)
    assert packed.scales.dtype == scale_dtype
    assert torch.equal(packed.scales.cpu(), scales)
    np.testing.assert_array_equal(packed.data.cpu().numpy(), codes.numpy())


def run_grad(rng, n, rows, dim, din, dout, idt=torch.int32, pad=-1, ids=None, accumulate=False,
             scale=1.3):
    if ids is None:
        # text-like frequencies: one token very often, most hardly ever
        ids = np.minimum(np.exp(rng.random(n) * np.log(rows + 1)).astype(np.int64) - 1, rows - 1)
        ids[rng.random(n) < 0.02] = -1
    d = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).to(din)
    want, bound = ref.embed_grad(ref.f64(d), ids, rows, scale, pad)
    start = torch.from_numpy(rng.standard_normal((rows, dim)).astype(np.float32)).to(dout)
    out = start.to(device())
    hs.embed_grad(d.to(device()), torch.from_numpy(ids).to(idt).to(device()), rows, scale=scale,
                  pad_id=pad, out=out, accumulate=accumulate)
    if accumulate:
        old = ref.f64(start)
        bound = bound + 2.0 ** -24 * (np.abs(want) + bound + np.abs(old))
        ok = (ids >= 0) & (ids < rows) & (ids != pad)
        absent = np.ones(rows, bool)
        absent[ids[ok]] = False
        assert torch.equal(out.cpu()[torch.from_numpy(absent)], start[torch.from_numpy(absent)])
        want = want + old
    ref.check(out, want, bound, dout, f"n={n} rows={rows} dim={dim}")
    return d, ids, out


@pytest.mark.parametrize("n,rows,dim", [
    (0, 5, 16), (1, 1, 1), (1, 1000, 8), (63, 7, 24), (64, 513, 40), (65, 511, 33), (129, 3, 520),
    (1000, 100_000, 16), (4095, 300, 64), (4096, 512, 72), (4097, 513, 72),
    (10_240, 700, 20), (10_241, 700, 20), (11_000, 200, 12), (5000, 1, 136),
    (20_011, 50_257, 100), (70_001, 9, 48), (300_000, 40_000, 24)])
@pytest.mark.parametrize("din,dout", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
def test_embed_grad_sizes(n, rows, dim, din, dout):
    rng = np.random.default_rng(n + rows + dim)
    run_grad(rng, n, rows, dim, din, dout, torch.int64 if n % 2 else torch.int32)


@pytest.mark.parametrize("n,rows,dim", [(1, 9001, 515), (40, 30_001, 515), (7, 70_000, 33),
                                        (300, 20_003, 2049), (2000, 40_000, 1)])
@pytest.mark.parametrize("din,dout", [(F32, BF16), (BF16, F32)])
def test_embed_grad_few_tokens_of_many(n, rows, dim, din, dout):
    """Rows of zeros of odd widths, written by both launches."""
    rng = np.random.default_rng(n + rows)
    ids = rng.integers(0, rows, n)
    ids[:2] = (rows - 1, 0)[:n]
    run_grad(rng, n, rows, dim, din, dout, ids=ids)


@pytest.mark.parametrize("dim,din", [(3, F32), (20, BF16), (128, F32), (129, F32), (256, BF16),
                                     (264, BF16)])
def test_embed_grad_runs_over_chunk_ends(dim, din):
    """Tokens of lengths around multiples of 8 to 64 places, and over 23 to 70 of those."""
    rng = np.random.default_rng(dim)
    runs = [8, 1, 7, 16, 9, 63, 64, 65, 128] + [c * k + e for c in (8, 16, 64)
                                              for k in (22, 23, 24, 25) for e in (-1, 0, 1)]
    runs += [8 * 63, 8 * 64, 8 * 65 + 1, 16 * 70, 64 * 70, 1, 64 * 30 + 5]
    for lengths in (runs, runs[::-1], [64 * 24], [8 * 24, 8 * 24], [5000, 1, 9000]):
        ids = np.repeat(np.arange(len(lengths)), lengths)
        run_grad(rng, len(ids), len(lengths), dim, din, F32, ids=rng.permutation(ids))
    # and where chunks have 64 places
    ids = np.concatenate([np.repeat(np.arange(len(runs)), runs), np.arange(len(runs), 200_000)])
    run_grad(rng, len(ids), 200_000, dim, din, F32, ids=rng.permutation(ids))


@pytest.mark.parametrize("dim", [64, 101, 1544])
@pytest.mark.parametrize("dout", [F32, BF16])
def test_embed_grad_accumulate_and_padding(dim, dout):
    rng = np.random.default_rng(dim)
    ids = rng.integers(-2, 44, 3000)
    run_grad(rng, 3000, 40, dim, BF16, dout, pad=11, ids=ids, accumulate=True)
    run_grad(rng, 3000, 40, dim, BF16, dout, pad=11, ids=ids)
    run_grad(rng, 50, 40, dim, F32, dout, ids=np.full(50, -1), accumulate=True)   # no token at all
    run_grad(rng, 50, 40, dim, F32, dout, ids=np.full(50, 40))


@pytest.mark.parametrize("din,dim", [
    (F32, 255), (F32, 257), (F32, 258), (F32, 259), (F32, 771), (F32, 1025), (F32, 2049),
    (BF16, 511), (BF16, 513), (BF16, 515), (BF16, 519), (BF16, 1025), (BF16, 2049)])
@pytest.mark.parametrize("dout", [F32, BF16])
def test_embed_grad_accumulates_each_column_once(din, dim, dout):
    """Widths whose last columns are fewer than a lane's, many of them where the row's last
    lane is in another wave than the one before: tokens that occur once, over a few and
    over many chunks."""
    rng = np.random.default_rng(dim)
    lengths = [1] * 300 + [2, 9, 40, 100, 300, 700]
    ids = rng.permutation(np.repeat(np.arange(len(lengths)), lengths))
    d, _, _ = run_grad(rng, len(ids), len(lengths) + 3, dim, din, dout, ids=ids, accumulate=True)
    args = (d.to(device()), torch.from_numpy(ids).to(device()), len(lengths) + 3)
    plain = hs.embed_grad(*args, out_dtype=dout)
    for _ in range(3):     # added to zeros: the plain gradient
        out = torch.zeros_like(plain)
        hs.embed_grad(*args, out=out, accumulate=True)
        assert torch.equal(out, plain)


@pytest.mark.parametrize("n", [1, 100, 4096, 30_000])
def test_embed_grad_one_token_and_all_distinct(n):
    rng = np.random.default_rng(n)
    run_grad(rng, n, 77, 72, BF16, F32, ids=np.full(n, 76))
    run_grad(rng, n, n, 72, BF16, F32, ids=rng.permutation(n))


def test_embed_grad_wide_keys():
    """Ids of more than 18 bits: three and four digits."""
    rng = np.random.default_rng(8)
    for n in (700, 9000):
        for rows in (300_001, 2 ** 24 + 5):
            ids = np.sort(rng.integers(rows - 40, rows, n))[::-1].copy()
            ids[::7] = rng.integers(0, 30, len(ids[::7]))
            d = torch.from_numpy(rng.standard_normal((n, 4)).astype(np.float32))
            out = hs.embed_grad(d.to(device()), torch.from_numpy(ids).to(device()), rows).cpu()
            want = torch.zeros(rows, 4, dtype=torch.float64)
            want.index_add_(0, torch.from_numpy(ids), d.double())
            cnt = np.bincount(ids).max()
            assert (out.double() - want).abs().max() <= (cnt + 2) * 2.0 ** -24 * cnt * 6


def test_embed_grad_offsets_past_32_bits():
    """More than 4 GiB of gradients, and of table: chosen rows and columns."""
    n, dim, rows = 280_000, 8192, 300_000
    dev = device()
    d = torch.zeros(n, dim, dtype=BF16, device=dev)
    ids = torch.arange(n, device=dev) + 7
    ids[-1000:] = rows - 1
    d[-1000:] = 1.0
    d[5] = 2.0
    d[-1001] = 3.0
    out = hs.embed_grad(d, ids, rows)
    assert torch.all(out[rows - 1] == 1000.0) and torch.all(out[12] == 2.0)
    assert torch.all(out[n - 1001 + 7] == 3.0)
    assert out[:7].abs().max().item() == 0 and out[n + 7:rows - 1].abs().max().item() == 0
    assert out[13:n - 1001 + 7].abs().max().item() == 0


def test_embed_grad_repeats_bit_for_bit_and_unaligned():
    rng = np.random.default_rng(4)
    d, ids, out = run_grad(rng, 50_000, 900, 72, BF16, F32)
    ids_d = torch.from_numpy(ids).to(torch.int32).to(device())
    again = hs.embed_grad(d.to(device()), ids_d, 900, scale=1.3, out_dtype=F32)
    assert torch.equal(out, again)
    # gradients that start 2 bytes past 16: the narrow accesses, the same sums
    buf = torch.zeros(50_000 * 72 + 8, dtype=BF16, device=device())
    odd = buf[1:1 + 50_000 * 72].view(50_000, 72)
    odd.copy_(d)
    tab = torch.full((900 * 72 + 3,), 9.0, device=device())
    res = tab[1:1 + 900 * 72].view(900, 72)
    hs.embed_grad(odd, ids_d, 900, scale=1.3, out=res)
    assert torch.equal(res, out)
    assert tab[0].item() == 9.0 and torch.all(tab[1 + 900 * 72:] == 9.0)


def test_embed_grad_matches_differences():
    """d(sum of w * embed(T)) / dT against differences of the forward pass in T (the
    lookup is linear: powers of two as steps make the differences exact up to rounding)."""
    rng = np.random.default_rng(5)
    rows, dim, n = 13, 24, 200
    t = torch.from_numpy(rng.integers(-8, 9, (rows, dim)).astype(np.float32))
    w = torch.from_numpy(rng.integers(-8, 9, (n, dim)).astype(np.float32))
    ids = torch.from_numpy(rng.integers(-1, rows, n)).to(device())
    grad = hs.embed_grad(w.to(device()), ids, rows, scale=0.5).cpu()

    def loss(x):
        return float((hs.embed(hs.RowTable(x.to(device())), ids, scale=0.5).cpu().double()
                      * w.double()).sum())

    for r, c in [(0, 0), (5, 23), (12, 7), (3, 11)]:
        up, down = t.clone(), t.clone()
        up[r, c] += 4.0
        down[r, c] -= 4.0
        # small integers times 1/2: every product and sum is exact
        assert (loss(up) - loss(down)) / 8.0 == float(grad[r, c])


def test_embed_and_grad_in_a_graph():
    """Both captured once and replayed on changing ids, with eager calls between, two
    graphs with workspaces of their own."""
    dev = device()
    rng = np.random.default_rng(9)
    rows, dim, n = 5000, 128, 6000
    table = hs.RowTable(torch.randn(rows, dim, device=dev).to(BF16))
    ids = torch.zeros(n, dtype=torch.int64, device=dev)
    d = torch.randn(n, dim, device=dev).to(BF16)
    s = torch.cuda.Stream(dev)
    graphs = []
    for _ in range(2):
        out = torch.empty(n, dim, dtype=BF16, device=dev)
        g_out = torch.empty(rows, dim, device=dev)
        ws = torch.empty(hs.hs_embed_grad_bytes(n, rows, dim), dtype=torch.uint8, device=dev)
        hs.embed(table, ids, out=out)     # (warm-up)
        hs.embed_grad(d, ids, rows, out=g_out, ws=ws)
        torch.cuda.synchronize(dev)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            hs.embed(table, ids, out=out)
            hs.embed_grad(d, ids, rows, out=g_out, ws=ws)
        graphs.append((g, out, g_out))
    for rep in range(4):
        ids.copy_(torch.from_numpy(rng.integers(-1, rows // (rep + 1), n)))
        want = hs.embed(table, ids), hs.embed_grad(d, ids, rows, out_dtype=F32)
        for g, out, g_out in graphs:
            out.fill_(-1)
            g_out.fill_(-1)
            torch.cuda.synchronize(dev)
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize(dev)
        for g, out, g_out in graphs:
            assert torch.equal(out, want[0]) and torch.equal(g_out, want[1])
