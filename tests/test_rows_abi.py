"""Refusals of the row-table operators: every entry point checks its arguments on the
host before any device call, so these run without a GPU."""
import ctypes
import os
import shutil

import pytest
import torch

import paper_2607_22578_amd as hs
from test_sanitizers import HIP_INC, HIP_LIB, ROOT, SAN, _env, _run

FAKE = 0x10000000   # never dereferenced: validation fails first, or there is nothing to do
BIG = 1 << 44       # apart from every FAKE range below
INVALID, UNSUP, WS, ALIGN = (hs.HS_ERR_INVALID_ARG, hs.HS_ERR_UNSUPPORTED, hs.HS_ERR_WORKSPACE,
                             hs.HS_ERR_ALIGNMENT)


def refused(code, call, *args, **kw):
    with pytest.raises(hs.HsError) as e:
        call(*args, **kw)
    assert e.value.status == code, (hs.hs_last_error(), args, kw)
    assert hs.hs_last_error()


def table(**kw):
    base = dict(data=FAKE, scale=BIG, rows=1000, dim=256, dtype=hs.HS_FP4_E2M1,
                scale_dtype=hs.HS_BF16, group=32)
    base.update(kw)
    return hs.hs_row_table(*(base[n] for n, _ in hs.hs_row_table._fields_))


BAD_TABLES = [
    (dict(rows=-1), INVALID), (dict(rows=2 ** 31), INVALID), (dict(dim=0), INVALID),
    (dict(dim=16385), INVALID), (dict(data=None), INVALID), (dict(scale=None), INVALID),
    (dict(dtype=9), UNSUP), (dict(group=16), UNSUP), (dict(group=0), UNSUP),
    (dict(dim=48), UNSUP), (dict(group=128, dim=192), UNSUP), (dict(scale_dtype=2), UNSUP),
    (dict(data=FAKE + 8), ALIGN), (dict(scale=BIG + 1), ALIGN),
    (dict(scale=BIG + 2, scale_dtype=hs.HS_F32), ALIGN),
    (dict(dtype=hs.HS_FP8_E4M3, scale=None), INVALID),
    (dict(dtype=hs.HS_FP8_E4M3, scale=BIG + 2), ALIGN),
    (dict(dtype=hs.HS_F32, data=FAKE + 4), ALIGN)]


@pytest.mark.parametrize("bad,code", BAD_TABLES)
def test_tables(bad, code):
    refused(code, hs.hs_embed, table(**bad), FAKE, 0, 4, 1.0, -1, 2 * BIG, hs.HS_F32)
    if bad.get("dtype") in (None, 9):
        refused(code, hs.hs_score_packed, table(**bad), 2 * BIG, hs.HS_F32, 4, 3 * BIG, hs.HS_F32,
                2 ** 31)


def test_embed():
    t = table()
    good = [t, FAKE, 0, 4, 1.0, -1, 2 * BIG, hs.HS_F32]
    for at, bad, code in [(1, None, INVALID), (1, FAKE + 2, ALIGN), (2, 2, INVALID),
                          (3, -1, INVALID), (3, 2 ** 30 + 1, INVALID),
                          (4, float("nan"), INVALID), (4, float("inf"), INVALID),
                          (6, None, INVALID), (6, 2 * BIG + 2, ALIGN), (7, hs.HS_FP8_E4M3, UNSUP),
                          (6, FAKE + 64, INVALID),       # inside the table
                          (1, 2 * BIG + 64, INVALID),    # ids inside out
                          (6, BIG + 64, INVALID)]:       # inside its scales
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_embed, *args)
    refused(ALIGN, hs.hs_embed, t, FAKE + 4, 1, 4, 1.0, -1, 2 * BIG, hs.HS_F32)
    assert hs._lib.hs_embed(None, FAKE, 0, 4, 1.0, -1, FAKE, 0, None) == INVALID
    hs.hs_embed(t, None, 0, 0, 1.0, -1, None, hs.HS_F32)             # no ids: nothing enqueued


def test_pack_rows():
    good = [FAKE, hs.HS_F32, 100, 64, 32, hs.HS_BF16, BIG, 2 * BIG]
    for at, bad, code in [(0, None, INVALID), (0, FAKE + 4, ALIGN), (1, 2, UNSUP),
                          (2, -1, INVALID), (3, 0, INVALID), (3, 48, UNSUP), (4, 48, UNSUP),
                          (5, 3, UNSUP), (6, None, INVALID), (6, BIG + 8, ALIGN),
                          (7, 2 * BIG + 1, ALIGN), (6, FAKE + 160, INVALID),
                          (7, BIG + 64, INVALID)]:
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_pack_rows, *args)
    hs.hs_pack_rows(None, hs.HS_F32, 0, 64, 32, hs.HS_BF16, None, None)


def test_embed_grad():
    need = hs.hs_embed_grad_bytes(100, 50, 64)
    assert need >= 4 * 100 * 4 + 51 * 4
    for bad in ((-1, 50, 64), (2 ** 30 + 1, 50, 64), (100, -1, 64), (100, 2 ** 31, 64),
                (100, 50, 0), (100, 50, 16385)):
        refused(INVALID, hs.hs_embed_grad_bytes, *bad)
    assert hs._lib.hs_embed_grad_bytes(1, 1, 1, None) == INVALID
    good = [FAKE, hs.HS_BF16, BIG, 0, 100, 50, 64, 1.0, -1, 0, 2 * BIG, hs.HS_F32, 3 * BIG, need]
    for at, bad, code in [(0, None, INVALID), (0, FAKE + 1, ALIGN), (1, 3, UNSUP),
                          (2, None, INVALID), (2, BIG + 2, ALIGN), (3, 7, INVALID),
                          (4, -1, INVALID), (5, -1, INVALID), (6, 0, INVALID),
                          (7, float("inf"), INVALID), (9, 2, INVALID), (10, None, INVALID),
                          (10, 2 * BIG + 2, ALIGN), (11, 2, UNSUP), (12, None, WS),
                          (12, 3 * BIG + 64, ALIGN), (13, need - 1, WS),
                          (10, FAKE + 64, INVALID)]:     # d_table inside d_out
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_embed_grad, *args)
    # nothing to write: an empty table, or nothing to add
    hs.hs_embed_grad(None, hs.HS_F32, None, 0, 0, 0, 8, 1.0, -1, 0, None, hs.HS_F32, FAKE, 1 << 30)
    hs.hs_embed_grad(None, hs.HS_F32, None, 0, 0, 9, 8, 1.0, -1, 1, FAKE, hs.HS_F32, FAKE, 1 << 30)


@pytest.mark.parametrize("accumulate", [0, 1])
def test_embed_grad_overlaps(accumulate):
    """The sort's launch writes rows of zeros while others still read ids, and the
    workspace all along: neither may lie on what the call reads or writes."""
    need = hs.hs_embed_grad_bytes(100, 50, 64)
    good = [FAKE, hs.HS_BF16, BIG, 0, 100, 50, 64, 1.0, -1, accumulate, 2 * BIG, hs.HS_F32,
            3 * BIG, need]
    for at, bad in [(2, 2 * BIG), (2, 2 * BIG + 50 * 64 * 4 - 4), (2, 2 * BIG - 396),   # ids
                    (12, FAKE), (12, FAKE + 100 * 64 * 2 - 256), (12, BIG), (12, BIG + 256),
                    (12, 2 * BIG), (12, 2 * BIG + 50 * 64 * 4 - 256),                   # ws
                    (10, 3 * BIG + need - 4), (0, 3 * BIG + need - 2), (2, 3 * BIG + need - 4)]:
        args = list(good)
        args[at] = bad
        refused(INVALID, hs.hs_embed_grad, *args)
    # int64 ids reach twice as far
    args = list(good)
    args[2], args[3] = 2 * BIG - 800 + 8, 1
    refused(INVALID, hs.hs_embed_grad, *args)
    # (a table of no rows, or nothing to add: the call writes nothing)
    hs.hs_embed_grad(FAKE, hs.HS_F32, FAKE, 0, 9, 0, 8, 1.0, -1, accumulate, None, hs.HS_F32, FAKE,
                     1 << 30)


def test_score_packed():
    t = table()
    good = [t, 2 * BIG, hs.HS_F32, 4, 3 * BIG, hs.HS_F32, 1000]
    for at, bad, code in [(0, table(dtype=hs.HS_BF16), UNSUP), (1, None, INVALID),
                          (1, 2 * BIG + 8, ALIGN), (2, 2, UNSUP), (3, -1, INVALID),
                          (3, 2 ** 20 + 1, INVALID), (4, None, INVALID), (4, 3 * BIG + 2, ALIGN),
                          (5, 3, UNSUP), (6, 999, INVALID), (6, 2 ** 40 + 1, INVALID),
                          (4, FAKE + 4096, INVALID), (4, 2 * BIG + 1024, INVALID)]:
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_score_packed, *args)
    hs.hs_score_packed(t, None, hs.HS_F32, 0, None, hs.HS_F32, 1000)
    hs.hs_score_packed(table(rows=0, data=None, scale=None), None, hs.HS_F32, 4, None, hs.HS_F32, 0)


def adjust(**kw):
    a = hs.hs_adjust()
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_adjust_scores():
    good = [adjust(), FAKE, 100, BIG, 100, hs.HS_F32, 4, 100]
    for at, bad, code in [(1, None, INVALID), (1, FAKE + 2, ALIGN), (2, 99, INVALID),
                          (3, None, INVALID), (3, BIG + 1, ALIGN), (4, 99, INVALID),
                          (5, hs.HS_FP8_E4M3, UNSUP), (6, -1, INVALID), (6, 2 ** 20 + 1, INVALID),
                          (7, -1, INVALID), (3, FAKE + 800, INVALID)]:    # overlapping rows
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_adjust_scores, *args)
    refused(INVALID, hs.hs_adjust_scores, adjust(), FAKE, 100, FAKE, 104, hs.HS_F32, 4, 100)
    refused(INVALID, hs.hs_adjust_scores, adjust(), FAKE, 2 ** 31, BIG, 2 ** 31, hs.HS_F32, 2 ** 20,
            2 ** 31 - 1)
    for bad, code in [(dict(n_seen=-1), INVALID), (dict(n_bias=2 ** 30 + 1), INVALID),
                      (dict(seen_off=FAKE, n_seen=3), INVALID),
                      (dict(bias_off=FAKE, bias_id=FAKE, n_bias=3), INVALID),
                      (dict(allow=FAKE, allow_stride=3), INVALID),
                      (dict(allow=FAKE, allow_stride=-4), INVALID),
                      (dict(allow=FAKE + 2), ALIGN), (dict(seen_off=FAKE + 4), ALIGN),
                      (dict(repetition=FAKE + 1), ALIGN), (dict(bias_off=FAKE + 4), ALIGN),
                      (dict(prompt_len=FAKE + 2), ALIGN), (dict(presence=FAKE + 2), ALIGN)]:
        refused(code, hs.hs_adjust_scores, adjust(**bad), *good[1:])
    assert hs._lib.hs_adjust_scores(None, FAKE, 100, BIG, 100, 0, 4, 100, None) == INVALID
    hs.hs_adjust_scores(adjust(), None, 100, None, 100, hs.HS_F32, 0, 100)
    hs.hs_adjust_scores(adjust(), None, 0, None, 0, hs.HS_BF16, 5, 0)


LISTS = ["seen_off", "seen", "prompt_len", "repetition", "frequency", "presence", "bias_off",
         "bias_id", "bias", "allow"]


def lists(**kw):
    """All lists and arrays of four rows (100 columns), each BIG apart from the others."""
    base = {n: (10 + i) * BIG for i, n in enumerate(LISTS)}
    base.update(n_seen=30, n_bias=20, allow_stride=4)
    base.update(kw)
    return adjust(**base)


@pytest.mark.parametrize("name,size", [
    ("seen_off", 40), ("seen", 120), ("prompt_len", 16), ("repetition", 16), ("frequency", 16),
    ("presence", 16), ("bias_off", 40), ("bias_id", 80), ("bias", 80), ("allow", 64)])
def test_adjust_scores_overlaps(name, size):
    """Other workgroups still read the lists, arrays and masks while out is written."""
    # out: four rows of 400 bytes, 512 apart
    for at in (BIG, BIG + 392, BIG + 512, BIG + 3 * 512 + 392, BIG - size + 8):
        for scores in (FAKE, BIG):                     # (out of place and in place)
            refused(INVALID, hs.hs_adjust_scores, lists(**{name: at}), scores, 128, BIG, 128,
                    hs.HS_F32, 4, 100)


def accepted(call, *args):
    """Validation passes: what fails, without a GPU, is the device call behind it."""
    try:
        call(*args)
    except hs.HsError as e:
        assert e.status == hs.HS_ERR_DEVICE, hs.hs_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch on made-up addresses")
@pytest.mark.parametrize("name,size", [("seen_off", 40), ("bias", 80), ("allow", 64)])
def test_adjust_scores_between_rows(name, size):
    """Lists before, behind and between the rows of out; a mask of each row behind its
    scores; lists of no entries anywhere."""
    rows = [hs.HS_F32, 4, 100]
    for at in (BIG - size, BIG + 3 * 512 + 400, BIG + 400):
        a = lists(**{name: at})
        accepted(hs.hs_adjust_scores, a, FAKE, 128, BIG, 128, *rows)
    a = lists(allow=BIG + 400, allow_stride=128)
    accepted(hs.hs_adjust_scores, a, BIG, 128, BIG, 128, *rows)
    a = lists(seen=BIG, n_seen=0)
    accepted(hs.hs_adjust_scores, a, BIG, 128, BIG, 128, *rows)
    # (a mask of 4 words a row, one word too far to the front)
    refused(INVALID, hs.hs_adjust_scores, lists(allow=BIG + 396, allow_stride=128), BIG, 128, BIG,
            128, *rows)
    refused(INVALID, hs.hs_adjust_scores, lists(allow=BIG + 400, allow_stride=127), BIG, 128, BIG,
            128, *rows)


def test_topk_rows():
    need = hs.hs_topk_rows_bytes(4, 100_000, 50)
    assert need >= 256
    for bad in ((-1, 10, 5), (2 ** 20 + 1, 10, 5), (4, -1, 5), (4, 2 ** 31, 5), (4, 10, 0),
                (4, 10, 1025)):
        refused(INVALID, hs.hs_topk_rows_bytes, *bad)
    assert hs._lib.hs_topk_rows_bytes(1, 1, 1, None) == INVALID
    good = [FAKE, hs.HS_F32, 100_000, 4, 100_000, 50, BIG, 2 * BIG, 3 * BIG, need]
    for at, bad, code in [(0, None, INVALID), (0, FAKE + 2, ALIGN), (1, 2, UNSUP),
                          (2, 99_999, INVALID), (3, -1, INVALID), (4, -1, INVALID),
                          (5, 0, INVALID), (5, 1025, INVALID), (6, None, INVALID),
                          (6, BIG + 2, ALIGN), (7, None, INVALID), (7, 2 * BIG + 1, ALIGN),
                          (8, None, WS), (8, 3 * BIG + 16, ALIGN), (9, need - 1, WS),
                          # outputs on the scores' last column, or on each other's
                          (6, FAKE + 4 * 400_000 - 4, INVALID), (7, FAKE, INVALID),
                          (7, BIG + 4 * 4 * 50 - 4, INVALID)]:
        args = list(good)
        args[at] = bad
        refused(code, hs.hs_topk_rows, *args)
    hs.hs_topk_rows(None, hs.HS_F32, 10, 0, 10, 5, None, None, FAKE, 1 << 20)


def test_topk_rows_workspace_overlaps():
    """The maxima are written while scores are still read; the outputs while maxima are."""
    need = hs.hs_topk_rows_bytes(4, 100_000, 50)
    good = [FAKE, hs.HS_F32, 100_000, 4, 100_000, 50, BIG, 2 * BIG, 3 * BIG, need]
    for at, bad in [(8, FAKE), (8, FAKE + 1_600_000 - 256), (8, BIG), (8, BIG + 512),
                    (8, 2 * BIG), (0, 3 * BIG + need - 4), (6, 3 * BIG + need - 4),
                    (7, 3 * BIG + need - 4)]:
        args = list(good)
        args[at] = bad
        refused(INVALID, hs.hs_topk_rows, *args)
    hs.hs_topk_rows(FAKE, hs.HS_F32, 10, 0, 10, 5, FAKE, FAKE, FAKE, 1 << 20)   # (no rows)


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch on made-up addresses")
def test_topk_rows_workspace_between_rows():
    """A workspace in what follows the columns of a row of scores."""
    need = hs.hs_topk_rows_bytes(4, 10_000, 50)
    assert need == 256
    args = [BIG, hs.HS_F32, 12_032, 4, 10_000, 50, 2 * BIG, 3 * BIG, BIG + 40_192, need]
    accepted(hs.hs_topk_rows, *args)
    args[8] = BIG + 48_128      # the second row's first columns
    refused(INVALID, hs.hs_topk_rows, *args)


def test_run_packed_refuses_before_it_begins(monkeypatch):
    """A table or masks that do not fit are found before anything is enqueued or made."""
    m = hs.MergedRetrieval(6, 64, 100, 3, hs.HS_F32, hs.HS_F32, device="cpu")

    def begun(*args, **kw):
        raise AssertionError("the window has begun")

    for name in ("hs_dedup", "hs_scatter", "hs_score_packed", "hs_deliver"):
        monkeypatch.setattr(hs, name, begun)
    keys, q = torch.zeros(6, dtype=torch.int64), torch.zeros(6, 64)

    def table(rows=100, dim=64, device="cpu"):
        return hs.RowTable(torch.zeros(rows, dim // 2, dtype=torch.uint8, device=device),
                           torch.zeros(rows, dim // 32, device=device), group=32)

    def words(*shape, dtype=torch.int32, device="cpu"):
        return torch.zeros(shape, dtype=dtype, device=device)

    t = table()
    for bad, err in [((table(rows=99),), ValueError), ((table(dim=96),), ValueError),
                     ((table(device="meta"),), ValueError),
                     ((hs.RowTable(torch.zeros(100, 64)),), TypeError),
                     ((hs.RowTable(torch.zeros(100, 64, dtype=torch.uint8), torch.zeros(100)),),
                      TypeError),
                     ((t, words(3)), ValueError), ((t, words(5, 4)), ValueError),
                     ((t, words(6, 5)), ValueError), ((t, words(1, 6, 4)), ValueError),
                     ((t, words(4, dtype=torch.int64)), TypeError),
                     ((t, words(4, device="meta")), ValueError),
                     ((t, words(4, 6).t()), ValueError)]:
        with pytest.raises(err):
            m.run_packed(keys, q, *bad)
        assert not hasattr(m, "packed_scores")


def test_python_functions_refuse():
    """The one-call functions' own checks (CPU tensors: no device call is reached)."""
    f = torch.zeros(4, 64)
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2)
    t = hs.RowTable(codes, scales, group=32)
    assert (t.rows, t.dim) == (4, 64)
    for call, err in [
            (lambda: hs.RowTable(torch.zeros(4)), ValueError),
            (lambda: hs.RowTable(f.t()), ValueError),
            (lambda: hs.RowTable(f, scales), ValueError),
            (lambda: hs.RowTable(codes), ValueError),                       # fp8 without scales
            (lambda: hs.RowTable(codes, scales[:, :1], group=32), ValueError),
            (lambda: hs.RowTable(codes, scales, group=48), ValueError),
            (lambda: hs.RowTable(f, scales, group=32), TypeError),
            (lambda: hs.RowTable(codes, scales.half(), group=32), TypeError),
            (lambda: hs.RowTable(torch.zeros(4, 64, dtype=torch.float16)), TypeError),
            (lambda: hs.pack_rows(f[:, :40].contiguous()), ValueError),
            (lambda: hs.pack_rows(f.double()), TypeError),
            (lambda: hs.pack_rows(f), TypeError),                           # not on a GPU
            (lambda: hs.embed(t, torch.zeros(3)), TypeError),
            (lambda: hs.embed(t, torch.zeros(3, dtype=torch.int32)), TypeError),
            (lambda: hs.embed_grad(f, torch.zeros(3, dtype=torch.int64), 9), ValueError),
            (lambda: hs.embed_grad(f, torch.zeros(4, dtype=torch.int64), 9, accumulate=True),
             ValueError),
            (lambda: hs.score_packed(hs.RowTable(f), f), TypeError),
            (lambda: hs.score_packed(t, torch.zeros(2, 32)), ValueError),
            (lambda: hs.score_packed(t, f.double()), TypeError),
            (lambda: hs.adjust_scores(f, seen=torch.zeros(3, dtype=torch.int32)), ValueError),
            (lambda: hs.adjust_scores(f, bias=torch.zeros(3)), ValueError),
            (lambda: hs.adjust_scores(f, allow=torch.zeros(3, dtype=torch.int32)), ValueError),
            (lambda: hs.adjust_scores(f, repetition=torch.zeros(3)), ValueError),
            (lambda: hs.adjust_scores(f.t()), ValueError),
            (lambda: hs.adjust_scores(torch.zeros(1, 8).expand(4, 8)), ValueError),
            (lambda: hs.topk_rows(f.t(), 3), ValueError),
            (lambda: hs.topk_rows(f.int(), 3), TypeError),
            (lambda: hs.topk_rows(f, 0), hs.HsError)]:
        with pytest.raises(err):
            call()


@pytest.mark.skipif(not os.path.isdir(HIP_INC) or shutil.which("g++") is None,
                    reason="needs the HIP headers and g++")
def test_validation_under_asan_ubsan(tmp_path):
    """rows_api.cpp with host-only launcher stubs under the host sanitizers."""
    inc = ["-D__HIP_PLATFORM_AMD__", "-I" + HIP_INC, "-I" + os.path.join(ROOT, "include")]
    objs = []
    for src, lang, std in [("paper_2607_22578_amd/csrc/api.cpp", "g++", "c++17"),
                           ("paper_2607_22578_amd/csrc/rows_api.cpp", "g++", "c++17"),
                           ("tests/sanitize/launch_stubs.cpp", "g++", "c++17"),
                           ("tests/sanitize/rows_stubs.cpp", "g++", "c++17"),
                           ("tests/sanitize/rows_driver.c", "gcc", "c11")]:
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([lang, "-std=" + std] + SAN + inc + ["-c", os.path.join(ROOT, src), "-o", obj],
             str(tmp_path))
        objs.append(obj)
    exe = str(tmp_path / "rows")
    _run(["g++", "-fsanitize=address,undefined"] + objs +
         ["-L" + HIP_LIB, "-lamdhip64", "-Wl,-rpath," + HIP_LIB, "-o", exe], str(tmp_path))
    import subprocess
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=_env())
    assert r.returncode == 0, r.stdout + r.stderr
    assert "all checks passed" in r.stdout


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(hs.hs_row_table) == 48
    assert ctypes.sizeof(hs.hs_adjust) == 13 * 8
