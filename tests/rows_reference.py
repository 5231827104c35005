"""Plain 64-bit references of the row-table operators (numpy, CPU) and the error
bounds that their fp32 arithmetic can be held to.

HALF[t] is half a step of type t relative to the value: what one rounding may be off."""
import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126   # (roundings of subnormal results are absolute: far below this)
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def f64(t):
    return t.detach().cpu().double().numpy()


def unpack(codes, scales, group):
    """fp64 rows of packed codes [n x d / 2] and scales [n x d / group] (tensors)."""
    c = codes.cpu().numpy()
    nib = np.empty((c.shape[0], c.shape[1] * 2), dtype=np.uint8)
    nib[:, 0::2], nib[:, 1::2] = c & 15, c >> 4
    return E2M1[nib] * np.repeat(f64(scales), group, axis=1)


def pack(rows, group, scale_dtype):
    """(codes, scales) as hs_pack_rows defines them: fp32 divisions, the nearest E2M1
    value, ties to the even code."""
    x = rows.detach().cpu().float().numpy().reshape(rows.shape[0], -1, group)
    s = torch.from_numpy(np.abs(x).max(axis=2) / np.float32(6)).to(scale_dtype)
    sf = s.float().numpy()[:, :, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(sf > 0, x / sf, np.float32(0)).astype(np.float32)
    mag = np.abs(q).astype(np.float64)
    # distances to the eight magnitudes; among equal ones the even code
    d = np.abs(mag[..., None] - E2M1[:8])
    best = d.min(axis=-1, keepdims=True)
    cand = d == best
    even = cand & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), cand.argmax(-1)).astype(np.uint8)
    code = np.where(q < 0, code | 8, code).astype(np.uint8).reshape(rows.shape[0], -1)
    return torch.from_numpy(code[:, 0::2] | (code[:, 1::2] << 4)), s


def embed(table, ids, scale, pad_id=-1):
    """table: fp64 [rows x dim] values."""
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < table.shape[0]) & (ids != pad_id)
    out = np.zeros(ids.shape + (table.shape[1],))
    out[ok] = table[ids[ok]] * float(np.float32(scale))
    return out


def embed_grad(d_out, ids, rows, scale, pad_id=-1):
    """(gradient, bound on the error of fp32 sums in any order): a sum of n terms and a
    scaling, each addition and the product off by at most 2^-24 of a partial sum, which is
    at most the sum of magnitudes."""
    d, ids = np.asarray(d_out), np.asarray(ids)
    ok = (ids >= 0) & (ids < rows) & (ids != pad_id)
    s = float(np.float32(scale))
    g, mag = np.zeros((rows, d.shape[-1])), np.zeros((rows, d.shape[-1]))
    np.add.at(g, ids[ok], d[ok])
    np.add.at(mag, ids[ok], np.abs(d[ok]))
    n = np.bincount(ids[ok].ravel(), minlength=rows)[:, None]
    return g * s, (n + 1) * 2.0 ** -24 * 1.01 * mag * abs(s)


def score_packed(values, x, group):
    """(scores, bound): the matrix cores add a group's exact products in fp32, at most one
    step (2^-23) off per addition; three parts of an fp32 x make it 3 per column; then a
    product and an addition per group and the join of up to four partial sums."""
    w, x = np.asarray(values), np.asarray(x)
    n = 3 * w.shape[1] + 2 * (w.shape[1] // group) + 8
    return x @ w.T, n * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def adjust(scores, seen=None, seen_off=None, prompt_len=None, repetition=None, frequency=None,
           presence=None, bias_id=None, bias=None, bias_off=None, allow=None):
    """(adjusted scores, sum of the magnitudes that the at most six fp32 operations
    round); lists are numpy arrays, allow a boolean [rows x cols]."""
    x = np.array(scores, dtype=np.float64)
    rows, cols = x.shape
    mag = np.abs(x)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for r in range(rows):
            if seen is not None:
                ids = seen[max(seen_off[r], 0):min(seen_off[r + 1], len(seen))]
                cut = 0 if prompt_len is None else int(prompt_len[r])
                late = ids[max(cut, 0):]
                hit = np.zeros(cols, bool)
                hit[ids[(ids >= 0) & (ids < cols)]] = True
                n = np.bincount(late[(late >= 0) & (late < cols)], minlength=cols)
                rep = 1.0 if repetition is None else float(repetition[r])
                v = np.where(x[r] > 0, x[r] / rep, x[r] * rep)
                x[r] = np.where(hit, v, x[r])
                f = 0.0 if frequency is None else float(frequency[r])
                p = 0.0 if presence is None else float(presence[r])
                mag[r] = np.maximum(mag[r], np.abs(x[r])) + np.abs(f * n) + (n > 0) * abs(p)
                x[r] = np.where(n > 0, x[r] - f * n - p, x[r])
            if bias_id is not None:
                lo, hi = max(bias_off[r], 0), min(bias_off[r + 1], len(bias_id))
                last = {int(c): float(b) for c, b in zip(bias_id[lo:hi], bias[lo:hi])}
                for c, b in last.items():
                    if 0 <= c < cols:
                        x[r, c] += b
                        mag[r, c] += abs(b)
            if allow is not None:
                x[r] = np.where(allow[r], x[r], -np.inf)
    return x, mag


def topk(scores, k):
    """(scores [rows x k] fp32, columns int32) by a stable sort; -inf and NaN never taken."""
    s = np.asarray(scores, dtype=np.float32)
    out = np.full((s.shape[0], k), -np.inf, dtype=np.float32)
    idx = np.full((s.shape[0], k), -1, dtype=np.int32)
    for r in range(s.shape[0]):
        cols = np.nonzero(s[r] > -np.inf)[0]
        order = cols[np.argsort(-s[r][cols], kind="stable")][:k]
        out[r, :len(order)], idx[r, :len(order)] = s[r][order] + np.float32(0), order
    return out, idx


def mask_words(allow):
    """int32 words of a boolean [.. x cols]."""
    a = np.asarray(allow)
    cols = a.shape[-1]
    pad = np.zeros(a.shape[:-1] + ((cols + 31) // 32 * 32,), dtype=bool)
    pad[..., :cols] = a
    b = np.packbits(pad.reshape(a.shape[:-1] + (-1, 32)), axis=-1, bitorder="little")
    return torch.from_numpy(np.ascontiguousarray(b).view("<i4").reshape(a.shape[:-1] + (-1,)))


def check(got, want, bound, dtype, what=""):
    """got (tensor of `dtype`) within bound plus one rounding to dtype of want; the same
    infinities and NaN."""
    g = f64(got)
    want = np.asarray(want)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(g), np.isnan(want), err_msg=what)
    np.testing.assert_array_equal(g[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)],
                                  err_msg=what)
    b = np.broadcast_to(np.asarray(bound, dtype=np.float64), want.shape)
    tol = b + HALF[dtype] * (np.abs(want) + b) + TINY
    off = np.abs(np.where(fine, g, 0.0) - np.where(fine, want, 0.0)) > np.where(fine, tol, 0.0)
    if off.any():
        at = tuple(np.argwhere(off)[0])
        raise AssertionError(f"{what}: {off.sum()} of {off.size} outputs off, first at {at}: got "
                             f"{g[at]!r}, want {want[at]!r} +- {tol[at]!r}")
