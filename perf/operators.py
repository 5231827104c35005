"""Performance cases of the row-table operators: both ends of a language model.

  embed     embedding lookup with scaling (hs.embed): token rows of an fp32, bf16,
            fp8 (row scales) or packed 4-bit (group scales) table;
  grad      its gradient with respect to the table (hs.embed_grad);
  packed    products of a few rows with a packed 4-bit table (hs.score_packed): the
            logits of a quantised head, or the scores of a few queries over a corpus;
  adjust    penalties for repeated tokens, biases and allow masks on the scores
            (hs.adjust_scores);
  topk      the k best columns of every row of scores (hs.topk_rows).

listed() names the cases, draw(rng) draws further ones from the same ranges,
prepare(case, seed) makes a state on the GPU, run(state) is one pass (the library's
kernels where `own` is true, else elementary torch operations), work(case) the bytes
and operations a pass cannot do without, exact(case, seed) the results in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
# the values of the eight non-negative E2M1 codes
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _embed(name, table, out, tokens, vocab, dim, group=0):
    return {"name": name, "op": "embed", "table": table, "out": out, "tokens": tokens,
            "vocab": vocab, "dim": dim, "group": group}


def _grad(name, dtype, out, tokens, vocab, dim):
    return {"name": name, "op": "grad", "dtype": dtype, "out": out, "tokens": tokens,
            "vocab": vocab, "dim": dim}


def _packed(name, dtype, scale, out, rows, table, dim, group):
    return {"name": name, "op": "packed", "dtype": dtype, "scale": scale, "out": out, "rows": rows,
            "table": table, "dim": dim, "group": group}


def _adjust(name, dtype, rows, vocab, seen, biases, masks):
    return {"name": name, "op": "adjust", "dtype": dtype, "rows": rows, "vocab": vocab,
            "seen": seen, "biases": biases, "masks": masks}


def _topk(name, dtype, rows, vocab, k):
    return {"name": name, "op": "topk", "dtype": dtype, "rows": rows, "vocab": vocab, "k": k}


def listed():
    return [
        # One decoding step of 32 sequences: a launch and 32 rows.
        _embed("lookup_step_bf16", "bf16", "bf16", 32, 32_000, 4_096),
        # A prefill's tokens from a 4-bit table that the head shares.
        _embed("lookup_prefill_fp4", "fp4", "bf16", 65_536, 131_072, 4_096, 32),
        # A short fine-tuning step: most table rows get a zero gradient.
        _grad("grad_short_bf16", "bf16", "bf16", 2_048, 32_000, 1_024),
        # fp32 training with sizes that divide by nothing.
        _grad("grad_ragged_f32", "f32", "f32", 10_007, 50_257, 771),
        # A training step of 256 sequences x 1,024 tokens, fp32 gradient of a bf16 model.
        _grad("grad_step_bf16", "bf16", "f32", 262_144, 131_072, 1_024),
        # The head for one token of one sequence: the table is streamed once.
        _packed("head_one_bf16", "bf16", "bf16", "f32", 1, 32_000, 4_096, 32),
        # fp32 states of a few sequences over a vocabulary of odd size.
        _packed("head_ragged_f32", "f32", "f32", "f32", 5, 50_257, 1_024, 128),
        # Few distinct queries over the 1M-chunk index held in four bits.
        _packed("queries_1m_bf16", "bf16", "bf16", "f32", 24, 1_000_000, 768, 64),
        # One sequence's logits.
        _adjust("adjust_one_f32", "f32", 1, 32_000, 300, 8, "rows"),
        # A serving batch: long histories, a grammar mask for each sequence.
        _adjust("adjust_batch_bf16", "bf16", 256, 131_072, 2_000, 50, "rows"),
        # One sequence's candidates.
        _topk("topk_one_f32", "f32", 1, 32_000, 50),
        # The chunks of 24 queries over the 1M-chunk index.
        _topk("topk_1m_f32", "f32", 24, 1_000_000, 100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "grad", "packed", "adjust", "topk"])
    if op == "embed":
        table = rng.choice(["f32", "bf16", "fp8", "fp4"])
        group = rng.choice([32, 64, 128]) if table == "fp4" else 0
        dim = group * rng.randint(1, 4_096 // group) if group else _log(rng, 64, 4_096)
        c = _embed("", table, rng.choice(["f32", "bf16"]), _log(rng, 1, 30_000),
                   _log(rng, 1_000, 131_072), dim, group)
    elif op == "grad":
        dim = _log(rng, 64, 2_048)
        c = _grad("", rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]),
                  _log(rng, 1, 130_000_000 // dim if dim > 500 else 262_144),
                  _log(rng, 1_000, 65_536), dim)
    elif op == "packed":
        group = rng.choice([32, 64, 128])
        dim = group * rng.randint(1, 4_096 // group)
        rows = _log(rng, 1, 48)
        most = min(700_000_000 // dim, 20_000_000 // rows)
        c = _packed("", rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]),
                    rng.choice(["f32", "bf16"]), rows, _log(rng, 1_000, most), dim, group)
    elif op == "adjust":
        rows = _log(rng, 1, 256)
        c = _adjust("", rng.choice(["f32", "bf16"]), rows, _log(rng, 1_000, 65_536),
                    _log(rng, 1, 4_000), _log(rng, 1, 300), rng.choice(["none", "one", "rows"]))
    else:
        rows = _log(rng, 1, 64)
        c = _topk("", rng.choice(["f32", "bf16"]), rows,
                  _log(rng, 1_000, 20_000_000 // rows), _log(rng, 1, 256))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device=DEVICE)


def _words(gen, n, vocab):
    """Token ids of text-like frequencies (rank r about as often as 1 / r), scattered
    over the vocabulary."""
    rank = torch.exp(_uniform(gen, n).double() * math.log(vocab)).long().clamp_(max=vocab) - 1
    place = torch.randperm(vocab, generator=gen, device=DEVICE)
    return place[rank].to(torch.int32)


def _pack(rows, group, scale_type):
    """4-bit codes (two a byte, the even column in the low half) and group scales."""
    n, d = rows.shape
    x = rows.view(n, d // group, group)
    scale = (x.abs().amax(2) / 6).to(scale_type)
    q = x / scale.float()[:, :, None]
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=rows.device)
    code = torch.bucketize(q.abs(), middles).to(torch.uint8)
    code = torch.where(q < 0, code | 8, code).view(n, d // 2, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, scale


def _packed_table(gen, n, d, group, scale_type):
    """Rows of a trained-looking table, made a slice at a time."""
    codes = torch.empty((n, d // 2), dtype=torch.uint8, device=DEVICE)
    scales = torch.empty((n, d // group), dtype=scale_type, device=DEVICE)
    step = max(1, (1 << 27) // d)
    for at in range(0, n, step):
        m = min(step, n - at)
        rows = _normal(gen, m, d) * (0.01 + 0.05 * _uniform(gen, m, 1))
        codes[at:at + m], scales[at:at + m] = _pack(rows, group, scale_type)
    return codes, scales


def _offsets(gen, rows, each):
    """Row starts of ragged lists of up to `each` entries, empty ones among them."""
    n = (_uniform(gen, rows) * (each + 1)).long().clamp_(max=each)
    n[-1] = each
    off = torch.zeros(rows + 1, dtype=torch.int64, device=DEVICE)
    off[1:] = torch.cumsum(n, 0)
    return off


def _library(state):
    """What a program that uses the library keeps beside its tensors: the table's handle, the
    outputs and the workspace."""
    import paper_2607_22578_amd as hs
    c, s = state["case"], state
    if c["op"] in ("embed", "packed"):
        s["handle"] = hs.RowTable(s["data"], s.get("scales"), group=c["group"])
    if c["op"] == "embed":
        s["buffer"] = torch.empty((c["tokens"], c["dim"]), dtype=TYPES[c["out"]], device=DEVICE)
    elif c["op"] == "grad":
        s["buffer"] = torch.empty((c["vocab"], c["dim"]), dtype=TYPES[c["out"]], device=DEVICE)
        s["ws"] = torch.empty(hs.hs_embed_grad_bytes(c["tokens"], c["vocab"], c["dim"]),
                              dtype=torch.uint8, device=DEVICE)
    elif c["op"] == "packed":
        s["buffer"] = torch.empty((c["rows"], c["table"]), dtype=TYPES[c["out"]], device=DEVICE)
    elif c["op"] == "adjust":
        s["buffer"] = torch.empty_like(s["scores"])
    else:
        s["buffer"] = (torch.empty((c["rows"], c["k"]), dtype=torch.float32, device=DEVICE),
                       torch.empty((c["rows"], c["k"]), dtype=torch.int32, device=DEVICE))
        s["ws"] = torch.empty(hs.hs_topk_rows_bytes(c["rows"], c["vocab"], c["k"]),
                              dtype=torch.uint8, device=DEVICE)
    s["hs"] = hs


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = {"case": c}
    if c["op"] == "embed":
        if c["table"] == "fp4":
            s["data"], s["scales"] = _packed_table(gen, c["vocab"], c["dim"], c["group"],
                                                   torch.bfloat16)
        elif c["table"] == "fp8":
            rows = 0.02 * _normal(gen, c["vocab"], c["dim"])
            s["scales"] = rows.abs().amax(1) / 448
            s["data"] = (rows / s["scales"][:, None]).to(torch.float8_e4m3fn)
        else:
            s["data"] = (0.02 * _normal(gen, c["vocab"], c["dim"])).to(TYPES[c["table"]])
        s["ids"] = _words(gen, c["tokens"], c["vocab"])
        if c["tokens"] > 4:   # the padded end of a batch
            s["ids"][-c["tokens"] // 50:] = -1
        s["scale"] = math.sqrt(c["dim"])
    elif c["op"] == "grad":
        s["grad"] = (1e-3 * _normal(gen, c["tokens"], c["dim"])).to(TYPES[c["dtype"]])
        s["ids"] = _words(gen, c["tokens"], c["vocab"])
        if c["tokens"] > 4:
            s["ids"][-c["tokens"] // 50:] = -1
        s["scale"] = math.sqrt(c["dim"])
    elif c["op"] == "packed":
        s["data"], s["scales"] = _packed_table(gen, c["table"], c["dim"], c["group"],
                                               TYPES[c["scale"]])
        s["x"] = _normal(gen, c["rows"], c["dim"]).to(TYPES[c["dtype"]])
    elif c["op"] == "adjust":
        s["scores"] = (4 * _normal(gen, c["rows"], c["vocab"])).to(TYPES[c["dtype"]])
        s["seen_off"] = _offsets(gen, c["rows"], c["seen"])
        s["seen"] = _words(gen, c["rows"] * c["seen"], c["vocab"])
        lens = s["seen_off"][1:] - s["seen_off"][:-1]
        s["prompt_len"] = (lens.double() * _uniform(gen, c["rows"]).double()).to(torch.int32)
        s["repetition"] = 1 + 0.3 * _uniform(gen, c["rows"])
        s["frequency"] = _uniform(gen, c["rows"]) - 0.2
        s["presence"] = _uniform(gen, c["rows"]) - 0.2
        s["bias_off"] = _offsets(gen, c["rows"], c["biases"])
        s["bias_id"] = _words(gen, c["rows"] * c["biases"], c["vocab"])
        s["bias"] = 5 * _normal(gen, c["rows"] * c["biases"])
        s["allow"] = None
        if c["masks"] != "none":
            shape = (c["rows"] if c["masks"] == "rows" else 1, (c["vocab"] + 31) // 32)
            s["allow"] = torch.randint(-2 ** 31, 2 ** 31, shape, generator=gen, device=DEVICE,
                                       dtype=torch.int64).to(torch.int32)
            if c["masks"] == "one":
                s["allow"] = s["allow"][0]
    else:
        s["scores"] = (4 * _normal(gen, c["rows"], c["vocab"])).to(TYPES[c["dtype"]])
        # what an allow mask leaves out
        s["scores"].masked_fill_(_uniform(gen, c["rows"], c["vocab"]) < 0.25, -math.inf)
    if own:
        _library(s)
    return s


# ------------------------------------------------------------------ one pass

def _values(codes, scales, group):
    """The fp32 rows that 4-bit codes and their group scales stand for."""
    value = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    n = codes.shape[0]
    v = torch.stack((value[(codes & 15).int()], value[(codes >> 4).int()]), 2)
    return (v.view(n, -1, group) * scales.float()[:, :, None]).view(n, -1)


def _plain_embed(s):
    c, ids = s["case"], s["ids"]
    inside = (ids >= 0) & (ids < c["vocab"])
    at = ids.clamp(0, c["vocab"] - 1)
    if c["table"] == "fp4":
        rows = _values(s["data"][at], s["scales"][at], c["group"])
    elif c["table"] == "fp8":
        rows = s["data"].view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
        rows = rows * s["scales"][at][:, None]
    else:
        rows = s["data"][at].float()
    rows = torch.where(inside[:, None], rows * s["scale"], 0.0)
    return rows.to(TYPES[c["out"]])


def _plain_grad(s):
    c, ids = s["case"], s["ids"]
    inside = (ids >= 0) & (ids < c["vocab"])
    total = torch.zeros((c["vocab"] + 1, c["dim"]), device=DEVICE)   # (the last row: padding)
    total.index_add_(0, torch.where(inside, ids, c["vocab"]), s["grad"].float())
    return (total[:-1] * s["scale"]).to(TYPES[c["out"]])


def _plain_packed(s):
    c = s["case"]
    rows = _values(s["data"], s["scales"], c["group"])
    return torch.matmul(s["x"].float(), rows.t()).to(TYPES[c["out"]])


def _entries(off, total):
    """Row and place in the row of each of a ragged list's first `total` entries; entries
    past the last row get row = rows."""
    at = torch.arange(total, device=off.device)
    row = torch.searchsorted(off[1:].contiguous(), at, right=True)
    return row, at - off[row.clamp(max=off.numel() - 2)]


def _plain_adjust(s):
    c = s["case"]
    rows, vocab = c["rows"], c["vocab"]
    x = s["scores"].float()
    row, place = _entries(s["seen_off"], s["seen"].numel())
    cell = row * vocab + s["seen"]          # (entries of no row land in an extra one)
    late = place >= s["prompt_len"][row.clamp(max=rows - 1)]
    seen = torch.zeros((rows + 1) * vocab, device=DEVICE)
    seen[cell] = 1.0
    count = torch.zeros((rows + 1) * vocab, device=DEVICE)
    count.index_add_(0, cell, late.float())
    seen, count = (t.view(rows + 1, vocab)[:rows] for t in (seen, count))
    rep = s["repetition"][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    row, _ = _entries(s["bias_off"], s["bias_id"].numel())
    cell = row * vocab + s["bias_id"]
    last = torch.full(((rows + 1) * vocab,), -1, dtype=torch.int64, device=DEVICE)
    last.index_reduce_(0, cell, torch.arange(cell.numel(), device=DEVICE), "amax")
    last = last.view(rows + 1, vocab)[:rows]
    x = torch.where(last >= 0, x + s["bias"][last.clamp(min=0)], x)
    if s["allow"] is not None:
        col = torch.arange(vocab, device=DEVICE)
        bit = s["allow"].view(-1, s["allow"].shape[-1])[:, col >> 5] >> (col & 31).int() & 1
        x = torch.where(bit != 0, x, -math.inf)
    return x.to(TYPES[c["dtype"]])


def _plain_topk(s):
    k = s["case"]["k"]
    v, i = torch.sort(s["scores"].float(), dim=1, descending=True, stable=True)
    v, i = v[:, :k], i[:, :k].to(torch.int32)
    return v.contiguous(), torch.where(v == -math.inf, -1, i)


PLAIN = {"embed": _plain_embed, "grad": _plain_grad, "packed": _plain_packed,
         "adjust": _plain_adjust, "topk": _plain_topk}


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return PLAIN[op](s)
    hs = s["hs"]
    if op == "embed":
        return hs.embed(s["handle"], s["ids"], scale=s["scale"], out=s["buffer"])
    if op == "grad":
        return hs.embed_grad(s["grad"], s["ids"], s["case"]["vocab"], scale=s["scale"],
                             out=s["buffer"], ws=s["ws"])
    if op == "packed":
        return hs.score_packed(s["handle"], s["x"], out=s["buffer"])
    if op == "adjust":
        return hs.adjust_scores(s["scores"], allow=s["allow"], seen=s["seen"],
                                seen_off=s["seen_off"], prompt_len=s["prompt_len"],
                                repetition=s["repetition"], frequency=s["frequency"],
                                presence=s["presence"], bias_id=s["bias_id"], bias=s["bias"],
                                bias_off=s["bias_off"], out=s["buffer"])
    return hs.topk_rows(s["scores"], s["case"]["k"], out=s["buffer"], ws=s["ws"])


# ------------------------------------------------------------------ what a pass needs

def _distinct(n, vocab):
    """Distinct tokens expected among n of _words."""
    r = np.arange(1, vocab + 1, dtype=np.float64)
    p = np.log((r + 1) / r) / math.log(vocab + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    c = case
    if c["op"] == "embed":
        d = c["dim"]
        row = {"f32": 4 * d, "bf16": 2 * d, "fp8": d + 4,
               "fp4": d // 2 + 2 * d // max(c["group"], 1)}[c["table"]]
        return {"bytes": _distinct(c["tokens"], c["vocab"]) * row
                + c["tokens"] * (4 + d * SIZE[c["out"]]), "flops": c["tokens"] * d}
    if c["op"] == "grad":
        return {"bytes": c["tokens"] * (4 + c["dim"] * SIZE[c["dtype"]])
                + c["vocab"] * c["dim"] * SIZE[c["out"]], "flops": c["tokens"] * c["dim"]}
    if c["op"] == "packed":
        n, d, m = c["table"], c["dim"], c["rows"]
        return {"bytes": n * (d // 2 + d // c["group"] * SIZE[c["scale"]])
                + m * (d * SIZE[c["dtype"]] + n * SIZE[c["out"]]), "flops": 2 * m * n * d}
    if c["op"] == "adjust":
        n = c["rows"] * c["vocab"]
        masks = {"none": 0, "one": 1, "rows": c["rows"]}[c["masks"]]
        return {"bytes": 2 * n * SIZE[c["dtype"]] + masks * ((c["vocab"] + 31) // 32) * 4
                + c["rows"] * (4 * c["seen"] + 8 * c["biases"]) // 2, "flops": n}
    n = c["rows"] * c["vocab"]
    return {"bytes": n * SIZE[c["dtype"]] + c["rows"] * c["k"] * 8, "flops": n}


# ------------------------------------------------------------------ 64 bits

def _wide(codes, scales, group):
    """Rows of a packed table in fp64, from the bits: s eem, e = 0 subnormal."""
    nib = torch.empty((codes.shape[0], codes.shape[1] * 2), dtype=torch.uint8,
                      device=codes.device)
    nib[:, 0::2], nib[:, 1::2] = codes & 15, codes >> 4
    e, m = (nib >> 1 & 3).double(), (nib & 1).double()
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2 ** (e - 1))
    mag = torch.where(nib >= 8, -mag, mag)
    return mag * scales.double().repeat_interleave(group, 1)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "embed":
        out = torch.zeros((c["tokens"], c["dim"]), dtype=torch.float64, device=DEVICE)
        for a in range(0, c["tokens"], 8_192):
            ids = s["ids"][a:a + 8_192].long()
            use = ids[ids >= 0]
            if c["table"] == "fp4":
                t = _wide(s["data"][use], s["scales"][use], c["group"])
            elif c["table"] == "fp8":
                t = s["data"].view(torch.uint8)[use].view(torch.float8_e4m3fn).double()
                t = t * s["scales"][use].double()[:, None]
            else:
                t = s["data"][use].double()
            out[a:a + 8_192][ids >= 0] = t * s["scale"]
        return out
    if c["op"] == "grad":
        ids = s["ids"].long()
        order = torch.argsort(ids, stable=True)
        order = order[ids[order] >= 0]
        total = torch.zeros((c["vocab"], c["dim"]), dtype=torch.float64, device=DEVICE)
        for a in range(0, c["dim"], 256):   # running sums along the sorted tokens, by column slices
            run_sum = torch.cumsum(s["grad"][order, a:a + 256].double(), 0)
            n = torch.bincount(ids[order], minlength=c["vocab"])
            end = torch.cumsum(n, 0)
            pad = torch.cat((torch.zeros_like(run_sum[:1]), run_sum))
            total[:, a:a + 256] = (pad[end] - pad[end - n]) * s["scale"]
        return total
    if c["op"] == "packed":
        x = s["x"].double()
        out = torch.empty((c["rows"], c["table"]), dtype=torch.float64, device=DEVICE)
        for a in range(0, c["table"], 32_768):
            t = _wide(s["data"][a:a + 32_768], s["scales"][a:a + 32_768], c["group"])
            out[:, a:a + 32_768] = (t @ x.t().contiguous()).t()
        return out
    if c["op"] == "adjust":
        vocab = c["vocab"]
        off, boff = s["seen_off"].tolist(), s["bias_off"].tolist()
        x = s["scores"].double()
        for r in range(c["rows"]):
            ids = s["seen"][off[r]:off[r + 1]].long()
            n = torch.bincount(ids[int(s["prompt_len"][r]):], minlength=vocab)
            hit = torch.bincount(ids, minlength=vocab) > 0
            rep = s["repetition"][r].double()
            v = torch.where(hit, torch.where(x[r] > 0, x[r] / rep, x[r] * rep), x[r])
            v = v - s["frequency"][r].double() * n - s["presence"][r].double() * (n > 0)
            b = dict(zip(s["bias_id"][boff[r]:boff[r + 1]].tolist(),
                         s["bias"][boff[r]:boff[r + 1]].tolist()))
            if b:
                v[torch.tensor(list(b), device=DEVICE)] += torch.tensor(
                    list(b.values()), dtype=torch.float64, device=DEVICE)
            if s["allow"] is not None:
                word = s["allow"] if s["allow"].dim() == 1 else s["allow"][r]
                bits = (word.long()[:, None] >> torch.arange(32, device=DEVICE) & 1).view(-1)
                v[bits[:vocab] == 0] = -math.inf
            x[r] = v
        return x
    # the k best by counting: an entry's rank is the number of entries before it in the order
    v = torch.empty((c["rows"], c["k"]), dtype=torch.float64, device=DEVICE)
    i = torch.full((c["rows"], c["k"]), -1, dtype=torch.int32, device=DEVICE)
    for r in range(c["rows"]):
        row = s["scores"][r].double()
        n = min(c["k"], int((row > -math.inf).sum()))
        v[r] = -math.inf
        if n:
            line = torch.topk(row, n).values[-1]
            at = torch.nonzero(row >= line)[:, 0]
            rank = torch.argsort(row[at], descending=True, stable=True)[:n]
            v[r, :n], i[r, :n] = row[at[rank]], at[rank].to(torch.int32)
    return v, i
