"""What is done with learned rows after training: normalised, dropped out, trained through, and scored against a table.

A case is one pass through one of the operators on rows in device memory, as a program that answers queries from
embeddings, or trains a head on them, makes it.  With ``own`` the pass goes through the entry points of
``paper_1903_00757_amd``; otherwise the same formulas are computed with elementary torch operations in 32 bits.

Fields of a case
  path      answer   rows -> root-mean-square norm in 8 bits -> scores against a 4-bit table   gv_norm_rows, gv_score_rows
            norm     rows -> root-mean-square norm in 8 bits                                   gv_norm_rows
            train    norm with dropout and residual, forward and backward                      gv_norm_rows, gv_norm_rows_backward
            drop     dropout, forward and backward                                             gv_drop_rows
            score    scores of query rows against a 4-bit table                                gv_score_rows
  rows, cols      rows of a batch (queries, for answer and score) and their length
  type            of the rows: f32, bf16, f16, or i8 (queries of score: 8-bit codes with a scale for each row)
  pad             the rows lie that many values further apart than they are long
  residual        a second row is added to each
  drop            probability that a value of the addend is dropped
  table, group    rows of the 4-bit table, and the columns that share a scale
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}
STREAM = 5  # of the generator: dropout


def _case(name, path, rows, cols, type, pad=0, residual=False, drop=0.0, table=0, group=0):
    return dict(name=name, path=path, rows=rows, cols=cols, type=type, pad=pad, residual=residual, drop=drop,
                table=table, group=group)


def listed():
    return [
        # one node asks a small graph for its neighbours: vertex and context row, added and normalised, against 10^4 rows
        _case("answer, one query", "answer", 1, 128, "f32", residual=True, table=10_000, group=32),
        # a server's batch of queries against four million rows
        _case("answer, 16 queries, d128", "answer", 16, 128, "f32", residual=True, table=4_000_000, group=32),
        # the query rows of a nightly job, long rows in 16 bits
        _case("norm, 65536 rows, d512", "norm", 65_536, 512, "bf16", residual=True),
        # a few rows of an odd length that lie in a wider matrix
        _case("norm, odd rows", "norm", 513, 1001, "f16", pad=7, residual=True),
        # a small step of a head's training: odd batch, no residual
        _case("train, small and odd", "train", 1021, 357, "f32", drop=0.3),
        # a million rows of the headline length in one step, dropout on the addend
        _case("train, million rows, d128", "train", 1 << 20, 128, "bf16", residual=True, drop=0.1),
        # a deep head's wide rows
        _case("train, wide rows", "train", 8192, 4096, "bf16", residual=True),
        # dropout by itself on long rows
        _case("drop, million rows, d512", "drop", 1 << 20, 512, "bf16", drop=0.1),
        # and on a small odd batch
        _case("drop, odd rows", "drop", 997, 353, "f32", pad=3, drop=0.5),
        # one query in full precision against a million rows
        _case("score, one query, d128", "score", 1, 128, "f32", table=1_000_000, group=32),
        # a few queries, odd sizes, a last group that is not full
        _case("score, 7 queries, odd", "score", 7, 500, "bf16", table=20_011, group=64),
        # many queries at a time, long rows
        _case("score, 64 queries, d512", "score", 64, 512, "bf16", table=1_000_000, group=128),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even on the logarithm's scale."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """The length of a row: one of those that the library trains, or any other."""
    return rng.choice([32, 64, 96, 128, 160, 256, 352, 512]) if rng.random() < 0.5 else _spread(rng, lo, hi)


def draw(rng):
    path = rng.choice(["answer", "norm", "train", "train", "drop", "score", "score"])
    pad = rng.choice([0, 0, 0, 1, 8, 33])
    if path in ("norm", "train", "drop"):
        # the gradient of a norm over a handful of values is a difference of nearly equal ones
        cols = _length(rng, 16 if path == "train" else 1, 8192)
        kind = rng.choice(["f32", "bf16", "bf16", "f16"])
        most = {"norm": 1 << 26, "train": 1 << 28, "drop": 1 << 30}[path] // SIZE[kind] // cols
        case = _case("", path, _spread(rng, 1, min(1 << 20, most)), cols, kind, pad,
                     residual=path != "drop" and rng.random() < 0.7,
                     drop=0.0 if path == "norm" else rng.choice([0.1, 0.1, 0.2, 0.5]) if path == "drop" or rng.random() < 0.6 else 0.0)
    else:
        cols = _length(rng, 1, 2048)
        queries = 1 if rng.random() < 0.4 else _spread(rng, 1, 64 if path == "score" else 16)
        table = _spread(rng, 100, min(4_000_000, (1 << 29) // cols, (1 << 26) // queries))
        case = _case("", path, queries, cols, rng.choice(["f32", "bf16", "f16", "i8", "i8"] if path == "score" else ["f32", "bf16", "f16"]),
                     pad, residual=path == "answer" and rng.random() < 0.7, table=table, group=rng.choice([32, 32, 64, 128]))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------- inputs


def _rows(gen, case, spread=0.5):
    """Rows as embeddings are: their lengths differ, and a few columns are larger than the others."""
    n, c = case["rows"], case["cols"]
    wide = torch.randn(n, c + case["pad"], device="cuda", generator=gen)
    wide *= torch.exp(spread * torch.randn(n, 1, device="cuda", generator=gen))
    wide *= torch.exp(0.5 * torch.randn(1, c + case["pad"], device="cuda", generator=gen))
    return wide.to(TYPES[case["type"]])[:, :c]


def _table(gen, n, cols, group):
    """A table of rows in 4 bits: byte b of a row holds columns 2 b (low half) and 2 b + 1 as two's complement, rows are
    filled up to whole 16 bytes; a bfloat16 scale for every `group` columns."""
    groups, wide = -(-cols // group), 32 * (-(-cols // 32))
    w = torch.randn(n, cols, device="cuda", generator=gen)
    w *= 0.3 * torch.exp(0.5 * torch.randn(n, 1, device="cuda", generator=gen))
    w = torch.nn.functional.pad(w, (0, groups * group - cols)).view(n, groups, group)
    s = (w.abs().amax(-1) / 7).to(torch.bfloat16)
    w = w / s.float().clamp_min(1e-30).unsqueeze(-1)
    q = w.round_().clamp_(-8, 7).view(n, -1)[:, :wide].to(torch.int8)
    return ((q[:, 0::2] & 15) | (q[:, 1::2] << 4)).view(torch.uint8).contiguous(), s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case=case, eps=EPS, seed=(seed * 0x9E3779B97F4A7C15 + 1) % (1 << 64), first=1000 * (seed % 1000))
    path, cols = case["path"], case["cols"]
    if path == "score" and case["type"] == "i8":
        state["x"] = torch.randint(-127, 128, (case["rows"], cols + case["pad"]), device="cuda", generator=gen,
                                   dtype=torch.int8)[:, :cols]
        state["x_scale"] = torch.exp(torch.randn(case["rows"], device="cuda", generator=gen) - 4)
    else:
        state["x"] = _rows(gen, case)
    if case["residual"]:
        state["residual"] = _rows(gen, case)
    if path in ("answer", "norm", "train"):
        state["gain"] = 1 + 0.2 * torch.randn(cols, device="cuda", generator=gen)
    if path in ("train", "drop"):
        state["grad"] = _rows(gen, case, spread=1.0)
    if path == "train" and case["residual"]:
        state["grad_sum"] = _rows(gen, case, spread=1.0)
    if path in ("answer", "score"):
        state["codes"], state["scales"] = _table(gen, case["table"], cols, case["group"])
    return state


# ---------------------------------------------------------------------------------------------------- plain forms


def _multiply(a, m):
    """High and low word of the products of 32-bit words with m (the int64 product wraps, its bits are right)."""
    p = a * m
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _kept(case, seed, first):
    """Which values of a batch are kept, and the factor on them: Philox4x32-10 with the seed as its key, one block of eight
    16-bit numbers for 8 columns of a row, counter (row, column / 8, stream)."""
    n, c = case["rows"], case["cols"]
    line = -(-c // 8)
    row = torch.arange(first, first + n, device="cuda").view(n, 1).expand(n, line)
    c0, c1 = row & 0xFFFFFFFF, row >> 32
    c2 = torch.arange(line, device="cuda").view(1, line).expand(n, line)
    c3 = torch.full_like(c2, STREAM)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _multiply(c0, 0xD2511F53)
        h1, l1 = _multiply(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    threshold = int(case["drop"] * 65536 + 0.5)
    return halves.view(n, 8 * line)[:, :c] >= threshold, 65536.0 / (65536 - threshold)


def _dropped(x, kept):
    return x if kept is None else torch.where(kept[0], x * kept[1], 0.0)


def _norm(state, kept=None):
    """(h, 1 / rms, h g) of a batch in 32 bits."""
    h = _dropped(state["x"].float(), kept)
    if "residual" in state:
        h = h + state["residual"].float()
    return h, torch.rsqrt(h.square().mean(-1, keepdim=True) + state["eps"]), h * state["gain"]


def _in_8_bits(rs, v):
    """(codes, scales): the largest |v| of a row becomes 127; the root mean square goes into the scale alone."""
    step = v.abs().amax(-1, keepdim=True) * (1.0 / 127.0)
    return torch.round(v * torch.reciprocal(step)), step * rs


def _weights(state):
    """The table in 32 bits."""
    case, codes = state["case"], state["codes"]
    n, cols = case["table"], case["cols"]
    q = torch.stack([codes & 15, codes >> 4], -1).view(n, -1)[:, :cols].float()
    q = q - 16.0 * (q > 7.5)
    return q * state["scales"].float().repeat_interleave(case["group"], dim=1)[:, :cols]


def run(state):
    case = state["case"]
    path = case["path"]
    if own:
        return _run_own(state, case, path)
    if path == "drop":
        kept = _kept(case, state["seed"], state["first"])
        return [_dropped(state[k].float(), kept).to(state[k].dtype) for k in ("x", "grad")]
    if path == "score":
        x = state["x"].float()
        if "x_scale" in state:
            x = x * state["x_scale"].view(-1, 1)
        return torch.matmul(x, _weights(state).t())
    kind = state["x"].dtype
    kept = _kept(case, state["seed"], state["first"]) if case["drop"] else None
    h, rs, v = _norm(state, kept)
    if path in ("norm", "answer"):
        q, scale = _in_8_bits(rs, v)
        if path == "answer":
            return torch.matmul(q * scale, _weights(state).t())
        return {"values": q * scale, "sum": h.to(kind)} if "residual" in state else {"values": q * scale}
    out = {"y": (v * rs).to(kind)}
    if "residual" in state or kept is not None:
        out["sum"] = h.to(kind)
        h = out["sum"].float()  # the backward pass has the sum as it was kept
    n = h * rs
    grad = state["grad"].float()
    u = grad * state["gain"]
    dh = rs * (u - n * (u * n).mean(-1, keepdim=True))
    if "grad_sum" in state:
        dh = dh + state["grad_sum"].float()
    out["grad_x"] = _dropped(dh, kept).to(kind)
    if "residual" in state:
        out["grad_residual"] = dh.to(kind)
    out["grad_gain"] = (grad * n).sum(0)
    return out


def _run_own(state, case, path):
    import paper_1903_00757_amd as gv

    x, drop = state["x"], dict(drop=case["drop"], seed=state["seed"], first_row=state["first"])
    if path == "drop":
        return [gv.gv_drop_rows(x, **drop), gv.gv_drop_rows(state["grad"], **drop)]
    if path == "score":
        return gv.gv_score_rows(state["codes"], state["scales"], x, group=case["group"], scale=state.get("x_scale"))
    if path == "answer":
        got = gv.gv_norm_rows(x, state["gain"], state.get("residual"), eps=state["eps"], out_type=torch.int8, keep_sum=False)
        return gv.gv_score_rows(state["codes"], state["scales"], got.out, group=case["group"], scale=got.scale)
    if path == "norm":
        got = gv.gv_norm_rows(x, state["gain"], state.get("residual"), eps=state["eps"], out_type=torch.int8)
        values = got.out * got.scale.view(-1, 1)  # the values that the codes stand for
        return {"values": values, "sum": got.sum} if "residual" in state else {"values": values}
    got = gv.gv_norm_rows(x, state["gain"], state.get("residual"), eps=state["eps"], keep_rstd=True, **drop)
    grads = gv.gv_norm_rows_backward(state["grad"], x if got.sum is None else got.sum, state["gain"], got.rstd,
                                     grad_sum=state.get("grad_sum"), **drop)
    out = {"y": got.out, "grad_x": grads.x, "grad_gain": grads.gain}
    if got.sum is not None:
        out["sum"] = got.sum
    if "residual" in state:
        out["grad_residual"] = grads.residual
    return out


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    path, n, c, es = case["path"], case["rows"], case["cols"], SIZE[case["type"]]
    moved = n * c * es  # one batch of rows
    if path == "drop":
        return {"bytes": 4 * moved, "flops": 2 * n * c}
    if path in ("answer", "score"):
        m = case["table"]
        table = m * (-(-c // 2) + 2 * -(-c // case["group"]))
        return {"bytes": table + moved * (2 if case["residual"] else 1) + 4 * n * m, "flops": 2 * n * m * c}
    if path == "norm":
        return {"bytes": moved * (3 if case["residual"] else 1) + 4 * n * c + 4 * c, "flops": 8 * n * c}
    kept = case["residual"] or case["drop"] > 0
    forward = 2 + (1 if case["residual"] else 0) + (1 if kept else 0)  # x, y, residual, sum
    backward = 3 + (1 if case["residual"] else 0)  # gradient of y, sum, gradient of x, gradient of the sum
    if case["residual"] and case["drop"] > 0:
        backward += 1  # the residual's gradient is another than the addend's
    return {"bytes": (forward + backward) * moved + 8 * c, "flops": 20 * n * c}


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _exact_keep(seed, first, n, c, p):
    """Philox4x32-10 with its products made of 16-bit halves."""
    def product(a, m):
        al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
        low, mid, other = al * ml, ah * ml, al * mh
        carry = (low >> 16) + (mid & 0xFFFF) + (other & 0xFFFF)
        return ah * mh + (mid >> 16) + (other >> 16) + (carry >> 16), ((carry & 0xFFFF) << 16) | (low & 0xFFFF)

    blocks = (c + 7) // 8
    at = torch.arange(n * blocks, device="cuda")
    row = at // blocks + first
    word = [row % (1 << 32), row // (1 << 32), at % blocks, torch.full_like(at, STREAM)]
    key = [seed % (1 << 32), seed >> 32]
    for r in range(10):
        a, b = product(word[0], 0xD2511F53), product(word[2], 0xCD9E8D57)
        word = [b[0] ^ word[1] ^ key[0], b[1], a[0] ^ word[3] ^ key[1], a[1]]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    drawn = torch.empty(n, blocks, 8, dtype=torch.int32, device="cuda")
    for w in range(4):
        drawn[:, :, 2 * w] = (word[w] % 65536).view(n, blocks)
        drawn[:, :, 2 * w + 1] = (word[w] // 65536).view(n, blocks)
    return drawn.view(n, 8 * blocks)[:, :c] >= math.floor(p * 65536 + 0.5)


def _exact_table(state, lo, hi):
    """Rows lo .. hi - 1 of the table in 64 bits."""
    case = state["case"]
    codes = state["codes"][lo:hi].to(torch.int64)
    c = case["cols"]
    column = torch.arange(c, device="cuda")
    nibble = (codes[:, column // 2] >> (4 * (column % 2))) & 15
    value = torch.where(nibble < 8, nibble, nibble - 16).double()
    return value * state["scales"][lo:hi].double()[:, column // case["group"]]


def _exact_scores(state, x):
    m, step = state["case"]["table"], max(1, (1 << 26) // state["case"]["cols"])
    return torch.cat([x @ _exact_table(state, lo, min(m, lo + step)).t().contiguous() for lo in range(0, m, step)], dim=1)


def exact(case, seed):
    state = prepare(case, seed)
    path, n, c, p = case["path"], case["rows"], case["cols"], case["drop"]
    if path == "score":
        x = state["x"].double()
        return _exact_scores(state, x * state["x_scale"].double()[:, None] if "x_scale" in state else x)
    step = max(1, (1 << 24) // c)  # rows at a time
    parts, grad_gain = [], torch.zeros(c, dtype=torch.float64, device="cuda")
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        inside = {k: state[k][lo:hi].double() for k in ("x", "residual", "grad", "grad_sum") if k in state}
        factor = None
        if p > 0:
            t = math.floor(p * 65536 + 0.5)
            factor = _exact_keep(state["seed"], state["first"] + lo, hi - lo, c, p).double() * (65536 / (65536 - t))
        if path == "drop":
            parts.append([inside["x"] * factor, inside["grad"] * factor])
            continue
        h = inside["x"] if factor is None else inside["x"] * factor
        h = h + inside["residual"] if "residual" in inside else h
        g = state["gain"].double()
        power = (h * h).sum(1, keepdim=True) / c + EPS
        if path in ("norm", "answer"):
            v = h * g
            largest = v.abs().max(dim=1, keepdim=True).values
            values = torch.round(v / largest * 127) * largest / 127 / power.sqrt()
            parts.append([values, h] if path == "norm" and "residual" in inside else [values])
            continue
        unit = h / power.sqrt()
        dy = inside["grad"]
        inner = (dy * g * unit).sum(1, keepdim=True) / c
        dh = (dy * g - unit * inner) / power.sqrt()
        dh = dh + inside["grad_sum"] if "grad_sum" in inside else dh
        grad_gain += (dy * unit).sum(0)
        row = {"y": unit * g, "grad_x": dh if factor is None else dh * factor}
        if factor is not None or "residual" in inside:
            row["sum"] = h
        if "residual" in inside:
            row["grad_residual"] = dh
        parts.append(row)
    if path == "train":
        out = {k: torch.cat([r[k] for r in parts]) for k in parts[0]}
        out["grad_gain"] = grad_gain
        return out
    whole = [torch.cat(column) for column in zip(*parts)]
    if path == "drop":
        return whole
    if path == "answer":
        return _exact_scores(state, whole[0])
    return {"values": whole[0], "sum": whole[1]} if len(whole) == 2 else {"values": whole[0]}
