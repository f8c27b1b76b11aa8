"""A table of embeddings in training and serving, as measurable cases: the lookup with scaling and dropout, the table's gradient by sorted
tokens, the update of the rows that a batch names, and dropout of token rows.

In front of the model a program turns item ids into rows, E = scale * table[ids], and drops a share of their values; behind
``longer_forward_backward`` (and the norms' backward pass) it sums the rows of dE into the table's gradient, one row for each item that
the batch names, and updates these rows.  What is dropped follows from a key, a site and the value's place alone, so that no mask is kept:

    value c of row r (user * L + place) is kept where h >= round(65536 p), and then counts 65536 / (65536 - round(65536 p)) times;
    h is half-word c mod 8 of the four words that Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3,
    2011) makes of the counter (c div 8 + 65536 site, r, step's low word, step's high word) under the key (seed's low word, its high word).

Tokens behind a user's length, and those whose id is no row of the table, have zero rows and take no part in a gradient.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INTS = {"i32": torch.int32, "i64": torch.int64}
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 10
MOST_TOKEN_VALUES = 512 * 5000 * 128         # rows of tokens of the largest listed lookup
MOST_GRAD_VALUES = 256 * 2000 * 128          # of the largest listed gradient
MOST_TABLE_VALUES = 1_000_003 * 128          # of the largest listed table


def _tokens(op, users, tokens, width, table=1, dtype="f32", **more):
    """Tokens [users, tokens] of `width` values; `table` rows.  ids: their type; fields: a token's ids in the buffer that `ids` is the
    second one of (1: it is the only one); skew: how ids are spread ("popular": the k-th most popular item as often as 1 / k); out:
    type of the rows that are written, or of the rows of dE; p: share of values that is dropped; dense: the gradient of every row of the table."""
    case = dict(op=op, users=users, tokens=tokens, width=width, table=table, dtype=dtype, ids="i64", fields=1, skew="popular", ragged=False,
                p=0.0, out=dtype, dense=False, residual=False)
    case.update(more)
    return case


def listed():
    return [
        # the items of a handful of short histories in full precision: launch and latency
        _tokens("lookup", 4, 64, 32, 1000, name="lookup_few"),
        # one token for each candidate of a serving request's users: rows of the widest model, any of them
        _tokens("lookup", 16, 1000, 256, 1_000_003, "bf16", skew="even", name="lookup_candidates"),
        # every item of a full training batch, a tenth of the values dropped
        _tokens("lookup", 256, 2000, 128, 1_000_003, "bf16", p=0.1, name="lookup_tokens"),
        # histories of very different length from fp32 master rows, ids beside other fields of the log
        _tokens("lookup", 512, 5000, 128, 500_009, "f32", out="bf16", ids="i32", fields=3, ragged=True, name="lookup_ragged"),
        # the step of a small model with a dense gradient of its table
        _tokens("gradient", 64, 96, 64, 1000, dense=True, name="gradient_few"),
        # every item of a full training batch, with the mask of its lookup; the gradient of the rows that it names
        _tokens("gradient", 256, 2000, 128, 1_000_003, p=0.1, name="gradient_tokens"),
        # histories of different length, one item in most places; every row of the table
        _tokens("gradient", 256, 2000, 96, 300_007, "bf16", ids="i32", ragged=True, skew="one", dense=True, name="gradient_dense"),
        # rows of a wide language model, of an odd width, from a small table
        _tokens("gradient", 3, 1501, 4099, 513, "bf16", skew="even", name="gradient_wide"),
        # the rows that a small batch names, fp32 copies
        _tokens("rows", 64, 96, 32, 1000, name="rows_few"),
        # the rows that a full training batch names, and their part of the global norm
        _tokens("rows", 256, 2000, 128, 1_000_003, out="bf16", name="rows_tokens"),
        # the rows of a small batch's global tokens in full precision, odd ones
        _tokens("dropout", 128, 4, 33, p=0.5, name="dropout_few"),
        # every raw token of a full training batch, added to the rows that a residual path carries
        _tokens("dropout", 256, 2000, 128, dtype="bf16", p=0.1, residual=True, ragged=True, name="dropout_residual"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("lookup", "gradient", "rows", "dropout"))
    while True:
        users, tokens, width, table = _log(rng, 1, 512), _log(rng, 1, 5000), _log(rng, 8, 8192), _log(rng, 16, 2_000_000)
        if rng.random() < 0.4:
            width = rng.choice((32, 64, 128, 256, 512, 1024, 4096))
        most = MOST_TOKEN_VALUES // 4 if op in ("lookup", "dropout") else MOST_GRAD_VALUES // 2
        if 4096 <= users * tokens * width <= most and table * width <= MOST_TABLE_VALUES // 2:
            break
    dtype = rng.choice(("f32", "bf16"))
    p = rng.choice((0.0, 0.1, 0.25, 0.5))
    more = dict(ragged=rng.random() < 0.4, ids=rng.choice(("i32", "i64")), fields=rng.choice((1, 1, 3)), skew=rng.choice(("popular", "popular", "even", "one")))
    if op == "dropout":
        return _tokens(op, users, tokens, width, dtype=dtype, ragged=more["ragged"], p=p or 0.3, residual=rng.random() < 0.5)
    if op == "lookup":
        return _tokens(op, users, tokens, width, table, dtype, out=rng.choice(("f32", "bf16")), p=p, **more)
    if op == "gradient":
        return _tokens(op, users, tokens, width, table, dtype, p=p, dense=rng.random() < 0.5, **more)
    return _tokens(op, users, tokens, width, table, out=rng.choice(("f32", "bf16")), **more)


# ---------------------------------------------------------------------------- what a pass cannot do without
def _there(case):
    n = case["users"] * case["tokens"]
    return n / 2 if case["ragged"] else n                # lengths are uniform over [0, tokens]


def _distinct(case):
    """How many rows of the table the tokens are expected to name."""
    n, rows = _there(case), case["table"]
    if case["skew"] == "even":
        return rows * -math.expm1(-n / rows)
    if case["skew"] == "one":
        return 1 + rows * -math.expm1(-0.1 * n / rows)
    # item k with probability log((k + 1) / k) / log(rows + 1), summed over steps of equal ratio
    total, steps, top = 0.0, 400, math.log(rows + 1)
    for i in range(steps):
        lo, hi = math.exp(top * i / steps), math.exp(top * (i + 1) / steps)
        total += (hi - lo) * -math.expm1(-n / (math.sqrt(lo * hi) * top))
    return min(total, n, rows)


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    every, there, d = case["users"] * case["tokens"], _there(case), case["width"]
    e, o = size[case["dtype"]], size[case["out"]]
    if case["op"] == "dropout":
        return {"bytes": (there * e * (2 if case["residual"] else 1) + every * e) * d, "flops": 2 * there * d}
    named = _distinct(case)
    if case["op"] == "lookup":
        return {"bytes": there * size[case["ids"]] + named * d * e + every * d * o, "flops": there * d}
    if case["op"] == "gradient":
        written = (case["table"] if case["dense"] else named) * (d + 1) * 4
        return {"bytes": there * (size[case["ids"]] + 8 + d * e) + 4 * named + written, "flops": there * d + 2 * named * d}
    return {"bytes": named * d * (28 + o) + 8 * named, "flops": 18 * named * d}


# ---------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(r, *shape):
    return torch.randn(*shape, generator=r, device="cuda")


def _ids(case, r):
    """Item ids as a log holds them, places behind a history's end filled with anything; one in fifty names no item."""
    B, L, R = case["users"], case["tokens"], case["table"]
    u = torch.rand(B, L, generator=r, device="cuda", dtype=torch.float64)
    k = torch.exp(u * math.log(R + 1)).floor().sub(1) if case["skew"] == "popular" else (u * R).floor()
    k = k.long().clamp_(0, R - 1)
    k = (k * 2654435761 + 12345) % R                     # popular items anywhere in the table (a few may fall together)
    if case["skew"] == "one":
        k = torch.where(torch.rand(B, L, generator=r, device="cuda") < 0.9, R // 2, k)
    k = torch.where(torch.rand(B, L, generator=r, device="cuda") < 0.02, -1, k)
    buf = torch.full((B, L, case["fields"]), 1 << 30, dtype=INTS[case["ids"]], device="cuda")
    ids = buf[:, :, 1] if case["fields"] > 1 else buf[:, :, 0]
    ids.copy_(k)
    lens = None
    if case["ragged"]:
        lens = torch.randint(0, L + 1, (B,), generator=r, device="cuda", dtype=torch.int32)
        ids.masked_fill_(torch.arange(L, device="cuda") >= lens[:, None], (1 << 31) - 1)
    return ids, lens


def prepare(case, seed):
    r = _generator(seed)
    s = _state(case, r, int(seed))
    if own:
        _library(s)
    return s


def _state(case, r, seed):
    B, L, d, R = case["users"], case["tokens"], case["width"], case["table"]
    s = dict(case=case, lens=None)
    # what the generator's key holds: a seed of 64 bits and the number of the step
    s["key"] = torch.tensor([(seed * 0x9E3779B97F4A7C15 + 1) % (1 << 63), 1000 + seed % 77], dtype=torch.int64, device="cuda")
    if case["op"] == "dropout":
        t = DTYPES[case["dtype"]]
        s["x"] = _randn(r, B, L, d).mul_(_randn(r, B, L, 1).exp_()).to(t)
        s["residual"] = _randn(r, B, L, d).to(t) if case["residual"] else None
        if case["ragged"]:
            s["lens"] = torch.randint(0, L + 1, (B,), generator=r, device="cuda", dtype=torch.int32)
            pad = (torch.arange(L, device="cuda") >= s["lens"][:, None])[..., None]
            for x in (s["x"], s["residual"]):
                if x is not None:
                    x.masked_fill_(pad, float("nan"))                  # padding holds anything
        s["y"] = torch.empty(B, L, d, dtype=t, device="cuda")
        return s
    s["ids"], s["lens"] = _ids(case, r)
    if case["op"] == "lookup":
        s["scale"] = math.sqrt(d)
        s["table"] = _randn(r, R, d).mul_(1 / math.sqrt(d)).to(DTYPES[case["dtype"]])
        s["e"] = torch.empty(B, L, d, dtype=DTYPES[case["out"]], device="cuda")
        return s
    most = min(B * L, R)
    whole = lambda n, fill: torch.full((n,), fill, dtype=torch.int32, device="cuda")
    s["order"] = {"tokens": whole(B * L, -1), "runs": whole(B * L, -1), "rows": whole(most, -1), "counts": whole(2, 0)}
    if case["op"] == "gradient":
        s["scale"] = math.sqrt(d)
        s["de"] = _randn(r, B, L, d).mul_(_randn(r, B, L, 1).exp_()).mul_(1e-3).to(DTYPES[case["dtype"]])
        if case["ragged"]:
            s["de"].masked_fill_((torch.arange(L, device="cuda") >= s["lens"][:, None])[..., None], float("nan"))
        s["grads"] = torch.zeros(R if case["dense"] else most, d, device="cuda")
        s["norms"] = torch.zeros(R if case["dense"] else most, device="cuda")
        return s
    # the rows' update: the gradient pass has left the order, the rows' gradients and their norms
    _plain_order(s)
    n = int(s["order"]["counts"][0])
    s["named"] = s["order"]["rows"][:n].long()
    s["g"], s["norms"] = torch.zeros(most, d, device="cuda"), torch.zeros(most, device="cuda")
    s["g"][:n] = _randn(r, n, d).mul_(_randn(r, n, 1).exp_()).mul_(0.01)
    s["norms"][:n] = s["g"][:n].double().square().sum(1).sqrt().float()
    s["max_norm"] = 1.0
    s["p"], s["m"] = _randn(r, R, d).mul_(0.05), _randn(r, R, d).mul_(0.003)
    s["v"] = _randn(r, R, d).mul_(0.01).square_().add_(1e-10)
    s["w"] = s["p"].to(DTYPES[case["out"]])
    s["norm"] = torch.zeros(2, device="cuda")
    return s


def _library(s):
    """What a program that calls the library has made once, when it made its buffers."""
    import paper_2505_04421_amd as lg
    case = s["case"]
    B, L, d = case["users"], case["tokens"], case["width"]
    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    s["lg"] = lg
    s["mask"] = lg.DropoutMask(case["p"], s["key"], SITE) if case["p"] else None
    if case["op"] in ("gradient", "rows"):
        o = s["order"]
        s["sorted"] = lg.TokenOrder(o["tokens"], o["runs"], o["rows"], o["counts"])
    if case["op"] == "gradient":
        s["ws_sort"] = scratch(lg.longer_sort_ids_workspace_bytes(B, L, case["table"]))
        s["ws"] = scratch(lg.longer_embedding_backward_workspace_bytes(B, L, d))
    if case["op"] == "rows":
        if s["w"] is s["p"]:                             # fp32 copies are a buffer of their own
            s["w"] = s["p"].clone()
        s["params"] = lg.AdamWRows(s["p"], s["m"], s["v"], s["w"], DECAY)
        s["list"] = lg.TensorList([s["norms"]])
        s["ws"] = scratch(lg.longer_grad_norm_workspace_bytes(s["list"]))


SITE = 3


# ---------------------------------------------------------------------------- the plain forms
def _plain_kept(s):
    """[rows, width]: whether a value is kept, and the factor of those that are."""
    case = s["case"]
    n, d = case["users"] * case["tokens"], case["width"]
    t = round(65536 * case["p"])
    low = 0xffffffff
    seed, step = s["key"][0], s["key"][1]
    k0, k1 = seed & low, seed >> 32 & low
    c0 = (torch.arange(-(-d // 8), device="cuda") + 65536 * SITE).expand(n, -1)
    c1 = torch.arange(n, device="cuda")[:, None].expand_as(c0)
    c2, c3 = (step & low).expand_as(c0), (step >> 32 & low).expand_as(c0)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # 64 bits of a product: the sign bit is a bit like the others
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    halves = torch.stack([h for c in (c0, c1, c2, c3) for h in (c & 0xffff, c >> 16)], -1)
    return (halves >= t).reshape(n, -1)[:, :d].reshape(case["users"], case["tokens"], d), 65536 / (65536 - t)


def _plain_valid(s):
    B, L = s["case"]["users"], s["case"]["tokens"]
    if s["lens"] is None:
        return torch.ones(B, L, dtype=torch.bool, device="cuda")
    return torch.arange(L, device="cuda") < s["lens"][:, None]


def _plain_named(s):
    ids = s["ids"].long()
    return _plain_valid(s) & (ids >= 0) & (ids < s["case"]["table"]), ids


def _plain_lookup(s):
    there, ids = _plain_named(s)
    e = s["table"][ids.masked_fill(~there, 0)].float() * s["scale"]
    if s["case"]["p"]:
        kept, f = _plain_kept(s)
        e = torch.where(kept, e * f, 0.0)
    s["e"].copy_(torch.where(there[..., None], e, 0.0))
    return {"e": s["e"]}


def _plain_order(s):
    there, ids = _plain_named(s)
    at = there.reshape(-1).nonzero()[:, 0]
    item, by = torch.sort(ids.reshape(-1)[at], stable=True)
    first = torch.ones_like(item, dtype=torch.bool)
    first[1:] = item[1:] != item[:-1]
    rows, runs, o = item[first], first.cumsum(0) - 1, s["order"]
    o["tokens"][:len(at)] = at[by].int()
    o["runs"][:len(at)] = runs.int()
    o["rows"][:len(rows)] = rows.int()
    o["counts"].copy_(torch.tensor([len(rows), len(at)]))
    return at[by], runs, rows


def _plain_gradient(s):
    at, runs, rows = _plain_order(s)
    d = s["case"]["width"]
    de = s["de"].float() * s["scale"]
    if s["case"]["p"]:
        kept, f = _plain_kept(s)
        de = torch.where(kept, de * f, 0.0)
    g = torch.zeros(len(rows), d, device="cuda").index_add_(0, runs, de.reshape(-1, d)[at])
    norm = g.square().sum(1).sqrt()
    s["norms"].zero_()
    if s["case"]["dense"]:
        s["grads"].zero_()
        s["grads"][rows], s["norms"][rows] = g, norm
    else:
        s["grads"][:len(rows)], s["norms"][:len(rows)] = g, norm
    return {"order": s["order"], "grads": s["grads"], "norms": s["norms"]}


def _plain_rows(s):
    norm = s["norms"].square().sum().sqrt()
    c = torch.clamp(s["max_norm"] / norm, max=1.0)
    i = s["named"]
    g = s["g"][:len(i)] * c
    m = s["m"][i] * BETA1 + g * (1 - BETA1)
    v = s["v"][i] * BETA2 + g * g * (1 - BETA2)
    p = s["p"][i]
    p = p - LR * (m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS) + DECAY * p)
    s["p"][i], s["m"][i], s["v"][i], s["w"][i] = p, m, v, p.to(s["w"].dtype)
    return {"norm": norm.reshape(1), "p": s["p"], "m": s["m"], "v": s["v"], "w": s["w"]}


def _plain_dropout(s):
    kept, f = _plain_kept(s)
    y = torch.where(kept, s["x"].float() * f, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    s["y"].copy_(torch.where(_plain_valid(s)[..., None], y, 0.0))
    return {"y": s["y"]}


# ---------------------------------------------------------------------------- the library's calls
def _own_lookup(s):
    s["lg"].longer_embedding(s["table"], s["ids"], s["lens"], s["scale"], s["mask"], s["e"])
    return {"e": s["e"]}


def _own_gradient(s):
    lg, table = s["lg"], s["case"]["table"]
    lg.longer_sort_ids(s["ids"], s["lens"], table, s["sorted"], s["ws_sort"])
    lg.longer_embedding_backward(s["sorted"], s["de"], s["scale"], s["mask"], s["case"]["dense"], s["grads"], s["norms"], s["ws"])
    return {"order": s["order"], "grads": s["grads"], "norms": s["norms"]}


def _own_rows(s):
    s["lg"].longer_grad_norm(s["list"], s["max_norm"], s["norm"], s["ws"])
    s["lg"].longer_adamw_rows(s["params"], s["sorted"], s["g"], s["norm"], LR, BETA1, BETA2, ADAM_EPS, STEP)
    return {"norm": s["norm"][:1], "p": s["p"], "m": s["m"], "v": s["v"], "w": s["w"]}


def _own_dropout(s):
    s["lg"].longer_dropout(s["x"], s["residual"], s["lens"], s["mask"], s["y"])
    return {"y": s["y"]}


PLAIN = {"lookup": _plain_lookup, "gradient": _plain_gradient, "rows": _plain_rows, "dropout": _plain_dropout}
OWN = {"lookup": _own_lookup, "gradient": _own_gradient, "rows": _own_rows, "dropout": _own_dropout}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def _times(a, b):
    """High and low word of the product of two 32-bit numbers, by halves."""
    a1, a0, b1, b0 = a >> 16, a & 0xffff, b >> 16, b & 0xffff
    low = a0 * b0
    mid = a1 * b0 + (low >> 16)                          # at most 2^32 - 2^16
    mid2 = a0 * b1 + (mid & 0xffff)
    return a1 * b1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xffff) << 16) + (low & 0xffff)


def _exact_factors(s):
    """[rows, width] in 64 bits: 0 where a value is dropped, what it counts where it is kept."""
    case, word = s["case"], 1 << 32
    n, d = case["users"] * case["tokens"], case["width"]
    seed, step = (int(v) for v in s["key"])
    out = torch.empty(n, -(-d // 8) * 8, dtype=torch.float64, device="cuda")
    share = round(65536 * case["p"])
    for a in range(0, n, 1 << 17):                       # (some rows at a time)
        b = min(n, a + (1 << 17))
        row = torch.arange(a, b, device="cuda")[:, None].repeat(1, -(-d // 8))
        block = torch.arange(row.shape[1], device="cuda")[None].repeat(b - a, 1) + (SITE << 16)
        x = [block, row, torch.full_like(row, step % word), torch.full_like(row, step // word)]
        key = [seed % word, seed // word]
        for i in range(10):
            hi0, lo0 = _times(x[0], 0xD2511F53)
            hi1, lo1 = _times(x[2], 0xCD9E8D57)
            x = [hi1 ^ x[1] ^ key[0], lo1, hi0 ^ x[3] ^ key[1], lo0]
            key = [(key[0] + 0x9E3779B9) % word, (key[1] + 0xBB67AE85) % word]
        for i in range(4):
            out[a:b, 2 * i::8] = (x[i] % 65536 >= share).double()
            out[a:b, 2 * i + 1::8] = (x[i] // 65536 >= share).double()
    return out[:, :d].mul_(65536 / (65536 - share))


def exact(case, seed):
    s = _state(dict(case), _generator(seed), int(seed))
    B, L, d, R = case["users"], case["tokens"], case["width"], case["table"]
    place = torch.arange(B * L, device="cuda")
    there = place >= 0 if s["lens"] is None else place % L < s["lens"].long().repeat_interleave(L)
    factors = _exact_factors(s) if case["p"] else None
    if case["op"] == "dropout":
        y = torch.zeros(B * L, d, dtype=torch.float64, device="cuda")
        y[there] = s["x"].reshape(-1, d)[there].double()
        dropped = factors == 0
        y = y.mul_(factors).masked_fill_(dropped, 0.0)
        if s["residual"] is not None:
            y[there] += s["residual"].reshape(-1, d)[there].double()
        return {"y": y.reshape(B, L, d)}
    ids = s["ids"].reshape(-1).long()
    at = (there & (ids >= 0) & (ids < R)).nonzero()[:, 0]
    if case["op"] == "lookup":
        e = torch.zeros(B * L, d, dtype=torch.float64, device="cuda")
        e[at] = s["table"].double()[ids[at]] * math.sqrt(d)
        if factors is not None:
            e.mul_(factors)
        return {"e": e.reshape(B, L, d)}
    if case["op"] == "gradient":
        g = torch.zeros(R, d, dtype=torch.float64, device="cuda")
        for a in range(0, len(at), 1 << 17):
            i = at[a:a + (1 << 17)]
            rows = s["de"].reshape(-1, d)[i].double() * math.sqrt(d)
            g.index_add_(0, ids[i], rows if factors is None else rows * factors[i])
        items = torch.unique(ids[at])                    # ascending
        o = {k: torch.full_like(t, -1) for k, t in s["order"].items()}
        by = at[torch.argsort(ids[at] * (B * L) + at)]   # by item, then by place
        o["tokens"][:len(at)] = by.int()
        o["runs"][:len(at)] = torch.searchsorted(items, ids[by]).int()
        o["rows"][:len(items)] = items.int()
        o["counts"] = torch.tensor([len(items), len(at)], dtype=torch.int32, device="cuda")
        norms = torch.linalg.vector_norm(g, dim=1)
        if not case["dense"]:
            grads, ns = torch.zeros_like(s["grads"], dtype=torch.float64), torch.zeros_like(s["norms"], dtype=torch.float64)
            grads[:len(items)], ns[:len(items)] = g[items], norms[items]
            g, norms = grads, ns
        return {"order": o, "grads": g, "norms": norms}
    norm = float(torch.linalg.vector_norm(s["norms"].double()))
    c = min(1.0, s["max_norm"] / norm) if norm else 1.0
    new = {k: s[k].double() for k in "pmvw"}
    for i, row in ((slice(a, a + 65536), s["named"][a:a + 65536]) for a in range(0, len(s["named"]), 65536)):
        g = c * s["g"][i][:len(row)].double()
        first = BETA1 * new["m"][row] + (1 - BETA1) * g
        second = BETA2 * new["v"][row] + (1 - BETA2) * g ** 2
        old = new["p"][row]
        to = old * (1 - LR * DECAY) - LR / (1 - BETA1 ** STEP) * first / (torch.sqrt(second / (1 - BETA2 ** STEP)) + ADAM_EPS)
        for k, t in (("p", to), ("m", first), ("v", second), ("w", to)):
            new[k][row] = t
    return {"norm": torch.tensor([norm], dtype=torch.float64), **new}
