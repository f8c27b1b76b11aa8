"""The training step around the model's gradients, as measurable cases: layer norm and its gradients, the global gradient norm with
clipping, and the AdamW update that follows them.

``longer_forward_backward`` takes token rows and gives back the gradient of every input and parameter.  In front of it a training
program normalises the rows of its embeddings, behind it it takes dH back through that norm, bounds the gradients by their
global norm and updates the parameters: fp32 master weights and moments, and the copy in the model's type that the kernels read.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5                                   # of the norm, as in the model's configurations
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 10
MOST_ROWS_ELEMENTS = 512 * 5000 * 128        # the largest listed rows
MOST_LIST_ELEMENTS = 1_000_003 * 128         # the largest listed update


def _rows(op, users, rows, width, dtype, ragged=False, of=0, grad="", **name):
    """Rows [users, rows, width]; `of`: rows per user in the buffer that they are the first ones of (0: no others)."""
    return dict(op=op, users=users, rows=rows, width=width, dtype=dtype, ragged=ragged, of=of, grad=grad, **name)


def _model(op, width, blocks, tokens, table, dtype="f32", **name):
    """The parameters of `blocks` transformer blocks (in the order of longer_block), the head, and a table of embeddings."""
    return dict(op=op, layout="model", width=width, blocks=blocks, tokens=tokens, table=table, dtype=dtype, max_norm=1.0, **name)


def _spread(op, tensors, most, mix, aligned, dtype, max_norm, **name):
    """`tensors` tensors of 1 to `most` values, their sizes spread over the logarithm."""
    return dict(op=op, layout="spread", tensors=tensors, most=most, mix=mix, aligned=aligned, dtype=dtype, max_norm=max_norm, **name)


def listed():
    return [
        # the tokens of a handful of short histories in full precision: launch and latency
        _rows("layer_norm", 4, 64, 32, "f32", name="norm_few"),
        # a final norm on the global rows of a batch's outputs, the first 8 of the 108 rows of each user
        _rows("layer_norm", 256, 8, 128, "bf16", of=108, name="norm_globals"),
        # every raw token of a full training batch
        _rows("layer_norm", 256, 2000, 128, "bf16", name="norm_tokens"),
        # the same for histories of very different length, the padding written as zeros
        _rows("layer_norm", 512, 5000, 128, "bf16", ragged=True, name="norm_ragged"),
        # rows of a wide language model, of an odd width
        _rows("layer_norm", 3, 1501, 4099, "f32", name="norm_wide"),
        # the global tokens of a small model's batch: gradients of few rows
        _rows("layer_norm_backward", 128, 4, 64, "bf16", grad="f32", name="grad_globals"),
        # the gradient of every raw token of a full training batch, as the model's backward pass hands it over
        _rows("layer_norm_backward", 256, 2000, 128, "bf16", grad="f32", name="grad_tokens"),
        # ragged wide rows whose gradients are kept in 16 bits
        _rows("layer_norm_backward", 7, 1023, 8191, "bf16", ragged=True, grad="bf16", name="grad_wide"),
        # the gradients of the headline model alone: 98 tensors, 1.2 million values
        _model("clip", 128, 6, 8, 0, name="clip_model"),
        # with the gradient of a table of embeddings at the widest model's width
        _model("clip", 256, 5, 8, 1_000_003, name="clip_table"),
        # norm and update, the headline model alone
        _model("update", 128, 6, 8, 0, name="update_model"),
        # norm and update with a table of embeddings
        _model("update", 128, 5, 8, 1_000_003, name="update_table"),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(("layer_norm", "layer_norm_backward", "clip", "update"))
    if op in ("layer_norm", "layer_norm_backward"):
        while True:
            users, rows, width = _log(rng, 1, 512), _log(rng, 1, 5000), _log(rng, 8, 8192)
            if rng.random() < 0.4:
                width = rng.choice((32, 64, 128, 256, 512, 1024, 2048, 4096, 8192))
            of = rows + _log(rng, 1, 128) if rng.random() < 0.25 else 0
            if 4096 <= users * max(rows, of) * width <= MOST_ROWS_ELEMENTS // 2:
                break
        dtype = rng.choice(("f32", "bf16"))
        grad = "" if op == "layer_norm" else rng.choice(("f32", dtype))
        return _rows(op, users, rows, width, dtype, rng.random() < 0.4, of, grad)
    if rng.random() < 0.4:
        width = rng.choice((32, 64, 128, 256))
        return _model(op, width, rng.randint(2, 9), rng.choice((1, 2, 4, 8)), _log(rng, 1000, 500_000), rng.choice(("f32", "bf16")))
    tensors = _log(rng, 1, 512)
    most = _log(rng, 64, min(1 << 25, MOST_LIST_ELEMENTS // tensors))
    return _spread(op, tensors, most, rng.randrange(1 << 20), rng.random() < 0.5, rng.choice(("f32", "bf16")), rng.choice((0.1, 1.0, 10.0)))


def _shapes(case):
    """The tensors of a list: (values, whether weight decay applies)."""
    if case["layout"] == "model":
        d = case["width"]
        f = 4 * d
        block = [(d, 0), (d, 0)] + [(d * d, 1), (d, 0)] * 4 + [(d, 0), (d, 0), (d * f, 1), (f, 0), (f * d, 1), (d, 0)]
        table = [(case["table"] * d, 1)] if case["table"] else []
        return block * case["blocks"] + [(case["tokens"] * d, 1), (1, 0)] + table
    r = random.Random(case["mix"])
    return [(int(math.exp(r.uniform(0.0, math.log(case["most"] + 0.5)))), r.randrange(2)) for _ in range(case["tensors"])]


def _places(case):
    """Where each tensor begins in the buffer that holds them all, and that buffer's size; gradient buffers of the model are
    dense up to the head's bias, which is padded to 4 values."""
    align = 4 if case["layout"] == "model" or case["aligned"] else 1
    at, starts = 0, []
    for n, _ in _shapes(case):
        starts.append(at)
        at += -(-n // align) * align
    return starts, at


def _cut(flat, case):
    return [flat[a:a + n] for a, (n, _) in zip(_places(case)[0], _shapes(case))]


def work(case):
    size = {"f32": 4, "bf16": 2, "": 0}
    if "users" in case:
        e, eg, d = size[case["dtype"]], size[case["grad"]], case["width"]
        every = case["users"] * case["rows"] * d
        there = every / 2 if case["ragged"] else every      # lengths are uniform over [0, rows]
        if case["op"] == "layer_norm":
            return {"bytes": there * e + every * e + 2 * d * e, "flops": 8 * there}
        return {"bytes": there * (e + eg) + every * eg + d * e + 8 * d, "flops": 14 * there}
    n = sum(n for n, _ in _shapes(case))
    if case["op"] == "clip":
        return {"bytes": 2 * n * size[case["dtype"]], "flops": 3 * n}
    return {"bytes": n * (24 + size[case["dtype"]] + 2), "flops": 18 * n}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def prepare(case, seed):
    r = _generator(seed)
    if "users" in case:
        return _prepare_rows(case, r)
    return _prepare_list(case, r)


def _randn(r, *shape):
    return torch.randn(*shape, generator=r, device="cuda")


def _prepare_rows(case, r):
    B, L, d, of = case["users"], case["rows"], case["width"], case["of"] or case["rows"]
    t = DTYPES[case["dtype"]]
    # token rows of heavy-tailed norm, off zero
    x = _randn(r, B, of, d).mul_(_randn(r, B, of, 1).exp_()).add_(0.25).to(t)
    gain = (0.9 + 0.2 * torch.rand(d, generator=r, device="cuda")).to(t)
    bias = (0.1 * torch.rand(d, generator=r, device="cuda") - 0.05).to(t)
    s = dict(case=case, x=x[:, :L], gain=gain, bias=bias, lens=None)
    if case["ragged"]:
        s["lens"] = torch.randint(0, L + 1, (B,), generator=r, device="cuda", dtype=torch.int32)
        pad = torch.arange(L, device="cuda") >= s["lens"][:, None]
        s["x"].masked_fill_(pad[..., None], float("nan"))       # padding holds anything
    if case["op"] == "layer_norm":
        s["y"] = torch.empty(B, L, d, dtype=t, device="cuda")
    else:
        s["dy"] = _randn(r, B, L, d).mul_(_randn(r, B, L, 1).exp_()).mul_(1e-3).to(DTYPES[case["grad"]])
        if case["ragged"]:
            s["dy"].masked_fill_(pad[..., None], float("nan"))
        s["dx"] = torch.empty_like(s["dy"])
        s["grads"] = torch.empty(2, d, device="cuda")
    if own:
        import paper_2505_04421_amd as lg
        s["lg"] = lg
        if case["op"] == "layer_norm_backward":
            n = lg.longer_layer_norm_backward_workspace_bytes(B, L, d)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


def _heavy(r, n, scale):
    return _randn(r, n).mul_(_randn(r, n).exp_()).mul_(scale)


def _prepare_list(case, r):
    starts, n = _places(case)
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    for v in _cut(inside, case):
        v.fill_(True)
    g = _heavy(r, n, 0.01).masked_fill_(~inside, float("nan")).to(DTYPES[case["dtype"]])     # between two tensors: anything
    s = dict(case=case, max_norm=case["max_norm"], flat_g=g, g=_cut(g, case), norm=torch.zeros(2, device="cuda"))
    if case["op"] == "clip":
        s["flat_out"] = torch.zeros_like(g)
        s["out"] = _cut(s["flat_out"], case)
    else:
        s["flat_p"] = _randn(r, n).mul_(0.05)
        s["flat_m"] = _heavy(r, n, 0.003)
        s["flat_v"] = _heavy(r, n, 0.01).square_().add_(1e-10)
        s["flat_w"] = s["flat_p"].to(torch.bfloat16)
        for k in "pmvw":
            s[k] = _cut(s["flat_" + k], case)
        s["decay"] = [DECAY * on for _, on in _shapes(case)]
    if own:
        # the lists that a training program makes once, when it makes its buffers
        import paper_2505_04421_amd as lg
        s["lg"] = lg
        s["grads"] = lg.TensorList(s["g"])
        s["ws"] = torch.empty(lg.longer_grad_norm_workspace_bytes(s["grads"]), dtype=torch.uint8, device="cuda")
        if case["op"] == "clip":
            s["clipped"] = lg.TensorList(s["out"])
        else:
            s["params"] = lg.AdamWList(s["p"], s["m"], s["v"], s["g"], s["w"], s["decay"])
    return s


# ---------------------------------------------------------------------------- the plain forms
def _valid(s):
    L = s["x"].shape[1]
    return (torch.arange(L, device="cuda") < s["lens"][:, None])[..., None]


def _standardised(s):
    x = s["x"].float()
    if s["lens"] is not None:
        x = torch.where(_valid(s), x, 0.0)
    c = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * r, r


def _plain_norm(s):
    y = _standardised(s)[0] * s["gain"].float() + s["bias"].float()
    if s["lens"] is not None:
        y = torch.where(_valid(s), y, 0.0)
    return {"y": y.to(s["x"].dtype)}


def _plain_norm_backward(s):
    xh, r = _standardised(s)
    dy = s["dy"].float()
    if s["lens"] is not None:
        dy = torch.where(_valid(s), dy, 0.0)
    q = dy * s["gain"].float()
    dx = r * (q - q.mean(-1, keepdim=True) - xh * (q * xh).mean(-1, keepdim=True))
    return {"dx": dx.to(s["dy"].dtype), "dgain": (dy * xh).sum((0, 1)), "dbias": dy.sum((0, 1))}


def _plain_global_norm(s):
    norm = torch.stack([v.float().square().sum() for v in s["g"]]).sum().sqrt()
    return norm, torch.clamp(s["max_norm"] / norm, max=1.0)


def _plain_clip(s):
    norm, c = _plain_global_norm(s)
    [o.copy_(v.float() * c) for v, o in zip(s["g"], s["out"])]
    return {"norm": norm.reshape(1), "clipped": s["flat_out"]}


def _plain_adamw(p, m, v, g, w, decay, c):
    g = g.float() * c
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    p.sub_(LR * (m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS) + decay * p))
    w.copy_(p)


def _plain_update(s):
    norm, c = _plain_global_norm(s)
    [_plain_adamw(*t, c) for t in zip(s["p"], s["m"], s["v"], s["g"], s["w"], s["decay"])]
    return {"norm": norm.reshape(1), "p": s["flat_p"], "m": s["flat_m"], "v": s["flat_v"], "w": s["flat_w"]}


# ---------------------------------------------------------------------------- the library's calls
def _own_norm(s):
    s["lg"].longer_layer_norm(s["x"], s["gain"], s["bias"], s["lens"], EPS, s["y"])
    return {"y": s["y"]}


def _own_norm_backward(s):
    s["lg"].longer_layer_norm_backward(s["x"], s["gain"], s["dy"], s["lens"], EPS, s["dx"], s["grads"], s["ws"])
    return {"dx": s["dx"], "dgain": s["grads"][0], "dbias": s["grads"][1]}


def _own_clip(s):
    s["lg"].longer_grad_norm(s["grads"], s["max_norm"], s["norm"], s["ws"])
    s["lg"].longer_clip_gradients(s["grads"], s["norm"], s["clipped"])
    return {"norm": s["norm"][:1], "clipped": s["flat_out"]}


def _own_update(s):
    s["lg"].longer_grad_norm(s["grads"], s["max_norm"], s["norm"], s["ws"])
    s["lg"].longer_adamw_step(s["params"], s["norm"], LR, BETA1, BETA2, ADAM_EPS, STEP)
    return {"norm": s["norm"][:1], "p": s["flat_p"], "m": s["flat_m"], "v": s["flat_v"], "w": s["flat_w"]}


PLAIN = {"layer_norm": _plain_norm, "layer_norm_backward": _plain_norm_backward, "clip": _plain_clip, "update": _plain_update}
OWN = {"layer_norm": _own_norm, "layer_norm_backward": _own_norm_backward, "clip": _own_clip, "update": _own_update}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    r = _generator(seed)
    if "users" not in case:
        return _exact_list(case, _prepare_list(dict(case), r))
    s = _prepare_rows(case, r)
    B, L, d = s["x"].shape
    n = torch.full((B,), L, device="cuda") if s["lens"] is None else s["lens"]
    there = (torch.arange(L, device="cuda").expand(B, L) < n[:, None]).reshape(-1).nonzero()[:, 0]
    x = s["x"].reshape(B * L, d)[there].double()
    gain, bias = s["gain"].double().requires_grad_(), s["bias"].double().requires_grad_()
    whole = torch.zeros(B * L, d, dtype=torch.float64, device="cuda")
    if case["op"] == "layer_norm":
        with torch.no_grad():
            whole[there] = torch.nn.functional.layer_norm(x, (d,), gain, bias, EPS)
        return {"y": whole.reshape(B, L, d)}
    x.requires_grad_()
    y = torch.nn.functional.layer_norm(x, (d,), gain, bias, EPS)
    dx, dgain, dbias = torch.autograd.grad(y, (x, gain, bias), s["dy"].reshape(B * L, d)[there].double())
    whole[there] = dx
    return {"dx": whole.reshape(B, L, d), "dgain": dgain, "dbias": dbias}


def _exact_list(case, s):
    g = [v.double() for v in s["g"]]
    norm = math.sqrt(math.fsum(float(torch.dot(v, v)) for v in g))
    c = case["max_norm"] / norm if norm > case["max_norm"] else 1.0
    at = torch.tensor([norm], dtype=torch.float64)
    flat = {k: s["flat_" + k].double() for k in (("out",) if case["op"] == "clip" else ("p", "m", "v", "w"))}
    for i, (a, (n, _)) in enumerate(zip(_places(case)[0], _shapes(case))):
        v = {k: t[a:a + n] for k, t in flat.items()}
        if case["op"] == "clip":
            v["out"].copy_(c * g[i])
            continue
        first = BETA1 * v["m"] + (1 - BETA1) * c * g[i]
        second = BETA2 * v["v"] + (1 - BETA2) * (c * g[i]) ** 2
        root = torch.sqrt(second / (1 - BETA2 ** STEP)) + ADAM_EPS
        new = v["p"] * (1 - LR * s["decay"][i]) - LR / (1 - BETA1 ** STEP) * first / root
        for k, t in (("p", new), ("m", first), ("v", second), ("w", new)):
            v[k].copy_(t)
    if case["op"] == "clip":
        return {"norm": at, "clipped": flat["out"]}
    return {"norm": at, **flat}
