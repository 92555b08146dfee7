"""What the operators at the two ends of a pipeline are measured on: a segment's rows [batch, rows, hidden] as the first stage makes
them out of tokens, as any stage normalises them and as the last stage turns them into a loss, with the gradients that go back.

A case is one of
  embed_fwd   rows of a table by token, times a scale; a token outside the table gives zeros
  embed_bwd   its gradient, added into the table's fp32 accumulators
  norm_fwd    layer norm of every row, with the rows' statistics
  norm_bwd    its gradient; those of gain and shift are added into fp32 accumulators
  loss_fwd    cross entropy of every row against its target over the whole vocabulary; a row without a target has loss 0
  loss_bwd    its gradient with respect to rows and weight, from the rows' log-sum-exp: a bf16 weight's is written in bf16, an fp32
              weight's added into its accumulators
for `batch` sequences of `rows` tokens each; `view`: the rows are a segment of longer sequences, so that they are strided; `blank`: the
share of tokens or targets that are none.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


def _case(what, dtype, batch, rows, hidden, vocab=0, view=False, blank=0.0):
    return dict(what=what, dtype=dtype, batch=batch, rows=rows, hidden=hidden, vocab=vocab, view=view, blank=blank)


def listed():
    return [
        # the smallest call: a few tokens of the tiny configuration's width, all latency
        dict(_case("embed_fwd", "f32", 1, 16, 256, 1000), name="embed fwd few tokens"),
        # a segment of a 30B model's sequence on the first stage
        dict(_case("embed_fwd", "bf16", 1, 4897, 7168, 50021), name="embed fwd 30b segment"),
        # two ragged sequences in training precision to check against, rows of odd width
        dict(_case("embed_bwd", "f32", 2, 1357, 515, 9973, view=True, blank=0.1), name="embed bwd ragged batch"),
        # a whole 7b sequence: many rows of the frequent tokens, few of the others
        dict(_case("embed_bwd", "bf16", 1, 32768, 4096, 50021), name="embed bwd 7b sequence"),
        # a segment of the tiny configuration: a launch of a few workgroups
        dict(_case("norm_fwd", "f32", 1, 256, 256), name="norm fwd tiny"),
        # a segment of a 7b sequence
        dict(_case("norm_fwd", "bf16", 1, 4096, 4096), name="norm fwd 7b segment"),
        # ragged batch, rows of odd width inside longer sequences
        dict(_case("norm_bwd", "bf16", 2, 1357, 2563, view=True), name="norm bwd ragged batch"),
        # the first segment of the longest sequence
        dict(_case("norm_bwd", "bf16", 1, 8774, 8192), name="norm bwd gqa segment"),
        # a segment of the tiny configuration with a small vocabulary
        dict(_case("loss_fwd", "f32", 1, 256, 256, 5003), name="loss fwd tiny"),
        # a segment of a 7b sequence on the last stage
        dict(_case("loss_fwd", "bf16", 1, 4099, 4096, 50021), name="loss fwd 7b segment"),
        # two padded sequences in the precision to check against
        dict(_case("loss_bwd", "f32", 2, 341, 1280, 20011, view=True, blank=0.3), name="loss bwd ragged batch"),
        # a segment of a 30B model's sequence with a large vocabulary: the largest
        dict(_case("loss_bwd", "bf16", 1, 6144, 7168, 100003, blank=0.1), name="loss bwd 30b segment"),
    ]


_MOST_BYTES = 2.0e9                                  # of a drawn embedding or layer norm
_MOST_FLOPS = 3 * 2.0 * 6144 * 7168 * 100003         # of a drawn loss; fp32 counts six times


def _spread(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))


def draw(rng):
    what = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "loss_fwd", "loss_fwd", "loss_bwd", "loss_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    batch = rng.choice([1, 1, 2, 3])
    rows, hidden = _spread(rng, 1, 16384), _spread(rng, 64, 8192)
    if rng.random() < 0.6:                           # widths are mostly heads times their width
        hidden = max(64, hidden // 64 * 64)
    vocab = 0 if what.startswith("norm") else _spread(rng, 300, 131072)
    view, blank = rng.random() < 0.3, 0.0 if what.startswith("norm") else rng.choice([0.0, 0.0, 0.1, 0.5, 0.95])
    while True:
        c = _case(what, dtype, batch, rows, hidden, vocab, view, blank)
        w = work(c)
        if w["bytes"] <= _MOST_BYTES and w["flops"] * (6 if dtype == "f32" else 1) <= _MOST_FLOPS:
            return c
        rows, vocab = max(1, rows * 3 // 4), vocab and max(300, vocab * 3 // 4)


def _rows(c, gen, dtype, scale=1.0):
    """[batch, rows, hidden]; as a view, the middle of sequences a little more than twice as long."""
    b, n, h = c["batch"], c["rows"], c["hidden"]
    if not c["view"]:
        return torch.empty((b, n, h), device="cuda", dtype=dtype).normal_(0, scale, generator=gen)
    return torch.empty((b, 2 * n + 3, h), device="cuda", dtype=dtype).normal_(0, scale, generator=gen)[:, n // 2:n // 2 + n]


def _tokens(c, gen):
    """Numbers of tokens as text has them: number i about as often as 1 / (i + 1); a share of them none (-1)."""
    b, n = c["batch"], 2 * c["rows"] + 3 if c["view"] else c["rows"]
    u = torch.rand((b, n), device="cuda", generator=gen, dtype=torch.float64)
    t = ((math.log(c["vocab"] + 1) * u).exp() - 1).long().clamp(0, c["vocab"] - 1)
    t = torch.where(torch.rand((b, n), device="cuda", generator=gen) < c["blank"], -1, t)
    return t[:, c["rows"] // 2:c["rows"] // 2 + c["rows"]] if c["view"] else t


def prepare(case, seed):
    c, t = case, _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    h, v = c["hidden"], c["vocab"]
    s = dict(c=c)

    def normal(*shape, dtype=t, mean=0.0, std=1.0):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=gen)

    if c["what"] == "embed_fwd":
        s.update(ids=_tokens(c, gen), table=normal(v, h, std=0.02), scale=math.sqrt(h))
    elif c["what"] == "embed_bwd":
        s.update(ids=_tokens(c, gen), dout=_rows(c, gen, t), scale=math.sqrt(h), acc=normal(v, h, dtype=torch.float32))
    elif c["what"].startswith("norm"):
        s.update(x=_rows(c, gen, t).add_(0.5), gain=normal(h, mean=1.0, std=0.1), shift=normal(h, std=0.1))
        if c["what"] == "norm_bwd":
            x = s["x"].float()
            s["mean"] = x.mean(2)
            s["rstd"] = ((x - s["mean"][..., None]).square().mean(2) + _EPS).rsqrt()
            s.update(dy=_rows(c, gen, t), dgain=normal(h, dtype=torch.float32), dshift=normal(h, dtype=torch.float32))
    else:
        # scores of a few units, as behind a final layer norm
        s.update(x=_rows(c, gen, t), weight=normal(v, h, std=2.0 / math.sqrt(h)), targets=_tokens(c, gen))
        if c["what"] == "loss_bwd":
            s["lse"] = torch.logsumexp(s["x"].float().reshape(-1, h) @ s["weight"].float().t(), 1).view(c["batch"], c["rows"])
            counted = (s["targets"] >= 0).sum().clamp(min=1)
            s["dloss"] = torch.rand((c["batch"], c["rows"]), device="cuda", generator=gen).add_(0.5) / counted
            if t == torch.float32:
                s["acc"] = normal(v, h, dtype=torch.float32, std=1e-4)
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _plain(s):
    c = s["c"]
    what, t, h, v = c["what"], _TYPES[c["dtype"]], c["hidden"], c["vocab"]
    if what == "embed_fwd":
        known = (s["ids"] >= 0) & (s["ids"] < v)
        out = s["table"][s["ids"].clamp(0, v - 1)].float() * s["scale"]
        return {"out": torch.where(known[..., None], out, 0.0).to(t)}
    if what == "embed_bwd":
        known = (s["ids"] >= 0) & (s["ids"] < v)
        d = torch.where(known[..., None], s["dout"].float() * s["scale"], 0.0)
        s["acc"].index_add_(0, s["ids"].clamp(0, v - 1).reshape(-1), d.reshape(-1, h))
        return {"dtable": s["acc"]}
    if what == "norm_fwd":
        x = s["x"].float()
        mean = x.mean(2)
        x = x - mean[..., None]
        rstd = (x.square().mean(2) + _EPS).rsqrt()
        return {"y": (x * rstd[..., None] * s["gain"].float() + s["shift"].float()).to(t), "mean": mean, "rstd": rstd}
    if what == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][..., None]
        xhat = (s["x"].float() - s["mean"][..., None]) * rstd
        g = dy * s["gain"].float()
        dx = (g - g.mean(2, keepdim=True) - xhat * (g * xhat).mean(2, keepdim=True)) * rstd
        s["dgain"] += (dy * xhat).sum((0, 1))
        s["dshift"] += dy.sum((0, 1))
        return {"dx": dx.to(t), "dgain": s["dgain"], "dshift": s["dshift"]}
    x, w, target = s["x"].float().reshape(-1, h), s["weight"].float(), s["targets"].reshape(-1)
    counted = (target >= 0) & (target < v)
    at = target.clamp(0, v - 1)[:, None]
    z = x @ w.t()
    if what == "loss_fwd":
        most = z.max(1).values
        lse = most + (z - most[:, None]).exp().sum(1).log()
        loss = torch.where(counted, lse - z.gather(1, at)[:, 0], 0.0)
        return {"loss": loss.view(s["targets"].shape), "lse": torch.where(counted, lse, 0.0).view(s["targets"].shape)}
    dz = (z - s["lse"].reshape(-1, 1)).exp()
    dz.scatter_add_(1, at, torch.full_like(dz[:, :1], -1.0))
    dz *= torch.where(counted, s["dloss"].reshape(-1), 0.0)[:, None]
    dx, dw = (dz @ w).to(t).view(s["x"].shape), dz.t() @ x
    if t == torch.float32:
        s["acc"] += dw
        dw = s["acc"]
    return {"dx": dx, "dweight": dw.to(t)}


def _own(s):
    import paper_2406_03488_amd as s1f
    c = s["c"]
    what, t = c["what"], _TYPES[c["dtype"]]

    def keep(name, make):        # buffers that a program allocates once
        if name not in s:
            s[name] = make()
        return s[name]

    def like(x):                 # a buffer with the strides of the rows that it goes with
        return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)

    def row_values():
        return torch.empty((c["batch"], c["rows"]), dtype=torch.float32, device="cuda")

    def bytes_of(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None

    if what == "embed_fwd":
        out = keep("out", lambda: torch.empty((c["batch"], c["rows"], c["hidden"]), dtype=t, device="cuda"))
        s1f.embed_fwd(s["ids"], s["table"], s["scale"], out)
        return {"out": out}
    if what == "embed_bwd":
        ws = keep("ws", lambda: bytes_of(s1f.embed_bwd_workspace_bytes(s["ids"], s["dout"], s["acc"])))
        s1f.embed_bwd(s["ids"], s["dout"], s["scale"], s["acc"], ws)
        return {"dtable": s["acc"]}
    if what == "norm_fwd":
        y, mean, rstd = keep("y", lambda: like(s["x"])), keep("mean", row_values), keep("rstd", row_values)
        s1f.layer_norm_fwd(s["x"], s["gain"], s["shift"], _EPS, y, mean, rstd)
        return {"y": y, "mean": mean, "rstd": rstd}
    if what == "norm_bwd":
        dx = keep("dx", lambda: like(s["x"]))
        ws = keep("ws", lambda: bytes_of(s1f.layer_norm_bwd_workspace_bytes(s["dy"], s["x"])))
        s1f.layer_norm_bwd(s["dy"], s["x"], s["gain"], s["mean"], s["rstd"], dx, s["dgain"], s["dshift"], ws)
        return {"dx": dx, "dgain": s["dgain"], "dshift": s["dshift"]}
    if what == "loss_fwd":
        loss, lse = keep("loss", row_values), keep("lse", row_values)
        ws = keep("ws", lambda: bytes_of(s1f.token_loss_fwd_workspace_bytes(s["x"], s["weight"])))
        s1f.token_loss_fwd(s["x"], s["weight"], s["targets"], loss, lse, ws)
        return {"loss": loss, "lse": lse}
    dx, dw = keep("dx", lambda: like(s["x"])), s["acc"] if t == torch.float32 else keep("dw", lambda: like(s["weight"]))
    ws = keep("ws", lambda: bytes_of(s1f.token_loss_bwd_workspace_bytes(s["x"], s["weight"])))
    s1f.token_loss_bwd(s["dloss"], s["x"], s["weight"], s["targets"], s["lse"], dx, dw, ws)
    return {"dx": dx, "dweight": dw}


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    n, h, v = c["batch"] * c["rows"], c["hidden"], c["vocab"]
    used = n * (1 - c["blank"])
    # tokens of a draw from 1 / (i + 1): about this many different ones (a table's rows that a call touches)
    kinds = sum(min(1.0, used / ((i + 1) * math.log(v + 1))) for i in range(min(v, 2000))) if v else 0
    if v > 2000:
        first, last = 2001, v + 1        # the rest as an integral of min(1, used / (x log v))
        knee = min(max(used / math.log(v + 1), first), last)
        kinds += knee - first + used / math.log(v + 1) * math.log(last / knee)
    kinds = min(kinds, used)
    if c["what"] == "embed_fwd":
        return {"bytes": n * 8 + kinds * h * e + n * h * e, "flops": used * h}
    if c["what"] == "embed_bwd":
        return {"bytes": n * 8 + used * h * e + 2 * kinds * h * 4, "flops": 2 * used * h}
    if c["what"] == "norm_fwd":
        return {"bytes": 2 * n * h * e + 8 * n + 2 * h * e, "flops": 8 * n * h}
    if c["what"] == "norm_bwd":
        return {"bytes": 3 * n * h * e + 8 * n + h * e + 16 * h, "flops": 16 * n * h}
    if c["what"] == "loss_fwd":
        return {"bytes": used * h * e + v * h * e + 16 * n, "flops": 2 * used * h * v}
    # scores again, then the products with the weight and with the rows
    return {"bytes": used * h * e + n * h * e + v * h * e + v * h * (2 if e == 2 else 8) + 16 * n, "flops": 6 * used * h * v}


def exact(case, seed):
    c = case
    if work(c)["flops"] > 4e13:
        return None
    s = prepare(c, seed)
    n, h, v = c["batch"] * c["rows"], c["hidden"], c["vocab"]
    shape = (c["batch"], c["rows"])
    if c["what"].startswith("embed"):
        ids = s["ids"].reshape(-1)
        rows = torch.nonzero((ids >= 0) & (ids < v))[:, 0]
        if c["what"] == "embed_fwd":
            out = torch.zeros((n, h), dtype=torch.float64, device="cuda")
            out[rows] = s["table"].double()[ids[rows]] * s["scale"]
            return {"out": out.view(*shape, h)}
        d = s["dout"].double().reshape(n, h)[rows] * s["scale"]
        return {"dtable": s["acc"].double().index_add_(0, ids[rows], d)}
    if c["what"] == "norm_fwd":
        x = s["x"].double()
        variance, mean = torch.var_mean(x, 2, correction=0)
        rstd = 1 / torch.sqrt(variance + _EPS)
        y = (x - mean[..., None]) * rstd[..., None] * s["gain"].double() + s["shift"].double()
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["what"] == "norm_bwd":
        x, dy, rstd = s["x"].double().reshape(n, h), s["dy"].double().reshape(n, h), s["rstd"].double().reshape(n)
        xhat = (x - s["mean"].double().reshape(n, 1)) * rstd[:, None]
        u = dy * s["gain"].double()
        along, mean = (u * xhat).sum(1) / h, u.sum(1) / h
        dx = torch.addcmul(u - mean[:, None], xhat, along[:, None], value=-1) * rstd[:, None]
        return {"dx": dx.view(*shape, h), "dgain": s["dgain"].double() + (dy * xhat).sum(0), "dshift": s["dshift"].double() + dy.sum(0)}
    target = s["targets"].reshape(-1)
    rows = torch.nonzero((target >= 0) & (target < v))[:, 0]       # the others take no part
    x, w, target = s["x"].double().reshape(n, h)[rows], s["weight"].double(), target[rows]
    chunk = max(1, (1 << 28) // v)
    loss, lse = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    dx, dw = torch.zeros((n, h), dtype=torch.float64, device="cuda"), torch.zeros((v, h), dtype=torch.float64, device="cuda")
    for i in range(0, len(rows), chunk):
        r, k = rows[i:i + chunk], target[i:i + chunk]
        z = x[i:i + chunk] @ w.T
        if c["what"] == "loss_fwd":
            lse[r] = torch.logsumexp(z, 1)
            loss[r] = lse[r] - z[torch.arange(len(r), device="cuda"), k]
            continue
        z.sub_(s["lse"].double().reshape(-1)[r][:, None]).exp_()
        z[torch.arange(len(r), device="cuda"), k] -= 1
        z *= s["dloss"].double().reshape(-1)[r][:, None]
        dx[r] = z @ w
        dw.addmm_(z.T, x[i:i + chunk])
    if c["what"] == "loss_fwd":
        return {"loss": loss.view(shape), "lse": lse.view(shape)}
    return {"dx": dx.view(*shape, h), "dweight": dw + s["acc"].double() if "acc" in s else dw}
