"""What a layer of a pipeline stage computes per segment around its attention: the rotation of queries and keys by their positions on
the way into the K/V cache, the same behind a norm of every head, and the gated feed-forward block, each with its gradient.

A case is one of
  rope_fwd   queries rotated; keys rotated and values as they are into rows of the caches
  rope_bwd   gradients of queries, and rows of the fp32 accumulators of keys and values, back to what the projections made
  norm_fwd   as rope_fwd, every head of queries and keys divided by its root mean square and scaled by a gain first
  norm_bwd   as rope_bwd; gradients of the gains are added into fp32 accumulators
  ffn_fwd    y = (act(x Wg^T) * (x Wu^T)) Wout^T, Wg and Wu the halves of one weight; x Wg^T and x Wu^T are kept where `keep` says so
  ffn_bwd    its gradient from what was kept: bf16 weights' are written in bf16, fp32 weights' added into their accumulators
for `batch` sequences of `rows` tokens.  Heads: `view`: queries, keys and values are parts of one projection's rows, else [batch, heads,
rows, dim]; `rotary` leading elements of a head are rotated, in pairs (2i, 2i + 1) if `pairs`, else (i, i + rotary / 2); `far`: the
position of the first token; `listed`: positions are a tensor (gaps where documents end), else they count on from `far`; `scale`: frequencies
of a context that many times as long as the trained one.  Rows: `view`: a segment of longer sequences.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-6
_BASE = 10000.0


def _heads(what, dtype, batch, rows, heads, kv_heads, dim, rotary=None, pairs=False, far=0, listed=False, scale=1.0, view=False):
    return dict(what=what, dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rotary=dim if rotary is None else rotary,
                pairs=pairs, far=far, listed=listed, scale=scale, view=view)


def _ffn(what, dtype, batch, rows, hidden, inner, act="silu", keep=True, view=False):
    return dict(what=what, dtype=dtype, batch=batch, rows=rows, hidden=hidden, inner=inner, act=act, keep=keep, view=view)


def listed():
    return [
        # a few tokens of the tiny configuration: the smallest call, all latency
        dict(_heads("rope_fwd", "f32", 1, 16, 4, 4, 64), name="rope fwd few tokens"),
        # a late segment of the longest sequence: far positions, frequencies of a longer context, one projection's rows
        dict(_heads("rope_fwd", "bf16", 1, 4097, 64, 8, 128, far=118000, scale=8.0, view=True), name="rope fwd gqa segment"),
        # two ragged sequences to check against, a part of each head in pairs, positions with gaps
        dict(_heads("rope_bwd", "f32", 2, 1357, 32, 32, 80, rotary=32, pairs=True, listed=True), name="rope bwd ragged batch"),
        # a segment of a 7b sequence
        dict(_heads("rope_bwd", "bf16", 1, 4096, 32, 32, 128, far=16384), name="rope bwd 7b segment"),
        # one more token behind a long sequence
        dict(_heads("norm_fwd", "bf16", 1, 1, 64, 8, 128, far=131071, view=True), name="norm fwd one token"),
        # a segment of a 30B model's sequence
        dict(_heads("norm_fwd", "bf16", 1, 4897, 56, 56, 128, far=4897, view=True), name="norm fwd 30b segment"),
        # two ragged sequences, part of each head rotated, in halves that do not start on 16 bytes
        dict(_heads("norm_bwd", "bf16", 2, 1357, 32, 32, 80, rotary=20, listed=True), name="norm bwd ragged batch"),
        # the first segment of the longest sequence
        dict(_heads("norm_bwd", "bf16", 1, 8774, 64, 8, 128, pairs=True, view=True), name="norm bwd gqa segment"),
        # a few tokens behind a 7b sequence, nothing kept: the weights are read once
        dict(_ffn("ffn_fwd", "bf16", 1, 16, 4096, 11008, keep=False), name="ffn fwd few tokens"),
        # a segment of a 7b sequence
        dict(_ffn("ffn_fwd", "bf16", 1, 4099, 4096, 11008), name="ffn fwd 7b segment"),
        # two ragged sequences in the precision to check against, rows of odd width between the projections
        dict(_ffn("ffn_bwd", "f32", 2, 341, 1280, 3413, act="gelu", view=True), name="ffn bwd ragged batch"),
        # a segment of a 30B model's sequence: the largest
        dict(_ffn("ffn_bwd", "bf16", 1, 4897, 7168, 19200), name="ffn bwd 30b segment"),
    ]


_MOST_BYTES = 5.0e8                                  # of drawn heads
_MOST_FLOPS = 12.0 * 4897 * 7168 * 19200             # of a drawn block; fp32 counts six times


def _spread(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))


def draw(rng):
    what = rng.choice(["rope_fwd", "rope_bwd", "norm_fwd", "norm_bwd", "ffn_fwd", "ffn_fwd", "ffn_bwd", "ffn_bwd"])
    dtype, batch, view = rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 1, 2, 3]), rng.random() < 0.4
    rows = _spread(rng, 1, 16384)
    if what.startswith("ffn"):
        hidden = _spread(rng, 64, 8192)
        inner = int(hidden * rng.uniform(1.0, 4.0))
        if rng.random() < 0.7:                       # widths are mostly multiples of a tile's
            hidden, inner = max(64, hidden // 64 * 64), max(64, inner // 64 * 64)
        act, keep = rng.choice(["silu", "silu", "gelu"]), what == "ffn_bwd" or rng.random() < 0.7
        while True:
            c = _ffn(what, dtype, batch, rows, hidden, inner, act, keep, view)
            if work(c)["flops"] * (6 if dtype == "f32" else 1) <= _MOST_FLOPS:
                return c
            rows = rows * 3 // 4
    dim = rng.choice([64, 80, 128, 128, 8 * rng.randint(2, 32)])
    kv_heads, group = rng.choice([1, 2, 4, 8, 8, 32]), rng.choice([1, 1, 2, 4, 7, 8])
    rotary = rng.choice([dim, dim, dim // 2, dim // 4 // 2 * 2, 2 * rng.randint(1, dim // 2)])
    far, scale = rng.choice([0, _spread(rng, 1, 1 << 20)]), rng.choice([1.0, 1.0, 4.0, 32.0])
    pairs, positions = rng.random() < 0.4, rng.random() < 0.4
    while True:
        c = _heads(what, dtype, batch, rows, kv_heads * group, kv_heads, dim, rotary, pairs, far, positions, scale, view)
        if work(c)["bytes"] <= _MOST_BYTES:
            return c
        rows = rows * 3 // 4


def _frequencies(rotary, scale):
    """Turns per token, in radians, of each pair: base^(-2i / rotary); of a context `scale` times as long slow pairs are slowed down that
    many times, fast ones not at all, those between in part."""
    i = torch.arange(rotary // 2, device="cuda", dtype=torch.float64)
    f = _BASE ** (-2 * i / max(rotary, 1))
    if scale == 1.0:
        return f, 1.0
    turns = 4096 * f / (2 * math.pi)                 # of a pair over the trained context
    fast = ((turns - 1) / (32 - 1)).clamp(0, 1)
    return f * fast + f / scale * (1 - fast), 0.1 * math.log(scale) + 1


def _rows(c, gen, dtype, scale):
    """[batch, rows, hidden]; as a view, the middle of sequences a little more than twice as long."""
    b, n, h = c["batch"], c["rows"], c["hidden"]
    if not c["view"]:
        return torch.empty((b, n, h), device="cuda", dtype=dtype).normal_(0, scale, generator=gen)
    return torch.empty((b, 2 * n + 3, h), device="cuda", dtype=dtype).normal_(0, scale, generator=gen)[:, n // 2:n // 2 + n]


def prepare(case, seed):
    c, t = case, _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=t, mean=0.0, std=1.0):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=gen)

    s = dict(c=c)
    if c["what"].startswith("ffn"):
        h, f = c["hidden"], c["inner"]
        s.update(x=_rows(c, gen, t, 1.0), w_in=normal(2 * f, h, std=1 / math.sqrt(h)), w_out=normal(h, f, std=1 / math.sqrt(f)))
        if c["what"] == "ffn_bwd":
            s["gate_up"] = (s["x"].float().reshape(-1, h) @ s["w_in"].float().t()).to(t).view(c["batch"], c["rows"], 2 * f)
            s["dy"] = _rows(c, gen, t, 1e-2)
            if t == torch.float32:
                s.update(acc_in=normal(2 * f, h, dtype=torch.float32, std=1e-2), acc_out=normal(h, f, dtype=torch.float32, std=1e-2))
        return s

    b, n, hq, hk, d = c["batch"], c["rows"], c["heads"], c["kv_heads"], c["dim"]
    at = n // 2 + 3                                  # the segment's first row of the caches, with rows of others around it
    s["freqs"], s["magnitude"] = _frequencies(c["rotary"], c["scale"])
    s["at"], s["positions"] = at, c["far"]
    if c["listed"]:
        steps = torch.randint(1, 3, (b, n), device="cuda", generator=gen)
        s["positions"] = c["far"] + steps.cumsum(1) - steps[:, :1]
    if c["what"].startswith("norm"):
        s.update(q_gain=normal(d, mean=1.0, std=0.1), k_gain=normal(d, mean=1.0, std=0.1))
    if c["what"] in ("rope_fwd", "norm_fwd", "norm_bwd"):
        if c["view"]:
            projected = normal(b, n, hq + 2 * hk, d).transpose(1, 2)
            s.update(q=projected[:, :hq], k=projected[:, hq:hq + hk], v=projected[:, hq + hk:])
        else:
            s.update(q=normal(b, hq, n, d), k=normal(b, hk, n, d), v=normal(b, hk, n, d))
    if c["what"].endswith("fwd"):
        s.update(q_rot=torch.zeros((b, hq, n, d), device="cuda", dtype=t), k_cache=normal(b, hk, at + n + 5, d), v_cache=normal(b, hk, at + n + 5, d))
        return s
    s.update(dq_rot=normal(b, hq, n, d), dk_acc=normal(b, hk, at + n + 5, d, dtype=torch.float32), dv_acc=normal(b, hk, at + n + 5, d, dtype=torch.float32))
    # gradients lie as what they are the gradients of
    if c["view"]:
        projected = torch.zeros((b, n, hq + 2 * hk, d), device="cuda", dtype=t).transpose(1, 2)
        s.update(dq=projected[:, :hq], dk=projected[:, hq:hq + hk], dv=projected[:, hq + hk:])
    else:
        s.update(dq=torch.zeros((b, hq, n, d), device="cuda", dtype=t), dk=torch.zeros((b, hk, n, d), device="cuda", dtype=t),
                 dv=torch.zeros((b, hk, n, d), device="cuda", dtype=t))
    if c["what"] == "norm_bwd":
        s.update(dq_gain=normal(d, dtype=torch.float32), dk_gain=normal(d, dtype=torch.float32))
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _angles(s, dtype):
    c = s["c"]
    p = s["positions"] if c["listed"] else torch.arange(c["far"], c["far"] + c["rows"], device="cuda").expand(c["batch"], c["rows"])
    a = p.double()[:, None, :, None] * s["freqs"]
    return (a.cos() * s["magnitude"]).to(dtype), (a.sin() * s["magnitude"]).to(dtype)


def _turned(x, c, cos, sin):
    """Heads with their pairs turned by the angles; by the opposite angles with -sin."""
    r = c["rotary"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["pairs"] else (x[..., :r // 2], x[..., r // 2:r])
    out = x.clone()
    if c["pairs"]:
        out[..., 0:r:2], out[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    else:
        out[..., :r // 2], out[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    return out


def _gelu_slope(g):
    t = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)


def _plain(s):
    c = s["c"]
    what, t = c["what"], _TYPES[c["dtype"]]
    if what.startswith("ffn"):
        h, f = c["hidden"], c["inner"]
        x, w_in, w_out = s["x"].float().reshape(-1, h), s["w_in"].float(), s["w_out"].float()
        shape = (c["batch"], c["rows"])
        z = x @ w_in.t() if what == "ffn_fwd" else s["gate_up"].float().view(-1, 2 * f)
        g, u = z[:, :f], z[:, f:]
        if c["act"] == "silu":
            sig = 1 / (1 + (-g).exp())
            a, slope = g * sig, sig * (1 + g * (1 - sig))
        else:
            a, slope = 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))), _gelu_slope(g)
        if what == "ffn_fwd":
            out = {"y": ((a * u) @ w_out.t()).to(t).view(*shape, h)}
            if c["keep"]:
                out["gate_up"] = z.to(t).view(*shape, 2 * f)
            return out
        dy = s["dy"].float().reshape(-1, h)
        dh = dy @ w_out
        dz = torch.cat([dh * u * slope, dh * a], 1)
        dx, dw_in, dw_out = (dz @ w_in).to(t).view(*shape, h), dz.t() @ x, dy.t() @ (a * u)
        if t == torch.float32:
            s["acc_in"] += dw_in
            s["acc_out"] += dw_out
            return {"dx": dx, "dw_in": s["acc_in"], "dw_out": s["acc_out"]}
        return {"dx": dx, "dw_in": dw_in.to(t), "dw_out": dw_out.to(t)}

    cos, sin = _angles(s, torch.float32)
    rows = slice(s["at"], s["at"] + c["rows"])
    if what.endswith("fwd"):
        q, k = s["q"].float(), s["k"].float()
        if what == "norm_fwd":
            q = q * (q.square().mean(3, keepdim=True) + _EPS).rsqrt() * s["q_gain"].float()
            k = k * (k.square().mean(3, keepdim=True) + _EPS).rsqrt() * s["k_gain"].float()
        s["q_rot"].copy_(_turned(q, c, cos, sin))
        s["k_cache"][:, :, rows] = _turned(k, c, cos, sin).to(t)
        s["v_cache"][:, :, rows] = s["v"]
        return {"q_rot": s["q_rot"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    out = {}
    for name, d in (("q", s["dq_rot"].float()), ("k", s["dk_acc"][:, :, rows])):
        d = _turned(d, c, cos, -sin)
        if what == "norm_bwd":
            x = s[name].float()
            r = (x.square().mean(3, keepdim=True) + _EPS).rsqrt()
            xhat, g = x * r, d * s[name + "_gain"].float()
            s[f"d{name}_gain"] += (d * xhat).sum((0, 1, 2))
            out[f"d{name}_gain"] = s[f"d{name}_gain"]
            d = r * (g - xhat * (g * xhat).mean(3, keepdim=True))
        out["d" + name] = s["d" + name].copy_(d)
    out["dv"] = s["dv"].copy_(s["dv_acc"][:, :, rows])
    return out


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

    def bytes_of(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None

    if what == "rope_fwd":
        s1f.rope_fwd(s["q"], s["k"], s["v"], s["freqs"], s["magnitude"], c["pairs"], s["positions"], s["at"], s["q_rot"], s["k_cache"], s["v_cache"])
        return {"q_rot": s["q_rot"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if what == "norm_fwd":
        s1f.qk_norm_rope_fwd(s["q"], s["k"], s["v"], s["q_gain"], s["k_gain"], _EPS, s["freqs"], s["magnitude"], c["pairs"], s["positions"], s["at"],
                             s["q_rot"], s["k_cache"], s["v_cache"])
        return {"q_rot": s["q_rot"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if what == "rope_bwd":
        s1f.rope_bwd(s["dq_rot"], s["dk_acc"], s["dv_acc"], s["freqs"], s["magnitude"], c["pairs"], s["positions"], s["at"], s["dq"], s["dk"], s["dv"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if what == "norm_bwd":
        ws = keep("ws", lambda: bytes_of(s1f.qk_norm_rope_bwd_workspace_bytes(s["dq_rot"], s["dk_acc"])))
        s1f.qk_norm_rope_bwd(s["dq_rot"], s["dk_acc"], s["dv_acc"], s["q"], s["k"], s["q_gain"], s["k_gain"], _EPS, s["freqs"], s["magnitude"],
                             c["pairs"], s["positions"], s["at"], s["dq"], s["dk"], s["dv"], s["dq_gain"], s["dk_gain"], ws)
        return {"dq_gain": s["dq_gain"], "dq": s["dq"], "dk_gain": s["dk_gain"], "dk": s["dk"], "dv": s["dv"]}
    act = s1f.SILU if c["act"] == "silu" else s1f.GELU_TANH
    if what == "ffn_fwd":
        y = keep("y", lambda: like(s["x"]))
        kept = keep("gate_up", lambda: torch.empty((c["batch"], c["rows"], 2 * c["inner"]), dtype=t, device="cuda")) if c["keep"] else None
        ws = keep("ws", lambda: bytes_of(s1f.gated_ffn_fwd_workspace_bytes(s["x"], s["w_in"], s["w_out"])))
        s1f.gated_ffn_fwd(s["x"], s["w_in"], s["w_out"], act, y, kept, ws)
        return {"y": y, "gate_up": kept} if c["keep"] else {"y": y}
    dx = keep("dx", lambda: like(s["x"]))
    if t == torch.float32:
        dw_in, dw_out = s["acc_in"], s["acc_out"]
    else:
        dw_in, dw_out = keep("dw_in", lambda: like(s["w_in"])), keep("dw_out", lambda: like(s["w_out"]))
    ws = keep("ws", lambda: bytes_of(s1f.gated_ffn_bwd_workspace_bytes(s["dy"], s["x"], s["w_in"], s["w_out"])))
    s1f.gated_ffn_bwd(s["dy"], s["x"], s["w_in"], s["w_out"], act, s["gate_up"], dx, dw_in, dw_out, ws)
    return {"dx": dx, "dw_in": dw_in, "dw_out": dw_out}


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    n = c["batch"] * c["rows"]
    if c["what"].startswith("ffn"):
        h, f = c["hidden"], c["inner"]
        if c["what"] == "ffn_fwd":
            return {"bytes": e * (2 * n * h + 3 * h * f + (2 * n * f if c["keep"] else 0)), "flops": 6 * n * h * f}
        # dy, x and what was kept, dx; the weights, their gradients (accumulators are read, too)
        return {"bytes": e * (3 * n * h + 2 * n * f + 3 * h * f) + (2 if e == 2 else 8) * 3 * h * f, "flops": 12 * n * h * f}
    q, kv, d = n * c["heads"], n * c["kv_heads"], c["dim"]
    turns, positions = 3 * (q + kv) * c["rotary"], 8 * n if c["listed"] else 0
    if c["what"].endswith("fwd"):
        norm = 4 * (q + kv) * d if c["what"] == "norm_fwd" else 0
        return {"bytes": 2 * e * (q + 2 * kv) * d + positions, "flops": turns + norm}
    moved = d * (2 * e * q + 2 * (4 + e) * kv) + positions
    if c["what"] == "rope_bwd":
        return {"bytes": moved, "flops": turns}
    return {"bytes": moved + e * (q + kv) * d + 16 * d, "flops": turns + 12 * (q + kv) * d}


def exact(case, seed):
    c = case
    if work(c)["flops"] > 4e13:
        return None
    s = prepare(c, seed)
    if c["what"].startswith("ffn"):
        h, f = c["hidden"], c["inner"]
        x, w_in, w_out = s["x"].double().reshape(-1, h), s["w_in"].double(), s["w_out"].double()
        shape = (c["batch"], c["rows"])
        z = torch.mm(x, w_in.T) if c["what"] == "ffn_fwd" else s["gate_up"].double().reshape(-1, 2 * f)
        gate, up = z.split(f, 1)
        k = math.sqrt(2 / math.pi)
        if c["act"] == "silu":
            half = torch.tanh(gate / 2)
            on = (1 + half) / 2
            act = gate * on
        else:
            half = torch.tanh(k * gate * (1 + 0.044715 * gate.square()))
            act = gate * (1 + half) / 2
        if c["what"] == "ffn_fwd":
            out = {"y": torch.mm(act * up, w_out.T).view(*shape, h)}
            if c["keep"]:
                out["gate_up"] = z.view(*shape, 2 * f)
            return out
        if c["act"] == "silu":
            slope = on + act * (1 - on)
        else:
            slope = (1 + half) / 2 + gate / 2 * (1 - half.square()) * k * (1 + 0.134145 * gate.square())
        dy = s["dy"].double().reshape(-1, h)
        back = torch.mm(dy, w_out)
        dgate, dup = back * up * slope, back * act
        dx = torch.mm(dgate, w_in[:f]).addmm_(dup, w_in[f:])
        dw_in, dw_out = torch.cat((torch.mm(dgate.T, x), torch.mm(dup.T, x))), torch.mm(dy.T, act * up)
        if c["dtype"] == "f32":
            dw_in, dw_out = s["acc_in"].double() + dw_in, s["acc_out"].double() + dw_out
        return {"dx": dx.view(*shape, h), "dw_in": dw_in, "dw_out": dw_out}

    # pairs as complex numbers, turned by a factor of length `magnitude`
    b, n, r, at = c["batch"], c["rows"], c["rotary"], s["at"]
    p = s["positions"] if c["listed"] else (torch.arange(n, device="cuda") + c["far"]).repeat(b, 1)
    angle = p.to(torch.float64).view(b, 1, n, 1) * s["freqs"].view(1, 1, 1, -1)
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)

    def rotate(x, by):
        head, rest = x[..., :r], x[..., r:]
        two = head.unflatten(3, (r // 2, 2)) if c["pairs"] else head.unflatten(3, (2, r // 2)).transpose(3, 4)
        z = torch.view_as_real(torch.complex(two[..., 0].contiguous(), two[..., 1].contiguous()) * by)
        if not c["pairs"]:
            z = z.transpose(3, 4)
        return torch.cat((z.flatten(3), rest), 3)

    if c["what"].endswith("fwd"):
        out = {"q_rot": None, "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
        for name in ("q", "k"):
            x = s[name].double()
            if c["what"] == "norm_fwd":
                x = x / torch.sqrt(torch.linalg.vecdot(x, x)[..., None] / c["dim"] + _EPS) * s[name + "_gain"].double()
            x = rotate(x, turn)
            if name == "q":
                out["q_rot"] = x
            else:
                out["k_cache"][:, :, at:at + n] = x
        out["v_cache"][:, :, at:at + n] = s["v"].double()
        return out
    out = {}
    for name, d in (("q", s["dq_rot"].double()), ("k", s["dk_acc"][:, :, at:at + n].double())):
        d = rotate(d, turn.conj())
        if c["what"] == "norm_bwd":
            x = s[name].double()
            root = torch.sqrt(torch.linalg.vecdot(x, x)[..., None] / c["dim"] + _EPS)
            out[f"d{name}_gain"] = s[f"d{name}_gain"].double() + (d * x / root).sum((0, 1, 2))
            d = d * s[name + "_gain"].double()
            d = d / root - x * (torch.linalg.vecdot(d, x)[..., None] / (c["dim"] * root ** 3))
        out["d" + name] = d
    out["dv"] = s["dv_acc"][:, :, at:at + n].double()
    return out
