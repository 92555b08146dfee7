"""Embedding, layer norm and token loss together with the attention, as the stages of a pipeline run them: segments forward in order, backward in reverse,
gradients in fp32 accumulators; captured into a graph; on a side stream; and their compiled forms against the Python ones."""
import numpy as np
import pytest
import torch

import paper_2406_03488_amd as s1f
from paper_2406_03488_amd import binding
from ends_harness import f64, normal, placed, row_values, space, tokens_of

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -17


class Model:
    """Tokens -> table -> norm -> attention (its rows as queries, keys and values) -> norm -> loss over the same table."""

    def __init__(self, dtype, batch=2, heads=2, tokens=333, vocab=411, seed=3):
        rng = np.random.default_rng(seed)
        self.b, self.h, self.n, self.v, self.d = batch, heads, tokens, vocab, 64
        hid = self.hid = heads * 64
        self.table = normal(rng, (vocab, hid), dtype, 0.3).cuda()
        self.gain = [normal(rng, (hid,), dtype, 0.2, 1.0).cuda() for _ in range(2)]
        self.shift = [normal(rng, (hid,), dtype, 0.2).cuda() for _ in range(2)]
        self.ids = tokens_of(rng, batch, tokens, vocab, 0.05)
        self.targets = tokens_of(rng, batch, tokens, vocab, 0.2)
        self.scale = 4.0
        self.dloss = torch.from_numpy(rng.random((batch, tokens)).astype(np.float32)).cuda() / tokens

    def reference(self):
        """Loss and gradients of the unsplit sequences by autograd in 64 bits on the CPU."""
        p = [t.cpu().double().requires_grad_() for t in (self.table, *self.gain, *self.shift)]
        table, g0, g1, b0, b1 = p
        ids, targets = self.ids.cpu(), self.targets.cpu()
        on = (ids >= 0) & (ids < self.v)
        x = torch.where(on[..., None], table[ids.clamp(0, self.v - 1)] * self.scale, 0.0)
        y = torch.nn.functional.layer_norm(x, (self.hid,), g0, b0, EPS)
        q = y.view(self.b, self.n, self.h, self.d).transpose(1, 2)
        a = torch.nn.functional.scaled_dot_product_attention(q, q, q, is_causal=True).transpose(1, 2).reshape(self.b, self.n, self.hid)
        z = torch.nn.functional.layer_norm(a, (self.hid,), g1, b1, EPS) @ table.T
        counted = (targets >= 0) & (targets < self.v)
        loss = torch.nn.functional.cross_entropy(z.flatten(0, 1), torch.where(counted, targets, -100).flatten(), ignore_index=-100, reduction="none")
        loss.backward(self.dloss.cpu().double().flatten())
        return loss.detach().view(self.b, self.n), [t.grad for t in p]

    def run(self, n_seg):
        """The library's calls, segment by segment: loss, and the gradients of table (tied: from both ends), gains and shifts."""
        t, b, n, hid = self.table.dtype, self.b, self.n, self.hid
        new = lambda: torch.full((b, n, hid), float("nan"), dtype=t, device="cuda")
        x, y, a, o = new(), new(), new(), new()
        heads = lambda r: r.view(b, -1, self.h, self.d).transpose(1, 2)
        kc = torch.full((b, self.h, n, self.d), float("nan"), dtype=t, device="cuda")
        vc = kc.clone()
        bounds = s1f.partition(n, n_seg, hid, self.h)
        segs, kept, loss = list(zip(bounds[:-1], bounds[1:])), [], torch.zeros((b, n), device="cuda")
        for i, j in segs:
            s = slice(i, j)
            m0, r0, m1, r1, one, lse = (row_values(b, j - i) for _ in range(6))
            s1f.embed_fwd(self.ids[:, s], self.table, self.scale, x[:, s])
            s1f.layer_norm_fwd(x[:, s], self.gain[0], self.shift[0], EPS, y[:, s], m0, r0)
            q, out = heads(y[:, s].contiguous()), heads(torch.empty((b, j - i, hid), dtype=t, device="cuda"))
            s1f.kv_append(q, q, i, kc, vc)
            attn_lse = torch.empty((b, self.h, j - i), device="cuda")
            s1f.seg_attn_fwd(q, kc, vc, i, out, attn_lse)
            a[:, s] = out.transpose(1, 2).reshape(b, j - i, hid)
            s1f.layer_norm_fwd(a[:, s], self.gain[1], self.shift[1], EPS, o[:, s], m1, r1)
            size = s1f.token_loss_fwd_workspace_bytes(o[:, s], self.table)
            s1f.token_loss_fwd(o[:, s], self.table, self.targets[:, s], one, lse, space(size)[0])
            loss[:, s] = one
            kept.append((m0, r0, m1, r1, q, out, attn_lse, lse))
        zero = lambda *shape: torch.zeros(shape, device="cuda")
        dtable, dg, db = zero(self.v, hid), [zero(hid), zero(hid)], [zero(hid), zero(hid)]
        dk, dv = zero(*kc.shape), zero(*kc.shape)
        for (i, j), (m0, r0, m1, r1, q, out, attn_lse, lse) in reversed(list(zip(segs, kept))):
            s, g = slice(i, j), self.dloss[:, i:j].contiguous()
            do, da, dy, dx = (torch.empty_strided(x[:, s].shape, x[:, s].stride(), dtype=t, device="cuda") for _ in range(4))
            s1f.token_loss_bwd(g, o[:, s], self.table, self.targets[:, s], lse, do, dtable, space(s1f.token_loss_bwd_workspace_bytes(o[:, s], self.table))[0])
            s1f.layer_norm_bwd(do, a[:, s], self.gain[1], m1, r1, da, dg[1], db[1], space(s1f.layer_norm_bwd_workspace_bytes(do, a[:, s]))[0])
            dout, dq, dks, dvs = heads(da.contiguous()), torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
            s1f.seg_attn_bwd(dout, q, kc, vc, out, attn_lse, i, dq, dk, dv, space(s1f.bwd_workspace_bytes(q, kc, i))[0])
            s1f.kv_grad_emit(dk, dv, i, dks, dvs)
            dy.copy_((dq.float() + dks.float() + dvs.float()).to(t).transpose(1, 2).reshape(b, j - i, hid))
            s1f.layer_norm_bwd(dy, x[:, s], self.gain[0], m0, r0, dx, dg[0], db[0], space(s1f.layer_norm_bwd_workspace_bytes(dy, x[:, s]))[0])
            s1f.embed_bwd(self.ids[:, s], dx, self.scale, dtable, space(s1f.embed_bwd_workspace_bytes(self.ids[:, s], dx, dtable))[0])
        return loss, [dtable, *dg, *db]


@pytest.mark.parametrize("n_seg", [1, 4])
def test_whole_model_fp32(n_seg):
    """Ten operations in a row, each within some 1e-6 of its result (fp32 sums of up to 411 terms); nothing between them is badly conditioned: rows of a norm
    have a deviation near 1, scores a few units.  1e-4 of the largest value, the attention's contract, leaves a factor of ten."""
    m = Model("f32")
    loss, grads = m.run(n_seg)
    want_loss, want = m.reference()
    assert np.abs(f64(loss) - want_loss.numpy()).max() <= 1e-4 * want_loss.abs().max().item()
    for got, w in zip(grads, want):
        assert np.abs(f64(got) - w.numpy()).max() <= 1e-4 * w.abs().max().item()


@pytest.mark.parametrize("n_seg", [1, 4])
def test_whole_model_bf16(n_seg):
    """A gradient passes about twelve roundings to bf16 (rows, probabilities, score gradients), of at most 2^-8 each and of either sign: together, were all at
    their largest, 12 * 2^-8; relative to the norm."""
    m = Model("bf16")
    loss, grads = m.run(n_seg)
    want_loss, want = m.reference()
    assert np.linalg.norm(f64(loss) - want_loss.numpy()) <= 12 * 2.0 ** -8 * want_loss.norm().item()
    for got, w in zip(grads, want):
        assert np.linalg.norm(f64(got) - w.numpy()) <= 12 * 2.0 ** -8 * w.norm().item()


def calls(rng, dtype, n=300, h=136, v=777, batch=2):
    """Every call on its own tensors: (function, arguments, outputs, what accumulates)."""
    x, y, dy, dx = (placed(normal(rng, (batch, n, h), dtype), "dense") for _ in range(4))
    table = normal(rng, (v, h), dtype).cuda()
    ids, targets = tokens_of(rng, batch, n, v, 0.1), tokens_of(rng, batch, n, v, 0.1)
    gamma, beta = normal(rng, (h,), dtype).cuda(), normal(rng, (h,), dtype).cuda()
    rows = lambda: torch.rand((batch, n), device="cuda")
    f32 = lambda *s: torch.zeros(s, device="cuda")
    mean, rstd, loss, lse, dloss = rows(), rows(), rows(), rows() + 5, rows() / n
    dg, db, acc, dw = f32(h), f32(h), f32(v, h), f32(v, h)
    out, dxl = torch.empty_like(x), torch.empty_like(x)
    size = max(s1f.embed_bwd_workspace_bytes(ids, dy, acc), s1f.layer_norm_bwd_workspace_bytes(dy, x), s1f.token_loss_fwd_workspace_bytes(x, table),
               s1f.token_loss_bwd_workspace_bytes(x, table))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")     # one for all: calls on a stream follow each other
    return {"embed_fwd": [[ids, table, 1.5, out], [out], []], "embed_bwd": [[ids, dy, 1.5, acc, ws], [], [acc]],
            "layer_norm_fwd": [[x, gamma, beta, 1e-5, y, mean, rstd], [y, mean, rstd], []],
            "layer_norm_bwd": [[dy, x, gamma, mean, rstd, dx, dg, db, ws], [dx], [dg, db]],
            "token_loss_fwd": [[x, table, targets, loss, lse, ws], [loss, lse], []],
            "token_loss_bwd": [[dloss, x, table, targets, lse, dxl, dw, ws], [dxl], [dw]]}


def run_all(c, change=lambda args: args):
    for name, (args, _, sums) in c.items():
        for a in sums:
            a.zero_()
        getattr(s1f, name)(*change(args))


def results(c):
    return [t.clone() for _, outs, sums in c.values() for t in outs + sums]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    """One graph of every call, with one workspace; new tokens and rows before each replay, eager work in between."""
    rng = np.random.default_rng(17)
    c = calls(rng, dtype)
    run_all(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_all(c)
    inputs = [c["embed_fwd"][0][0], c["token_loss_fwd"][0][2]], [c["layer_norm_fwd"][0][0], c["layer_norm_bwd"][0][0]]
    for turn in range(4):
        for t in inputs[0]:
            t.copy_(tokens_of(rng, *t.shape, 777, 0.2 if turn else 1.0))
        for t in inputs[1]:
            t.copy_(normal(rng, t.shape, dtype))
        run_all(c)
        want = results(c)
        torch.cuda.synchronize()
        for _, outs, _ in c.values():
            for t in outs:
                t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(c), want)), turn


def test_on_the_current_stream():
    c = calls(np.random.default_rng(18), "bf16")
    run_all(c)
    want = results(c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run_all(c)
        got = results(c)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


class Sub(torch.Tensor):
    pass


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_compiled_forms_give_what_the_python_forms_give(dtype):
    c = calls(np.random.default_rng(19), dtype)
    native = binding._native()
    assert native is not binding._PythonForms
    for name, (args, _, _) in c.items():
        assert getattr(native, name)(*args) == 0, name
        assert getattr(native, name)(*([args[0].as_subclass(Sub)] + args[1:])) == -1, name
    run_all(c)
    want = results(c)
    run_all(c, lambda args: [args[0].as_subclass(Sub)] + args[1:])     # a subclass goes through the Python forms
    assert all(torch.equal(a, b) for a, b in zip(results(c), want))


def test_compiled_forms_leave_what_does_not_fit_to_the_python_forms():
    """Every argument in turn replaced by one of another shape, type, layout or place: -1, nothing launched, and the Python forms refuse it."""
    native = binding._native()
    c = calls(np.random.default_rng(20), "bf16")
    for name, (args, _, _) in c.items():
        for i, a in enumerate(args):
            if not isinstance(a, torch.Tensor) or a.dtype == torch.uint8:
                continue
            bad = [a.cpu(), a[..., :-1], a.double() if a.dtype != torch.int64 else a.int(), a[None]]
            if a.dim() > 1:
                bad.append(a.transpose(0, 1))
            for b in bad:
                put = args[:i] + [b] + args[i + 1:]
                assert getattr(native, name)(*put) == -1, (name, i)
                with pytest.raises((TypeError, ValueError)):
                    getattr(s1f, name)(*put)
        assert getattr(native, name)(*args[:-1]) == -1
    with pytest.raises(s1f.S1FError):
        s1f.embed_bwd(*c["embed_bwd"][0][:-1], None)
    with pytest.raises(s1f.S1FError):
        s1f.token_loss_bwd(*c["token_loss_bwd"][0][:-1], torch.empty(64, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()


def test_tied_gradients_of_two_calls_add_up():
    """Accumulators hold what was there: two calls give the sum of each."""
    c = calls(np.random.default_rng(21), "f32")
    args, _, (dw,) = c["token_loss_bwd"]
    dw.zero_()
    s1f.token_loss_bwd(*args)
    once = dw.clone()
    s1f.token_loss_bwd(*args)
    assert torch.equal(dw, once + once)
