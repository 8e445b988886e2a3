"""Norm, activation and dropout between the layers of a GraphSage model, as a training loop uses them: forward pass, backward pass, optimiser steps,
against the definition differentiated by torch in 64 bits.

Tolerance of the fp32 models: a layer's sums have at most 2 * 48 products, each term off by a few 2^-24, and enter a norm that divides by deviations
of order one; three layers, forward and back, stay below 10 * 6 * 100 * 2^-24 = 4e-4 of a result's norm in the worst case, and a value below
ten times that of the largest one."""
import math

import numpy as np
import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import inputs

pytestmark = pytest.mark.gpu

N = 5_000


def mask(keys, channels, p, seed, site):
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    blocks, keys = -(-channels // 8), np.asarray(keys).astype(np.uint64)[:, None]
    c = [np.broadcast_to(x, (len(keys), blocks)) for x in (keys & low, keys >> shift, np.arange(blocks, dtype=np.uint64)[None], np.full((1, 1), 0x64720000 + site, dtype=np.uint64))]
    k0, k1 = seed % 2**32, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k0), b & low, (a >> shift) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2**32, (k1 + 0xBB67AE85) % 2**32
    halves = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(len(keys), -1)[:, :channels]
    return torch.from_numpy(halves >= np.uint64(round(p * 65536)))


def act(n, kind):
    return {"none": lambda: n, "relu": lambda: torch.relu(n), "silu": lambda: n * torch.sigmoid(n), "gelu": lambda: n * 0.5 * torch.erfc(-n / math.sqrt(2))}[kind]()


def between(z, l, b, ids, how, params):
    if how["over"] is None:
        h = torch.relu(z)
    else:
        per = z.reshape(z.shape[0], how["groups"], -1)
        over = (2,) if how["over"] == "rows" else (0, 2)
        var, mean = torch.var_mean(per, dim=over, correction=0, keepdim=True)
        hat = ((per - mean) / torch.sqrt(var + how["eps"])).reshape(z.shape)
        h = act(hat * params[l][0] + params[l][1], how["activation"])
    if how["p"] > 0:
        keep = mask(ids.numpy() + (b << 32), z.shape[1], how["p"], how["seed"], l)
        t = round(how["p"] * 65536)
        h = torch.where(keep, h * (65536 / (65536 - t) if t < 65536 else 0.0), torch.zeros((), dtype=torch.float64))
    return h


def reference(views, feats, layers, norms, how, d_outs=None):
    """Outputs and, with a loss sum(d_out * H^k), the gradients of weights, norms and rows."""
    params = [[p.double().requires_grad_() for p in layer] for layer in layers]
    nps = {l + 1: [p.double().requires_grad_() for p in q] for l, q in enumerate(norms)}
    outs, rows, loss = [], [], 0.0
    for b, v in enumerate(views):
        ids, nio = v.node_ids.cpu().long(), v.node_id_offsets.cpu().tolist()
        rep, off = v.repr_map.cpu().long(), v.nbr_offsets.cpu().long()
        h = feats[ids].double().requires_grad_()
        rows.append((ids, h))
        for l, (ws, wn, bias) in enumerate(params):
            first, drop = nio[l + 1] - nio[l], nio[l + 1] - nio[1]
            n_out = h.shape[0] - first
            lo, hi = off[drop], off[drop + n_out]
            cnt = off[drop + 1:drop + n_out + 1] - off[drop:drop + n_out]
            dst = torch.repeat_interleave(torch.arange(n_out), cnt)
            agg = torch.zeros((n_out, h.shape[1]), dtype=torch.float64).index_add(0, dst, h[rep[lo:hi] - nio[l]]) / cnt.clamp(min=1).double()[:, None]
            h = h[first:] @ ws + agg @ wn + bias
            if l + 1 < len(params):
                h = between(h, l + 1, b, ids[nio[l + 1]:], how, nps)
        outs.append(h.detach())
        if d_outs is not None:
            loss = loss + (h * d_outs[b].double().cpu()).sum()
    if d_outs is not None:
        loss.backward()
    return torch.cat(outs), params, nps, rows


class Run:
    def __init__(self, dims, fanouts, counts, precision=mg.GEMM_FP32):
        self.graph = inputs.erdos_renyi_graph(N, 10 * N, seed=3)
        self.feats = inputs.normal_features(N, dims[0], seed=4)
        self.layers = inputs.random_bias_layers(dims, seed=5)
        self.ctx = mg.Context(0)
        self.ctx.load_graph(self.graph.row_offsets.cuda(), self.graph.nbrs.cuda())
        self.ctx.load_features(self.feats.cuda())
        self.model = self.ctx.model(self.layers, precision)
        targets = inputs.distinct_targets(N, sum(counts), seed=6)
        self.dense = self.ctx.sample_many(targets, np.cumsum([0] + counts), fanouts, list(range(len(counts))))
        self.views = [self.dense.view(b) for b in range(len(counts))]
        g = torch.Generator().manual_seed(7)
        self.norms = [[1 + 0.3 * torch.randn(d, generator=g), 0.3 * torch.randn(d, generator=g)] for d in dims[1:-1]]
        self.d_out = torch.randn(sum(counts), dims[-1], generator=g)
        self.counts, self.dims = counts, dims

    def set(self, how):
        self.model.set_norm(how["over"], how["groups"], [n[0] for n in self.norms], [n[1] for n in self.norms], how["eps"], how["activation"])
        self.model.set_dropout(how["p"], how["seed"])

    def forward(self):
        out = torch.empty(sum(self.counts), self.dims[-1], device="cuda")
        return self.ctx.forward(self.model, self.dense, out)


def near(got, want, rel=4e-4):
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape
    assert float((got - want).norm() / want.norm()) < rel
    assert float((got - want).abs().max() / want.abs().max()) < 10 * rel


def how(over, groups=1, activation="silu", p=0.0, seed=11, eps=1e-3):
    return dict(over=over, groups=groups, activation=activation, p=p, seed=seed, eps=eps)


CASES = [([16, 24, 8], [4, 3], [40], how("rows")), ([48, 32, 40, 8], [4, 3, 2], [30, 1, 17], how("batch", 4, "gelu", 0.4)), ([16, 32, 32, 8], [3, 3, 2], [25, 40], how("rows", 8, "none", 0.2)),
         ([32, 48, 12], [5, 4], [60, 3], how(None, p=0.5, seed=2**63 + 5)), ([16, 16, 4], [4, 3], [9] * 70, how("batch", 2, "silu", 0.1)), ([12, 20, 4], [4, 3], [33], how("batch", 20, "gelu")),
         ([16, 8], [4], [50], how("rows", p=0.5))]


@pytest.mark.parametrize("dims,fanouts,counts,what", CASES)
def test_training_step(dims, fanouts, counts, what):
    r = Run(dims, fanouts, counts)
    r.set(what)
    plain = r.forward().clone()
    r.ctx.keep_layer_outputs(True)
    out = r.forward()
    assert torch.equal(out, plain)                 # the norm in the layers' place or beside them
    grads, g_h0, ids = r.ctx.backward(r.model, r.dense, r.d_out.cuda(), want_h0_grad=True)
    want, params, nps, rows = reference(r.views, r.feats, r.layers, r.norms, what, torch.split(r.d_out, counts))
    near(out, want)
    for l, (got, p) in enumerate(zip(grads, params)):
        for x, y in zip(got, p):
            if y.dim() == 1 and what["over"] == "batch" and l + 1 < len(r.layers) and what["groups"] == len(y):
                # a norm takes away what is added to all values of a group: where a channel is a group, the gradient of its bias in front is
                # zero, a sum of terms that are as large as those of the weights' gradients
                assert float(y.grad.abs().max()) < 1e-12
                assert float(x.norm()) < 4e-4 * float(p[0].grad.norm())
                continue
            near(x.view(y.shape), y.grad)
    if what["over"] and len(dims) > 2:
        for l, got in enumerate(r.model.norm_grads()):
            for x, y in zip(got, nps[l + 1]):
                near(x, y.grad)
    at = 0
    for node_ids, h in rows:
        n = len(node_ids)
        got_ids, got = ids[at:at + n].cpu().long(), g_h0[at:at + n].cpu()
        place = torch.empty(N, dtype=torch.long)
        place[node_ids] = torch.arange(n)
        near(got, h.grad[place[got_ids]])
        at += n
    # the same again: what the dropout keeps goes by the seed, and a new seed keeps others
    again = r.ctx.backward(r.model, r.dense, r.d_out.cuda())
    for a, b in zip(again, grads):
        near(a[0], b[0], 1e-5)
    if what["p"] and len(dims) > 2:
        r.model.set_dropout(what["p"], what["seed"] + 1)
        for a, b in zip(r.ctx.backward(r.model, r.dense, r.d_out.cuda()), grads):
            near(a[0], b[0], 1e-5)                 # the backward pass goes by its forward pass
        assert not torch.equal(r.forward(), out)


@pytest.mark.parametrize("over", ["rows", "batch"])
@pytest.mark.parametrize("step", ["sgd", "adagrad"])
def test_steps_move_the_norms(over, step):
    r = Run([16, 32, 24, 8], [4, 3, 2], [40, 20])
    what = how(over, 4, "gelu", 0.3)
    r.set(what)
    r.ctx.keep_layer_outputs(True)
    layers, norms = [[p.double() for p in q] for q in r.layers], [[p.double() for p in q] for q in r.norms]
    sums = [[torch.zeros_like(p) for p in q] for q in layers + norms]
    for i in range(3):
        seed = 100 + i
        r.model.set_dropout(what["p"], seed)
        out = r.forward()
        r.ctx.backward(r.model, r.dense, r.d_out.cuda())
        r.ctx.sgd_step(r.model, 1e-3) if step == "sgd" else r.ctx.adagrad_step(r.model, 1e-2)
        want, params, nps, _ = reference(r.views, r.feats, layers, norms, {**what, "seed": seed}, torch.split(r.d_out, r.counts))
        near(out, want, 4e-4 * (i + 1))
        with torch.no_grad():
            for q, ps, ss in zip(layers + norms, params + [nps[l + 1] for l in range(len(norms))], sums):
                for j, (p, s) in enumerate(zip(ps, ss)):
                    s += p.grad.view(s.shape) ** 2
                    q[j] = q[j] - (1e-3 * p.grad if step == "sgd" else 1e-2 * p.grad / (s.view(p.shape).sqrt() + 1e-10)).view(q[j].shape)


def test_tensor_core_layers_and_many_mini_batches():
    for over in ("rows", "batch", None):
        what = how(over, 8 if over else 1, "relu", 0.5)
        outs = []
        for precision in (mg.GEMM_FP32, mg.GEMM_TF32):
            r = Run([64, 128, 64, 16], [6, 4, 3], [150] * 9, precision)
            r.set(what)
            r.ctx.set_layer_window(2)
            r.model.set_intermediates(torch.float16)
            outs.append(r.forward().clone())
            r.ctx.keep_layer_outputs(True)
            near(r.forward(), outs[-1], 1e-6)
            outs.append(r.ctx.backward(r.model, r.dense, r.d_out.cuda()))
        near(outs[2], outs[0], 1e-2)                 # operands of ten bits
        for a, b in zip(outs[3], outs[1]):
            near(a[0], b[0], 3e-2)                   # (a ReLU's side of zero goes by them here and there)
            near(a[2], b[2], 3e-2)


def test_the_plain_model_is_as_it_was():
    r = Run([64, 128, 16], [6, 4], [150, 70], mg.GEMM_TF32)
    r.ctx.keep_layer_outputs(True)
    out = r.forward().clone()
    grads = r.ctx.backward(r.model, r.dense, r.d_out.cuda())
    r.set(how("batch", 4, p=0.3))
    assert not torch.equal(r.forward(), out)
    r.model.set_norm(None)
    r.model.set_dropout(0.0)
    assert torch.equal(r.forward(), out)
    for a, b in zip(r.ctx.backward(r.model, r.dense, r.d_out.cuda()), grads):
        near(a[0], b[0], 1e-5)
    r.model.set_dropout(1.0, 3)
    layers = r.layers
    near(r.forward(), layers[-1][2].expand(220, 16), 1e-6)      # all of the first layer dropped: the last one's bias


def test_gradients_of_the_norm_are_the_callers_own():
    r = Run([16, 32, 8], [4, 3], [40])
    r.set(how("rows", 4))
    r.ctx.keep_layer_outputs(True)
    r.forward()
    d_out = r.d_out.cuda()
    r.ctx.backward(r.model, r.dense, d_out)
    want = [t.clone() for q in r.model.norm_grads() for t in q]
    other = 3 * d_out
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):      # a stream that is behind
        torch.cuda._sleep(100_000_000)
        got = [t for q in r.model.norm_grads() for t in q]
    r.ctx.backward(r.model, r.dense, other)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_mini_batches_without_targets():
    for over in ("rows", "batch"):
        r = Run([16, 32, 24, 8], [4, 3, 2], [5])
        r.set(how(over, 4, p=0.3))
        r.ctx.keep_layer_outputs(True)
        for counts in ([0, 0], [0, 7, 0]):
            ends = np.cumsum([0] + counts).tolist()
            dense = r.ctx.sample_many(torch.arange(sum(counts), dtype=torch.int32, device="cuda"), ends, [4, 3, 2], list(range(1, len(counts) + 1)))
            out = r.ctx.forward(r.model, dense, torch.zeros(max(1, sum(counts)), 8, device="cuda"))
            assert bool(out.isfinite().all()) and bool(out.any()) == (sum(counts) > 0)
            if sum(counts) == 0:
                continue                              # (no forward pass that a backward pass could follow)
            grads, g_h0, _ = r.ctx.backward(r.model, dense, torch.ones_like(out), want_h0_grad=True)
            assert bool(g_h0.isfinite().all())
            for t in [t for q in grads + r.model.norm_grads() for t in q]:
                assert bool(t.isfinite().all()) and bool(t.any())


def test_refusals():
    r = Run([16, 24, 8], [4, 3], [40])
    for call in (lambda: r.model.set_norm("rows", 5), lambda: r.model.set_norm("rows", 0), lambda: r.model.set_norm("batch", 2, eps=0.0), lambda: r.model.set_dropout(1.5),
                 lambda: r.model.set_dropout(float("nan"))):
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.code == -1
    with pytest.raises(mg.MgError) as e:
        r.model.norm_grads()
    assert e.value.code == -2
    r.set(how("rows", 2, p=0.2))
    with pytest.raises(AssertionError):
        r.model.set_norm("rows", 2, [torch.ones(24)] * 2)
    out = r.forward()
    for call in (lambda: r.ctx.backward(r.model, r.dense, r.d_out.cuda()), lambda: r.ctx.forward_noalloc(r.model, r.dense, out), lambda: r.model.norm_grads()):
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.code == -2
    r.ctx.keep_layer_outputs(True)
    r.forward()
    r.model.set_norm("batch", 2)
    with pytest.raises(mg.MgError) as e:          # the forward pass was of the norm before
        r.ctx.backward(r.model, r.dense, r.d_out.cuda())
    assert e.value.code == -2
