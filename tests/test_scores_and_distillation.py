"""Log probabilities, distillation and their gradients against their definitions in 64 bits, at the sizes, types, strides and masks where the kernels are
cut differently, and in the ways a program may call them.

Tolerances, in units of u = 2^-24, half a step of fp32.  With d = scale (x - m): d is two roundings, 2 |d|; an exponential of d is off by that, by
2 |d| of its base's change and by 8 of its own, so by 4 |d| + 8 of itself.  A sum of n of them adds its chain, the number of additions that one value goes
through: below min(n, 1024) / 32 + n / 256 + 64 in every kernel here.  A logarithm is off by the relative error of what it is taken of and 2 of its own
value.  What follows from these stands beside each formula; h is half a step of a gradient's type."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import build

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
INF = float("inf")


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def smallest(dtype):      # half the distance of subnormal numbers
    return {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]


def chain(n):
    return min(n, 1024) / 32 + n / 256 + 64


# ---- definitions ----------------------------------------------------------------------------------------------------
def rows_of(x, scale):
    """z, m, sum exp(z - m), p, and the relative error of the sum in units."""
    z = x.double() * scale
    m = z.max(-1, keepdim=True).values
    m = torch.where(m == -INF, torch.zeros_like(m), m)
    e = torch.exp(z - m)
    s = e.sum(-1, keepdim=True)
    d = torch.where(e > 0, (z - m).abs(), torch.zeros_like(e))
    p = e / s
    off = chain(x.shape[-1]) + 8 + 4 * (p * d).sum(-1, keepdim=True)
    return z, m, s, p, d, off


def scores(x, labels, scale):
    """log_prob, entropy, lse, log p of every class; and how far each may be off."""
    z, m, s, p, d, off = rows_of(x, scale)
    log_s = torch.log(s)
    lse = m + log_s
    nothing = (z == -INF).all(-1, keepdim=True)      # lse = -infinity, entropy 0, log probabilities -infinity
    log_p = torch.where(nothing, -INF, (z - m) - log_s)
    valid = (labels >= 0) & (labels < x.shape[-1])
    at = torch.where(valid, labels, 0).long()[..., None]
    log_prob = torch.where(valid, log_p.gather(-1, at)[..., 0], 0.0)
    entropy = torch.where(nothing, 0.0, torch.special.entr(p)).sum(-1)
    # lse: m one rounding, its sum with log s another; log p: d, log s and their difference
    lse_off = U * (2 * m.abs() + 2 * lse.abs() + off + 2 * log_s.abs())
    log_p_off = U * (2 * (z - m).abs() + off + 4 * log_s.abs() + 2 * log_p.abs())
    # entropy = log s - w / s, w the sum of e d: each term off by 4 |d| + 8 and one product of itself, the sum by its chain, the quotient by the sum and a rounding
    mean_d = (p * d).sum(-1)
    entropy_off = U * (off[..., 0] + 4 * log_s[..., 0].abs() + 2 * entropy.abs() + 4 * (p * d * d).sum(-1) + mean_d * (off[..., 0] + chain(x.shape[-1]) + 16))
    log_prob_off = torch.where(valid, log_p_off.gather(-1, at)[..., 0], 0.0)
    return (log_prob, log_prob_off), (entropy, entropy_off), (lse[..., 0], lse_off[..., 0]), (log_p, log_p_off)


def scores_backward(x, lse, labels, g, entropy, h, l, scale, dtype):
    z = x.double() * scale
    log_p = z - lse.double()[..., None]
    p = torch.exp(log_p)
    zero = torch.zeros(x.shape[:-1], dtype=torch.float64, device=x.device)
    valid = (labels >= 0) & (labels < x.shape[-1]) if labels is not None else zero.bool()
    g = torch.where(valid, g.double(), zero) if g is not None else zero
    h, l = (t.double() if t is not None else zero for t in (h, l))
    entropy = entropy.double() if entropy is not None else zero
    at_label = torch.zeros_like(z)
    if labels is not None:
        at_label.scatter_(-1, torch.where(valid, labels, 0).long()[..., None], g[..., None])
    g, h, l, entropy = (t[..., None] for t in (g, h, l, entropy))
    inner = torch.where(p > 0, log_p, 0.0) + entropy
    d = at_label + p * (l - g - h * inner)
    d = torch.where((g == 0) & (h == 0) & (l == 0) | (lse == -INF)[..., None], 0.0, d) * scale
    # p: log p one rounding and 2 |log p| of the base's change, the exponential 8; the bracket: five roundings; the sum with g, the scale
    size = p * (g.abs() + l.abs() + h.abs() * (torch.where(p > 0, log_p.abs(), 0.0) + entropy.abs()))
    off = U * scale * (size * (8 * torch.where(p > 0, log_p.abs(), 0.0) + 24) + 2 * at_label.abs()) + 2 * U * d.abs()
    return d, off + half_step(dtype) * 1.01 * d.abs() + smallest(dtype) + 2.0 ** -126 * scale * (g.abs() + l.abs() + h.abs() * 100)


def teacher(ids, values, lse, classes, scale):
    """valid, q, log q; and how far log q may be off, in units."""
    valid = (ids >= 0) & (ids < classes)
    v = torch.where(valid, values.double() * scale, -INF)
    shift = torch.logsumexp(v, -1, keepdim=True) if lse is None else lse.double()[..., None]
    shift = torch.where(shift == -INF, 0.0, shift)
    log_q = v - shift
    fine = torch.where(log_q > -INF, log_q.abs(), 0.0)
    off = 2 * torch.where(v > -INF, v.abs(), 0.0) + 4 * shift.abs() + 2 * fine + chain(ids.shape[-1]) + 8
    return valid, torch.exp(log_q), torch.where(log_q > -INF, log_q, 0.0), off


def distill(x, ids, values, teacher_lse, scale):
    _, _, lse, (log_p, log_p_off) = scores(x, torch.zeros(x.shape[:-1], dtype=torch.int64, device=x.device), scale)
    valid, q, log_q, q_off = teacher(ids, values, teacher_lse, x.shape[-1], scale)
    at = torch.where(valid, ids, 0).long()
    on = valid & (q > 0)
    term = torch.where(on, q * (log_q - log_p.gather(-1, at)), 0.0)
    # each term: log q and log p, q (its logarithm's error and 4 |log q| + 8), the difference and the product; then the chain over the entries
    off = torch.where(on, U * q * (q_off + 2) + q * log_p_off.gather(-1, at) + U * term.abs() * (q_off + 4 * log_q.abs() + 16 + chain(ids.shape[-1])), 0.0)
    return (term.sum(-1), off.sum(-1)), lse


def distill_backward(x, lse, ids, values, teacher_lse, d_loss, scale, dtype):
    log_p = x.double() * scale - lse.double()[..., None]
    p = torch.exp(log_p)
    valid, q, log_q, q_off = teacher(ids, values, teacher_lse, x.shape[-1], scale)
    q_off = q_off + 4 * log_q.abs() + 12
    at = torch.where(valid, ids, 0).long()
    q = torch.where(valid, q, 0.0)
    named, named_off = torch.zeros_like(p), torch.zeros_like(p)
    named.scatter_add_(-1, at, q)
    named_off.scatter_add_(-1, at, q * q_off)
    mass, mass_off = q.sum(-1, keepdim=True), (q * (q_off + chain(ids.shape[-1]))).sum(-1, keepdim=True)
    g = d_loss.double()[..., None]
    zero = (mass == 0) | (g == 0) | (lse == -INF)[..., None]
    d = torch.where(zero, 0.0, scale * g * (p * mass - named))
    off = U * scale * g.abs() * (p * mass * (8 * torch.where(p > 0, log_p.abs(), 0.0) + 24) + p * mass_off + named_off + named * (ids.shape[-1] + 2)) + 4 * U * d.abs()
    return d, torch.where(zero, 0.0, off + half_step(dtype) * 1.01 * d.abs() + smallest(dtype) + 2.0 ** -126 * scale * g.abs())


def test_the_gradients_are_the_losses():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(6, 9, dtype=torch.float64, generator=g)
    x[1, 4] = -INF
    labels = torch.tensor([0, 3, -100, 8, 9, 2])
    c = torch.randn(3, 6, dtype=torch.float64, generator=g)

    def loss(v):
        (lp, _), (h, _), (lse, _), _ = scores(v, labels, 0.7)
        return (lp * c[0] + h * c[1] + lse * c[2]).sum()

    (_, _), (h, _), (lse, _), _ = scores(x, labels, 0.7)
    got = scores_backward(x, lse, labels, c[0], h, c[1], c[2], 0.7, torch.float32)[0]
    for r in range(6):
        for j in range(9):
            if x[r, j] > -INF:
                step = torch.zeros_like(x)
                step[r, j] = 1e-6
                assert abs(float((loss(x + step) - loss(x - step)) / 2e-6 - got[r, j])) < 1e-7
    assert got[1, 4] == 0
    ids = torch.tensor([[0, 3, 3], [1, -1, 2], [-1, 9, -1], [8, 0, 1], [5, 5, 5], [2, 1, 0]])
    values = torch.randn(6, 3, dtype=torch.float64, generator=g)
    values[5, 1] = -INF
    for t_lse in (None, torch.randn(6, dtype=torch.float64, generator=g) + 2):
        (_, _), (lse, _) = distill(x, ids, values, t_lse, 0.7)
        got = distill_backward(x, lse, ids, values, t_lse, c[0], 0.7, torch.float32)[0]
        for r in range(6):
            for j in range(9):
                if x[r, j] > -INF:
                    step = torch.zeros_like(x)
                    step[r, j] = 1e-6
                    up, down = ((distill(x + s, ids, values, t_lse, 0.7)[0][0] * c[0]).sum() for s in (step, -step))
                    assert abs(float((up - down) / 2e-6 - got[r, j])) < 1e-7
        assert not got[2].any()


# ---- on the GPU -----------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ctx():
    return mg.Context(0)


def logits_of(rows, classes, dtype, seed, pad=0, shift=0, spread=3.0, masked=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((rows * (classes + pad) + shift + 8,), float("nan"), device="cuda", dtype=dtype)
    m = wide[shift:shift + rows * (classes + pad)].view(rows, classes + pad)[:, :classes]
    v = torch.randn(rows, classes, generator=g, device="cuda") * spread
    if masked:
        v.masked_fill_(torch.rand(rows, classes, generator=g, device="cuda") < masked, -INF)
        v[0::5] = torch.where(torch.arange(classes, device="cuda") == seed % classes, 1.5, -INF)      # one class is left
    m.copy_(v)
    return m


def some_labels(rows, classes, seed, dtype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    bad = torch.tensor([-100, -1, classes, classes + 5], device="cuda")
    return torch.where(torch.rand(rows, generator=g, device="cuda") < 0.25, bad[labels % 4], labels).to(dtype)


def near(got, want, off):
    """Equal where there is no number or an infinite one, near elsewhere."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got == INF, want == INF) and torch.equal(got == -INF, want == -INF)
    fine = want.isfinite()
    off = off.nan_to_num(0.0, 0.0)      # (rows that allow nothing: exactly)
    worst = ((got - want).abs() / off.clamp(min=1e-300))[fine]
    assert (worst <= 1).all(), float(worst.max())


def top_of(x, k):
    """The k best of each row, equal ones by ascending class, NaN first."""
    order = torch.where(x.isnan(), INF, x.float())
    first = torch.sort(x.isnan().to(torch.int32), dim=-1, descending=True, stable=True).indices
    second = torch.sort(order.gather(-1, first), dim=-1, descending=True, stable=True).indices
    return first.gather(-1, second)[..., :k]


def check_scores(ctx, x, labels, top, scale):
    r = ctx.log_probs(x, labels, top=top, scale=scale)
    (lp, lp_off), (h, h_off), (lse, lse_off), (log_p, log_p_off) = scores(x, labels, torch.tensor(scale, dtype=torch.float32).double().item())
    near(r.log_prob, lp, lp_off)
    near(r.entropy, h, h_off)
    near(r.lse, lse, lse_off)
    if top:
        best = top_of(x, top)
        assert torch.equal(r.top_ids.long(), best)
        near(r.top_log_probs, log_p.gather(-1, best), log_p_off.gather(-1, best))
    else:
        assert r.top_ids is None and r.top_log_probs is None
    return r


SIZES = [(1, 1), (3, 2), (5, 31), (64, 16), (411, 100), (70, 101), (130, 172), (33, 255), (40, 257), (19, 600), (21, 1000), (9, 1025), (12, 2048), (7, 4099), (600, 4096), (5, 20_001), (150, 9000),
         (2, 50_257), (1, 131_073), (300, 33_000), (1, 1_000_003), (20_000, 47)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,classes", SIZES)
def test_log_probs(ctx, dtype, rows, classes):
    for top, pad, shift, scale, masked in ((0, 0, 0, 1.0, 0.0), (min(5, classes), 3, 1, 0.6, 0.3), (min(32, classes), 8, 0, 2.5, 0.0), (1, 0, 3, 1.0, 0.9)):
        x = logits_of(rows, classes, TYPES[dtype], rows + top, pad, shift, masked=masked)
        r = check_scores(ctx, x, some_labels(rows, classes, 3, torch.int32 if top else torch.int64), top, scale)
        again = ctx.log_probs(x, top=top, scale=scale)
        assert again.log_prob is None and torch.equal(again.lse, r.lse) and torch.equal(again.entropy, r.entropy)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [4, 100, 1000, 5000, 40_000, 300_000])
def test_equal_values_and_long_rows_of_few(ctx, classes):
    """Ties go to the lowest class, wherever they lie."""
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((6, classes), -2.0, device="cuda", dtype=dtype)
        x[1, ::3] = 5.0
        x[2] = torch.randint(0, 3, (classes,), device="cuda").to(dtype)
        x[3, classes // 2:] = 0.0
        x[3, -1] = -0.0
        x[4] = -torch.arange(classes, device="cuda").to(dtype)
        x[5] = torch.arange(classes, device="cuda").to(dtype)
        check_scores(ctx, x, torch.arange(6, device="cuda") % classes, min(32, classes), 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [3, 150, 1500, 30_000, 250_000])
def test_rows_without_a_class_and_bad_values(ctx, classes):
    for dtype in (torch.float32, torch.float16):
        lowest = torch.finfo(dtype).min
        x = logits_of(9, classes, dtype, 5)
        x[0] = -INF                         # nothing is allowed
        x[1] = lowest                       # a mask of the type's lowest value over all: every class alike
        x[2, 1:] = lowest                   # ... over all but one
        x[3, 2] = float("nan")
        x[4, 1] = INF
        x[5, :-1] = -INF
        x[6] = float("nan")
        x[7, 0], x[7, -1] = -INF, float("nan")
        labels = torch.tensor([0, 1, 0, 1, 1, classes - 1, 0, -100, 2], device="cuda")
        r = ctx.log_probs(x, labels, top=3)
        assert r.lse[0] == -INF and r.entropy[0] == 0 and r.log_prob[0] == -INF and (r.top_log_probs[0] == -INF).all() and r.top_ids[0].tolist() == [0, 1, 2]
        for row in (3, 4, 6, 7):
            assert r.lse[row].isnan() and r.entropy[row].isnan() and r.top_log_probs[row].isnan().all()
        assert r.log_prob[3].isnan() and r.log_prob[4].isnan() and r.log_prob[6].isnan() and r.log_prob[7] == 0
        assert torch.equal(r.top_ids.long(), top_of(x, 3))
        fine = torch.tensor([1, 2, 5, 8], device="cuda")
        (lp, lp_off), (h, h_off), (lse, lse_off), _ = scores(x[fine], labels[fine], 1.0)
        near(r.log_prob[fine], lp, lp_off)
        near(r.entropy[fine], h, h_off)
        near(r.lse[fine], lse, lse_off)
        ones = torch.ones(9, device="cuda")
        d = ctx.log_probs_backward(x, r.lse, labels, ones, r.entropy, 0.5 * ones, 0.25 * ones)
        assert not d[0].any() and all(d[row].isnan().any() for row in (3, 4, 6, 7))
        want, off = scores_backward(x[fine], r.lse[fine], labels[fine], ones[fine], r.entropy[fine], 0.5 * ones[fine], 0.25 * ones[fine], 1.0, dtype)
        near(d[fine], want, off)
        zero = torch.zeros(9, device="cuda")      # no gradient comes in: none goes out, whatever the row holds
        assert not ctx.log_probs_backward(x, r.lse, labels, zero, r.entropy, zero, zero).any()
        assert not ctx.log_probs_backward(x, r.lse, torch.full_like(labels, -100), ones).any()
        ids = torch.arange(3, device="cuda").expand(9, 3).contiguous()
        loss, lse = ctx.distill(x, ids, torch.zeros(9, 3, device="cuda"))
        assert loss[0] == INF and lse[0] == -INF and all(loss[row].isnan() for row in (3, 4, 6, 7)) and loss[8].isfinite()
        d = ctx.distill_backward(ones, x, lse, ids, torch.zeros(9, 3, device="cuda"))
        assert not d[0].any() and d[3].isnan().any() and d[8].isfinite().all()
        none = torch.full_like(ids, -1)
        assert not ctx.distill(x[:3], none[:3], torch.zeros(3, 3, device="cuda"))[0].any()
        assert not ctx.distill_backward(ones, x, lse, none, torch.zeros(9, 3, device="cuda")).any()
        assert not ctx.distill_backward(zero, x, lse, ids, torch.zeros(9, 3, device="cuda")).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,classes", SIZES)
def test_log_probs_backward(ctx, dtype, rows, classes):
    g = torch.Generator(device="cuda").manual_seed(2)
    for pad, shift, out_pad, scale, masked, parts in ((0, 0, 0, 1.0, 0.0, "g"), (3, 1, 5, 0.6, 0.3, "ghl"), (8, 0, 0, 2.5, 0.0, "h"), (0, 3, 0, 1.0, 0.2, "l"), (2, 0, 2, 1.0, 0.0, "gl")):
        x = logits_of(rows, classes, TYPES[dtype], rows, pad, shift, masked=masked)
        labels = some_labels(rows, classes, 3, torch.int32 if pad else torch.int64)
        r = ctx.log_probs(x, labels, scale=scale)
        d = {k: torch.randn(rows, generator=g, device="cuda") for k in "ghl"}
        d["g"][rows // 2] = 0.0
        how = dict(d_log_prob=d["g"] if "g" in parts else None, entropy=r.entropy if "h" in parts else None, d_entropy=d["h"] if "h" in parts else None, d_lse=d["l"] if "l" in parts else None)
        scale32 = torch.tensor(scale, dtype=torch.float32).double().item()
        want, off = scores_backward(x, r.lse, labels, how["d_log_prob"], how["entropy"], how["d_entropy"], how["d_lse"], scale32, TYPES[dtype])
        got = ctx.log_probs_backward(x, r.lse, labels, scale=scale, **how)
        near(got, want, off)
        out = logits_of(rows, classes, TYPES[dtype], 1, out_pad, shift)
        whole = out.as_strided((rows, out.stride(0)), out.stride(), out.storage_offset())
        assert ctx.log_probs_backward(x, r.lse, labels, scale=scale, out=out, **how) is out
        assert torch.equal(out, got) and whole[:, classes:].isnan().all()
        assert torch.equal(ctx.log_probs_backward(x, r.lse, labels, scale=scale, out=x, **how), got)      # in place


def some_teacher(rows, classes, entries, seed, ids_type=torch.int32, dtype=torch.float32, twice=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, classes, (rows, entries), generator=g, device="cuda")      # the same class twice, now and then
    values = torch.randn(rows, entries, generator=g, device="cuda") * 3
    none = torch.rand(rows, entries, generator=g, device="cuda") < 0.2
    bad = torch.tensor([-1, classes, -7, 2**31 - 1], device="cuda")
    ids = torch.where(none, bad[ids % 4], ids)
    ids[rows // 2] = -1
    values = torch.where(none, torch.where(ids % 2 == 0, float("nan"), INF), values)      # what is no pair may hold anything
    if entries > 1:
        values[0, 1] = -INF
        ids[0, 1] = 0
    return ids.to(ids_type), values.to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,classes,entries", [(1, 1, 1), (3, 2, 2), (64, 16, 5), (411, 100, 10), (70, 101, 32), (130, 172, 33), (19, 600, 64), (9, 1025, 100), (12, 2048, 256), (7, 4099, 50),
                                                  (600, 4096, 20), (5, 20_001, 1024), (2, 50_257, 50), (300, 33_000, 64), (1, 1_000_003, 200), (20_000, 47, 8)])
def test_distill(ctx, dtype, rows, classes, entries):
    for pad, shift, scale, masked, wide, t_type, with_lse in ((0, 0, 1.0, 0.0, False, "f32", False), (3, 1, 0.5, 0.0, True, "bf16", True), (8, 0, 2.0, 0.2, False, "f16", False)):
        x = logits_of(rows, classes, TYPES[dtype], rows, pad, shift, masked=masked)
        ids, values = some_teacher(rows, classes, entries, 5, torch.int64 if wide else torch.int32, TYPES[t_type])
        if masked:      # a class that the student does not allow costs an infinite loss: not here
            x.scatter_(1, torch.where((ids >= 0) & (ids < classes), ids, 0).long(), torch.zeros((), device="cuda", dtype=x.dtype).expand(rows, entries))
        t_lse = torch.full((rows,), 9.5, device="cuda") if with_lse else None
        if pad:      # rows of the teacher's that lie apart
            ids, values = (torch.cat([t, t[:, :1]], 1)[:, :entries] for t in (ids, values))
        scale32 = torch.tensor(scale, dtype=torch.float32).double().item()
        loss, lse = ctx.distill(x, ids, values, scale=scale, teacher_lse=t_lse)
        (want, off), (want_lse, lse_off) = distill(x, ids, values, t_lse, scale32)
        near(loss, want, off)
        near(lse, want_lse, lse_off)
        assert loss[rows // 2] == 0
        d_loss = torch.randn(rows, device="cuda")
        d_loss[0] = 1.0
        got = ctx.distill_backward(d_loss, x, lse, ids, values, scale=scale, teacher_lse=t_lse)
        want, off = distill_backward(x, lse, ids, values, t_lse, d_loss, scale32, TYPES[dtype])
        near(got, want, off)
        out = logits_of(rows, classes, TYPES[dtype], 1, 5 if pad else 0, shift)
        whole = out.as_strided((rows, out.stride(0)), out.stride(), out.storage_offset())
        ctx.distill_backward(d_loss, x, lse, ids, values, scale=scale, teacher_lse=t_lse, out=out)
        assert torch.equal(out, got) and whole[:, classes:].isnan().all()
        assert torch.equal(ctx.distill_backward(d_loss, x, lse, ids, values, scale=scale, teacher_lse=t_lse, out=x), got)      # in place


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [7, 8, 63, 153, 172, 1023, 1024, 1026, 1500, 2048, 2049, 6144, 6151, 16_400, 70_003, 140_001])
def test_best_classes_wherever_they_lie(ctx, classes):
    """The best at the rows' ends, at the borders of what a thread, a round and a row's part hold, and rising or falling along the row."""
    for dtype in (torch.float32, torch.bfloat16):
        for rows in (1, 40):
            x = logits_of(rows, classes, dtype, classes, 1, 1, spread=0.5)
            g = torch.Generator(device="cuda").manual_seed(classes)
            at = torch.cat([torch.tensor([0, classes - 1, classes // 2], device="cuda"), torch.randint(0, classes, (9,), generator=g, device="cuda")]).unique()
            x[:, at] = (10 + torch.randperm(len(at), generator=g, device="cuda")).to(dtype)
            if rows > 1:
                x[1] = (torch.arange(classes, device="cuda") / classes).to(dtype)      # rising: many equal ones in two bytes
                x[2] = -(torch.arange(classes, device="cuda") / classes).to(dtype)
                x[3, :classes // 3] = 9.0
            check_scores(ctx, x, some_labels(rows, classes, 1), min(32, classes), 0.8)
            check_scores(ctx, x, some_labels(rows, classes, 2), min(7, classes), 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [1100, 2500, 6151, 16_400, 70_003, 300_007])
def test_many_equal_values_and_few_classes_that_are_allowed(ctx, classes):
    """Rows of which many more classes are as good as the last of the best than there is room for, or fewer allowed than are asked for."""
    for dtype in (torch.float32, torch.float16):
        for rows in (1, 30):
            g = torch.Generator(device="cuda").manual_seed(classes + rows)
            x = torch.full((rows, classes + 3), float("nan"), dtype=dtype, device="cuda")[:, 1:1 + classes]
            some = lambda n: torch.randint(0, classes, (n,), generator=g, device="cuda")
            for r in range(rows):
                x[r] = (-INF, torch.finfo(dtype).min, 0.0, -1e4)[r % 4]
                x[r, some((0, 1, 5, 20, 90, 600)[r // 4 % 6])] = torch.randn(1, generator=g, device="cuda").item()
                if r % 3 == 1:
                    x[r, some(9)] = torch.randn(9, generator=g, device="cuda").to(dtype)
            if rows > 1:
                x[24] = (torch.arange(classes, device="cuda") // 7 / classes).to(dtype)      # rising by sevens
                x[25, some(900)] = float("nan")
                x[26, some(40)], x[27, some(40)] = float("nan"), INF
                x[28] = -INF
                x[28, [0, classes - 1]] = 1.0
                x[29, classes // 2:] = -INF
            for top in (32, 5):
                r = ctx.log_probs(x, top=top)
                best = top_of(x, top)
                assert torch.equal(r.top_ids.long(), best)
                fine = slice(0, 25)
                (_, _), (_, _), (lse, lse_off), (log_p, log_p_off) = scores(x[fine], some_labels(len(x[fine]), classes, 1), 1.0)
                near(r.lse[fine], lse, lse_off)
                near(r.top_log_probs[fine], log_p.gather(-1, best[fine]), log_p_off.gather(-1, best[fine]))


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [1, 2, 5, 8, 9, 16, 20, 31, 32, 33])
def test_many_rows_of_few_classes(ctx, classes):
    for dtype in (torch.float32, torch.float16):
        for pad, masked in ((0, 0.0), (3, 0.4)):
            x = logits_of(40_001, classes, dtype, classes, pad, 1 if pad else 0, masked=masked)
            x[5] = -INF
            x[6], x[7] = 1.0, -0.0
            x[7, ::2] = 0.0
            check_scores(ctx, x, some_labels(40_001, classes, 1), classes if classes < 33 else 32, 0.5)
            check_scores(ctx, x, some_labels(40_001, classes, 2, torch.int32), 1, 1.0)
            x[8, 0], x[9, classes // 2] = float("nan"), INF
            r = ctx.log_probs(x, top=classes if classes < 33 else 32)
            assert r.lse[8].isnan() and r.lse[9].isnan() and torch.equal(r.top_ids.long(), top_of(x, r.top_ids.shape[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(1, 8), (7, 153), (300, 153), (3000, 172), (50, 1024), (33, 2047), (257, 4), (900, 12), (5, 2048)])
def test_runs_of_rows_with_and_without_gradients(ctx, rows, classes):
    """Rows that lie one behind the other: every third without a label, some without any gradient, some that allow nothing, as the first and the last of all."""
    for dtype in (torch.float32, torch.float16):
        x = logits_of(rows, classes, dtype, rows)
        x = x.contiguous()
        labels = torch.randint(0, classes, (rows,), device="cuda")
        labels[::3] = -100
        x[rows // 2] = -INF
        r = ctx.log_probs(x, labels)
        g, h, l = torch.randn(3, rows, device="cuda")
        h[1::4] = l[1::4] = 0.0
        for how in (dict(d_log_prob=g), dict(d_log_prob=g, entropy=r.entropy, d_entropy=h, d_lse=l)):
            want, off = scores_backward(x, r.lse, labels, how["d_log_prob"], how.get("entropy"), how.get("d_entropy"), how.get("d_lse"), 1.0, dtype)
            got = ctx.log_probs_backward(x, r.lse, labels, **how)
            near(got, want, off)
            assert not got[rows // 2].any()
            inplace = x.clone()
            assert torch.equal(ctx.log_probs_backward(inplace, r.lse, labels, out=inplace, **how), got)


@pytest.mark.gpu
def test_shapes_and_nothing(ctx):
    x = logits_of(24, 50, torch.float32, 1).view(2, 3, 4, 50)
    labels = torch.randint(0, 50, (2, 3, 4), device="cuda")
    r = ctx.log_probs(x, labels, top=2)
    flat = ctx.log_probs(x.view(24, 50), labels.view(24), top=2)
    assert r.log_prob.shape == (2, 3, 4) and r.top_ids.shape == (2, 3, 4, 2) and torch.equal(r.top_ids.view(24, 2), flat.top_ids) and torch.equal(r.lse.view(24), flat.lse)
    d = ctx.log_probs_backward(x, r.lse, labels, torch.ones_like(r.lse))
    assert d.shape == x.shape
    loss, lse = ctx.distill(x, r.top_ids, r.top_log_probs)
    assert loss.shape == (2, 3, 4) and ctx.distill_backward(torch.ones_like(loss), x, lse, r.top_ids, r.top_log_probs).shape == x.shape
    apart = x.transpose(1, 2)      # rows that do not lie one behind the other
    assert torch.equal(ctx.log_probs(apart).lse, r.lse.transpose(1, 2))
    r = ctx.log_probs(x[:0], labels[:0], top=3)
    assert r.lse.shape == (0, 3, 4) and r.top_ids.shape == (0, 3, 4, 3)
    assert ctx.log_probs_backward(x[:0], r.lse, labels[:0], r.lse).shape == (0, 3, 4, 50)
    assert ctx.distill(x[:0], r.top_ids, r.top_log_probs)[0].shape == (0, 3, 4)
    one = x[0, 0, :1].expand(7, 50)      # one row over and over
    assert (ctx.log_probs(one).lse == ctx.log_probs(x[0, 0, :1]).lse).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(1, 70_000), (9, 300), (500, 6000), (3000, 100)])
def test_runs_alike_on_other_streams_and_captured(ctx, rows, classes):
    x, labels = logits_of(rows, classes, torch.float32, 1), some_labels(rows, classes, 2)
    ids, values = some_teacher(rows, classes, 20, 3)
    d = torch.randn(rows, device="cuda")

    def all_of():
        r = ctx.log_probs(x, labels, top=7)
        grad = ctx.log_probs_backward(x, r.lse, labels, d, r.entropy, d, d)
        loss, lse = ctx.distill(x, ids, values, 0.5)
        return r.log_prob, r.entropy, r.lse, r.top_ids, r.top_log_probs, grad, loss, lse, ctx.distill_backward(d, x, lse, ids, values, 0.5)

    first = all_of()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(all_of())
    torch.cuda.synchronize()
    for other in got:
        assert all(torch.equal(a, b) for a, b in zip(first, other))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, all_of()))
    for seed in (4, 5):
        x.copy_(logits_of(rows, classes, torch.float32, seed))
        labels.copy_(some_labels(rows, classes, seed))
        torch.cuda.synchronize()
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = all_of()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.gpu
def test_more_than_two_to_the_31_elements(ctx):
    rows, classes = 45_000, 50_257      # 4.5 GB
    x = torch.zeros(rows, classes, dtype=torch.bfloat16, device="cuda")
    x[-1, -3], x[-1, 7], x[44_000, 5] = 20.0, 19.0, 3.0
    labels = torch.full((rows,), classes - 3, device="cuda")
    r = ctx.log_probs(x, labels, top=2)
    few = torch.tensor([0, 43_999, 44_000, rows - 1], device="cuda")
    (lp, lp_off), _, (lse, lse_off), _ = scores(x[few], labels[few], 1.0)
    near(r.log_prob[few], lp, lp_off)
    near(r.lse[few], lse, lse_off)
    assert r.top_ids[few].tolist() == [[0, 1], [0, 1], [5, 0], [classes - 3, 7]]
    g = torch.ones(rows, device="cuda")
    ids, values = r.top_ids, r.top_log_probs
    d = ctx.distill_backward(g, x, r.lse, ids, values)
    want, off = distill_backward(x[few], r.lse[few], ids[few], values[few], None, g[few], 1.0, torch.bfloat16)
    near(d[few], want, off)
    ctx.log_probs_backward(x, r.lse, labels, g, out=d)
    want, off = scores_backward(x[few], r.lse[few], labels[few], g[few], None, None, None, 1.0, torch.bfloat16)
    near(d[few], want, off)


@pytest.mark.gpu
def test_refusals(ctx):
    x, labels, lse = torch.randn(12, 16, device="cuda"), torch.zeros(12, dtype=torch.int64, device="cuda"), torch.zeros(12, device="cuda")
    ids, values = torch.zeros(12, 4, dtype=torch.int32, device="cuda"), torch.zeros(12, 4, device="cuda")
    many = torch.zeros(12, 1025, dtype=torch.int32, device="cuda")
    bad = [lambda: ctx.log_probs(x, top=33), lambda: ctx.log_probs(x, top=-1), lambda: ctx.log_probs(x, top=17), lambda: ctx.log_probs(x, scale=0.0), lambda: ctx.log_probs(x, scale=-1.0),
           lambda: ctx.log_probs(x, scale=float("nan")), lambda: ctx.log_probs(x, scale=INF), lambda: ctx.log_probs(x[:, :0]), lambda: ctx.log_probs_backward(x, lse, None, lse),
           lambda: ctx.log_probs_backward(x, lse, d_entropy=lse), lambda: ctx.log_probs_backward(x, None, labels, lse), lambda: ctx.log_probs_backward(x[:8], lse[:8], labels[:8], lse[:8], out=x[2:10]),
           lambda: ctx.log_probs_backward(x, lse, labels, lse, out=torch.empty(1, 16, device="cuda").expand(12, 16)), lambda: ctx.distill(x, ids[:, :0], values[:, :0]),
           lambda: ctx.distill(x, many, many.float()), lambda: ctx.distill(x, ids, values, scale=0.0), lambda: ctx.distill_backward(None, x, lse, ids, values)]
    for call in bad:
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.code == -1
    wrong = [lambda: ctx.log_probs(x.cpu()), lambda: ctx.log_probs(x.double()), lambda: ctx.log_probs(x[0]), lambda: ctx.log_probs(x, labels[:3]), lambda: ctx.log_probs(x, labels.float()),
             lambda: ctx.log_probs(x, labels.cpu()), lambda: ctx.log_probs_backward(x, lse[:3], labels, lse), lambda: ctx.log_probs_backward(x, lse, labels, lse.double()),
             lambda: ctx.log_probs_backward(x, lse, labels, lse, out=x.half()), lambda: ctx.distill(x, ids[:3], values[:3]), lambda: ctx.distill(x, ids, values[:, :3]),
             lambda: ctx.distill(x, ids.float(), values), lambda: ctx.distill(x, ids, values.double()), lambda: ctx.distill(x, ids, values, teacher_lse=lse[:2])]
    for call in wrong:
        with pytest.raises(AssertionError):
            call()


# ---- a training step ------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dims,count,entries", [([16, 16, 40], 60, 5), ([64, 128, 172], 500, 20)])
def test_a_step_of_learned_rows_against_labels_and_a_teacher(ctx, dims, count, entries):
    """Looked-up rows through two layers of a GraphSage model to both losses and back: every gradient against the formulas' in 64 bits."""
    from paper_2202_02365_b200 import inputs
    n, classes = 900, dims[-1]
    graph = inputs.erdos_renyi_graph(n, 8000, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    kinds = torch.randint(-1, 50, (n,), generator=gen, device="cuda")      # what a node is of; -1: unknown
    table = torch.randn(50, dims[0], generator=gen, device="cuda")
    layers = inputs.random_bias_layers(dims, seed=5)
    own = mg.Context(0)
    own.load_graph(graph.row_offsets.cuda(), graph.nbrs.cuda())
    rows = own.embedding(table, kinds, scale=0.5)
    own.load_features(rows)
    own.keep_layer_outputs(True)
    targets = inputs.distinct_targets(n, count, seed=6)
    d = own.sample(targets, [5, 4], seed=7)
    model = own.model(layers, mg.GEMM_FP32)
    logits = torch.empty(count, classes, device="cuda")
    own.forward(model, d, logits)
    labels = torch.randint(-1, classes, (count,), generator=gen, device="cuda")
    big = torch.randn(count, classes, generator=gen, device="cuda") * 2
    best = own.log_probs(big, top=entries)      # the teacher
    r = own.log_probs(logits, labels)
    loss, lse = own.distill(logits, best.top_ids, best.top_log_probs, scale=0.5)
    d_lp, d_loss = torch.full((count,), -0.3, device="cuda"), torch.full((count,), 0.7, device="cuda")
    d_logits = own.log_probs_backward(logits, r.lse, labels, d_lp) + own.distill_backward(d_loss, logits, lse, best.top_ids, best.top_log_probs, scale=0.5)
    grads, d_h0, ids = own.backward(model, d, d_logits, want_h0_grad=True)
    d_table = own.embedding_backward(d_h0, kinds[ids.long()], 50, scale=0.5)

    # the same by torch's autograd in 64 bits
    v = d.view(0)
    nodes = v.node_ids.cpu().long()
    k64 = kinds.cpu()
    t64 = table.cpu().double().requires_grad_()
    w64 = [tuple(w.double().requires_grad_() for w in layer) for layer in layers]
    h = torch.where((k64 >= 0)[:, None], 0.5 * t64[k64.clamp(min=0)], 0.0)[nodes]
    out = _layers(h, v, w64)
    logp = torch.log_softmax(out, 1)
    lab = labels.cpu()
    total = -0.3 * torch.where((lab >= 0), logp.gather(1, lab.clamp(min=0)[:, None])[:, 0], 0.0).sum()
    q = torch.softmax(0.5 * best.top_log_probs.cpu().double(), 1)
    logp = torch.log_softmax(0.5 * out, 1).gather(1, best.top_ids.cpu().long())
    total = total + 0.7 * (q * (q.log() - logp)).sum()
    total.backward()
    assert (logits.cpu().double() - out.detach()).abs().max() <= 1e-4 * out.detach().abs().max()
    got_total = -0.3 * r.log_prob.double().sum() + 0.7 * loss.double().sum()
    assert abs(float(got_total) - float(total)) <= 1e-4 * abs(float(total))
    for (gs, gn, gb), (ws, wn, wb) in zip(grads, w64):
        for got, want in ((gs, ws.grad), (gn, wn.grad), (gb, wb.grad)):
            assert (got.cpu().double() - want).abs().max() <= 4e-4 * want.abs().max()
    assert (d_table.cpu().double() - t64.grad).abs().max() <= 4e-4 * t64.grad.abs().max()


def _layers(h, view, weights):
    """Two GraphSage layers over a mini-batch's arrays, with autograd: rows of the last delta out first, as the arrays have it."""
    ids_off, ends, rmap = (t.cpu().long() for t in (view.node_id_offsets, view.nbr_offsets, view.repr_map))
    n_nodes, start = view.node_ids.numel(), 0      # start: where h's rows begin in node_ids
    for l, (ws, wn, b) in enumerate(weights):
        first = int(ids_off[l + 1])      # rows from here on have neighbours at this layer
        mine = torch.arange(first, n_nodes)
        at = mine - int(ids_off[1])
        rows = []
        for i in at.tolist():
            e = rmap[int(ends[i]):int(ends[i + 1])] - start
            rows.append(h[e].mean(0) if len(e) else torch.zeros(h.shape[1], dtype=h.dtype))
        out = h[mine - start] @ ws + torch.stack(rows) @ wn + b
        h = torch.relu(out) if l + 1 < len(weights) else out
        start = first
    return h


# ---- refusals that need no GPU --------------------------------------------------------------------------------------
HOST = r"""
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include "mg_loss_plan.cuh"
int mg_fail(mg_ctx*, int code, const char*, ...) { return code; }
int mg_cuda_fail(mg_ctx*, cudaError_t, const char*) { return MG_ERR_CUDA; }
void mg_prof_begin(mg_ctx*, int) {}
void mg_prof_end(mg_ctx*, int, int64_t) {}

static mg_ctx context;
static int bad = 0;
#define EXPECT(code, call) do { const int got = (call); if (got != (code)) { printf("line %d: %d\n", __LINE__, got); ++bad; } } while (0)

int main() {
    char *base = reinterpret_cast<char*>(1ull << 30), *far = base + (1ll << 42), *more = base + (1ll << 44);   // (addresses are only compared)
    float *f = reinterpret_cast<float*>(more), *odd = reinterpret_cast<float*>(more + 2);
    const mg_logits z{base, 100, 50, 100, MG_DTYPE_F32, 1.f};
    const auto fwd = [&](auto change, int32_t top = 5, const void* labels = nullptr, int wide = 0, const float* lp = nullptr, const float* lse = nullptr) {
        mg_logits a = z; change(a); return check_log_probs(&context, &a, labels, wide, top, lp, f, lse, reinterpret_cast<int32_t*>(f), f);
    };
    const auto same = [](mg_logits&) {};
    EXPECT(MG_OK, fwd(same));
    EXPECT(MG_OK, fwd([](mg_logits& a) { a.stride = 0; }));
    EXPECT(MG_OK, fwd([](mg_logits& a) { a.rows = 0; a.x = nullptr; }));
    EXPECT(MG_OK, fwd([](mg_logits& a) { a.classes = 1 << 28; a.rows = 1; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.classes = (1 << 28) + 1; a.rows = 1; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.classes = 0; }, 0));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.x = nullptr; }));
    EXPECT(MG_ERR_ARG, fwd([&](mg_logits& a) { a.x = base + 2; }));
    EXPECT(MG_OK, fwd([&](mg_logits& a) { a.x = base + 2; a.dtype = MG_DTYPE_BF16; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.dtype = 3; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.rows = -1; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.rows = 1ll << 31; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.stride = -1; }));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.stride = (1ll << 28) + 1; }));
    for (const float s : {0.f, -1.f, (float)NAN, (float)INFINITY}) EXPECT(MG_ERR_ARG, fwd([&](mg_logits& a) { a.scale = s; }));
    EXPECT(MG_ERR_ARG, fwd(same, -1));
    EXPECT(MG_ERR_ARG, fwd(same, 33));
    EXPECT(MG_ERR_ARG, fwd([](mg_logits& a) { a.classes = 4; }));
    EXPECT(MG_OK, fwd([](mg_logits& a) { a.classes = 5; }));
    EXPECT(MG_ERR_ARG, fwd(same, 5, nullptr, 0, f));
    EXPECT(MG_OK, fwd(same, 5, far + 4, 0, f));
    EXPECT(MG_ERR_ARG, fwd(same, 5, far + 4, 1, f));
    EXPECT(MG_ERR_ARG, fwd(same, 5, far, 1, odd));
    EXPECT(MG_ERR_ARG, fwd(same, 5, far, 1, f, odd));
    EXPECT(MG_ERR_ARG, check_log_probs(&context, nullptr, nullptr, 0, 0, nullptr, nullptr, nullptr, nullptr, nullptr));

    struct B { const float* lse; const void* labels; const float *g, *entropy, *h, *l; const void* d; int64_t ds; };
    const B ok{f, far, f, f, f, f, far, 100};
    const auto bwd = [&](auto change) { B a = ok; change(a); return check_log_probs_backward(&context, &z, a.lse, a.labels, 1, a.g, a.entropy, a.h, a.l, a.d, a.ds); };
    EXPECT(MG_OK, bwd([](B&) {}));
    EXPECT(MG_OK, bwd([&](B& a) { a.d = base; }));
    EXPECT(MG_OK, bwd([](B& a) { a.labels = nullptr; a.g = nullptr; a.entropy = nullptr; a.h = nullptr; a.l = nullptr; }));
    EXPECT(MG_ERR_ARG, bwd([&](B& a) { a.d = base + 400; }));
    EXPECT(MG_ERR_ARG, bwd([&](B& a) { a.d = base; a.ds = 104; }));
    EXPECT(MG_ERR_ARG, bwd([](B& a) { a.ds = 99; }));
    EXPECT(MG_ERR_ARG, bwd([](B& a) { a.d = nullptr; }));
    EXPECT(MG_ERR_ARG, bwd([](B& a) { a.lse = nullptr; }));
    EXPECT(MG_ERR_ARG, bwd([](B& a) { a.labels = nullptr; }));
    EXPECT(MG_ERR_ARG, bwd([](B& a) { a.entropy = nullptr; }));
    EXPECT(MG_ERR_ARG, bwd([&](B& a) { a.l = odd; }));

    const mg_teacher t{base + (1ll << 36), base + (1ll << 37), nullptr, 64, 64, 0, MG_DTYPE_F16, 64};
    const auto teach = [&](auto change) { mg_teacher a = t; change(a); return check_distill(&context, &z, &a, f, nullptr); };
    EXPECT(MG_OK, teach([](mg_teacher&) {}));
    EXPECT(MG_OK, teach([](mg_teacher& a) { a.entries = 1024; a.ids_stride = a.values_stride = 1024; }));
    EXPECT(MG_OK, teach([](mg_teacher& a) { a.ids_stride = a.values_stride = 0; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.entries = 1025; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.entries = 0; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.ids = nullptr; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.values = nullptr; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.dtype = 7; }));
    EXPECT(MG_ERR_ARG, teach([](mg_teacher& a) { a.ids_stride = -1; }));
    EXPECT(MG_ERR_ARG, teach([&](mg_teacher& a) { a.ids = base + 4; a.ids_are_i64 = 1; }));
    EXPECT(MG_ERR_ARG, teach([&](mg_teacher& a) { a.lse = odd; }));
    EXPECT(MG_ERR_ARG, check_distill(&context, &z, &t, nullptr, nullptr));
    EXPECT(MG_ERR_ARG, check_distill(&context, &z, nullptr, f, nullptr));
    EXPECT(MG_OK, check_distill_backward(&context, &z, f, &t, f, far, 100));
    EXPECT(MG_ERR_ARG, check_distill_backward(&context, &z, f, &t, nullptr, far, 100));
    EXPECT(MG_ERR_ARG, check_distill_backward(&context, &z, nullptr, &t, f, far, 100));
    EXPECT(MG_ERR_ARG, check_distill_backward(&context, &z, f, &t, f, base + 4, 100));
    return bad;
}
"""


def test_refusals_on_the_host(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    source, program = tmp_path / "host.cu", str(tmp_path / "host")
    source.write_text(HOST)
    made = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xcompiler", "-w", "-I", build.CSRC,
                           "-I", os.path.join(build.ROOT, "include"), str(source), "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([program], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
