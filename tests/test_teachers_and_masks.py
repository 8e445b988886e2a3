"""Rows of a teacher's that hold no pair or allow no class, with a normaliser of their own that is no number, in every kernel of the distillation; gradients
of classes that are masked, and of rows far from zero or masked all over by a finite value."""
import pytest
import torch

import paper_2202_02365_b200 as mg
from test_scores_and_distillation import INF, TYPES, ctx, distill, distill_backward, logits_of, near, rows_of, scores_backward, some_labels, some_teacher  # noqa: F401
from test_scores_and_distillation import U
from test_table_rows_at_length import run_program

NAN = float("nan")


def teacher_rows(classes, entries, dtype, seed):
    """Twelve rows of pairs, and the teacher's lse: nothing to learn in rows 0 .. 7 (no pair, or none of a probability), pairs beside slots that are none in 8 .. 10, an lse that
    is no number with pairs of numbers in 11."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, classes, (12, entries), generator=g, device="cuda")
    values = (torch.randn(12, entries, generator=g, device="cuda") * 3).to(dtype)
    lse = torch.full((12,), 9.5, device="cuda")
    slot = torch.arange(entries, device="cuda")
    bad = torch.tensor([-1, classes, -7, 2**31 - 1], device="cuda")[slot % 4]
    anything = torch.tensor([NAN, INF, -INF, 2.0], device="cuda", dtype=dtype)[slot % 4]
    for r, l in enumerate((-INF, NAN, INF, 9.5)):      # no pair
        ids[r], values[r], lse[r] = bad, anything, l
    values[4], lse[4] = -INF, -INF                     # pairs, all of a probability of zero: a row that allows the teacher no class
    values[5] = -INF
    ids[6], lse[6] = torch.where(slot % 2 == 0, bad, ids[6]), -INF
    values[6] = torch.where(slot % 2 == 0, anything, torch.full_like(anything, -INF))
    values[7], lse[7] = -INF, INF
    for r in (8, 9, 10):
        ids[r] = torch.where((slot + r) % 3 == 0, bad, ids[r])
        values[r] = torch.where((slot + r) % 3 == 0, anything, values[r])
    values[9, ::2] = torch.where((slot + 9) % 3 == 0, anything, torch.full_like(anything, -INF))[::2]
    ids[8:11, 1 % entries], values[8:11, 1 % entries] = 0, 1.0      # (one pair at least)
    ids[11, 0], values[11, 0], lse[11] = 0, 1.0, NAN
    return ids, values, lse


# eight lanes, 32, a block of 64, of 128, parts of a row; their gradients by eight lanes, 32 and by blocks, by what there are of classes and of entries
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [5, 47, 172, 900, 2500, 9000, 50_257, 300_000])
def test_a_teachers_rows_without_pairs_whatever_their_normaliser(ctx, classes, dtype):
    for entries, t_type in ((1, "f32"), (7, "f16"), (60, "f32"), (200, "bf16"), (300, "f32")):
        x = logits_of(12, classes, TYPES[dtype], classes)
        ids, values, t_lse = teacher_rows(classes, entries, TYPES[t_type], entries)
        loss, lse = ctx.distill(x, ids, values, scale=0.5, teacher_lse=t_lse)
        d_loss = torch.linspace(0.5, 1.5, 12, device="cuda")
        d = ctx.distill_backward(d_loss, x, lse, ids, values, scale=0.5, teacher_lse=t_lse)
        assert (loss[:8] == 0).all(), loss
        assert not d[:8].any()
        fine = slice(8, 11)
        (want, off), (want_lse, lse_off) = distill(x[fine], ids[fine], values[fine], t_lse[fine], 0.5)
        near(loss[fine], want, off)
        near(lse[fine], want_lse, lse_off)
        want, off = distill_backward(x[fine], lse[fine], ids[fine], values[fine], t_lse[fine], d_loss[fine], 0.5, TYPES[dtype])
        near(d[fine], want, off)
        assert loss[11].isnan() and d[11].isnan().all()
        # the same teacher's log probabilities as they come: rows that allow it nothing, and one that allows all
        logits = logits_of(3, max(classes, 3), torch.float32, 1)
        logits[:2] = -INF
        best = ctx.log_probs(logits, top=min(entries, 3))
        loss, lse = ctx.distill(x[:3], best.top_ids, best.top_log_probs, teacher_lse=torch.where(best.lse == -INF, best.lse, 0.0))
        assert (loss[:2] == 0).all() and loss[2].isfinite()
        d = ctx.distill_backward(d_loss[:3], x[:3], lse, best.top_ids, best.top_log_probs, teacher_lse=torch.where(best.lse == -INF, best.lse, 0.0))
        assert not d[:2].any() and d[2].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,pad", [(300, 5, 0), (300, 172, 0), (33, 172, 3), (9, 1000, 1), (5, 4099, 0), (3, 50_257, 0)])
def test_masked_classes_under_a_large_gradient_of_the_entropy(ctx, rows, classes, pad):
    """A loss that is scaled up, or summed up far: what is not allowed still gets zero, not zero times infinity."""
    x = logits_of(rows, classes, torch.float32, classes, pad, masked=0.3)
    x[1:, 1] = -1e30
    labels = some_labels(rows, classes, 3)
    r = ctx.log_probs(x, labels)
    for size in (1e9, 1e30):
        h = torch.linspace(-1.0, 1.0, rows, device="cuda") * size
        want, off = scores_backward(x, r.lse, labels, None, r.entropy, h, None, 1.0, torch.float32)
        got = ctx.log_probs_backward(x, r.lse, labels, entropy=r.entropy, d_entropy=h)
        near(got, want, off)
        assert not got[x == -INF].any()


SHIFTS = {torch.float32: (0.0, 40.0, -300.0, 1e4, -1e6, 3e7, -1e9, 1e30), torch.float16: (0.0, 200.0, -3e4, 6e4), torch.bfloat16: (0.0, 100.0, 3e4, -1e30)}


def far_rows(classes, dtype, seed, pad, shift):
    """Rows about values far from zero, masked all over by a finite value, all over but for some classes, and without a class."""
    shifts = SHIFTS[dtype]
    x = logits_of(2 * len(shifts) + 10, classes, dtype, seed, pad, shift, masked=0.3)
    lowest = torch.finfo(dtype).min
    for i, by in enumerate(shifts):
        x[2 * i:2 * i + 2] = (x[2 * i:2 * i + 2].double() + by).to(dtype)
    last = x[2 * len(shifts):]
    last[0] = lowest
    last[1] = max(-1e9, lowest)
    last[2:4] = torch.where(last[2:4] == -INF, -INF, lowest)      # some are not allowed, the others masked
    last[4, classes // 2:] = lowest
    last[5, 1:] = lowest
    last[6] = -INF
    last[7] = lowest / 2
    last[8] = torch.where(last[8] == -INF, lowest, torch.full_like(last[8], lowest / 2))
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("classes", [1, 5, 20, 153, 172, 1000, 2500, 6151, 50_257, 300_007])
def test_gradients_by_the_rows_sums(ctx, classes, dtype):
    """Probabilities as exact as the forward call's, where lse is rounded to less than its sum's logarithm.  Beside the roundings that scores_backward and distill_backward count: the
    sum's relative error, its logarithm, and two roundings of x - m."""
    dtype = TYPES[dtype]
    for pad, shift, scale in ((0, 0, 1.0), (3, 1, 0.6), (0, 0, 2.5)):
        x = far_rows(classes, dtype, classes, pad, shift)
        rows = len(x)
        if scale > 1:      # (times the scale no value is beyond fp32)
            x.clamp_(min=torch.finfo(dtype).min / 4).masked_fill_(x <= torch.finfo(dtype).min / 4, torch.finfo(dtype).min / 4)
        labels = some_labels(rows, classes, 3)
        scale32 = torch.tensor(scale, dtype=torch.float32).double().item()
        most = x.double().max(1, keepdim=True).values
        about = x.double() - torch.where(most == -INF, 0.0, most)      # the same gradient, from numbers of an ordinary size
        _, _, s, p, far, sum_off = rows_of(about, scale32)
        log_s = torch.log(s)
        p_off = U * p * (sum_off + 4 * log_s.abs() + 4 * far)
        row_sums = torch.full((rows, 2), float("nan"), device="cuda")
        r = ctx.log_probs(x, labels, scale=scale, row_sums=row_sums)
        lse = scale32 * row_sums[:, 0].double() + row_sums[:, 1].double()
        assert torch.equal(lse == -INF, r.lse == -INF) and ((lse - r.lse.double()).abs() <= 2 * U * (scale32 * row_sums[:, 0].double().abs() + lse.abs()))[lse.isfinite()].all()
        g, h, l = torch.randn(3, rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(classes))
        for how in (dict(d_log_prob=g), dict(d_log_prob=g, entropy=r.entropy, d_entropy=h, d_lse=l), dict(d_lse=l)):
            want, off = scores_backward(about, log_s[:, 0], labels, how.get("d_log_prob"), how.get("entropy"), how.get("d_entropy"), how.get("d_lse"), scale32, dtype)
            sizes = [how[k].double().abs()[:, None] if k in how else 0.0 for k in ("d_log_prob", "d_entropy", "d_lse")]
            inner = torch.where(p > 0, torch.log(p).abs(), 0.0) + r.entropy.double().abs()[:, None]
            off = off + scale32 * p_off * (sizes[0] + sizes[1] * (inner + 1) + sizes[2])
            got = ctx.log_probs_backward(x, None, labels, scale=scale, row_sums=row_sums, **how)
            near(got, want, off)
            near(ctx.log_probs_backward(x, r.lse, labels, scale=scale, row_sums=row_sums, out=logits_of(rows, classes, dtype, 1, 5, 0), **how), want, off)      # (by another kernel)
            near(ctx.log_probs_backward(x.clone(), None, labels, scale=scale, row_sums=row_sums, **how), want, off)      # (rows one behind the other)
        ids, values = some_teacher(rows, classes, 20, 5)
        sums = torch.empty(rows, 2, device="cuda")
        ctx.distill(x, ids, values, scale=scale, row_sums=sums)
        want, off = distill_backward(about, log_s[:, 0], ids, values, None, l, scale32, dtype)
        off = off + scale32 * l.double().abs()[:, None] * 1.001 * p_off
        for by in (sums, row_sums):
            got = ctx.distill_backward(l, x, None, ids, values, scale=scale, row_sums=by)
            near(got, want, off)
        inplace = torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda").copy_(x)
        assert torch.equal(ctx.distill_backward(l, inplace, None, ids, values, scale=scale, row_sums=row_sums, out=inplace), got)
        inplace = torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda").copy_(x)
        assert torch.equal(ctx.log_probs_backward(inplace, None, labels, scale=scale, row_sums=row_sums, out=inplace, d_lse=l), ctx.log_probs_backward(x, None, labels, scale=scale, row_sums=row_sums, d_lse=l))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(4, 20), (4, 172), (4, 6151), (4, 250_000)])
def test_a_row_that_is_masked_all_over_by_a_finite_value(ctx, rows, classes):
    for value in (-1e9, torch.finfo(torch.float32).min):
        x = torch.full((rows, classes), value, device="cuda")
        row_sums = torch.empty(rows, 2, device="cuda")
        ctx.log_probs(x, row_sums=row_sums)
        d = ctx.log_probs_backward(x, None, d_lse=torch.ones(rows, device="cuda"), row_sums=row_sums)
        assert ((d * classes - 1).abs() <= 1e-4).all()      # (n sums of one: below 2^-24 (n / 256 + 128) by the chains, 6e-5)


@pytest.mark.gpu
def test_refusals_of_row_sums(ctx):
    x, labels, g = torch.randn(3, 8, 16, device="cuda")[0], torch.zeros(8, dtype=torch.int64, device="cuda"), torch.ones(8, device="cuda")
    good = torch.empty(8, 2, device="cuda")
    for bad in (good[:7], good.double(), good.cpu(), torch.empty(2, 8, device="cuda").t(), good[:, :1], good.view(16)):
        for call in (lambda: ctx.log_probs(x, row_sums=bad), lambda: ctx.log_probs_backward(x, g, labels, g, row_sums=bad)):
            with pytest.raises(AssertionError):
                call()
    with pytest.raises(mg.MgError) as e:
        ctx.log_probs(x, row_sums=torch.empty(17, device="cuda")[1:].view(8, 2))
    assert e.value.code == -1
    with pytest.raises(mg.MgError):
        ctx.log_probs_backward(x, None, labels, g)
    ctx.log_probs(x, labels, row_sums=good)
    assert good.isfinite().all()


PLANS = r"""
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include "mg_loss_plan.cuh"
int mg_fail(mg_ctx*, int code, const char*, ...) { return code; }
int mg_cuda_fail(mg_ctx*, cudaError_t, const char*) { return MG_ERR_CUDA; }
void mg_prof_begin(mg_ctx*, int) {}
void mg_prof_end(mg_ctx*, int, int64_t) {}

int main() {
    int bad = 0;
    for (const int dtype : {MG_DTYPE_F32, MG_DTYPE_F16, MG_DTYPE_BF16})
        for (const int64_t rows : {(int64_t)1, (int64_t)500, (int64_t)40'000, (int64_t)1 << 30})
            for (int32_t classes = 1; classes < 1100; ++classes)
                for (int32_t top = 0; top <= MG_MAX_TOP && top <= classes; ++top)
                    for (const bool threads : {false, true}) {
                        const mg_logits z{nullptr, classes, rows, classes, dtype, 1.f};
                        const ForwardPlan p = plan_forward(&z, top, threads, 148);
                        const int vec = dtype == MG_DTYPE_F32 ? 4 : 8;
                        const bool by_lanes = p.lanes >= 8 && p.lanes <= 32 && top <= p.lanes && p.nv * vec <= 32 && p.nv * p.lanes >= (classes + 2 * (vec - 1)) / vec;
                        const bool by_threads = p.lanes == 1 && threads && classes <= 32, wide = p.lanes == 0 && p.threads >= 64;
                        if (!by_lanes && !by_threads && !wide) { printf("%d classes, %d best: %d lanes of %d\n", classes, top, p.lanes, p.nv); ++bad; }
                    }
    return bad ? 1 : 0;
}
"""


def test_a_row_has_as_many_lanes_as_best_classes(tmp_path):
    run_program(tmp_path, PLANS)
