"""Rows of a teacher's that hold no pair or allow no class, with a normaliser of their own that is no number, in every kernel of the distillation; gradients
of classes that are masked."""
import pytest
import torch

from test_scores_and_distillation import INF, TYPES, ctx, distill, distill_backward, logits_of, near, scores_backward, some_labels  # noqa: F401

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
