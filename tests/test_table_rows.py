"""Rows looked up by id and their gradient against their definitions in 64 bits, at the sizes, types, strides and ids where the kernels are cut
differently, and in the ways a program may call them.

Tolerances.  u = 2^-24 is half a step of fp32, h half a step of the result's type (0 for fp32, whose roundings are counted with the others).  A
looked-up value is one product, rounded to fp32 and to the type.  A sum is off by at most (chain + 2) u times the sum of its magnitudes, the chain being
the number of additions that one value goes through: below the length of its group, and below 512 in every kernel here; the scale and what is
added to are one rounding each."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import build

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def smallest(dtype):      # half the distance of subnormal numbers
    return {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]


# ---- definitions (the scale is a float of 32 bits) -------------------------------------------------------------------
def in_32_bits(scale):
    return torch.tensor(scale, dtype=torch.float32).double().item()


def looked_up(table, ids, scale):
    valid = (ids >= 0) & (ids < table.shape[0])
    y = torch.zeros(*ids.shape, table.shape[1], dtype=torch.float64, device=table.device)
    y[valid] = in_32_bits(scale) * table[ids[valid].long()].double()
    return y


def summed_up(d_y, ids, n_rows, scale):
    """The gradient, the sums of its magnitudes and the number of places of each row."""
    ids, d_y = ids.reshape(-1).long(), d_y.reshape(-1, d_y.shape[-1]).double() * in_32_bits(scale)
    valid = (ids >= 0) & (ids < n_rows)
    out = torch.zeros(n_rows, d_y.shape[1], dtype=torch.float64, device=d_y.device)
    size = torch.zeros_like(out)
    out.index_add_(0, ids[valid], d_y[valid])
    size.index_add_(0, ids[valid], d_y[valid].abs())
    return out, size, torch.bincount(ids[valid], minlength=n_rows)


def test_the_gradient_is_the_lookups():
    g = torch.Generator().manual_seed(1)
    table = torch.randn(5, 3, dtype=torch.float64, generator=g, requires_grad=True)
    ids = torch.tensor([4, -1, 0, 4, 5, 2, 4])
    d_y = torch.randn(7, 3, dtype=torch.float64, generator=g)
    (torch.where(((ids >= 0) & (ids < 5))[:, None], 1.5 * table[ids.clamp(0, 4)], 0.0) * d_y).sum().backward()
    got = summed_up(d_y, ids, 5, 1.5)[0]
    assert torch.allclose(got, table.grad, rtol=1e-14)
    for r, c in ((4, 0), (0, 2), (1, 1)):      # and that of differences
        step = torch.zeros(5, 3, dtype=torch.float64)
        step[r, c] = 1e-6
        slope = ((looked_up(table.detach() + step, ids, 1.5) - looked_up(table.detach() - step, ids, 1.5)) * d_y).sum() / 2e-6
        assert abs(float(slope - got[r, c])) < 1e-8


# ---- on the GPU -----------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ctx():
    return mg.Context(0)


def matrix(rows, cols, dtype, seed, pad=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), device="cuda", dtype=dtype)
    m = wide[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    return m


def ids_of(n, n_rows, seed, kind="skewed", dtype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(n, generator=g, device="cuda").double()
    ids = (u ** {"skewed": 4.0, "even": 1.0, "padded": 2.0, "one": 60.0}[kind] * n_rows).long().clamp(max=n_rows - 1)
    if kind == "padded":
        bad = torch.tensor([-1, -100, n_rows, n_rows + 7, -2**31], device="cuda")
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.3, bad[torch.randint(0, 5, (n,), generator=g, device="cuda")], ids)
    return ids.to(dtype)


def check_lookup(got, table, ids, scale):
    want = looked_up(table, ids, scale)
    assert ((got.double() - want).abs() <= (U + half_step(got.dtype)) * 1.001 * want.abs() + smallest(got.dtype)).all()


SIZES = [(1, 1, 1), (3, 2, 7), (512, 10_000, 16), (1000, 50, 100), (4096, 4096, 128), (4097, 100_000, 101), (77, 3, 768), (20_000, 14_824, 64), (300, 1000, 1030), (70_000, 70_001, 8),
         (65, 5, 4100)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,n_rows,dim", SIZES)
def test_lookup(ctx, dtype, n, n_rows, dim):
    for kind, wide, pad, shift, scale in (("even", True, 0, 0, 1.0), ("padded", False, 3, 1, 11.3)):
        table = matrix(n_rows, dim, TYPES[dtype], 3, pad, shift)
        ids = ids_of(n, n_rows, 4, kind, torch.int64 if wide else torch.int32)
        for to in (None, torch.float32, torch.bfloat16):
            check_lookup(ctx.embedding(table, ids, scale, dtype=to), table, ids, scale)
        out = matrix(n, dim, TYPES[dtype], 5, 8 if pad else 2, shift)
        around = out.as_strided((n, out.stride(0)), out.stride(), out.storage_offset())[:, dim:] if n > 1 else out[:, dim:]
        assert ctx.embedding(table, ids, scale, out=out) is out and around[:-1].isnan().all()
        check_lookup(out, table, ids, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,pad,shift", [(2, 0, 0), (6, 0, 2), (36, 0, 0), (36, 4, 4), (36, 2, 2), (50, 0, 0), (100, 0, 0), (100, 2, 6), (602, 6, 0), (300, 0, 4), (8, 0, 1), (128, 4, 0), (2052, 0, 0)])
def test_widths_and_beginnings_between_vectors(ctx, dim, pad, shift):
    """Rows of 4, 8 and 16 bytes' multiples that begin at others, of each pair of types, both ways."""
    ids = ids_of(700, 90, 1, "padded")
    for dtype in TYPES.values():
        table, d_y = matrix(90, dim, dtype, 2, pad, shift), matrix(700, dim, dtype, 3, pad, shift)
        for to in TYPES.values():
            check_lookup(ctx.embedding(table, ids, 1.7, dtype=to), table, ids, 1.7)
            out = matrix(700, dim, to, 4, pad, shift)
            ctx.embedding(table, ids, 1.7, out=out)
            check_lookup(out, table, ids, 1.7)
            want, size, count = summed_up(d_y, ids, 90, 1.7)
            check_sums(ctx.embedding_backward(d_y, ids, 90, 1.7, dtype=to), want, size, count)
            out = matrix(90, dim, to, 5, pad, shift)
            around = out.as_strided((90, out.stride(0)), out.stride(), out.storage_offset())[:, dim:]
            ctx.embedding_backward(d_y, ids, 90, 1.7, out=out)
            check_sums(out, want, size, count)
            assert around[:-1].isnan().all()


@pytest.mark.gpu
def test_lookup_of_nothing_and_of_shapes(ctx):
    table = matrix(9, 12, torch.float32, 1)
    assert ctx.embedding(table, torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0, 12)
    ids = torch.tensor([[[3], [8]], [[-1], [9]]], device="cuda")
    got = ctx.embedding(table, ids, 2.0)
    assert got.shape == (2, 2, 1, 12) and torch.equal(got[0, 0, 0], table[3] * 2) and not got[1].any()
    assert torch.equal(ctx.embedding(table, torch.tensor(5, device="cuda")), table[5])
    assert not ctx.embedding(table[:0], ids).any()
    table[3, 2], table[3, 4] = float("nan"), float("inf")
    got = ctx.embedding(table, torch.tensor([3, -1, 2], device="cuda"), 0.5)
    assert got[0, 2].isnan() and got[0, 4] == float("inf") and not got[1].any() and torch.equal(got[2], table[2] * 0.5)
    got = ctx.embedding(table, ids.view(2, 2).t())      # ids that do not lie one behind the other
    assert torch.equal(got[1, 0], table[8])
    high = torch.tensor([2**32 + 3, -2**32, 2**63 - 1], device="cuda")      # their low halves are rows
    assert not ctx.embedding(table, high).any()


def check_groups(groups, ids, n_rows):
    flat = ids.reshape(-1).long()
    valid = (flat >= 0) & (flat < n_rows)
    count = int(groups.count)
    distinct, sizes = torch.unique(flat[valid], return_counts=True)
    assert count == len(distinct) and torch.equal(groups.ids[:count].long(), distinct) and groups.ids.dtype == ids.dtype
    ends = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), sizes.cumsum(0)])
    assert torch.equal(groups.starts[:count + 1].long(), ends)
    of = torch.repeat_interleave(torch.arange(count, device="cuda"), sizes)
    assert torch.equal(groups.group_of[:len(of)].long(), of) and (groups.group_of[len(of):] == -1).all()
    key = torch.where(valid, flat, n_rows)
    assert torch.equal(groups.order.long(), torch.argsort(key, stable=True))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["skewed", "even", "padded", "one"])
@pytest.mark.parametrize("n,n_rows", [(1, 1), (2, 1), (31, 5), (1000, 255), (1000, 256), (4096, 257), (4097, 65_535), (8192, 65_536), (12_289, 20_000_000), (100_000, 3), (543_000, 2_000_000),
                                      (1_500_007, 2**31 - 2), (3_000_001, 14_824)])
def test_groups(ctx, n, n_rows, kind):
    for dtype in (torch.int64, torch.int32):
        ids = ids_of(n, n_rows, n, kind, dtype)
        if n > 5 and dtype == torch.int64:
            ids[3] = 2**40 + 1
        check_groups(ctx.id_groups(ids, n_rows), ids, n_rows)


@pytest.mark.gpu
def test_groups_of_nothing(ctx):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    check_groups(ctx.id_groups(none, 5), none, 5)
    bad = torch.full((5000,), -1, device="cuda")
    check_groups(ctx.id_groups(bad, 5), bad, 5)
    check_groups(ctx.id_groups(bad, 0), bad, 0)
    for ids in (torch.arange(9000, device="cuda"), torch.arange(9000, device="cuda").flip(0), torch.zeros(9000, dtype=torch.int64, device="cuda")):
        check_groups(ctx.id_groups(ids, 9000), ids, 9000)
        check_groups(ctx.id_groups(ids, 1), ids, 1)


def check_sums(got, want, size, count, before=None):
    chain = count.clamp(max=512)[:, None].double()
    if before is not None:
        want, size = want + before.double(), size + before.double().abs()
    bound = (chain + 3) * U * size + half_step(got.dtype) * 1.001 * want.abs() + smallest(got.dtype)
    assert ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() / bound).max())


def check_gradient(ctx, d_y, ids, n_rows, scale):
    want, size, count = summed_up(d_y, ids, n_rows, scale)
    groups = ctx.id_groups(ids, n_rows)
    for to in (None, torch.float32, torch.bfloat16):
        got = ctx.embedding_backward(d_y, groups if to else ids, n_rows, scale, dtype=to)
        assert got.dtype == (to or d_y.dtype)
        check_sums(got, want, size, count)
        assert not got[count == 0].any()
    distinct, rows = ctx.embedding_backward_rows(d_y, ids, n_rows, scale)
    assert torch.equal(distinct.long(), torch.nonzero(count)[:, 0])
    assert torch.equal(rows, ctx.embedding_backward(d_y, groups, n_rows, scale)[count > 0])
    before = matrix(n_rows, d_y.shape[-1], torch.float32, 9, 4)
    before[count == 0] = float("nan")      # what is not touched may hold anything
    kept = before.clone()
    ctx.embedding_backward(d_y, groups, n_rows, scale, out=before, accumulate=True)
    assert before[count == 0].isnan().all()
    check_sums(before[count > 0], want[count > 0], size[count > 0], count[count > 0], kept[count > 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,n_rows,dim", SIZES)
def test_gradient(ctx, dtype, n, n_rows, dim):
    for kind, wide, pad, shift, scale in (("skewed", True, 0, 0, 1.0), ("padded", False, 3, 1, 11.3)):
        check_gradient(ctx, matrix(n, dim, TYPES[dtype], 6, pad, shift), ids_of(n, n_rows, 7, kind, torch.int64 if wide else torch.int32), n_rows, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_rows,dim,kind", [(300_000, 4, 128, "even"), (200_000, 1000, 100, "one"), (400_000, 1, 32, "even"), (100_000, 300_000, 192, "skewed"), (33_000, 7, 1024, "skewed")])
def test_gradient_of_many_places(ctx, n, n_rows, dim, kind):
    check_gradient(ctx, matrix(n, dim, torch.float32, 8), ids_of(n, n_rows, 9, kind), n_rows, 0.25)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [15, 16, 17, 33, 1023, 1024, 1025, 4097, 12_345])
def test_ids_that_begin_and_end_anywhere(ctx, n):
    """Runs of equal ids of every length around a chunk's, from every place on; ids that are none among them."""
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.randint(1, 50, (n,), generator=g, device="cuda"))[:n]
    ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, -1, ids)
    for order in (ids, ids[torch.randperm(n, generator=g, device="cuda")]):
        for dim in (4, 12, 40, 128, 257, 520):
            d_y = matrix(n, dim, torch.float32, dim)
            want, size, count = summed_up(d_y, order, n, 1.0)
            got = ctx.embedding_backward(d_y, order, n)
            check_sums(got, want, size, count)
            assert not got[count == 0].any()
            check_sums(ctx.embedding_backward(d_y.bfloat16(), order, n, dtype=torch.float32), *summed_up(d_y.bfloat16(), order, n, 1.0))


@pytest.mark.gpu
def test_long_sums_of_drifting_values(ctx):
    """All values of a group have one sign and grow along it: a lost or doubled part is far outside the bound."""
    n, dim = 250_000, 36
    d_y = (1 + torch.arange(n, device="cuda").float()[:, None] / n).expand(n, dim).contiguous()
    for ids in (torch.zeros(n, dtype=torch.int64, device="cuda"), torch.arange(n, device="cuda") // 100_000, torch.arange(n, device="cuda") % 3):
        want, size, count = summed_up(d_y, ids, 3, 1.0)
        check_sums(ctx.embedding_backward(d_y, ids, 3), want, size, count)


@pytest.mark.gpu
def test_gradient_of_nothing_and_of_shapes(ctx):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert not ctx.embedding_backward(torch.empty(0, 12, device="cuda"), none, 7).any()
    distinct, rows = ctx.embedding_backward_rows(torch.empty(0, 12, device="cuda"), none, 7)
    assert distinct.shape == (0,) and rows.shape == (0, 12)
    d_y = torch.ones(2, 3, 4, device="cuda")
    ids = torch.tensor([[1, 1, -1], [9, 0, 1]], device="cuda")
    got = ctx.embedding_backward(d_y, ids, 2, 0.5)
    assert got.tolist() == [[0.5] * 4, [1.5] * 4]
    d_y[0, 2] = float("nan")      # the row of an id that is none
    d_y[1, 1] = float("inf")
    got = ctx.embedding_backward(d_y, ids, 2)
    assert (got[0] == float("inf")).all() and (got[1] == 3).all()
    bad = torch.full((6,), -1, device="cuda")
    assert not ctx.embedding_backward(d_y.view(6, 4), bad, 2).any()
    assert ctx.embedding_backward(d_y.view(6, 4), bad, 0).shape == (0, 4)
    same = torch.ones(1, 4, device="cuda").expand(50, 4)      # one row over and over
    assert (ctx.embedding_backward(same, torch.zeros(50, dtype=torch.int64, device="cuda"), 1) == 50).all()


@pytest.mark.gpu
def test_runs_alike_and_on_other_streams(ctx):
    d_y, ids = matrix(120_000, 100, torch.float32, 1), ids_of(120_000, 5000, 2)
    first = ctx.embedding_backward(d_y, ids, 5000)
    for _ in range(3):
        assert torch.equal(ctx.embedding_backward(d_y, ids, 5000), first)
    side = [torch.cuda.Stream() for _ in range(3)]
    table = matrix(5000, 100, torch.float32, 3)
    torch.cuda.synchronize()
    got = []
    for s in side:      # several at once, each with a workspace of its own
        with torch.cuda.stream(s):
            got.append((ctx.embedding_backward(d_y, ids, 5000), ctx.embedding(table, ids), ctx.embedding_backward_rows(d_y, ids, 5000)))
    torch.cuda.synchronize()
    for d_table, y, (distinct, rows) in got:
        assert torch.equal(d_table, first) and torch.equal(y, table[ids]) and torch.equal(rows, first[distinct])


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_rows,dim", [(300, 50, 16), (9000, 2000, 100), (60_000, 100_000, 128)])
def test_captured_and_replayed(ctx, n, n_rows, dim):
    d_y, table = matrix(n, dim, torch.float32, 1), matrix(n_rows, dim, torch.float32, 2)
    ids = ids_of(n, n_rows, 3)
    ctx.embedding_backward(d_y, ids, n_rows)
    graphs = []
    torch.cuda.synchronize()
    for _ in range(2):      # two graphs, replayed at once
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, ctx.embedding(table, ids, 3.0), ctx.embedding_backward(d_y, ids, n_rows, 3.0)))
    for seed in (4, 5, 6):
        ids.copy_(ids_of(n, n_rows, seed, "padded"))
        d_y.copy_(matrix(n, dim, torch.float32, seed))
        torch.cuda.synchronize()
        for (g, _, _), s in zip(graphs, (torch.cuda.Stream(), torch.cuda.Stream())):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want, size, count = summed_up(d_y, ids, n_rows, 3.0)
        for _, y, d_table in graphs:
            check_lookup(y, table, ids, 3.0)
            check_sums(d_table, want, size, count)


@pytest.mark.gpu
def test_more_than_two_to_the_31_elements(ctx):
    n, dim = 5_000_001, 512      # rows of half precision: 5 GB each
    table = torch.empty(n, dim, dtype=torch.float16, device="cuda")
    table.copy_((torch.arange(n, device="cuda") % 1021).half()[:, None].expand(n, dim))
    ids = torch.arange(n, device="cuda", dtype=torch.int32).flip(0)
    y = ctx.embedding(table, ids)
    for i in (0, 1, 4_194_303, 4_194_304, n - 1):
        assert (y[i] == (n - 1 - i) % 1021).all()
    assert torch.equal(y[:, 511], table[:, 3].flip(0))
    d = ctx.embedding_backward(y, ids, n)
    assert torch.equal(d[:, 0], table[:, 0]) and torch.equal(d[:, 511], table[:, 511])
    # few rows, far apart
    del table, y, d
    far = torch.empty(20, 1 << 28, dtype=torch.float16, device="cuda")[:, :64]
    far.copy_(torch.arange(20, device="cuda").half()[:, None].expand(20, 64))
    ids = torch.tensor([19, 0, 11], device="cuda")
    assert ctx.embedding(far, ids)[:, 0].tolist() == [19, 0, 11]
    ctx.embedding_backward(torch.ones(3, 64, dtype=torch.float16, device="cuda"), ids, 20, out=far, accumulate=True)
    assert far[:, 63].tolist() == [v + (v in (19, 0, 11)) for v in range(20)]


@pytest.mark.gpu
def test_refusals(ctx):
    table, ids, d_y = torch.randn(12, 16, device="cuda"), torch.arange(8, device="cuda"), torch.randn(8, 16, device="cuda")
    bad = [lambda: ctx.embedding(table, ids, float("nan")), lambda: ctx.embedding(table, ids, float("inf")), lambda: ctx.embedding(table, ids, out=table[:8]),
           lambda: ctx.embedding(table, ids, out=torch.randn(1, 16, device="cuda").expand(8, 16)), lambda: ctx.embedding_backward(d_y, ids, 12, float("inf")),
           lambda: ctx.embedding_backward(table[:8], ids, 12, out=table), lambda: ctx.id_groups(ids, -1), lambda: ctx.id_groups(ids, 2**31 - 1)]
    for call in bad:
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.code == -1
    groups = ctx.id_groups(ids, 12)
    wrong = [lambda: ctx.embedding(table.cpu(), ids), lambda: ctx.embedding(table.double(), ids), lambda: ctx.embedding(table, ids.cpu()), lambda: ctx.embedding(table, ids.float()),
             lambda: ctx.embedding(table[0], ids), lambda: ctx.embedding(table, ids, out=torch.empty(8, 15, device="cuda")), lambda: ctx.embedding(table, ids, out=torch.empty(16, 8, device="cuda").t()),
             lambda: ctx.embedding(table, ids, dtype=torch.float16, out=torch.empty(8, 16, device="cuda")), lambda: ctx.embedding_backward(d_y[:7], ids, 12),
             lambda: ctx.embedding_backward(d_y, groups, 13), lambda: ctx.embedding_backward(d_y[:7], groups, 12), lambda: ctx.embedding_backward(d_y, ids, 12, accumulate=True),
             lambda: ctx.embedding_backward(d_y, ids, 12, out=torch.empty(11, 16, device="cuda"))]
    for call in wrong:
        with pytest.raises(AssertionError):
            call()


# ---- refusals that need no GPU --------------------------------------------------------------------------------------
HOST = r"""
#include <cstdarg>
#include <cstdio>
#include "mg_rows_plan.cuh"
int mg_fail(mg_ctx*, int code, const char*, ...) { return code; }
int mg_cuda_fail(mg_ctx*, cudaError_t, const char*) { return MG_ERR_CUDA; }
void mg_prof_begin(mg_ctx*, int) {}
void mg_prof_end(mg_ctx*, int, int64_t) {}

static mg_ctx context;
static int bad = 0;
#define EXPECT(code, call) do { const int got = (call); if (got != (code)) { printf("line %d: %d\n", __LINE__, got); ++bad; } } while (0)

int main() {
    char *base = reinterpret_cast<char*>(1ull << 30), *far = base + (1ll << 42), *ids = base + (1ll << 44), *more = base + (1ll << 45);   // (addresses are only compared)
    const int64_t huge = (1ll << 31) - 1;
    struct L { const void* table; int64_t ts; int td; int64_t rows; int32_t dim; const void* ids; int wide; int64_t n; float scale; const void* y; int64_t ys; int yd; };
    const L ok{base, 16, MG_DTYPE_F32, 100, 16, ids, 1, 50, 2.f, far, 16, MG_DTYPE_F16};
    const auto lookup = [&](auto change) { L a = ok; change(a); return check_lookup(&context, a.table, a.ts, a.td, a.rows, a.dim, a.ids, a.wide, a.n, a.scale, a.y, a.ys, a.yd); };
    EXPECT(MG_OK, lookup([](L&) {}));
    EXPECT(MG_OK, lookup([](L& a) { a.ts = 0; }));
    EXPECT(MG_OK, lookup([](L& a) { a.n = 0; a.ids = a.y = nullptr; }));
    EXPECT(MG_OK, lookup([](L& a) { a.rows = 0; a.table = nullptr; }));
    EXPECT(MG_OK, lookup([&](L& a) { a.y = base + 6400; }));
    EXPECT(MG_OK, lookup([](L& a) { a.scale = -1.f; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.y = base + 6396; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.y = base - 50 * 32 + 2; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.table = nullptr; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.ids = nullptr; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.y = nullptr; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.td = 3; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.yd = -1; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.dim = 0; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.dim = (1 << 22) + 1; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.n = -1; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.n = huge; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.rows = -1; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.rows = huge; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.ids = ids + 4; }));
    EXPECT(MG_OK, lookup([&](L& a) { a.ids = ids + 4; a.wide = 0; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.ids = ids + 2; a.wide = 0; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.table = base + 2; }));
    EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.y = far + 1; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.ys = 15; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.ys = 0; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.ts = -1; }));
    EXPECT(MG_ERR_ARG, lookup([](L& a) { a.ts = (1ll << 28) + 1; }));
    for (const float s : {(float)NAN, (float)INFINITY}) EXPECT(MG_ERR_ARG, lookup([&](L& a) { a.scale = s; }));

    struct G { const void* ids; int wide; int64_t n, rows; const void *order, *of, *gids, *starts, *count, *ws; size_t bytes; };
    const G good{ids, 0, 10000, 500, base, base + 80000, far, far + 8000, far + 16000, more, 1 << 30};
    if (plan_groups(1024, 500).bytes || !plan_groups(1025, 500).bytes) { printf("small\n"); ++bad; }
    const auto groups = [&](auto change) { G a = good; change(a); return check_groups(&context, a.ids, a.wide, a.n, a.rows, a.order, a.of, a.gids, a.starts, a.count, a.ws, a.bytes); };
    EXPECT(MG_OK, groups([](G&) {}));
    EXPECT(MG_OK, groups([](G& a) { a.bytes = plan_groups(a.n, a.rows).bytes; }));
    EXPECT(MG_ERR_CAPACITY, groups([](G& a) { a.bytes = plan_groups(a.n, a.rows).bytes - 1; }));
    EXPECT(MG_ERR_CAPACITY, groups([](G& a) { a.ws = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([&](G& a) { a.ws = more + 8; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.order = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.of = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.gids = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.starts = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.count = nullptr; }));
    EXPECT(MG_ERR_ARG, groups([&](G& a) { a.order = base + 2; }));
    EXPECT(MG_ERR_ARG, groups([&](G& a) { a.wide = 1; a.gids = far + 4; }));
    EXPECT(MG_ERR_ARG, groups([&](G& a) { a.n = huge; }));
    EXPECT(MG_ERR_ARG, groups([&](G& a) { a.rows = huge; }));
    EXPECT(MG_ERR_ARG, groups([](G& a) { a.ids = nullptr; }));

    struct S { const void* d; int64_t ds; int dd; int64_t n, rows; int32_t dim; float scale; const void *order, *of, *gids; int wide; const void *starts, *count; int into; const void* out; int64_t os; int od; const void* ws; size_t bytes; };
    const S fine{base, 16, MG_DTYPE_F32, 1000, 500, 16, 1.f, ids, ids + 20000, ids + 4000, 0, ids + 8000, ids + 16000, MG_ROWS_TABLE, far, 16, MG_DTYPE_F32, more, 1 << 30};
    const auto sums = [&](auto change) { S a = fine; change(a); return check_sums(&context, a.d, a.ds, a.dd, a.n, a.rows, a.dim, a.scale, a.order, a.of, a.gids, a.wide, a.starts, a.count, a.into, a.out, a.os, a.od, a.ws, a.bytes); };
    EXPECT(MG_OK, sums([](S&) {}));
    EXPECT(MG_OK, sums([](S& a) { a.into = MG_ROWS_COMPACT; }));
    EXPECT(MG_OK, sums([](S& a) { a.bytes = sums_workspace(a.n, a.rows, a.dim); }));
    if (sums_workspace(fine.n, fine.rows, fine.dim)) EXPECT(MG_ERR_CAPACITY, sums([](S& a) { a.bytes = sums_workspace(a.n, a.rows, a.dim) - 1; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.into = 3; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.into = -1; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.dd = 4; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.od = 4; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.dim = 0; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.out = a.d; }));
    EXPECT(MG_ERR_ARG, sums([&](S& a) { a.out = base + 64000 - 4; }));
    EXPECT(MG_OK, sums([&](S& a) { a.out = base + 64000; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.os = 12; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.order = nullptr; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.starts = nullptr; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.count = nullptr; }));
    EXPECT(MG_ERR_ARG, sums([](S& a) { a.scale = NAN; }));
    EXPECT(MG_ERR_ARG, sums([&](S& a) { a.ws = more + 4; }));
    EXPECT(MG_ERR_ARG, sums([&](S& a) { a.n = huge; }));
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
