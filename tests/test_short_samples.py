"""Group norm over many short samples whose rows are wide or cut by alignment: values and gradients against the definition in 64 bits, and the memory that a
call asks for, which goes by the blocks that work on it and not by the samples."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import api, build
from test_between_layers import ACTS, HOST, TYPES, check_norm, ctx, rows_of  # noqa: F401


def workspace(ctx, rows, channels, groups, dtype, per_sample, backward, offsets=None):
    spec = api.NormSpec(rows, channels, groups, api.ROW_TYPES[TYPES[dtype]], 0, 1e-5, len(offsets) - 1 if offsets is not None else 0,
                        offsets.ctypes.data if offsets is not None else None, per_sample, None, None, None)
    need = C.c_size_t(0)
    ctx._check(ctx.lib.mg_group_norm_workspace(ctx.handle, C.byref(spec), backward, C.byref(need)))
    return need.value


# matrices of 0.1 to 1.6 GB.  Sums by channel of a few blocks in each of 148 multiprocessors: below 50 MB; what goes by the sample would be 8 bytes a
# channel of each, up to four times the matrix
@pytest.mark.gpu
@pytest.mark.parametrize("rows,per,channels,groups,dtype", [(200_000, 1, 2048, 32, "f32"), (200_000, 1, 4096, 32, "f16"), (131_072, 1, 1280, 32, "f16"), (131_072, 2, 1024, 32, "f16"),
                                                            (131_072, 2, 512, 32, "f16"), (100_000, 4, 512, 512, "f32"), (96_000, 16, 4096, 32, "f16")])
def test_what_a_call_asks_for(ctx, rows, per, channels, groups, dtype):  # noqa: F811
    for backward in (0, 1):
        assert workspace(ctx, rows, channels, groups, dtype, per, backward) < 50_000_000


# more samples than six for each of 148 multiprocessors: single rows of one run of channels and of many, of every vector width, with groups that a run's
# end cuts; several rows; more groups than a block's shared memory has room for
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels,groups,pad,shift", [(1000, 2048, 32, 0, 0), (950, 4104, 3, 0, 0), (901, 2001, 1, 0, 0), (1300, 1028, 257, 0, 4), (905, 4098, 2, 3, 1), (889, 1025, 5, 0, 0), (920, 6000, 6000, 0, 0)])
def test_wide_rows(ctx, dtype, rows, channels, groups, pad, shift):  # noqa: F811
    x = rows_of(rows, channels, TYPES[dtype], 3, pad, shift)
    i = (rows + channels) % 4
    drop = (None, mg.Dropout(0.5, 3, 1), mg.Dropout(0.2, 4, row_keys=torch.randint(0, 2**40, (rows,)).cuda()), None)[i]
    check_norm(ctx, x, "rows", groups, ACTS[(i + channels // 2) % 4], drop)
    check_norm(ctx, x, "rows", groups, "relu", mg.Dropout(0.4, 6))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("channels,groups,pad,shift", [(602, 2, 0, 0), (300, 300, 0, 0), (1030, 2, 0, 0), (2048, 8, 8, 0), (515, 5, 0, 1)])
def test_short_samples(ctx, dtype, channels, groups, pad, shift):  # noqa: F811
    samples = ([3, 0, 1, 7, 15, 0, 16, 2] * 120)[:-3] + [0, 0]
    x = rows_of(sum(samples) + 2, channels, TYPES[dtype], 3, pad, shift)
    x[-2:] = float("nan")
    i = (channels + groups) % 4
    for drop in (None, mg.Dropout(0.3, 9, row_keys=torch.randint(0, 2**40, (len(x),)).cuda())):
        first = check_norm(ctx, x, samples, groups, ACTS[i], drop)
    for a, b in zip(first, check_norm(ctx, x, samples, groups, ACTS[i], drop)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_more_blocks_than_samples_with_rows(ctx):  # noqa: F811
    samples = [0] * 1000 + [5, 0, 9]
    check_norm(ctx, rows_of(14, 1100, torch.float32, 3), samples, 11, "silu", mg.Dropout(0.3, 9))
    check_norm(ctx, rows_of(14, 1100, torch.float32, 3), [0] * 1000, 11, "silu")


@pytest.mark.gpu
def test_in_place_and_captured(ctx):  # noqa: F811
    x, how = rows_of(5 * 1000, 1100, torch.float16, 3).view(1000, 5, 1100), dict(activation="gelu", dropout=mg.Dropout(0.4, 6))
    d_y = rows_of(5 * 1000, 1100, torch.float16, 9).view(1000, 5, 1100)
    y, mean, rstd = ctx.group_norm(x, 11, **how)
    grads = ctx.group_norm_backward(d_y, x, mean, rstd, 11, **how)
    inout = x.clone()
    ctx.group_norm(inout, 11, out=inout, **how)
    assert torch.equal(inout, y)
    for given in (d_y.clone(), x.clone()):
        got = ctx.group_norm_backward(given if torch.equal(given, d_y) else d_y, given if torch.equal(given, x) else x, mean, rstd, 11, out=given, **how)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ctx.group_norm(x, 11, **how)
        held = (*held, *ctx.group_norm_backward(d_y, x, held[1], held[2], 11, **how))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, (y, mean, rstd, *grads)))


# bad values stay in their sample and group, in runs that share the group and runs that do not
@pytest.mark.gpu
def test_bad_values(ctx):  # noqa: F811
    x = rows_of(950, 4101, torch.float32, 3)[:, :4098]      # single elements, runs of 256
    clean = x.clone()
    x[5, 2000], x[650, 4097] = float("nan"), float("inf")
    got, want = ctx.group_norm(x, 6), ctx.group_norm(clean, 6)
    bad = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
    bad[5, 1366:2049] = bad[650, 3415:] = True
    assert torch.equal(got[0][~bad], want[0][~bad]) and bool(got[0][bad].isnan().all())
    a, b = (ctx.group_norm_backward(torch.ones_like(x), v, s[1], s[2], 6) for v, s in ((x, got), (clean, want)))
    assert torch.equal(a[0][~bad], b[0][~bad]) and bool(a[0][bad].isnan().all())


# every array that the plan lays out lies in what the call asks for, at every alignment, and that has a bound of its own
PLANS = HOST[:HOST.index("int main")] + r"""
#include <random>
int main() {
    std::mt19937 rng(1);
    const auto pick = [&](int64_t lo, int64_t hi) { return (int64_t)std::exp(std::uniform_real_distribution<double>(std::log((double)lo), std::log(hi + 0.99))(rng)); };
#define NEED(x) do { if (!(x)) { printf("line %d: %s (rows %lld channels %d groups %d samples %lld dtype %d backward %d vec %d)\n", __LINE__, #x, (long long)s.rows, s.channels, s.groups, (long long)n, s.dtype, backward, v); return 1; } } while (0)
    std::vector<int64_t> ends;
    int wide = 0;
    for (int i = 0; i < 40000; ++i) {
        mg_norm_spec s{};
        s.groups = (int)pick(1, i % 3 ? 64 : 3000); s.channels = s.groups * (int)pick(1, i % 50 ? 300 : 5000); s.dtype = (int)(rng() % 3); s.eps = 1.f;
        s.rows_per_sample = pick(1, 20);
        s.rows = s.rows_per_sample * pick(500, 1'000'000);
        if (s.rows >= 1ll << 31) continue;
        if (rng() % 2) {
            s.n_samples = (int)pick(500, MG_MAX_BATCHES);
            ends.assign(1, 0);
            for (int k = 0; k < s.n_samples; ++k) ends.push_back(ends.back() + (int64_t)(rng() % 17));
            s.rows = ends.back() + 1;
            s.sample_offsets = ends.data();
        }
        const int backward = rng() % 2;
        const int64_t n = sample_count(&s);
        int v = 0;
        if (norm_mode(&s) != NORM_TILES || !short_samples(&s, 148)) continue;
        const size_t have = call_workspace(&s, 148, backward);
        NEED(have <= 16 * 8ull * s.channels * 2 + (2ull * 128 << 20) + (1 << 20) && (backward || have <= 8ull * (MG_MAX_BATCHES + 2)));
        for (const int* at = vec_widths(s.dtype); *at; ++at) {
            v = *at;
            if (s.channels % v) continue;
            NormPlan p;
            TileArgs a;
            plan_samples(&s, 148, backward, v, &p, &a);
            NEED(p.bytes <= have && p.block_grid >= 1 && a.samples == n && a.tiles == 0);
            if (p.cluster) continue;
            ++wide;
            NEED(p.block_grid <= n && p.cleared == 0 && a.results.tx <= 8 && a.run <= v * 256 && (a.run == s.channels || a.run % v == 0) && a.run <= (v << a.results.tx));
            NEED(!s.sample_offsets || p.at_table + 8ull * (n + 1) <= p.at_group_parts);
            NEED(!backward || (p.n_parts == p.block_grid && p.n_parts <= 1024 && p.at_group_parts + 8ull * p.block_grid * s.groups <= p.at_parts && p.at_parts + 8ull * p.n_parts * s.channels <= p.bytes));
        }
    }
    return wide < 1000;
}
"""


def test_plans_on_the_host(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    source, program = tmp_path / "host.cu", str(tmp_path / "host")
    source.write_text(PLANS)
    made = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xcompiler", "-w", "-I", build.CSRC,
                           "-I", os.path.join(build.ROOT, "include"), str(source), "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([program], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
