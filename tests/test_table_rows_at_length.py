"""Gradients of looked-up rows where ids are many: how the sorted places are cut, and how exact the sums stay."""
import dataclasses
import os
import shutil
import subprocess
import types

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import build
from test_table_rows import check_sums, ctx  # noqa: F401

# ---- how a call is cut, on the host ---------------------------------------------------------------------------------
PLANS = r"""
#include <cstdarg>
#include <cstdio>
#include "mg_rows_plan.cuh"
int mg_fail(mg_ctx*, int code, const char*, ...) { return code; }
int mg_cuda_fail(mg_ctx*, cudaError_t, const char*) { return MG_ERR_CUDA; }
void mg_prof_begin(mg_ctx*, int) {}
void mg_prof_end(mg_ctx*, int, int64_t) {}

int main() {
    int bad = 0;
    const int64_t most = (1ll << 31) - 2;
    for (const int sms : {8, 148})
        for (const int32_t dim : {1, 16, 17, 33, 64, 100, 256, 300, 4100, 70'000, 1 << 22})
            for (const int64_t n : {(int64_t)1, (int64_t)15, (int64_t)16, (int64_t)17, (int64_t)131'071, (int64_t)131'073, (int64_t)139'263, (int64_t)1'000'003, (int64_t)33'000'000, (int64_t)1'000'000'007, most})
                for (const int64_t rows : {(int64_t)1, (int64_t)5'000'000, most}) {
                    const SumPlan p = plan_sums(n, rows, dim, sms);
                    const bool covers = p.chunk >= 1 && p.chunks >= 1 && (int64_t)p.chunk * p.chunks >= n && (int64_t)p.chunk * (p.chunks - 1) < n;
                    const bool room = p.chunks <= 8192 && p.at_begun == 8 * (size_t)p.chunks * p.pitch && p.bytes >= p.at_begun + 4 * (size_t)p.chunks && p.pitch >= dim;
                    if (!covers || !room) { printf("%lld places of %d, %d multiprocessors: chunks %d of %d\n", (long long)n, dim, sms, p.chunks, p.chunk); ++bad; }
                }
    return bad ? 1 : 0;
}
"""


def run_program(tmp_path, program):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    source, out = tmp_path / "program.cu", str(tmp_path / "program")
    source.write_text(program)
    made = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xcompiler", "-w", "-I", build.CSRC,
                           "-I", os.path.join(build.ROOT, "include"), str(source), "-o", out], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([out], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout


def test_every_place_is_in_one_of_few_chunks(tmp_path):
    run_program(tmp_path, PLANS)


def test_groups_of_another_device_are_refused():
    """Their addresses are read by kernels: before any call of the library."""
    here, there = torch.device("meta"), torch.device("cpu")
    ctx = types.SimpleNamespace(device=here)
    d_y = torch.empty(5, 4, device=here)
    some = lambda n, device: torch.empty(n, dtype=torch.int32, device=device)
    good = mg.IdGroups(some(5, here), some(5, here), some(3, here), some(4, here), some(1, here), 3)
    assert mg.Context._grouped(ctx, d_y, good, 3)[1] is good
    for field in ("order", "group_of", "ids", "starts", "count"):
        with pytest.raises(AssertionError):
            mg.Context._grouped(ctx, d_y, dataclasses.replace(good, **{field: getattr(good, field).new_empty(getattr(good, field).shape, device=there)}), 3)


# ---- on the GPU -----------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,stretches", [(100_000, 65_536, 1), (100_000, 65_536, 50), (40_000, 262_144, 2), (9000, 1 << 20, 3), (30_000_000, 16, 1), (3_000_001, 36, 2), (30_000_000, 16, 9000),
                                             (200_000, 3000, 3)])
def test_sums_of_many_places_stay_within_their_bound(ctx, n, dim, stretches):
    """One row over and over, of values whose fp32 sums are rounded the same way each time: a chain of some thousand additions is off by more than 512 roundings can be."""
    values = torch.tensor([1 + 0.9 * 2.0 ** -13, 0.1, 0.7, -0.1, 1 + 0.9 * 2.0 ** -14, 3.0], device="cuda")
    row = values[torch.arange(dim, device="cuda") % 6]
    n_rows = stretches + 3
    one_by_one = (torch.arange(n, device="cuda", dtype=torch.int32) % stretches) + 1      # (its places lie apart)
    ids = torch.where(torch.arange(n, device="cuda") % 1000 == 7, -1, one_by_one)
    ids[-1] = n_rows - 1                                                                  # an id of one place
    count = torch.bincount(ids[ids >= 0].long(), minlength=n_rows)
    for dtype in (torch.float32, torch.bfloat16):
        d_y = row.to(dtype).expand(n, dim)
        want = count[:, None].double() * d_y[0].double()
        got = ctx.embedding_backward(d_y, ids, n_rows, dtype=torch.float32)
        check_sums(got, want, want.abs(), count)
        assert not got[count == 0].any()
        distinct, rows = ctx.embedding_backward_rows(d_y, ids, n_rows, dtype=torch.float32)
        assert torch.equal(rows, got[distinct.long()])


# ---- kernels by themselves: what no call of the library makes happen ------------------------------------------------
COMMON = r"""
#include <cstdarg>
#include <cstdio>
#include <vector>
#include "mgdense.h"
#include "mg_rows_sums.cuh"
using namespace mgrows;

static int bad = 0;
#define EXPECT(is, what) do { if (!(is)) { printf("line %d: %s\n", __LINE__, what); ++bad; } } while (0)
template <typename T> static T* device(const std::vector<T>& v) {
    T* p = nullptr;
    cudaMalloc(&p, v.size() * sizeof(T));
    cudaMemcpy(p, v.data(), v.size() * sizeof(T), cudaMemcpyHostToDevice);
    return p;
}
template <typename T> static std::vector<T> host(const T* p, size_t n) {
    std::vector<T> v(n);
    cudaMemcpy(v.data(), p, n * sizeof(T), cudaMemcpyDeviceToHost);
    return v;
}

"""
JOIN = COMMON + r"""
// 5,000 chunks by one block, in several rounds: ids of two to forty shares, each of which begins in the chunk that the one before ends in.
static void join() {
    const int chunk = 16, chunks = 5000, dim = 128, spans[] = {2, 3, 40, 2, 5, 33, 2, 2};
    std::vector<float> shares((size_t)chunks * 2 * dim), want;
    std::vector<int32_t> begun(chunks, -1), starts;
    for (size_t i = 0; i < shares.size(); ++i) shares[i] = (float)(i / dim % 13 + 1);
    int first = 0;
    for (int g = 0;; ++g) {
        const int span = spans[g % 8];
        starts.push_back(first * chunk + 8);
        if (first + span > chunks) break;
        begun[first] = g;
        float sum = 0.f;
        for (int i = 0; i < span; ++i) sum += shares[((size_t)(first + i) * 2 + (i == 0)) * dim];
        want.push_back(sum);
        first += span - 1;
    }
    const int groups = (int)want.size();
    SumArgs a = {};
    a.n = (int64_t)chunks * chunk; a.n_rows = a.n; a.dim = dim; a.scale = 1.f; a.into = MG_ROWS_COMPACT; a.out_stride = dim; a.chunk = chunk; a.chunks = chunks; a.pitch = dim;
    a.starts = device(starts); a.shares = device(shares); a.begun = device(begun);
    float* out = device(std::vector<float>((size_t)groups * dim, -1.f));
    a.out = out;
    for (int t = 0; t < 20; ++t) {
        cudaMemset(out, 0xFF, sizeof(float) * groups * dim);
        k_join_shares<float><<<1, kJoinThreads>>>(a);
        const std::vector<float> got = host(out, (size_t)groups * dim);
        int wrong = 0;
        for (int g = 0; g < groups; ++g)
            for (int c = 0; c < dim; ++c) wrong += got[(size_t)g * dim + c] != want[g];
        EXPECT(wrong == 0, "shares");
    }
}

int main() {
    join();
    EXPECT(cudaDeviceSynchronize() == cudaSuccess, cudaGetErrorString(cudaGetLastError()));
    return bad ? 1 : 0;
}
"""


GROUPS = COMMON + r"""
// Groups of 3,000 sorted keys below 100 (`some`) or that are none: what is said of their number.
static int32_t groups(bool some, bool failed, int first_tile, int tiles, const std::vector<uint64_t>& told, int polls) {
    const int n = 3000, none = 100;
    std::vector<uint32_t> keys(n, none);
    if (some) for (int i = 0; i < n; ++i) keys[i] = i * none / n;
    SortShared shared = {};
    shared.failed = failed;
    shared.ticket[kMaxPasses] = first_tile;
    int32_t *ids = device(std::vector<int32_t>(none)), *starts = device(std::vector<int32_t>(none + 1)), *of = device(std::vector<int32_t>(n)), *count = device(std::vector<int32_t>(1, 12345));
    k_sort_groups<4><<<tiles, kSortThreads>>>(device(keys), n, none, device(std::vector<SortShared>(1, shared)), device(told), 0, ids, starts, of, count, polls);
    return host(count, 1)[0];
}

int main() {
    const std::vector<uint64_t> nothing(3, 0);
    EXPECT(groups(true, false, 0, 3, nothing, 1 << 20) == 100, "all is well");
    EXPECT(groups(false, false, 0, 3, nothing, 1 << 20) == 0, "no group");
    EXPECT(groups(true, true, 0, 3, nothing, 1 << 20) == -1, "the sort has failed");
    EXPECT(groups(false, true, 0, 3, nothing, 1 << 20) == -1, "the sort has failed, no key of a row came out of it");
    // the third tile by itself: the second has said how many it has, the first never says anything, which the second lane waits for
    EXPECT(groups(true, false, 2, 1, {0, kChainTag | kChainOwn | 34, 0}, 8) == -1, "a wait has run out");
    EXPECT(groups(true, false, 2, 1, {0, 0, 0}, 8) == -1, "a wait has run out");
    EXPECT(cudaDeviceSynchronize() == cudaSuccess, cudaGetErrorString(cudaGetLastError()));
    return bad ? 1 : 0;
}
"""


@pytest.mark.gpu
def test_shares_in_several_rounds(tmp_path):
    run_program(tmp_path, JOIN)


@pytest.mark.gpu
def test_a_wait_that_has_run_out_is_told(tmp_path):
    """On the device: waits of a few polls for a word that nobody writes."""
    run_program(tmp_path, GROUPS)
