"""Gradients of looked-up rows where ids are many: how the sorted places are cut, and how exact the sums stay."""
import os
import shutil
import subprocess

import pytest

from paper_2202_02365_b200 import build

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


def run_on_the_host(tmp_path, program):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    source, out = tmp_path / "host.cu", str(tmp_path / "host")
    source.write_text(program)
    made = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O0", "-Xcompiler", "-w", "-I", build.CSRC,
                           "-I", os.path.join(build.ROOT, "include"), str(source), "-o", out], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([out], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout


def test_every_place_is_in_one_of_few_chunks(tmp_path):
    run_on_the_host(tmp_path, PLANS)
