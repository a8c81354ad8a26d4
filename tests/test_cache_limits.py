"""The paged key/value cache's calls with the largest numbers that their arguments hold, without a GPU: refused, or taken without an overflow."""
import glob
import os
import shutil
import subprocess

import pytest

from paper_2410_09426_amd import binding as fq
from paper_2410_09426_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LLVM = "/opt/rocm/lib/llvm/bin"

DRIVE = r"""
#include "flatquant.h"
#include <stdint.h>
#include <stdio.h>
#define CHECK(cond) do { if (!(cond)) { printf("line %d: %s\n", __LINE__, #cond); return 1; } } while (0)
int main(void) {
    char* far = (char*)0x10000000;      /* addresses that are never followed */
    fq_kv_cache cache = {(uint8_t*)far, (uint32_t*)(far + 0x1000000), (uint8_t*)(far + 0x2000000), (uint32_t*)(far + 0x3000000), 8, 16, 4, 4, 3};
    fq_kv_batch batch = {(int32_t*)(far + 0x4000000), (int32_t*)(far + 0x4001000), (int32_t*)(far + 0x4002000), 3, 5, 4, 4, INT64_MAX, INT64_MAX};
    char *q = far + 0x8000000, *out = far + 0x8100000, *work = far + 0x10000000;
    int64_t need = fq_cache_attention_workspace(&cache, &batch, 8);
    CHECK(need >= 0);
    /* hints of any size; a query that is not aligned ends the call before a device is touched */
    for (int window = 0; window <= 100; window += 100) {
        CHECK(flatquant_cache_attention(&cache, &batch, q + 8, 1024, 8, 0.1f, window, 3, out, 1024, work, need, 0) == FQ_MISALIGNED);
        CHECK(flatquant_cache_attention(&cache, &batch, q + 8, 1024, 8, 0.1f, window ? INT32_MAX : 0, INT32_MAX, out, 1024, work, need, 0) == FQ_MISALIGNED);
    }
    batch.max_rows = 64;
    need = fq_cache_attention_workspace(&cache, &batch, 8);
    CHECK(flatquant_cache_tree_attention(&cache, &batch, q + 8, 1024, 8, 0.1f, (uint64_t*)(far + 0x9000000), out, 1024, work, need, 0) == FQ_MISALIGNED);
    /* rows of the page table that lie further apart than memory goes */
    for (int k = 47; k < 63; ++k) {
        batch.table_stride = (int64_t)1 << k;
        CHECK(flatquant_cache_write(&cache, &batch, q, 512, out, 512, 0, 0, 1, 0.9f, 0.9f, 0) == FQ_UNSUPPORTED_SHAPE);
        CHECK(flatquant_cache_read(&cache, &batch, q, 512, out, 512, 0) == FQ_UNSUPPORTED_SHAPE);
        CHECK(flatquant_cache_attention(&cache, &batch, q, 1024, 8, 0.1f, 0, 0, out, 1024, work, need, 0) == FQ_UNSUPPORTED_SHAPE);
    }
    batch.table_stride = INT64_MAX;
    CHECK(flatquant_cache_read(&cache, &batch, q, 512, out, 512, 0) == FQ_UNSUPPORTED_SHAPE);
    batch.B = 1;                        /* of one sequence the distance means nothing */
    CHECK(flatquant_cache_read(&cache, &batch, q + 8, 512, out, 512, 0) == FQ_MISALIGNED);
    CHECK(flatquant_cache_read(&cache, &batch, cache.k_codes, 512, out, 512, 0) == FQ_INVALID_ARG);
    printf("limits ok\n");
    return 0;
}
"""


def test_largest_numbers_under_the_undefined_behaviour_sanitizer(tmp_path):
    """The argument checks compiled with -fsanitize=undefined (host pass only; the kernels' objects are the library's own).  No call gets past them."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    objs = [o for o in glob.glob(os.path.join(build.CSRC, "*.o")) if os.path.basename(o) != "fq_api.o"]
    if not (os.path.exists(hipcc) and os.path.exists(LLVM + "/clang")) or len(objs) < 5:
        pytest.skip("needs hipcc, its clang and the library's object files (python -m paper_2410_09426_amd.build)")
    api = tmp_path / "fq_api.o"
    subprocess.run([hipcc, "-O1", "-g", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-w", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
                    "-c", os.path.join(build.CSRC, "fq_api.hip"), "-o", str(api)], check=True, capture_output=True)
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-w", "-fno-gpu-sanitize", "-fsanitize=undefined", str(api), *objs,
                    "-o", str(tmp_path / "libflatquant_limits.so")], check=True, capture_output=True)
    (tmp_path / "drive.c").write_text(DRIVE)
    subprocess.run([LLVM + "/clang", "-std=c99", "-g", "-w", "-fsanitize=undefined", "-I", os.path.join(ROOT, "include"), str(tmp_path / "drive.c"),
                    "-o", str(tmp_path / "drive"), "-L", str(tmp_path), "-lflatquant_limits", f"-Wl,-rpath,{tmp_path}"], check=True, capture_output=True)
    r = subprocess.run([str(tmp_path / "drive")], capture_output=True, text=True)
    assert r.returncode == 0 and "limits ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def test_page_table_rows_too_far_apart_are_refused():
    """Whatever else is asked for, nothing to do included."""
    cache = fq.KvCache(*[4096 * k for k in range(1, 5)], 8, 16, 4, 4, 3)
    for B, stride, want in ((2, 2 ** 47, fq.FQ_OK), (2, 2 ** 47 + 1, fq.FQ_UNSUPPORTED_SHAPE), (3, 2 ** 62, fq.FQ_UNSUPPORTED_SHAPE), (1, 2 ** 62, fq.FQ_OK)):
        batch = fq.KvBatch(4096, 4096, 4096, B, 0, 4, stride, 1, 64)
        assert fq.flatquant_cache_read(cache, batch, 4096, 512, 4096, 512, check=False) == want, (B, stride)
