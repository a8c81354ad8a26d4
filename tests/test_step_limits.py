"""The calls of a step with the largest numbers that their arguments hold, without a GPU: refused, or taken without an overflow; and what the compiler made of
the kernels."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2410_09426_amd import build
from test_cache_built import _private_bytes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVE = r"""
#include "flatquant.h"
#include <stdint.h>
#include <stdio.h>
#define CHECK(cond) do { if (!(cond)) { printf("line %d: %s\n", __LINE__, #cond); return 1; } } while (0)
int main(void) {
    char* far = (char*)0x10000000;      /* addresses that are never followed */
    fq_kv_cache cache = {(uint8_t*)far, (uint32_t*)(far + 0x1000000), (uint8_t*)(far + 0x2000000), (uint32_t*)(far + 0x3000000), 8, 16, 4, 4, 3};
    fq_kv_batch batch = {(int32_t*)(far + 0x4000000), (int32_t*)(far + 0x4001000), (int32_t*)(far + 0x4002000), 3, 5, 4, 4, INT64_MAX, INT64_MAX};
    fq_page_pool pool = {(int32_t*)(far + 0x5000000), (int64_t*)(far + 0x5100000), (int64_t*)(far + 0x5200000), 8};
    char *q = far + 0x8000000, *out = far + 0x8100000, *work = far + 0x10000000;
    /* something at the end of every call is not aligned: it ends before a device is touched */
    int32_t* odd = (int32_t*)(far + 0x6000001);
#define ADVANCE() flatquant_cache_advance(&batch, &pool, 16, 8, odd, (int32_t*)(far + 0x6100000), (int32_t*)(far + 0x6200000), 0, 0, 0)
    CHECK(ADVANCE() == FQ_MISALIGNED);
    pool.capacity = INT32_MAX;
    CHECK(ADVANCE() == FQ_MISALIGNED);
    pool.capacity = INT64_MAX;
    CHECK(ADVANCE() == FQ_UNSUPPORTED_SHAPE);
    pool.capacity = 8;
    for (int k = 47; k < 63; ++k) {
        batch.table_stride = (int64_t)1 << k;
        CHECK(ADVANCE() == FQ_UNSUPPORTED_SHAPE);
    }
    batch.table_stride = ((int64_t)1 << 48) / 3;
    CHECK(ADVANCE() == FQ_MISALIGNED);
    batch.B = 0xffffff;
    CHECK(ADVANCE() == FQ_UNSUPPORTED_SHAPE);
    batch.table_stride = 1 << 20;
    batch.table_width = 1 << 20;
    batch.T = 1 << 29;
    CHECK(ADVANCE() == FQ_MISALIGNED);
    CHECK(flatquant_cache_advance(&batch, &pool, 16, INT64_MAX, odd, odd, odd, 0, 0, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(flatquant_cache_advance(&batch, &pool, INT32_MAX, 8, odd, odd, odd, 0, 0, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(flatquant_cache_advance(&batch, &pool, INT32_MIN, 8, odd, odd, odd, 0, 0, 0) == FQ_INVALID_ARG);
    batch.T = INT64_MAX;
    CHECK(ADVANCE() == FQ_UNSUPPORTED_SHAPE);
    /* rope: counts, strides */
#define ROPE(Hq, sq, T, per) flatquant_head_rope(q, sq, Hq, 0, 0, 0, T, (int32_t*)(far + 0x6000002), (uint64_t*)far, 128, 0, 0, 0, 1.0f, 0, 0, per, out + ((int64_t)1 << 52), sq, 0, 0, 0)
    CHECK(ROPE(65535, 65535 * 128, 32000, 0) == FQ_MISALIGNED);
    CHECK(ROPE(65535, 65535 * 128, 1 << 29, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(INT32_MAX, INT64_MAX, 1, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(32768, 32768 * 128, 1, 1) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(3, (int64_t)1 << 40, 256, 0) == FQ_MISALIGNED);
    CHECK(ROPE(3, ((int64_t)1 << 40) + 8, 256, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(3, INT64_MAX - 7, 1 << 29, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(3, 384, INT64_MAX, 0) == FQ_UNSUPPORTED_SHAPE);
    CHECK(ROPE(INT32_MIN, 384, 5, 0) == FQ_INVALID_ARG);
    CHECK(flatquant_head_rope(q, 384, 3, 0, 0, 0, 5, (int32_t*)far, (uint64_t*)far, INT32_MIN, 0, 0, 0, 1.0f, 0, 0, 0, out, 384, 0, 0, 0) == FQ_INVALID_ARG);
    CHECK(flatquant_head_rope(q, 384, 3, 0, 0, 0, 5, (int32_t*)far, (uint64_t*)far, INT32_MAX, 0, 0, 0, 1.0f, 0, 0, 0, out, 384, 0, 0, 0) == FQ_UNSUPPORTED_SHAPE);
    /* attention: what the call checks by itself before the checks that all attention has */
    batch.B = 3; batch.T = 5; batch.table_width = batch.table_stride = 4;
#define SCORED(Hq, so, bytes) flatquant_cache_scored_attention(&cache, &batch, q + 8, so, Hq, 0.1f, 3e38f, (float*)(far + 0x6000000), (int32_t*)(far + 0x7000000), INT32_MAX, INT32_MAX, 0, out, so, work, bytes, 0)
    CHECK(SCORED(8, 1024, INT64_MAX) == FQ_MISALIGNED);
    CHECK(SCORED(8, 1024, (int64_t)1 << 40) == FQ_MISALIGNED);
    CHECK(SCORED(INT32_MAX - 3, 1024, 1) == FQ_INVALID_ARG);
    CHECK(SCORED(1 << 24, INT64_MAX, INT64_MAX) != FQ_OK);
    CHECK(SCORED(INT32_MIN, INT64_MIN, INT64_MIN) == FQ_INVALID_ARG);
    batch.T = 1 << 29;
    CHECK(SCORED(8, 1024, (int64_t)1 << 40) == FQ_UNSUPPORTED_SHAPE);
    batch.T = 1 << 28; batch.B = 0x3fffff;
    CHECK(SCORED(4, ((int64_t)1 << 20) - 8, (int64_t)1 << 60) != FQ_OK);
    batch.B = INT64_MAX; batch.T = INT64_MAX;
    CHECK(SCORED(8, 1024, 1) == FQ_UNSUPPORTED_SHAPE);
    double f[2] = {1e308, -1e308};
    uint64_t turns[2];
    CHECK(fq_rope_turns(f, 2, turns) == FQ_OK && fq_rope_turns(f, INT32_MIN, turns) == FQ_INVALID_ARG);
    puts("ok");
    return 0;
}
"""


def test_largest_numbers_under_the_undefined_behaviour_sanitizer(tmp_path):
    """The argument checks compiled for the host with the sanitizer (the kernels' objects are the library's own).  No call gets past them."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    clang = "/opt/rocm/lib/llvm/bin/clang"
    objs = [os.path.join(build.CSRC, s.replace(".hip", ".o")) for s in build.SOURCES if s != "fq_api.hip"]
    if not (os.path.exists(hipcc) and os.path.exists(clang) and all(map(os.path.exists, objs))):
        pytest.skip("needs hipcc, its clang and the library's object files (python -m paper_2410_09426_amd.build)")
    api = tmp_path / "fq_api.o"
    subprocess.run([hipcc, "-O1", "-g", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-w", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
                    "-c", os.path.join(build.CSRC, "fq_api.hip"), "-o", str(api)], check=True, capture_output=True)
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-w", "-fno-gpu-sanitize", "-Xarch_host", "-fsanitize=undefined", str(api), *objs,
                    "-o", str(tmp_path / "libflatquant_limits.so")], check=True, capture_output=True)
    (tmp_path / "drive.c").write_text(DRIVE)
    subprocess.run([clang, "-std=c99", "-g", "-w", "-fsanitize=undefined", "-I", os.path.join(ROOT, "include"), str(tmp_path / "drive.c"),
                    "-o", str(tmp_path / "drive"), "-L", str(tmp_path), "-lflatquant_limits", f"-Wl,-rpath,{tmp_path}"], check=True, capture_output=True)
    r = subprocess.run([str(tmp_path / "drive")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout[-2000:] + r.stderr[-4000:]


def test_kernels_keep_no_array_in_memory(tmp_path):
    """Where 8 or 16 waves share the registers a few values that the loop does not touch may be spilled; nothing else lies in memory."""
    for source, names in (("fq_advance.hip", ("advance_kernel", "advance_rows_kernel")), ("fq_rope.hip", ("rope_kernel", "rope_matrix_kernel", "rope_matrix_few_kernel"))):
        kernels = _private_bytes(tmp_path, source)
        assert all(any(n in k for k in kernels) for n in names) and not any(kernels.values()), kernels
    kernels = _private_bytes(tmp_path, "fq_scored_attention.hip")
    for name in ("whole_attention_kernel", "balanced_attention_kernel", "shared_attention_kernel"):
        assert sum(name in k for k in kernels) >= 18, name
    for k, used in kernels.items():
        crowded = re.search(r"whole_attention_kernelILi(\d)ELi(\d)ELi1ELi(8|16)E", k)
        assert used == 0 or (crowded and used <= 24), (k, used)
