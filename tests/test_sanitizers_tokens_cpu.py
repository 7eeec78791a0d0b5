"""The host code of the operators over tokens and a vocabulary (validation, plans, workspace sizes, launch set-up) under AddressSanitizer and
UndefinedBehaviorSanitizer with launches stubbed: every entry point over a sweep of sizes, valid and invalid.  CPU only."""
import os
import subprocess
import tempfile

import pytest

from test_sanitizers_cpu import CSRC, HIPCC, ROOT, SAN_ENV, _run

DRIVER = r'''
#include "ngconv.h"
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
static unsigned long long st = 0x9E3779B97F4A7C15ull;
static unsigned long long rnd64(void) { st ^= st << 13; st ^= st >> 7; st ^= st << 17; return st; }
/* a size spread over its logarithm, now and then a border or something out of range */
static long long size(int bits)
{
    static const long long odd[] = {0, -1, 1, 0x7fffffffll, 0x80000000ll, 1ll << 40, -(1ll << 31), (1ll << 20) - 1, 1ll << 21};
    if (rnd64() % 12 == 0) return odd[rnd64() % 9];
    return 1 + (long long)(rnd64() >> (64 - 1 - rnd64() % bits));
}
int main(void)
{
    setenv("NGC_DRY_RUN", "1", 1);
    ngc_reload_switches();
    char *p = (char *)(size_t)0x7000000000;                      /* never dereferenced: nothing is launched */
    const size_t big = (size_t)1 << 60;
    long ok = 0, calls = 0;
    for (int it = 0; it < 60000; ++it) {
        const int dt = (int)(rnd64() % 13 == 0 ? rnd64() % 5 - 1 : rnd64() % 2);
        const long long rows = size(it % 3 ? 14 : 31), wide = size(it % 3 ? 13 : 31), many = size(it % 3 ? 17 : 31);
        const int w = (int)(wide > 0x7fffffff ? -1 : wide), v = (int)(many > 0x7fffffff ? -1 : many), off = rnd64() % 4 ? 0 : 4;
        void *a = p + off;
        float *f = (float *)(p + off);
        int64_t *ids = (int64_t *)p;
        const size_t need[4] = {ngc_embedding_workspace_bytes(rows, v, w), ngc_layer_norm_workspace_bytes(dt, rows, w),
                                ngc_linear_xent_workspace_bytes(dt, rows, w, v, 0), ngc_linear_xent_workspace_bytes(dt, rows, w, v, 1)};
        int rc[16], n = 0;
        rc[n++] = ngc_embedding(dt, rows, v, w, 2.f, a, ids, a, 0);
        rc[n++] = ngc_embedding_bwd(dt, rows, v, w, 2.f, a, ids, f, p, need[0], 0);
        rc[n++] = ngc_layer_norm(dt, rows, w, it % 50 ? 1e-5f : nanf(""), a, f, it % 3 ? f : NULL, a, it % 4 ? f : NULL, f, 0);
        rc[n++] = ngc_layer_norm_bwd(dt, rows, w, a, it % 3 ? f : NULL, f, f, a, a, it % 4 ? f : NULL, f, p, need[1], 0);
        rc[n++] = ngc_linear_xent(dt, rows, w, v, a, a, ids, f, f, p, need[2], 0);
        rc[n++] = ngc_linear_xent_bwd(dt, rows, w, v, a, a, ids, f, f, it % 5 ? a : NULL, a, p, need[3], 0);
        for (int i = 0; i < n; ++i, ++calls) ok += rc[i] == NGC_OK;
        /* one byte less than needed is refused */
        if (rc[1] == NGC_OK && ngc_embedding_bwd(dt, rows, v, w, 2.f, a, ids, f, p, need[0] - 1, 0) != NGC_WORKSPACE_TOO_SMALL) return 3;
        if (rc[4] == NGC_OK && ngc_linear_xent(dt, rows, w, v, a, a, ids, f, f, p, need[2] - 1, 0) != NGC_WORKSPACE_TOO_SMALL) return 4;
        if (rc[5] == NGC_OK && ngc_linear_xent_bwd(dt, rows, w, v, a, a, ids, f, f, a, a, p, need[3] - 1, 0) != NGC_WORKSPACE_TOO_SMALL) return 5;
        if (need[2] > big || need[3] > big) return 6;
    }
    printf("tokens clean: %ld calls, %ld accepted\n", calls, ok);
    return ok > 20000 ? 0 : 7;
}
'''


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_host_code_is_clean_under_asan_and_ubsan_with_launches_stubbed():
    from concurrent.futures import ThreadPoolExecutor
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    with tempfile.TemporaryDirectory() as td:
        def compile_one(name):
            obj = os.path.join(td, name.replace(".hip", ".o"))
            _run([HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-fPIC", "-Wno-unused-command-line-argument",
                  "-Wno-inline-asm", "-Wno-unknown-cuda-version", *san, "-c", os.path.join(CSRC, name), "-o", obj], timeout=600)
            return obj

        with ThreadPoolExecutor(max_workers=5) as ex:
            objs = list(ex.map(compile_one, ["api_tokens.hip", "embedding.hip", "layer_norm.hip", "linear_xent.hip", "switches.hip"]))
        drv, drv_o, stub, stub_o, exe = (os.path.join(td, n) for n in ("drv.c", "drv.o", "images.c", "images.o", "drv"))
        with open(drv, "w") as f:
            f.write(DRIVER)
        clang = "/opt/rocm/lib/llvm/bin/clang"
        _run([clang, "-O1", "-g", "-D_GNU_SOURCE", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"),
              "-c", drv, "-o", drv_o], timeout=300)
        # each host-only object registers a device image: an empty one will do, nothing is launched
        images = sorted({sym for sym in _run(["nm", "-u", *objs]).stdout.split() if sym.startswith("__hip_fatbin_")})
        with open(stub, "w") as f:
            f.write("".join(f"const unsigned char {sym}[4096] __attribute__((aligned(4096))) = {{0}};\n" for sym in images))
        _run([clang, "-c", stub, "-o", stub_o])
        _run([HIPCC, "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", exe, drv_o, stub_o, *objs], timeout=600)
        r = subprocess.run([exe], env={**os.environ, **SAN_ENV, "NGC_DRY_RUN": "1"}, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0 and "tokens clean" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
