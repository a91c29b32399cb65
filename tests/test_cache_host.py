"""Host side of the paged cache (lr_cache_api.cu) against a fake CUDA runtime: what is ordered before what, and what an error leaves.

The fake keeps device memory on the host and counts the device work that nothing has waited for.  Its launch of the
chunk kernel can do what one does that ran into its limit of a wait: a count of finished parts stays.
"""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2607_18253_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNTIME = r"""
#include <cstdlib>
#include <cstring>
static int pending;
extern "C" {
int fake_pending() { return pending; }
int cudaMalloc(void **p, size_t n) { return (*p = std::malloc(n)) ? 0 : 2; }
int cudaFree(void *p) { std::free(p); return 0; }
int cudaMemset(void *p, int v, size_t n) { std::memset(p, v, n); ++pending; return 0; }
int cudaMemsetAsync(void *p, int v, size_t n, void *) { std::memset(p, v, n); ++pending; return 0; }
int cudaMemcpy(void *d, const void *s, size_t n, int) { std::memcpy(d, s, n); ++pending; return 0; }
int cudaMemcpyAsync(void *d, const void *s, size_t n, int, void *) { std::memcpy(d, s, n); ++pending; return 0; }
int cudaStreamSynchronize(void *) { pending = 0; return 0; }
int cudaDeviceSynchronize() { pending = 0; return 0; }
int cudaGetDevice(int *d) { *d = 0; return 0; }
int cudaDeviceGetAttribute(int *v, int, int) { *v = 4; return 0; }
const char *cudaGetErrorString(int) { return "fake"; }
void **__cudaRegisterFatBinary(void *) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
char __cudaInitModule(void **) { return 1; }
}
"""

LAUNCHES = r"""
#include "latency_router.h"
#include "lr_cache.cuh"
static int give_up, record;
extern "C" void fake_chunk(int status, int gives_up) { record = status; give_up = gives_up; }
namespace lr {
static uint32_t *counts;
cudaError_t launch_cache_write(const RwLaunch &, bool, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_cache_read(const RwLaunch &, bool, int, bool, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_attend_step(const AttendLaunch &, bool, int, int, int, cudaStream_t) { return cudaSuccess; }
cudaError_t attend_step_init() { return cudaSuccess; }
cudaError_t attend_chunk_init() { return cudaSuccess; }
int attend_step_ctas(int sms) { return 4 * sms; }
int encode_maps(const CacheDev &, bool, CacheMaps &m) { return m.box = 0; }
cudaError_t launch_attend_chunk(const AttendLaunch &a, const CacheMaps &, bool, int, int, cudaStream_t) {
    counts = a.done;
    if (record && !*a.c.status) *a.c.status = record;  // as the kernels: the first error stays
    if (give_up) {
        a.done[3] = 1;
        if (!*a.c.status) *a.c.status = LR_ECUDA;
    }
    return cudaSuccess;
}
}
extern "C" unsigned fake_count() { return lr::counts ? lr::counts[3] : ~0u; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    nvcc = build._nvcc()
    if not (os.path.exists(nvcc) or shutil.which(nvcc)):
        pytest.skip("no nvcc")
    at = tmp_path_factory.mktemp("fake")
    (at / "launches.cu").write_text(LAUNCHES)
    (at / "runtime.cpp").write_text(RUNTIME)
    out = str(at / "libfake.so")
    r = subprocess.run([nvcc, "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", *build.ARCH, "-cudart", "none", "-shared",
                        "-Xlinker", "-Bsymbolic", "-I", build.INCLUDE, "-I", build.CSRC, "-o", out, os.path.join(build.CSRC, "lr_cache_api.cu"), str(at / "launches.cu"), str(at / "runtime.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    so = ctypes.CDLL(out)
    P = ctypes.c_void_p
    so.lr_cache_attend.argtypes = [P, P, ctypes.c_int32, P, ctypes.c_int64, ctypes.c_int64, ctypes.c_float, ctypes.c_int32,
                                   ctypes.c_int32, P, ctypes.c_int64, ctypes.c_int64, P, P]
    so.lr_cache_status.argtypes = [P, P]
    so.lr_cache_destroy.argtypes = [P]
    return so


@pytest.fixture
def cache(lib):
    from paper_2607_18253_gb300 import router as R
    cfg = R._CacheConfig(8, 2, 64, 0, 0, 16, 4, 4, 1 << 20, 1 << 21, None, None, 2048, 128, 64, 0, 0, 0)
    h = ctypes.c_void_p()
    assert lib.lr_cache_create(ctypes.byref(cfg), ctypes.byref(h)) == R.LR_OK
    yield h
    lib.fake_chunk(0, 0)
    assert lib.lr_cache_destroy(h) == R.LR_OK


def attend(lib, h):
    from paper_2607_18253_gb300 import router as R
    b = R._CacheBatch(1, 64, 16, 16, 16, 4, 4)
    assert lib.lr_cache_attend(h, ctypes.byref(b), 64, 16, 512, 64, 0.125, 0, 0, 16, 512, 64, None, None) == R.LR_OK


def test_a_new_handle_is_ready_on_every_stream(lib, cache):
    # counts and status word are set by work of the default stream, which streams that do not block on it would not wait for
    assert lib.fake_pending() == 0


@pytest.mark.parametrize("earlier", [0, 1])
def test_counts_start_again_after_a_launch_that_gave_up(lib, cache, earlier):
    # the word keeps the first error, an earlier LR_EINVAL too
    from paper_2607_18253_gb300 import router as R
    if earlier:
        lib.fake_chunk(R.LR_EINVAL, 0)
        attend(lib, cache)
    lib.fake_chunk(0, 1)
    attend(lib, cache)
    assert lib.fake_count() == 1
    assert lib.lr_cache_status(cache, None) == (R.LR_EINVAL if earlier else R.LR_ECUDA)
    assert lib.fake_count() == 0
    assert lib.lr_cache_status(cache, None) == R.LR_OK
