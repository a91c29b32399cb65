"""What the calls on trees and kept tokens refuse before anything is launched (host side, against a fake CUDA runtime)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2607_18253_gb300 import build
from test_cache_host import LAUNCHES, RUNTIME

MORE = r"""
namespace lr {
static int launched;
cudaError_t launch_weigh(const WeighLaunch &, const CacheMaps &, bool, int, int, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_select(const SelectLaunch &, int, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_keep(const KeepLaunch &, int, int, cudaStream_t) { ++launched; return cudaSuccess; }
}
extern "C" int fake_launched() { return lr::launched; }
"""

I32, I64, F = ctypes.c_int32, ctypes.c_int64, ctypes.c_float


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    nvcc = build._nvcc()
    if not (os.path.exists(nvcc) or shutil.which(nvcc)):
        pytest.skip("no nvcc")
    at = tmp_path_factory.mktemp("fake")
    (at / "launches.cu").write_text(LAUNCHES + MORE)
    (at / "runtime.cpp").write_text(RUNTIME)
    out = str(at / "libfake.so")
    r = subprocess.run([nvcc, "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", *build.ARCH, "-cudart", "none", "-shared",
                        "-Xlinker", "-Bsymbolic", "-I", build.INCLUDE, "-I", build.CSRC, "-o", out, os.path.join(build.CSRC, "lr_cache_api.cu"),
                        os.path.join(build.CSRC, "lr_cache_tokens.cu"), str(at / "launches.cu"), str(at / "runtime.cpp")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    so = ctypes.CDLL(out)
    P = ctypes.c_void_p
    so.lr_cache_attend_tree.argtypes = [P, P, I32, P, I64, I64, P, I64, I32, F, I32, I32, P, I64, I64, P, P]
    so.lr_cache_weigh.argtypes = [P, P, I32, P, I64, I64, P, F, I32, I32, F, P, I64, I64, I64, P]
    so.lr_cache_select.argtypes = [P, P, P, I64, I64, I64, I32, P, I32, I32, P, P, P]
    so.lr_cache_keep.argtypes = [P, P, I32, P, I32, P, P, P, I64, I64, I64, P]
    so.lr_cache_last_error.argtypes = [P]
    so.lr_cache_last_error.restype = ctypes.c_char_p
    so.lr_cache_destroy.argtypes = [P]
    return so


@pytest.fixture
def cache(lib):
    from paper_2607_18253_gb300 import router as R
    cfg = R._CacheConfig(8, 2, 64, 0, 0, 16, 4, 4, 1 << 20, 1 << 21, None, None, 2048, 128, 64, 0, 0, 0)
    h = ctypes.c_void_p()
    assert lib.lr_cache_create(ctypes.byref(cfg), ctypes.byref(h)) == R.LR_OK
    yield h
    assert lib.lr_cache_destroy(h) == R.LR_OK


def batch(n=1, max_q=64):
    from paper_2607_18253_gb300 import router as R
    return ctypes.byref(R._CacheBatch(n, max_q, 16, 16, 16, 4, 4))


def good(name):
    return {"tree": dict(T=64, q=16, qt=512, qh=64, tree=16, stride=2, words=2, scale=0.125, window=0, sinks=0, out=16, ot=512, oh=64, lse=None),
            "weigh": dict(T=64, q=16, qt=512, qh=64, lse=16, scale=0.125, window=0, sinks=0, decay=1.0, w=16, wb=32, wt=2, wh=1),
            "select": dict(w=16, wb=32, wt=2, wh=1, cap=8, budget=None, sinks=2, recent=6, kept=16, count=16),
            "keep": dict(cap=8, kept=16, heads=2, count=16, start=None, w=None, wb=0, wt=0, wh=0)}[name]


FN = {"tree": "lr_cache_attend_tree", "weigh": "lr_cache_weigh", "select": "lr_cache_select", "keep": "lr_cache_keep"}


def call(lib, h, name, b=None, **kw):
    a = dict(good(name), **kw)
    return getattr(lib, FN[name])(h, batch() if b is None else b, *a.values(), None)


@pytest.mark.parametrize("name", list(FN))
def test_good_calls_are_launched(lib, cache, name):
    before = lib.fake_launched()
    assert call(lib, cache, name) == 0
    assert lib.fake_launched() == before + (name != "tree")


NAN, INF = float("nan"), float("inf")
BAD = ([("tree", k) for k in (dict(T=-1), dict(tree=None), dict(tree=18), dict(words=1), dict(words=-1), dict(words=1 << 31 - 1, stride=-1),
                              dict(scale=0.0), dict(scale=NAN), dict(window=-1), dict(sinks=-1), dict(q=None), dict(q=8), dict(out=None),
                              dict(qt=7), dict(oh=4))]
       + [("weigh", k) for k in (dict(T=-1), dict(q=None), dict(q=24), dict(lse=None), dict(lse=6), dict(scale=INF), dict(scale=-1.0),
                                 dict(window=-1), dict(sinks=(1 << 30) + 1), dict(decay=-0.5), dict(decay=NAN), dict(decay=INF), dict(w=None),
                                 dict(w=2), dict(wb=-1), dict(wt=-1), dict(wh=-1), dict(qh=9))]
       + [("select", k) for k in (dict(cap=-1), dict(cap=7), dict(sinks=-1), dict(recent=-1), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1),
                                  dict(w=None), dict(wb=-8), dict(kept=None), dict(count=None))]
       + [("keep", k) for k in (dict(cap=-1), dict(kept=None), dict(count=None), dict(heads=0), dict(heads=3), dict(w=2), dict(w=16, wh=-1))])


@pytest.mark.parametrize("name,kw", BAD)
def test_bad_calls_are_refused(lib, cache, name, kw):
    from paper_2607_18253_gb300 import router as R
    before = lib.fake_launched()
    assert call(lib, cache, name, **kw) == R.LR_EINVAL
    assert lib.lr_cache_last_error(cache) and lib.fake_launched() == before


@pytest.mark.parametrize("name", list(FN))
def test_batches_out_of_range(lib, cache, name):
    from paper_2607_18253_gb300 import router as R
    before = lib.fake_launched()
    assert call(lib, cache, name, batch(n=5)) == R.LR_ECAPACITY
    assert call(lib, cache, name, batch(n=-1)) == R.LR_EINVAL
    assert call(lib, cache, name, batch(max_q=0)) == R.LR_EINVAL
    assert call(lib, cache, name, batch(n=0)) == R.LR_OK
    assert getattr(lib, FN[name])(None, batch(), *good(name).values(), None) == R.LR_EINVAL
    assert lib.fake_launched() == before


def test_more_drafted_tokens_than_mask_bits(lib, cache):
    assert call(lib, cache, "tree", batch(max_q=65)) != 0
    assert b"tree_words" in lib.lr_cache_last_error(cache)
    assert call(lib, cache, "tree", batch(max_q=65), words=3) == 0


@pytest.mark.parametrize("name", list(FN))
def test_a_batch_without_q_start(lib, cache, name):
    # the choice and the move do not use it
    from paper_2607_18253_gb300 import router as R
    b = ctypes.byref(R._CacheBatch(1, 64, None, 16, 16, 4, 4))
    before = lib.fake_launched()
    assert call(lib, cache, name, b) == (R.LR_OK if name in ("select", "keep") else R.LR_EINVAL)
    assert lib.fake_launched() == before + (name in ("select", "keep"))
    for bad in (R._CacheBatch(1, 64, None, None, 16, 4, 4), R._CacheBatch(1, 64, None, 16, None, 4, 4)):
        assert call(lib, cache, name, ctypes.byref(bad)) == R.LR_EINVAL


@pytest.mark.parametrize("name,kw", [("select", dict(kept=18)), ("select", dict(count=17)), ("select", dict(budget=6)), ("keep", dict(kept=18)),
                                     ("keep", dict(count=17)), ("keep", dict(start=6))])
def test_lists_that_are_not_aligned_are_refused(lib, cache, name, kw):
    # (a kernel that read them would fault)
    from paper_2607_18253_gb300 import router as R
    before = lib.fake_launched()
    assert call(lib, cache, name, **kw) == R.LR_EINVAL
    assert b"aligned" in lib.lr_cache_last_error(cache) and lib.fake_launched() == before
