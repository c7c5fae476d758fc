"""What the feed-forward calls hand to their kernels, read on the host: `csrc/ffn.cu` is compiled as plain C++ with the bodies of its
device functions left out and its launches recorded, so that no device is needed and no address is followed."""
import ctypes
import os
import re
import subprocess

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2408_11500_b200", "csrc")

BEFORE = r"""
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>
#undef __grid_constant__
#define __grid_constant__
#undef __launch_bounds__
#define __launch_bounds__(...)
#undef __cluster_dims__
#define __cluster_dims__(...)
template <typename C, typename K, typename... A>
cudaError_t recorded_launch(const C* cfg, K, const A&... args) { record(*cfg, args...); return cudaSuccess; }
#define cudaLaunchKernelEx recorded_launch
"""

AFTER = r"""
struct Seen { int64_t kernel, bias, bias2, reach; };     // biases' addresses; `reach`: numbers of each that the launch may ask for
static Seen seen[64];
static int count;
namespace sgcn {
namespace {
void record(const cudaLaunchConfig_t&, const Params& P) { seen[count++] = {0, (int64_t)P.b, (int64_t)P.b2, (int64_t)P.items / ((int64_t)P.tiles_m * P.tiles_n * P.splits) * P.cols}; }
void record(const cudaLaunchConfig_t&, const FinishArgs& A) { seen[count++] = {1, (int64_t)A.b, (int64_t)A.b2, (int64_t)A.p * A.cols}; }
void record(const cudaLaunchConfig_t&, const PackArgs&) { seen[count++] = {2, 0, 0, 0}; }
void record(const cudaLaunchConfig_t&, const SumArgs&) { seen[count++] = {3, 0, 0, 0}; }
void record(const cudaLaunchConfig_t&, const JoinArgs&) { seen[count++] = {4, 0, 0, 0}; }
void record(const cudaLaunchConfig_t& c, const RowsArgs& A) { seen[count++] = {5, (int64_t)A.b, (int64_t)A.b2, (int64_t)c.gridDim.y * A.out_s}; }
void record(const cudaLaunchConfig_t& c, const LittleArgs& A) { seen[count++] = {6, (int64_t)A.b, (int64_t)A.b2, (int64_t)(c.gridDim.x / A.tiles_n) * A.out_s}; }
}  // namespace
void set_error(const char*, ...) {}
void count_launch(int) {}
}  // namespace sgcn
static CUresult encoded(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                        CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) { return CUDA_SUCCESS; }
extern "C" {
int launches_seen(int64_t* to) { const int n = count; for (int i = 0; i < n; ++i) for (int k = 0; k < 4; ++k) to[4 * i + k] = (&seen[i].kernel)[k]; count = 0; return n; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return ""; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    *fn = (void*)encoded, *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
}
"""


def host_only(source):
    """The source without the bodies of its __device__ and __global__ functions."""
    out, at = [], 0
    for m in re.finditer(r"__(?:device|global)__", source):
        if m.start() < at:
            continue
        open_ = source.index("{", m.end())
        depth, end = 1, open_ + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(source[end], 0)
            end += 1
        out.append(source[at:open_] + "{}")
        at = end
    return "".join(out) + source[at:]


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    folder = tmp_path_factory.mktemp("ffn_host")
    with open(os.path.join(CSRC, "ffn.cu")) as f:
        body = host_only(re.sub(r"//[^\n]*", "", f.read()))
    path, lib = folder / "ffn_host.cpp", folder / "ffn_host.so"
    path.write_text(BEFORE + body.replace('#include "common.cuh"', f'#include "{CSRC}/common.cuh"') + AFTER)
    subprocess.run(["g++", "-std=c++17", "-O0", "-w", "-fpermissive", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", str(path), "-o", str(lib)], check=True)
    lib = ctypes.CDLL(str(lib))
    for name in ("slicegcn_ffn_workspace_bytes", "slicegcn_ffn_forward", "slicegcn_ffn_backward"):
        from paper_2408_11500_b200 import binding as B
        getattr(lib, name).argtypes = B.ARGTYPES[name]
    return lib


AT = 1 << 40             # addresses that nobody follows
X, W, W2, BIAS, BIAS2, OUT, WS = (AT + i * (1 << 36) for i in range(7))


def _launches(library, n, p, ins, outs, gated, dtype, grad, back):
    from paper_2408_11500_b200 import binding as B
    code = {"bf16": B.BF16, "fp32": B.F32}
    d = B.make_ffn_desc(n, p, ins, outs, W, W2 if gated else None, BIAS, BIAS2 if gated else None, act=B.ACT_SILU, dtype=code[dtype], grad_dtype=code[grad])
    if back:
        s = library.slicegcn_ffn_backward(ctypes.byref(d), X, OUT, OUT, OUT, OUT if gated else None, OUT, OUT if gated else None, None, WS, 1 << 36, None)
    else:
        s = library.slicegcn_ffn_forward(ctypes.byref(d), X, None, OUT, None, WS, 1 << 36, None)
    assert s == B.OK
    seen = (ctypes.c_int64 * 256)()
    return [tuple(seen[4 * i:4 * i + 4]) for i in range(library.launches_seen(seen))]


PRODUCT, FINISH = 0, 1
SHAPES = [(300, 1, 1024, 1024), (2708, 1, 1433, 16), (100, 1, 4096, 64), (16, 1, 64, 2500), (700, 1, 2000, 130), (40, 2, 900, 300), (5000, 1, 800, 72), (6, 1, 256, 1024),
          (169_343, 1, 256, 1024), (232_965, 1, 602, 128), (20_001, 8, 32, 64), (200, 1, 25, 14)]


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")], ids=str)
def test_no_launch_may_ask_for_biases_past_their_end(library, types, gated):
    """A launch that is given biases has slices x columns of them, whatever pieces its product is cut into; and they do arrive somewhere."""
    pieces = 0
    for n, p, ins, outs in SHAPES:
        for back in (False, True):
            seen = _launches(library, n, p, ins, outs, gated, *types, back)
            pieces += any(s[0] == FINISH and s[1] for s in seen)
            for kernel, bias, bias2, reach in seen:
                assert not (bias or bias2) or reach <= p * outs, (n, p, ins, outs, back, kernel)
                assert bias in (0, BIAS) and bias2 in (0, BIAS2)
            assert sum(s[1] == BIAS for s in seen) == 1 and sum(s[2] == BIAS2 for s in seen) == int(gated), (n, p, ins, outs, back)
    assert pieces > 1          # products in pieces are among them
