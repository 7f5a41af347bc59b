"""Without a GPU: which launches small problems make where a cluster of 16 blocks fits the device, and where it does not (a part of a
GPU).  The norm's and the 4-bit quantisation's host code runs on stand-ins for the CUDA runtime that note the launches; the kernels,
compiled to the intermediate form only, never run."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2409_12517_b200 import binding as B
from paper_2409_12517_b200 import build as libbuild

P = 4096

RUNTIME = r"""
#include <cuda_runtime.h>
int fake_device = 0, fake_clusters[3] = {4, 0, 0}, launches = 0;
int grid[64], cluster[64];
static void note(int g, int c) { if (launches < 64) { grid[launches] = g; cluster[launches] = c; } ++launches; }
namespace fp8mlp {
void set_cuda_error(const char*, cudaError_t) {}
void count_launch() {}
int clear_float(float*, cudaStream_t) { note(1, 0); return 0; }
}
extern "C" {
int* at_device() { return &fake_device; }
int* at_launches() { return &launches; }
int* at_grid() { return grid; }
int* at_cluster() { return cluster; }
cudaError_t cudaGetDevice(int* d) { *d = fake_device; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaSuccess; }
// device 0 holds such clusters, device 1 none, device 2 does not know the size
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) {
    *n = fake_clusters[fake_device];
    return fake_device == 2 ? cudaErrorInvalidClusterSize : cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* cfg, const void*, void**) {
    int c = 0;
    for (unsigned i = 0; i < cfg->numAttrs; ++i)
        if (cfg->attrs[i].id == cudaLaunchAttributeClusterDimension) c = cfg->attrs[i].val.clusterDim.x;
    note(cfg->gridDim.x, c);
    return cudaSuccess;
}
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, void*, void*, void*, void*, int*) {}
char __cudaInitModule(void**) { return 0; }
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("host")
    (at / "runtime.cpp").write_text(RUNTIME)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-std=c++17", "-O0", "-Xcompiler", "-fPIC", "-c"]
    runs = [subprocess.Popen([nvcc, "-gencode", "arch=compute_100a,code=compute_100a", "-Xcicc", "-O0", *flags, "-o", str(at / f"{f}.o"),
                              str(libbuild.CSRC / f"{f}.cu")]) for f in ("norm", "fp4")]
    runs.append(subprocess.Popen([nvcc, *flags, "-o", str(at / "runtime.o"), str(at / "runtime.cpp")]))
    assert all(r.wait() == 0 for r in runs)
    subprocess.check_call(["g++", "-shared", "-Wl,-Bsymbolic", "-o", str(at / "host.so"), *(str(at / f"{f}.o") for f in ("norm", "fp4", "runtime"))])
    L = C.CDLL(str(at / "host.so"))
    p, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
    L.fp8mlp_rmsnorm.argtypes = [i64, i64, i32, p, i64, p, i64, p, i64, p, f32, i32, p, i64, p, p, p, p]
    L.fp8mlp_rmsnorm_backward.argtypes = [i64, i64, i32, p, i64, p, i64, p, p, p, i64, p, i64, p, p, p]
    L.fp8mlp_quantize_fp4.argtypes = [p, i32, i64, i64, i64, i32, i32, i32, p, p, p, i64, p, p]
    for n in ("device", "launches", "grid", "cluster"):
        getattr(L, f"at_{n}").restype = C.POINTER(i32)

    def made(device, call):
        """(grid, cluster) of each launch of a call on that device; the clearing of a maximum is one of (1, 0)."""
        L.at_device()[0], L.at_launches()[0] = device, 0
        assert call(L) == B.OK
        return [(L.at_grid()[i], L.at_cluster()[i]) for i in range(L.at_launches()[0])]
    return made


def norm(T, amax=P):
    return lambda L: L.fp8mlp_rmsnorm(T, 4096, B.BF16, P, 4096, None, 0, None, 0, None, 1e-5, B.RMS_SAME, 2 * P, 4096, None, amax, None, None)


def norm_backward(T):
    return lambda L: L.fp8mlp_rmsnorm_backward(T, 4096, B.BF16, P, 4096, 2 * P, 4096, None, P, None, 0, 3 * P, 4096, P, P, None)


def quantise(rows):
    return lambda L: L.fp8mlp_quantize_fp4(P, B.BF16, rows, 1024, 1024, 0, B.NVFP4, B.SCALE_FROM_CURRENT_AMAX, P, 2 * P, P, 512, P, None)


def test_one_cluster_where_it_fits(host):
    assert host(0, norm(16)) == host(0, norm(32)) == [(16, 16)]
    assert host(0, norm_backward(32)) == [(16, 16)]
    assert host(0, quantise(256)) == [(16, 16)]
    assert host(0, norm(1)) == [(1, 0)] and host(0, norm(16, amax=None)) == [(16, 0)]
    assert host(0, norm(40)) == [(1, 0), (40, 0)] and len(host(0, norm_backward(40))) == 2 and len(host(0, quantise(400))) == 3


@pytest.mark.parametrize("device", [1, 2])
def test_several_launches_where_it_does_not(host, device):
    """As large problems run: the maximum cleared first, the gain's gradient added up by a second launch, a pass for the maximum."""
    assert host(device, norm(16)) == [(1, 0), (16, 0)] and host(device, norm(32)) == [(1, 0), (32, 0)]
    assert host(device, norm_backward(32)) == [(32, 0), (64, 0)]
    made = host(device, quantise(256))
    assert len(made) == 3 and all(c == 0 for _, c in made) and made[2] == (16, 0)
    assert host(device, norm(1)) == [(1, 0)]
