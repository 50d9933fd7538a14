"""Programs that call the operators' C entry points on a runtime that is made up: launches are counted and never run, so that made-up addresses do and any status or
size can be tried without a device.  The library's own object files, linked with these functions in place of the CUDA runtime."""
import os
import subprocess

RUNTIME = r"""
#include <cuda_runtime.h>
#include <stdio.h>
#include <string.h>
#include "mpode.h"
static cudaError_t stale = cudaSuccess, refuse = cudaSuccess;      // what an earlier call has left; what a launch answers
static cudaError_t occupancy = cudaSuccess;                        // what the question for clusters answers
static long long launches = 0;
static dim3 grid;
extern "C" {
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
unsigned __cudaPushCallConfiguration(dim3 g, dim3, size_t, struct CUstream_st*) { grid = g; return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3 g, dim3, void**, size_t, cudaStream_t) { ++launches; grid = g; return refuse; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**) { ++launches; grid = c->gridDim; return refuse; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { *n = 8; return occupancy; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaGetLastError() { const cudaError_t e = stale; stale = cudaSuccess; return e; }
const char* cudaGetErrorString(cudaError_t) { return "made up"; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* q) { *f = nullptr; *q = cudaDriverEntryPointSymbolNotFound; return cudaSuccess; }
}
static const void* at(int i) { return (const void*)((1ull << 40) + ((unsigned long long)i << 36)); }
static void* to(int i) { return const_cast<void*>(at(i)); }
"""


def run(tmp_path, body):
    """What a program with `body` as the inside of main prints, in words."""
    from paper_2510_23498_b200 import build
    objects = [os.path.join(build.HERE, "_build", n + ".o") for n in ("recurrence", "residual", "residual_forward", "residual_backward", "dropout", "tensormap")]
    build.build(force=not all(os.path.exists(o) for o in objects))
    src = tmp_path / "t.cpp"
    src.write_text(RUNTIME + "int main() {\n" + body + "\nreturn 0; }\n")
    exe = str(tmp_path / "t")
    cuda = os.path.dirname(os.path.dirname(build._nvcc()))
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(cuda, "include"), "-I", os.path.join(build.HERE, "..", "include"), str(src), *objects, "-o", exe], check=True)
    return subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.split()
