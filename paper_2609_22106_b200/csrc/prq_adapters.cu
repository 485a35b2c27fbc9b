// Low-rank adapters beside a projection: h = x A^T of each row's adapter, then y = base + scale * h B^T.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "prq_internal.h"
#include "prq_kernels.h"
#include "prq_ptx.cuh"

namespace prq {
namespace {

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

__device__ __forceinline__ int rank_of(const AdapterParams& p, int slot) {
    return p.ranks ? min(max(p.ranks[slot], 0), p.max_rank) : p.max_rank;
}

// h[m, p, r] = scale * sum_k x[m, k] A[p, r, k]: a block per row, a warp per (p, r).
__global__ void __launch_bounds__(256) adapters_h_kernel(const __grid_constant__ AdapterParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const long long m = blockIdx.x;
    const int slot = p.row_adapter[m];
    if (slot < 0 || slot >= p.n_slots) return;
    const int rank = rank_of(p, slot), lane = threadIdx.x & 31;
    const float scale = p.scale ? p.scale[slot] : 1.0f;
    for (int i = threadIdx.x >> 5; i < p.n_parts * rank; i += 8) {
        const int part = i / rank, r = i - part * rank;
        const uint4* a = reinterpret_cast<const uint4*>(p.A + ((static_cast<long long>(slot) * p.n_parts + part) * p.max_rank + r) * p.K);
        const uint4* x = reinterpret_cast<const uint4*>(p.x + m * p.ldx);
        float sum = 0.0f;
        for (int k = lane; k < p.K / 8; k += 32) {
            const uint4 va = a[k], vx = x[k];
            const uint32_t *wa = &va.x, *wx = &vx.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum = fmaf(bf16_lo(wa[j]), bf16_lo(wx[j]), sum);
                sum = fmaf(bf16_hi(wa[j]), bf16_hi(wx[j]), sum);
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) p.h[(m * p.n_parts + part) * p.max_rank + r] = sum * scale;
    }
}

template <class T>
__global__ void __launch_bounds__(256) adapters_y_kernel(const __grid_constant__ AdapterParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= p.N) return;
    int part = 0;
    while (n >= p.part_end[part]) ++part;
    for (long long m = blockIdx.y; m < p.M; m += gridDim.y) {
        const int slot = p.row_adapter[m];
        const int rank = slot < 0 || slot >= p.n_slots ? 0 : rank_of(p, slot);
        const T* from = static_cast<const T*>(p.base) + m * p.ldbase + n;
        T* to = static_cast<T*>(p.y) + m * p.ldy + n;
        if (rank == 0) {
            if (to != from) *to = *from;
            continue;
        }
        const float* h = p.h + (m * p.n_parts + part) * p.max_rank;
        const uint16_t* b = p.B + (static_cast<long long>(slot) * p.N + n) * p.max_rank;
        float sum = 0.0f;
        for (int r = 0; r < rank; ++r) sum = fmaf(h[r], __uint_as_float(static_cast<uint32_t>(b[r]) << 16), sum);
        *to = static_cast<T>(static_cast<float>(*from) + sum);
    }
}

}  // namespace

size_t adapters_workspace_bytes(int M, int n_parts, int max_rank) { return sizeof(float) * M * n_parts * max_rank; }

cudaError_t launch_adapters(const AdapterParams& p, bool bf16, int num_sms, cudaStream_t stream, int* launches) {
    cudaLaunchConfig_t cfg = {};
    cfg.stream = stream;
    cfg.blockDim = dim3(256);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(p.M);
    cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_h_kernel, p);
    if (e != cudaSuccess) return e;
    cfg.gridDim = dim3((p.N + 255) / 256, std::min(p.M, 65535));
    *launches = 2;
    return bf16 ? cudaLaunchKernelEx(&cfg, adapters_y_kernel<__nv_bfloat16>, p) : cudaLaunchKernelEx(&cfg, adapters_y_kernel<float>, p);
}

}  // namespace prq
