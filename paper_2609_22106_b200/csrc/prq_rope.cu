// Position rotation of query and key heads, with or without the RMS norm of each head in front.
//
// A pair (a, b) of a head in a row at position m turns by m f_i.  The angle is kept as a fraction of a turn: f_i / 2 pi in units
// of 2^-64, times m, modulo 2^64 -- exact integer arithmetic, so that the angle of a far position is as exact as that of
// a near one.  (In fp32, m f_i is off by up to 0.03 radian at position 10^6.)  What is left of the turn is cut into an octant and
// a remainder of at most pi / 4, whose sine and cosine are Taylor polynomials.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "prq_internal.h"
#include "prq_kernels.h"
#include "prq_ptx.cuh"

namespace prq {
namespace {

// cos and sin of `turns` * 2^-64 turns.  The quadrant is the nearest one, so that the remainder t is within an eighth of a turn
// (theta <= pi / 4); the next Taylor terms are theta^11 / 11! < 1.8e-9 and theta^10 / 10! < 2.5e-8, theta^12 / 12! < 1.2e-10.
__device__ __forceinline__ void cos_sin(uint64_t turns, float* c, float* s) {
    const uint32_t hi = static_cast<uint32_t>(turns >> 32);
    const uint32_t quadrant = (hi + 0x20000000u) >> 30;
    const float t = static_cast<float>(static_cast<int32_t>(hi - (quadrant << 30)));   // 2^-32 turns, |t| <= 2^29
    const float theta = t * 1.4629180792671596e-9f;                                    // 2 pi / 2^32
    const float u = theta * theta;
    float sn = fmaf(u, 1.0f / 362880.0f, -1.0f / 5040.0f);
    sn = fmaf(u, sn, 1.0f / 120.0f);
    sn = fmaf(u, sn, -1.0f / 6.0f);
    sn = fmaf(theta * u, sn, theta);
    float cs = fmaf(u, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    cs = fmaf(u, cs, -1.0f / 720.0f);
    cs = fmaf(u, cs, 1.0f / 24.0f);
    cs = fmaf(u, cs, -0.5f);
    cs = fmaf(u, cs, 1.0f);
    const bool swap = quadrant & 1;
    const float a = swap ? sn : cs, b = swap ? cs : sn;
    // quadrants 0 .. 3: (c, s), (-s, c), (-c, -s), (s, -c)
    *c = (quadrant == 1 || quadrant == 2) ? -a : a;
    *s = (quadrant & 2) ? -b : b;
}

__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }   // nearest, ties to even

// Any head size, rotated part, stride and alignment: a warp per head, the head in shared memory.
constexpr int kAnyWarps = 4;
template <class T, bool kInterleaved, bool kNorm>
__global__ void __launch_bounds__(kAnyWarps * 32) rotate_any_kernel(const __grid_constant__ RotateParams p) {
    __shared__ float head_s[kAnyWarps][512];
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* z = head_s[warp];
    const int heads = p.t[0].heads + p.t[1].heads, D = p.head_dim, half = p.rot_dim / 2;
    const long long tasks = static_cast<long long>(p.M) * heads;
    for (long long i = static_cast<long long>(blockIdx.x) * kAnyWarps + warp; i < tasks; i += static_cast<long long>(gridDim.x) * kAnyWarps) {
        const long long m = i / heads;
        int h = static_cast<int>(i - m * heads);
        const bool key = h >= p.t[0].heads;
        const HeadRows& t = p.t[key];
        if (key) h -= p.t[0].heads;
        const int pos = p.positions[m];
        if (pos == PRQ_POSITION_NONE) continue;
        const T* x = static_cast<const T*>(t.x) + m * t.ldx + h * t.hsx;
        T* out = static_cast<T*>(t.out) + m * t.ldout + h * t.hsout;
        float sum = 0.0f;
        for (int j = lane; j < D; j += 32) {
            const float v = load(x + j);
            z[j] = v;
            sum = fmaf(v, v, sum);
        }
        __syncwarp();
        float r = 1.0f;
        if (kNorm) {
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            r = rsqrtf(sum / D + p.eps);
        }
        auto element = [&](int j) { return kNorm ? (t.weight ? z[j] * r * t.weight[j] : z[j] * r) : z[j]; };
        for (int j = lane; j < half; j += 32) {
            const int ja = kInterleaved ? 2 * j : j, jb = kInterleaved ? 2 * j + 1 : j + half;
            const float a = element(ja), b = element(jb);
            float c, s;
            cos_sin(p.turns[j] * static_cast<uint64_t>(static_cast<int64_t>(pos)), &c, &s);
            c *= p.factor;
            s *= p.factor;
            store(out + ja, a * c - b * s);
            store(out + jb, b * c + a * s);
        }
        for (int j = 2 * half + lane; j < D; j += 32) store(out + j, element(j));
        __syncwarp();
    }
}

template <class T, bool kInterleaved, bool kNorm>
cudaError_t launch(const RotateParams& p, int num_sms, cudaStream_t stream) {
    const long long tasks = static_cast<long long>(p.M) * (p.t[0].heads + p.t[1].heads);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>((tasks + kAnyWarps - 1) / kAnyWarps, num_sms * 16ll)));
    cfg.blockDim = dim3(kAnyWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, rotate_any_kernel<T, kInterleaved, kNorm>, p);
}

}  // namespace

cudaError_t launch_rotate_heads(const RotateParams& p, bool interleaved, bool norm, bool bf16, int num_sms, cudaStream_t stream) {
    auto of_type = [&](auto zero) {
        using T = decltype(zero);
        if (interleaved) return norm ? launch<T, true, true>(p, num_sms, stream) : launch<T, true, false>(p, num_sms, stream);
        return norm ? launch<T, false, true>(p, num_sms, stream) : launch<T, false, false>(p, num_sms, stream);
    };
    return bf16 ? of_type(__nv_bfloat16()) : of_type(0.0f);
}

}  // namespace prq
