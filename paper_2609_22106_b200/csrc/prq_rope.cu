// Position rotation of query and key heads, with or without the RMS norm of each head in front.
//
// A pair (a, b) of a head in a row at position m turns by m f_i.  The angle is kept as a fraction of a turn: f_i / 2 pi in units
// of 2^-64, times m, modulo 2^64 -- exact integer arithmetic, so that the angle of a far position is as exact as that of
// a near one.  (In fp32, m f_i is off by up to 0.03 radian at position 10^6.)  What is left of the turn is cut into the nearest quadrant and
// a remainder of at most pi / 4, whose sine and cosine are Taylor polynomials.
#include <cuda_bf16.h>
#include <type_traits>
#include <cuda_runtime.h>

#include "prq_internal.h"
#include "prq_kernels.h"
#include "prq_ptx.cuh"

namespace prq {
namespace {

// cos and sin of `turns` * 2^-64 turns.  The quadrant is the nearest one, so that the remainder t is within an eighth of a turn
// (theta <= pi / 4); the next Taylor terms are theta^11 / 11! < 1.8e-9 and theta^12 / 12! < 1.2e-10.
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

// Any head size, rotated part, stride and alignment: a warp per head, the head in shared memory, angles worked out for every head anew.  Simple
// and slow for many rows: 4096 rows of 32 + 8 heads of 128, bf16, an odd row stride, 105 us (110 with the norm), where the kernel below
// takes 9.5 (13.7) on whole 16 bytes; 1533 rows of 20 + 20 heads of 80, fp32, 21 and 7.8; 4096 rows of 16 + 4 heads of 80, of which 20 turn, 26,
// where 80 take 7.1; 64 rows 3.4 and 2.0, one row 1.6 either way.  (In place, in L2.)
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

// Two fp32 values that one instruction works on, low half first.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ float lo(f32x2 v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float hi(f32x2 v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
__device__ __forceinline__ f32x2 swapped(f32x2 v) { return pair(hi(v), lo(v)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Eight elements of a head, 16 bytes (bf16) or 32 (fp32).  Ordinary loads: rows may be rotated in place.
template <class T>
struct Eight {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) raw[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void unpack(f32x2 (&v)[4]) const {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[2 * i] = pair(__uint_as_float(raw[i].x), __uint_as_float(raw[i].y));
                v[2 * i + 1] = pair(__uint_as_float(raw[i].z), __uint_as_float(raw[i].w));
            }
        }
    }
    static __device__ __forceinline__ void store(T* p, const f32x2 (&v)[4]) {
        if constexpr (sizeof(T) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(lo(v[i]), hi(v[i]));   // nearest, ties to even
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            reinterpret_cast<float4*>(p)[0] = make_float4(lo(v[0]), hi(v[0]), lo(v[1]), hi(v[1]));
            reinterpret_cast<float4*>(p)[1] = make_float4(lo(v[2]), hi(v[2]), lo(v[3]), hi(v[3]));
        }
    }
};

// The fast kernels take head sizes and rotated parts that are multiples of 16, rows and heads on 16 bytes.  A head is cut into units of 16
// elements that hold eight whole pairs: elements 8 u .. 8 u + 7 of both halves (half layout), or 16 u .. 16 u + 15 (interleaved,
// and what does not turn).  A lane has one unit, kLanes lanes a head, a warp 32 / kLanes heads at a time and kTimes such groups of
// one tensor; the warps of a CTA share a row (blockIdx.y: where it has more heads than that).
constexpr int kRotateWarps = 8;
template <class T, bool kInterleaved, bool kNorm, int kLanes>
struct Unit {
    int u, g, ea, eb;      // unit, head of the group; the unit's two eights
    bool inside, rotated;
    f32x2 wa[4], wb[4];

    __device__ __forceinline__ Unit(const RotateParams& p) {
        const int lane = threadIdx.x & 31;
        u = lane % kLanes;
        g = lane / kLanes;
        inside = u < p.head_dim / 16 && g < 32 / kLanes;
        rotated = u < p.rot_dim / 16;
        ea = kInterleaved || !rotated ? 16 * u : 8 * u;   // (what does not turn begins at 16 units of what does)
        eb = kInterleaved || !rotated ? ea + 8 : ea + p.rot_dim / 2;
    }
    __device__ __forceinline__ void load_weight(const float* weight) {   // 16-byte aligned, or null
        const bool w = weight && inside;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float4 va = w ? __ldg(reinterpret_cast<const float4*>(weight + ea) + j) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
            const float4 vb = w ? __ldg(reinterpret_cast<const float4*>(weight + eb) + j) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
            wa[2 * j] = pair(va.x, va.y);
            wa[2 * j + 1] = pair(va.z, va.w);
            wb[2 * j] = pair(vb.x, vb.y);
            wb[2 * j + 1] = pair(vb.z, vb.w);
        }
    }
    // Norm (its sum over the head's lanes: all of the warp take part) and rotation of the two eights.
    __device__ __forceinline__ void turn(f32x2 (&a)[4], f32x2 (&b)[4], const f32x2 (&c)[4], const f32x2 (&s)[4], float inv_dim, float eps) const {
        if (kNorm) {
            f32x2 sum2 = mul2(a[0], a[0]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j) sum2 = fma2(a[j], a[j], sum2);
                sum2 = fma2(b[j], b[j], sum2);
            }
            float sum = lo(sum2) + hi(sum2);
#pragma unroll
            for (int d = kLanes / 2; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const float r = rsqrtf(fmaf(sum, inv_dim, eps));
            const f32x2 r2 = pair(r, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = mul2(mul2(a[j], r2), wa[j]);
                b[j] = mul2(mul2(b[j], r2), wb[j]);
            }
        }
        if (!rotated) return;
        f32x2 ta[4], tb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (kInterleaved) {
                // element pair j of the first eight is pair j of the unit, of the second eight pair 4 + j
                const float c0 = j & 1 ? hi(c[j / 2]) : lo(c[j / 2]), s0 = j & 1 ? hi(s[j / 2]) : lo(s[j / 2]);
                const float c1 = j & 1 ? hi(c[2 + j / 2]) : lo(c[2 + j / 2]), s1 = j & 1 ? hi(s[2 + j / 2]) : lo(s[2 + j / 2]);
                ta[j] = fma2(swapped(a[j]), pair(-s0, s0), mul2(a[j], pair(c0, c0)));
                tb[j] = fma2(swapped(b[j]), pair(-s1, s1), mul2(b[j], pair(c1, c1)));
            } else {
                ta[j] = fma2(b[j], pair(-lo(s[j]), -hi(s[j])), mul2(a[j], c[j]));
                tb[j] = fma2(a[j], s[j], mul2(b[j], c[j]));
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = ta[j];
            b[j] = tb[j];
        }
    }
};

// Cosines and sines of a row's pairs, a pair a thread; `mine` is the thread's first one.  A unit's eight pairs lie in two fours, next to those
// of the other units: a warp's 16-byte loads meet no bank twice.
template <int kLanes>
using Angles = float[4][kLanes][4];   // cosines of pairs 0 .. 3 of every unit, of pairs 4 .. 7, sines of both
template <int kLanes>
__device__ __forceinline__ void turn_pairs(const RotateParams& p, uint64_t mine, int pos, Angles<kLanes>& angle) {
    for (int i = threadIdx.x; i < p.rot_dim / 2; i += blockDim.x) {
        float c, s;
        cos_sin((i == static_cast<int>(threadIdx.x) ? mine : p.turns[i]) * static_cast<uint64_t>(static_cast<int64_t>(pos)), &c, &s);
        angle[i >> 2 & 1][i >> 3][i & 3] = c * p.factor;
        angle[2 + (i >> 2 & 1)][i >> 3][i & 3] = s * p.factor;
    }
}
template <int kLanes>
__device__ __forceinline__ void read_pairs(const Angles<kLanes>& angle, int u, f32x2 (&c)[4], f32x2 (&s)[4]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const ulonglong2 vc = *reinterpret_cast<const ulonglong2*>(angle[j][u]), vs = *reinterpret_cast<const ulonglong2*>(angle[2 + j][u]);
        c[2 * j] = vc.x;
        c[2 * j + 1] = vc.y;
        s[2 * j] = vs.x;
        s[2 * j + 1] = vs.y;
    }
}

// A row, or a slice of its heads, per CTA.  Bound by memory for many rows: what hides its latency is 128 bytes of loads per lane in flight
// (kTimes = 4 for bf16, 2 for fp32) and 24 warps per SM.  The angles, a pair a thread, are worked out beside the loads.  (Rows that came
// through a ring in shared memory by bulk copies, CTAs going from row to row, took longer: one barrier per row holds all warps.)  8192
// rows of 40 heads of 128, bf16: 26.4 us, 6.35 TB/s; 4096 rows with the norm: 16.7 us, 5.0 TB/s, its instructions count there.  For few rows
// the chain position -> angle -> result is what takes the time: one row 1.8 us, as long as an empty launch behind another.
template <class T, bool kInterleaved, bool kNorm, int kLanes, int kTimes>
__global__ void __launch_bounds__(kRotateWarps * 32, 3) rotate_kernel(const __grid_constant__ RotateParams p, int warps_q) {
    constexpr int kHeads = 32 / kLanes;
    __shared__ __align__(16) Angles<kLanes> angle_s;
    Unit<T, kInterleaved, kNorm, kLanes> unit(p);
    const int warp = blockIdx.y * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const bool key = warp >= warps_q;
    const HeadRows& t = p.t[key];
    const int head = (key ? warp - warps_q : warp) * (kHeads * kTimes) + unit.g;
    const uint64_t turns = static_cast<int>(threadIdx.x) < p.rot_dim / 2 ? p.turns[threadIdx.x] : 0;
    const long long m = blockIdx.x;
    const T* x = static_cast<const T*>(t.x) + m * t.ldx + head * t.hsx;
    T* out = static_cast<T*>(t.out) + m * t.ldout + head * t.hsout;
    grid_dependency_wait();
    grid_launch_dependents();
    const int pos = p.positions[m];
    Eight<T> ra[kTimes], rb[kTimes];
#pragma unroll
    for (int n = 0; n < kTimes; ++n) {
        ra[n].zero();
        rb[n].zero();
        if (unit.inside && head + n * kHeads < t.heads) {
            ra[n].load(x + n * kHeads * t.hsx + unit.ea);
            rb[n].load(x + n * kHeads * t.hsx + unit.eb);
        }
    }
    if (kNorm) unit.load_weight(t.weight);
    if (pos == PRQ_POSITION_NONE) return;
    turn_pairs<kLanes>(p, turns, pos, angle_s);
    __syncthreads();
    f32x2 c[4], s[4];
    read_pairs<kLanes>(angle_s, unit.u, c, s);
    const float inv_dim = 1.0f / p.head_dim;
#pragma unroll
    for (int n = 0; n < kTimes; ++n) {
        f32x2 a[4], b[4];
        ra[n].unpack(a);
        rb[n].unpack(b);
        unit.turn(a, b, c, s, inv_dim, p.eps);
        if (unit.inside && head + n * kHeads < t.heads) {
            Eight<T>::store(out + n * kHeads * t.hsout + unit.ea, a);
            Eight<T>::store(out + n * kHeads * t.hsout + unit.eb, b);
        }
    }
}

template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 blocks, int threads, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class T, bool kInterleaved, bool kNorm>
cudaError_t launch_of(const RotateParams& p, int num_sms, cudaStream_t stream) {
    const int heads = p.t[0].heads + p.t[1].heads;
    bool wide = p.head_dim % 16 == 0 && p.rot_dim % 16 == 0 && p.head_dim <= 256;
    for (const HeadRows& t : p.t) {
        constexpr long long kUnit = 16 / sizeof(T);
        if (t.heads == 0) continue;
        wide = wide && ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.out) | reinterpret_cast<uintptr_t>(t.weight)) & 15) == 0 && t.ldx % kUnit == 0 && t.ldout % kUnit == 0 &&
               t.hsx % kUnit == 0 && t.hsout % kUnit == 0;
    }
    if (!wide) {
        const long long tasks = static_cast<long long>(p.M) * heads;
        return launch(rotate_any_kernel<T, kInterleaved, kNorm>, dim3(static_cast<unsigned>(std::min<long long>((tasks + kAnyWarps - 1) / kAnyWarps, num_sms * 16ll))),
                      kAnyWarps * 32, stream, p);
    }
    // lanes of a head: a power of two, for the norm's sum over them; without one, five or six where that is a head's units (20 + 20 heads of 80, 1533
    // rows, fp32: 9.2 us with eight, 8.6 so)
    const int units = p.head_dim / 16, lanes = !kNorm && (units == 5 || units == 6) ? units : units <= 4 ? 4 : units <= 8 ? 8 : 16, at_once = 32 / lanes;
    constexpr int kMany = 8 / sizeof(T);
    const auto its = [&](int times) { return (p.t[0].heads + at_once * times - 1) / (at_once * times) + (p.t[1].heads + at_once * times - 1) / (at_once * times); };
    // few rows: as long as the warps with one group of heads each are all on the GPU at once (40 heads of 128: up to 236 rows.  64 rows:
    // 1.95 us, with kMany groups 2.6; 200 to 300 rows: 2.8 - 3.0 either way; 400 rows: 3.8 and 3.2)
    const bool few = static_cast<long long>(p.M) * its(1) <= 16ll * num_sms;
    const int times = few ? 1 : kMany, all = its(times), slices = (all + kRotateWarps - 1) / kRotateWarps, warps = (all + slices - 1) / slices;
    const int warps_q = (p.t[0].heads + at_once * times - 1) / (at_once * times);
    auto of = [&](auto lanes_c) {
        constexpr int kLanes = decltype(lanes_c)::value;
        return launch(few ? rotate_kernel<T, kInterleaved, kNorm, kLanes, 1> : rotate_kernel<T, kInterleaved, kNorm, kLanes, kMany>, dim3(p.M, slices), warps * 32,
                      stream, p, warps_q);
    };
    if constexpr (!kNorm) {
        if (lanes == 5) return of(std::integral_constant<int, 5>());
        if (lanes == 6) return of(std::integral_constant<int, 6>());
    }
    return lanes == 4 ? of(std::integral_constant<int, 4>()) : lanes == 8 ? of(std::integral_constant<int, 8>()) : of(std::integral_constant<int, 16>());
}

}  // namespace

cudaError_t launch_rotate_heads(const RotateParams& p, bool interleaved, bool norm, bool bf16, int num_sms, cudaStream_t stream) {
    auto of_type = [&](auto zero) {
        using T = decltype(zero);
        if (interleaved) return norm ? launch_of<T, true, true>(p, num_sms, stream) : launch_of<T, true, false>(p, num_sms, stream);
        return norm ? launch_of<T, false, true>(p, num_sms, stream) : launch_of<T, false, false>(p, num_sms, stream);
    };
    return bf16 ? of_type(__nv_bfloat16()) : of_type(0.0f);
}

}  // namespace prq
