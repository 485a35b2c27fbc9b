// C-ABI entry points of what stands beside the projections: low-rank adapters, position rotation of heads.  Argument checks
// and launches; the contract of every call is in include/prq.h.
#include <cmath>
#include <cstring>
#include <new>

#include "prq_internal.h"
#include "prq_kernels.h"

using namespace prq;

namespace {

constexpr int kMaxAdapterRows = 1 << 23;   // (items, and with them grids, stay within 31 bits)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A description as it is used: fields checked, sums done.
prq_status read_adapters(const prq_adapters* a, AdapterParams* p) {
    if (!a || a->struct_size < sizeof(prq_adapters)) return PRQ_ERR_INVALID_ARG;
    if (a->n_slots < 1 || a->max_rank < 8 || a->max_rank > PRQ_ADAPTER_MAX_RANK || a->max_rank % 8) return PRQ_ERR_INVALID_ARG;
    if (a->K < 32 || a->K % 32 || a->n_parts < 1 || a->n_parts > PRQ_MULTI_MAX) return PRQ_ERR_INVALID_ARG;
    long long N = 0;
    for (int i = 0; i < a->n_parts; ++i) {
        if (a->part_N[i] < 1 || (i + 1 < a->n_parts && a->part_N[i] % 8)) return PRQ_ERR_INVALID_ARG;
        N += a->part_N[i];
        if (N > (1ll << 30)) return PRQ_ERR_INVALID_ARG;
        p->part_end[i] = static_cast<int>(N);
    }
    for (int i = a->n_parts; i < kMaxBatch; ++i) p->part_end[i] = static_cast<int>(N);
    p->A = static_cast<const uint16_t*>(a->A);
    p->B = static_cast<const uint16_t*>(a->B);
    p->scale = a->scale;
    p->ranks = a->ranks;
    p->K = a->K;
    p->N = static_cast<int>(N);
    p->n_slots = a->n_slots;
    p->max_rank = a->max_rank;
    p->n_parts = a->n_parts;
    return PRQ_OK;
}

// [low, high] of YaRN's ramp over the pair index.
long double pair_of_turns(const prq_rope_opts& o, long double base, long double turns) {
    const long double two_pi = 2.0l * acosl(-1.0l);
    return o.rot_dim * logl(o.original_positions / (turns * two_pi)) / (2.0l * logl(base));
}

prq_status rotate(const prq_rope* r, const int32_t* positions, int M, const prq_heads* q, const prq_heads* k, bool norm, float eps, prq_dtype dtype,
                  prq_stream_t stream) {
    if (!r || !q || M < 0 || (dtype != PRQ_F32 && dtype != PRQ_BF16)) return PRQ_ERR_INVALID_ARG;
    if (norm && !(eps > 0.0f && std::isfinite(eps))) return PRQ_ERR_INVALID_ARG;
    if (M == 0) return PRQ_OK;
    RotateParams p;
    std::memset(&p, 0, sizeof(p));
    const prq_heads* in[2] = {q, k};
    const uintptr_t size = dtype == PRQ_F32 ? 4 : 2;
    long long heads = 0;
    for (int i = 0; i < 2; ++i) {
        if (!in[i] || in[i]->heads == 0) continue;
        const prq_heads& h = *in[i];
        if (h.heads < 0 || h.heads > (1 << 16) || !h.x || !h.out) return PRQ_ERR_INVALID_ARG;
        // results on top of one another (that no row meets another row's heads is the caller's part: any order of strides is open)
        if ((h.heads > 1 && std::llabs(h.hsout) < r->head_dim) || (M > 1 && std::llabs(h.ldout) < r->head_dim)) return PRQ_ERR_INVALID_ARG;
        if (h.x == h.out && (h.ldx != h.ldout || h.hsx != h.hsout)) return PRQ_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(h.x) % size || reinterpret_cast<uintptr_t>(h.out) % size) return PRQ_ERR_ALIGNMENT;
        if (norm && reinterpret_cast<uintptr_t>(h.weight) % 4) return PRQ_ERR_ALIGNMENT;
        p.t[i] = HeadRows{h.x, h.out, h.ldx, h.hsx, h.ldout, h.hsout, h.heads, norm ? h.weight : nullptr};
        heads += h.heads;
    }
    if (heads == 0) return PRQ_OK;
    if (!positions) return PRQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(positions) % 4) return PRQ_ERR_ALIGNMENT;
    int sms = 0, *status;   // (no wait of these kernels can run out)
    const prq_status st = current_device_ready(&sms, &status);
    if (st != PRQ_OK) return st;
    p.positions = positions;
    p.M = M;
    p.head_dim = r->head_dim;
    p.rot_dim = r->rot_dim;
    p.eps = eps;
    p.factor = static_cast<float>(r->attention_factor);
    std::memcpy(p.turns, r->turns, sizeof(p.turns));
    const cudaError_t e = launch_rotate_heads(p, r->layout == PRQ_ROPE_INTERLEAVED, norm, dtype == PRQ_BF16, sms, static_cast<cudaStream_t>(stream));
    count_launches(e == cudaSuccess);
    return e == cudaSuccess ? PRQ_OK : PRQ_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t prq_adapters_workspace_bytes(const prq_adapters* a, int M) {
    AdapterParams p;
    if (M < 1 || M >= kMaxAdapterRows || read_adapters(a, &p) != PRQ_OK) return 0;
    return adapters_workspace_bytes(M, p.n_slots, p.n_parts, p.max_rank, true);
}

prq_status prq_linear_adapters(const prq_adapters* a, const int32_t* row_adapter, const void* x, int M, int ldx, const void* base, int ldbase,
                               void* y, int ldy, prq_dtype y_dtype, void* workspace, size_t workspace_bytes, prq_stream_t stream) {
    AdapterParams p;
    std::memset(&p, 0, sizeof(p));
    prq_status st = read_adapters(a, &p);
    if (st != PRQ_OK) return st;
    if (M == 0) return PRQ_OK;
    if (M < 0 || M >= kMaxAdapterRows || (y_dtype != PRQ_F32 && y_dtype != PRQ_BF16) || !row_adapter || !x || !base || !y || !p.A || !p.B) return PRQ_ERR_INVALID_ARG;
    if (ldx < p.K || ldbase < p.N || ldy < p.N || (base == y && ldbase != ldy)) return PRQ_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(base) || !aligned16(y) || !aligned16(p.A) || !aligned16(p.B)) return PRQ_ERR_ALIGNMENT;
    const int unit = y_dtype == PRQ_F32 ? 4 : 8;
    if (ldx % 8 || ldbase % unit || ldy % unit) return PRQ_ERR_ALIGNMENT;
    for (const void* v : {static_cast<const void*>(row_adapter), static_cast<const void*>(p.scale), static_cast<const void*>(p.ranks)})
        if (reinterpret_cast<uintptr_t>(v) % 4) return PRQ_ERR_ALIGNMENT;
    const size_t need = adapters_workspace_bytes(M, p.n_slots, p.n_parts, p.max_rank, false);
    if (need) {
        if (!workspace || workspace_bytes < need) return PRQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return PRQ_ERR_ALIGNMENT;
    }
    int sms = 0;
    st = current_device_ready(&sms, &p.status);
    if (st != PRQ_OK) return st;
    p.row_adapter = row_adapter;
    p.x = static_cast<const uint16_t*>(x);
    p.base = base;
    p.y = y;
    p.h = workspace;
    p.ldx = ldx;
    p.ldbase = ldbase;
    p.ldy = ldy;
    p.M = M;
    // developer switch: lets a test watch a wait run out
    const int limit = developer_switch("PRQ_WAIT_LIMIT_CYCLES", 0);
    p.wait_limit = limit ? limit : kDefaultWaitLimitCycles;
    int launches = 0;
    const cudaError_t e = launch_adapters(p, y_dtype == PRQ_BF16, sms, static_cast<cudaStream_t>(stream), &launches);
    count_launches(launches);
    return e == cudaSuccess ? PRQ_OK : PRQ_ERR_CUDA;
}

prq_status prq_fold_adapter(const int32_t* perm, const float* s, int K, const uint16_t* A, int rows, uint16_t* out) {
    if (!perm || !s || !A || !out || K < 1 || rows < 1) return PRQ_ERR_INVALID_ARG;
    return fold_adapter(perm, s, K, A, rows, out);
}

prq_status prq_rope_create(const prq_rope_opts* opts, prq_rope** out) {
    if (!opts || !out || opts->struct_size < sizeof(prq_rope_opts)) return PRQ_ERR_INVALID_ARG;
    prq_rope_opts o = *opts;
    auto otherwise = [](double& v, double value) { if (v == 0.0) v = value; };
    if (o.rot_dim == 0) o.rot_dim = o.head_dim;
    otherwise(o.base, 10000.0);
    otherwise(o.factor, 1.0);
    if (o.head_dim < 2 || o.head_dim > 512 || o.rot_dim < 2 || o.rot_dim % 2 || o.rot_dim > o.head_dim || o.rot_dim > 2 * kMaxPairs) return PRQ_ERR_INVALID_ARG;
    if (o.layout != PRQ_ROPE_HALF && o.layout != PRQ_ROPE_INTERLEAVED) return PRQ_ERR_INVALID_ARG;
    if (!(o.base > 1.0) || !std::isfinite(o.base) || !(o.factor >= 1.0) || !std::isfinite(o.factor)) return PRQ_ERR_INVALID_ARG;
    const float attention_factor = static_cast<float>(o.attention_factor);   // (what a kernel multiplies by)
    if (!(o.attention_factor >= 0.0) || !std::isfinite(attention_factor) || (o.attention_factor > 0.0 && attention_factor == 0.0f)) return PRQ_ERR_INVALID_ARG;

    long double base = o.base, low = 0.0l, high = 0.0l, attention = 1.0l;
    const long double two_pi = 2.0l * acosl(-1.0l);
    switch (o.scaling) {
        case PRQ_ROPE_UNSCALED:
            o.factor = 1.0;
            break;
        case PRQ_ROPE_LINEAR:
            break;
        case PRQ_ROPE_BASE:
            if (o.rot_dim <= 2) return PRQ_ERR_INVALID_ARG;
            base *= powl(o.factor, static_cast<long double>(o.rot_dim) / (o.rot_dim - 2));
            break;
        case PRQ_ROPE_YARN:
            otherwise(o.beta_fast, 32.0);
            otherwise(o.beta_slow, 1.0);
            if (o.original_positions < 1 || !(o.beta_slow > 0.0) || !(o.beta_fast > o.beta_slow) || !std::isfinite(o.beta_fast)) return PRQ_ERR_INVALID_ARG;
            low = fmaxl(floorl(pair_of_turns(o, base, o.beta_fast)), 0.0l);
            high = fminl(ceill(pair_of_turns(o, base, o.beta_slow)), o.rot_dim - 1.0l);
            attention = 0.1l * logl(o.factor) + 1.0l;
            break;
        case PRQ_ROPE_WAVELENGTH:
            otherwise(o.low_factor, 1.0);
            otherwise(o.high_factor, 4.0);
            if (o.original_positions < 1 || !(o.low_factor > 0.0) || !(o.high_factor > o.low_factor) || !std::isfinite(o.high_factor)) return PRQ_ERR_INVALID_ARG;
            break;
        default:
            return PRQ_ERR_INVALID_ARG;
    }
    prq_rope* r = new (std::nothrow) prq_rope;
    if (!r) return PRQ_ERR_OOM;
    r->head_dim = o.head_dim;
    r->rot_dim = o.rot_dim;
    r->layout = o.layout;
    r->attention_factor = o.attention_factor > 0.0 ? o.attention_factor : static_cast<double>(attention);
    for (int i = 0; i < o.rot_dim / 2; ++i) {
        long double f = powl(base, -2.0l * i / o.rot_dim);
        if (o.scaling == PRQ_ROPE_LINEAR) {
            f /= o.factor;
        } else if (o.scaling == PRQ_ROPE_YARN || o.scaling == PRQ_ROPE_WAVELENGTH) {
            // share of the scaled frequency
            const long double t = o.scaling == PRQ_ROPE_YARN ? (i - low) / fmaxl(high - low, 0.001l)
                                                             : (o.high_factor - o.original_positions * f / two_pi) / (o.high_factor - o.low_factor);
            const long double share = fminl(fmaxl(t, 0.0l), 1.0l);
            f = f / o.factor * share + f * (1.0l - share);
        }
        r->f[i] = static_cast<double>(f);
        r->turns[i] = static_cast<uint64_t>(f / two_pi * 18446744073709551616.0l + 0.5l);   // f <= 1 radian: under a sixth of a turn
    }
    *out = r;
    return PRQ_OK;
}

void prq_rope_free(prq_rope* r) { delete r; }

prq_status prq_rope_frequencies(const prq_rope* r, double* f, double* attention_factor) {
    if (!r) return PRQ_ERR_INVALID_ARG;
    if (f) std::memcpy(f, r->f, sizeof(double) * (r->rot_dim / 2));
    if (attention_factor) *attention_factor = r->attention_factor;
    return PRQ_OK;
}

prq_status prq_rotate_heads(const prq_rope* r, const int32_t* positions, int M, const prq_heads* q, const prq_heads* k, prq_dtype dtype,
                            prq_stream_t stream) {
    return rotate(r, positions, M, q, k, false, 0.0f, dtype, stream);
}

prq_status prq_norm_rotate_heads(const prq_rope* r, const int32_t* positions, int M, const prq_heads* q, const prq_heads* k, float eps,
                                 prq_dtype dtype, prq_stream_t stream) {
    return rotate(r, positions, M, q, k, true, eps, dtype, stream);
}

}  // extern "C"
