// Low-rank adapters beside a projection: h = scale * x A^T with the adapter of each row, then y = base + h B^T.
//
// An item is rows of one adapter, from anywhere in a window of 4096 rows.  Few rows: one launch, in which a cluster has an item, sums its h and adds
// h B^T.  Many rows: two launches, the first one for h, the second one streams y past it.  Items are worked out on the device, so that a
// captured call follows its row table.  Sums are fp32; h goes into the second product as two bf16 terms (hi = bf16(h), lo = bf16(h - hi):
// 16 bits and more of its significand), whose products with B the tensor cores sum in fp32.  In a bf16 y the bits that are lost do not show; an
// fp32 y is off by 3.1 to 3.6e-7 of its size (97 rows of K = 9728, rank 32) where a product in fp32 is by 0.7 to 0.9e-7: a third term, half again as many
// products, would be the price of the rest.
//
// Up to rank 32 both products use mma.sync (16 x 8 x 16, bf16): they hold 16 to 64 flop per byte of y, too little for its rate to become the
// bound.  Rows may stand in any order, and sums stay in the registers of the lane that stores them.  The order of a reduction's elements is
// free, so the k index of every fragment is permuted such that a lane's share of a row is 16 (or 8) contiguous bytes in both operands.
// With higher ranks the loads of fragments from shared memory become the bound of y, and many tiles go through tcgen05.mma.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "prq_internal.h"
#include "prq_kernels.h"
#include "prq_ptx.cuh"

namespace prq {
namespace {

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// Eight columns of y as they are stored.
template <class T>
struct Columns {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = raw[i];
    }
    // the sum is rounded once, to nearest
    __device__ __forceinline__ void add(const float (&d)[8]) {
        if constexpr (sizeof(T) == 2) {
            uint32_t* w = &raw[0].x;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16(bf16_lo(w[i]) + d[2 * i], bf16_hi(w[i]) + d[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t* w = &raw[i / 4].x + i % 4;
                *w = __float_as_uint(__uint_as_float(*w) + d[i]);
            }
        }
    }
};

// ---------------------------------------------------------------- items
// Up to 16 rows each, or up to 128, so that A and B are read seldom and h and y have whole tiles.
constexpr int kFewRows = 16, kManyRows = 128;
constexpr int kFewCall = 512;         // rows of a call up to which items are small where one pass takes all ranks
constexpr int kWindow = 4096;         // rows that are put in the order of their adapters together
constexpr int kSortedSlots = 511;     // pools of more adapters, and calls of up to 32 rows: 32 rows that follow one another are grouped

struct __align__(16) Item {
    int slot, rows, rank, pad;        // rows: 0 -- no such item; rank: 0 -- no adapter
    int row[kManyRows];
};

constexpr int kItemsSoon = 24;        // items times passes that clusters of eight CTAs work off in two turns
// All ranks of all parts are summed in passes of up to 64, which small items take one after another and large ones at the same time.
int passes_of(int n_parts, int max_rank) { return (n_parts * ((max_rank + 15) & ~15) + 63) / 64; }
// Small items and one launch, or large ones and two: a rule on what the host knows, which is the pool's size and not what a batch uses of it.
// One pass: small up to 512 rows (o of 387 rows, rank 32: 10.1 us, with large items 12.0; gate / up of 512 rows, rank 16: 21 and 20; of 768: 28
// and 21), and wherever adapters may have fewer rows than such an item (q / k / v, rank 16, 1000 rows of a pool of 64: all of them in use 23 and 80,
// four in use 23 and 18; of a pool of 500 102 and 582, 23 and 18).  Several passes: large where there cannot be more items than clusters
// work off soon (q / k / v, rank 64, one row: 9.1 and 17 with a small item; 48 rows of a pool of 4: 10 to 12 and 21; of 8: 11 to 21 and 21),
// small where adapters may have few rows (200 rows of a pool of 64: all in use 46 and 130, four in use 38 and 14; 256 of a pool of 32: 36 and 71,
// 36 and 16).  And small where rows are put in order 32 at a time.
// What the rule costs where a large pool has four adapters in use (q / k / v, as it is, and in a pool of four): rank 16, 200 rows of a pool of 64 to
// 600 22 and 9 us, 1000 23 and 18, 4096 of a pool of 500 50 and 34, of 600 62; rank 64, 200 rows of a pool of 64 to 600 38 and 14, 1000 39
// and 28, 2000 of a pool of 200 or 500 79 and 43, 4096 of a pool of 500 163 and 68, of 600 183.
bool small_items(int M, int n_slots, int passes) {
    const long long room = static_cast<long long>(kFewRows) * n_slots;
    if (n_slots > kSortedSlots) return true;
    if (passes == 1) return M <= kFewCall || M < room;
    return (M < n_slots ? M : n_slots) * passes > kItemsSoon && M < room;
}
// rows per window, items that a window may have, windows, items in all
AdapterItems plan_items(int M, int n_slots, bool small) {
    AdapterItems t;
    if (n_slots > kSortedSlots) {
        t.window = M < 32 ? M : 32;
        t.per_window = t.window;
    } else {
        t.window = M < kWindow ? M : kWindow;
        const int kinds = n_slots + 1 < t.window ? n_slots + 1 : t.window;
        t.per_window = t.window / (small ? kFewRows : kManyRows) + kinds;   // whole ones, and a rest of each adapter
    }
    t.windows = static_cast<int>((M + static_cast<long long>(t.window) - 1) / t.window);
    t.n = t.windows * t.per_window;   // (under 2^23 rows: 31 bits hold that, and all grids)
    return t;
}

constexpr int kHThreads = 512, kHWarps = kHThreads / 32;

struct FindShared {
    uint16_t count[kHWarps][kSortedSlots + 1];   // rows per warp and adapter (the last one: none), then the rows in front of them
    int warp_items[kHWarps];
    int slot, first, rows, all, bare;   // all: items of the window; bare: those of them, the last ones, whose rows have no adapter
    int row[kManyRows];
};

// The CTA's item: the index-th one of the window at m0.  Every thread keeps up to eight rows and their places among the rows of
// their adapter (a warp's rows follow one another, so that the order is that of the rows and a prompt's stay together).
template <int kItemRows, int kSteps>
__device__ __forceinline__ void find_item(const AdapterParams& p, int m0, int n, int index, FindShared& f) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kinds = p.n_slots + 1;
    const int steps = (n + kHThreads - 1) / kHThreads, begin = warp * steps * 32;
    int slot[kSteps], place[kSteps];
    unsigned same[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int m = begin + 32 * s + lane;
        slot[s] = -1;
        if (s < steps && m < n) slot[s] = p.row_adapter[m0 + m];
    }
    for (int i = lane; i < kinds; i += 32) f.count[warp][i] = 0;
    if (threadIdx.x == 0) f.rows = 0;
    __syncwarp();
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (s >= steps) break;
        const bool inside = begin + 32 * s + lane < n;
        if (inside && static_cast<unsigned>(slot[s]) >= static_cast<unsigned>(p.n_slots)) slot[s] = p.n_slots;
        if (!inside) slot[s] = -1;
        same[s] = __match_any_sync(0xffffffffu, slot[s]);
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (s >= steps) break;
        const int leader = __ffs(same[s]) - 1;
        int at = 0;
        if (lane == leader && slot[s] >= 0) {
            at = f.count[warp][slot[s]];
            f.count[warp][slot[s]] = static_cast<uint16_t>(at + __popc(same[s]));
        }
        place[s] = __shfl_sync(0xffffffffu, at, leader) + __popc(same[s] & ((1u << lane) - 1));
        __syncwarp();
    }
    __syncthreads();
    // a thread per adapter: its rows in front of each warp, its items, and the items of the adapters before it
    int rows = 0;
    const int kind = threadIdx.x;
    if (kind < kinds) {
#pragma unroll
        for (int w = 0; w < kHWarps; ++w) {
            const int c = f.count[w][kind];
            f.count[w][kind] = static_cast<uint16_t>(rows);
            rows += c;
        }
    }
    const int items = (rows + kItemRows - 1) / kItemRows;
    int sum = items;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 31) f.warp_items[warp] = sum;
    __syncthreads();
    int first = sum - items;
#pragma unroll
    for (int w = 0; w < kHWarps; ++w) first += w < warp ? f.warp_items[w] : 0;
    if (kind == kinds - 1) {
        f.all = first + items;
        f.bare = items;
    }
    if (index >= first && index < first + items) {
        f.slot = kind;
        f.first = (index - first) * kItemRows;
        f.rows = min(kItemRows, rows - f.first);
    }
    __syncthreads();
    if (f.rows > 0) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s >= steps) break;
            if (slot[s] != f.slot) continue;
            const int at = f.count[warp][slot[s]] + place[s] - f.first;
            if (at >= 0 && at < kItemRows) f.row[at] = m0 + begin + 32 * s + lane;
        }
    }
    __syncthreads();
}

// The same for small items within 32 rows that follow one another, for any number of adapters, by one warp: items in the order of their
// first rows, those without an adapter last.
__device__ __forceinline__ void find_item_of_32(const AdapterParams& p, int m0, int n, int index, FindShared& f) {
    constexpr int kItemRows = kFewRows;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int slot = lane < n ? p.row_adapter[m0 + lane] : -2;
        if (lane < n && static_cast<unsigned>(slot) >= static_cast<unsigned>(p.n_slots)) slot = -1;
        const unsigned same = __match_any_sync(0xffffffffu, slot), before = (1u << lane) - 1;
        const int nth = __popc(same & before);
        const bool leads = lane < n && nth % kItemRows == 0;
        const unsigned leaders = __ballot_sync(0xffffffffu, leads), bare = __ballot_sync(0xffffffffu, leads && slot < 0), other = leaders & ~bare;
        const bool chosen = leads && (slot < 0 ? __popc(other) + __popc(bare & before) : __popc(other & before)) == index;
        const unsigned who = __ballot_sync(0xffffffffu, chosen);
        if (lane == 0) {
            f.rows = 0;
            f.all = __popc(leaders);
            f.bare = __popc(bare);
        }
        __syncwarp();
        if (who) {
            const int first = __shfl_sync(0xffffffffu, nth, __ffs(who) - 1);
            if ((same & who) && nth >= first && nth < first + kItemRows) f.row[nth - first] = m0 + lane;
            if (chosen) {
                f.slot = slot;
                f.rows = min(kItemRows, __popc(same) - nth);
            }
        }
    }
    __syncthreads();
}

struct Workspace {
    int* counts;       // items of each window that have something to do: its first ones
    Item* items;
    uint4* h;          // M x ranks / 4: (hi, lo) of four ranks
};
__host__ __device__ inline size_t counts_bytes(const AdapterItems& t) { return (sizeof(int) * t.windows + 15) / 16 * 16; }
__host__ __device__ inline Workspace views(void* at, const AdapterItems& t) {
    Item* items = reinterpret_cast<Item*>(static_cast<uint8_t*>(at) + counts_bytes(t));
    return Workspace{static_cast<int*>(at), items, reinterpret_cast<uint4*>(items + t.n)};
}

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

// ---------------------------------------------------------------- h
// An item and 8 kRankTiles ranks at a time per cluster, whose CTAs split K.  Rows of x and of A come into a ring in shared memory, kStageK of K
// at a time; a warp has 16 rows and one 32 of K in kWarpsK.  (With items of 16 rows a stage has 32s of K for eight of the 16 warps; the others' sums
// are zeros.)  Few rows: what is on its way at once sets the pace (a CTA's share of K is a few stages), so the pieces are long.  Row stride in the ring: 64 bytes off a multiple of 128, so that the eight lanes of a 16-byte load (two
// rows, four lanes each) meet no bank twice.
template <int kRankTiles, int kItemRows>
struct HShared {
    static constexpr int kRanks = 8 * kRankTiles, kRows = kItemRows + kRanks;
    static constexpr int kStageK = kItemRows == kFewRows ? 256 : 128, kStages = kItemRows == kFewRows && kRankTiles <= 6 ? 4 : 3;
    static constexpr int kRowBytes = 2 * kStageK + 64, kTiles = kItemRows / 16, kWarpsK = kHWarps / kTiles;
    union {
        uint8_t ring[kStages][kRows][kRowBytes];
        FindShared find;
        float part[kWarpsK][kItemRows][kRanks + 4];   // sums of the warps
    };
    int row[kItemRows];
};
struct Found { int slot, rows, rank, all, bare; };
// The nth item of a window, its rows in sh.row.
template <int kRankTiles, int kItemRows>
__device__ __forceinline__ Found find(const AdapterParams& p, int window, int nth, HShared<kRankTiles, kItemRows>& sh) {
    const int m0 = window * p.items.window, n = min(p.items.window, p.M - m0);
    if (kItemRows == kFewRows && (p.n_slots > kSortedSlots || p.M <= 32)) find_item_of_32(p, m0, n, nth, sh.find);
    else if (kItemRows == kFewRows && n <= kHThreads) find_item<kItemRows, 1>(p, m0, n, nth, sh.find);   // (what is executed once counts by its instructions' way here, too)
    else find_item<kItemRows, kWindow / kHThreads>(p, m0, n, nth, sh.find);
    Found f{sh.find.slot, sh.find.rows, 0, sh.find.all, sh.find.bare};
    if (static_cast<int>(threadIdx.x) < f.rows) sh.row[threadIdx.x] = sh.find.row[threadIdx.x];
    if (f.rows > 0 && f.slot >= 0 && f.slot < p.n_slots) f.rank = p.ranks ? min(max(p.ranks[f.slot], 0), p.max_rank) : p.max_rank;
    __syncthreads();   // (the ring takes the table's memory)
    return f;
}
__device__ __forceinline__ int part_of(int f, int pad_rank) { return (f >= pad_rank) + (f >= 2 * pad_rank) + (f >= 3 * pad_rank); }

// Sums of the warps over this CTA's share of K, for ranks r0 .. (of all parts, padded), left in sh.part.
template <int kRankTiles, int kItemRows>
__device__ __forceinline__ void sum_h(const AdapterParams& p, const Found& item, int r0, int cta, int ctas, HShared<kRankTiles, kItemRows>& sh) {
    using Shared = HShared<kRankTiles, kItemRows>;
    constexpr int kRows = Shared::kRows, kStageK = Shared::kStageK, kStages = Shared::kStages, kRowBytes = Shared::kRowBytes;
    constexpr int kTiles = Shared::kTiles, kWarpsK = Shared::kWarpsK;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int steps = item.rank > 0 ? p.K / 32 : 0, k0 = steps * cta / ctas * 32, k1 = steps * (cta + 1) / ctas * 32;
    const int stages = (k1 - k0 + kStageK - 1) / kStageK;
    // a thread has the same 16 bytes of every kAtOnce-th row in each stage
    constexpr int kPieces = kStageK / 8, kAtOnce = kHThreads / kPieces, kMine = (kRows + kAtOnce - 1) / kAtOnce;
    const int piece = threadIdx.x % kPieces, my_row = threadIdx.x / kPieces;
    const uint16_t* from[kMine];   // null: no such row
    const uint16_t* A = p.A + static_cast<long long>(item.slot) * p.n_parts * p.max_rank * p.K + k0 + 8 * piece;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int r = my_row + i * kAtOnce;
        from[i] = nullptr;
        if (i * kAtOnce < kItemRows) {   // (kItemRows is a multiple of kAtOnce)
            if (r < item.rows) from[i] = p.x + sh.row[r] * p.ldx + k0 + 8 * piece;
        } else {
            const int f = r0 + r - kItemRows, part = part_of(f, p.pad_rank), k = f - part * p.pad_rank;
            if (r < kRows && part < p.n_parts && k < item.rank) from[i] = A + static_cast<long long>(part * p.max_rank + k) * p.K;
        }
    }
    static_assert(kItemRows % kAtOnce == 0, "rows of x and of A in different turns");
    const uint32_t to = smem_u32(sh.ring[0][0]) + my_row * kRowBytes + 16 * piece;
    auto ask = [&](int stage, int place) {
        if (stage < stages && k0 + stage * kStageK + 8 * piece < k1) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                if (from[i]) copy16(to + place * (kRows * kRowBytes) + i * kAtOnce * kRowBytes, from[i] + stage * kStageK);
            }
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) ask(i, i);

    float acc[kRankTiles][4];
#pragma unroll
    for (int t = 0; t < kRankTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = 0.0f;
    const int tile = warp % kTiles, kw = warp / kTiles;
    int place = 0;
    for (int s = 0; s < stages; ++s) {
        copies_wait<kStages - 2>();
        __syncthreads();   // this stage is there for all, and the one before it has been read
        ask(s + kStages - 1, place == 0 ? kStages - 1 : place - 1);
        const int here = min(kStageK, k1 - k0 - s * kStageK);
        if (tile * 16 < item.rows) {
            const uint8_t* at = sh.ring[place][0] + 16 * q;
#pragma unroll
            for (int k = 32 * kw; k < kStageK; k += 32 * kWarpsK) {   // (what ranks and rows that do not exist leave there reaches no sum that is read)
                if (k >= here) break;
                const uint4 va = *reinterpret_cast<const uint4*>(at + (16 * tile + g) * kRowBytes + 2 * k);
                const uint4 vb = *reinterpret_cast<const uint4*>(at + (16 * tile + 8 + g) * kRowBytes + 2 * k);
#pragma unroll
                for (int t = 0; t < kRankTiles; ++t) {
                    const uint4 a = *reinterpret_cast<const uint4*>(at + (kItemRows + 8 * t + g) * kRowBytes + 2 * k);
                    mma_bf16(acc[t], va.x, vb.x, va.y, vb.y, a.x, a.y);
                    mma_bf16(acc[t], va.z, vb.z, va.w, vb.w, a.z, a.w);
                }
            }
        }
        place = place == kStages - 1 ? 0 : place + 1;
    }
    copies_wait<0>();
    __syncthreads();
    if (tile * 16 < item.rows) {
#pragma unroll
        for (int t = 0; t < kRankTiles; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<float2*>(&sh.part[kw][16 * tile + 8 * k + g][8 * t + 2 * q]) = make_float2(acc[t][2 * k], acc[t][2 * k + 1]);
    }
    __syncthreads();
}
// The CTA's sum of ranks j .. j + 3 of row m.
template <class Shared>
__device__ __forceinline__ float4 cta_sum(const Shared& sh, int m, int j) {
    float4 sum = *reinterpret_cast<const float4*>(&sh.part[0][m][j]);
#pragma unroll
    for (int k = 1; k < Shared::kWarpsK; ++k) {
        const float4 u = *reinterpret_cast<const float4*>(&sh.part[k][m][j]);
        sum.x += u.x; sum.y += u.y; sum.z += u.z; sum.w += u.w;
    }
    return sum;
}
// Four sums, of ranks r .. r + 3 of a part, scaled and split in two terms; nothing behind the adapter's rank.
__device__ __forceinline__ uint4 two_terms(float4 sum, float scale, int r, int rank) {
    const float v[4] = {r < rank ? sum.x * scale : 0.0f, r + 1 < rank ? sum.y * scale : 0.0f, r + 2 < rank ? sum.z * scale : 0.0f, r + 3 < rank ? sum.w * scale : 0.0f};
    uint4 h;
    h.x = pack_bf16(v[0], v[1]);
    h.y = pack_bf16(v[2], v[3]);
    const auto rest = [](float v, float hi) { return fabsf(hi) <= 3.4e38f ? v - hi : 0.0f; };   // (an infinite sum stays one)
    h.z = pack_bf16(rest(v[0], bf16_lo(h.x)), rest(v[1], bf16_hi(h.x)));
    h.w = pack_bf16(rest(v[2], bf16_lo(h.y)), rest(v[3], bf16_hi(h.y)));
    return h;
}

// Many rows: h of an item goes to the workspace, for the second launch.  4096 rows of q / k / v (K = 2560), rank 16: 15 us, of which the loop over
// K takes 7 (21 MB of x), finding the rows 2.4, set-up 1, the first loads 1.6, the cluster's exchange 3.  Every CTA pushes its sums to
// the one that adds them up; fetching them took 2 us more.
// kOnce: there is a cluster for each item that there could be.  (The loop over items costs registers: 0.3 to 0.6 us per call.)
template <int kRankTiles>
struct ManyHShared : HShared<kRankTiles, kManyRows> {
    float4 got[kManyRows * 8 * kRankTiles / 4 + 8];   // sums of the cluster's CTAs for this CTA's share of them, one CTA behind the other
    int todo;                                         // items of the window that have something to do, as the cluster's first CTA found them
};
template <int kRankTiles, bool kOnce>
__global__ void __launch_bounds__(kHThreads, 1) adapters_many_h_kernel(const __grid_constant__ AdapterParams p) {
    using Shared = ManyHShared<kRankTiles>;
    constexpr int kRanks = Shared::kRanks;
    extern __shared__ __align__(128) uint8_t smem[];
    Shared& sh = *reinterpret_cast<Shared*>(smem);
    const int ctas = p.cluster, cta = cluster_ctarank(), r0 = blockIdx.y * kRanks, ranks = p.n_parts * p.pad_rank;
    const int window = blockIdx.x / ctas / p.h_clusters, begin = blockIdx.x / ctas - window * p.h_clusters;
    const Workspace ws = views(p.h, p.items);
    grid_dependency_wait();
    grid_launch_dependents();
    int nth = begin;
    while (true) {
        if (ctas > 1) cluster_arrive();   // (the others' shared memory may be written to once all have come by here)
        const Found item = find<kRankTiles, kManyRows>(p, window, nth, sh);
        const int todo = p.base == p.y ? item.all - item.bare : item.all;
        if (cta == 0 && blockIdx.y == 0) {
            Item& to = ws.items[window * p.items.per_window + nth];
            if (static_cast<int>(threadIdx.x) < item.rows) to.row[threadIdx.x] = sh.row[threadIdx.x];
            if (threadIdx.x == 0) {
                *reinterpret_cast<int4*>(&to) = make_int4(item.slot, item.rows, item.rank, 0);
                if (nth == 0) ws.counts[window] = todo;
            }
        }
        // (a cluster without work meets all the same: the number of meetings does not depend on what each CTA read, but on what its first one did)
        sum_h<kRankTiles, kManyRows>(p, item, r0, cta, ctas, sh);
        // the cluster's sums: a share of them in each CTA
        const int quads = (item.rank > 0 ? item.rows : 0) * (kRanks / 4), share = (quads + ctas - 1) / ctas;
        const float to_share = share > 0 ? 1.0f / share : 0.0f;
        if (ctas > 1) cluster_wait();
        for (int i = threadIdx.x; i < quads; i += kHThreads) {
            const int c = __float2int_rd((i + 0.5f) * to_share);   // i / share (i + 0.5 is 2^-13 of itself and more away from a border)
            st_cluster(cluster_map(smem_u32(&sh.got[cta * share + i - c * share]), c), cta_sum(sh, i / (kRanks / 4), i % (kRanks / 4) * 4));
        }
        if (!kOnce && cta == 0 && static_cast<int>(threadIdx.x) < ctas) st_cluster(cluster_map(smem_u32(&sh.todo), threadIdx.x), todo);
        const float scale = item.rank > 0 && p.scale ? p.scale[item.slot] : 1.0f;
        if (ctas > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        const int i0 = min(quads, share * cta), mine = min(quads, i0 + share) - i0;
        for (int i = threadIdx.x; i < mine; i += kHThreads) {
            const int m = (i0 + i) / (kRanks / 4), f = r0 + (i0 + i) % (kRanks / 4) * 4;
            if (f >= ranks) continue;
            float4 sum = sh.got[i];
            for (int k = 1; k < ctas; ++k) {
                const float4 u = sh.got[k * share + i];
                sum.x += u.x; sum.y += u.y; sum.z += u.z; sum.w += u.w;
            }
            ws.h[static_cast<long long>(sh.row[m]) * (ranks / 4) + f / 4] = two_terms(sum, scale, f - part_of(f, p.pad_rank) * p.pad_rank, item.rank);
        }
        nth += p.h_clusters;
        if (kOnce || nth >= sh.todo) break;
        __syncthreads();   // (rows and sums have been read)
    }
}

// ---------------------------------------------------------------- y
// In both forms a lane has eight columns that follow one another: column 2 q + e of the j-th 8-column fragment stands for column 8 q + 2 j + e
// of a block of 32.  bf16: the accumulators begin with base (their sum is cut to 24 bits, and then rounded to 8); fp32: base is added to
// the sum.  What lies behind an adapter's rank may be anything: `masked` clears it in a lane's four ranks of B.
__device__ __forceinline__ uint2 masked(uint2 b, int left) {
    b.x &= left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u;
    b.y &= left >= 4 ? 0xffffffffu : left == 3 ? 0xffffu : 0u;
    return b;
}
template <class T>
__device__ __forceinline__ void begin_sum(float (&acc)[4][4], const Columns<T>& v, int e) {   // e: 0 -- row g, 2 -- row g + 8
    if constexpr (sizeof(T) == 2) {
        const uint32_t w[4] = {v.raw[0].x, v.raw[0].y, v.raw[0].z, v.raw[0].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            acc[j][e] = bf16_lo(w[j]);
            acc[j][e + 1] = bf16_hi(w[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j][e] = acc[j][e + 1] = 0.0f;
    }
}
template <class T>
__device__ __forceinline__ Columns<T> end_sum(const float (&acc)[4][4], const Columns<T>& v, int e) {
    Columns<T> to;
    if constexpr (sizeof(T) == 2) {
        to.raw[0] = make_uint4(pack_bf16(acc[0][e], acc[0][e + 1]), pack_bf16(acc[1][e], acc[1][e + 1]), pack_bf16(acc[2][e], acc[2][e + 1]),
                               pack_bf16(acc[3][e], acc[3][e + 1]));
    } else {
        const float d[8] = {acc[0][e], acc[0][e + 1], acc[1][e], acc[1][e + 1], acc[2][e], acc[2][e + 1], acc[3][e], acc[3][e + 1]};
        to = v;
        to.add(d);
    }
    return to;
}
// The last columns of a matrix whose width is no multiple of eight (their accumulators began with zero).
template <class T>
__device__ __forceinline__ void add_last(const float (&acc)[4][4], int e, int cols, const T* from, T* to) {
#pragma unroll
    for (int n = 0; n < 8; ++n)
        if (n < cols) to[n] = static_cast<T>(static_cast<float>(from[n]) + acc[n / 2][e + (n & 1)]);
}
// Part and columns of the unit-th `width` columns of y (p.unit_end: units up to the end of each part).
struct Unit { int part, n0, end; };
__device__ __forceinline__ Unit unit_of(const AdapterParams& p, int unit, int width) {
    int part = 0, first = 0, from = 0;
#pragma unroll
    for (int i = 0; i < kMaxBatch - 1; ++i)
        if (unit >= p.unit_end[i]) {   // (of parts that do not exist: all units)
            part = i + 1;
            first = p.unit_end[i];
            from = p.part_end[i];
        }
    return Unit{part, from + width * (unit - first), p.part_end[part]};
}
// Rows without an adapter, where y is not base: copied bit for bit.
template <class T>
__device__ __forceinline__ void copy_rows(const AdapterParams& p, const int* row, int rows, int n0, int n1, int thread, int threads) {
    constexpr int kPiece = 16 / sizeof(T);
    const int pieces = (n1 - n0 + kPiece - 1) / kPiece;
    for (int i = thread; i < rows * pieces; i += threads) {
        const int m = i / pieces, n = n0 + (i - m * pieces) * kPiece;
        const T* from = static_cast<const T*>(p.base) + row[m] * p.ldbase + n;
        T* to = static_cast<T*>(p.y) + row[m] * p.ldy + n;
        if (n + kPiece <= n1) {
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
        } else {
            for (int j = 0; n + j < n1; ++j) to[j] = from[j];
        }
    }
}

// Few rows: one launch.  Every CTA of an item's cluster gets all of its sums, and a share of the columns: 64 per warp, straight from memory.
// Bound by a chain of latencies, not by bytes: one row of q / k / v, rank 16, 7.0 us (finding it 1, loads of x and A 2, exchange 1, loads of
// B and base, products and stores 2); 64 rows with 58 adapters 15.3 us, 27 MB.  Two launches took 7.1 and 18.9.
template <int kRankTiles>
struct FewShared : HShared<kRankTiles, kFewRows> {
    uint4 h[kFewRows * PRQ_MULTI_MAX * PRQ_ADAPTER_MAX_RANK / 4];   // [rank / 4][row]
    float4 got[8][kFewRows * 8 * kRankTiles / 4];                    // from each CTA of the cluster
    int todo;                                                        // as above
};
template <class T, int kRankTiles, bool kOnce>
__global__ void __launch_bounds__(kHThreads, 1) adapters_few_kernel(const __grid_constant__ AdapterParams p, int passes, int units) {
    using Shared = FewShared<kRankTiles>;
    constexpr int kRanks = Shared::kRanks;
    extern __shared__ __align__(128) uint8_t smem[];
    Shared& sh = *reinterpret_cast<Shared*>(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int ctas = p.cluster, cta = cluster_ctarank(), pad_rank = p.pad_rank, ranks = p.n_parts * pad_rank;
    const int window = blockIdx.x / ctas / p.h_clusters;
    int nth = blockIdx.x / ctas - window * p.h_clusters;
    grid_dependency_wait();
    grid_launch_dependents();
    while (true) {
        if (ctas > 1) cluster_arrive();   // (the others' shared memory may be written to once all have come by here)
        const Found item = find<kRankTiles, kFewRows>(p, window, nth, sh);
        const int rows = item.rows, rank = item.rank, stride = ctas * kHWarps;
        if (rank > 0) {
            // this warp's columns' share of B is on its way into L2 meanwhile
            for (int unit = cta * kHWarps + warp + lane * stride; unit < units; unit += 32 * stride) {
                const Unit at = unit_of(p, unit, 64);
                prefetch_l2(p.B + (static_cast<long long>(item.slot) * p.N + at.n0) * p.max_rank, min(64, at.end - at.n0) * p.max_rank * 2);
            }
        }
        const float scale = rank > 0 && p.scale ? p.scale[item.slot] : 1.0f;
        const int quads = rank > 0 ? rows * (kRanks / 4) : 0;
        // (a cluster without work meets all the same, so that the number of meetings does not depend on what each CTA read)
        for (int pass = 0; pass < passes; ++pass) {
            sum_h<kRankTiles, kFewRows>(p, item, pass * kRanks, cta, ctas, sh);
            if (ctas > 1) cluster_wait();
            for (int i = threadIdx.x; i < quads; i += kHThreads) {
                const float4 sum = cta_sum(sh, i / (kRanks / 4), i % (kRanks / 4) * 4);
                for (int c = 0; c < ctas; ++c) st_cluster(cluster_map(smem_u32(&sh.got[cta][i]), c), sum);
            }
            if (!kOnce && cta == 0 && static_cast<int>(threadIdx.x) < ctas) st_cluster(cluster_map(smem_u32(&sh.todo), threadIdx.x), p.base == p.y ? item.all - item.bare : item.all);
            if (ctas > 1) {
                cluster_arrive();
                cluster_wait();
            } else {
                __syncthreads();
            }
            for (int i = threadIdx.x; i < quads; i += kHThreads) {
                const int m = i / (kRanks / 4), f = pass * kRanks + i % (kRanks / 4) * 4;
                if (f >= ranks) continue;
                float4 sum = sh.got[0][i];
                for (int c = 1; c < ctas; ++c) {
                    const float4 u = sh.got[c][i];
                    sum.x += u.x; sum.y += u.y; sum.z += u.z; sum.w += u.w;
                }
                sh.h[f / 4 * kFewRows + m] = two_terms(sum, scale, f - part_of(f, pad_rank) * pad_rank, rank);
            }
            __syncthreads();
            if (ctas > 1 && pass + 1 < passes) cluster_arrive();   // (what was got has been read)
        }

        const bool mine[2] = {g < rows, 8 + g < rows};
        // (lanes whose row does not exist load and store nothing)
        const long long row[2] = {mine[0] ? sh.row[g] : 0, mine[1] ? sh.row[8 + g] : 0};
#pragma unroll 1
        for (int unit = cta * kHWarps + warp; unit < units && rows > 0; unit += stride) {
            const Unit at = unit_of(p, unit, 64);
            if (rank == 0) {
                if (p.base != p.y) copy_rows<T>(p, sh.row, rows, at.n0, min(at.end, at.n0 + 64), lane, 32);
                continue;
            }
            Columns<T> v[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = at.n0 + 32 * j + 8 * q;
                    v[i][j] = Columns<T>{};
                    if (mine[i] && col + 8 <= at.end) v[i][j].load(static_cast<const T*>(p.base) + row[i] * p.ldbase + col);
                }
            float acc[2][4][4];
            const uint16_t* B = p.B + (static_cast<long long>(item.slot) * p.N + at.n0 + 8 * (g >> 1) + (g & 1)) * p.max_rank + 4 * q;
            const uint4* H = sh.h + (at.part * (pad_rank / 4) + q) * kFewRows + g;
            const int n_left = at.end - at.n0 - 8 * (g >> 1) - (g & 1);   // columns of this lane's row of B up to the end
#pragma unroll 1
            for (int k = 0; k < rank; k += 16) {
                const int left = rank - k - 4 * q;
                uint2 b[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int n = 32 * (j / 4) + 2 * (j % 4);
                    b[j] = make_uint2(0, 0);
                    if (n < n_left && left > 0) b[j] = *reinterpret_cast<const uint2*>(B + static_cast<long long>(n) * p.max_rank + k);
                }
                const uint4 ha = H[k / 4 * kFewRows], hb = H[k / 4 * kFewRows + 8];   // (of a row that does not exist: reaches no sum that is stored)
                if (k == 0) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 2; ++i) begin_sum<T>(acc[j], v[i][j], 2 * i);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (left < 4) b[j] = masked(b[j], left);
                    mma_bf16(acc[j / 4][j % 4], ha.x, hb.x, ha.y, hb.y, b[j].x, b[j].y);
                    mma_bf16(acc[j / 4][j % 4], ha.z, hb.z, ha.w, hb.w, b[j].x, b[j].y);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = at.n0 + 32 * j + 8 * q, cols = at.end - col;
                    if (!mine[i] || cols <= 0) continue;
                    T* to = static_cast<T*>(p.y) + row[i] * p.ldy + col;
                    if (cols >= 8) end_sum<T>(acc[j], v[i][j], 2 * i).store(to);
                    else add_last<T>(acc[j], 2 * i, cols, static_cast<const T*>(p.base) + row[i] * p.ldbase + col, to);
                }
        }
        nth += p.h_clusters;
        if (kOnce || nth >= sh.todo) break;
        __syncthreads();   // (rows and sums have been read)
    }
}

// Many rows: a CTA has every y_items-th item of a window, and `span` tiles of kCols columns of one part.  4096 rows of q / k / v in place, rank
// 16: 25 us for 101 MB, 4 TB/s (a copy in place of that pattern takes 20 to 22).  It waits for its loads (the long scoreboard is the largest
// stall); no pipe is more than a third busy, and HBM a quarter when the launch stands alone.  Tiles of base and B come into a ring in shared memory; a
// warp has 16 of the item's rows, whose h it keeps in registers, and all columns.  In the ring a row of B stands where the fragment's
// lane wants it (row n of a block of 32 at 8 ((n % 8) / 2) + 2 (n / 8) + n % 2), with a stride of 32 bytes off a multiple of 64; of base,
// odd rows have the halves of their 128 bytes swapped: no lane of a load meets another one's bank.
constexpr int kManyThreads = 256, kManyStages = 3;
template <class T>
constexpr int kManyCols = 128 / sizeof(T);                           // 128 bytes of y per row and tile
__host__ __device__ inline int b_stride(int max_rank) { return 2 * ((max_rank + 15) & ~15) + (max_rank % 32 <= 16 && max_rank % 32 > 0 ? 0 : 32); }
template <class T>
__host__ __device__ inline int many_stage_bytes(int max_rank) { return kManyRows * 128 + kManyCols<T> * b_stride(max_rank); }

template <class T, int kSteps16>
__global__ void __launch_bounds__(kManyThreads, kSteps16 == 1 ? 3 : 2) adapters_many_y_kernel(const __grid_constant__ AdapterParams p, int units, int span) {
    constexpr int kCols = kManyCols<T>, kBlocks = kCols / 32, kPieceCols = 16 / sizeof(T);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ const T* base_s[kManyRows];
    __shared__ int row_s[kManyRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int pad_rank = p.pad_rank, quads = p.n_parts * pad_rank / 4, stride = b_stride(p.max_rank), stage_bytes = many_stage_bytes<T>(p.max_rank);
    const Workspace ws = views(p.h, p.items);
    const int turn = blockIdx.x / units, window = turn / p.y_items;
    const Unit at = unit_of(p, blockIdx.x - turn * units, kCols * span);
    const int stop = min(at.end, at.n0 + kCols * span), tiles = (stop - at.n0 + kCols - 1) / kCols;
    grid_dependency_wait();
    grid_launch_dependents();
    for (int nth = turn - window * p.y_items, todo = 0x7fffffff; nth < todo; nth += p.y_items) {
        const Item& item = ws.items[window * p.items.per_window + nth];
        todo = ws.counts[window];
        const int4 head = *reinterpret_cast<const int4*>(&item);
        const int listed = threadIdx.x < kManyRows ? item.row[threadIdx.x] : 0;
        const int slot = head.x, rows = head.y, rank = head.z;
        if (nth >= todo) return;
        if (rank == 0) {
            if (p.base != p.y) copy_rows<T>(p, item.row, rows, at.n0, stop, threadIdx.x, kManyThreads);
            continue;
        }
        if (static_cast<int>(threadIdx.x) < rows) {
            row_s[threadIdx.x] = listed;
            base_s[threadIdx.x] = static_cast<const T*>(p.base) + listed * p.ldbase + at.n0;
        }
        __syncthreads();

        // a thread copies one piece of every kRowStep-th row of base, and of one row of B one in kBThreads
        constexpr int kRowStep = kManyThreads / 8, kBThreads = kManyThreads / kCols;
        const int piece = threadIdx.x & 7, b_row = threadIdx.x / kBThreads, in = b_row & 31;
        const T* base_from[kManyRows / kRowStep];
#pragma unroll
        for (int i = 0; i < kManyRows / kRowStep; ++i) {
            const int r = (threadIdx.x >> 3) + i * kRowStep;
            base_from[i] = r < rows ? base_s[r] + piece * kPieceCols : nullptr;
        }
        const uint32_t base_to = smem_u32(smem) + (threadIdx.x >> 3) * 128 + 16 * (piece ^ ((threadIdx.x >> 3 & 1) << 2));   // (kRowStep is even)
        const uint16_t* b_from = p.B + (static_cast<long long>(slot) * p.N + at.n0 + b_row) * p.max_rank + 8 * (threadIdx.x % kBThreads);
        const uint32_t b_to = smem_u32(smem) + kManyRows * 128 + ((b_row & ~31) + 8 * ((in & 7) >> 1) + 2 * (in >> 3) + (in & 1)) * stride + 16 * (threadIdx.x % kBThreads);
        const int b_pieces = p.max_rank / 8 - threadIdx.x % kBThreads, width = stop - at.n0;
        auto ask = [&](int tile, int place) {
            const int n = tile * kCols;
            if (n + (piece + 1) * kPieceCols <= width) {
#pragma unroll
                for (int i = 0; i < kManyRows / kRowStep; ++i)
                    if (base_from[i]) copy16(base_to + place * stage_bytes + i * (kRowStep * 128), base_from[i] + n);
            }
            if (n + b_row < width) {
                const uint16_t* b = b_from + static_cast<long long>(n) * p.max_rank;
                for (int i = 0; i < b_pieces; i += kBThreads) copy16(b_to + place * stage_bytes + 16 * i, b + 8 * i);
            }
            copies_commit();
        };
#pragma unroll
        for (int i = 0; i < kManyStages - 1; ++i) ask(i, i);

        // h of rows g and 8 + g of the warp's 16 (of a row that exists, where they do not)
        const int ra = 16 * warp + g, rb = ra + 8;
        const bool working = 16 * warp < rows, has_a = ra < rows, has_b = rb < rows;
        const long long ma = working ? row_s[has_a ? ra : 0] : 0, mb = working ? row_s[has_b ? rb : 0] : 0;
        uint4 ha[kSteps16], hb[kSteps16];
        if (working) {
            const uint4* H = ws.h + at.part * (pad_rank / 4) + q;
#pragma unroll
            for (int k = 0; k < kSteps16; ++k) {
                ha[k] = hb[k] = make_uint4(0, 0, 0, 0);
                if (16 * k < rank) {
                    ha[k] = H[ma * quads + 4 * k];
                    hb[k] = H[mb * quads + 4 * k];
                }
            }
        }
        T* ya = static_cast<T*>(p.y) + ma * p.ldy + at.n0 + 8 * q;
        T* yb = static_cast<T*>(p.y) + mb * p.ldy + at.n0 + 8 * q;
        const uint32_t swap = (ra & 1) << 6;   // (rb's is the same)
        int place = 0;
        // one tile; `whole`: all of its columns, and all of the rank's steps, exist
        auto one_tile = [&](int tile, auto whole) {
            constexpr bool kWhole = decltype(whole)::value;
            const uint8_t *a_s = smem + place * stage_bytes + ra * 128, *b_s = smem + place * stage_bytes + kManyRows * 128 + g * stride + 8 * q;
            const int n = tile * kCols;
#pragma unroll
            for (int block = 0; block < kBlocks; ++block) {
                const int cols = kWhole ? 8 : width - n - 32 * block - 8 * q;   // from this lane's first one up to the end
                Columns<T> va, vb;
#pragma unroll
                for (int i = 0; i < 8 / kPieceCols; ++i) {   // (8 columns: one piece of bf16, two of fp32)
                    const uint32_t off = (static_cast<uint32_t>((32 * block + 8 * q) / kPieceCols + i) * 16) ^ swap;
                    va.raw[i] = vb.raw[i] = make_uint4(0, 0, 0, 0);
                    if (cols >= 8) {
                        va.raw[i] = *reinterpret_cast<const uint4*>(a_s + off);
                        vb.raw[i] = *reinterpret_cast<const uint4*>(a_s + 8 * 128 + off);
                    }
                }
                float acc[4][4];
                begin_sum<T>(acc, va, 0);
                begin_sum<T>(acc, vb, 2);
#pragma unroll
                for (int k = 0; k < kSteps16; ++k) {
                    if (!kWhole && 16 * k >= rank) break;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint2 b = *reinterpret_cast<const uint2*>(b_s + (32 * block + 8 * j) * stride + 32 * k);
                        if (!kWhole && rank - 16 * k < 16) b = masked(b, rank - 16 * k - 4 * q);
                        mma_bf16(acc[j], ha[k].x, hb[k].x, ha[k].y, hb[k].y, b.x, b.y);
                        mma_bf16(acc[j], ha[k].z, hb[k].z, ha[k].w, hb[k].w, b.x, b.y);
                    }
                }
                if (cols >= 8) {
                    if (has_a) end_sum<T>(acc, va, 0).store(ya + n + 32 * block);
                    if (has_b) end_sum<T>(acc, vb, 2).store(yb + n + 32 * block);
                } else if (cols > 0) {
                    const T* from = static_cast<const T*>(p.base) + at.n0 + n + 32 * block + 8 * q;
                    if (has_a) add_last<T>(acc, 0, cols, from + ma * p.ldbase, ya + n + 32 * block);
                    if (has_b) add_last<T>(acc, 2, cols, from + mb * p.ldbase, yb + n + 32 * block);
                }
            }
        };
#pragma unroll 1
        for (int tile = 0; tile < tiles; ++tile) {
            copies_wait<kManyStages - 2>();
            __syncthreads();   // this tile is there for all, and the one before it has been read
            ask(tile + kManyStages - 1, place == 0 ? kManyStages - 1 : place - 1);
            if (working) {
                if (rank == 16 * kSteps16 && (tile + 1) * kCols <= width) one_tile(tile, std::true_type());
                else one_tile(tile, std::false_type());
            }
            place = place == kManyStages - 1 ? 0 : place + 1;
        }
        copies_wait<0>();
        __syncthreads();   // (the item's rows and tiles have been read)
    }
}

// Many rows, high ranks: the tensor core takes its operands from shared memory, and its accumulators are in tensor memory.  Tiles of an item's
// rows and kRowBytes of each of them, in columns of one part; a CTA per SM has an equal share of all tiles, one
// after another.  A tile of base comes into shared memory while the one before is done; the tensor core multiplies the item's h, which stays in
// shared memory as 128 x 2 rank (hi, then lo against the same B), with the next tile's B into one of two accumulators in tensor memory
// while the threads take this tile out of the other one, add base in its place, and store rows from there.
// Operands lie in the tensor core's swizzled layout of 128 bytes of K per row (ranks above 64 take two such blocks): the pieces of a
// row, which neighbouring threads copy, stay within 128 bytes.  (Without swizzle each goes to a line of shared memory of its own, and
// the copies of one tile of B took 2500 cycles instead of 300.)  Rows of base: piece i of row r (16 bytes) at
// i ^ (r & 7), so that eight threads with a row each meet no bank twice.
// 4096 rows of gate / up in place, rank 64: 88 us for 319 MB, 3.6 TB/s; with fragments from shared memory (mma.sync) 110.  It waits: all warps of
// the SM's only CTA are in the same phase (tensor core, tile out, stores, loads of the tile after the next one), and one tile of loads is on its
// way meanwhile.  The long scoreboard is the largest stall; HBM is 44 % busy, the load and store pipe 31 %, issue 36 %.
constexpr int kHighThreads = 512, kHighWarps = kHighThreads / 32;
constexpr int kKBytes = 128;      // of K per row of an operand's block
struct HighShared { int blocks, h, base, b, total; };   // blocks of K; bytes of h, a tile of base, of B, and in all, with two of each tile
__host__ __device__ inline HighShared high_shared(int pad_rank, int row_bytes, int cols) {
    HighShared t;
    t.blocks = pad_rank <= 64 ? 1 : 2;
    t.h = 2 * t.blocks * kManyRows * kKBytes;
    t.base = kManyRows * row_bytes;
    t.b = t.blocks * cols * kKBytes;
    t.total = 1024 + t.h + 2 * (t.base + t.b);   // (the first kilobyte: alignment)
    return t;
}
// Where 16-byte piece c of row r of an operand with `rows` rows lies.
__device__ __forceinline__ uint32_t operand_at(int r, int c, int rows) { return (c >> 3) * rows * kKBytes + r * kKBytes + 16 * ((c ^ r) & 7); }
__device__ __forceinline__ uint64_t operand_desc(uint32_t at) { return make_smem_desc(at, 16, 8 * kKBytes, kSwizzle128B); }
// The nth item of all windows that has something to do; -1 and the number of them in `all` if there are not so many.
__device__ __forceinline__ int nth_item(const int* counts, const AdapterItems& t, int nth, int* shared, int* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = 0;
    for (int w0 = 0; w0 < t.windows; w0 += kHighThreads) {
        const int w = w0 + threadIdx.x, c = w < t.windows ? counts[w] : 0;
        int before = c;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += v;
        }
        if (lane == 31) shared[warp] = before;
        if (threadIdx.x == 0) shared[kHighWarps] = -1;
        __syncthreads();
        int here = 0;
        before += sum - c;
        for (int i = 0; i < kHighWarps; ++i) {
            if (i < warp) before += shared[i];
            here += shared[i];
        }
        if (nth >= before && nth < before + c) shared[kHighWarps] = w * t.per_window + nth - before;
        __syncthreads();
        const int found = shared[kHighWarps];
        __syncthreads();
        if (found >= 0) return found;
        sum += here;
    }
    *all = sum;
    return -1;
}

template <class T, int kRowBytes>
__global__ void __launch_bounds__(kHighThreads, 1) adapters_high_y_kernel(const __grid_constant__ AdapterParams p, int tiles_per_item) {
    constexpr int kCols = kRowBytes / sizeof(T), kPieces = kRowBytes / 16, kPieceCols = 16 / sizeof(T), kTmemCols = 2 * kCols;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int row_s[kManyRows], search_s[kHighWarps + 1];
    __shared__ __align__(8) uint64_t done[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int pad_rank = p.pad_rank, ranks = p.n_parts * pad_rank;
    const HighShared lay = high_shared(pad_rank, kRowBytes, kCols);
    uint8_t* base_tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem) + 1023) & ~uintptr_t(1023));
    uint8_t *h_tile = base_tiles + 2 * lay.base, *b_tiles = h_tile + lay.h;
    const Workspace ws = views(p.h, p.items);
    const bool in_place = p.base == p.y;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&done[0]), 1);
        mbar_init(smem_u32(&done[1]), 1);
        abort_s = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    grid_dependency_wait();
    grid_launch_dependents();

    // This CTA's share of all tiles: [at_tile, stop_tile), counted item after item of those that have something to do.  (In one window, those
    // are its first ones.)
    int active = 0;
    if (p.items.windows == 1) active = ws.counts[0];
    else nth_item(ws.counts, p.items, 0x7fffffff, search_s, &active);
    const long long all_tiles = static_cast<long long>(active) * tiles_per_item;
    long long at_tile = all_tiles * blockIdx.x / gridDim.x;
    const long long stop_tile = all_tiles * (blockIdx.x + 1) / gridDim.x;
    unsigned count = 0;            // tiles that were multiplied: accumulator and phase
    bool ok = true;
#pragma unroll 1
    while (ok && at_tile < stop_tile) {
        // ---- the tiles of one part of one item
        const int nth = static_cast<int>(at_tile / tiles_per_item);
        int in_item = static_cast<int>(at_tile - static_cast<long long>(nth) * tiles_per_item);
        const int index = p.items.windows == 1 ? nth : nth_item(ws.counts, p.items, nth, search_s, &active);
        const Item& item = ws.items[index];
        int part = 0, n0 = 0, end = p.part_end[0];
        while (true) {
            const int n = (end - n0 + kCols - 1) / kCols;
            if (in_item < n) break;
            in_item -= n;
            n0 = end;
            end = p.part_end[++part];
        }
        n0 += in_item * kCols;
        const int tiles = static_cast<int>(min(stop_tile - at_tile, static_cast<long long>((end - n0 + kCols - 1) / kCols)));
        const int width = min(end - n0, kCols * tiles);
        at_tile += tiles;
        const int4 head = *reinterpret_cast<const int4*>(&item);
        const int listed = threadIdx.x < kManyRows ? item.row[threadIdx.x] : 0;
        const int slot = head.x, rows = head.y, rank = head.z;
        if (rank == 0) {   // (of an adapter whose rank is 0: in place too)
            if (!in_place) copy_rows<T>(p, item.row, rows, n0, n0 + width, threadIdx.x, kHighThreads);
            continue;
        }
        if (static_cast<int>(threadIdx.x) < rows) {
            row_s[threadIdx.x] = listed;
        }
        // B holds zeros behind the rank up to the end of the k step (h does too)
        if (rank & 15)
            for (int i = threadIdx.x; i < 2 * lay.b / 16; i += kHighThreads) reinterpret_cast<uint4*>(b_tiles)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();

        const T* base = static_cast<const T*>(p.base) + n0;
        T* y = static_cast<T*>(p.y) + n0;
        const uint16_t* B = p.B + (static_cast<long long>(slot) * p.N + n0) * p.max_rank;
        // What a thread copies of a tile, worked out once: a piece of every kRowsOn-th row of base ...
        constexpr int kRowsOn = kHighThreads / kPieces, kMyRows = kManyRows / kRowsOn;
        const int base_piece = threadIdx.x % kPieces, base_row = threadIdx.x / kPieces;
        const T* base_from[kMyRows];   // null: no such row
#pragma unroll
        for (int i = 0; i < kMyRows; ++i) {
            const int r = base_row + i * kRowsOn;
            base_from[i] = r < rows ? base + row_s[r] * p.ldbase + base_piece * kPieceCols : nullptr;
        }
        const uint32_t base_to = smem_u32(base_tiles) + base_row * kRowBytes + 16 * (base_piece ^ (base_row & 7));
        static_assert(kRowsOn % 8 == 0, "the swizzle of a thread's rows is the same");
        // ... and of B pieces that are kHighThreads apart (a rank of 8, 16, 32, 64 or 128: the same one of every so many-th row)
        const int b_whole = rank / 8, b_pieces = (rank + 7) / 8, b_row = threadIdx.x / b_pieces, b_piece = threadIdx.x - b_row * b_pieces;
        const int b_rows_on = kHighThreads / b_pieces, b_pieces_on = kHighThreads - b_rows_on * b_pieces;
        const bool b_regular = b_pieces_on == 0 && (rank & 7) == 0;
        const uint16_t* b_from = B + static_cast<long long>(b_row) * p.max_rank + 8 * b_piece;
        const uint32_t b_to = smem_u32(b_tiles) + operand_at(b_row, b_piece, kCols);
        const long long b_step = static_cast<long long>(b_rows_on) * p.max_rank, b_tile_step = static_cast<long long>(kCols) * p.max_rank;
        auto ask_b = [&](int tile) {
            if (tile < tiles) {
                const int n = tile * kCols, here = min(kCols, width - n);
                if (b_regular) {   // (b_rows_on is a multiple of 8: the swizzle of a thread's rows is the same)
                    const uint16_t* from = b_from + tile * b_tile_step;
                    uint32_t to = b_to + (tile & 1) * lay.b;
                    for (int row = b_row; row < here; row += b_rows_on) {
                        copy16(to, from);
                        from += b_step;
                        to += b_rows_on * kKBytes;
                    }
                } else {
                    for (int row = b_row, c = b_piece; row < here;) {
                        const uint16_t* from = B + static_cast<long long>(n + row) * p.max_rank + 8 * c;
                        const uint32_t off = (tile & 1) * lay.b + operand_at(row, c, kCols);
                        if (c < b_whole) {
                            copy16(smem_u32(b_tiles) + off, from);
                        } else {   // the piece that the rank ends in
                            const uint4 v = *reinterpret_cast<const uint4*>(from);
                            const uint2 first = masked(make_uint2(v.x, v.y), rank - 8 * c), second = masked(make_uint2(v.z, v.w), rank - 8 * c - 4);
                            *reinterpret_cast<uint4*>(b_tiles + off) = make_uint4(first.x, first.y, second.x, second.y);
                        }
                        row += b_rows_on;
                        c += b_pieces_on;
                        if (c >= b_pieces) {
                            c -= b_pieces;
                            ++row;
                        }
                    }
                }
            }
            copies_commit();
        };
        auto ask_base = [&](int tile) {
            const int n = tile * kCols;
            if (tile < tiles && n + (base_piece + 1) * kPieceCols <= width) {
#pragma unroll
                for (int i = 0; i < kMyRows; ++i)
                    if (base_from[i]) copy16(base_to + (tile & 1) * lay.base + i * (kRowsOn * kRowBytes), base_from[i] + n);
            }
            copies_commit();
        };
        // h: hi, then lo (of four ranks each in the workspace, of eight here)
        for (int m = warp; m < rows; m += kHighWarps) {
            const uint2* from = reinterpret_cast<const uint2*>(ws.h + static_cast<long long>(row_s[m]) * (ranks / 4) + part * (pad_rank / 4));
            for (int c = lane; c < pad_rank / 2; c += 32)
                copy8(smem_u32(h_tile) + (c & 1) * (lay.h / 2) + operand_at(m, c >> 2, kManyRows) + 8 * (c >> 1 & 1), from + c);
        }
        ask_b(0);
        ask_base(0);
        ask_b(1);
        ask_base(1);

        const uint64_t h_desc = operand_desc(smem_u32(h_tile));
        const int k_steps = (rank + 15) / 16;
        auto multiply = [&](int tile) {   // one thread
            const unsigned number = count + tile;
            const uint64_t b_desc = operand_desc(smem_u32(b_tiles) + (tile & 1) * lay.b);
            for (int term = 0; term < 2; ++term)
                for (int k = 0; k < k_steps; ++k) {
                    // (16 of K: 32 bytes on; a block of 64 of K: the next one)
                    const uint64_t h_at = h_desc + ((term * (lay.h / 2) + (k >> 2) * kManyRows * kKBytes + (k & 3) * 32) >> 4);
                    const uint64_t b_at = b_desc + (((k >> 2) * kCols * kKBytes + (k & 3) * 32) >> 4);
                    tc_mma_bf16(tmem + (number & 1) * kCols, h_at, b_at, make_idesc_bf16(kCols), term | k);
                }
            tc_commit(smem_u32(&done[number & 1]));
        };
        // Takes a tile out: a warp has 32 rows (the lanes of tensor memory that it can read) and a quarter of the columns, 64 bytes of each
        // row at a time.
        const int my_row = 32 * (warp & 3) + lane, quarter = warp >> 2;
        constexpr int kRow = kPieces / 4, kAtOnce = 32 / kRow;   // lanes that store a row's quarter, rows at once
        const int out_piece = quarter * kRow + lane % kRow, out_row = 32 * (warp & 3) + lane / kRow;
        T* to[32 / kAtOnce];
#pragma unroll
        for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int r = out_row + kAtOnce * i;
            to[i] = r < rows ? y + row_s[r] * p.ldy + out_piece * kPieceCols : nullptr;
        }
        auto take = [&](int tile) {
            uint8_t* base_tile = base_tiles + (tile & 1) * lay.base;
            const uint32_t sums = tmem + ((32u * (warp & 3)) << 16) + ((count + tile) & 1) * kCols + quarter * (kCols / 4);
            uint8_t* mine = base_tile + my_row * kRowBytes;
#pragma unroll
            for (int part64 = 0; part64 < kPieces / 16; ++part64) {
                constexpr int kHere = 4 * kPieceCols;   // columns in 64 bytes
                uint32_t d[kHere];
                if constexpr (kHere == 32) tmem_ld_32x32(sums + part64 * kHere, d);
                else tmem_ld_32x16(sums + part64 * kHere, d);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int piece = quarter * (kPieces / 4) + 4 * part64 + i;
                    uint4* at16 = reinterpret_cast<uint4*>(mine + 16 * (piece ^ (my_row & 7)));
                    uint4 v = *at16;
                    uint32_t* w = &v.x;
                    if constexpr (sizeof(T) == 2) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            w[j] = pack_bf16(bf16_lo(w[j]) + __uint_as_float(d[8 * i + 2 * j]), bf16_hi(w[j]) + __uint_as_float(d[8 * i + 2 * j + 1]));
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(__uint_as_float(w[j]) + __uint_as_float(d[4 * i + j]));
                    }
                    *at16 = v;
                    // the last columns of a matrix whose width is no multiple of a piece
                    const int n = tile * kCols + piece * kPieceCols, cols = width - n;
                    if (cols > 0 && cols < kPieceCols && my_row < rows) {
#pragma unroll
                        for (int j = 0; j < kPieceCols; ++j)
                            if (j < cols) y[row_s[my_row] * p.ldy + n + j] = static_cast<T>(static_cast<float>(base[row_s[my_row] * p.ldbase + n + j]) + __uint_as_float(d[i * kPieceCols + j]));
                    }
                }
            }
            __syncwarp();
            const int n = tile * kCols;
            if (n + (out_piece + 1) * kPieceCols <= width) {
#pragma unroll
                for (int i = 0; i < 32 / kAtOnce; ++i) {
                    const int r = out_row + kAtOnce * i;
                    if (to[i]) *reinterpret_cast<uint4*>(to[i] + n) = *reinterpret_cast<const uint4*>(base_tile + r * kRowBytes + 16 * (out_piece ^ (r & 7)));
                }
            }
        };
        copies_wait<3>();            // h and the first B
        fence_proxy_async_smem();    // (what copies and threads wrote, before the tensor core reads it)
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (threadIdx.x == 0) multiply(0);
#pragma unroll 1
        for (int tile = 0; tile < tiles; ++tile) {
            copies_wait<1>();            // this tile's base and the next one's B
            fence_proxy_async_smem();
            tc_fence_before_sync();      // (the accumulator that is written next has been read)
            __syncthreads();
            tc_fence_after_sync();
            if (tile + 1 < tiles && threadIdx.x == 0) multiply(tile + 1);
            // A warp takes the tile out as a whole or not at all.  Whether a wait ran out is the CTA's answer at the barrier behind the tile: nothing
            // is multiplied, asked for or taken out after one did.
            const unsigned number = count + tile;
            const bool gives_up = p.wait_limit < 0 && threadIdx.x == 0 && static_cast<long long>(number) + 1 >= -p.wait_limit;
            const bool there = __all_sync(0xffffffffu, !gives_up && mbar_wait(smem_u32(&done[number & 1]), number >> 1 & 1, &abort_s,
                                                                              p.wait_limit < 0 ? kWaitLimitCycles : p.wait_limit));
            tc_fence_after_sync();
            if (there) take(tile);
            ok = __syncthreads_and(there);   // (the tile's places are free)
            if (!ok) {
                // products that are still on their way read shared memory and write tensor memory
                for (unsigned i = number; i < count + min(tiles, tile + 2); ++i) mbar_wait_after_abort(smem_u32(&done[i & 1]), i >> 1 & 1);
                break;
            }
            ask_b(tile + 2);
            ask_base(tile + 2);
        }
        copies_wait<0>();
        count += tiles;
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
    }
    if (!ok && threadIdx.x == 0) atomicExch(p.status, PRQ_ERR_TIMEOUT);
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kTmemCols);
}

template <class... Params, class... Args>
cudaError_t launch_kernel(void (*kernel)(Params...), dim3 blocks, int threads, int cluster, size_t smem, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class Kernel>
cudaError_t allow_shared(Kernel kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
}
struct Passes { int passes, tiles; };   // tiles: eights of ranks per pass
Passes passes_of(const AdapterParams& p) {
    const int passes = passes_of(p.n_parts, p.max_rank), tiles = (p.n_parts * p.pad_rank / 8 + passes - 1) / passes;
    return Passes{passes, tiles <= 2 ? 2 : tiles <= 4 ? 4 : tiles <= 6 ? 6 : 8};
}
template <class F>
cudaError_t with_tiles(int tiles, F&& f) {
    return tiles == 2 ? f(std::integral_constant<int, 2>()) : tiles == 4 ? f(std::integral_constant<int, 4>())
         : tiles == 6 ? f(std::integral_constant<int, 6>()) : f(std::integral_constant<int, 8>());
}
// Pieces of `width` columns of all parts; where the kernel looks for them, up to the end of each part too.
int pieces_of(const AdapterParams& p, int width, int* ends = nullptr) {
    int n = 0;
    for (int i = 0; i < kMaxBatch; ++i) {
        n += (p.part_end[i] - (i ? p.part_end[i - 1] : 0) + width - 1) / width;
        if (ends) ends[i] = n;
    }
    return n;
}
template <class T, int kRowBytes>
cudaError_t launch_high_y(const AdapterParams& p, int num_sms, cudaStream_t stream) {
    static OncePerDevice once;
    constexpr int kCols = kRowBytes / sizeof(T);
    const auto kernel = adapters_high_y_kernel<T, kRowBytes>;
    const cudaError_t e = once([&] { return allow_shared(kernel, high_shared(kRowBytes == 512 ? 64 : PRQ_ADAPTER_MAX_RANK, kRowBytes, kCols).total); });
    if (e != cudaSuccess) return e;
    const int tiles = pieces_of(p, kCols);
    const long long most = static_cast<long long>(tiles) * p.items.n;
    return launch_kernel(kernel, dim3(static_cast<unsigned>(std::min<long long>(most, num_sms))), kHighThreads, 1, high_shared(p.pad_rank, kRowBytes, kCols).total, stream, p, tiles);
}
template <class T, int kSteps16>
cudaError_t launch_many_y(const AdapterParams& p, int units, int span, cudaStream_t stream) {
    static OncePerDevice once;
    const auto kernel = adapters_many_y_kernel<T, kSteps16>;
    const cudaError_t e = once([&] { return allow_shared(kernel, kManyStages * many_stage_bytes<T>(16 * kSteps16)); });
    if (e != cudaSuccess) return e;
    return launch_kernel(kernel, dim3(units * p.y_items * p.items.windows), kManyThreads, 1, kManyStages * many_stage_bytes<T>(p.max_rank), stream, p, units, span);
}
template <class T>
cudaError_t launch_few(AdapterParams p, cudaStream_t stream) {
    const Passes t = passes_of(p);
    const int units = pieces_of(p, 64, p.unit_end);
    return with_tiles(t.tiles, [&](auto tiles) {
        static OncePerDevice once;
        using Shared = FewShared<decltype(tiles)::value>;
        static_assert(sizeof(Shared) <= 227 * 1024, "shared memory");
        const auto kernel = adapters_few_kernel<T, decltype(tiles)::value, true>, looping = adapters_few_kernel<T, decltype(tiles)::value, false>;
        const cudaError_t e = once([&] {
            const cudaError_t first = allow_shared(kernel, sizeof(Shared));
            return first != cudaSuccess ? first : allow_shared(looping, sizeof(Shared));
        });
        if (e != cudaSuccess) return e;
        return launch_kernel(p.h_clusters == p.items.per_window ? kernel : looping, dim3(p.h_clusters * p.items.windows * p.cluster), kHThreads, p.cluster, sizeof(Shared), stream, p, t.passes, units);
    });
}
cudaError_t launch_many_h(const AdapterParams& p, cudaStream_t stream) {
    const Passes t = passes_of(p);
    return with_tiles(t.tiles, [&](auto tiles) {
        static OncePerDevice once;
        using Shared = ManyHShared<decltype(tiles)::value>;
        static_assert(sizeof(Shared) <= 227 * 1024, "shared memory");
        const auto kernel = adapters_many_h_kernel<decltype(tiles)::value, true>, looping = adapters_many_h_kernel<decltype(tiles)::value, false>;
        const cudaError_t e = once([&] {
            const cudaError_t first = allow_shared(kernel, sizeof(Shared));
            return first != cudaSuccess ? first : allow_shared(looping, sizeof(Shared));
        });
        if (e != cudaSuccess) return e;
        return launch_kernel(p.h_clusters == p.items.per_window ? kernel : looping, dim3(p.h_clusters * p.items.windows * p.cluster, t.passes), kHThreads, p.cluster, sizeof(Shared), stream, p);
    });
}
template <class T>
cudaError_t launch_many_y(AdapterParams p, int num_sms, cudaStream_t stream) {
    // Tensor memory for ranks above 32 where a CTA has many tiles (gate / up of 4096 tokens, 16 tiles of 256 columns per SM: rank 64 125 us
    // with mma.sync, 109 to 111 so; rank 32 84 and 98; q / k / v, five per SM: rank 64 68 either way, rank 32 42 and 54; 1024 tokens of gate / up,
    // rank 64: 47 either way), and for ranks above 64, whose h mma.sync's registers do not hold.
    const int items = (p.M + kManyRows - 1) / kManyRows;
    if (p.pad_rank > 64) return launch_high_y<T, 256>(p, num_sms, stream);
    if (p.pad_rank > 32 && static_cast<long long>(pieces_of(p, 512 / sizeof(T))) * items >= 8ll * num_sms) return launch_high_y<T, 512>(p, num_sms, stream);
    // a CTA's tiles: one where there are few of them, up to four for less to set up (q / k / v of 4096 rows, rank 16: 41 us with four, 48 with
    // one, 45 with eight; o of 387 rows, rank 32: 13.1 with one, 14.9 with four)
    int span = static_cast<int>(std::max<long long>(1, std::min<long long>(4, static_cast<long long>(pieces_of(p, kManyCols<T>)) * items / (6ll * num_sms))));
    while (static_cast<long long>(pieces_of(p, kManyCols<T> * span)) * p.y_items * p.items.windows > 0x7fffffffll) span *= 2;   // (a grid's limit)
    const int units = pieces_of(p, kManyCols<T> * span, p.unit_end), steps = p.pad_rank / 16;
    return steps == 1 ? launch_many_y<T, 1>(p, units, span, stream) : steps == 2 ? launch_many_y<T, 2>(p, units, span, stream) : launch_many_y<T, 4>(p, units, span, stream);
}

}  // namespace

size_t adapters_workspace_bytes(int M, int n_slots, int n_parts, int max_rank, bool any_fewer) {
    // (several passes: a few rows need some where a middling number does not)
    if (any_fewer) return std::max(adapters_workspace_bytes(M, n_slots, n_parts, max_rank, false),
                                   adapters_workspace_bytes(std::max(1, std::min(M, kItemsSoon / passes_of(n_parts, max_rank))), n_slots, n_parts, max_rank, false));
    if (small_items(M, n_slots, passes_of(n_parts, max_rank))) return 0;
    const AdapterItems items = plan_items(M, n_slots, false);
    const size_t ranks = n_parts * ((max_rank + 15) & ~15);
    return counts_bytes(items) + sizeof(Item) * items.n + 4 * ranks * static_cast<size_t>(M);
}

cudaError_t launch_adapters(const AdapterParams& in, bool bf16, int num_sms, cudaStream_t stream, int* launches) {
    AdapterParams p = in;
    p.pad_rank = (p.max_rank + 15) & ~15;
    const bool few = small_items(p.M, p.n_slots, passes_of(p.n_parts, p.max_rank));
    const int passes = few ? 1 : passes_of(p.n_parts, p.max_rank);
    p.items = plan_items(p.M, p.n_slots, few);
    const int full = p.M / kManyRows, items = few ? p.items.n : full + std::min(p.n_slots, full) / 4 + 1;
    // CTAs of a cluster: as many as let all items (of large ones, those of the rows, and of some more adapters) be on the GPU at once, with 8
    // steps of K each (4 for many rows), and of small items with an adapter of 640 KB per CTA and more in any case (q / k / v of rank 64, 200
    // rows of a pool of 64, four of them in use: 64 us without that, 38 so; all in use: 76 and 46).
    p.cluster = 1;
    const long long bytes = 2ll * p.pad_rank * (static_cast<long long>(p.n_parts) * p.K + p.N), sixth = num_sms / 18;
    for (int c = 2; c <= 8; ++c) {
        const bool at_once = static_cast<long long>(items) * passes * c <= sixth * (18 / c) * c;
        if ((at_once || (few && bytes >= 655360ll * c)) && p.K / 32 >= (few ? 8 : 4) * c) p.cluster = c;
    }
    // How many items there are is not known here, and a pool of 64 may be used by four adapters: clusters, and CTAs of y, for as many items as
    // run at once, each with every so many-th one.  (1000 rows of a pool of 64, four in use: 18 us, with a cluster for each item that there
    // could be 36; pool of 500: 18 and 193.)
    const int windows = p.items.windows, whole = p.items.window / kManyRows;
    p.h_clusters = std::min(p.items.per_window, static_cast<int>(std::max<long long>(1, (sixth * (18 / p.cluster) / passes + windows - 1) / windows)));
    if (few) {
        const cudaError_t e = bf16 ? launch_few<__nv_bfloat16>(p, stream) : launch_few<float>(p, stream);
        *launches = e == cudaSuccess;
        return e;
    }
    p.y_items = std::min(p.items.per_window, whole + whole / 4 + 8);
    cudaError_t e = launch_many_h(p, stream);
    if (e != cudaSuccess) return e;
    ++*launches;
    e = bf16 ? launch_many_y<__nv_bfloat16>(p, num_sms, stream) : launch_many_y<float>(p, num_sms, stream);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace prq
