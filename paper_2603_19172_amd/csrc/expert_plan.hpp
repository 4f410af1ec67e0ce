// The plan of a call on a layer's experts, shared by the formats whose table entries are six pointers: pairs sorted by expert, and the list
// of tiles of rows.
#pragma once
#include "common.hpp"

namespace dymoe {

// A tile of an expert: all that a workgroup has to know before its first load of weights.
template <class Entry>
struct __attribute__((aligned(16))) ExpertTile {
    int32_t first, pairs;             // the expert's first position, its pairs
    int32_t tile0, tiles;             // its first tile, its tiles
    Entry mat;
};

template <class Entry>
struct ExpertPlan {
    int32_t* meta;        // [8]: tiles, wide tiles behind them
    int32_t* perm;        // [P] position -> pair
    int32_t* where;       // [P] pair -> position, -1: left out
    ExpertTile<Entry>* tiles;
};

template <class Entry>
__host__ __device__ inline ExpertPlan<Entry> expert_plan(int32_t* p, long P)
{
    static_assert(sizeof(Entry) == 48, "six pointers");
    ExpertPlan<Entry> r;
    r.meta = p;
    r.perm = r.meta + 8;
    r.where = r.perm + P;
    r.tiles = (ExpertTile<Entry>*)(p + 8 + (2 * P + 3) / 4 * 4);
    return r;
}

// bytes of a plan of P pairs and at most that many tiles
static inline size_t expert_plan_bytes(size_t P, size_t tiles) { return (8 + (2 * P + 3) / 4 * 4 + 16 * tiles) * 4; }

template <class Entry>
__device__ __forceinline__ bool expert_present(const Entry& x)
{
    return (x.q[0] != nullptr) & (x.q[1] != nullptr) & (x.q[2] != nullptr) & (x.s[0] != nullptr) & (x.s[1] != nullptr) & (x.s[2] != nullptr);
}

// Counting sort of the pairs by expert and the list of tiles, by one workgroup: tall tiles first, then wide ones, by expert.  A pair's turn
// in its expert is what the counter held before it: kept in registers (in `where` beyond the first kPlanKeep pairs of a thread)
// until the experts' first positions are known, so that there is one pass of atomics.  The turns come in any order, and nothing that is
// computed depends on it.  The sorted pairs and the tiles' experts pass through LDS where they fit: written from the threads that
// know them, 16384 pairs cost 7 us in stores of four bytes each, and an expert's sixteen records 3 us in one thread.  16384 pairs of 128
// experts 12.1 us with 2048 rows' codes beside it, 488 pairs 4.6: latencies of one workgroup's passes, not bytes.
constexpr int kPlanThreads = 1024;
constexpr int kPlanKeep = 16;
constexpr int kPlanPairs = kPlanKeep * kPlanThreads;
constexpr int kPlanTiles = 4096;

static_assert(kPlanThreads == DYMOE_MAX_EXPERTS, "a thread for every expert");

struct ExpertPlanLds {
    int count[DYMOE_MAX_EXPERTS], at[DYMOE_MAX_EXPERTS], tile0[DYMOE_MAX_EXPERTS], wave[3][kPlanThreads / kWave];
    uint16_t owner[kPlanTiles], perm[kPlanPairs];
};

// Tiles of SMALL rows (small), else of WIDE rows for experts of up to as many pairs (0: none are) and of TALL rows for the others.
template <int SMALL, int WIDE, int TALL, class Entry>
__device__ __forceinline__ void make_expert_plan(ExpertPlanLds& lds, const int32_t* __restrict__ idx, const Entry* __restrict__ table, long P, int E,
                                                 int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const ExpertPlan<Entry> pp = expert_plan<Entry>(plan, P);
    int e_of[kPlanKeep], turn[kPlanKeep];
#pragma unroll
    for (int i = 0; i < kPlanKeep; i++) {
        const long p = tid + (long)i * kPlanThreads;
        e_of[i] = p < P ? idx[p] : -1;
    }
    const bool held = tid < E && expert_present(table[tid]);
    lds.count[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPlanKeep; i++)
        if ((unsigned)e_of[i] < (unsigned)E) turn[i] = atomicAdd(&lds.count[e_of[i]], 1);
    for (long p = tid + (long)kPlanPairs; p < P; p += kPlanThreads) {
        const int e = idx[p];
        if ((unsigned)e < (unsigned)E) pp.where[p] = atomicAdd(&lds.count[e], 1);
    }
    __syncthreads();
    int n = lds.count[tid];
    if (n > 0 && !held) {
        atomicOr(flags, DYMOE_FLAG_FORMAT_MISSING);
        n = 0;
    }
    const bool one = WIDE > 0 && !small && n <= WIDE;             // a wide tile
    const int rows = small ? SMALL : one ? WIDE : TALL, m = (n + rows - 1) / rows;
    const int n_in = wave_scan_dpp_i32(n), m2_in = wave_scan_dpp_i32(one ? 0 : m), m1_in = wave_scan_dpp_i32(one ? m : 0);
    if (lane == kWave - 1) {
        lds.wave[0][wave] = n_in;
        lds.wave[1][wave] = m2_in;
        lds.wave[2][wave] = m1_in;
    }
    __syncthreads();
    constexpr int kUnroll = WIDE > 0 ? kPlanThreads / kWave : 4;       // (16 without wide tiles: 14 registers to scratch memory)
    int n0 = n_in - n, t2 = m2_in, t1 = m1_in, all2 = 0, all1 = 0;
#pragma unroll kUnroll
    for (int w = 0; w < kPlanThreads / kWave; w++) {
        const int a2 = lds.wave[1][w], a1 = lds.wave[2][w];
        if (w < wave) {
            n0 += lds.wave[0][w];
            t2 += a2;
            t1 += a1;
        }
        all2 += a2;
        all1 += a1;
    }
    const int t0 = one ? all2 + t1 - m : t2 - m;
    // (in 16-byte pieces: a record put together first would pass through scratch memory)
    auto record = [&](ExpertTile<Entry>* to, int e, int first, int pairs, int tile0, int tiles) {
        uint4* const at = (uint4*)to;
        const uint2* const mat = (const uint2*)(table + e);
        store_global(at, make_uint4((uint32_t)first, (uint32_t)pairs, (uint32_t)tile0, (uint32_t)tiles));
#pragma unroll
        for (int i = 0; i < 3; i++) {
            const uint2 lo = load_global<uint2>(mat + 2 * i), hi = load_global<uint2>(mat + 2 * i + 1);
            store_global(at + 1 + i, make_uint4(lo.x, lo.y, hi.x, hi.y));
        }
    };
    lds.at[tid] = n > 0 ? n0 : -1;
    lds.count[tid] = n;
    lds.tile0[tid] = t0;
    for (int i = 0; i < m; i++) {
        if (t0 + i < kPlanTiles) lds.owner[t0 + i] = (uint16_t)tid;
        else record(&pp.tiles[t0 + i], tid, n0, n, t0, m);
    }
    if (tid == 0) {
        pp.meta[0] = all2;
        pp.meta[1] = all1;
    }
    __syncthreads();
    for (int i = tid; i < min(all1 + all2, kPlanTiles); i += kPlanThreads) {
        const int e = lds.owner[i], c = lds.count[e];
        const int per = small ? SMALL : c <= WIDE ? WIDE : TALL;
        record(&pp.tiles[i], e, lds.at[e], c, lds.tile0[e], (c + per - 1) / per);
    }
    const bool fits = P <= kPlanPairs;
    auto place = [&](long p, int x, int rank) {
        int at = -1;
        if ((unsigned)x < (unsigned)E && lds.at[x] >= 0) {
            at = lds.at[x] + rank;
            if (fits) lds.perm[at] = (uint16_t)p;
            else pp.perm[at] = (int32_t)p;
        }
        pp.where[p] = at;
    };
#pragma unroll
    for (int i = 0; i < kPlanKeep; i++) {
        const long p = tid + (long)i * kPlanThreads;
        if (p < P) place(p, e_of[i], turn[i]);
    }
    for (long p = tid + (long)kPlanPairs; p < P; p += kPlanThreads) place(p, idx[p], pp.where[p]);
    if (!fits) return;
    __syncthreads();
    int sorted = 0;
    for (int w = 0; w < kPlanThreads / kWave; w++) sorted += lds.wave[0][w];
    for (int i = tid; i < sorted; i += kPlanThreads) pp.perm[i] = lds.perm[i];
}

}  // namespace dymoe
