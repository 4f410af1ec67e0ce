// Products in microscaled 4-bit floating point: a matrix (dymoe_matmul_mx4) and a layer's SwiGLU experts (dymoe_moe_ffn_mx4).
//   y[t, n] = sum over blocks b of 32 columns of 2^(ex[t, b] + ew[n, b]) sum_{j in b} xq[t, j] wq[n, j]
// A block's sum is exact; the sum over the blocks is taken in fp32 (mfma_mx4), in an order that belongs to the shape of the call.
#include <type_traits>

#include "expert_plan.hpp"
#include "mx4_device.hpp"
#include "mx4_rule.hpp"

namespace dymoe {

int mx4_quantize(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, uint8_t* codes, uint8_t* scale, hipStream_t st);

using Mx4Plan = ExpertPlan<dymoe_expert_mx4>;

// The plan by the first workgroup, the codes of the activations by the others, a wavefront 512 columns of a row: neither needs the other.  A step's 256
// columns of all tokens lie together (128 bytes a token, 8 of exponents), so that a tile's rows are neighbours in memory whatever H is: a power of
// two from row to row sends them to few channels (512 tokens, 2 of 8 experts of 14336 x 4096 218 -> 211 us, 2047 tokens 471 -> 457).
template <int DT>
__global__ __launch_bounds__(kPlanThreads) void mx4_prep_kernel(const int32_t* __restrict__ idx, const dymoe_expert_mx4* __restrict__ table, long P,
                                                                int E, int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags,
                                                                const char* __restrict__ x, int rows, int units, int per_row, int K, char* __restrict__ codes,
                                                                char* __restrict__ scale)
{
    __shared__ ExpertPlanLds lds;
    if (blockIdx.x == 0) {
        make_expert_plan<kMx4SmallRows, 0, kMx4TallRows>(lds, idx, table, P, E, small, plan, flags);
        return;
    }
    const int unit = (int)(blockIdx.x - 1) * (kPlanThreads / kWave) + threadIdx.x / kWave;
    if (unit >= units) return;
    const int part = unit / per_row, col0 = (unit - part * per_row) * 512;
    const long row = part;
    const int col = col0 + (threadIdx.x & (kWave - 1)) * 8, Kp = (int)up_to(K, 256);
    const Raw8<DT> v = load8<DT>(x + row * K * dtype_bytes(DT), col, K);
    const uint32_t byte = mx4_exponent(quad_max_u32(peak_f32_bits<DT>(peak8<DT>(v, 0u)))), q = mx4_codes8<DT>(v, byte);
    if (col >= Kp) return;
    const long at = ((long)(col >> 8) * rows + row) * 256 + (col & 255);
    *(DYMOE_GLOBAL uint32_t*)(codes + at / 2) = q;
    if ((col & 31) == 0) *(DYMOE_GLOBAL uint8_t*)(scale + at / 32) = (uint8_t)byte;
}

enum { kMx4Plain = 0, kMx4Up = 1, kMx4Down = 2 };

struct Mx4Args {
    const char *x, *xs;               // codes of the rows, Kp / 2 bytes each, and their exponents, Kp / 32 (up: 256 columns of all tokens after
                                      // another); or the rows themselves
    long ldx;                         // those: bytes from row to row
    const int32_t* idx;               // and the experts of a few tokens' pairs, their weights and table
    const float* gate;
    const dymoe_expert_mx4* table;
    unsigned* flags;
    int x_dtype, K, E;
    const int32_t* plan;              // experts
    const char *w, *ws;               // the plain product
    const float* bias;
    void* out;                        // up: codes of the intermediate's rows, ldo / 2 bytes each, or in tiles (tall ones)
    uint8_t* out_scale;               // up: their exponents
    long ldo, P;
    int rows, Kp, N, k, out_dtype;
    int splits;                       // tall tiles of the down projection: parts of K, P rows of outputs each
};

// A strip of 32 weight rows: codes and exponents.  One behind the last of the matrix has no bytes, and is read as zeros.
struct Mx4Strip {
    BufferSrc q, s;
    __device__ __forceinline__ void set(const void* codes, const void* scale, long strip, int strips, int Kp)
    {
        const long at = min(strip, strips - 1L);
        q.set((const char*)codes + at * 16 * Kp, strip < strips ? 16u * (uint32_t)Kp : 0u);
        s.set((const char*)scale + at * Kp, strip < strips ? (uint32_t)Kp : 0u);
    }
};

__device__ __forceinline__ uint32_t load_u32(const BufferSrc& s, uint32_t lane, uint32_t all)
{
    return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(s.r, (int)lane, (int)all, 0);
}

// The codes of `rows` rows into LDS, Kp / 2 + 16 bytes apart, and their exponents behind them, Kp / 32 apart, by a whole workgroup (mx4_fuse_bytes).
__device__ __forceinline__ int mx4_lds_row(int Kp) { return (Kp >> 1) + 16; }

template <int DT>
__device__ __forceinline__ void mx4_rows_to_lds(const char* x, long ldx, int rows, int K, int Kp, char* lds)
{
    const int per = Kp >> 3, n = rows * per;
    char* const exps = lds + rows * mx4_lds_row(Kp);
    // (per is a multiple of 32 and so is the number of threads: four lanes that share a block are in step)
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int r = i / per, col = (i - r * per) * 8;
        const Raw8<DT> v = load8<DT>(x + r * ldx, col, K);
        const uint32_t byte = mx4_exponent(quad_max_u32(peak_f32_bits<DT>(peak8<DT>(v, 0u))));
        *(uint32_t*)(lds + r * mx4_lds_row(Kp) + (col >> 1)) = mx4_codes8<DT>(v, byte);
        if ((col & 31) == 0) exps[r * (Kp >> 5) + (col >> 5)] = (char)byte;
    }
    __syncthreads();
}

__device__ __forceinline__ void mx4_rows_to_lds(int dt, const char* x, long ldx, int rows, int K, int Kp, char* lds)
{
    if (dt == DYMOE_OUT_F32) mx4_rows_to_lds<DYMOE_OUT_F32>(x, ldx, rows, K, Kp, lds);
    else if (dt == DYMOE_OUT_F16) mx4_rows_to_lds<DYMOE_OUT_F16>(x, ldx, rows, K, Kp, lds);
    else mx4_rows_to_lds<DYMOE_OUT_BF16>(x, ldx, rows, K, Kp, lds);
}

// ----------------------------------------------------------------------------
// Tiles of up to 32 rows where rows or columns are too few for the tiles below (decode batches, narrow matrices): a stream of weights.  KS
// wavefronts share a strip of 32 weight rows (of W1 and of W3 in the up projection) and take the 256-column tiles of K in turn; a workgroup of NW
// has NW / KS strips.  Nothing is shared before the end: weights and codes come straight into registers, a tile ahead of a wavefront's products, and
// the sums of a strip's wavefronts meet in LDS.
// Bound by the weights' bytes: 61 tokens on 8 of 128 experts of 768 x 2048, up 34.9 us (6.0 TB/s), down 19.2 (5.4); 61 x 1536 x 2048 4.3 us, a
// start, eight wavefronts' share of K and the sums' way through LDS.
// XT: the rows lie in tiles as the weights do, and a load of theirs is 1 KiB of contiguous memory too: 61 x 1536 x 2048 4.1 us and 5.0 row by row.  A
// call that converts its rows writes them so.
// FUSE: the rows come as they are, few enough for every workgroup to convert them for itself, behind its first loads of weights; the experts' pairs
// are then looked through by every workgroup too: the one of a pair that comes first among those of its expert (or 32, 64, ... behind
// the first) takes the next 32 of them, and a pair's position is its number.
template <int MODE, int NW, int KS, bool FUSE = false, bool XT = false>
__global__ __launch_bounds__(64 * NW) void mx4_small_kernel(const Mx4Args A)
{
    constexpr int S = MODE == kMx4Up ? 2 : 1, kRows = 32, kStrips = NW / KS;
    constexpr int kParts = KS > 4 ? 4 : KS;      // wavefronts that finish a strip
    constexpr int kV = 16 / kParts;              // registers of a fragment that each of them finishes
    static_assert(NW % KS == 0 && (KS == 8 || KS == 4 || KS == 2 || KS == 1), "");
    static_assert(!FUSE || MODE != kMx4Down, "");
    extern __shared__ __attribute__((aligned(16))) char s_rows[];
    __shared__ float s_red[KS > 1 ? kStrips * kParts : 1][S][16][kWave];
    __shared__ uint32_t s_peak[kStrips][kParts][32];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5, mine = wave / KS, part = wave - mine * KS;
    const int strips = (A.N + 31) / 32, all = MODE == kMx4Up ? (int)(A.ldo >> 5) : strips, nblk = (all + kStrips - 1) / kStrips;
    const Mx4Plan pp = expert_plan<dymoe_expert_mx4>(const_cast<int32_t*>(A.plan), A.P);
    int row0, rows, bx;
    Mx4Strip w[S];
    if (MODE == kMx4Plain) {
        const int tiles = (A.rows + kRows - 1) / kRows, block = blockIdx.x / tiles;
        bx = block * kStrips + mine;
        row0 = (blockIdx.x - block * tiles) * kRows;
        rows = min(kRows, A.rows - row0);
        w[0].set(A.w, A.ws, bx, strips, A.Kp);
    } else if (FUSE) {
        const int pair = blockIdx.x / nblk;
        bx = (blockIdx.x - pair * nblk) * kStrips + mine;
        const int my_e = lane < A.P ? A.idx[lane] : -1, e = __builtin_amdgcn_readlane(my_e, pair);
        if ((unsigned)e >= (unsigned)A.E) return;
        const uint64_t its = __ballot(my_e == e);
        const int rank = __popcll(its & ((1ull << pair) - 1));
        if (rank & (kRows - 1)) return;
        const dymoe_expert_mx4 ex = A.table[e];
        if (!expert_present(ex)) {
            if (tid == 0) atomicOr(A.flags, DYMOE_FLAG_FORMAT_MISSING);
            return;
        }
        rows = min(kRows, __popcll(its) - rank);
        uint64_t left = its >> pair << pair;                 // this tile's pairs and those behind it
        const int want = min(ln, rows - 1);
        for (int i = 0; i < want; i++) left &= left - 1;
        row0 = __builtin_ctzll(left);                        // this lane's pair
        w[0].set(ex.q[0], ex.s[0], bx, strips, A.Kp);
        w[S - 1].set(ex.q[1], ex.s[1], bx, strips, A.Kp);
    } else {
        const int tile = blockIdx.x / nblk;
        bx = (blockIdx.x - tile * nblk) * kStrips + mine;
        if (tile >= pp.meta[0]) return;
        const ExpertTile<dymoe_expert_mx4> t = pp.tiles[tile];
        const int i = (tile - t.tile0) * kRows;
        row0 = t.first + i;
        rows = min(kRows, t.pairs - i);
        w[0].set(t.mat.q[MODE == kMx4Up ? 0 : 2], t.mat.s[MODE == kMx4Up ? 0 : 2], bx, strips, A.Kp);
        if (MODE == kMx4Up) w[S - 1].set(t.mat.q[1], t.mat.s[1], bx, strips, A.Kp);
    }
    struct Tile {
        uint4 w[S][4], x[4];
        uint32_t ws[S], xs;
    };
    const uint32_t lane16 = (uint32_t)lane * 16u, lane4 = (uint32_t)lane * 4u;
    const int nkt = A.Kp >> 8;
    uint32_t off, offs;
    const uint32_t step_x = XT ? 4096u : MODE == kMx4Up ? (uint32_t)A.rows * 128u : 128u;
    BufferSrc x, xs;
    // (the tile as an argument: captured, the compiler copies all of its registers once more in every step)
    auto load_w = [&](Tile& t, int kt) {
#pragma unroll
        for (int s = 0; s < S; s++) {
#pragma unroll
            for (int c = 0; c < 4; c++) t.w[s][c] = w[s].q.template load<true>(lane16 + (uint32_t)(c * 1024), (uint32_t)kt * 4096u);
            t.ws[s] = load_u32(w[s].s, lane4, (uint32_t)kt * 256u);
        }
    };
    auto load_x = [&](Tile& t, int kt) {
        if (FUSE) return;
#pragma unroll
        for (int c = 0; c < 4; c++) t.x[c] = x.load(off + (uint32_t)c * (XT ? 1024u : 16u), (uint32_t)kt * step_x);
        t.xs = load_u32(xs, offs, (uint32_t)kt * (step_x >> 4));
    };
    Tile tile;
    int kt = part;
    if (kt < nkt) load_w(tile, kt);               // (the weights need nothing of the rows)
    if (FUSE) {
        mx4_rows_to_lds(A.x_dtype, A.x, A.ldx, A.rows, A.K, A.Kp, s_rows);
        const int row = MODE == kMx4Up ? row0 / A.k : row0 + min(ln, rows - 1);
        off = (uint32_t)(row * mx4_lds_row(A.Kp)) + 64u * (uint32_t)kb;
        offs = (uint32_t)(A.rows * mx4_lds_row(A.Kp) + row * (A.Kp >> 5)) + 4u * (uint32_t)kb;
    } else if (XT) {
        off = lane16;
        offs = lane4;
    } else {
        const int r = min(ln, rows - 1);                                     // rows behind the last: computed and dropped
        const uint32_t row = MODE == kMx4Up ? (uint32_t)(pp.perm[row0 + r] / A.k) : (uint32_t)r;
        off = row * (MODE == kMx4Up ? 128u : (uint32_t)(A.Kp >> 1)) + 64u * (uint32_t)kb;
        offs = row * (MODE == kMx4Up ? 8u : (uint32_t)(A.Kp >> 5)) + 4u * (uint32_t)kb;
    }
    const long from = MODE == kMx4Up ? 0 : row0;
    const uint32_t held = XT ? (uint32_t)(rows + 31) / 32u * 32u : MODE == kMx4Up ? A.rows : rows;
    x.set(A.x + from * (A.Kp >> 1), held * (uint32_t)(A.Kp >> 1));
    xs.set(A.xs + from * (A.Kp >> 5), held * (uint32_t)(A.Kp >> 5));
    if (kt < nkt) load_x(tile, kt);
    float16_t acc[S] = {};
    auto multiply = [&](const Tile& t) {
#pragma unroll
        for (int s = 0; s < S; s++) {
            acc[s] = mfma_mx4<0, 0>(t.w[s][0], t.x[0], acc[s], t.ws[s], t.xs);
            acc[s] = mfma_mx4<1, 1>(t.w[s][1], t.x[1], acc[s], t.ws[s], t.xs);
            acc[s] = mfma_mx4<2, 2>(t.w[s][2], t.x[2], acc[s], t.ws[s], t.xs);
            acc[s] = mfma_mx4<3, 3>(t.w[s][3], t.x[3], acc[s], t.ws[s], t.xs);
        }
    };
    for (; kt < nkt; kt += KS) {
        if (FUSE) {
#pragma unroll
            for (int c = 0; c < 4; c++) tile.x[c] = *(const uint4*)(s_rows + off + kt * 128 + c * 16);
            tile.xs = *(const uint32_t*)(s_rows + offs + kt * 8);
        }
        multiply(tile);
        __builtin_amdgcn_sched_barrier(0);
        if (kt + KS < nkt) {
            load_w(tile, kt + KS);
            load_x(tile, kt + KS);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // the strip's sums: register kV * part + i of this lane, from the wavefronts in their order
    float sum[S][kV];
    if constexpr (KS == 1) {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int i = 0; i < 16; i++) sum[s][i] = acc[s][i];
    } else {
        const int at = mine * kParts + (part & (kParts - 1));
        auto put = [&]() {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int i = 0; i < 16; i++) s_red[at][s][i][lane] = acc[s][i];
        };
        if constexpr (KS > kParts) {
            if (part >= kParts) put();
            __syncthreads();
            if (part < kParts) {
#pragma unroll
                for (int s = 0; s < S; s++)
#pragma unroll
                    for (int i = 0; i < 16; i++) acc[s][i] += s_red[at][s][i][lane];
                put();                          // (its own place, read by none but it)
            }
        } else {
            put();
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int i = 0; i < kV; i++) {
                const int reg = kV * (part & (kParts - 1)) + i;
                float v = s_red[mine * kParts][s][reg][lane];
#pragma unroll
                for (int q = 1; q < kParts; q++) v += s_red[mine * kParts + q][s][reg][lane];
                sum[s][i] = v;
            }
    }
    // register 4 g + i: weight row 8 g + 4 kb + i, token ln
    if constexpr (MODE == kMx4Up) {
        uint32_t h[kV], m = 0;
#pragma unroll
        for (int i = 0; i < kV; i++) {
            h[i] = __float_as_uint(silu_times(sum[0][i], sum[S - 1][i]));
            m = max(m, h[i] & 0x7fffffffu);
        }
        const auto halves = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        uint32_t peak = max(halves[0], halves[1]);
        if constexpr (KS > 1) {
            if (part < kParts && kb == 0) s_peak[mine][part][ln] = peak;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kParts; q++) peak = max(peak, s_peak[mine][q][ln]);
        }
        if (part >= kParts || bx >= all) return;
        const uint32_t byte = mx4_exponent(peak);
        const float unit = mx4_unit(byte);
        const long out = (FUSE ? (long)row0 : (long)(row0 + ln)) * A.ldo + 32L * bx;
#pragma unroll
        for (int g = 0; g < kV / 4; g++) {
            uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, __uint_as_float(h[4 * g]), __uint_as_float(h[4 * g + 1]), unit, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(h[4 * g + 2]), __uint_as_float(h[4 * g + 3]), unit, 1);
            const auto both = __builtin_amdgcn_permlane32_swap(q, q, false, false);
            q = byte == 255u ? 0u : (both[0] & 0xffffu) | (both[1] << 16);
            if (kb == 0 && ln < rows) *(DYMOE_GLOBAL uint32_t*)((char*)A.out + out / 2 + 4 * (kV / 4 * part + g)) = q;
        }
        if (kb == 0 && ln < rows && part == 0) *(DYMOE_GLOBAL uint8_t*)(A.out_scale + out / 32) = (uint8_t)byte;
    } else {
        if (part >= kParts || ln >= rows) return;
#pragma unroll
        for (int g = 0; g < kV / 4; g++) {
            const int n = 32 * bx + 8 * (kV / 4 * part + g) + 4 * kb, left = A.N - n;
            if (left <= 0) continue;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[i] = sum[0][4 * g + i];
                if (MODE == kMx4Plain && A.bias) v[i] += A.bias[min(n + i, A.N - 1)];
            }
            store_any4(A.out, (long)(row0 + ln) * A.ldo + n, MODE == kMx4Plain ? A.out_dtype : DYMOE_OUT_F32, left, v);
        }
    }
}

// The down projection of a few tokens with the sum over their slots: a workgroup owns 16 outputs of one token.  The tiles of its pairs, one pair behind
// the other, are dealt to the wavefronts in equal runs, D tiles of a wavefront on their way; the intermediate's codes wait in LDS.  The
// matrix instruction's 32 weight rows are those 16 twice (the second half of the lanes asks for the same lines): with 32 outputs a workgroup, one
// token on 4096 outputs would have half as many workgroups as there are compute units.  Bound by the weights' bytes and its own start: two
// experts of 14336 x 4096 13.8 us (4.5 TB/s; the up projection before it 22.0, 5.7).
constexpr int kMx4LastWaves = 16;

template <int D>
__global__ __launch_bounds__(64 * kMx4LastWaves) void mx4_thin_down_kernel(const Mx4Args A)
{
    extern __shared__ __attribute__((aligned(16))) char s_rows[];
    __shared__ float s_sum[kMx4LastWaves][16], s_gate[64];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    // the workgroups of one strip go to one XCD, whose L2 then has the weights that several tokens need
    const int nblk = (A.N + 15) / 16, j = blockIdx.x >> 3;
    const int t = j % A.rows, bx = j / A.rows * 8 + (blockIdx.x & 7);
    if (bx >= nblk) return;
    const int k = A.k, nkt = A.Kp >> 8, strips = (A.N + 31) / 32, items = k * nkt;
    const int first = items * wave / kMx4LastWaves, last = items * (wave + 1) / kMx4LastWaves;
    const uint32_t row = (uint32_t)((lane >> 5) * 32 + (bx & 1) * 16 + (lane & 15));
    struct Tile {
        uint4 w[4];
        uint32_t ws;
    } ring[D];
    Mx4Strip w;
    int ask = first, ask_slot = first / nkt, ask_kt = first - ask_slot * nkt;
    auto open = [&](int slot) {
        // (an expert that is not there: a strip without bytes, read as zeros)
        const int e = __builtin_amdgcn_readfirstlane(A.idx[t * k + slot]);
        dymoe_expert_mx4 ex = {};
        if ((unsigned)e < (unsigned)A.E) ex = A.table[e];
        w.set(ex.q[2], ex.s[2], expert_present(ex) ? bx >> 1 : strips, strips, A.Kp);
    };
    auto request = [&](Tile& tl) {
        if (ask >= last) return;
#pragma unroll
        for (int c = 0; c < 4; c++) tl.w[c] = w.q.template load<true>(row * 16u + (uint32_t)(c * 1024), (uint32_t)ask_kt * 4096u);
        tl.ws = load_u32(w.s, row * 4u, (uint32_t)ask_kt * 256u);
        ask++;
        if (++ask_kt == nkt && ask < last) {
            ask_kt = 0;
            open(++ask_slot);
        }
    };
    if (first < last) open(ask_slot);
#pragma unroll
    for (int d = 0; d < D; d++) request(ring[d]);
    // the pairs' codes and exponents; zeros for one that is left out, whose row nobody wrote and whose weight may be no number
    const int per = A.Kp >> 5, exps = k * mx4_lds_row(A.Kp);             // 16-byte chunks of a row's codes, and bytes of its exponents
    for (int i = tid; i < k * per; i += 64 * kMx4LastWaves) {
        const int slot = i / per, c = i - slot * per, pair = t * k + slot, e = A.idx[pair];
        uint4 q = make_uint4(0, 0, 0, 0);
        uint8_t x = 0;
        const bool here = (unsigned)e < (unsigned)A.E && expert_present(A.table[e]);
        if (c == 0) s_gate[slot] = here ? A.gate[pair] : 0.0f;
        if (here) {
            q = load_global<uint4>(A.x + ((long)pair * (A.Kp >> 1) + c * 16));
            x = *(const DYMOE_GLOBAL uint8_t*)(A.xs + ((long)pair * per + c));
        }
        *(uint4*)(s_rows + slot * mx4_lds_row(A.Kp) + c * 16) = q;
        s_rows[exps + slot * per + c] = (char)x;
    }
    __syncthreads();
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float16_t acc = {};
    int slot = first / nkt, kt = first - slot * nkt;
    const int half = lane >> 5;
    for (int i = first; i < last;) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            if (i < last) {
                const char* const xr = s_rows + slot * mx4_lds_row(A.Kp) + kt * 128 + half * 64;
                const uint32_t xe = *(const uint32_t*)(s_rows + exps + slot * per + kt * 8 + half * 4);
                acc = mfma_mx4<0, 0>(ring[d].w[0], *(const uint4*)xr, acc, ring[d].ws, xe);
                acc = mfma_mx4<1, 1>(ring[d].w[1], *(const uint4*)(xr + 16), acc, ring[d].ws, xe);
                acc = mfma_mx4<2, 2>(ring[d].w[2], *(const uint4*)(xr + 32), acc, ring[d].ws, xe);
                acc = mfma_mx4<3, 3>(ring[d].w[3], *(const uint4*)(xr + 48), acc, ring[d].ws, xe);
                __builtin_amdgcn_sched_barrier(0);
                request(ring[d]);
                __builtin_amdgcn_sched_barrier(0);
                i++;
                if (++kt == nkt || i == last) {
                    // register 4 g + i holds row 8 g + 4 (lane / 32) + i, of which the first 16 are wanted
                    const float gate = s_gate[slot];
#pragma unroll
                    for (int v = 0; v < 8; v++) y[v] = fmaf(gate, acc[v], y[v]);
#pragma unroll
                    for (int v = 0; v < 16; v++) acc[v] = 0.0f;
                    kt = 0;
                    slot++;
                }
            }
        }
    }
    if ((lane & 31) == 0) {
#pragma unroll
        for (int v = 0; v < 8; v++) s_sum[wave][8 * (v >> 2) + 4 * half + (v & 3)] = y[v];
    }
    __syncthreads();
    const int n = 16 * bx + tid;
    if (tid >= 16 || n >= A.N) return;
    float sum = s_sum[0][tid];
#pragma unroll
    for (int v = 1; v < kMx4LastWaves; v++) sum += s_sum[v][tid];
    store_out(A.out, t * A.ldo + n, A.out_dtype, sum);
}

// ----------------------------------------------------------------------------
// Tiles of up to 32 NTF rows and 128 S weight rows (S / 2 times 128 of W1 and of W3 in the up projection): a workgroup of four wavefronts walks K
// in steps of 256 columns.
//  * Weights come straight into registers: a tile's bytes lie in the order of the matrix instruction's operand, so a wavefront's load is 1 KiB
//    of contiguous memory.  A register is requested anew, for the step after the next, as soon as the last instruction that reads it has been
//    issued.
//  * The rows' codes and exponents are shared by the wavefronts through three LDS buffers that global memory fills directly, two steps ahead; the 16-byte chunks of
//    a row's 128 bytes are turned by its number, which spreads the operand reads (one chunk of 32 rows) over all banks (conflicts in 2.5 % of the
//    cycles).  Rows in tiles (XT) come and lie in the operand's order by themselves: 512 x 4096 x 14336 22.9 us, 28.7 row by row.
// 2047 x 14336 x 4096: 72 to 77 us from box to box, 3.1 to 3.3 PFLOP/s, the matrix units busy in 51 % of a compute unit's busy cycles and 37 % of the launch's;
// codes made before, row by row: 80 us beside 77; with zeros in place of random codes 62 and 58 (the clock is the power's to set); 8192 x 8192 x 8192
// 4.0 PFLOP/s, 4.7 with zeros, of 5.3 to 6.4 that these instructions reach on random codes from registers alone.  Experts with 128 rows each, 8 of 14336 x 4096: the stream of weights, 4.3 TB/s beside the rows' copies from L2 (with 8
// rows 5.6): a compute unit's requests for either wait in one queue.
constexpr uint32_t kMx4Row = 128;           // bytes of a row of a step
template <int NTF>
constexpr uint32_t kMx4Buf = 32u * NTF * (kMx4Row + 8u);
template <int S>
constexpr uint32_t kMx4EpiRow = S == 2 ? 272 : 144;      // epilogue: bytes of a row of 32 S sums in LDS, 16 of them padding
template <int S>
constexpr uint32_t kMx4EpiWave = 32 * kMx4EpiRow<S>;

__device__ __forceinline__ int mx4_turn(int row) { return (row >> 1) & 7; }      // (the row's parity is half of the banks already)

template <int S, int D>
struct Mx4Weights {
    uint4 r[D][S][4];              // codes of this step and of those behind it
    uint32_t e[D][S];              // exponents
    Mx4Strip strip[S];

    __device__ __forceinline__ void codes(int p, int c, uint32_t lane16, int step)
    {
#pragma unroll
        for (int s = 0; s < S; s++) r[p][s][c] = strip[s].q.load(lane16 + (uint32_t)(c * 1024), (uint32_t)step * 4096u);
    }
    __device__ __forceinline__ void scales(int p, uint32_t lane16, int step)
    {
#pragma unroll
        for (int s = 0; s < S; s++) e[p][s] = load_u32(strip[s].s, lane16 >> 2, (uint32_t)step * 256u);
    }
};

template <int MODE, int NTF, int S, int D, int RR, bool XT>
__device__ __forceinline__ void mx4_tile(const Mx4Args& A, const int32_t* perm, Mx4Weights<S, D>& w, int row0, int rows, long held_at, int bx, int step0, int steps, void* out,
                                         uint32_t base)
{
    constexpr int kMask = 0x2 | 0x4;             // vector and scalar arithmetic may cross; products, LDS and memory accesses may not
    constexpr uint32_t kBuf = kMx4Buf<NTF>, kExp = 32u * NTF * kMx4Row;
    constexpr int kCopies = NTF + (NTF + 3) / 4;
    constexpr int R = RR < 4 * NTF ? RR : 4 * NTF;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const uint32_t lane16 = (uint32_t)lane * 16u;
    const int end = steps - 1;
    float16_t acc[S][NTF] = {};
    // copies: rows 32 i + 8 wave + lane / 8, chunk lane % 8 turned (XT: chunk `wave` of all rows); exponents of fragment `wave` (and wave + 4)
    const long kStepX = XT ? 4096 : MODE == kMx4Up ? A.rows * 128L : 128, kStepE = kStepX >> 4;
    const char* const xb = A.x + (MODE == kMx4Up ? 0 : held_at * (A.Kp >> 1)) + step0 * kStepX;
    const char* const sb = A.xs + (MODE == kMx4Up ? 0 : held_at * (A.Kp >> 5)) + step0 * kStepE;
    uint32_t off[NTF], offs[(NTF + 3) / 4];
    auto source = [&](int r) {                   // rows behind the last: computed and dropped
        r = min(r, rows - 1);
        return MODE == kMx4Up ? (uint32_t)(perm[row0 + r] / A.k) : (uint32_t)r;
    };
    const int rb = 8 * wave + (lane >> 3);
#pragma unroll
    for (int i = 0; i < NTF; i++)
        off[i] = XT ? (uint32_t)i * 16u * (uint32_t)A.Kp + (uint32_t)wave * 1024u + lane16 : source(32 * i + rb) * (MODE == kMx4Up ? 128u : (uint32_t)(A.Kp >> 1)) + 16u * (uint32_t)((lane & 7) ^ mx4_turn(rb));
    // (wavefronts without a fragment of their own copy the last one's exponents again: the count of copies is then every wavefront's)
#pragma unroll
    for (int i = 0; i < (NTF + 3) / 4; i++)
        offs[i] = XT ? (uint32_t)min(wave + 4 * i, NTF - 1) * (uint32_t)A.Kp + (lane16 >> 2) : source(32 * min(wave + 4 * i, NTF - 1) + (lane >> 1)) * (MODE == kMx4Up ? 8u : (uint32_t)(A.Kp >> 5)) + 4u * (uint32_t)(lane & 1);
    auto copy = [&](int step, uint32_t buf) {
#pragma unroll
        for (int i = 0; i < NTF; i++)
            lds_copy16(xb + step * kStepX, off[i], __builtin_amdgcn_readfirstlane(base + buf + (uint32_t)(i * 4096 + wave * 1024)));
#pragma unroll
        for (int i = 0; i < (NTF + 3) / 4; i++)
            lds_copy4(sb + step * kStepE, offs[i], __builtin_amdgcn_readfirstlane(base + buf + kExp + (uint32_t)(min(wave + 4 * i, NTF - 1) * 256)));
    };
#pragma unroll
    for (int p = 0; p < D; p++) copy(min(p, end), (uint32_t)p * kBuf);
#pragma unroll
    for (int p = 0; p < D; p++) {
        // (in the loop's order: what the compiler waits for at the loop's head is then what a step behind another needs)
        w.scales(p, lane16, step0 + min(p, end));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 4; c++) {
            w.codes(p, c, lane16, step0 + min(p, end));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    wait_lds_copies<(D - 1) * kCopies + 5 * D * S>();        // the first copies are older than everything else
    __syncthreads();
    const uint32_t xa0 = XT ? base + lane16 : base + (uint32_t)ln * kMx4Row + (((uint32_t)kb << 6) ^ ((uint32_t)mx4_turn(ln) << 4));
    const uint32_t xe0 = base + kExp + (XT ? lane16 >> 2 : (uint32_t)ln * 8u + (uint32_t)kb * 4u);
    uint32_t at = 0;
    // Step ks multiplies what its buffer and registers hold and requests the codes of the rows and of the weights D steps on.
    auto step = [&](int ks, auto slot) __attribute__((always_inline)) {
        constexpr int p = slot();
        const int after = min(ks + D, end);
        // What a step waits for first is requested first, and the copies behind its first products: the compiler does not count them, so that
        // a wait of its own for a load that copies were issued behind is one for younger loads too.
        uint32_t now[S];
#pragma unroll
        for (int s = 0; s < S; s++) asm volatile("v_mov_b32 %0, %1" : "=v"(now[s]) : "v"(w.e[p][s]));      // (here, and not at the end of the loop)
        __builtin_amdgcn_sched_barrier(kMask);
        w.scales(p, lane16, step0 + after);
        uint32_t xe[NTF];
#pragma unroll
        for (int f = 0; f < NTF; f++) xe[f] = lds_read4(xe0 + at + (uint32_t)f * 256u);
        // the operands of the next R products of a chunk and a fragment are read while this one's are issued
        uint4 op[R];
        auto read = [&](int o) { return XT ? lds_read16(xa0 + at + (uint32_t)((o / NTF) * 1024 + (o % NTF) * 4096)) : lds_read16(((xa0 + at) ^ (uint32_t)((o / NTF) << 4)) + (uint32_t)(o % NTF) * (32u * kMx4Row)); };
#pragma unroll
        for (int o = 0; o < R; o++) op[o] = read(o);
        auto chunk = [&](auto which) __attribute__((always_inline)) {
            constexpr int c = which();
#pragma unroll
            for (int f = 0; f < NTF; f++) {
                const int o = c * NTF + f;
                __builtin_amdgcn_sched_barrier(kMask);
#pragma unroll
                for (int s = 0; s < S; s++) acc[s][f] = mfma_mx4<c, c>(w.r[p][s][c], op[o % R], acc[s][f], now[s], xe[f]);
                __builtin_amdgcn_sched_barrier(kMask);
                if (o + R < 4 * NTF) op[o % R] = read(o + R);
            }
            if constexpr (c == 0) copy(after, at == 0 ? D * kBuf : at - kBuf);         // (the buffer of the step before)
            w.codes(p, c, lane16, step0 + after);
            __builtin_amdgcn_sched_barrier(kMask);
        };
        chunk(std::integral_constant<int, 0>());
        chunk(std::integral_constant<int, 1>());
        chunk(std::integral_constant<int, 2>());
        chunk(std::integral_constant<int, 3>());
        // behind the next step's copies: the loads of codes of the step that asked for them, and all of the steps since
        wait_lds_copies<4 * S + (D - 1) * (kCopies + 5 * S)>();
        __syncthreads();
        at = at == D * kBuf ? 0 : at + kBuf;
    };
    int ks = 0;
    for (; ks + D <= steps; ks += D) {
        step(ks, std::integral_constant<int, 0>());
        step(ks + 1, std::integral_constant<int, 1>());
        if constexpr (D > 2) step(ks + 2, std::integral_constant<int, 2>());
        if constexpr (D > 3) step(ks + 3, std::integral_constant<int, 3>());
    }
    if (ks < steps) step(ks, std::integral_constant<int, 0>());
    if constexpr (D > 2)
        if (ks + 1 < steps) step(ks + 1, std::integral_constant<int, 1>());
    if constexpr (D > 3)
        if (ks + 2 < steps) step(ks + 2, std::integral_constant<int, 2>());
    // (the copies requested beyond the end: the buffers are the epilogue's now)
    wait_lds_copies<0>();
    __syncthreads();

    // A lane holds, of its token's row, four neighbouring outputs in each group of four registers.  The intermediate goes into tiles, where a fragment's
    // 32 rows of a block are 512 bytes, and comes back as the down projection's rows: 512 tokens, 2 of 8 experts of 14336 x 4096 212 -> 202 us, 2047
    // tokens 459 -> 438.  (Not from strips: tiles of few rows would read all 32, 61 tokens on 8 of 128 experts of 768 x 2048 63 -> 66.)
    if constexpr (MODE == kMx4Up) {
        // the halves of a wavefront hold a block together: 16 numbers each
#pragma unroll
        for (int u = 0; u < S / 2; u++) {
            const int block = (4 * bx + wave) * (S / 2) + u;
            if (block * 32 >= A.ldo) continue;
#pragma unroll
            for (int f = 0; f < NTF; f++) {
                const int row = 32 * f + ln;
                float h[16];
                uint32_t peak = 0;
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    h[i] = silu_times(acc[2 * u][f][i], acc[2 * u + 1][f][i]);
                    peak = max(peak, __float_as_uint(h[i]) & 0x7fffffffu);
                }
                const auto both = __builtin_amdgcn_permlane32_swap(peak, peak, false, false);
                const uint32_t byte = mx4_exponent(max(both[0], both[1]));
                const float unit = mx4_unit(byte);
                uint32_t q[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, h[8 * i], h[8 * i + 1], unit, 0);
                    q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], h[8 * i + 2], h[8 * i + 3], unit, 1);
                    q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], h[8 * i + 4], h[8 * i + 5], unit, 2);
                    q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], h[8 * i + 6], h[8 * i + 7], unit, 3);
                    if (byte == 255u) q[i] = 0;
                }
                const auto a = __builtin_amdgcn_permlane32_swap(q[0], q[0], false, false), b = __builtin_amdgcn_permlane32_swap(q[1], q[1], false, false);
                const uint4 all = make_uint4((a[0] & 0xffffu) | (a[1] << 16), (a[0] >> 16) | (a[1] & 0xffff0000u), (b[0] & 0xffffu) | (b[1] << 16),
                                             (b[0] >> 16) | (b[1] & 0xffff0000u));
                if (row >= rows) continue;
                if (kb == 0) store_global((char*)out + mx4_tile_byte(held_at + row, 32L * block, A.ldo), all);
                else *(DYMOE_GLOBAL uint8_t*)(A.out_scale + mx4_tile_exponent(held_at + row, 32L * block, A.ldo)) = (uint8_t)byte;
            }
        }
    } else {
        // the wavefront turns a fragment round in an LDS area of its own, so that a row leaves in whole lines
        constexpr int kOut = 8 * S;                 // lanes to a row of the wavefront's 32 S sums
        const uint32_t area = base + (uint32_t)wave * kMx4EpiWave<S>, wr = area + (uint32_t)ln * kMx4EpiRow<S> + (uint32_t)kb * 16u;
        const int dt = MODE == kMx4Plain ? A.out_dtype : DYMOE_OUT_F32;
        const int n = (4 * bx + wave) * 32 * S + 4 * (lane & (kOut - 1)), left = A.N - n;
        float add[4] = {0.f, 0.f, 0.f, 0.f};
        if (MODE == kMx4Plain && A.bias) {
#pragma unroll
            for (int i = 0; i < 4; i++) add[i] = A.bias[min(n + i, A.N - 1)];
        }
#pragma unroll
        for (int f = 0; f < NTF; f++) {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int g = 0; g < 4; g++)
                    lds_write16(wr + (uint32_t)(128 * s + 32 * g), make_uint4(__float_as_uint(acc[s][f][4 * g]), __float_as_uint(acc[s][f][4 * g + 1]),
                                                                              __float_as_uint(acc[s][f][4 * g + 2]), __float_as_uint(acc[s][f][4 * g + 3])));
            // (a wavefront's LDS accesses execute in order and the area is its own: no barrier)
#pragma unroll
            for (int j = 0; j < 32 * kOut / 64; j++) {
                const int rr = lane / kOut + 64 / kOut * j, row = 32 * f + rr;
                const uint4 u = lds_read16(area + (uint32_t)rr * kMx4EpiRow<S> + (uint32_t)(lane & (kOut - 1)) * 16u);
                if (row >= rows || left <= 0) continue;
                const float v[4] = {__uint_as_float(u.x) + add[0], __uint_as_float(u.y) + add[1], __uint_as_float(u.z) + add[2], __uint_as_float(u.w) + add[3]};
                store_any4(out, (long)(row0 + row) * A.ldo + n, dt, left, v);
            }
        }
    }
}

// Neighbouring units that an XCD takes at a time: workgroups go to the 8 XCDs, each with an L2 of its own, in turn, and units that read the same
// weights (the tiles of a matrix or expert, for one column block) are neighbours.
constexpr int kMx4Run = 8;
__device__ __forceinline__ long mx4_unit_of_group() { return ((long)(blockIdx.x >> 3) / kMx4Run * 8 + (blockIdx.x & 7)) * kMx4Run + (blockIdx.x >> 3) % kMx4Run; }
static long mx4_groups(long units) { return ((units + kMx4Run - 1) / kMx4Run + 7) / 8 * 8 * kMx4Run; }
static dim3 mx4_grid(long units) { return dim3((unsigned)mx4_groups(units)); }

__device__ __forceinline__ uint32_t mx4_lds_base(char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)p; }

// weight rows of a workgroup's block: of the up projection, those of W1
template <int MODE, int S>
constexpr int kMx4Cols = 128 * (MODE == kMx4Up ? S / 2 : S);

template <int MODE, int MAXF, int S, int D, int RR, bool XT = false>
__global__ __launch_bounds__(256, MAXF * S <= 8 ? 2 : 1) void mx4_tall_kernel(const Mx4Args A)
{
    extern __shared__ __attribute__((aligned(1024))) char lds_raw[];
    const uint32_t base = mx4_lds_base(lds_raw);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    constexpr int kCols = kMx4Cols<MODE, S>, kRows = 32 * MAXF;
    const int strips = (A.N + 31) / 32, nblk = (int)(((MODE == kMx4Up ? A.ldo : A.N) + kCols - 1) / kCols);
    const Mx4Plan pp = expert_plan<dymoe_expert_mx4>(const_cast<int32_t*>(A.plan), A.P);
    const long unit = mx4_unit_of_group();
    Mx4Weights<S, D> w;
    int row0, rows, bx, step0 = 0, steps = A.Kp >> 8;
    long held_at;
    void* out = A.out;
    if (MODE == kMx4Plain) {
        const int tiles = (A.rows + kRows - 1) / kRows;
        if (unit >= (long)tiles * nblk) return;
        bx = (int)(unit / tiles);
        row0 = (int)(unit - (long)bx * tiles) * kRows;
        rows = min(kRows, A.rows - row0);
        held_at = row0;
#pragma unroll
        for (int s = 0; s < S; s++) w.strip[s].set(A.w, A.ws, (4L * bx + wave) * S + s, strips, A.Kp);
    } else {
        const int splits = MODE == kMx4Down ? A.splits : 1;
        if (unit >= (long)pp.meta[0] * nblk * splits) return;
        const ExpertTile<dymoe_expert_mx4> t = pp.tiles[unit / (nblk * splits)];
        long local = unit - (long)t.tile0 * (nblk * splits);
        if (MODE == kMx4Down) {
            const int part = (int)(local / ((long)t.tiles * nblk));
            local -= (long)part * t.tiles * nblk;
            step0 = steps * part / splits;
            steps = steps * (part + 1) / splits - step0;
            out = (float*)out + part * A.P * A.ldo;
        }
        bx = (int)(local / t.tiles);
        const int i = (int)(local - (long)bx * t.tiles) * kRows;
        row0 = t.first + i;
        rows = min(kRows, t.pairs - i);
        held_at = 32L * (t.first / 32 + t.tile0) + i;
#pragma unroll
        for (int s = 0; s < S; s++) {
            if (MODE == kMx4Up) w.strip[s].set(s & 1 ? t.mat.q[1] : t.mat.q[0], s & 1 ? t.mat.s[1] : t.mat.s[0], (4L * bx + wave) * (S / 2) + s / 2, strips, A.Kp);
            else w.strip[s].set(t.mat.q[2], t.mat.s[2], (4L * bx + wave) * S + s, strips, A.Kp);
        }
    }
    // one instantiation per number of fragments of 32 rows: the accumulators then sit in fixed registers for the whole loop
#define DYMOE_MX4_TILE(NTF) mx4_tile<MODE, NTF, S, D, RR, XT>(A, pp.perm, w, row0, rows, held_at, bx, step0, steps, out, base)
    switch ((rows + 31) >> 5) {
    case 1: DYMOE_MX4_TILE(1); break;
    case 2: DYMOE_MX4_TILE(MAXF < 2 ? MAXF : 2); break;
    case 3: DYMOE_MX4_TILE(MAXF < 3 ? MAXF : 3); break;
    default: DYMOE_MX4_TILE(MAXF); break;
    }
#undef DYMOE_MX4_TILE
}

// three buffers or more, or the epilogue's areas
template <int MAXF, int S, int D>
constexpr int kMx4Lds = (int)((D + 1) * kMx4Buf<MAXF> > 4 * kMx4EpiWave<S> ? (D + 1) * kMx4Buf<MAXF> : 4 * kMx4EpiWave<S>);

// A shape's instantiation: the tile's fragments of 32 rows, strips of a wavefront, steps ahead, operands ahead.
#define DYMOE_MX4_TILE32(MODE, XT) mx4_tall_kernel<MODE, 1, 1, 4, 4, XT>
#define DYMOE_MX4_TILE64(MODE, XT) mx4_tall_kernel<MODE, 2, 1, 3, 4, XT>
#define DYMOE_MX4_TILE64W(MODE, XT) mx4_tall_kernel<MODE, 2, 2, 2, 4, XT>
#define DYMOE_MX4_TILE128(MODE, XT) mx4_tall_kernel<MODE, 4, 2, 2, 3, XT>

// per-device set-up, with the device current
int mx4_init()
{
    auto allow = [](const void* f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess; };
    auto plain = [&](auto xt) {
        constexpr bool XT = decltype(xt)::value;
        return allow((const void*)DYMOE_MX4_TILE32(kMx4Plain, XT), kMx4Lds<1, 1, 4>) && allow((const void*)DYMOE_MX4_TILE64(kMx4Plain, XT), kMx4Lds<2, 1, 3>) &&
               allow((const void*)DYMOE_MX4_TILE64W(kMx4Plain, XT), kMx4Lds<2, 2, 2>) && allow((const void*)DYMOE_MX4_TILE128(kMx4Plain, XT), kMx4Lds<4, 2, 2>);
    };
    bool ok = plain(std::false_type()) && plain(std::true_type());
    ok = ok && allow((const void*)DYMOE_MX4_TILE128(kMx4Up, false), kMx4Lds<4, 2, 2>) && allow((const void*)DYMOE_MX4_TILE128(kMx4Down, true), kMx4Lds<4, 2, 2>);
    ok = ok && allow((const void*)mx4_small_kernel<kMx4Plain, 8, 8, true>, (int)kMx4FuseBytes) &&
         allow((const void*)mx4_small_kernel<kMx4Up, 4, 4, true>, (int)kMx4FuseBytes) && allow((const void*)mx4_thin_down_kernel<2>, (int)kMx4FuseBytes);
    return ok ? DYMOE_OK : DYMOE_EHIP;
}

// y[t] = sum over the slots, in their order, of gate times the pair's output, which is the sum of its parts.  A workgroup takes 2048 outputs of a
// token.  Bound by the pairs' bytes: 16376 pairs of 2048 outputs 22.1 us (6.1 TB/s).
template <int PARTS>
__global__ __launch_bounds__(256) void mx4_combine_kernel(const float* __restrict__ part, long ldp, long P, const int32_t* __restrict__ where,
                                                          const float* __restrict__ gate, int H, int k, int out_dtype, void* __restrict__ y)
{
    const int blocks = (H + 2047) / 2048;
    const long t = blockIdx.x / blocks;
    const int h = (int)(blockIdx.x - t * blocks) * 2048 + threadIdx.x * 8;
    if (h >= H) return;
    constexpr int kAhead = PARTS > 1 ? 2 : 4;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll kAhead
    for (int j = 0; j < k; j++) {
        const int at = where[t * k + j];
        if (at < 0) continue;
        const float g = gate[t * k + j];
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < PARTS; p++) {
            const float* const from = part + (p * P + at) * ldp + h;
            const float4 a = load_global<float4>(from), b = load_global<float4>(from + 4);
            const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = p == 0 ? w[i] : v[i] + w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] = fmaf(g, v[i], sum[i]);
    }
    const float lo[4] = {sum[0], sum[1], sum[2], sum[3]}, hi[4] = {sum[4], sum[5], sum[6], sum[7]};
    store_any4(y, t * H + h, out_dtype, H - h, lo);
    store_any4(y, t * H + h + 4, out_dtype, H - h - 4, hi);
}

// a launch's threads have to stay below 2^32
static bool fits_grid(long groups, int threads) { return groups < (1L << 32) / threads; }

}  // namespace dymoe

using namespace dymoe;

extern "C" size_t dymoe_matmul_mx4_workspace_bytes(int T, int N, int K)
{
    if (T < 0 || N <= 0 || K <= 0 || K > DYMOE_MX4_MAX_K) return 0;
    return mx4_mat_layout(T, K).total;
}

extern "C" int dymoe_matmul_mx4(dymoe_ctx* ctx, const void* x, int x_dtype, const uint8_t* x_scale, long ldx, const uint8_t* w,
                                const uint8_t* w_scale, const float* bias, int T, int N, int K, int out_dtype, void* y, long ldy,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    DYMOE_REQUIRE(T >= 0 && N > 0 && K > 0 && ldy >= N);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16 || x_dtype == DYMOE_DTYPE_MX4);
    DYMOE_REQUIRE(out_dtype == DYMOE_OUT_BF16 || out_dtype == DYMOE_OUT_F32 || out_dtype == DYMOE_OUT_F16);
    const bool coded = x_dtype == DYMOE_DTYPE_MX4;
    DYMOE_REQUIRE(coded ? ldx == up_to(K, kMx4TileCols) : ldx >= K);
    DYMOE_REQUIRE(w && w_scale);
    if (T > 0) DYMOE_REQUIRE(x && y && (coded ? x_scale != nullptr : workspace != nullptr));
    DYMOE_REQUIRE(dymoe_aligned(x, coded ? 16 : dtype_bytes(x_dtype)) && dymoe_aligned(y, dtype_bytes(out_dtype)) && dymoe_aligned(w, 16));
    DYMOE_REQUIRE(dymoe_aligned(x_scale, 4) && dymoe_aligned(w_scale, 4) && dymoe_aligned(bias, 4) && dymoe_aligned(workspace, 256));
    if (K > DYMOE_MX4_MAX_K || T > (1 << 24) || N > (1 << 24)) return DYMOE_ENOTSUP;
    const Mx4MatLayout L = mx4_mat_layout(T, K);
    if (!coded && T > 0 && workspace_bytes < L.total) return DYMOE_ENOSPC;
    // (the other shapes are taken while tiles are few, or with up to 32 rows: 2^19 strips of 512 threads at most)
    const long n128 = (N + 127L) / 128, n256 = (N + 255L) / 256, t128 = (T + 127L) / 128;
    if (!fits_grid(mx4_groups(t128 * n256), 256)) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const Mx4MatChoice c = mx4_mat_choice(T, N, K, coded, ctx->num_cu);
    Mx4Args A = {};
    A.x = (const char*)x;
    A.xs = (const char*)x_scale;
    if (c.fuse) {
        A.ldx = ldx * dtype_bytes(x_dtype);
        A.x_dtype = x_dtype;
        A.K = K;
    } else if (!coded) {
        const int rc = mx4_quantize(ctx, x, x_dtype, T, K, ldx, 1, (uint8_t*)ws + L.xq, (uint8_t*)ws + L.xs, st);
        if (rc != DYMOE_OK) return rc;
        A.x = ws + L.xq;
        A.xs = ws + L.xs;
    }
    A.w = (const char*)w;
    A.ws = (const char*)w_scale;
    A.bias = bias;
    A.out = y;
    A.ldo = ldy;
    A.rows = T;
    A.Kp = (int)L.Kp;
    A.N = N;
    A.out_dtype = out_dtype;
    const long groups = (T + 31L) / 32 * ((N + 31L) / 32);
    auto run = [&](void (*kernel)(const Mx4Args), dim3 grid, int threads, int lds) {
        dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, kernel, grid, dim3((unsigned)threads), lds, st, A);
    };
    // rows converted in the call lie in tiles, codes made before row by row
    auto launch = [&](auto xt) {
        constexpr bool XT = decltype(xt)::value;
        const long t32 = (T + 31L) / 32, t64 = (T + 63L) / 64;
        switch (c.shape) {
        case Mx4MatShape::kSmall:
            if (c.waves == 8) run(mx4_small_kernel<kMx4Plain, 8, 8, false, XT>, dim3((unsigned)groups), 512, 0);
            else run(mx4_small_kernel<kMx4Plain, 4, 4, false, XT>, dim3((unsigned)groups), 256, 0);
            break;
        case Mx4MatShape::kTile32: run(DYMOE_MX4_TILE32(kMx4Plain, XT), mx4_grid(t32 * n128), 256, kMx4Lds<1, 1, 4>); break;
        case Mx4MatShape::kTile64: run(DYMOE_MX4_TILE64(kMx4Plain, XT), mx4_grid(t64 * n128), 256, kMx4Lds<2, 1, 3>); break;
        case Mx4MatShape::kTile64w: run(DYMOE_MX4_TILE64W(kMx4Plain, XT), mx4_grid(t64 * n256), 256, kMx4Lds<2, 2, 2>); break;
        default: run(DYMOE_MX4_TILE128(kMx4Plain, XT), mx4_grid(t128 * n256), 256, kMx4Lds<4, 2, 2>);
        }
    };
    if (c.fuse) run(mx4_small_kernel<kMx4Plain, 8, 8, true, false>, dim3((unsigned)groups), 512, (int)mx4_fuse_bytes(T, L.Kp));
    else if (coded) launch(std::false_type());
    else launch(std::true_type());
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

extern "C" size_t dymoe_moe_ffn_mx4_workspace_bytes(int T, int H, int F, int E, int k)
{
    if (T < 0 || H <= 0 || F <= 0 || E <= 0 || k <= 0 || k > E) return 0;
    return mx4_ffn_layout(T, H, F, E, k).total;
}

extern "C" int dymoe_moe_ffn_mx4(dymoe_ctx* ctx, const void* x, int x_dtype, const int32_t* idx, const float* w, const dymoe_expert_mx4* table,
                                 int T, int H, int F, int E, int k, int out_dtype, void* y, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    DYMOE_REQUIRE(T >= 0 && H > 0 && F > 0 && E > 0 && k > 0 && k <= E);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(out_dtype == DYMOE_OUT_BF16 || out_dtype == DYMOE_OUT_F32 || out_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(table && workspace);
    if (T > 0) DYMOE_REQUIRE(x && idx && w && y);
    DYMOE_REQUIRE(dymoe_aligned(x, dtype_bytes(x_dtype)) && dymoe_aligned(y, dtype_bytes(out_dtype)) && dymoe_aligned(workspace, 256));
    DYMOE_REQUIRE(dymoe_aligned(idx, 4) && dymoe_aligned(w, 4) && dymoe_aligned(table, 8));
    if (E > DYMOE_MAX_EXPERTS || H > DYMOE_MX4_MAX_K || F > DYMOE_MX4_MAX_K) return DYMOE_ENOTSUP;
    const long P = (long)T * k;
    if (P >= 1L << 29 || (long)T * up_to(H, kMx4TileCols) / 2 >= 1L << 32) return DYMOE_ENOTSUP;      // (32-bit offsets into the codes)
    const Mx4FfnLayout L = mx4_ffn_layout(T, H, F, E, k);
    if (workspace_bytes < L.total) return DYMOE_ENOSPC;
    // Tall tiles' workgroups; K is in parts only where they are few.  (Strips are taken for up to 20 E pairs, or 32 tokens: 2048 tiles of 4096 strips at
    // most, four to a workgroup of 256 threads.)
    const long tall = P / kMx4TallRows + (E < P ? E : P);
    if (!fits_grid(mx4_groups(tall * (long)(L.Fp / 128)), 256) || !fits_grid(mx4_groups(tall * ((H + 255L) / 256)), 256) ||
        !fits_grid(T * ((H + 2047L) / 2048), 256))
        return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const Mx4FfnChoice c = mx4_ffn_choice(T, H, F, E, k, ctx->num_cu);
    Mx4Args A = {};
    A.out = ws + L.hq;
    A.out_scale = (uint8_t*)ws + L.hs;
    A.ldo = (long)L.Fp;
    A.P = P;
    A.rows = T;
    A.Kp = (int)L.Hp;
    A.N = F;
    A.k = k;
    A.splits = 1;
    auto run = [&](void (*kernel)(const Mx4Args), dim3 grid, int threads, int lds) {
        dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, kernel, grid, dim3((unsigned)threads), lds, st, A);
    };
    // from the up to the down projection
    auto turn = [&](void* out, long ldo, int dt) {
        A.x = ws + L.hq;
        A.xs = ws + L.hs;
        A.out = out;
        A.ldo = ldo;
        A.Kp = (int)L.Fp;
        A.N = H;
        A.out_dtype = dt;
    };
    if (c.shape == Mx4FfnShape::kThin) {
        A.x = (const char*)x;
        A.ldx = (long)H * dtype_bytes(x_dtype);
        A.x_dtype = x_dtype;
        A.K = H;
        A.idx = idx;
        A.gate = w;
        A.table = table;
        A.flags = ctx->device_flags;
        A.E = E;
        run(mx4_small_kernel<kMx4Up, 4, 4, true>, dim3((unsigned)(P * (long)(L.Fp / 32))), 256, (int)mx4_fuse_bytes(T, L.Hp));
        turn(y, H, out_dtype);
        run(mx4_thin_down_kernel<2>, dim3((unsigned)(8L * T * (((H + 15L) / 16 + 7) / 8))), 64 * kMx4LastWaves, (int)mx4_fuse_bytes(k, L.Fp));
        DYMOE_HIP_LAUNCH_CHECK();
        return DYMOE_OK;
    }
    const bool small = c.shape == Mx4FfnShape::kSmall;
    int32_t* const plan = (int32_t*)(ws + L.plan);
    const int per_row = (int)((L.Hp + 511) / 512);
    const int units = T * per_row;              // (at most 2^25: T times Hp is below 2^33)
    auto prep = mx4_prep_kernel<DYMOE_OUT_BF16>;
    if (x_dtype == DYMOE_OUT_F32) prep = mx4_prep_kernel<DYMOE_OUT_F32>;
    else if (x_dtype == DYMOE_OUT_F16) prep = mx4_prep_kernel<DYMOE_OUT_F16>;
    dymoe_launch(ctx, DYMOE_K_MX4_ROWS, prep, dim3((unsigned)(1 + (units + 15) / 16)), dim3(kPlanThreads), 0, st, idx, table, P, E, (int)small, plan,
                 ctx->device_flags, (const char*)x, T, units, per_row, H, ws + L.xq, ws + L.xs);
    A.x = ws + L.xq;
    A.xs = ws + L.xs;
    A.plan = plan;
    auto strips = [&](long n, int each) { return dim3((unsigned)(L.max_tiles * ((n + each - 1) / each))); };
    const long fs = (long)(L.Fp / 32), hs = (H + 31L) / 32;
    if (!small) run(DYMOE_MX4_TILE128(kMx4Up, false), mx4_grid(tall * (long)(L.Fp / 128)), 256, kMx4Lds<4, 2, 2>);
    else if (c.up_waves == 4) run(mx4_small_kernel<kMx4Up, 4, 4>, strips(fs, 1), 256, 0);
    else if (c.up_waves == 2) run(mx4_small_kernel<kMx4Up, 4, 2>, strips(fs, 2), 256, 0);
    else run(mx4_small_kernel<kMx4Up, 4, 1>, strips(fs, 4), 256, 0);
    turn(ws + L.part, (long)mx4_round((size_t)H, 8), DYMOE_OUT_F32);
    A.splits = c.splits;
    if (!small) run(DYMOE_MX4_TILE128(kMx4Down, true), mx4_grid(tall * ((H + 255L) / 256) * c.splits), 256, kMx4Lds<4, 2, 2>);
    else if (c.down_waves == 8) run(mx4_small_kernel<kMx4Down, 8, 8>, strips(hs, 1), 512, 0);
    else if (c.down_waves == 4) run(mx4_small_kernel<kMx4Down, 4, 4>, strips(hs, 1), 256, 0);
    else if (c.down_waves == 2) run(mx4_small_kernel<kMx4Down, 4, 2>, strips(hs, 2), 256, 0);
    else run(mx4_small_kernel<kMx4Down, 4, 1>, strips(hs, 4), 256, 0);
    auto combine = c.splits == 1 ? mx4_combine_kernel<1> : c.splits == 2 ? mx4_combine_kernel<2> : mx4_combine_kernel<4>;
    dymoe_launch(ctx, DYMOE_K_MX4_ROWS, combine, dim3((unsigned)(T * ((H + 2047L) / 2048))), dim3(256), 0, st, (const float*)(ws + L.part), A.ldo, P,
                 expert_plan<dymoe_expert_mx4>(plan, P).where, w, H, k, out_dtype, y);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
