// Products in 8-bit integers with a scale for each token and each channel: a matrix (dymoe_matmul_int8) and a layer's SwiGLU
// experts (dymoe_moe_ffn_int8).
//   y[t, n] = xs[t] ws[n] sum_k xq[t, k] wq[n, k]
// The sums are whole numbers of 32 bits (127 * 127 * K < 2^31 up to K = 131072), so their order does not matter and every split of K gives
// the same bits.
#include <type_traits>

#include "int8_device.hpp"
#include "int8_rule.hpp"

namespace dymoe {

int quantize_rows(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, void* codes, float* scale, hipStream_t st);

// A tile of an expert: all that a workgroup has to know before its first load of weights.
struct __attribute__((aligned(16))) I8TileRec {
    int32_t first, pairs;             // the expert's first position, its pairs
    int32_t tile0, tiles;             // its first tile, its tiles
    dymoe_expert_i8 mat;
};

struct I8Plan {
    int32_t* meta;        // [8]: tiles, wide tiles behind them
    int32_t* perm;        // [P] position -> pair
    int32_t* where;       // [P] pair -> position, -1: left out
    I8TileRec* tiles;
};

__host__ __device__ inline I8Plan i8_plan(int32_t* p, long P)
{
    I8Plan r;
    r.meta = p;
    r.perm = r.meta + 8;
    r.where = r.perm + P;
    r.tiles = (I8TileRec*)(p + 8 + (2 * P + 3) / 4 * 4);
    return r;
}

__device__ __forceinline__ bool i8_present(const dymoe_expert_i8& x)
{
    return (x.q[0] != nullptr) & (x.q[1] != nullptr) & (x.q[2] != nullptr) & (x.s[0] != nullptr) & (x.s[1] != nullptr) & (x.s[2] != nullptr);
}

// Counting sort of the pairs by expert and the list of tiles, by one workgroup: tall tiles first, then wide ones, by expert.  A pair's turn
// in its expert is what the counter held before it: kept in registers (in `where` beyond the first kI8PlanKeep pairs of a thread)
// until the experts' first positions are known, so that there is one pass of atomics.  The turns come in any order, and nothing that is
// computed depends on it.  The sorted pairs and the tiles' experts pass through LDS where they fit: written from the threads that
// know them, 16384 pairs cost 7 us in stores of four bytes each, and an expert's sixteen records 3 us in one thread.  16384 pairs of 128
// experts 12.1 us with 2048 rows' codes beside it, 488 pairs 4.6: latencies of one workgroup's passes, not bytes.
constexpr int kI8PlanThreads = 1024;
constexpr int kI8PlanKeep = 16;
constexpr int kI8PlanPairs = kI8PlanKeep * kI8PlanThreads;
constexpr int kI8PlanTiles = 4096;

static_assert(kI8PlanThreads == DYMOE_MAX_EXPERTS, "a thread for every expert");

struct I8PlanLds {
    int count[DYMOE_MAX_EXPERTS], at[DYMOE_MAX_EXPERTS], tile0[DYMOE_MAX_EXPERTS], wave[3][kI8PlanThreads / kWave];
    uint16_t owner[kI8PlanTiles], perm[kI8PlanPairs];
};

__device__ __forceinline__ void i8_make_plan(I8PlanLds& lds, const int32_t* __restrict__ idx, const dymoe_expert_i8* __restrict__ table, long P, int E,
                                             int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const I8Plan pp = i8_plan(plan, P);
    int e_of[kI8PlanKeep], turn[kI8PlanKeep];
#pragma unroll
    for (int i = 0; i < kI8PlanKeep; i++) {
        const long p = tid + (long)i * kI8PlanThreads;
        e_of[i] = p < P ? idx[p] : -1;
    }
    const bool held = tid < E && i8_present(table[tid]);
    lds.count[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kI8PlanKeep; i++)
        if ((unsigned)e_of[i] < (unsigned)E) turn[i] = atomicAdd(&lds.count[e_of[i]], 1);
    for (long p = tid + (long)kI8PlanPairs; p < P; p += kI8PlanThreads) {
        const int e = idx[p];
        if ((unsigned)e < (unsigned)E) pp.where[p] = atomicAdd(&lds.count[e], 1);
    }
    __syncthreads();
    int n = lds.count[tid];
    if (n > 0 && !held) {
        atomicOr(flags, DYMOE_FLAG_FORMAT_MISSING);
        n = 0;
    }
    const bool one = !small && n <= kI8TileWide;             // a wide tile
    const int rows = small ? kI8TileSmall : one ? kI8TileWide : kI8TileRows, m = (n + rows - 1) / rows;
    const int n_in = wave_scan_dpp_i32(n), m2_in = wave_scan_dpp_i32(one ? 0 : m), m1_in = wave_scan_dpp_i32(one ? m : 0);
    if (lane == kWave - 1) {
        lds.wave[0][wave] = n_in;
        lds.wave[1][wave] = m2_in;
        lds.wave[2][wave] = m1_in;
    }
    __syncthreads();
    int n0 = n_in - n, t2 = m2_in, t1 = m1_in, all2 = 0, all1 = 0;
    for (int w = 0; w < kI8PlanThreads / kWave; w++) {
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
    auto record = [&](I8TileRec* to, int e, int first, int pairs, int tile0, int tiles) {
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
        if (t0 + i < kI8PlanTiles) lds.owner[t0 + i] = (uint16_t)tid;
        else record(&pp.tiles[t0 + i], tid, n0, n, t0, m);
    }
    if (tid == 0) {
        pp.meta[0] = all2;
        pp.meta[1] = all1;
    }
    __syncthreads();
    for (int i = tid; i < min(all1 + all2, kI8PlanTiles); i += kI8PlanThreads) {
        const int e = lds.owner[i], c = lds.count[e];
        const int per = small ? kI8TileSmall : c <= kI8TileWide ? kI8TileWide : kI8TileRows;
        record(&pp.tiles[i], e, lds.at[e], c, lds.tile0[e], (c + per - 1) / per);
    }
    const bool fits = P <= kI8PlanPairs;
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
    for (int i = 0; i < kI8PlanKeep; i++) {
        const long p = tid + (long)i * kI8PlanThreads;
        if (p < P) place(p, e_of[i], turn[i]);
    }
    for (long p = tid + (long)kI8PlanPairs; p < P; p += kI8PlanThreads) place(p, idx[p], pp.where[p]);
    if (!fits) return;
    __syncthreads();
    int sorted = 0;
    for (int w = 0; w < kI8PlanThreads / kWave; w++) sorted += lds.wave[0][w];
    for (int i = tid; i < sorted; i += kI8PlanThreads) pp.perm[i] = lds.perm[i];
}

// The plan by the first workgroup, the codes of the activations by the others, four rows each: neither needs the other, and a launch of its
// own would cost either as much as its work.  CH: 16 bytes a thread times CH hold a row.
template <int DT, int CH>
__global__ __launch_bounds__(kI8PlanThreads) void i8_prep_kernel(const int32_t* __restrict__ idx, const dymoe_expert_i8* __restrict__ table, long P,
                                                                 int E, int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags,
                                                                 const char* __restrict__ x, int T, int K, char* __restrict__ codes,
                                                                 float* __restrict__ scale)
{
    __shared__ I8PlanLds lds;
    if (blockIdx.x == 0) {
        i8_make_plan(lds, idx, table, P, E, small, plan, flags);
        return;
    }
    constexpr int kThreads = kI8PlanThreads / 4;                 // to a row
    const int t = threadIdx.x % kThreads, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const long row = (long)(blockIdx.x - 1) * 4 + threadIdx.x / kThreads;
    const int Kp = (int)up_to(K, 128);
    const char* const src = x + row * K * dtype_bytes(DT);
    Raw8<DT> v[CH];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; c++) v[c] = load8<DT>(src, (c * kThreads + t) * 8, row < T ? K : 0);
#pragma unroll
    for (int c = 0; c < CH; c++) m = peak8<DT>(v[c], m);
    m = wave_max_u32(peak_bits<DT>(m));
    if (lane == 0) lds.count[wave] = (int)m;
    __syncthreads();
    if (row >= T) return;
    const int w0 = wave & ~3;
    m = max(max((uint32_t)lds.count[w0], (uint32_t)lds.count[w0 + 1]), max((uint32_t)lds.count[w0 + 2], (uint32_t)lds.count[w0 + 3]));
    float sc;
    const RowQ q = row_q(peak_value<DT>(m), sc);
    if (t == 0) scale[row] = sc;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int col = (c * kThreads + t) * 8;
        if (col < Kp) store_global(codes + row * Kp + col, codes8<DT>(v[c], q));
    }
}

template <int DT>
static void i8_prep_launch(dymoe_ctx* ctx, const int32_t* idx, const dymoe_expert_i8* table, long P, int E, int small, int32_t* plan, const void* x,
                           int T, int K, void* codes, float* scale, hipStream_t st)
{
    const dim3 grid((unsigned)(1 + (T + 3L) / 4)), block(kI8PlanThreads);
    auto kernel = K <= 4096 ? i8_prep_kernel<DT, 2> : i8_prep_kernel<DT, 8>;
    dymoe_launch(ctx, DYMOE_K_INT8_PLAN, kernel, grid, block, 0, st, idx, table, P, E, small, plan, ctx->device_flags, (const char*)x, T, K,
                 (char*)codes, scale);
}

// (a row of more than 16384 values: its codes by a launch of their own, this one for the plan)
__global__ __launch_bounds__(kI8PlanThreads) void i8_plan_kernel(const int32_t* __restrict__ idx, const dymoe_expert_i8* __restrict__ table, long P,
                                                                 int E, int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags)
{
    __shared__ I8PlanLds lds;
    i8_make_plan(lds, idx, table, P, E, small, plan, flags);
}

// One weight matrix as a launch reads it: codes in tiles, scales.
struct I8Mat {
    const char* q;
    const float* s;
};

struct I8Args {
    const char* x;                    // codes of the rows, Kp columns each
    const float* xs;
    const int32_t* plan;              // grouped products
    I8Mat w;                          // the plain product
    const float* bias;
    void* out;
    long ldo, P;
    int rows, Kp, N, k, out_dtype, aligned, tiled;     // aligned: the plain product's rows start where four outputs may be stored at once
};

// Memory that a wavefront's loads share a base in: the base in scalar registers, a lane's offset and the load's own in 32 bits each.
struct I8Src {
    __amdgpu_buffer_rsrc_t r;

    __device__ __forceinline__ void set(const void* p, uint32_t bytes)
    {
        const uint64_t u = (uint64_t)p;
        const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)u), hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32));
        r = __builtin_amdgcn_make_buffer_rsrc((void*)(((uint64_t)hi << 32) | lo), 0, (int)bytes, 0x00020000);
    }
    // NT: streamed through once
    template <bool NT = false>
    __device__ __forceinline__ uint4 load(uint32_t lane, uint32_t all) const
    {
        return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)lane, (int)all, NT ? 2 : 0));
    }
};

enum { kI8Plain = 0, kI8Up = 1, kI8Down = 2 };

__device__ __forceinline__ i32x16_t mfma_i8(const uint4 a, const uint4 b, const i32x16_t c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
}

// An output of a product: the sum's conversion, its product with the row's scale and the multiply-add round once each, in every shape alike,
// whatever the compiler would contract.
__device__ __forceinline__ float i8_value(int sum, float xs, float sc, float add) { return fmaf((float)sum * xs, sc, add); }

// a u / (1 + e^-a).  The instruction for powers of two takes t = -a log2 e, a product that rounds by up to 2^-24 of itself; at |a| = 80 that
// alone moves the power by 2^-18.  What it leaves out, -a - t ln 2, is an exact difference and goes to the result as the factor 1 + that.
// In steps of 2^-24: exp 2, the factor 1.5, 1 + e^-a 1, the reciprocal 2, the products 1 each: 8.5 at most.  (Beyond 128 e^-a is 0
// or infinite, and log2 e times a could leave the range; from -87.3 down the reciprocal is below the normal numbers, and the result 0.
// 512 tokens on eight experts of 14336 351 us, as with the rounded t alone.)
__device__ __forceinline__ float silu_times(float a, float u)
{
    constexpr float kLn2 = 0x1.62e43p-1f, kRest = -0x1.05c61p-29f;          // their sum: ln 2 to 2^-54
    const float x = __builtin_amdgcn_fmed3f(a, -128.0f, 128.0f), t = x * -1.44269504f;
    const float p = 1.0f + fmaf(t, -kRest, fmaf(t, -kLn2, -x));
    return a * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), p, 1.0f)) * u;
}

// ----------------------------------------------------------------------------
// A few rows (decode): a stream of weights.  A workgroup owns 16 weight rows (of W1 and of W3 in the up projection), its wavefronts take the
// 128-column tiles of K in turn and meet in LDS; every wavefront requests its first kI8Ahead tiles before anything else, so that the
// rows' quantisation, which every workgroup then does for itself where the rows are few, costs no launch and hides behind them.
// v_mfma_i32_16x16x64_i8: lane l holds weight row l % 16 and row l % 16 of the codes, columns 64 (l / 32) + 32 j + 16 (l / 16 % 2) of a
// tile in its j-th product (any order of columns will do that is the same on both sides).
// Bound by the weights' bytes: one token on two experts of 14336 x 4096, up 39.1 us (6.0 TB/s) and down 24.1 us (4.9 TB/s); a matrix of
// 128256 x 4096 and one token 83 us (6.3 TB/s).
constexpr int kI8Ahead = 4;
constexpr int kI8ThinWaves = 8;
__device__ __forceinline__ i32x4_t mfma16_i8(const uint4 a, const uint4 b, const i32x4_t c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
}

template <int S>
struct I8Thin {
    uint4 w[kI8Ahead][S][2];
    I8Src q[S];                // the strips
    uint32_t off;              // this lane's 16 bytes of the first product, in the sixteen rows' half of the strip
    int kt, nkt, by;           // next tile to multiply, tiles, distance of this wavefront's tiles

    __device__ __forceinline__ void load(int d, int tile)
    {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int j = 0; j < 2; j++) w[d][s][j] = q[s].template load<true>(off + (uint32_t)(j * 2048), (uint32_t)tile * 4096u);
    }
    __device__ __forceinline__ void start(int first, int tiles, int stride, int half, int lane)
    {
        kt = first;
        nkt = tiles;
        by = stride;
        off = (uint32_t)((lane >> 4 & 1) * 1024 + (lane >> 5) * 512 + half * 256 + (lane & 15) * 16);
#pragma unroll
        for (int d = 0; d < kI8Ahead; d++)
            if (kt + d * by < nkt) load(d, kt + d * by);
    }
    // row(col): 16 codes of this lane's row from column col on
    template <class Row>
    __device__ __forceinline__ void run(i32x4_t (&acc)[S], int lane, Row row)
    {
        const int col = 64 * (lane >> 5) + 16 * (lane >> 4 & 1);
        while (kt < nkt) {
#pragma unroll
            for (int d = 0; d < kI8Ahead; d++) {
                if (kt < nkt) {
                    const uint4 b0 = row(kt * 128 + col), b1 = row(kt * 128 + col + 32);
#pragma unroll
                    for (int s = 0; s < S; s++) {
                        acc[s] = mfma16_i8(w[d][s][0], b0, acc[s]);
                        acc[s] = mfma16_i8(w[d][s][1], b1, acc[s]);
                    }
                    if (kt + kI8Ahead * by < nkt) load(d, kt + kI8Ahead * by);
                }
                kt += by;
            }
        }
    }
};

// The codes of `rows` rows into LDS (Kp + 16 bytes apart) and their scales, by a whole workgroup.
template <int DT>
__device__ __forceinline__ void i8_rows_to_lds(const char* x, long pitch, int rows, int K, int Kp, char* s_codes, float* s_scale, uint32_t* s_max)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, n = blockDim.x, waves = n / kWave;
    if (3 * rows >= waves || K <= 1024) {           // a wavefront a row: nothing to hand over
        for (int r = wave; r < rows; r += waves) {
            uint32_t m = 0;
#pragma unroll 2
            for (int col = lane * 8; col < K; col += kWave * 8) m = peak8<DT>(load8<DT>(x + r * pitch, col, K), m);
            float sc;
            const RowQ q = row_q(peak_value<DT>(wave_max_u32(peak_bits<DT>(m))), sc);
            if (lane == 0) s_scale[r] = sc;
#pragma unroll 2
            for (int col = lane * 8; col < Kp; col += kWave * 8)
                *(uint2*)(s_codes + (long)r * (Kp + 16) + col) = codes8<DT>(load8<DT>(x + r * pitch, col, K), q);
        }
        __syncthreads();
        return;
    }
    for (int r = 0; r < rows; r++) {
        uint32_t m = 0;
        for (int col = tid * 8; col < K; col += n * 8) m = peak8<DT>(load8<DT>(x + r * pitch, col, K), m);
        m = wave_max_u32(peak_bits<DT>(m));
        if (lane == 0) s_max[r * waves + wave] = m;
    }
    __syncthreads();
    for (int r = 0; r < rows; r++) {
        uint32_t m = 0;
        for (int w = 0; w < waves; w++) m = max(m, s_max[r * waves + w]);
        float sc;
        const RowQ q = row_q(peak_value<DT>(m), sc);
        if (tid == 0) s_scale[r] = sc;
        for (int col = tid * 8; col < Kp; col += n * 8)
            *(uint2*)(s_codes + (long)r * (Kp + 16) + col) = codes8<DT>(load8<DT>(x + r * pitch, col, K), q);
    }
    __syncthreads();
}

__device__ __forceinline__ void i8_rows_to_lds(int dt, const char* x, long pitch, int rows, int K, int Kp, char* s_codes, float* s_scale, uint32_t* s_max)
{
    if (dt == DYMOE_OUT_F32) i8_rows_to_lds<DYMOE_OUT_F32>(x, pitch, rows, K, Kp, s_codes, s_scale, s_max);
    else if (dt == DYMOE_OUT_F16) i8_rows_to_lds<DYMOE_OUT_F16>(x, pitch, rows, K, Kp, s_codes, s_scale, s_max);
    else i8_rows_to_lds<DYMOE_OUT_BF16>(x, pitch, rows, K, Kp, s_codes, s_scale, s_max);
}

struct I8ThinArgs {
    const char* x;            // FUSE: the rows themselves, else their codes
    const float* xs;
    const int32_t* idx;       // experts: [P]
    const float* gate;
    const dymoe_expert_i8* table;
    unsigned* flags;
    I8Mat w;
    const float* bias;
    void* out;
    long ldx, ldo;            // ldx: bytes from row to row
    int x_dtype, rows, K, Kp, N, E, k, P, out_dtype;
};

// The plain product of up to 16 rows, and the up projection of up to 64 pairs: the workgroup of a pair that comes first among those of its
// expert (or 16, 32, ... behind the first) takes the next sixteen of them.
template <int MODE, bool FUSE>
__global__ __launch_bounds__(64 * kI8ThinWaves, 4) void i8_thin_kernel(const I8ThinArgs A)
{
    constexpr int S = MODE == kI8Up ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) char s_codes[];
    __shared__ int s_sum[kI8ThinWaves][S][4][kWave];
    __shared__ float s_scale[kI8ThinRows];
    __shared__ uint32_t s_max[kI8ThinRows * kI8ThinWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 15;
    const int nblk = (A.N + 15) / 16;
    const int pair = blockIdx.x / nblk, bx = blockIdx.x - pair * nblk;
    int rows = A.rows, mine = min(ln, A.rows - 1);          // this lane's row: a token of the plain product, a pair of the experts
    const float *sa, *sb;
    I8Thin<S> thin;
    const long strip = (long)(bx >> 1) * 32 * A.Kp;
    const uint32_t bytes = 32u * (uint32_t)A.Kp;
    if (MODE == kI8Plain) {
        thin.q[0].set(A.w.q + strip, bytes);
        sa = sb = A.w.s;
    } else {
        const int my_e = lane < A.P ? A.idx[lane] : -1;
        const int e = __builtin_amdgcn_readlane(my_e, pair);
        if ((unsigned)e >= (unsigned)A.E) return;
        const uint64_t all = __ballot(my_e == e);
        const int rank = __popcll(all & ((1ull << pair) - 1));
        if (rank & (kI8ThinRows - 1)) return;
        const dymoe_expert_i8 ex = A.table[e];
        if (!i8_present(ex)) {
            if (tid == 0) atomicOr(A.flags, DYMOE_FLAG_FORMAT_MISSING);
            return;
        }
        rows = min(kI8ThinRows, __popcll(all) - rank);
        uint64_t left = all >> pair << pair;                 // this tile's pairs and those behind it
        const int want = min(ln, rows - 1);
        for (int i = 0; i < want; i++) left &= left - 1;
        mine = __builtin_ctzll(left);
        thin.q[0].set((const char*)ex.q[0] + strip, bytes);
        thin.q[S - 1].set((const char*)ex.q[S - 1] + strip, bytes);
        sa = ex.s[0];
        sb = ex.s[1];
    }
    const int nkt = A.Kp >> 7;
    thin.start(wave, nkt, kI8ThinWaves, bx & 1, lane);
    const int token = MODE == kI8Up ? mine / A.k : mine;
    i32x4_t acc[S] = {};
    if constexpr (FUSE) {
        i8_rows_to_lds(A.x_dtype, A.x, A.ldx, MODE == kI8Up ? A.P / A.k : A.rows, A.K, A.Kp, s_codes, s_scale, s_max);
        const char* const row = s_codes + token * (A.Kp + 16);
        thin.run(acc, lane, [&](int col) { return *(const uint4*)(row + col); });
    } else {
        const char* const row = A.x + (long)token * A.ldx;
        thin.run(acc, lane, [&](int col) { return load_global<uint4>(row + col); });
    }
#pragma unroll
    for (int s = 0; s < S; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) s_sum[wave][s][i][lane] = acc[s][i];
    __syncthreads();
    // wavefronts 0 .. 3 finish weight rows 4 (l / 16) + wave of row l % 16
    if (wave >= 4 || ln >= rows) return;
    int sum[S];
#pragma unroll
    for (int s = 0; s < S; s++) {
        sum[s] = 0;
#pragma unroll
        for (int w = 0; w < kI8ThinWaves; w++) sum[s] += s_sum[w][s][wave][lane];
    }
    const int n = 16 * bx + 4 * (lane >> 4) + wave;
    if (n >= A.N) return;
    const float xs = FUSE ? s_scale[token] : A.xs[token];
    if (MODE == kI8Up) {
        ((DYMOE_GLOBAL float*)A.out)[mine * A.ldo + n] = silu_times(i8_value(sum[0], xs, sa[n], 0.0f), i8_value(sum[S - 1], xs, sb[n], 0.0f));
    } else {
        store_out(A.out, mine * A.ldo + n, A.out_dtype, i8_value(sum[0], xs, sa[n], A.bias ? A.bias[n] : 0.0f));
    }
}

// The down projection of up to kI8FuseRows tokens with the sum over their slots: a workgroup owns 16 outputs of one token; its wavefronts
// share out the token's pairs, or a pair's tiles where there are fewer pairs than wavefronts.  Every workgroup quantises the
// intermediate's rows itself.
constexpr int kI8LastWaves = 16;

__global__ __launch_bounds__(64 * kI8LastWaves) void i8_thin_down_kernel(const I8ThinArgs A)
{
    extern __shared__ __attribute__((aligned(16))) char s_codes[];
    __shared__ int s_sum[64][16];
    __shared__ float s_scale[64];
    __shared__ uint32_t s_max[64 * kI8LastWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    // the workgroups of one strip go to one XCD, whose L2 then has the weights that several tokens need
    const int nblk = (A.N + 15) / 16, j = blockIdx.x >> 3;
    const int t = j % A.rows, bx = j / A.rows * 8 + (blockIdx.x & 7);
    if (bx >= nblk) return;
    const int k = A.k, seg = max(1, kI8LastWaves / k), units = k * seg;
    const long strip = (long)(bx >> 1) * 32 * A.Kp;
    const uint32_t bytes = 32u * (uint32_t)A.Kp;
    const int nkt = A.Kp >> 7;
    I8Thin<1> thin;
    bool ok = false;
    auto begin = [&](int u) {
        const int e = __builtin_amdgcn_readfirstlane(A.idx[t * k + u / seg]);
        ok = (unsigned)e < (unsigned)A.E;
        if (ok) {
            const dymoe_expert_i8 ex = A.table[e];
            ok = i8_present(ex);
            thin.q[0].set((const char*)ex.q[2] + strip, bytes);
        }
        if (ok) thin.start(u % seg, nkt, seg, bx & 1, lane);
    };
    if (wave < units) begin(wave);
    i8_rows_to_lds<DYMOE_OUT_F32>(A.x + (long)t * k * A.ldx, A.ldx, k, A.K, A.Kp, s_codes, s_scale, s_max);
    for (int u = wave; u < units; u += kI8LastWaves) {
        if (u != wave) begin(u);
        i32x4_t acc[1] = {};
        if (ok) {
            const char* const row = s_codes + (long)(u / seg) * (A.Kp + 16);
            thin.run(acc, lane, [&](int col) { return *(const uint4*)(row + col); });
        }
        if ((lane & 15) == 0) {
#pragma unroll
            for (int i = 0; i < 4; i++) s_sum[u][4 * (lane >> 4) + i] = acc[0][i];
        }
    }
    __syncthreads();
    const int n = 16 * bx + tid;
    if (tid >= 16 || n >= A.N) return;
    float y = 0.0f;
    for (int i = 0; i < k; i++) {
        const int e = A.idx[t * k + i];
        if ((unsigned)e >= (unsigned)A.E || !i8_present(A.table[e])) continue;
        int sum = 0;
        for (int s = 0; s < seg; s++) sum += s_sum[i * seg + s][tid];
        y = fmaf(A.gate[t * k + i], (float)sum * s_scale[i] * A.table[e].s[2][n], y);
    }
    store_out(A.out, t * A.ldo + n, A.out_dtype, y);
}

// ----------------------------------------------------------------------------
// Tiles of up to 128 rows.  A workgroup of four wavefronts owns S strips of 32 weight rows a wavefront and walks K in steps of KT tiles of 128
// columns.
//  * Weights come straight into registers: a tile's bytes lie in the order of the matrix instruction's operand, so a wavefront's load is 1 KiB
//    of contiguous memory.  A register is requested anew, for the next step, as soon as the last instruction that reads it has been issued.
//  * The rows' codes are shared by the wavefronts through two LDS buffers that global memory fills directly; the 16-byte chunks
//    of a row are turned by its number, which spreads the operand reads (one chunk of 32 rows) over all banks.
//  * Several workgroups on a compute unit, one's waits, prologue and epilogue covered by the others' products.
// Two shapes: S = 2, KT = 2 (128 accumulator registers a lane, two workgroups a compute unit) reads half as much LDS for a product; S = 1,
// KT = 1 (64, four workgroups) has more loads on their way and twice as many workgroups, for calls that the weights' bytes bound.
// 2048 x 14336 x 4096: 126 us, 1.91 POP/s, with random codes.  On a card where it took 131: 102 us on zeros, since the clock follows the power
// (products from registers alone reach 4.4 POP/s on quiet data and 3.4 on random), 129 without its copies of rows, 113 without its loads
// of weights, 104 to 108 with neither: the products and their LDS reads are what is left.
template <int S>
constexpr uint32_t kI8EpiRow = S == 2 ? 272 : 144;     // epilogue: bytes of a row of 32 S sums in LDS, 16 of them padding
template <int S>
constexpr uint32_t kI8EpiWave = 32 * kI8EpiRow<S>;

template <int S, int KT>
struct I8Strips {
    uint4 r[S][4 * KT];       // chunk j = 4 * (tile of the step) + 16-byte chunk of the lane's half of that tile
};

// chunk c of a tile of a strip
__device__ __forceinline__ uint4 i8_chunk(const I8Src& q, uint32_t lane16, int tile, int c)
{
    return q.load(lane16 + (uint32_t)(c * 1024), (uint32_t)tile * 4096u);
}

template <int NTF, int KT>
struct I8Stage {
    static constexpr int kCopies = NTF * KT;    // an instruction of the workgroup fills 4 KiB
    const char* base;
    uint32_t off[kCopies];
    uint32_t lds;
};

struct I8Ops {
    uint4 t0, t1;
};

// What a row's chunks are turned by in LDS: sixteen rows' chunks of one number then lie on 64 different banks.
template <int KT>
__device__ __forceinline__ int i8_turn(int row)
{
    return KT == 2 ? row & 15 : (row >> 1) & 7;      // (rows of 128 bytes: the row's parity is half of the banks already)
}

// The first TILES tiles of a step.  The operands of the next pair of chunks are read while the products of this one are issued.
template <int NTF, int S, int KT, int TILES>
__device__ __forceinline__ void i8_step(I8Strips<S, KT>& w, const I8Src (&q)[S], uint32_t lane16, int tile_next, int nkt, uint32_t xa,
                                        i32x16_t (&acc)[S][NTF])
{
    constexpr int kStepMask = 0x2 | 0x4;        // vector and scalar arithmetic may cross; products, LDS and memory accesses may not
    constexpr int kPairs = 2 * TILES;
    I8Ops ops;
    ops.t0 = lds_read16(xa);
    ops.t1 = lds_read16(xa ^ 16u);
#pragma unroll
    for (int jj = 0; jj < kPairs; jj++) {
#pragma unroll
        for (int tf = 0; tf < NTF; tf++) {
            const bool wrap = tf == NTF - 1;
            const bool last = wrap && jj == kPairs - 1;
            const int nj = wrap ? jj + 1 : jj, nf = wrap ? 0 : tf + 1;
            I8Ops nxt = ops;
            if (!last) {
                // chunks 2 nj, 2 nj + 1 of the lane's columns: position 8 * tile + 4 * half + chunk, the half already in xa
                const uint32_t at = (xa ^ (uint32_t)(((nj >> 1) << 7) | ((nj & 1) << 5))) + (uint32_t)nf * (32 * 128 * KT);
                nxt.t0 = lds_read16(at);
                nxt.t1 = lds_read16(at ^ 16u);
            }
            __builtin_amdgcn_sched_barrier(kStepMask);
#pragma unroll
            for (int s = 0; s < S; s++) acc[s][tf] = mfma_i8(w.r[s][2 * jj], ops.t0, acc[s][tf]);
#pragma unroll
            for (int s = 0; s < S; s++) acc[s][tf] = mfma_i8(w.r[s][2 * jj + 1], ops.t1, acc[s][tf]);
            ops = nxt;
            __builtin_amdgcn_sched_barrier(kStepMask);
        }
        const int tile = min(tile_next + (jj >> 1), nkt - 1), c = 2 * (jj & 1);
#pragma unroll
        for (int s = 0; s < S; s++) {
            w.r[s][2 * jj] = i8_chunk(q[s], lane16, tile, c);
            w.r[s][2 * jj + 1] = i8_chunk(q[s], lane16, tile, c + 1);
        }
        __builtin_amdgcn_sched_barrier(kStepMask);
    }
}

// four neighbouring outputs of a row
__device__ __forceinline__ void i8_store4(void* out, long at, int dt, bool whole, int left, const float (&v)[4])
{
    if (whole) {
        if (dt == DYMOE_OUT_F32) {
            store_global((float*)out + at, make_float4(v[0], v[1], v[2], v[3]));
        } else if (dt == DYMOE_OUT_F16) {
            store_global((uint16_t*)out + at, make_uint2(pack_half2(v[0], v[1]), pack_half2(v[2], v[3])));
        } else {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            const bf16x4_t b = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            store_global((uint16_t*)out + at, __builtin_bit_cast(uint2, b));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (i < left) store_out(out, at + i, dt, v[i]);
}

// Epilogue.  A lane holds, of its token's row, four neighbouring outputs in each group of four registers; the wavefront turns a fragment
// round in an LDS area of its own, so that a row leaves in whole lines.
template <int MODE, int NTF, int S>
__device__ __forceinline__ void i8_finish(const I8Args& A, const int32_t* perm, const i32x16_t (&acc)[S][NTF], const float* sa, const float* sb,
                                          int row0, int rows, int bx, uint32_t xs_base)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const uint32_t area = xs_base + (uint32_t)wave * kI8EpiWave<S>;
    const uint32_t wr = area + (uint32_t)ln * kI8EpiRow<S> + (uint32_t)kb * 16u;
    const bool vec = MODE != kI8Plain || A.aligned;
    const int dt = MODE == kI8Plain ? A.out_dtype : DYMOE_OUT_F32;
    if constexpr (MODE == kI8Up && S == 2) {
        const int n = (4 * bx + wave) * 32 + 4 * (lane & 7), left = A.N - n;
#pragma unroll
        for (int tf = 0; tf < NTF; tf++) {
            const int r = min(32 * tf + ln, rows - 1);
            const float xs = A.xs[perm[row0 + r] / A.k];
#pragma unroll
            for (int g = 0; g < 4; g++) {
                float h[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int f = min((4 * bx + wave) * 32 + 8 * g + 4 * kb + i, A.N - 1);
                    h[i] = silu_times(i8_value(acc[0][tf][4 * g + i], xs, sa[f], 0.0f), i8_value(acc[S - 1][tf][4 * g + i], xs, sb[f], 0.0f));
                }
                lds_write16(wr + 32u * g, make_uint4(__float_as_uint(h[0]), __float_as_uint(h[1]), __float_as_uint(h[2]), __float_as_uint(h[3])));
            }
            // (a wavefront's LDS accesses execute in order and the area is its own: no barrier)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int rr = (lane >> 3) + 8 * j, row = 32 * tf + rr;
                const uint4 u = lds_read16(area + (uint32_t)rr * kI8EpiRow<S> + (uint32_t)(lane & 7) * 16u);
                if (row >= rows || left <= 0) continue;
                const float v[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
                i8_store4(A.out, (long)(row0 + row) * A.ldo + n, dt, left >= 4, left, v);
            }
        }
        return;
    }
    constexpr int kOut = 8 * S;                 // lanes to a row of the wavefront's 32 S sums
    auto put = [&](int tf) {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int g = 0; g < 4; g++)
                lds_write16(wr + (uint32_t)(s * 128 + g * 32), make_uint4((uint32_t)acc[s][tf][4 * g], (uint32_t)acc[s][tf][4 * g + 1],
                                                                          (uint32_t)acc[s][tf][4 * g + 2], (uint32_t)acc[s][tf][4 * g + 3]));
    };
    if constexpr (MODE == kI8Up) {
        // one strip a wavefront: wavefronts 0, 1 have W1's sums of 64 features, 2, 3 have W3's of the same
        const int f = 4 * (lane & 15), n = 64 * bx + f, left = A.N - n;
        float c1[4], c3[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            c1[i] = sa[min(n + i, A.N - 1)];
            c3[i] = sb[min(n + i, A.N - 1)];
        }
#pragma unroll
        for (int tf = 0; tf < NTF; tf++) {
            put(tf);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const int rr = 8 * wave + 4 * j + (lane >> 4), row = 32 * tf + rr;
                const uint32_t from = xs_base + (uint32_t)(f >> 5) * kI8EpiWave<S> + (uint32_t)rr * kI8EpiRow<S> + (uint32_t)(f & 31) * 4u;
                const uint4 a = lds_read16(from), u = lds_read16(from + 2 * kI8EpiWave<S>);
                if (row >= rows || left <= 0) continue;
                const float xs = A.xs[perm[row0 + row] / A.k];
                const uint32_t av[4] = {a.x, a.y, a.z, a.w}, uv[4] = {u.x, u.y, u.z, u.w};
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = silu_times(i8_value((int)av[i], xs, c1[i], 0.0f), i8_value((int)uv[i], xs, c3[i], 0.0f));
                i8_store4(A.out, (long)(row0 + row) * A.ldo + n, dt, left >= 4, left, v);
            }
            __syncthreads();
        }
    } else {
        const int n = (4 * bx + wave) * 32 * S + 4 * (lane & (kOut - 1)), left = A.N - n;
        float sc[4], add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            sc[i] = sa[min(n + i, A.N - 1)];
            if (MODE == kI8Plain && A.bias) add[i] = A.bias[min(n + i, A.N - 1)];
        }
#pragma unroll
        for (int tf = 0; tf < NTF; tf++) {
            put(tf);
            // (a wavefront's LDS accesses execute in order and the area is its own: no barrier)
#pragma unroll
            for (int j = 0; j < 32 * kOut / 64; j++) {
                const int rr = lane / kOut + 64 / kOut * j, row = 32 * tf + rr;
                const uint4 u = lds_read16(area + (uint32_t)rr * kI8EpiRow<S> + (uint32_t)(lane & (kOut - 1)) * 16u);
                if (row >= rows || left <= 0) continue;
                const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
                float v[4];
                const float xs = A.xs[row0 + row];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = i8_value((int)w4[i], xs, sc[i], add[i]);
                i8_store4(A.out, (long)(row0 + row) * A.ldo + n, dt, left >= 4 && vec, left, v);
            }
        }
    }
}

// qw: this wavefront's strips; sa, sb: the scales of the matrices
template <int MODE, int NTF, int S, int KT>
__device__ __forceinline__ void i8_tile(const I8Args& A, const int32_t* perm, const I8Src (&qw)[S], const float* sa, const float* sb,
                                        int row0, int rows, int bx, uint32_t xs_base, uint32_t buf_bytes)
{
    constexpr int kLanes = 8 * KT;              // lanes (16-byte chunks) to a row of a step
    constexpr int kRowsWave = 64 / kLanes;      // rows that a wavefront's copy fills
    constexpr uint32_t kRow = 128 * KT;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const uint32_t lane16 = (uint32_t)lane * 16u;
    i32x16_t acc[S][NTF] = {};
    I8Stage<NTF, KT> stage;
    const int rb = kRowsWave * wave + lane / kLanes;                         // (a thread's rows are turned alike)
    const int chunk = (lane & (kLanes - 1)) ^ i8_turn<KT>(rb);
#pragma unroll
    for (int i = 0; i < I8Stage<NTF, KT>::kCopies; i++) {
        const int r = min(4 * kRowsWave * i + rb, rows - 1);                 // rows behind the last: computed and dropped
        const uint32_t src = MODE == kI8Up ? (uint32_t)(perm[row0 + r] / A.k) : (uint32_t)r;
        stage.off[i] = src * (uint32_t)A.Kp + 16u * (uint32_t)chunk;          // below 4 GiB: checked by the launcher
    }
    stage.base = A.x + (MODE == kI8Up ? 0 : (long)row0 * A.Kp);
    stage.lds = __builtin_amdgcn_readfirstlane(xs_base + (uint32_t)wave * 1024u);
    const int nkt = A.Kp >> 7, steps = (nkt + KT - 1) / KT;
    // (two tiles a step: the last step's second may lie behind the rows' end: its chunks are then those of the first, and go unused)
    const uint32_t back = KT == 2 && (nkt & 1) && (chunk & 8) ? 128u : 0u;
    auto copy = [&](int ks, uint32_t at) {
        const char* const base = stage.base + (long)ks * kRow;
        const uint32_t less = ks == steps - 1 ? back : 0u;
#pragma unroll
        for (int i = 0; i < I8Stage<NTF, KT>::kCopies; i++) lds_copy16(base, stage.off[i] - less, stage.lds + at + (uint32_t)i * 4096u);
    };
    const uint32_t xa0 = xs_base + (uint32_t)ln * kRow + (((uint32_t)kb << 6) ^ ((uint32_t)i8_turn<KT>(ln) << 4));
    I8Strips<S, KT> w;
    copy(0, 0);
#pragma unroll
    for (int j = 0; j < 4 * KT; j++)
#pragma unroll
        for (int s = 0; s < S; s++) w.r[s][j] = i8_chunk(qw[s], lane16, min(j >> 2, nkt - 1), j & 3);
    wait_lds_copies<0>();
    __syncthreads();
    uint32_t at = 0;
    for (int ks = 0; ks < nkt / KT; ks++) {
        copy(min(ks + 1, steps - 1), at ^ buf_bytes);
        i8_step<NTF, S, KT, KT>(w, qw, lane16, KT * (ks + 1), nkt, xa0 + at, acc);
        wait_lds_copies<4 * S * KT>();          // the copies are older than the loads of weights
        __syncthreads();
        at ^= buf_bytes;
    }
    if constexpr (KT == 2) {
        if (nkt & 1) {
            i8_step<NTF, S, KT, 1>(w, qw, lane16, nkt - 1, nkt, xa0 + at, acc);
            __syncthreads();
        }
    }

    i8_finish<MODE, NTF, S>(A, perm, acc, sa, sb, row0, rows, bx, xs_base);
}

// Tiles of up to 160 rows for calls that the weights' bytes bound (experts that meet a few dozen tokens to some hundred): one strip a
// wavefront, four tiles of weights on their way in registers, the rows' codes through registers into two LDS buffers.  Bytes on
// their way are what sets the rate of such a stream; with the rows copied to LDS directly, as above, the loads of weights could run
// ahead by one step only, because a count of outstanding loads that lets the copies through has to wait for all loads before them.
// Eight experts of 14336 x 4096, 64 to 160 pairs each: up 218 us (4.3 TB/s of weights).  On a card where it took 230: 217 without its products, 208
// without its rows, 238 with non-temporal loads of the weights.
constexpr int kI8Deep = 4;

template <int MODE, int NTF>
__device__ __forceinline__ void i8_wide_tile(const I8Args& A, const int32_t* perm, const I8Src& qw, const float* sa, const float* sb, int row0,
                                             int rows, int bx, uint32_t xs_base)
{
    constexpr uint32_t kBuf = 32u * NTF * 128u;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const uint32_t lane16 = (uint32_t)lane * 16u;
    i32x16_t acc[1][NTF] = {};
    const int rb = 8 * wave + (lane >> 3);
    const uint32_t chunk = (uint32_t)((lane & 7) ^ i8_turn<1>(rb)) * 16u;
    uint32_t off[NTF];
#pragma unroll
    for (int i = 0; i < NTF; i++) {
        const int r = min(32 * i + rb, rows - 1);                            // rows behind the last: computed and dropped
        off[i] = (MODE == kI8Up ? (uint32_t)(perm[row0 + r] / A.k) : (uint32_t)r) * (uint32_t)A.Kp + chunk;
    }
    I8Src base;
    base.set(A.x + (MODE == kI8Up ? 0 : (long)row0 * A.Kp), MODE == kI8Up ? (uint32_t)A.rows * (uint32_t)A.Kp : (uint32_t)rows * (uint32_t)A.Kp);
    const int nkt = A.Kp >> 7;
    uint4 w[kI8Deep][4], xr[2][NTF];
    auto load_w = [&](uint4 (&to)[4], int tile, int c) { to[c] = i8_chunk(qw, lane16, min(tile, nkt - 1), c); };
    auto load_x = [&](uint4 (&to)[NTF], int tile) {
#pragma unroll
        for (int i = 0; i < NTF; i++) to[i] = base.load(off[i], (uint32_t)min(tile, nkt - 1) * 128u);
    };
    auto put_x = [&](const uint4 (&from)[NTF], uint32_t buf) {
#pragma unroll
        for (int i = 0; i < NTF; i++) lds_write16(xs_base + buf + (uint32_t)(i * 4096 + wave * 1024) + lane16, from[i]);
    };
    load_x(xr[0], 0);
#pragma unroll
    for (int d = 0; d < kI8Deep; d++) {
#pragma unroll
        for (int c = 0; c < 4; c++) load_w(w[d], d, c);
    }
    load_x(xr[1], 1);
    put_x(xr[0], 0);
    load_x(xr[0], 2);
    __syncthreads();
    const uint32_t xa0 = xs_base + (uint32_t)ln * 128u + (((uint32_t)kb << 6) ^ ((uint32_t)i8_turn<1>(ln) << 4));
    constexpr int kMask = 0x2 | 0x4;             // vector and scalar arithmetic may cross; products, LDS and memory accesses may not
    auto step = [&](int k, auto slot) __attribute__((always_inline)) {
        constexpr int d = slot(), odd = d & 1;   // k % 4, k % 2
        put_x(xr[odd ^ 1], odd ? 0u : kBuf);
        load_x(xr[odd ^ 1], k + 3);
        __builtin_amdgcn_sched_barrier(kMask);
        const uint32_t xa = xa0 + (odd ? kBuf : 0u);
        I8Ops ops;
        ops.t0 = lds_read16(xa);
        ops.t1 = lds_read16(xa ^ 16u);
#pragma unroll
        for (int jj = 0; jj < 2; jj++) {
#pragma unroll
            for (int tf = 0; tf < NTF; tf++) {
                const bool wrap = tf == NTF - 1, last = wrap && jj == 1;
                I8Ops nxt = ops;
                if (!last) {
                    const uint32_t at = (xa ^ (uint32_t)((wrap ? jj + 1 : jj) << 5)) + (uint32_t)(wrap ? 0 : tf + 1) * 4096u;
                    nxt.t0 = lds_read16(at);
                    nxt.t1 = lds_read16(at ^ 16u);
                }
                __builtin_amdgcn_sched_barrier(kMask);
                acc[0][tf] = mfma_i8(w[d][2 * jj], ops.t0, acc[0][tf]);
                acc[0][tf] = mfma_i8(w[d][2 * jj + 1], ops.t1, acc[0][tf]);
                ops = nxt;
                __builtin_amdgcn_sched_barrier(kMask);
            }
            load_w(w[d], k + kI8Deep, 2 * jj);
            load_w(w[d], k + kI8Deep, 2 * jj + 1);
            __builtin_amdgcn_sched_barrier(kMask);
        }
        __syncthreads();
    };
    int k = 0;
    for (; k + 4 <= nkt; k += 4) {
        step(k, std::integral_constant<int, 0>());
        step(k + 1, std::integral_constant<int, 1>());
        step(k + 2, std::integral_constant<int, 2>());
        step(k + 3, std::integral_constant<int, 3>());
    }
    if (k < nkt) step(k, std::integral_constant<int, 0>());
    if (k + 1 < nkt) step(k + 1, std::integral_constant<int, 1>());
    if (k + 2 < nkt) step(k + 2, std::integral_constant<int, 2>());
    i8_finish<MODE, NTF, 1>(A, perm, acc, sa, sb, row0, rows, bx, xs_base);
}

// Neighbouring units that an XCD takes at a time.  Calls with 4, 8, 16, 32 and 64, one card: 2048 x 14336 x 4096 133, 133, 137, 138 and 139 us,
// 2048 x 4096 x 14336 151, 145, 149, 148 and 150, 2048 x 1536 x 2048 18.1, 18.2, 19.6, 19.2 and 30.5; the experts (2 of 8 of 14336 x 4096,
// 2048 tokens) 942, 930, 914, 916 and 976.
constexpr int kI8Run = 16, kI8RunPlain = 8;

// columns of a workgroup's block
template <int MODE, int S>
constexpr int kI8Cols = (MODE == kI8Up ? 64 : 128) * S;

template <int S>
struct I8Unit {
    I8Src qw[S];              // this wavefront's strips
    const float *sa, *sb;     // the matrices' scales
    int row0, rows, bx;
};

// Workgroups go to the 8 XCDs, each with an L2 of its own, in turn.  A unit is a tile and a column block; units that read the same weights
// (the tiles of a matrix or expert, for one column block) are neighbours, and an XCD takes runs of neighbours.
template <int RUN>
__device__ __forceinline__ long i8_run() { return (long)((blockIdx.x >> 3) / RUN) * 8 + (blockIdx.x & 7); }
template <int RUN>
__device__ __forceinline__ int i8_turn_in_run() { return (blockIdx.x >> 3) % RUN; }

// strip nt of a matrix; strips behind the last re-read it
__device__ __forceinline__ void i8_strip(I8Src& to, const I8Args& A, const void* q, long nt)
{
    const long strip = 32L * A.Kp;
    to.set((const char*)q + min(nt, (A.N + 31) / 32 - 1L) * strip, (uint32_t)strip);
}

template <int S>
__device__ __forceinline__ bool i8_plain_unit(const I8Args& A, I8Unit<S>& u, int wave)
{
    const int cols = kI8Cols<kI8Plain, S>, nblk = (A.N + cols - 1) / cols, tiles = (A.rows + kI8TileRows - 1) / kI8TileRows;
    const long unit = i8_run<kI8RunPlain>() * kI8RunPlain + i8_turn_in_run<kI8RunPlain>();
    if (unit >= (long)tiles * nblk) return false;
    u.bx = (int)(unit / tiles);
    u.row0 = (int)(unit - (long)u.bx * tiles) * kI8TileRows;
    u.rows = min(kI8TileRows, A.rows - u.row0);
#pragma unroll
    for (int s = 0; s < S; s++) i8_strip(u.qw[s], A, A.w.q, (4L * u.bx + wave) * S + s);
    u.sa = u.sb = A.w.s;
    return true;
}

// unit `unit` of the tiles from `first` on, tiles of ROWS rows
template <int MODE, int S, int ROWS>
__device__ __forceinline__ void i8_expert_unit(const I8Args& A, const I8Plan& pp, int first, long unit, I8Unit<S>& u)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int cols = kI8Cols<MODE, S>, nblk = (A.N + cols - 1) / cols;
    const I8TileRec t = pp.tiles[first + unit / nblk];
    const long local = unit - (long)(t.tile0 - first) * nblk;
    u.bx = (int)(local / t.tiles);
    const int i = (int)(local - (long)u.bx * t.tiles) * ROWS;
    u.row0 = t.first + i;
    u.rows = min(ROWS, t.pairs - i);
    const dymoe_expert_i8& ex = t.mat;
    if (MODE == kI8Up) {
        u.sa = ex.s[0];
        u.sb = ex.s[1];
        if constexpr (S == 2) {
            i8_strip(u.qw[0], A, ex.q[0], 4L * u.bx + wave);
            i8_strip(u.qw[S - 1], A, ex.q[1], 4L * u.bx + wave);
        } else {
            i8_strip(u.qw[0], A, wave < 2 ? ex.q[0] : ex.q[1], 2L * u.bx + (wave & 1));
        }
    } else {
#pragma unroll
        for (int s = 0; s < S; s++) i8_strip(u.qw[s], A, ex.q[2], (4L * u.bx + wave) * S + s);
        u.sa = u.sb = ex.s[2];
    }
}

__device__ __forceinline__ uint32_t lds_base(char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)p; }

template <int S, int KT>
__global__ __launch_bounds__(256, S == 2 ? 2 : 4) void i8_matmul_kernel(const I8Args A)
{
    extern __shared__ __attribute__((aligned(1024))) char xs_raw[];
    constexpr uint32_t kBuf = (uint32_t)kI8TileRows * 128 * KT;
    I8Unit<S> u;
    if (!i8_plain_unit<S>(A, u, __builtin_amdgcn_readfirstlane(threadIdx.x / kWave))) return;
#define DYMOE_I8_TILE(NTF) i8_tile<kI8Plain, NTF, S, KT>(A, nullptr, u.qw, u.sa, u.sb, u.row0, u.rows, u.bx, lds_base(xs_raw), kBuf)
    // one instantiation per number of fragments of 32 rows: the accumulators then sit in fixed registers for the whole loop
    switch ((u.rows + 31) >> 5) {
    case 1: DYMOE_I8_TILE(1); break;
    case 2: DYMOE_I8_TILE(2); break;
    case 3: DYMOE_I8_TILE(3); break;
    default: DYMOE_I8_TILE(4); break;
    }
#undef DYMOE_I8_TILE
}

// The plain product where its tiles are fewer than the chip takes: G groups of four wavefronts share a tile of 128 x 128 outputs and split K,
// each with LDS buffers of its own; at the end a fragment after the other meets in LDS and the groups finish eight of its rows each.  (Alone on
// a compute unit a step costs 0.8 us, the latency of its copies; 256 x 4096 outputs over 4096 columns took 32 of them, 26.8 us, and in four
// groups 22.)
template <int NTF, int G>
__device__ __forceinline__ void i8_split_tile(const I8Args& A, const I8Unit<1>& u, int wave, int group, uint32_t xs_base)
{
    constexpr uint32_t kBuf = (uint32_t)kI8TileRows * 128;
    const int lane = threadIdx.x & (kWave - 1), ln = lane & 31, kb = lane >> 5;
    const uint32_t lane16 = (uint32_t)lane * 16u, own = xs_base + (uint32_t)group * 2u * kBuf;
    const int nkt = A.Kp >> 7, per = (nkt + G - 1) / G, first = group * per;
    const int tiles = max(0, min(per, nkt - first));
    i32x16_t acc[1][NTF] = {};
    I8Stage<NTF, 1> stage;
    const int rb = 8 * wave + (lane >> 3);
    const uint32_t chunk = (uint32_t)((lane & 7) ^ i8_turn<1>(rb)) * 16u;
#pragma unroll
    for (int i = 0; i < NTF; i++) stage.off[i] = (uint32_t)min(32 * i + rb, u.rows - 1) * (uint32_t)A.Kp + chunk;
    stage.base = A.x + (long)u.row0 * A.Kp;
    stage.lds = __builtin_amdgcn_readfirstlane(own + (uint32_t)wave * 1024u);
    auto copy = [&](int k, uint32_t at) {
        const char* const base = stage.base + (long)min(first + k, nkt - 1) * 128;       // (past a group's last: its bytes go unused)
#pragma unroll
        for (int i = 0; i < NTF; i++) lds_copy16(base, stage.off[i], stage.lds + at + (uint32_t)i * 4096u);
    };
    const uint32_t xa0 = own + (uint32_t)ln * 128u + (((uint32_t)kb << 6) ^ ((uint32_t)i8_turn<1>(ln) << 4));
    I8Strips<1, 1> w;
    copy(0, 0);
#pragma unroll
    for (int j = 0; j < 4; j++) w.r[0][j] = i8_chunk(u.qw[0], lane16, min(first, nkt - 1), j);
    wait_lds_copies<0>();
    __syncthreads();
    uint32_t at = 0;
    for (int k = 0; k < per; k++) {
        if (k < tiles) {
            copy(k + 1, at ^ kBuf);
            i8_step<NTF, 1, 1, 1>(w, u.qw, lane16, first + k + 1, nkt, xa0 + at, acc);
            wait_lds_copies<4>();               // the copies are older than the loads of weights
        }
        __syncthreads();
        at ^= kBuf;
    }
    // fragments in turn: [group][wavefront][row of 32 sums]
    const uint32_t area = xs_base + (uint32_t)(group * 4 + wave) * kI8EpiWave<1>;
    const int n = (4 * u.bx + wave) * 32 + 4 * (lane & 7), left = A.N - n;
    float sc[4], add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        sc[i] = u.sa[min(n + i, A.N - 1)];
        if (A.bias) add[i] = A.bias[min(n + i, A.N - 1)];
    }
#pragma unroll
    for (int tf = 0; tf < NTF; tf++) {
#pragma unroll
        for (int g = 0; g < 4; g++)
            lds_write16(area + (uint32_t)ln * kI8EpiRow<1> + (uint32_t)(kb * 16 + g * 32),
                        make_uint4((uint32_t)acc[0][tf][4 * g], (uint32_t)acc[0][tf][4 * g + 1], (uint32_t)acc[0][tf][4 * g + 2],
                                   (uint32_t)acc[0][tf][4 * g + 3]));
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4 / G; j++) {
            const int rr = 8 * (group + G * j) + (lane >> 3), row = 32 * tf + rr;
            uint32_t sum[4] = {0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < G; g++) {
                const uint32_t from = xs_base + (uint32_t)(g * 4 + wave) * kI8EpiWave<1> + (uint32_t)rr * kI8EpiRow<1>;
                const uint4 p = lds_read16(from + (uint32_t)(lane & 7) * 16u);
                sum[0] += p.x;
                sum[1] += p.y;
                sum[2] += p.z;
                sum[3] += p.w;
            }
            if (row >= u.rows || left <= 0) continue;
            const float xs = A.xs[u.row0 + row];
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = i8_value((int)sum[i], xs, sc[i], add[i]);
            i8_store4(A.out, (long)(u.row0 + row) * A.ldo + n, A.out_dtype, left >= 4 && A.aligned, left, v);
        }
        __syncthreads();
    }
}

template <int G>
constexpr int kI8SplitLds = G * 2 * kI8TileRows * 128;

template <int G>
__global__ __launch_bounds__(256 * G, 4) void i8_split_kernel(const I8Args A)
{
    extern __shared__ __attribute__((aligned(1024))) char xs_raw[];
    static_assert(4 * G * kI8EpiWave<1> <= kI8SplitLds<G>, "the epilogue areas fit in the buffers");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    I8Unit<1> u;
    if (!i8_plain_unit<1>(A, u, wave & 3)) return;
    const uint32_t xs = lds_base(xs_raw);
    switch ((u.rows + 31) >> 5) {
    case 1: i8_split_tile<1, G>(A, u, wave & 3, wave >> 2, xs); break;
    case 2: i8_split_tile<2, G>(A, u, wave & 3, wave >> 2, xs); break;
    case 3: i8_split_tile<3, G>(A, u, wave & 3, wave >> 2, xs); break;
    default: i8_split_tile<4, G>(A, u, wave & 3, wave >> 2, xs); break;
    }
}

// Experts.  One that more than kI8TileWide pairs go to takes tiles of 128 rows and two strips a wavefront; the others, whose weights' bytes
// bound them, one wide tile.  Runs of the two kinds alternate in proportion, so that the chip multiplies while it reads.
// The whole call with 160, 128 and 96 as the wide tiles' limit, and with tall tiles alone: 512 tokens, 2 of 8 experts of 14336 x 4096 355, 375, 392
// and 393 us, 2048 tokens 913, 915, 916 and 914; 2048 tokens, 8 of 128 experts of 768 x 2048, loads skewed, 253, 250, 249 and 244, 512 tokens 137, 139,
// 136 and 132.  Up and down: 218 and 111 us (512 tokens, large experts; 4.3 TB/s of weights), 115 and 88 (2048, small ones, loads skewed).
template <int MODE>
__global__ __launch_bounds__(256, 2) void i8_experts_kernel(const I8Args A)
{
    extern __shared__ __attribute__((aligned(1024))) char xs_raw[];
    const uint32_t xs = lds_base(xs_raw);
    const I8Plan pp = i8_plan(const_cast<int32_t*>(A.plan), A.P);
    const int tall = pp.meta[0], wide = pp.meta[1];
    const int c2 = kI8Cols<MODE, 2>, c1 = kI8Cols<MODE, 1>;
    const long units2 = (long)tall * ((A.N + c2 - 1) / c2), units1 = (long)wide * ((A.N + c1 - 1) / c1);
    const long runs2 = (units2 + kI8Run - 1) / kI8Run, runs1 = (units1 + kI8Run - 1) / kI8Run, runs = runs1 + runs2;
    const long run = i8_run<kI8Run>();
    if (run >= runs) return;
    const long before = run * runs2 / runs, upto = (run + 1) * runs2 / runs;      // runs of tall tiles before this one, and with it
    if (upto > before) {
        const long unit = before * kI8Run + i8_turn_in_run<kI8Run>();
        if (unit >= units2) return;
        I8Unit<2> u;
        i8_expert_unit<MODE, 2, kI8TileRows>(A, pp, 0, unit, u);
#define DYMOE_I8_TILE(NTF) i8_tile<MODE, NTF, 2, 2>(A, pp.perm, u.qw, u.sa, u.sb, u.row0, u.rows, u.bx, xs, (uint32_t)kI8TileRows * 256u)
        switch ((u.rows + 31) >> 5) {
        case 1: DYMOE_I8_TILE(1); break;
        case 2: DYMOE_I8_TILE(2); break;
        case 3: DYMOE_I8_TILE(3); break;
        default: DYMOE_I8_TILE(4); break;
        }
#undef DYMOE_I8_TILE
    } else {
        const long unit = (run - before) * kI8Run + i8_turn_in_run<kI8Run>();
        if (unit >= units1) return;
        I8Unit<1> u;
        i8_expert_unit<MODE, 1, kI8TileWide>(A, pp, tall, unit, u);
#define DYMOE_I8_TILE(NTF) i8_wide_tile<MODE, NTF>(A, pp.perm, u.qw[0], u.sa, u.sb, u.row0, u.rows, u.bx, xs)
        switch ((u.rows + 31) >> 5) {
        case 1: DYMOE_I8_TILE(1); break;
        case 2: DYMOE_I8_TILE(2); break;
        case 3: DYMOE_I8_TILE(3); break;
        case 4: DYMOE_I8_TILE(4); break;
        default: DYMOE_I8_TILE(5); break;
        }
#undef DYMOE_I8_TILE
    }
}

template <int KT>
constexpr int kI8Lds = 2 * kI8TileRows * 128 * KT;
static_assert(2 * kI8TileWide * 128 <= kI8Lds<2>, "the wide tiles' buffers fit in the tall ones'");
static_assert(4 * kI8EpiWave<2> <= kI8Lds<2> && 4 * kI8EpiWave<1> <= kI8Lds<1>, "the epilogue areas fit in the buffers");
static_assert(sizeof(I8TileRec) == 64 && offsetof(I8TileRec, mat) == 16, "as the plan writes it");
static_assert(4 * kI8EpiWave<1> <= 2 * 32 * 128 * 4, "also in those of a wide tile");

// per-device set-up, with the device current
int i8_init()
{
    auto allow = [](const void* f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess; };
    bool ok = allow((const void*)i8_matmul_kernel<2, 2>, kI8Lds<2>) && allow((const void*)i8_experts_kernel<kI8Up>, kI8Lds<2>) &&
              allow((const void*)i8_experts_kernel<kI8Down>, kI8Lds<2>);
    ok = ok && allow((const void*)i8_split_kernel<2>, kI8SplitLds<2>) && allow((const void*)i8_split_kernel<4>, kI8SplitLds<4>);
    ok = ok && allow((const void*)i8_thin_kernel<kI8Up, true>, (int)kI8FuseBytes) &&
         allow((const void*)i8_thin_down_kernel, (int)kI8FuseBytes);
    return ok ? DYMOE_OK : DYMOE_EHIP;
}

// workgroups for `units` units and `kinds` kinds of them, whose last runs need not be whole
static dim3 i8_grid(long units, int kinds, int run)
{
    return dim3((unsigned)(((units + run - 1) / run + kinds - 1 + 7) / 8 * 8 * run));
}

// ----------------------------------------------------------------------------
// Tiles of up to 32 NTF rows where rows or columns are too few for the shapes above (decode batches on experts, narrow matrices): a workgroup
// owns 32 weight rows (of W1 and of W3 in the up projection) and its NW wavefronts take the 128-column tiles of K in turn.  Nothing is
// shared before the end: weights and codes come straight into registers, D tiles of a wavefront on their way, and the sums meet in LDS.
// A load of codes that lie row by row touches a line for each of its 64 lanes; the plain product therefore has its rows quantised into
// the weights' tile layout (A.tiled), where it is 1 KiB of contiguous memory.
// 61 x 1536 x 2048: 6.2 us (10.8 in tiles of 128 x 128); 61 tokens, 8 of 128 experts of 768 x 2048: up 61 us (6.5 TB/s), down 31 (6.4 TB/s).
template <int MODE, int NTF, int NW, int D>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 2 : 3) void i8_small_kernel(const I8Args A)
{
    constexpr int S = MODE == kI8Up ? 2 : 1, kSums = S * NTF, kRows = 32 * NTF;
    __shared__ int s_red[4][kSums][16][kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const int nblk = (A.N + 31) / 32;
    const I8Plan pp = i8_plan(const_cast<int32_t*>(A.plan), A.P);
    const long strip = 32L * A.Kp;
    int row0, rows, bx;
    I8Src q[S], x;
    const float *sa, *sb;
    if (MODE == kI8Plain) {
        const int tiles = (A.rows + kRows - 1) / kRows;
        bx = blockIdx.x / tiles;
        row0 = (blockIdx.x - bx * tiles) * kRows;
        rows = min(kRows, A.rows - row0);
        q[0].set(A.w.q + bx * strip, (uint32_t)strip);
        sa = sb = A.w.s;
    } else {
        const int tile = blockIdx.x / nblk;
        bx = blockIdx.x - tile * nblk;
        if (tile >= pp.meta[0]) return;
        const I8TileRec t = pp.tiles[tile];
        const int i = (tile - t.tile0) * kRows;
        row0 = t.first + i;
        rows = min(kRows, t.pairs - i);
        q[0].set((const char*)t.mat.q[MODE == kI8Up ? 0 : 2] + bx * strip, (uint32_t)strip);
        q[S - 1].set((const char*)t.mat.q[MODE == kI8Up ? 1 : 2] + bx * strip, (uint32_t)strip);
        sa = t.mat.s[MODE == kI8Up ? 0 : 2];
        sb = t.mat.s[MODE == kI8Up ? 1 : 2];
    }
    struct Tile {
        uint4 w[S][4], x[NTF][4];
    };
    const uint32_t lane16 = (uint32_t)lane * 16u;
    uint32_t off[NTF];
    const int nkt = A.Kp >> 7;
    // bytes from one 16-byte chunk of a lane's columns to the next, and from one tile to the next
    const uint32_t chunk = MODE == kI8Plain && A.tiled ? 1024u : 16u, step = MODE == kI8Plain && A.tiled ? 4096u : 128u;
    auto load_w = [&](Tile& t, int kt) {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int c = 0; c < 4; c++) t.w[s][c] = q[s].template load<true>(lane16 + (uint32_t)(c * 1024), (uint32_t)kt * 4096u);
    };
    auto load_x = [&](Tile& t, int kt) {
#pragma unroll
        for (int f = 0; f < NTF; f++)
#pragma unroll
            for (int c = 0; c < 4; c++) t.x[f][c] = x.load(off[f], (uint32_t)kt * step + (uint32_t)c * chunk);
    };
    Tile ring[D];
    int kt = wave;
#pragma unroll
    for (int d = 0; d < D; d++)
        if (kt + d * NW < nkt) load_w(ring[d], kt + d * NW);               // (the weights need nothing of the rows)
#pragma unroll
    for (int f = 0; f < NTF; f++) {
        const int r = min(32 * f + ln, rows - 1);                            // rows behind the last: computed and dropped
        off[f] = (MODE == kI8Up ? (uint32_t)(pp.perm[row0 + r] / A.k) : (uint32_t)r) * (uint32_t)A.Kp + 64u * (uint32_t)kb;
        if (MODE == kI8Plain && A.tiled) off[f] = (uint32_t)min(f, (rows - 1) >> 5) * (uint32_t)strip + lane16;
    }
    const int held = MODE == kI8Up ? A.rows : MODE == kI8Plain && A.tiled ? (rows + 31) & ~31 : rows;
    x.set(A.x + (MODE == kI8Up ? 0 : (long)row0 * A.Kp), (uint32_t)held * (uint32_t)A.Kp);
#pragma unroll
    for (int d = 0; d < D; d++)
        if (kt + d * NW < nkt) load_x(ring[d], kt + d * NW);
    i32x16_t acc[S][NTF] = {};
    auto multiply = [&](const Tile& t) {
#pragma unroll
        for (int c = 0; c < 4; c++)
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int f = 0; f < NTF; f++) acc[s][f] = mfma_i8(t.w[s][c], t.x[f][c], acc[s][f]);
    };
    while (kt < nkt) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            if (kt < nkt) {
                multiply(ring[d]);
                __builtin_amdgcn_sched_barrier(0);
                if (kt + D * NW < nkt) {
                    load_w(ring[d], kt + D * NW);
                    load_x(ring[d], kt + D * NW);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            kt += NW;
        }
    }
    auto put = [&](int at) {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int f = 0; f < NTF; f++)
#pragma unroll
                for (int i = 0; i < 16; i++) s_red[at][s * NTF + f][i][lane] = acc[s][f][i];
    };
    if constexpr (NW == 8) {
        if (wave >= 4) put(wave - 4);
        __syncthreads();
        if (wave < 4) {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int f = 0; f < NTF; f++)
#pragma unroll
                    for (int i = 0; i < 16; i++) acc[s][f][i] += s_red[wave][s * NTF + f][i][lane];
            put(wave);                          // (its own place, read by none but it)
        }
    } else {
        put(wave);
    }
    __syncthreads();
    // a wavefront finishes four registers of a fragment: weight rows 8 g + 4 kb + 0 .. 3, token ln
    for (int item = wave; item < 4 * NTF; item += NW) {
        const int f = item >> 2, g = item & 3, row = 32 * f + ln;
        if (row >= rows) continue;
        const int n = 32 * bx + 8 * g + 4 * kb, left = A.N - n;
        if (left <= 0) continue;
        const float xs = A.xs[MODE == kI8Up ? pp.perm[row0 + row] / A.k : row0 + row];
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int m = min(n + i, A.N - 1);
            auto sum = [&](int at) {
                int all = 0;
#pragma unroll
                for (int w = 0; w < 4; w++) all += s_red[w][at][4 * g + i][lane];
                return all;
            };
            v[i] = i8_value(sum(f), xs, sa[m], MODE == kI8Plain && A.bias ? A.bias[m] : 0.0f);
            if (MODE == kI8Up) v[i] = silu_times(v[i], i8_value(sum(NTF + f), xs, sb[m], 0.0f));
        }
        const bool whole = left >= 4 && (MODE != kI8Plain || A.aligned);
        i8_store4(A.out, (long)(row0 + row) * A.ldo + n, MODE == kI8Plain ? A.out_dtype : DYMOE_OUT_F32, whole, left, v);
    }
}

// y[t] = sum over the slots, in their order, of gate times the pair's output.  A workgroup takes 2048 outputs of a token.  Bound by the pairs'
// bytes: 16384 pairs of 2048 outputs 24 us (5.9 TB/s).
__global__ __launch_bounds__(256) void i8_combine_kernel(const float* __restrict__ part, long ldp, const int32_t* __restrict__ where,
                                                         const float* __restrict__ gate, int H, int k, int out_dtype, int aligned,
                                                         void* __restrict__ y)
{
    const int blocks = (H + 2047) / 2048;
    const long t = blockIdx.x / blocks;
    const int h = (int)(blockIdx.x - t * blocks) * 2048 + threadIdx.x * 8;
    if (h >= H) return;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int j = 0; j < k; j++) {
        const int at = where[t * k + j];
        if (at < 0) continue;
        const float g = gate[t * k + j];
        const float4 a = load_global<float4>(part + at * ldp + h), b = load_global<float4>(part + at * ldp + h + 4);
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] = fmaf(g, v[i], sum[i]);
    }
    const float lo[4] = {sum[0], sum[1], sum[2], sum[3]}, hi[4] = {sum[4], sum[5], sum[6], sum[7]};
    i8_store4(y, t * H + h, out_dtype, aligned && h + 4 <= H, H - h, lo);
    i8_store4(y, t * H + h + 4, out_dtype, aligned && h + 8 <= H, H - h - 4, hi);
}

}  // namespace dymoe

using namespace dymoe;

extern "C" size_t dymoe_matmul_int8_workspace_bytes(int T, int N, int K)
{
    if (T < 0 || N <= 0 || K <= 0 || K > DYMOE_INT8_MAX_K) return 0;
    return i8_mat_layout(T, K).total;
}

extern "C" int dymoe_matmul_int8(dymoe_ctx* ctx, const void* x, int x_dtype, const float* x_scale, long ldx, const int8_t* w,
                                 const float* w_scale, const float* bias, int T, int N, int K, int out_dtype, void* y, long ldy,
                                 void* workspace, size_t workspace_bytes, void* stream)
{
    DYMOE_REQUIRE(T >= 0 && N > 0 && K > 0 && ldy >= N);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16 || x_dtype == DYMOE_DTYPE_I8);
    DYMOE_REQUIRE(out_dtype == DYMOE_OUT_BF16 || out_dtype == DYMOE_OUT_F32 || out_dtype == DYMOE_OUT_F16);
    const bool coded = x_dtype == DYMOE_DTYPE_I8;
    DYMOE_REQUIRE(coded ? ldx == up_to(K, 128) : ldx >= K);
    DYMOE_REQUIRE(w && w_scale);
    if (T > 0) DYMOE_REQUIRE(x && y && (coded ? x_scale != nullptr : workspace != nullptr));
    DYMOE_REQUIRE(dymoe_aligned(x, coded ? 16 : dtype_bytes(x_dtype)) && dymoe_aligned(y, dtype_bytes(out_dtype)) && dymoe_aligned(w, 16));
    DYMOE_REQUIRE(dymoe_aligned(x_scale, 4) && dymoe_aligned(w_scale, 4) && dymoe_aligned(bias, 4) && dymoe_aligned(workspace, 256));
    if (K > DYMOE_INT8_MAX_K) return DYMOE_ENOTSUP;
    if (T > (1 << 24) || N > (1 << 24)) return DYMOE_ENOTSUP;
    const I8MatLayout L = i8_mat_layout(T, K);
    if (!coded && T > 0 && workspace_bytes < L.total) return DYMOE_ENOSPC;
    if (i8_strip_units(T, N) > 0x7fff0000L) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const I8MatChoice c = i8_mat_choice(T, N, K, coded, ctx->num_cu);
    const bool small = c.shape == I8MatShape::kSmall32 || c.shape == I8MatShape::kSmall64, fuse = c.fuse;
    I8Args A = {};
    A.x = (const char*)x;
    A.xs = x_scale;
    if (!coded && !fuse) {
        A.tiled = small;
        const int rc = quantize_rows(ctx, x, x_dtype, T, K, ldx, small, ws + L.xq, (float*)(ws + L.xs), st);
        if (rc != DYMOE_OK) return rc;
        A.x = ws + L.xq;
        A.xs = (const float*)(ws + L.xs);
    }
    A.w.q = (const char*)w;
    A.w.s = w_scale;
    A.bias = bias;
    A.out = y;
    A.ldo = ldy;
    A.rows = T;
    A.Kp = (int)L.Kp;
    A.N = N;
    A.out_dtype = out_dtype;
    if (c.shape == I8MatShape::kThin) {
        I8ThinArgs B = {};
        B.x = A.x;
        B.xs = A.xs;
        B.w = A.w;
        B.bias = bias;
        B.out = y;
        B.ldx = fuse ? ldx * dtype_bytes(x_dtype) : (long)L.Kp;
        B.ldo = ldy;
        B.x_dtype = x_dtype;
        B.rows = T;
        B.K = K;
        B.Kp = (int)L.Kp;
        B.N = N;
        B.out_dtype = out_dtype;
        const dim3 grid((unsigned)((N + 15) / 16)), block(64 * kI8ThinWaves);
        if (fuse) dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_thin_kernel<kI8Plain, true>, grid, block, T * (L.Kp + 16), st, B);
        else dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_thin_kernel<kI8Plain, false>, grid, block, 0, st, B);
        DYMOE_HIP_LAUNCH_CHECK();
        return DYMOE_OK;
    }
    A.aligned = dymoe_aligned(y, 4 * dtype_bytes(out_dtype)) && ldy % 4 == 0;
    const long tiles = (T + kI8TileRows - 1L) / kI8TileRows, strips = (N + 31L) / 32;
    const dim3 grid1 = i8_grid(tiles * ((N + 127L) / 128), 1, kI8RunPlain);
    switch (c.shape) {
    case I8MatShape::kSmall32:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_small_kernel<kI8Plain, 1, 8, 4>, dim3((unsigned)strips), dim3(512), 0, st, A);
        break;
    case I8MatShape::kSmall64:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_small_kernel<kI8Plain, 2, 8, 3>, dim3((unsigned)i8_strip_units(T, N)), dim3(512), 0, st, A);
        break;
    case I8MatShape::kSplit4:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_split_kernel<4>, grid1, dim3(1024), kI8SplitLds<4>, st, A);
        break;
    case I8MatShape::kSplit2:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_split_kernel<2>, grid1, dim3(512), kI8SplitLds<2>, st, A);
        break;
    case I8MatShape::kOne:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_matmul_kernel<1, 1>, grid1, dim3(256), kI8Lds<1>, st, A);
        break;
    default:
        dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_matmul_kernel<2, 2>, i8_grid(tiles * ((N + 255L) / 256), 1, kI8RunPlain), dim3(256), kI8Lds<2>, st, A);
    }
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

extern "C" size_t dymoe_moe_ffn_int8_workspace_bytes(int T, int H, int F, int E, int k)
{
    if (T < 0 || H <= 0 || F <= 0 || E <= 0 || k <= 0 || k > E) return 0;
    return i8_ffn_layout(T, H, F, E, k).total;
}

extern "C" int dymoe_moe_ffn_int8(dymoe_ctx* ctx, const void* x, int x_dtype, const int32_t* idx, const float* w,
                                  const dymoe_expert_i8* table, int T, int H, int F, int E, int k, int out_dtype, void* y,
                                  void* workspace, size_t workspace_bytes, void* stream)
{
    DYMOE_REQUIRE(T >= 0 && H > 0 && F > 0 && E > 0 && k > 0 && k <= E);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(out_dtype == DYMOE_OUT_BF16 || out_dtype == DYMOE_OUT_F32 || out_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(table && workspace);
    if (T > 0) DYMOE_REQUIRE(x && idx && w && y);
    DYMOE_REQUIRE(dymoe_aligned(x, dtype_bytes(x_dtype)) && dymoe_aligned(y, dtype_bytes(out_dtype)) && dymoe_aligned(workspace, 256));
    DYMOE_REQUIRE(dymoe_aligned(idx, 4) && dymoe_aligned(w, 4) && dymoe_aligned(table, 8));
    if (E > DYMOE_MAX_EXPERTS || H > DYMOE_INT8_MAX_K || F > DYMOE_INT8_MAX_K) return DYMOE_ENOTSUP;
    if ((long)T * k >= 1L << 29 || (long)T * up_to(H, 128) >= 1L << 32) return DYMOE_ENOTSUP;      // (32-bit offsets into the codes)
    const I8FfnLayout L = i8_ffn_layout(T, H, F, E, k);
    if (workspace_bytes < L.total) return DYMOE_ENOSPC;
    const long up = (long)L.max_tiles * ((F + 31L) / 32), down = (long)L.max_tiles * ((H + 31L) / 32);      // workgroups at most
    if (up > 0x7fff0000L || down > 0x7fff0000L || T * ((H + 2047L) / 2048) >= 1L << 23) return DYMOE_ENOTSUP;      // (256 threads a row, 2^32 a grid)
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const long P = (long)T * k;
    const I8FfnShape shape = i8_ffn_choice(T, H, F, E, k);
    if (shape == I8FfnShape::kThin) {
        I8ThinArgs B = {};
        B.x = (const char*)x;
        B.idx = idx;
        B.table = table;
        B.flags = ctx->device_flags;
        B.out = ws + L.h;
        B.ldx = (long)H * dtype_bytes(x_dtype);
        B.ldo = (long)L.Fp;
        B.x_dtype = x_dtype;
        B.rows = T;
        B.K = H;
        B.Kp = (int)L.Hp;
        B.N = F;
        B.E = E;
        B.k = k;
        B.P = (int)P;
        dymoe_launch(ctx, DYMOE_K_INT8_UP, i8_thin_kernel<kI8Up, true>, dim3((unsigned)(P * ((F + 15) / 16))), dim3(64 * kI8ThinWaves),
                     T * (L.Hp + 16), st, B);
        B.x = ws + L.h;
        B.gate = w;
        B.out = y;
        B.ldx = (long)L.Fp * 4;
        B.ldo = H;
        B.K = F;
        B.Kp = (int)L.Fp;
        B.N = H;
        B.out_dtype = out_dtype;
        dymoe_launch(ctx, DYMOE_K_INT8_DOWN, i8_thin_down_kernel, dim3((unsigned)(8 * T * (((H + 15) / 16 + 7) / 8))), dim3(64 * kI8LastWaves),
                     k * (L.Fp + 16), st, B);
        DYMOE_HIP_LAUNCH_CHECK();
        return DYMOE_OK;
    }
    const bool small = shape == I8FfnShape::kSmall;
    // Workgroups at most: an expert of n pairs has n / 128 + 1 tall tiles at half as many column blocks, or one wide tile.
    const long tall = P / kI8TileRows + P / (kI8TileWide + 1), wide = E < P ? E : P;
    int32_t* const plan = (int32_t*)(ws + L.plan);
    int rc = DYMOE_OK;
    if (H <= 16384) {
        auto prep = i8_prep_launch<DYMOE_OUT_BF16>;
        if (x_dtype == DYMOE_OUT_F32) prep = i8_prep_launch<DYMOE_OUT_F32>;
        else if (x_dtype == DYMOE_OUT_F16) prep = i8_prep_launch<DYMOE_OUT_F16>;
        prep(ctx, idx, table, P, E, small, plan, x, T, H, ws + L.xq, (float*)(ws + L.xs), st);
    } else {
        rc = quantize_rows(ctx, x, x_dtype, T, H, H, 0, ws + L.xq, (float*)(ws + L.xs), st);
        if (rc != DYMOE_OK) return rc;
        dymoe_launch(ctx, DYMOE_K_INT8_PLAN, i8_plan_kernel, dim3(1), dim3(kI8PlanThreads), 0, st, idx, table, P, E, (int)small, plan, ctx->device_flags);
    }
    I8Args A = {};
    A.x = ws + L.xq;
    A.xs = (const float*)(ws + L.xs);
    A.plan = plan;
    A.out = ws + L.h;
    A.ldo = (long)L.Fp;
    A.P = P;
    A.Kp = (int)L.Hp;
    A.N = F;
    A.k = k;
    A.rows = T;
    const dim3 up_grid = i8_grid(tall * ((F + 127L) / 128) + wide * ((F + 63L) / 64), 2, kI8Run);
    const dim3 down_grid = i8_grid(tall * ((H + 255L) / 256) + wide * ((H + 127L) / 128), 2, kI8Run);
    if (small) dymoe_launch(ctx, DYMOE_K_INT8_UP, i8_small_kernel<kI8Up, 1, 4, 1>, dim3((unsigned)up), dim3(256), 0, st, A);
    else dymoe_launch(ctx, DYMOE_K_INT8_UP, i8_experts_kernel<kI8Up>, up_grid, dim3(256), kI8Lds<2>, st, A);
    rc = quantize_rows(ctx, ws + L.h, DYMOE_OUT_F32, P, F, (long)L.Fp, 0, ws + L.hq, (float*)(ws + L.hs), st);
    if (rc != DYMOE_OK) return rc;
    A.x = ws + L.hq;
    A.xs = (const float*)(ws + L.hs);
    A.out = ws + L.part;
    A.ldo = (long)L.Hp;
    A.Kp = (int)L.Fp;
    A.N = H;
    if (small) dymoe_launch(ctx, DYMOE_K_INT8_DOWN, i8_small_kernel<kI8Down, 1, 4, 1>, dim3((unsigned)down), dim3(256), 0, st, A);
    else dymoe_launch(ctx, DYMOE_K_INT8_DOWN, i8_experts_kernel<kI8Down>, down_grid, dim3(256), kI8Lds<2>, st, A);
    const dim3 grid((unsigned)(T * ((H + 2047L) / 2048)));
    dymoe_launch(ctx, DYMOE_K_INT8_COMBINE, i8_combine_kernel, grid, dim3(256), 0, st, (const float*)(ws + L.part), (long)L.Hp,
                 i8_plan(plan, P).where, w, H, k, out_dtype, H % 4 == 0 && dymoe_aligned(y, 4 * dtype_bytes(out_dtype)), y);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
