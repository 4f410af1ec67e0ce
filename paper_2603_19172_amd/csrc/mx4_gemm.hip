// Products in microscaled 4-bit floating point: a matrix (dymoe_matmul_mx4) and a layer's SwiGLU experts (dymoe_moe_ffn_mx4).
//   y[t, n] = sum over blocks b of 32 columns of 2^(ex[t, b] + ew[n, b]) sum_{j in b} xq[t, j] wq[n, j]
// A block's sum is exact; the sum over the blocks is taken in fp32, in an order that belongs to the shape of the call.
#include <type_traits>

#include "expert_plan.hpp"
#include "mx4_device.hpp"
#include "mx4_layout.hpp"

namespace dymoe {

int mx4_quantize(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, uint8_t* codes, uint8_t* scale, hipStream_t st);
void experts_combine(dymoe_ctx* ctx, int kernel_id, const float* part, long ldp, const int32_t* where, const float* gate, int T, int H, int k,
                     int out_dtype, void* y, hipStream_t st);

using Mx4Plan = ExpertPlan<dymoe_expert_mx4>;

// The plan by the first workgroup, the codes of the activations by the others, a wavefront 512 columns of a row: neither needs the other.
template <int DT>
__global__ __launch_bounds__(kPlanThreads) void mx4_prep_kernel(const int32_t* __restrict__ idx, const dymoe_expert_mx4* __restrict__ table, long P,
                                                                int E, int small, int32_t* __restrict__ plan, unsigned* __restrict__ flags,
                                                                const char* __restrict__ x, long units, int per_row, int K, char* __restrict__ codes,
                                                                char* __restrict__ scale)
{
    __shared__ ExpertPlanLds lds;
    if (blockIdx.x == 0) {
        make_expert_plan<kMx4SmallRows, 0, kMx4TallRows>(lds, idx, table, P, E, small, plan, flags);
        return;
    }
    const long unit = (blockIdx.x - 1L) * (kPlanThreads / kWave) + threadIdx.x / kWave;
    if (unit >= units) return;
    const long row = unit / per_row;
    const int col = (int)(unit - row * per_row) * 512 + (threadIdx.x & (kWave - 1)) * 8, Kp = (int)up_to(K, 256);
    const Raw8<DT> v = load8<DT>(x + row * K * dtype_bytes(DT), col, K);
    const uint32_t byte = mx4_exponent(quad_max_u32(peak_f32_bits<DT>(peak8<DT>(v, 0u)))), q = mx4_codes8<DT>(v, byte);
    if (col >= Kp) return;
    *(DYMOE_GLOBAL uint32_t*)(codes + (row * Kp + col) / 2) = q;
    if ((col & 31) == 0) *(DYMOE_GLOBAL uint8_t*)(scale + (row * Kp + col) / 32) = (uint8_t)byte;
}

enum { kMx4Plain = 0, kMx4Up = 1, kMx4Down = 2 };

struct Mx4Args {
    const char *x, *xs;               // codes of the rows, Kp / 2 bytes each, and their exponents, Kp / 32
    const int32_t* plan;              // experts
    const char *w, *ws;               // the plain product
    const float* bias;
    void* out;                        // up: codes of the intermediate's rows, ldo / 2 bytes each
    uint8_t* out_scale;               // up: their exponents, ldo / 32
    long ldo, P;
    int rows, Kp, N, k, out_dtype, aligned;     // aligned: the plain product's rows start where four outputs may be stored at once
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

// ----------------------------------------------------------------------------
// Tiles of up to 32 NTF rows: a workgroup owns 32 weight rows (of W1 and of W3 in the up projection) and its NW wavefronts take the 256-column
// tiles of K in turn.  Nothing is shared before the end: weights and codes come straight into registers, D tiles of a wavefront on their
// way, and the sums meet in LDS.
template <int MODE, int NTF, int NW, int D>
__global__ __launch_bounds__(64 * NW) void mx4_small_kernel(const Mx4Args A)
{
    constexpr int S = MODE == kMx4Up ? 2 : 1, kSums = S * NTF, kRows = 32 * NTF;
    __shared__ float s_red[4][kSums][16][kWave];
    __shared__ uint32_t s_peak[NTF][4][32];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const int strips = (A.N + 31) / 32, nblk = MODE == kMx4Up ? (int)up_to(A.N, 256) / 32 : strips;
    const Mx4Plan pp = expert_plan<dymoe_expert_mx4>(const_cast<int32_t*>(A.plan), A.P);
    int row0, rows, bx;
    Mx4Strip w[S];
    if (MODE == kMx4Plain) {
        const int tiles = (A.rows + kRows - 1) / kRows;
        bx = blockIdx.x / tiles;
        row0 = (blockIdx.x - bx * tiles) * kRows;
        rows = min(kRows, A.rows - row0);
        w[0].set(A.w, A.ws, bx, strips, A.Kp);
    } else {
        const int tile = blockIdx.x / nblk;
        bx = blockIdx.x - tile * nblk;
        if (tile >= pp.meta[0]) return;
        const ExpertTile<dymoe_expert_mx4> t = pp.tiles[tile];
        const int i = (tile - t.tile0) * kRows;
        row0 = t.first + i;
        rows = min(kRows, t.pairs - i);
        w[0].set(t.mat.q[MODE == kMx4Up ? 0 : 2], t.mat.s[MODE == kMx4Up ? 0 : 2], bx, strips, A.Kp);
        if (MODE == kMx4Up) w[S - 1].set(t.mat.q[1], t.mat.s[1], bx, strips, A.Kp);
    }
    struct Tile {
        uint4 w[S][4], x[NTF][4];
        uint32_t ws[S], xs[NTF];
    };
    const uint32_t lane16 = (uint32_t)lane * 16u, lane4 = (uint32_t)lane * 4u;
    const int nkt = A.Kp >> 8;
    uint32_t off[NTF], offs[NTF];
    BufferSrc x, xs;
    auto load_w = [&](Tile& t, int kt) {
#pragma unroll
        for (int s = 0; s < S; s++) {
#pragma unroll
            for (int c = 0; c < 4; c++) t.w[s][c] = w[s].q.template load<true>(lane16 + (uint32_t)(c * 1024), (uint32_t)kt * 4096u);
            t.ws[s] = load_u32(w[s].s, lane4, (uint32_t)kt * 256u);
        }
    };
    auto load_x = [&](Tile& t, int kt) {
#pragma unroll
        for (int f = 0; f < NTF; f++) {
#pragma unroll
            for (int c = 0; c < 4; c++) t.x[f][c] = x.load(off[f] + (uint32_t)c * 16u, (uint32_t)kt * 128u);
            t.xs[f] = load_u32(xs, offs[f], (uint32_t)kt * 8u);
        }
    };
    Tile ring[D];
    int kt = wave;
#pragma unroll
    for (int d = 0; d < D; d++)
        if (kt + d * NW < nkt) load_w(ring[d], kt + d * NW);               // (the weights need nothing of the rows)
#pragma unroll
    for (int f = 0; f < NTF; f++) {
        const int r = min(32 * f + ln, rows - 1);                            // rows behind the last: computed and dropped
        const uint32_t row = MODE == kMx4Up ? (uint32_t)(pp.perm[row0 + r] / A.k) : (uint32_t)r;
        off[f] = row * (uint32_t)(A.Kp >> 1) + 64u * (uint32_t)kb;
        offs[f] = row * (uint32_t)(A.Kp >> 5) + 4u * (uint32_t)kb;
    }
    const long from = MODE == kMx4Up ? 0 : row0;
    const uint32_t held = MODE == kMx4Up ? A.rows : rows;
    x.set(A.x + from * (A.Kp >> 1), held * (uint32_t)(A.Kp >> 1));
    xs.set(A.xs + from * (A.Kp >> 5), held * (uint32_t)(A.Kp >> 5));
#pragma unroll
    for (int d = 0; d < D; d++)
        if (kt + d * NW < nkt) load_x(ring[d], kt + d * NW);
    float16_t acc[S][NTF] = {};
    auto multiply = [&](const Tile& t) {
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int f = 0; f < NTF; f++) {
                acc[s][f] = mfma_mx4<0, 0>(t.w[s][0], t.x[f][0], acc[s][f], t.ws[s], t.xs[f]);
                acc[s][f] = mfma_mx4<1, 1>(t.w[s][1], t.x[f][1], acc[s][f], t.ws[s], t.xs[f]);
                acc[s][f] = mfma_mx4<2, 2>(t.w[s][2], t.x[f][2], acc[s][f], t.ws[s], t.xs[f]);
                acc[s][f] = mfma_mx4<3, 3>(t.w[s][3], t.x[f][3], acc[s][f], t.ws[s], t.xs[f]);
            }
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
    auto sum = [&](int at, int i) {
        float all = s_red[0][at][i][lane];
#pragma unroll
        for (int w = 1; w < 4; w++) all += s_red[w][at][i][lane];
        return all;
    };
    // a wavefront finishes four registers of a fragment: weight rows 8 g + 4 kb + 0 .. 3, token ln
    constexpr int kGroups = NW / 4, kEach = (NTF + kGroups - 1) / kGroups;
    const int g = wave & 3;
    if constexpr (MODE == kMx4Up) {
        uint32_t h[kEach][4];
#pragma unroll
        for (int j = 0; j < kEach; j++) {
            const int f = (wave >> 2) + kGroups * j;
            if (f >= NTF) continue;
            uint32_t peak = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                h[j][i] = __float_as_uint(silu_times(sum(f, 4 * g + i), sum(NTF + f, 4 * g + i)));
                peak = max(peak, h[j][i] & 0x7fffffffu);
            }
            const auto both = __builtin_amdgcn_permlane32_swap(peak, peak, false, false);
            if (kb == 0) s_peak[f][g][ln] = max(both[0], both[1]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; j++) {
            const int f = (wave >> 2) + kGroups * j, row = 32 * f + ln;
            if (f >= NTF) continue;
            const uint32_t byte = mx4_exponent(max(max(s_peak[f][0][ln], s_peak[f][1][ln]), max(s_peak[f][2][ln], s_peak[f][3][ln])));
            const float unit = mx4_unit(byte);
            uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, __uint_as_float(h[j][0]), __uint_as_float(h[j][1]), unit, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(h[j][2]), __uint_as_float(h[j][3]), unit, 1);
            const auto both = __builtin_amdgcn_permlane32_swap(q, q, false, false);
            q = byte == 255u ? 0u : (both[0] & 0xffffu) | (both[1] << 16);
            if (kb != 0 || row >= rows) continue;
            const long at = (long)(row0 + row) * A.ldo + 32 * bx;
            *(DYMOE_GLOBAL uint32_t*)((char*)A.out + at / 2 + 4 * g) = q;
            if (g == 0) *(DYMOE_GLOBAL uint8_t*)(A.out_scale + at / 32) = (uint8_t)byte;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kEach; j++) {
            const int f = (wave >> 2) + kGroups * j, row = 32 * f + ln;
            if (f >= NTF || row >= rows) continue;
            const int n = 32 * bx + 8 * g + 4 * kb, left = A.N - n;
            if (left <= 0) continue;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[i] = sum(f, 4 * g + i);
                if (MODE == kMx4Plain && A.bias) v[i] += A.bias[min(n + i, A.N - 1)];
            }
            const bool whole = left >= 4 && (MODE != kMx4Plain || A.aligned);
            store_out4(A.out, (long)(row0 + row) * A.ldo + n, MODE == kMx4Plain ? A.out_dtype : DYMOE_OUT_F32, whole, left, v);
        }
    }
}

// ----------------------------------------------------------------------------
// Tiles of up to 32 NTF rows and 128 S weight rows (S / 2 times 128 of W1 and of W3 in the up projection): a workgroup of four wavefronts walks K
// in steps of 256 columns.
//  * Weights come straight into registers: a tile's bytes lie in the order of the matrix instruction's operand, so a wavefront's load is 1 KiB
//    of contiguous memory.  A register is requested anew, for the step after the next, as soon as the last instruction that reads it has been
//    issued.
//  * The rows' codes and exponents are shared by the wavefronts through three LDS buffers that global memory fills directly, two steps ahead; the 16-byte chunks of
//    a row's 128 bytes are turned by its number, which spreads the operand reads (one chunk of 32 rows) over all banks.
constexpr uint32_t kMx4Row = 128;           // bytes of a row of a step
template <int NTF>
constexpr uint32_t kMx4Buf = 32u * NTF * (kMx4Row + 8u);
constexpr uint32_t kMx4EpiRow = 144;        // epilogue: bytes of a row of 32 sums in LDS, 16 of them padding
constexpr uint32_t kMx4EpiWave = 32 * kMx4EpiRow;

__device__ __forceinline__ int mx4_turn(int row) { return (row >> 1) & 7; }      // (the row's parity is half of the banks already)

template <int S>
struct Mx4Weights {
    uint4 r[2][S][4];              // codes of an even step and of an odd one
    uint32_t e[2][S];              // exponents
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

template <int MODE, int NTF, int S>
__device__ __forceinline__ void mx4_tile(const Mx4Args& A, const int32_t* perm, Mx4Weights<S>& w, int row0, int rows, int bx, uint32_t base)
{
    constexpr int kMask = 0x2 | 0x4;             // vector and scalar arithmetic may cross; products, LDS and memory accesses may not
    constexpr uint32_t kBuf = kMx4Buf<NTF>, kExp = 32u * NTF * kMx4Row;
    constexpr int kCopies = NTF + (NTF + 3) / 4;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const uint32_t lane16 = (uint32_t)lane * 16u;
    const int steps = A.Kp >> 8, end = steps - 1;
    float16_t acc[S][NTF] = {};
    // copies: rows 32 i + 8 wave + lane / 8, chunk lane % 8 turned; exponents of fragment `wave` (and wave + 4)
    const char* const xb = A.x + (MODE == kMx4Up ? 0 : (long)row0 * (A.Kp >> 1));
    const char* const sb = A.xs + (MODE == kMx4Up ? 0 : (long)row0 * (A.Kp >> 5));
    uint32_t off[NTF], offs[(NTF + 3) / 4];
    auto source = [&](int r) {                   // rows behind the last: computed and dropped
        r = min(r, rows - 1);
        return MODE == kMx4Up ? (uint32_t)(perm[row0 + r] / A.k) : (uint32_t)r;
    };
    const int rb = 8 * wave + (lane >> 3);
#pragma unroll
    for (int i = 0; i < NTF; i++) off[i] = source(32 * i + rb) * (uint32_t)(A.Kp >> 1) + 16u * (uint32_t)((lane & 7) ^ mx4_turn(rb));
    // (wavefronts without a fragment of their own copy the last one's exponents again: the count of copies is then every wavefront's)
#pragma unroll
    for (int i = 0; i < (NTF + 3) / 4; i++) offs[i] = source(32 * min(wave + 4 * i, NTF - 1) + (lane >> 1)) * (uint32_t)(A.Kp >> 5) + 4u * (uint32_t)(lane & 1);
    auto copy = [&](int step, uint32_t buf) {
#pragma unroll
        for (int i = 0; i < NTF; i++)
            lds_copy16(xb + (long)step * 128, off[i], __builtin_amdgcn_readfirstlane(base + buf + (uint32_t)(i * 4096 + wave * 1024)));
#pragma unroll
        for (int i = 0; i < (NTF + 3) / 4; i++)
            lds_copy4(sb + (long)step * 8, offs[i], __builtin_amdgcn_readfirstlane(base + buf + kExp + (uint32_t)(min(wave + 4 * i, NTF - 1) * 256)));
    };
    copy(0, 0);
    copy(min(1, end), kBuf);
#pragma unroll
    for (int p = 0; p < 2; p++) {
#pragma unroll
        for (int c = 0; c < 4; c++) w.codes(p, c, lane16, min(p, end));
        w.scales(p, lane16, min(p, end));
    }
    wait_lds_copies<kCopies + 10 * S>();        // the first copies are older than everything else
    __syncthreads();
    const uint32_t xa0 = base + (uint32_t)ln * kMx4Row + (((uint32_t)kb << 6) ^ ((uint32_t)mx4_turn(ln) << 4));
    const uint32_t xe0 = base + kExp + (uint32_t)ln * 8u + (uint32_t)kb * 4u;
    uint32_t at = 0;
    // Step ks multiplies what its buffer and registers hold and requests the codes of the rows and of the weights two steps on.
    auto step = [&](int ks, auto parity) __attribute__((always_inline)) {
        constexpr int p = parity();
        const int after = min(ks + 2, end);
        copy(after, at == 0 ? 2 * kBuf : at - kBuf);
        uint32_t xe[NTF];
#pragma unroll
        for (int f = 0; f < NTF; f++) xe[f] = lds_read4(xe0 + at + (uint32_t)f * 256u);
        uint4 op = lds_read16(xa0 + at);
        auto chunk = [&](auto which) __attribute__((always_inline)) {
            constexpr int c = which();
#pragma unroll
            for (int f = 0; f < NTF; f++) {
                constexpr int last = NTF - 1;
                uint4 nxt = op;
                if (!(f == last && c == 3))
                    nxt = lds_read16(((xa0 + at) ^ (uint32_t)((f == last ? c + 1 : c) << 4)) + (uint32_t)(f == last ? 0 : f + 1) * (32u * kMx4Row));
                __builtin_amdgcn_sched_barrier(kMask);
#pragma unroll
                for (int s = 0; s < S; s++) acc[s][f] = mfma_mx4<c, c>(w.r[p][s][c], op, acc[s][f], w.e[p][s], xe[f]);
                op = nxt;
                __builtin_amdgcn_sched_barrier(kMask);
            }
            w.codes(p, c, lane16, after);
            __builtin_amdgcn_sched_barrier(kMask);
        };
        chunk(std::integral_constant<int, 0>());
        chunk(std::integral_constant<int, 1>());
        chunk(std::integral_constant<int, 2>());
        chunk(std::integral_constant<int, 3>());
        w.scales(p, lane16, after);
        __builtin_amdgcn_sched_barrier(kMask);
        wait_lds_copies<kCopies + 10 * S>();    // behind the next step's copies: its and this step's loads of weights, this step's copies
        __syncthreads();
        at = at == 2 * kBuf ? 0 : at + kBuf;
    };
    int ks = 0;
    for (; ks + 2 <= steps; ks += 2) {
        step(ks, std::integral_constant<int, 0>());
        step(ks + 1, std::integral_constant<int, 1>());
    }
    if (ks < steps) step(ks, std::integral_constant<int, 0>());
    // (the copies requested beyond the end: the buffers are the epilogue's now)
    wait_lds_copies<0>();
    __syncthreads();

    // A lane holds, of its token's row, four neighbouring outputs in each group of four registers.
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
                const long out = (long)(row0 + row) * A.ldo + 32L * block;
                if (kb == 0) store_global((char*)A.out + out / 2, all);
                else *(DYMOE_GLOBAL uint8_t*)(A.out_scale + out / 32) = (uint8_t)byte;
            }
        }
    } else {
        // the wavefront turns a fragment round in an LDS area of its own, so that a row leaves in whole lines
        const uint32_t area = base + (uint32_t)wave * kMx4EpiWave, wr = area + (uint32_t)ln * kMx4EpiRow + (uint32_t)kb * 16u;
        const bool vec = MODE != kMx4Plain || A.aligned;
        const int dt = MODE == kMx4Plain ? A.out_dtype : DYMOE_OUT_F32;
#pragma unroll
        for (int s = 0; s < S; s++) {
            const int n = ((4 * bx + wave) * S + s) * 32 + 4 * (lane & 7), left = A.N - n;
            float add[4] = {0.f, 0.f, 0.f, 0.f};
            if (MODE == kMx4Plain && A.bias) {
#pragma unroll
                for (int i = 0; i < 4; i++) add[i] = A.bias[min(n + i, A.N - 1)];
            }
#pragma unroll
            for (int f = 0; f < NTF; f++) {
#pragma unroll
                for (int g = 0; g < 4; g++)
                    lds_write16(wr + 32u * g, make_uint4(__float_as_uint(acc[s][f][4 * g]), __float_as_uint(acc[s][f][4 * g + 1]),
                                                         __float_as_uint(acc[s][f][4 * g + 2]), __float_as_uint(acc[s][f][4 * g + 3])));
                // (a wavefront's LDS accesses execute in order and the area is its own: no barrier)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int rr = (lane >> 3) + 8 * j, row = 32 * f + rr;
                    const uint4 u = lds_read16(area + (uint32_t)rr * kMx4EpiRow + (uint32_t)(lane & 7) * 16u);
                    if (row >= rows || left <= 0) continue;
                    const float v[4] = {__uint_as_float(u.x) + add[0], __uint_as_float(u.y) + add[1], __uint_as_float(u.z) + add[2], __uint_as_float(u.w) + add[3]};
                    store_out4(A.out, (long)(row0 + row) * A.ldo + n, dt, left >= 4 && vec, left, v);
                }
            }
        }
    }
}

// Neighbouring units that an XCD takes at a time: workgroups go to the 8 XCDs, each with an L2 of its own, in turn, and units that read the same
// weights (the tiles of a matrix or expert, for one column block) are neighbours.
constexpr int kMx4Run = 8;
__device__ __forceinline__ long mx4_unit_of_group() { return ((long)(blockIdx.x >> 3) / kMx4Run * 8 + (blockIdx.x & 7)) * kMx4Run + (blockIdx.x >> 3) % kMx4Run; }
static dim3 mx4_grid(long units) { return dim3((unsigned)(((units + kMx4Run - 1) / kMx4Run + 7) / 8 * 8 * kMx4Run)); }

__device__ __forceinline__ uint32_t mx4_lds_base(char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)p; }

// weight rows of a workgroup's block: of the up projection, those of W1
template <int MODE, int S>
constexpr int kMx4Cols = 128 * (MODE == kMx4Up ? S / 2 : S);

template <int MODE, int MAXF, int S>
__global__ __launch_bounds__(256, MAXF * S <= 8 ? 2 : 1) void mx4_tall_kernel(const Mx4Args A)
{
    extern __shared__ __attribute__((aligned(1024))) char lds_raw[];
    const uint32_t base = mx4_lds_base(lds_raw);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    constexpr int kCols = kMx4Cols<MODE, S>, kRows = 32 * MAXF;
    const int strips = (A.N + 31) / 32, nblk = (int)(((MODE == kMx4Up ? A.ldo : A.N) + kCols - 1) / kCols);
    const Mx4Plan pp = expert_plan<dymoe_expert_mx4>(const_cast<int32_t*>(A.plan), A.P);
    const long unit = mx4_unit_of_group();
    Mx4Weights<S> w;
    int row0, rows, bx;
    if (MODE == kMx4Plain) {
        const int tiles = (A.rows + kRows - 1) / kRows;
        if (unit >= (long)tiles * nblk) return;
        bx = (int)(unit / tiles);
        row0 = (int)(unit - (long)bx * tiles) * kRows;
        rows = min(kRows, A.rows - row0);
#pragma unroll
        for (int s = 0; s < S; s++) w.strip[s].set(A.w, A.ws, (4L * bx + wave) * S + s, strips, A.Kp);
    } else {
        if (unit >= (long)pp.meta[0] * nblk) return;
        const ExpertTile<dymoe_expert_mx4> t = pp.tiles[unit / nblk];
        const long local = unit - (long)t.tile0 * nblk;
        bx = (int)(local / t.tiles);
        const int i = (int)(local - (long)bx * t.tiles) * kRows;
        row0 = t.first + i;
        rows = min(kRows, t.pairs - i);
#pragma unroll
        for (int s = 0; s < S; s++) {
            if (MODE == kMx4Up) w.strip[s].set(s & 1 ? t.mat.q[1] : t.mat.q[0], s & 1 ? t.mat.s[1] : t.mat.s[0], (4L * bx + wave) * (S / 2) + s / 2, strips, A.Kp);
            else w.strip[s].set(t.mat.q[2], t.mat.s[2], (4L * bx + wave) * S + s, strips, A.Kp);
        }
    }
    // one instantiation per number of fragments of 32 rows: the accumulators then sit in fixed registers for the whole loop
#define DYMOE_MX4_TILE(NTF) mx4_tile<MODE, NTF, S>(A, pp.perm, w, row0, rows, bx, base)
    switch ((rows + 31) >> 5) {
    case 1: DYMOE_MX4_TILE(1); break;
    case 2: DYMOE_MX4_TILE(2); break;
    case 3: DYMOE_MX4_TILE(3); break;
    default: DYMOE_MX4_TILE(MAXF); break;
    }
#undef DYMOE_MX4_TILE
}

template <int MAXF>
constexpr int kMx4Lds = 3 * kMx4Buf<MAXF>;
static_assert(4 * kMx4EpiWave <= 3 * kMx4Buf<4>, "the epilogue areas fit in the buffers of a whole tile");

// per-device set-up, with the device current
int mx4_init()
{
    auto allow = [](const void* f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess; };
    const bool ok = allow((const void*)mx4_tall_kernel<kMx4Plain, 4, 2>, kMx4Lds<4>) && allow((const void*)mx4_tall_kernel<kMx4Up, 4, 2>, kMx4Lds<4>) &&
                    allow((const void*)mx4_tall_kernel<kMx4Down, 4, 2>, kMx4Lds<4>);
    return ok ? DYMOE_OK : DYMOE_EHIP;
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
    const long groups = (T + 31L) / 32 * ((N + 31L) / 32);
    if (!fits_grid(groups, 512)) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    Mx4Args A = {};
    A.x = (const char*)x;
    A.xs = (const char*)x_scale;
    if (!coded) {
        const int rc = mx4_quantize(ctx, x, x_dtype, T, K, ldx, 0, (uint8_t*)ws + L.xq, (uint8_t*)ws + L.xs, st);
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
    A.aligned = dymoe_aligned(y, 4 * dtype_bytes(out_dtype)) && ldy % 4 == 0;
    if (T > 64)
        dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_tall_kernel<kMx4Plain, 4, 2>, mx4_grid((T + 127L) / 128 * ((N + 255L) / 256)), dim3(256), kMx4Lds<4>, st, A);
    else
        dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_small_kernel<kMx4Plain, 1, 8, 1>, dim3((unsigned)groups), dim3(512), 0, st, A);
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
    const long up = (long)L.max_tiles * (long)(L.Fp / 32), down = (long)L.max_tiles * ((H + 31L) / 32);
    if (!fits_grid(up, 512) || !fits_grid(down, 512) || !fits_grid(T * ((H + 2047L) / 2048), 256)) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    int32_t* const plan = (int32_t*)(ws + L.plan);
    const int per_row = (int)((L.Hp + 511) / 512);
    const long units = (long)T * per_row;
    const dim3 grid((unsigned)(1 + (units + 15) / 16));
    auto prep = mx4_prep_kernel<DYMOE_OUT_BF16>;
    if (x_dtype == DYMOE_OUT_F32) prep = mx4_prep_kernel<DYMOE_OUT_F32>;
    else if (x_dtype == DYMOE_OUT_F16) prep = mx4_prep_kernel<DYMOE_OUT_F16>;
    const int small = T <= 32 || P <= 20L * E;
    const long tall = P / kMx4TallRows + (E < P ? E : P);
    dymoe_launch(ctx, DYMOE_K_MX4_ROWS, prep, grid, dim3(kPlanThreads), 0, st, idx, table, P, E, small, plan, ctx->device_flags, (const char*)x,
                 units, per_row, H, ws + L.xq, ws + L.xs);
    Mx4Args A = {};
    A.x = ws + L.xq;
    A.xs = ws + L.xs;
    A.plan = plan;
    A.out = ws + L.hq;
    A.out_scale = (uint8_t*)ws + L.hs;
    A.ldo = (long)L.Fp;
    A.P = P;
    A.Kp = (int)L.Hp;
    A.N = F;
    A.k = k;
    A.rows = T;
    if (small) dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_small_kernel<kMx4Up, 1, 8, 1>, dim3((unsigned)up), dim3(512), 0, st, A);
    else dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_tall_kernel<kMx4Up, 4, 2>, mx4_grid(tall * (long)(L.Fp / 128)), dim3(256), kMx4Lds<4>, st, A);
    A.x = ws + L.hq;
    A.xs = ws + L.hs;
    A.out = ws + L.part;
    A.ldo = (long)mx4_round((size_t)H, 8);
    A.Kp = (int)L.Fp;
    A.N = H;
    if (small) dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_small_kernel<kMx4Down, 1, 8, 1>, dim3((unsigned)down), dim3(512), 0, st, A);
    else dymoe_launch(ctx, DYMOE_K_MX4_PRODUCT, mx4_tall_kernel<kMx4Down, 4, 2>, mx4_grid(tall * ((H + 255L) / 256)), dim3(256), kMx4Lds<4>, st, A);
    experts_combine(ctx, DYMOE_K_MX4_ROWS, (const float*)(ws + L.part), A.ldo, expert_plan<dymoe_expert_mx4>(plan, P).where, w, T, H, k, out_dtype,
                    y, st);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
