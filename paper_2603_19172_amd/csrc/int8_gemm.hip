// Products in 8-bit integers with a scale for each token and each channel: a matrix (dymoe_matmul_int8) and a layer's SwiGLU
// experts (dymoe_moe_ffn_int8).
//   y[t, n] = xs[t] ws[n] sum_k xq[t, k] wq[n, k]
// The sums are whole numbers of 32 bits (127 * 127 * K < 2^31 up to K = 131072), so their order does not matter and every split of K gives
// the same bits.
#include <float.h>

#include "int8_device.hpp"
#include "int8_layout.hpp"

namespace dymoe {

int quantize_rows(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, void* codes, float* scale, hipStream_t st);

struct I8Plan {
    int32_t* offsets;     // [E + 1] first position of each expert
    int32_t* meta;        // [8]: tiles
    int32_t* perm;        // [P] position -> pair
    int32_t* where;       // [P] pair -> position, -1: left out
    int32_t* tiles;       // [4 max_tiles]: expert, first position, rows, unused
};

__host__ __device__ inline I8Plan i8_plan(int32_t* p, int E, long P)
{
    I8Plan r;
    r.offsets = p;
    r.meta = r.offsets + E + 1;
    r.perm = r.meta + 8;
    r.where = r.perm + P;
    r.tiles = r.where + P;
    return r;
}

__device__ __forceinline__ bool i8_present(const dymoe_expert_i8& x)
{
    return (x.q[0] != nullptr) & (x.q[1] != nullptr) & (x.q[2] != nullptr) & (x.s[0] != nullptr) & (x.s[1] != nullptr) & (x.s[2] != nullptr);
}

// Counting sort of the pairs by expert and the list of tiles, by one workgroup.
constexpr int kI8PlanThreads = 1024;

__global__ __launch_bounds__(kI8PlanThreads) void i8_plan_kernel(const int32_t* __restrict__ idx, const dymoe_expert_i8* __restrict__ table,
                                                                 long P, int E, int tile_rows, int32_t* __restrict__ plan,
                                                                 unsigned* __restrict__ flags)
{
    __shared__ int s_count[DYMOE_MAX_EXPERTS], s_at[DYMOE_MAX_EXPERTS], s_wave[2][kI8PlanThreads / kWave];
    __shared__ int s_held[DYMOE_MAX_EXPERTS];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const I8Plan pp = i8_plan(plan, E, P);
    if (tid < E) {
        s_count[tid] = 0;
        s_held[tid] = i8_present(table[tid]);
    }
    __syncthreads();
    for (long p = tid; p < P; p += kI8PlanThreads) {
        const int e = idx[p];
        if ((unsigned)e < (unsigned)E) atomicAdd(&s_count[e], 1);
    }
    __syncthreads();
    int n = tid < E ? s_count[tid] : 0;
    if (n > 0 && !s_held[tid]) {
        atomicOr(flags, DYMOE_FLAG_FORMAT_MISSING);
        n = 0;
    }
    const int tiles = (n + tile_rows - 1) / tile_rows;
    const int n_in = wave_scan_dpp_i32(n), t_in = wave_scan_dpp_i32(tiles);
    if (lane == kWave - 1) {
        s_wave[0][wave] = n_in;
        s_wave[1][wave] = t_in;
    }
    __syncthreads();
    int n0 = n_in - n, t0 = t_in - tiles;
    for (int w = 0; w < wave; w++) {
        n0 += s_wave[0][w];
        t0 += s_wave[1][w];
    }
    if (tid < E) {
        s_at[tid] = n0;
        pp.offsets[tid] = n0;
        if (tid == E - 1) pp.offsets[E] = n0 + n;
        for (int i = 0; i < tiles; i++) {
            int32_t* const t = pp.tiles + 4L * (t0 + i);
            t[0] = tid;
            t[1] = n0 + i * tile_rows;
            t[2] = min(tile_rows, n - i * tile_rows);
        }
    }
    if (tid == kI8PlanThreads - 1) pp.meta[0] = t0 + tiles;
    __syncthreads();
    // (an expert's pairs come in any order: nothing that is computed depends on it)
    for (long p = tid; p < P; p += kI8PlanThreads) {
        const int e = idx[p];
        int at = -1;
        if ((unsigned)e < (unsigned)E && s_held[e]) {
            at = atomicAdd(&s_at[e], 1);
            pp.perm[at] = (int32_t)p;
        }
        pp.where[p] = at;
    }
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
    const dymoe_expert_i8* table;
    I8Mat w;                          // the plain product
    const float* bias;
    void* out;
    long ldo, P;
    int rows, Kp, N, E, k, out_dtype;
};

enum { kI8Plain = 0, kI8Up = 1, kI8Down = 2 };

__device__ __forceinline__ i32x16_t mfma_i8(const uint4 a, const uint4 b, const i32x16_t c)
{
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ float silu_times(float a, float u) { return a * __builtin_amdgcn_rcpf(1.0f + __expf(-a)) * u; }

// Tiles of one fragment (up to 32 rows): the four wavefronts of a workgroup share two strips of 32 weight rows and split K.  Nothing is
// shared before the end: weights and rows come straight into registers.
template <int MODE>
__global__ __launch_bounds__(256) void i8_small_kernel(const I8Args A)
{
    __shared__ __attribute__((aligned(16))) int s_red[4 * 2 * 16 * kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int ln = lane & 31, kb = lane >> 5;
    const int cols = MODE == kI8Up ? 32 : 64;
    const int nblk = (A.N + cols - 1) / cols;
    const int tile = blockIdx.x / nblk, bx = blockIdx.x - tile * nblk;
    int row0, rows;
    const char *qa, *qb;
    const float *sa, *sb;
    const I8Plan pp = i8_plan(const_cast<int32_t*>(A.plan), A.E, A.P);
    const long strip = 32L * A.Kp;
    const long last = (A.N + 31) / 32 - 1;
    if (MODE == kI8Plain) {
        row0 = tile * kI8TileSmall;
        rows = min(kI8TileSmall, A.rows - row0);
        qa = A.w.q + 2L * bx * strip;
        qb = A.w.q + min(2L * bx + 1, last) * strip;
        sa = sb = A.w.s;
    } else {
        if (tile >= pp.meta[0]) return;
        const int e = pp.tiles[4 * tile];
        row0 = pp.tiles[4 * tile + 1];
        rows = pp.tiles[4 * tile + 2];
        const dymoe_expert_i8 ex = A.table[e];
        if (MODE == kI8Up) {
            qa = (const char*)ex.q[0] + bx * strip;
            qb = (const char*)ex.q[1] + bx * strip;
            sa = ex.s[0];
            sb = ex.s[1];
        } else {
            qa = (const char*)ex.q[2] + 2L * bx * strip;
            qb = (const char*)ex.q[2] + min(2L * bx + 1, last) * strip;
            sa = sb = ex.s[2];
        }
    }
    const int r = min(ln, rows - 1);                  // rows behind the last: computed and dropped
    const long src = MODE == kI8Up ? pp.perm[row0 + r] / A.k : row0 + r;
    const char* const xp = A.x + src * A.Kp + 64 * kb;
    i32x16_t acc[2] = {};
    const int nkt = A.Kp >> 7;
    for (int kt = wave; kt < nkt; kt += 4) {
        uint4 a[4], b[4], t[4];
#pragma unroll
        for (int c = 0; c < 4; c++) {
            a[c] = load_global<uint4>(qa + (long)kt * 4096 + c * 1024 + lane * 16);
            b[c] = load_global<uint4>(qb + (long)kt * 4096 + c * 1024 + lane * 16);
            t[c] = load_global<uint4>(xp + (long)kt * 128 + c * 16);
        }
#pragma unroll
        for (int c = 0; c < 4; c++) {
            acc[0] = mfma_i8(a[c], t[c], acc[0]);
            acc[1] = mfma_i8(b[c], t[c], acc[1]);
        }
    }
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 16; i++) s_red[((wave * 2 + s) * 16 + i) * kWave + lane] = acc[s][i];
    __syncthreads();
    // wavefront w finishes registers 4 w .. 4 w + 3 of both strips: weight rows 8 w + 4 kb + 0 .. 3, token ln
    float v[2][4];
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int* const at = s_red + (s * 16 + 4 * wave + i) * kWave + lane;
            v[s][i] = (float)(at[0] + at[2048] + at[4096] + at[6144]);
        }
    if (ln >= rows) return;
    const float xs = A.xs[src];
    const int n0 = cols * bx + 8 * wave + 4 * kb;
    if (MODE == kI8Up) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int n = n0 + i;
            if (n < A.N) store_out(A.out, (row0 + ln) * A.ldo + n, DYMOE_OUT_BF16, silu_times(v[0][i] * xs * sa[n], v[1][i] * xs * sb[n]));
        }
        return;
    }
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int n = n0 + 32 * s + i;
            if (n >= A.N) continue;
            float o = v[s][i] * xs * sa[n];
            if (MODE == kI8Plain && A.bias) o += A.bias[n];
            store_out(A.out, (long)(row0 + ln) * A.ldo + n, MODE == kI8Plain ? A.out_dtype : DYMOE_OUT_F32, o);
        }
}

// y[t] = sum over the slots, in their order, of gate times the pair's output
__global__ __launch_bounds__(256) void i8_combine_kernel(const float* __restrict__ part, long ldp, const int32_t* __restrict__ where,
                                                         const float* __restrict__ gate, int T, int H, int k, int out_dtype,
                                                         void* __restrict__ y)
{
    const int per = (H + 3) / 4;
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    const long t = i / per;
    const int h = (int)(i - t * per) * 4;
    if (t >= T) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j = 0; j < k; j++) {
        const int at = where[t * k + j];
        if (at < 0) continue;
        const float g = gate[t * k + j];
        const float4 v = load_global<float4>(part + at * ldp + h);
        sum.x = fmaf(g, v.x, sum.x);
        sum.y = fmaf(g, v.y, sum.y);
        sum.z = fmaf(g, v.z, sum.z);
        sum.w = fmaf(g, v.w, sum.w);
    }
    const float o[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int u = 0; u < 4; u++)
        if (h + u < H) store_out(y, t * H + h + u, out_dtype, o[u]);
}

}  // namespace dymoe

using namespace dymoe;

extern "C" size_t dymoe_matmul_int8_workspace_bytes(int T, int N, int K)
{
    if (T < 0 || N <= 0 || K <= 0 || K > DYMOE_INT8_MAX_K) return 0;
    return i8_mat_layout(T, N, K).total;
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
    const I8MatLayout L = i8_mat_layout(T, N, K);
    if (!coded && T > 0 && workspace_bytes < L.total) return DYMOE_ENOSPC;
    const long blocks = ((T + kI8TileSmall - 1L) / kI8TileSmall) * ((N + 63L) / 64);
    if (blocks > 0x7fffffffL) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    I8Args A = {};
    A.x = (const char*)x;
    A.xs = x_scale;
    if (!coded) {
        const int rc = quantize_rows(ctx, x, x_dtype, T, K, ldx, 0, ws + L.xq, (float*)(ws + L.xs), st);
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
    dymoe_launch(ctx, DYMOE_K_MATMUL_INT8, i8_small_kernel<kI8Plain>, dim3((unsigned)blocks), dim3(256), 0, st, A);
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
    if ((long)T * k > 0x7fffffffL / 4) return DYMOE_ENOTSUP;
    const I8FfnLayout L = i8_ffn_layout(T, H, F, E, k);
    if (workspace_bytes < L.total) return DYMOE_ENOSPC;
    const long up = (long)L.max_tiles * ((F + 31L) / 32), down = (long)L.max_tiles * ((H + 63L) / 64);
    if (up > 0x7fffffffL || down > 0x7fffffffL || (long)T * ((H + 3) / 4) > 0x7fffffffL * 256L) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const long P = (long)T * k;
    int rc = quantize_rows(ctx, x, x_dtype, T, H, H, 0, ws + L.xq, (float*)(ws + L.xs), st);
    if (rc != DYMOE_OK) return rc;
    int32_t* const plan = (int32_t*)(ws + L.plan);
    dymoe_launch(ctx, DYMOE_K_INT8_PLAN, i8_plan_kernel, dim3(1), dim3(kI8PlanThreads), 0, st, idx, table, P, E, kI8TileSmall, plan,
                 ctx->device_flags);
    I8Args A = {};
    A.x = ws + L.xq;
    A.xs = (const float*)(ws + L.xs);
    A.plan = plan;
    A.table = table;
    A.out = ws + L.h;
    A.ldo = (long)L.Fp;
    A.P = P;
    A.Kp = (int)L.Hp;
    A.N = F;
    A.E = E;
    A.k = k;
    dymoe_launch(ctx, DYMOE_K_INT8_UP, i8_small_kernel<kI8Up>, dim3((unsigned)up), dim3(256), 0, st, A);
    rc = quantize_rows(ctx, ws + L.h, DYMOE_OUT_BF16, P, F, (long)L.Fp, 0, ws + L.hq, (float*)(ws + L.hs), st);
    if (rc != DYMOE_OK) return rc;
    A.x = ws + L.hq;
    A.xs = (const float*)(ws + L.hs);
    A.out = ws + L.part;
    A.ldo = (long)L.Hp;
    A.Kp = (int)L.Fp;
    A.N = H;
    dymoe_launch(ctx, DYMOE_K_INT8_DOWN, i8_small_kernel<kI8Down>, dim3((unsigned)down), dim3(256), 0, st, A);
    const long items = (long)T * ((H + 3) / 4);
    dymoe_launch(ctx, DYMOE_K_INT8_COMBINE, i8_combine_kernel, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, st,
                 (const float*)(ws + L.part), (long)L.Hp, i8_plan(plan, E, P).where, w, T, H, k, out_dtype, y);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
