// Dynamic 8-bit quantisation of rows (tokens, or the channels of a weight matrix), one scale a row.
//
// a = max |x|, scale = a / 127, code = rint(127 x / a).  A stream of bytes: 2 read and 1 written a value (bf16 or fp16).  A row stays in
// the registers of the threads that share it between the search for its largest value and its codes, so it is read once.  A wavefront
// takes a row of up to 2048 values where the rows are many; with few rows, or longer ones, the four wavefronts of a workgroup share
// one, and beyond 16384 values sixteen.  8191 rows of 14336 in bf16 65 us, 5.4 TB/s, what a copy of a GiB reaches on this card (5.2 to
// 5.5); 24 rows of 4096 2.6 us, a launch's latencies.
#include "int8_device.hpp"

namespace dymoe {

// byte of a tile-layout matrix that holds code (row, col), col a multiple of 8: see dymoe_expert_fmt, 8 bits
__device__ __forceinline__ long tile_byte(long row, long col, long Kp)
{
    const long tile = (row >> 5) * (Kp >> 7) + (col >> 7);
    const int in = (int)(col & 127);
    return tile * 4096 + ((in & 63) >> 4) * 1024 + ((in >> 6) * 32 + (row & 31)) * 16 + (in & 15);
}

template <int DT, int WAVES, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void quantize_rows_kernel(const char* __restrict__ x, long rows, long K, long ldx,
                                                                                      int tiles, long out_rows, char* __restrict__ codes,
                                                                                      float* __restrict__ scale)
{
    constexpr int kRows = WAVES == 1 ? 4 : 1;             // rows a workgroup takes
    __shared__ uint32_t s_max[WAVES];
    const int wave = threadIdx.x / kWave;
    const long row = (long)blockIdx.x * kRows + (WAVES == 1 ? wave : 0);
    const int t = WAVES == 1 ? (threadIdx.x & (kWave - 1)) : threadIdx.x;
    if (row >= out_rows) return;
    const long Kp = up_to(K, 128);
    const char* const src = x + row * ldx * dtype_bytes(DT);
    const bool real = row < rows;                         // (tiles end with whole strips: rows behind the last are zero)
    Raw8<DT> v[CH];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const long col = (long)(c * 64 * WAVES + t) * 8;
        v[c] = load8<DT>(src, col, real ? K : 0);
    }
#pragma unroll
    for (int c = 0; c < CH; c++) m = peak8<DT>(v[c], m);
    m = wave_max_u32(peak_bits<DT>(m));
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & (kWave - 1)) == 0) s_max[wave] = m;
        __syncthreads();
        m = s_max[0];
#pragma unroll
        for (int w = 1; w < WAVES; w++) m = max(m, s_max[w]);
    }
    float sc;
    const RowQ q = row_q(peak_value<DT>(m), sc);
    if (real && t == 0) scale[row] = sc;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const long col = (long)(c * 64 * WAVES + t) * 8;
        if (col < Kp) {
            const long at = tiles ? tile_byte(row, col, Kp) : row * Kp + col;
            store_global(codes + at, codes8<DT>(v[c], q));
        }
    }
}

template <int DT>
static int quantize_rows_launch(dymoe_ctx* ctx, const void* x, long rows, long K, long ldx, int tiles, void* codes, float* scale, hipStream_t st)
{
    const long out_rows = tiles ? up_to(rows, 32) : rows, Kp = up_to(K, 128);
#define DYMOE_QROWS(WAVES, CH)                                                                                                  \
    dymoe_launch(ctx, DYMOE_K_QUANTIZE_ROWS, quantize_rows_kernel<DT, WAVES, CH>,                                               \
                 dim3((unsigned)(WAVES == 1 ? (out_rows + 3) / 4 : out_rows)), dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, st,      \
                 (const char*)x, rows, K, ldx, tiles, out_rows, (char*)codes, scale)
    // A wavefront a row of up to 2048 values once there are eight for a compute unit, else a workgroup a row: 2048 rows of 768 3.4 us and 4.1, of
    // 2048 4.0 / 4.5, 16384 rows 8.4 / 14.1 and 16.9 / 18.0; 512 rows 4.5 / 4.1 and 3.4 / 3.0.  Rows of 4096 are a workgroup's at any number: 65536
    // of them 137 us, by a wavefront each 147.
    const bool many = out_rows >= 8L * ctx->num_cu;
    if (Kp <= 512) DYMOE_QROWS(1, 1);
    else if (Kp <= 1024 && many) DYMOE_QROWS(1, 2);
    else if (Kp <= 2048 && many) DYMOE_QROWS(1, 4);
    else if (Kp <= 2048) DYMOE_QROWS(4, 1);
    else if (Kp <= 4096) DYMOE_QROWS(4, 2);
    else if (Kp <= 8192) DYMOE_QROWS(4, 4);
    else if (Kp <= 16384) DYMOE_QROWS(4, 8);
    else if (Kp <= 32768) DYMOE_QROWS(16, 4);
    else if (Kp <= 65536) DYMOE_QROWS(16, 8);
    else DYMOE_QROWS(16, 16);
#undef DYMOE_QROWS
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

// rows of a launch at most: 1024 threads a row stay below the 2^32 of a grid
constexpr long kRowsLaunch = 1L << 21;

int quantize_rows(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, void* codes, float* scale, hipStream_t st)
{
    auto launch = quantize_rows_launch<DYMOE_OUT_BF16>;
    if (dtype == DYMOE_OUT_F32) launch = quantize_rows_launch<DYMOE_OUT_F32>;
    else if (dtype == DYMOE_OUT_F16) launch = quantize_rows_launch<DYMOE_OUT_F16>;
    for (long r = 0; r < rows; r += kRowsLaunch) {
        const long n = rows - r < kRowsLaunch ? rows - r : kRowsLaunch;
        const int rc = launch(ctx, (const char*)x + r * ldx * dtype_bytes(dtype), n, K, ldx, tiles, (char*)codes + r * up_to(K, 128), scale + r, st);
        if (rc != DYMOE_OK) return rc;
    }
    return DYMOE_OK;
}

}  // namespace dymoe

extern "C" int dymoe_quantize_rows(dymoe_ctx* ctx, const void* x, int x_dtype, long rows, long K, long ldx, int layout, int8_t* codes,
                                   float* scale, void* stream)
{
    DYMOE_REQUIRE(rows >= 0 && K > 0 && ldx >= K);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(layout == DYMOE_LAYOUT_ROWMAJOR || layout == DYMOE_LAYOUT_TILE);
    if (K > DYMOE_INT8_MAX_K || rows > 0x7fffffe0L) return DYMOE_ENOTSUP;
    if (rows > 0) {
        DYMOE_REQUIRE(x && codes && scale);
        DYMOE_REQUIRE(dymoe_aligned(x, dymoe::dtype_bytes(x_dtype)) && dymoe_aligned(codes, 16) && dymoe_aligned(scale, 4));
    }
    if (!ctx) return DYMOE_ENOCTX;
    if (rows == 0) return DYMOE_OK;
    return dymoe::quantize_rows(ctx, x, x_dtype, rows, K, ldx, layout == DYMOE_LAYOUT_TILE, codes, scale, (hipStream_t)stream);
}
