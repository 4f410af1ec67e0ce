// Rows to the microscaled 4-bit format and back.
//
// a = max |x| of 32 columns, e = floor(log2 a) - 2, code = x / 2^e to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  A stream of bytes: 2 read and
// 17 / 32 written a value (bf16 or fp16).  Four neighbouring lanes share a block, so nothing leaves the vector unit and every value is read once.
// 8191 x 14336 bf16: to rows 51 us (5.8 TB/s), to tiles 53; back 61 and 55.
#include "mx4_device.hpp"

namespace dymoe {

// A lane takes 8 columns at a time.  Row by row a wavefront takes 512 neighbouring columns of a row at once, in tiles 8 rows by 64 columns: a
// chunk's 8 rows are then 128 bytes that lie together.
template <int TILES>
struct Mx4Spread {
    long row, col;        // of this lane's first 8 columns
    static constexpr int kRows = TILES ? 8 : 1, kCols = TILES ? 64 : 512;
    // unit: kRows rows by CH * kCols columns
    __device__ __forceinline__ Mx4Spread(long unit, int per_row, int cols)
    {
        const int lane = threadIdx.x & (kWave - 1);
        const long r = unit / per_row;
        row = r * kRows + (TILES ? lane >> 3 : 0);
        col = (unit - r * per_row) * cols + (TILES ? lane & 7 : lane) * 8;
    }
};

template <int DT, int TILES, int CH>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const char* __restrict__ x, long rows, int K, long ldx, long out_rows, long units,
                                                           int per_row, uint8_t* __restrict__ codes, uint8_t* __restrict__ scale)
{
    using S = Mx4Spread<TILES>;
    const long unit = (long)blockIdx.x * 4 + threadIdx.x / kWave;
    if (unit >= units) return;
    const int Kp = (int)up_to(K, 256);
    const S at(unit, per_row, CH * S::kCols);
    const char* const src = x + at.row * ldx * dtype_bytes(DT);
    const int real = at.row < rows ? K : 0;               // (tiles end with whole strips: rows behind the last are zero)
    Raw8<DT> v[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) v[c] = load8<DT>(src, at.col + c * S::kCols, real);
    uint32_t bytes = 0;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const long col = at.col + c * S::kCols;
        const uint32_t byte = mx4_exponent(quad_max_u32(peak_f32_bits<DT>(peak8<DT>(v[c], 0u))));
        const uint32_t q = mx4_codes8<DT>(v[c], byte);
        if (TILES) bytes |= byte << (8 * c);
        if (col >= Kp || at.row >= out_rows) continue;
        *(DYMOE_GLOBAL uint32_t*)(codes + (TILES ? mx4_tile_byte(at.row, col, Kp) : (at.row * Kp + col) / 2)) = q;
        if (!TILES && (col & 31) == 0) *(DYMOE_GLOBAL uint8_t*)(scale + (at.row * Kp + col) / 32) = (uint8_t)byte;
    }
    if constexpr (TILES) {
        // four lanes hold the exponents of blocks 0 and 2 of half a row of the tile, the four beside them 1 and 3: a word
        static_assert(CH * S::kCols == 128, "half a tile at a time");
        const int lane = threadIdx.x & (kWave - 1);
        const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)bytes, 0x141, 0xF, 0xF, true);       // row_half_mirror: from the four beside
        if ((lane & 7) == 0 && at.row < out_rows)
            *(DYMOE_GLOBAL uint32_t*)(scale + mx4_tile_exponent(at.row, at.col, Kp)) = __builtin_amdgcn_perm(other, bytes, 0x05010400u);
    }
}

// code number i of eight, times the unit: exact in fp32
__device__ __forceinline__ float mx4_value(uint32_t q, int i, float unit, bool number)
{
    const uint32_t c = q >> (4 * i), m = c & 7;
    // 0.5 is the one subnormal number; the others' two exponent bits count from 2^0 on
    const float v = m < 2 ? 0.5f * (float)m : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1u) << 22);
    const float s = c & 8 ? -v : v;
    return number ? s * unit : __builtin_nanf("");
}

// eight values of a row, `left` of them inside it (a stream that this kernel does not read again: non-temporal, 8191 rows of 14336 53 us and 70)
template <int DT>
__device__ __forceinline__ void mx4_store8(void* y, long at, int left, const float (&v)[8])
{
    if (left < 8) {
#pragma unroll
        for (int i = 0; i < 7; i++)
            if (i < left) store_out(y, at + i, DT, v[i]);
        return;
    }
    if constexpr (DT == DYMOE_OUT_F32) {
#pragma unroll
        for (int i = 0; i < 8; i += 4)
            __builtin_nontemporal_store(any16_t{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])},
                                        (DYMOE_GLOBAL any16_t*)((float*)y + at + i));
    } else {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (DT == DYMOE_OUT_F16) u[i] = pack_half2(v[2 * i], v[2 * i + 1]);
            else {
                const bf16x2_t b = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
                u[i] = __builtin_bit_cast(uint32_t, b);
            }
        }
        __builtin_nontemporal_store(any16_t{u[0], u[1], u[2], u[3]}, (DYMOE_GLOBAL any16_t*)((uint16_t*)y + at));
    }
}

template <int DT, int TILES, int CH>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale, long rows, int K,
                                                             long units, int per_row, void* __restrict__ y, long ldy)
{
    using S = Mx4Spread<TILES>;
    const long unit = (long)blockIdx.x * 4 + threadIdx.x / kWave;
    if (unit >= units) return;
    const int Kp = (int)up_to(K, 256);
    const S at(unit, per_row, CH * S::kCols);
    if (at.row >= rows) return;
    uint32_t q[CH], e[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const long col = at.col + c * S::kCols;
        if (col >= K) continue;
        q[c] = *(const DYMOE_GLOBAL uint32_t*)(codes + (TILES ? mx4_tile_byte(at.row, col, Kp) : (at.row * Kp + col) / 2));
        e[c] = *(const DYMOE_GLOBAL uint8_t*)(scale + (TILES ? mx4_tile_exponent(at.row, col, Kp) : (at.row * Kp + col) / 32));
    }
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const long col = at.col + c * S::kCols;
        if (col >= K) continue;
        const float unit2 = mx4_unit(e[c]);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = mx4_value(q[c], i, unit2, e[c] != 255u);
        mx4_store8<DT>(y, at.row * ldy + col, (int)(K - col), v);
    }
}

// wavefronts of a launch at most: 64 threads each stay below the 2^32 of a grid
constexpr long kMx4Units = 1L << 25;

// rows of a launch: whole strips
static long mx4_rows_launch(long rows, int tiles, int per_row)
{
    const long n = kMx4Units / per_row * (tiles ? 8 : 1) / 32 * 32;
    return rows < n ? rows : n;
}

template <int DT, int TILES>
static int mx4_quantize_launch(dymoe_ctx* ctx, const void* x, long rows, long K, long ldx, uint8_t* codes, uint8_t* scale, hipStream_t st)
{
    constexpr int CH = 2;        // (in tiles, 61 x 2048 3.0 us and 3.6 with four, 8191 x 14336 52 and 56)
    using S = Mx4Spread<TILES>;
    const long Kp = up_to(K, 256);
    const int per_row = (int)((Kp + CH * S::kCols - 1) / (CH * S::kCols));
    const long step = mx4_rows_launch(rows, TILES, per_row);
    for (long r = 0; r < rows; r += step) {
        const long n = rows - r < step ? rows - r : step, out = TILES ? up_to(n, 32) : n, units = (out + S::kRows - 1) / S::kRows * per_row;
        dymoe_launch(ctx, DYMOE_K_MX4_ROWS, mx4_quantize_kernel<DT, TILES, CH>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st,
                     (const char*)x + r * ldx * dtype_bytes(DT), n, (int)K, ldx, out, units, per_row, codes + r * Kp / 2, scale + r * Kp / 32);
    }
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

int mx4_quantize(dymoe_ctx* ctx, const void* x, int dtype, long rows, long K, long ldx, int tiles, uint8_t* codes, uint8_t* scale, hipStream_t st)
{
    auto launch = tiles ? mx4_quantize_launch<DYMOE_OUT_BF16, 1> : mx4_quantize_launch<DYMOE_OUT_BF16, 0>;
    if (dtype == DYMOE_OUT_F32) launch = tiles ? mx4_quantize_launch<DYMOE_OUT_F32, 1> : mx4_quantize_launch<DYMOE_OUT_F32, 0>;
    else if (dtype == DYMOE_OUT_F16) launch = tiles ? mx4_quantize_launch<DYMOE_OUT_F16, 1> : mx4_quantize_launch<DYMOE_OUT_F16, 0>;
    return launch(ctx, x, rows, K, ldx, codes, scale, st);
}

template <int DT, int TILES>
static int mx4_dequantize_launch(dymoe_ctx* ctx, const uint8_t* codes, const uint8_t* scale, long rows, long K, void* y, long ldy, hipStream_t st)
{
    constexpr int CH = TILES ? 4 : 2;
    using S = Mx4Spread<TILES>;
    const long Kp = up_to(K, 256);
    const int per_row = (int)((Kp + CH * S::kCols - 1) / (CH * S::kCols));
    const long step = mx4_rows_launch(rows, TILES, per_row);
    for (long r = 0; r < rows; r += step) {
        const long n = rows - r < step ? rows - r : step, units = (n + S::kRows - 1) / S::kRows * per_row;
        dymoe_launch(ctx, DYMOE_K_MX4_ROWS, mx4_dequantize_kernel<DT, TILES, CH>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st,
                     codes + r * Kp / 2, scale + r * Kp / 32, n, (int)K, units, per_row, (char*)y + r * ldy * dtype_bytes(DT), ldy);
    }
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

}  // namespace dymoe

using namespace dymoe;

extern "C" int dymoe_quantize_mx4(dymoe_ctx* ctx, const void* x, int x_dtype, long rows, long K, long ldx, int layout, uint8_t* codes,
                                  uint8_t* scale, void* stream)
{
    DYMOE_REQUIRE(rows >= 0 && K > 0 && ldx >= K);
    DYMOE_REQUIRE(x_dtype == DYMOE_OUT_BF16 || x_dtype == DYMOE_OUT_F32 || x_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(layout == DYMOE_LAYOUT_ROWMAJOR || layout == DYMOE_LAYOUT_TILE);
    if (K > DYMOE_MX4_MAX_K || rows > 0x7fffffe0L) return DYMOE_ENOTSUP;
    if (rows > 0) {
        DYMOE_REQUIRE(x && codes && scale);
        DYMOE_REQUIRE(dymoe_aligned(x, dtype_bytes(x_dtype)) && dymoe_aligned(codes, 16) && dymoe_aligned(scale, 4));
    }
    if (!ctx) return DYMOE_ENOCTX;
    if (rows == 0) return DYMOE_OK;
    return mx4_quantize(ctx, x, x_dtype, rows, K, ldx, layout == DYMOE_LAYOUT_TILE, codes, scale, (hipStream_t)stream);
}

extern "C" int dymoe_dequantize_mx4(dymoe_ctx* ctx, const uint8_t* codes, const uint8_t* scale, long rows, long K, int layout, int out_dtype,
                                    void* y, long ldy, void* stream)
{
    DYMOE_REQUIRE(rows >= 0 && K > 0 && ldy >= K);
    DYMOE_REQUIRE(out_dtype == DYMOE_OUT_BF16 || out_dtype == DYMOE_OUT_F32 || out_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(layout == DYMOE_LAYOUT_ROWMAJOR || layout == DYMOE_LAYOUT_TILE);
    if (K > DYMOE_MX4_MAX_K || rows > 0x7fffffe0L) return DYMOE_ENOTSUP;
    if (rows > 0) {
        DYMOE_REQUIRE(y && codes && scale);
        DYMOE_REQUIRE(dymoe_aligned(y, dtype_bytes(out_dtype)) && dymoe_aligned(codes, 16) && dymoe_aligned(scale, 4));
    }
    if (!ctx) return DYMOE_ENOCTX;
    if (rows == 0) return DYMOE_OK;
    const bool tiles = layout == DYMOE_LAYOUT_TILE;
    auto launch = tiles ? mx4_dequantize_launch<DYMOE_OUT_BF16, 1> : mx4_dequantize_launch<DYMOE_OUT_BF16, 0>;
    if (out_dtype == DYMOE_OUT_F32) launch = tiles ? mx4_dequantize_launch<DYMOE_OUT_F32, 1> : mx4_dequantize_launch<DYMOE_OUT_F32, 0>;
    else if (out_dtype == DYMOE_OUT_F16) launch = tiles ? mx4_dequantize_launch<DYMOE_OUT_F16, 1> : mx4_dequantize_launch<DYMOE_OUT_F16, 0>;
    return launch(ctx, codes, scale, rows, K, y, ldy, (hipStream_t)stream);
}
