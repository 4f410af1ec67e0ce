// The training side of the router that scores (dymoe_route_scored): the balance loss with its counts, and the logits' gradient.
//
// A token's shares p = s / sum s come from fp32 exponentials of differences to its largest logit, so that no scores are too small to be
// divided; with sigmoids u = e^(min(l, 0) - min(m, 0)) / (1 + e^-|l|) is s e^(-min(m, 0)).  One wavefront per token, lane l holding experts l,
// l + 64, ...  Sums over tokens are held in 64 bits and taken in an order that follows from T and E alone.
// Latencies and vector arithmetic, not bytes: 8191 tokens of 256 experts, fp32, loss 6.9 + 5.8 us, gradient 9.8 (16.8 MB: 3.3); 24 of 128 4.6 and 3.9.
#include <float.h>

#include "int8_device.hpp"

namespace dymoe {

constexpr int kBalanceWaves = 8;
constexpr int kBalanceGroups = 256;       // workgroups of the first launch at most
constexpr int kBalanceOne = 32;           // tokens that one workgroup takes, with the loss in the same launch

// e^x, x <= 0 or NaN: the instruction for powers of two of the rounded product, and what the rounding left out as a factor.  Below 2^-126: 0.
__device__ __forceinline__ float exp_neg(float x)
{
    constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;          // their sum: log2 e to 2^-50
    const float y = fmaxf(x, -128.0f), t = y * kLog2e;
    const float p = __builtin_amdgcn_exp2f(t);
    return fmaf(p, kLn2 * fmaf(y, kRest, fmaf(y, kLog2e, -t)), p);
}

template <int DT>
__device__ __forceinline__ float load_logit(const char* logits, long at)
{
    float v;
    if constexpr (DT == DYMOE_OUT_F32) v = ((const DYMOE_GLOBAL float*)logits)[at];
    else if constexpr (DT == DYMOE_OUT_F16) v = (float)((const DYMOE_GLOBAL _Float16*)logits)[at];
    else v = bf16_bits_to_f32(((const DYMOE_GLOBAL uint16_t*)logits)[at]);
    return v;
}

// A masked logit is minus infinity, as dymoe_route_scored has it; NaN goes with the masked ones and is reported.
template <int DT>
__device__ __forceinline__ float masked_logit(float v, bool& bad)
{
    constexpr float lowest = DT == DYMOE_OUT_F32 ? -FLT_MAX : DT == DYMOE_OUT_F16 ? -65504.0f : -0x1.fep127f;
    bad |= v != v;
    return v > lowest ? v : -__builtin_inff();
}

// s e^(-min(m, 0)) of a sigmoid, e^(l - m) of a softmax; rest: 1 - s of a sigmoid, 1 of a softmax
__device__ __forceinline__ float scaled_score(float l, float m, bool sigmoid, float& rest)
{
    const bool masked = l == -__builtin_inff();
    rest = 1.0f;
    if (!sigmoid) return masked ? 0.0f : exp_neg(l - m);
    const float e = exp_neg(-fabsf(l)), one = __builtin_amdgcn_rcpf(1.0f + e);
    rest = masked ? 0.0f : (l > 0.0f ? e : 1.0f) * one;
    return masked ? 0.0f : exp_neg(fminf(l, 0.0f) - fminf(m, 0.0f)) * one;
}

// The scores of a token, up to a common factor, and one over their sum (0 where there are none).  Returns whether one is no number.
template <int NPL, int DT>
__device__ __forceinline__ void load_token(const char* logits, long t, int E, int lane, float (&raw)[NPL])
{
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        const int e = lane + 64 * i;
        raw[i] = e < E ? load_logit<DT>(logits, t * E + e) : -__builtin_inff();
    }
}

template <int NPL, int DT>
__device__ __forceinline__ bool token_scores(const float (&raw)[NPL], bool sigmoid, float (&l)[NPL], float (&u)[NPL], float (&rest)[NPL], float& m,
                                             float& inv)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NPL; i++) l[i] = masked_logit<DT>(raw[i], bad);
    m = l[0];
#pragma unroll
    for (int i = 1; i < NPL; i++) m = fmaxf(m, l[i]);
    m = wave_max_dpp(m);
    bad |= !sigmoid && m == __builtin_inff();
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        u[i] = scaled_score(l[i], m, sigmoid, rest[i]);
        sum += u[i];
    }
    sum = wave_sum(sum);
    inv = sum > 0.0f ? __builtin_amdgcn_rcpf(sum) : 0.0f;
    return __ballot(bad) != 0;
}

constexpr int kBalanceFinish = 1024;      // threads of the second launch

// ONE: the whole call.  Otherwise sums [groups][E] and counts [groups][E + 1] of the workgroup's tokens.
template <int NPL, int DT, bool ONE>
__global__ __launch_bounds__(64 * kBalanceWaves) void route_balance_kernel(const char* __restrict__ logits, const int32_t* __restrict__ idx,
                                                                           const uint8_t* __restrict__ keep, int T, int E, int k, int sigmoid,
                                                                           double* __restrict__ sums, int* __restrict__ often, float coef,
                                                                           int32_t* __restrict__ counts, float* __restrict__ mean,
                                                                           float* __restrict__ loss, int* __restrict__ done)
{
    constexpr int kHalf = kBalanceWaves / 2;
    __shared__ double s_sum[kHalf][64 * NPL < 128 ? 128 : 64 * NPL];
    __shared__ int s_often[64 * NPL + 1 < 512 ? 512 : 64 * NPL + 1];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    for (int e = tid; e <= E; e += blockDim.x) s_often[e] = 0;
    __syncthreads();
    double acc[NPL];
#pragma unroll
    for (int i = 0; i < NPL; i++) acc[i] = 0.0;
    int tokens = 0;
    // the next token's loads are on their way while this one is worked on
    float raw[NPL];
    int chosen = -1, part = 1;
    const long step = (long)gridDim.x * kBalanceWaves;
    auto request = [&](long t) {
        load_token<NPL, DT>(logits, t, E, lane, raw);
        chosen = lane < k ? idx[t * k + lane] : -1;
        part = keep ? keep[t] : 1;
    };
    long t = (long)blockIdx.x * kBalanceWaves + wave;
    if (t < T) request(t);
    for (; t < T; t += step) {
        float now[NPL];
#pragma unroll
        for (int i = 0; i < NPL; i++) now[i] = raw[i];
        const int e = chosen, in = part;
        if (t + step < T) request(t + step);
        if (in == 0) continue;
        if ((unsigned)e < (unsigned)E) atomicAdd(&s_often[e], 1);
        float l[NPL], u[NPL], rest[NPL], m, inv;
        const bool bad = token_scores<NPL, DT>(now, sigmoid, l, u, rest, m, inv);
#pragma unroll
        for (int i = 0; i < NPL; i++) acc[i] += bad ? (double)__builtin_nanf("") : (double)(u[i] * inv);
        tokens++;
    }
    if (lane == 0) atomicAdd(&s_often[E], tokens);
    if (wave >= kHalf) {
#pragma unroll
        for (int i = 0; i < NPL; i++) s_sum[wave - kHalf][lane + 64 * i] = acc[i];
    }
    __syncthreads();
    if (wave < kHalf) {
#pragma unroll
        for (int i = 0; i < NPL; i++) s_sum[wave][lane + 64 * i] += acc[i];
    }
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x) {
        double sum = s_sum[0][e];
#pragma unroll
        for (int w = 1; w < kHalf; w++) sum += s_sum[w][e];
        if (ONE) s_sum[0][e] = sum;
        else sums[(long)blockIdx.x * E + e] = sum;
    }
    if (!ONE) {
        if (blockIdx.x == 0 && tid == 0) *done = 0;       // (for the launch behind this one)
        for (int e = tid; e <= E; e += blockDim.x) often[(long)blockIdx.x * (E + 1) + e] = s_often[e];
        return;
    }
    __syncthreads();
    const int all = s_often[E];
    const double inv = all > 0 ? 1.0 / (double)all : 0.0;
    double term = 0.0;
    for (int e = tid; e <= E; e += blockDim.x) {
        counts[e] = s_often[e];
        if (e == E) continue;
        const double p = s_sum[0][e] * inv;
        mean[e] = (float)p;
        term += (double)s_often[e] * p;
    }
    __syncthreads();
    double* const s_term = &s_sum[0][0];        // (at least 512 of them)
    s_term[tid] = term;
    __syncthreads();
    for (int d = 64 * kBalanceWaves / 2; d > 0; d /= 2) {
        if (tid < d) s_term[tid] += s_term[tid + d];
        __syncthreads();
    }
    if (tid == 0) *loss = (float)((double)coef * (double)E * inv / (double)k * s_term[0]);
}

// Counts, means and the loss from the sums of `groups` workgroups: a workgroup joins them for 32 experts, 32 threads each; the one that comes last adds
// up the workgroups' shares of the loss.  (By one workgroup for all experts, 256 of them and 256 workgroups' sums took 46 us one after
// the other and 14 us eight at a time: its chain of loads.)
__global__ __launch_bounds__(kBalanceFinish) void route_balance_finish_kernel(const double* __restrict__ sums, const int* __restrict__ often, int groups,
                                                                              int E, int k, float coef, int32_t* __restrict__ counts,
                                                                              float* __restrict__ mean, float* __restrict__ loss,
                                                                              double* __restrict__ terms, int* __restrict__ done)
{
    __shared__ double s_sum[32][33];
    __shared__ int s_often[32][33], s_tokens[kBalanceFinish / kWave];
    static_assert(kBalanceGroups <= 8 * 32 && kBalanceFinish == 32 * 32, "eight workgroups' sums a thread");
    const int tid = threadIdx.x, col = tid & 31, slice = tid >> 5, e = blockIdx.x * 32 + col;
    double v[8];
    int n[8], tokens = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int g = slice + 32 * i;
        const bool in = g < groups && e < E;
        v[i] = in ? sums[(long)g * E + e] : 0.0;
        n[i] = in ? often[(long)g * (E + 1) + e] : 0;
    }
    if (tid < groups) tokens = often[(long)tid * (E + 1) + E];
    double sum = v[0];
    int c = n[0];
#pragma unroll
    for (int i = 1; i < 8; i++) {
        sum += v[i];
        c += n[i];
    }
    s_sum[slice][col] = sum;
    s_often[slice][col] = c;
    tokens = wave_sum_dpp_i32(tokens);
    if ((tid & (kWave - 1)) == 0) s_tokens[tid / kWave] = tokens;
    __syncthreads();
    if (tid < kWave) {
        tokens = 0;
        for (int w = 0; w < kBalanceFinish / kWave; w++) tokens += s_tokens[w];
        const double inv = tokens > 0 ? 1.0 / (double)tokens : 0.0;
        double term = 0.0;
        if (tid < 32 && e < E) {
            sum = s_sum[0][col];
            c = s_often[0][col];
            for (int i = 1; i < 32; i++) {
                sum += s_sum[i][col];
                c += s_often[i][col];
            }
            counts[e] = c;
            const double p = sum * inv;
            mean[e] = (float)p;
            term = (double)c * p;
        }
        if (tid == 0 && blockIdx.x == 0) counts[E] = tokens;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) term += __shfl_xor(term, o, kWave);
        if (tid == 0) {
            __hip_atomic_store(&terms[blockIdx.x], term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const bool last = __hip_atomic_fetch_add(done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
            if (last) {
                double all = 0.0;
                for (unsigned w = 0; w < gridDim.x; w++) all += __hip_atomic_load(&terms[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                *loss = (float)((double)coef * (double)E * inv / (double)k * all);
            }
        }
    }
}

// Between a wavefront's LDS accesses that other lanes' are ordered with: nothing to wait for, but the compiler may not carry values across.
__device__ __forceinline__ void lds_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct RouteGradArgs {
    const char* logits;
    const int32_t* idx;
    const float* dw;             // or NULL
    const int32_t* counts;       // or NULL: without the loss
    const float* dloss;          // or NULL: 1
    const uint8_t* keep;
    void* grad;
    int T, E, k, sigmoid, renorm, grad_dtype;
    float factor, coef;
};

// With p the shares, q the chosen experts' shares of their sum and r = 1 - s of a sigmoid (1 of a softmax):
//   the loss:                 r p (g - sum p g),  g = dloss coef E counts / (tokens^2 k)
//   weights, renorm:          factor r q (dw - sum q dw) at the chosen experts
//   weights, without it:      factor s (dw - sum s dw) (softmax), factor s (1 - s) dw (sigmoid)
template <int NPL, int DT>
__global__ __launch_bounds__(256) void route_grad_kernel(const RouteGradArgs A)
{
    __shared__ float s_area[4][64 * NPL];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, E = A.E, k = A.k;
    const bool sigmoid = A.sigmoid;
    float g[NPL];
#pragma unroll
    for (int i = 0; i < NPL; i++) g[i] = 0.0f;
    if (A.counts) {
        const float tokens = (float)A.counts[E];
        const float c = tokens > 0.0f ? (A.dloss ? *A.dloss : 1.0f) * A.coef * (float)E / tokens / (tokens * (float)k) : 0.0f;
#pragma unroll
        for (int i = 0; i < NPL; i++) g[i] = lane + 64 * i < E ? c * (float)A.counts[lane + 64 * i] : 0.0f;
    }
    for (long t = (long)blockIdx.x * 4 + wave; t < A.T; t += (long)gridDim.x * 4) {
        float raw[NPL], l[NPL], u[NPL], rest[NPL], m, inv;
        load_token<NPL, DT>(A.logits, t, E, lane, raw);
        // (a slot's loads are on their way beside them)
        int e = -1;
        float dw = 0.0f, x = -__builtin_inff();
        bool ignored = false;
        if (A.dw && lane < k) {
            e = A.idx[t * k + lane];
            dw = A.dw[t * k + lane];
            if ((unsigned)e >= (unsigned)E) e = -1;
            else x = masked_logit<DT>(load_logit<DT>(A.logits, t * E + e), ignored);
        }
        bool bad = token_scores<NPL, DT>(raw, sigmoid, l, u, rest, m, inv);
        float out[NPL];
#pragma unroll
        for (int i = 0; i < NPL; i++) out[i] = 0.0f;
        const bool part = A.counts && (!A.keep || A.keep[t] != 0);
        if (part) {
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; i++) dot = fmaf(u[i] * inv, g[i], dot);
            dot = wave_sum(dot);
#pragma unroll
            for (int i = 0; i < NPL; i++) out[i] = u[i] * inv * (g[i] - dot);
        }
        if (A.dw) {
            float v, row = 0.0f, unused;
            if (A.renorm) {
                const float top = wave_max_dpp(x), s = scaled_score(x, top, sigmoid, unused), sum = wave_sum(s);
                const float q = sum > 0.0f ? s / sum : 0.0f;
                const float dot = wave_sum(q != 0.0f ? q * dw : 0.0f);
                v = q != 0.0f ? A.factor * (q * (dw - dot)) : 0.0f;
            } else if (sigmoid) {
                v = x > -__builtin_inff() ? A.factor * (scaled_score(x, 0.0f, true, unused) * dw) : 0.0f;
            } else {
                const float s = scaled_score(x, m, false, unused) * inv;
                const float one = s != 0.0f ? s * dw : 0.0f;
                v = A.factor * one;
                row = A.factor * wave_sum(one);
            }
            // To the lanes that hold the experts, through an LDS area of the wavefront's own (its LDS accesses execute in order).  An expert in
            // several slots (a slot finds another's number where it left its own): their sum, slot after slot.
            float* const area = s_area[wave];
            if (e >= 0) area[e] = __int_as_float(lane);
            lds_in_order();
            const bool again = e >= 0 && __float_as_int(area[max(e, 0)]) != lane;
            if (__ballot(again) == 0) {
                lds_in_order();
#pragma unroll
                for (int i = 0; i < NPL; i++) area[lane + 64 * i] = 0.0f;
                lds_in_order();
                if (e >= 0) area[e] = v;
                lds_in_order();
#pragma unroll
                for (int i = 0; i < NPL; i++) out[i] += area[lane + 64 * i];
                lds_in_order();
            } else {
                for (int j = 0; j < k; j++) {
                    const int to = __builtin_amdgcn_readlane(e, j);
                    const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j));
#pragma unroll
                    for (int i = 0; i < NPL; i++) out[i] += to == lane + 64 * i ? add : 0.0f;
                }
            }
            if (row != 0.0f) {
#pragma unroll
                for (int i = 0; i < NPL; i++) out[i] = fmaf(-row, u[i] * inv, out[i]);
            }
        }
        bad = bad && (part || A.dw);
#pragma unroll
        for (int i = 0; i < NPL; i++) {
            const int to = lane + 64 * i;
            if (to >= E) continue;
            // (a masked logit's terms are products with 0, and what they are taken of may be no number)
            const float grad = l[i] == -__builtin_inff() ? 0.0f : out[i] * rest[i];
            store_out(A.grad, t * E + to, A.grad_dtype, bad ? __builtin_nanf("") : grad);
        }
    }
}

static long balance_groups(long T) { return T <= kBalanceOne ? 1 : T < kBalanceGroups * (long)kBalanceWaves ? (T + kBalanceWaves - 1) / kBalanceWaves : kBalanceGroups; }

struct BalanceLayout {
    size_t sums, often, terms, done, total;
};

static BalanceLayout balance_layout(long T, long E)
{
    BalanceLayout L;
    const size_t g = (size_t)balance_groups(T);
    L.sums = 0;
    L.often = g * (size_t)E * 8;
    L.terms = (L.often + g * (size_t)(E + 1) * 4 + 7) / 8 * 8;
    L.done = L.terms + (size_t)(E + 31) / 32 * 8;
    L.total = (L.done + 4 + 255) / 256 * 256;
    return L;
}

template <int DT>
static void route_balance_launch(dymoe_ctx* ctx, const void* logits, const int32_t* idx, const uint8_t* keep, int T, int E, int k, int sigmoid,
                                 float coef, int32_t* counts, float* mean, float* loss, char* ws, hipStream_t st)
{
    const int groups = (int)balance_groups(T);
    const BalanceLayout L = balance_layout(T, E);
    double* const sums = (double*)(ws + L.sums);
    int *const often = (int*)(ws + L.often), *const done = (int*)(ws + L.done);
#define DYMOE_BALANCE(NPL)                                                                                                              \
    do {                                                                                                                                \
        auto kernel = groups == 1 ? route_balance_kernel<NPL, DT, true> : route_balance_kernel<NPL, DT, false>;                          \
        dymoe_launch(ctx, DYMOE_K_ROUTE_BALANCE, kernel, dim3((unsigned)groups), dim3(64 * kBalanceWaves), 0, st, (const char*)logits,   \
                     idx, keep, T, E, k, sigmoid, sums, often, coef, counts, mean, loss, done);                                          \
    } while (0)
    if (E <= 64) DYMOE_BALANCE(1);
    else if (E <= 128) DYMOE_BALANCE(2);
    else if (E <= 256) DYMOE_BALANCE(4);
    else if (E <= 512) DYMOE_BALANCE(8);
    else DYMOE_BALANCE(16);
#undef DYMOE_BALANCE
    if (groups > 1)
        dymoe_launch(ctx, DYMOE_K_ROUTE_BALANCE, route_balance_finish_kernel, dim3((unsigned)((E + 31) / 32)), dim3(kBalanceFinish), 0, st, sums, often, groups, E, k,
                     coef, counts, mean, loss, (double*)(ws + L.terms), done);
}

template <int DT>
static void route_grad_launch(dymoe_ctx* ctx, const RouteGradArgs& A, hipStream_t st)
{
    const long blocks = (A.T + 3L) / 4;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
#define DYMOE_GRAD(NPL) dymoe_launch(ctx, DYMOE_K_ROUTE_BALANCE, route_grad_kernel<NPL, DT>, grid, dim3(256), 0, st, A)
    if (A.E <= 64) DYMOE_GRAD(1);
    else if (A.E <= 128) DYMOE_GRAD(2);
    else if (A.E <= 256) DYMOE_GRAD(4);
    else if (A.E <= 512) DYMOE_GRAD(8);
    else DYMOE_GRAD(16);
#undef DYMOE_GRAD
}

}  // namespace dymoe

using namespace dymoe;

extern "C" size_t dymoe_route_balance_workspace_bytes(int T, int E)
{
    if (T < 0 || E <= 0) return 0;
    return balance_layout(T, E).total;
}

extern "C" int dymoe_route_balance(dymoe_ctx* ctx, const void* logits, int dtype, const int32_t* idx, const uint8_t* keep, int T, int E, int k,
                                   int score, float coef, int32_t* counts, float* mean, float* loss, void* workspace, size_t workspace_bytes,
                                   void* stream)
{
    DYMOE_REQUIRE(T >= 0 && E > 0 && k > 0 && k <= E);
    DYMOE_REQUIRE(dtype == DYMOE_OUT_BF16 || dtype == DYMOE_OUT_F32 || dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(score == DYMOE_SCORE_SIGMOID || score == DYMOE_SCORE_SOFTMAX);
    DYMOE_REQUIRE(coef >= -FLT_MAX && coef <= FLT_MAX);
    DYMOE_REQUIRE(counts && mean && loss && workspace);
    if (T > 0) DYMOE_REQUIRE(logits && idx);
    DYMOE_REQUIRE(dymoe_aligned(logits, dtype_bytes(dtype)) && dymoe_aligned(idx, 4) && dymoe_aligned(counts, 4) && dymoe_aligned(mean, 4));
    DYMOE_REQUIRE(dymoe_aligned(loss, 4) && dymoe_aligned(workspace, 256));
    if (E > DYMOE_MAX_EXPERTS || k > 64 || T >= 1 << 25) return DYMOE_ENOTSUP;
    if (workspace_bytes < balance_layout(T, E).total) return DYMOE_ENOSPC;
    if (!ctx) return DYMOE_ENOCTX;
    auto launch = route_balance_launch<DYMOE_OUT_BF16>;
    if (dtype == DYMOE_OUT_F32) launch = route_balance_launch<DYMOE_OUT_F32>;
    else if (dtype == DYMOE_OUT_F16) launch = route_balance_launch<DYMOE_OUT_F16>;
    launch(ctx, logits, idx, keep, T, E, k, score == DYMOE_SCORE_SIGMOID, coef, counts, mean, loss, (char*)workspace, (hipStream_t)stream);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}

extern "C" int dymoe_route_scored_backward(dymoe_ctx* ctx, const void* logits, int dtype, const int32_t* idx, const float* dw, int T, int E, int k,
                                           int score, int renorm, float factor, const int32_t* counts, float coef, const float* dloss,
                                           const uint8_t* keep, int grad_dtype, void* grad, void* stream)
{
    DYMOE_REQUIRE(T >= 0 && E > 0 && k > 0 && k <= E);
    DYMOE_REQUIRE(dtype == DYMOE_OUT_BF16 || dtype == DYMOE_OUT_F32 || dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(grad_dtype == DYMOE_OUT_BF16 || grad_dtype == DYMOE_OUT_F32 || grad_dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(score == DYMOE_SCORE_SIGMOID || score == DYMOE_SCORE_SOFTMAX);
    DYMOE_REQUIRE(factor > 0.0f && factor <= FLT_MAX && coef >= -FLT_MAX && coef <= FLT_MAX);
    DYMOE_REQUIRE(dw || counts);
    if (T > 0) DYMOE_REQUIRE(logits && grad && (!dw || idx));
    DYMOE_REQUIRE(dymoe_aligned(logits, dtype_bytes(dtype)) && dymoe_aligned(grad, dtype_bytes(grad_dtype)) && dymoe_aligned(idx, 4));
    DYMOE_REQUIRE(dymoe_aligned(dw, 4) && dymoe_aligned(counts, 4) && dymoe_aligned(dloss, 4));
    if (E > DYMOE_MAX_EXPERTS || k > 64 || T >= 1 << 25) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    RouteGradArgs A = {};
    A.logits = (const char*)logits;
    A.idx = idx;
    A.dw = dw;
    A.counts = counts;
    A.dloss = dloss;
    A.keep = keep;
    A.grad = grad;
    A.T = T;
    A.E = E;
    A.k = k;
    A.sigmoid = score == DYMOE_SCORE_SIGMOID;
    A.renorm = renorm != 0;
    A.grad_dtype = grad_dtype;
    A.factor = factor;
    A.coef = coef;
    auto launch = route_grad_launch<DYMOE_OUT_BF16>;
    if (dtype == DYMOE_OUT_F32) launch = route_grad_launch<DYMOE_OUT_F32>;
    else if (dtype == DYMOE_OUT_F16) launch = route_grad_launch<DYMOE_OUT_F16>;
    launch(ctx, A, (hipStream_t)stream);
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
