// The training side of the router that scores (dymoe_route_scored): the balance loss with its counts, and the logits' gradient.
//
// A token's shares p = s / sum s come from fp32 exponentials of differences to its largest logit, so that no scores are too small to be
// divided; with sigmoids u = e^(min(l, 0) - min(m, 0)) / (1 + e^-|l|) is s e^(-min(m, 0)).  One wavefront per token, lane l holding experts l,
// l + 64, ...  Sums over tokens are held in 64 bits and taken in an order that follows from T and E alone.
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

// s e^(-min(m, 0)) of a sigmoid, e^(l - m) of a softmax
__device__ __forceinline__ float scaled_score(float l, float m, bool sigmoid)
{
    if (l == -__builtin_inff()) return 0.0f;
    if (!sigmoid) return exp_neg(l - m);
    return exp_neg(fminf(l, 0.0f) - fminf(m, 0.0f)) * __builtin_amdgcn_rcpf(1.0f + exp_neg(-fabsf(l)));
}

// 1 - s of a sigmoid
__device__ __forceinline__ float rest_of(float l)
{
    const float e = exp_neg(-fabsf(l));
    return (l > 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e);
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
__device__ __forceinline__ bool token_scores(const float (&raw)[NPL], bool sigmoid, float (&l)[NPL], float (&u)[NPL], float& m, float& inv)
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
        u[i] = scaled_score(l[i], m, sigmoid);
        sum += u[i];
    }
    sum = wave_sum(sum);
    inv = sum > 0.0f ? __builtin_amdgcn_rcpf(sum) : 0.0f;
    return __ballot(bad) != 0;
}

// counts, means and the loss from the sums of `groups` workgroups, by one workgroup
__device__ __forceinline__ void balance_finish(const double* sums, const int* often, int groups, int E, int k, float coef, int32_t* counts, float* mean,
                                               float* loss, double* s_part, int* s_often)
{
    const int tid = threadIdx.x, n = blockDim.x;
    const int slices = max(1, n / (E + 1)), slice = tid / (E + 1);
    // expert E: the tokens that take part
    for (int e0 = 0; e0 <= E; e0 += n) {
        const int e = e0 + (slices > 1 ? tid - slice * (E + 1) : tid);
        double sum = 0.0;
        int c = 0;
        if (slice < slices || slices == 1) {
            // (eight workgroups' at a time: one after the other their loads cost 45 us for 256 of them)
            const int first = slices > 1 ? slice : 0;
            for (int g0 = first; g0 < groups && e <= E; g0 += 8 * slices) {
                double v[8];
                int n8[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int g = g0 + i * slices;
                    v[i] = g < groups && e < E ? sums[(long)g * E + e] : 0.0;
                    n8[i] = g < groups ? often[(long)g * (E + 1) + e] : 0;
                }
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    sum += v[i];
                    c += n8[i];
                }
            }
        }
        if (slices > 1) {
            s_part[tid] = sum;
            s_often[tid] = c;
            __syncthreads();
            if (slice == 0 && e <= E) {
                for (int s = 1; s < slices; s++) {
                    sum += s_part[tid + s * (E + 1)];
                    c += s_often[tid + s * (E + 1)];
                }
            }
            __syncthreads();
        }
        if ((slices == 1 || slice == 0) && e <= E) {
            counts[e] = c;
            if (e < E) s_part[e] = sum;
            s_often[e] = c;
        }
    }
    __syncthreads();
    const int tokens = s_often[E];
    const double inv = tokens > 0 ? 1.0 / (double)tokens : 0.0;
    double term = 0.0;
    for (int e = tid; e < E; e += n) {
        const double p = s_part[e] * inv;
        mean[e] = (float)p;
        term += (double)s_often[e] * p;
    }
    __syncthreads();
    // the loss: lane by lane, then in LDS, in a fixed order
    s_part[tid] = term;
    __syncthreads();
    for (int d = n / 2; d > 0; d /= 2) {
        if (tid < d) s_part[tid] += s_part[tid + d];
        __syncthreads();
    }
    if (tid == 0) *loss = (float)((double)coef * (double)E * inv / (double)k * s_part[0]);
}

constexpr int kBalanceFinish = 1024;      // threads of the second launch

// ONE: the whole call.  Otherwise sums [groups][E] and counts [groups][E + 1] of the workgroup's tokens.
template <int NPL, int DT, bool ONE>
__global__ __launch_bounds__(64 * kBalanceWaves) void route_balance_kernel(const char* __restrict__ logits, const int32_t* __restrict__ idx,
                                                                           const uint8_t* __restrict__ keep, int T, int E, int k, int sigmoid,
                                                                           double* __restrict__ sums, int* __restrict__ often, float coef,
                                                                           int32_t* __restrict__ counts, float* __restrict__ mean,
                                                                           float* __restrict__ loss)
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
        float l[NPL], u[NPL], m, inv;
        const bool bad = token_scores<NPL, DT>(now, sigmoid, l, u, m, inv);
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

__global__ __launch_bounds__(kBalanceFinish) void route_balance_finish_kernel(const double* __restrict__ sums, const int* __restrict__ often, int groups,
                                                                              int E, int k, float coef, int32_t* __restrict__ counts,
                                                                              float* __restrict__ mean, float* __restrict__ loss)
{
    __shared__ double s_part[kBalanceFinish];
    __shared__ int s_often[kBalanceFinish + 1];
    balance_finish(sums, often, groups, E, k, coef, counts, mean, loss, s_part, s_often);
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
        float raw[NPL], l[NPL], u[NPL], m, inv;
        load_token<NPL, DT>(A.logits, t, E, lane, raw);
        bool bad = token_scores<NPL, DT>(raw, sigmoid, l, u, m, inv);
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
            int e = -1;
            float x = -__builtin_inff(), dw = 0.0f;
            if (lane < k) {
                e = A.idx[t * k + lane];
                bool ignored = false;
                if ((unsigned)e < (unsigned)E) {
                    x = masked_logit<DT>(load_logit<DT>(A.logits, t * E + e), ignored);
                    dw = A.dw[t * k + lane];
                } else {
                    e = -1;
                }
            }
            float v, row = 0.0f;
            if (A.renorm) {
                const float top = wave_max_dpp(x), s = scaled_score(x, top, sigmoid), sum = wave_sum(s);
                const float q = sum > 0.0f ? s / sum : 0.0f;
                const float dot = wave_sum(q != 0.0f ? q * dw : 0.0f);
                v = q != 0.0f ? A.factor * (q * (dw - dot)) : 0.0f;
            } else if (sigmoid) {
                v = x > -__builtin_inff() ? A.factor * (scaled_score(x, 0.0f, true) * dw) : 0.0f;
            } else {
                const float s = scaled_score(x, m, false) * inv;
                const float one = s != 0.0f ? s * dw : 0.0f;
                v = A.factor * one;
                row = A.factor * wave_sum(one);
            }
            // to the lanes that hold the experts
            for (int j = 0; j < k; j++) {
                const int to = __builtin_amdgcn_readlane(e, j);
                const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j));
#pragma unroll
                for (int i = 0; i < NPL; i++) out[i] += to == lane + 64 * i ? add : 0.0f;
            }
            if (row != 0.0f) {
#pragma unroll
                for (int i = 0; i < NPL; i++) out[i] = fmaf(-row, u[i] * inv, out[i]);
            }
        }
        bad = bad && (part || A.dw);
#pragma unroll
        for (int i = 0; i < NPL; i++) {
            const int e = lane + 64 * i;
            if (e >= E) continue;
            float v = out[i];
            if (sigmoid) v = l[i] == -__builtin_inff() ? 0.0f : v * rest_of(l[i]);
            store_out(A.grad, t * E + e, A.grad_dtype, bad ? __builtin_nanf("") : v);
        }
    }
}

static long balance_groups(long T) { return T <= kBalanceOne ? 1 : T < kBalanceGroups * (long)kBalanceWaves ? (T + kBalanceWaves - 1) / kBalanceWaves : kBalanceGroups; }

struct BalanceLayout {
    size_t sums, often, total;
};

static BalanceLayout balance_layout(long T, long E)
{
    BalanceLayout L;
    const size_t g = (size_t)balance_groups(T);
    L.sums = 0;
    L.often = g * (size_t)E * 8;
    L.total = (L.often + g * (size_t)(E + 1) * 4 + 255) / 256 * 256;
    return L;
}

template <int DT>
static void route_balance_launch(dymoe_ctx* ctx, const void* logits, const int32_t* idx, const uint8_t* keep, int T, int E, int k, int sigmoid,
                                 float coef, int32_t* counts, float* mean, float* loss, char* ws, hipStream_t st)
{
    const int groups = (int)balance_groups(T);
    const BalanceLayout L = balance_layout(T, E);
    double* const sums = (double*)(ws + L.sums);
    int* const often = (int*)(ws + L.often);
#define DYMOE_BALANCE(NPL)                                                                                                              \
    do {                                                                                                                                \
        auto kernel = groups == 1 ? route_balance_kernel<NPL, DT, true> : route_balance_kernel<NPL, DT, false>;                          \
        dymoe_launch(ctx, DYMOE_K_ROUTE_BALANCE, kernel, dim3((unsigned)groups), dim3(64 * kBalanceWaves), 0, st, (const char*)logits,   \
                     idx, keep, T, E, k, sigmoid, sums, often, coef, counts, mean, loss);                                                \
    } while (0)
    if (E <= 64) DYMOE_BALANCE(1);
    else if (E <= 128) DYMOE_BALANCE(2);
    else if (E <= 256) DYMOE_BALANCE(4);
    else if (E <= 512) DYMOE_BALANCE(8);
    else DYMOE_BALANCE(16);
#undef DYMOE_BALANCE
    if (groups > 1)
        dymoe_launch(ctx, DYMOE_K_ROUTE_BALANCE, route_balance_finish_kernel, dim3(1), dim3(kBalanceFinish), 0, st, sums, often, groups, E, k, coef, counts,
                     mean, loss);
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
