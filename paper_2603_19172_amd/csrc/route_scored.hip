// Routing by scores: sigmoid or softmax of the router's logits, a bias that decides who is chosen but not with which weight, a
// selection among the best groups of experts, top-k, weights divided by their sum and scaled.
//
// One wavefront per token, lane l holding experts l, l + 64, ...; nothing is shared between tokens.  Scores are numbers of 64 bits: with
// a bias the order of two experts depends on how s + b is rounded, and of 8192 tokens with 256 experts a few have neighbours nearer
// than 32 bits tell apart.  A round of the top-k looks for the largest key, the compared value rounded to 32 bits in an order-preserving
// pattern (six instructions through the vector unit); only where two experts share that pattern are the 64 bits looked at.
// 8192 tokens, 8 of 256 experts in 4 of 8 groups: 14.7 us, bound by its 64-bit arithmetic and the rounds' dependent steps (the bytes take 2 us).  The
// groups are 4.5 us of it, the exponentials 3; one token 5.5 us, and 2047 of 128 experts without groups: latencies.
#include <float.h>

#include "int8_device.hpp"

namespace dymoe {

// 1 / d, d in [1, 1e308]: the instruction's estimate and two Newton steps
__device__ __forceinline__ double inverse(double d)
{
    double r = __builtin_amdgcn_rcp(d);
    r = fma(fma(-d, r, 1.0), r, r);
    return fma(fma(-d, r, 1.0), r, r);
}

// e^x for |x| <= 709: x = n ln 2 + r, |r| <= 0.3466, and the Taylor polynomial of degree 13, whose next term is below 2^-57 of the sum.
// (Half the instructions of the library's, which four experts a lane spend a third of the kernel on.)
__device__ __forceinline__ double exp_of(double x)
{
    const double n = __builtin_rint(x * 1.4426950408889634);
    const double r = fma(n, -2.3190468138462996e-17, fma(n, -0.6931471805599453, x));
    double p = 1.0 / 6227020800.0;
    p = fma(p, r, 1.0 / 479001600.0);
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

__device__ __forceinline__ double lane_double(double v, int lane)       // lane the same for the whole wavefront
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

__device__ __forceinline__ uint32_t order_key(float f)
{
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// NPL: experts a lane holds.  DT: type of the logits.
template <int NPL, int DT>
__global__ __launch_bounds__(256) void route_scored_kernel(const char* __restrict__ logits, const float* __restrict__ bias, int T, int E,
                                                           int k, int sigmoid, int groups, int top_groups, int best, uint32_t per_group, int renorm,
                                                           float factor, int32_t* __restrict__ idx, float* __restrict__ w,
                                                           float* __restrict__ scores)
{
    extern __shared__ double s_value[];                       // a wavefront's compared values, where there are groups
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const long t = (long)blockIdx.x * 4 + wave;
    if (t >= T) return;                                       // (no barriers below)
    const double kLow = -__builtin_inf();
    const float lowest = DT == DYMOE_OUT_F32 ? -FLT_MAX : DT == DYMOE_OUT_F16 ? -65504.0f : -0x1.fep127f;

    float l[NPL];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        const int e = lane + 64 * i;
        l[i] = -__builtin_inff();
        if (e < E) {
            const long at = t * E + e;
            if constexpr (DT == DYMOE_OUT_F32) l[i] = ((const DYMOE_GLOBAL float*)logits)[at];
            else if constexpr (DT == DYMOE_OUT_F16) l[i] = (float)((const DYMOE_GLOBAL _Float16*)logits)[at];
            else l[i] = bf16_bits_to_f32(((const DYMOE_GLOBAL uint16_t*)logits)[at]);
            l[i] += 0.0f;                                     // (-0 is 0: the two are one number and tie)
            bad |= l[i] != l[i];
            if (!(l[i] > lowest)) l[i] = -__builtin_inff();   // masked; NaN ranks with the masked ones
        }
    }
    // scores
    double s[NPL], c[NPL];
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < NPL; i++) s[i] = l[i] == -__builtin_inff() ? 0.0 : inverse(1.0 + exp_of(-(double)fminf(fmaxf(l[i], -700.0f), 700.0f)));
    } else {
        uint32_t mk = 0;
#pragma unroll
        for (int i = 0; i < NPL; i++) mk = max(mk, order_key(l[i]));
        mk = wave_max_u32(mk);
        const float m = __uint_as_float(mk & 0x80000000u ? mk ^ 0x80000000u : ~mk);
        bad |= m == __builtin_inff();
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < NPL; i++) {
            // (a difference beyond 700 is a score below 2^-1000: 0 in the call's types)
            s[i] = l[i] == -__builtin_inff() ? 0.0 : exp_of(fmax((double)l[i] - (double)m, -700.0));
            sum += s[i];
        }
        sum = wave_sum_f64(sum);
        const double inv = sum > 0.0 ? inverse(sum) : 0.0;
#pragma unroll
        for (int i = 0; i < NPL; i++) s[i] *= inv;
    }
    bad = __ballot(bad) != 0;
    // what is compared: the score with its bias, or, in the same order, the logit
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        const int e = lane + 64 * i;
        c[i] = l[i] == -__builtin_inff() ? kLow : bias ? s[i] + (double)bias[min(e, E - 1)] : groups > 1 && best == 2 ? s[i] : (double)l[i];
        if (c[i] != c[i]) c[i] = kLow;
    }
    uint32_t key[NPL];
    uint64_t kept = ~0ull;
    const int per = E / groups;
    if (groups > 1) {
        double* const v = s_value + wave * (NPL * 64);
#pragma unroll
        for (int i = 0; i < NPL; i++) v[lane + 64 * i] = c[i];
        __builtin_amdgcn_wave_barrier();
        // lanes to a group: a power of two, so that a group's lanes meet in a butterfly
        int lg = 1;
        while (2 * lg * groups <= 64) lg *= 2;
        const int g = lane / lg, part = lane & (lg - 1);
        double v1 = kLow, v2 = kLow;
        if (g < groups)
            for (int j = part; j < per; j += lg) {
                const double d = v[g * per + j];
                v2 = fmax(v2, fmin(v1, d));
                v1 = fmax(v1, d);
            }
        for (int o = 1; o < lg; o *= 2) {
            const double a = __shfl_xor(v1, o, kWave), b = __shfl_xor(v2, o, kWave);
            v2 = fmax(fmax(v2, b), fmin(v1, a));
            v1 = fmax(v1, a);
        }
        const double value = best == 2 && v2 > kLow ? v1 + v2 : v1;
        int rank = 0;
        for (int h = 0; h < groups; h++) {
            const double o = lane_double(value, h * lg);
            rank += (o > value) || (o == value && h < g);
        }
        const uint64_t in = __ballot(g < groups && part == 0 && rank < top_groups);
        kept = 0;
        for (int h = 0; h < groups; h++) kept |= ((in >> (h * lg)) & 1ull) << h;
        // (the order inside the groups is the logits' where no bias moves it)
        if (!bias && best == 2) {
#pragma unroll
            for (int i = 0; i < NPL; i++) c[i] = (double)l[i];
        }
    }
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        const int e = lane + 64 * i;
        const bool in = e < E && (groups == 1 || ((kept >> ((uint32_t)e * per_group >> 21)) & 1ull));      // its group, e / per
        key[i] = in ? order_key((float)c[i]) : 0u;            // 0: cannot be chosen
    }
    if (scores) {
#pragma unroll
        for (int i = 0; i < NPL; i++) {
            const int e = lane + 64 * i;
            if (e < E) scores[t * E + e] = bad ? __builtin_nanf("") : (float)s[i];
        }
    }
    // A lane keeps its keys in falling order, so that a round compares one key a lane: the lane that has the round's
    // largest gives it up and shows its next.
    int which[NPL];
#pragma unroll
    for (int i = 0; i < NPL; i++) which[i] = i;
    // (Batcher's merging network: 1, 5, 19 or 63 comparisons)
#pragma unroll
    for (int p = 1; p < NPL; p *= 2)
#pragma unroll
        for (int d = p; d >= 1; d /= 2)
#pragma unroll
            for (int j = d % p; j + d < NPL; j += 2 * d)
#pragma unroll
                for (int i = 0; i < d; i++)
                    if (i + j + d < NPL && (i + j) / (2 * p) == (i + j + d) / (2 * p)) {
                        const bool swap = key[i + j + d] > key[i + j];
                        const uint32_t ka = key[i + j], kb = key[i + j + d];
                        const int wa = which[i + j], wb = which[i + j + d];
                        key[i + j] = swap ? kb : ka;
                        key[i + j + d] = swap ? ka : kb;
                        which[i + j] = swap ? wb : wa;
                        which[i + j + d] = swap ? wa : wb;
                    }
    int mine = 0;
    for (int j = 0; j < k; j++) {
        const uint32_t top = wave_max_u32(key[0]);
        uint64_t at = __ballot(key[0] == top);
        int owner = __builtin_ctzll(at), first;
        // more than one expert with that key, in several lanes or in one lane's next place
        const uint64_t again = NPL > 1 ? __ballot(key[0] == top && key[NPL > 1 ? 1 : 0] == top) : 0;
        if (((at & (at - 1)) | again) == 0) {
            first = 64 * __builtin_amdgcn_readlane(which[0], owner) + owner;
        } else {
            // the largest of the 64-bit values (without a bias the keys are the logits themselves), then the lowest index
            double best = kLow, of[NPL];
            if (bias) {
#pragma unroll
                for (int i = 0; i < NPL; i++) {
                    of[i] = kLow;
#pragma unroll
                    for (int u = 0; u < NPL; u++) of[i] = which[i] == u ? c[u] : of[i];
                    best = fmax(best, key[i] == top ? of[i] : kLow);
                }
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) best = fmax(best, __shfl_xor(best, o, kWave));
            }
            uint32_t low = 0xffffffffu;
#pragma unroll
            for (int i = 0; i < NPL; i++)
                if (key[i] == top && (!bias || of[i] == best)) low = min(low, (uint32_t)(64 * which[i] + lane));
            first = (int)~wave_max_u32(~low);
            owner = first & 63;
            // to the front of its lane
            const int slot = first >> 6;
            if (lane == owner) {
#pragma unroll
                for (int i = NPL - 1; i > 0; i--)
                    if (key[i] == top && which[i] == slot) {
                        which[i] = which[0];
                        which[0] = slot;
                    }
            }
        }
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i + 1 < NPL; i++) {
                key[i] = key[i + 1];
                which[i] = which[i + 1];
            }
            key[NPL - 1] = 0u;
        }
        if (lane == j) mine = first;
    }
    double weight = 0.0;
#pragma unroll
    for (int i = 0; i < NPL; i++) {
        const double v = __shfl(s[i], mine & 63, kWave);
        if (lane < k && (mine >> 6) == i) weight = v;
    }
    if (renorm) {
        const double sum = wave_sum_f64(weight);
        weight = sum > 0.0 ? weight / sum : 0.0;
    }
    if (lane < k) {
        idx[t * k + lane] = mine;
        w[t * k + lane] = bad ? __builtin_nanf("") : (float)(weight * (double)factor);
    }
}

template <int DT>
static void route_scored_launch(dymoe_ctx* ctx, const void* logits, const float* bias, int T, int E, int k, int sigmoid, int groups,
                                int top_groups, int best, int renorm, float factor, int32_t* idx, float* w, float* scores, hipStream_t st)
{
    const dim3 grid((unsigned)((T + 3L) / 4));
#define DYMOE_RSCORED(NPL)                                                                                                        \
    dymoe_launch(ctx, DYMOE_K_ROUTE_SCORED, route_scored_kernel<NPL, DT>, grid, dim3(256), groups > 1 ? 4 * NPL * 64 * 8 : 0, st, \
                 (const char*)logits, bias, T, E, k, sigmoid, groups, top_groups, best,                   \
                 (uint32_t)((1 << 21) / (E / groups) + 1), renorm, factor, idx, w, scores)
    if (E <= 64) DYMOE_RSCORED(1);
    else if (E <= 128) DYMOE_RSCORED(2);
    else if (E <= 256) DYMOE_RSCORED(4);
    else if (E <= 512) DYMOE_RSCORED(8);
    else DYMOE_RSCORED(16);
#undef DYMOE_RSCORED
}

}  // namespace dymoe

extern "C" int dymoe_route_scored(dymoe_ctx* ctx, const void* logits, int dtype, const float* bias, int T, int E, int k, int score,
                                  int groups, int top_groups, int group_best, int renorm, float factor, int32_t* idx, float* w,
                                  float* scores, void* stream)
{
    DYMOE_REQUIRE(T >= 0 && E > 0 && k > 0 && k <= E);
    DYMOE_REQUIRE(dtype == DYMOE_OUT_BF16 || dtype == DYMOE_OUT_F32 || dtype == DYMOE_OUT_F16);
    DYMOE_REQUIRE(score == DYMOE_SCORE_SIGMOID || score == DYMOE_SCORE_SOFTMAX);
    DYMOE_REQUIRE(groups >= 1 && E % groups == 0 && top_groups >= 1 && top_groups <= groups);
    DYMOE_REQUIRE(group_best == 1 || group_best == 2);
    DYMOE_REQUIRE((long)top_groups * (E / groups) >= k);
    DYMOE_REQUIRE(factor > 0.0f && factor <= FLT_MAX);
    if (T > 0) DYMOE_REQUIRE(logits && idx && w);
    DYMOE_REQUIRE(dymoe_aligned(logits, dymoe::dtype_bytes(dtype)) && dymoe_aligned(idx, 4) && dymoe_aligned(w, 4));
    DYMOE_REQUIRE(dymoe_aligned(bias, 4) && dymoe_aligned(scores, 4));
    if (E > DYMOE_MAX_EXPERTS || k > 64 || groups > 64 || T >= 1 << 26) return DYMOE_ENOTSUP;
    if (!ctx) return DYMOE_ENOCTX;
    if (T == 0) return DYMOE_OK;
    auto launch = dymoe::route_scored_launch<DYMOE_OUT_BF16>;
    if (dtype == DYMOE_OUT_F32) launch = dymoe::route_scored_launch<DYMOE_OUT_F32>;
    else if (dtype == DYMOE_OUT_F16) launch = dymoe::route_scored_launch<DYMOE_OUT_F16>;
    // tokens of a launch at most: 64 threads a token, and a grid has to stay below 2^32 of them
    constexpr int kTokens = 1 << 25;
    for (int t = 0; t < T; t += kTokens) {
        const int n = T - t < kTokens ? T - t : kTokens;
        launch(ctx, (const char*)logits + (size_t)t * E * dymoe::dtype_bytes(dtype), bias, n, E, k, score == DYMOE_SCORE_SIGMOID, groups, top_groups,
               group_best, renorm, factor, idx + (size_t)t * k, w + (size_t)t * k, scores ? scores + (size_t)t * E : nullptr, (hipStream_t)stream);
    }
    DYMOE_HIP_LAUNCH_CHECK();
    return DYMOE_OK;
}
