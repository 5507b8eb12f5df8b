// Losses that look at one token a position (clipped policy loss with a KL term, paired preference loss) and their gradient.
//
// Both rest on lp = z[a] - log(sum of exp z), z = logits / T, and on one number a row, the slope d loss / d lp:
// dlogits = dloss * slope / T * ([c == a] - softmax(z)[c]).
#include "worker_common.cuh"

namespace bz {

namespace {

struct TokenArgs {
    int64_t ld, v, ld_d;
    const int32_t* index;
    double inv_t;             // 1 / T
    float temperature, c;     // c = log2(e) / T
    const float *old_logp, *ref_logp, *advantage;
    float clip_low, clip_high, kl;
    const float* dloss;
    float *loss, *logp;
    float4* stats;            // largest logit, sum of e^((s - that)/T), slope, place in dloss
};

// lp of a logit in a row of maximum m and sum s.
__device__ __forceinline__ double log_probability(float logit, float m, float s, double inv_t) {
    if (logit == -INFINITY) return -INFINITY;
    return (static_cast<double>(logit) - static_cast<double>(m)) * inv_t - log(static_cast<double>(s));
}

struct PolicyRow {
    float loss, slope;
};
__device__ __forceinline__ PolicyRow policy_row(const TokenArgs& a, int64_t i, double lp) {
    double loss = 0.0, slope = 0.0;
    const double adv = a.advantage[i];
    if (adv != 0.0) {   // a NaN goes on
        const double r = a.old_logp != nullptr ? exp(lp - static_cast<double>(a.old_logp[i])) : 1.0;
        const double lo = 1.0 - static_cast<double>(a.clip_low), hi = 1.0 + static_cast<double>(a.clip_high);
        const bool held = adv > 0.0 ? r > hi : adv < 0.0 && r < lo;
        loss = -(held ? (adv > 0.0 ? hi : lo) : r) * adv;
        slope = held ? 0.0 : -r * adv;
    }
    if (a.kl != 0.f) {
        const double d = static_cast<double>(a.ref_logp[i]) - lp, e = expm1(d), k = a.kl;
        loss += k * (isinf(e) ? e : e - d);
        slope -= k * e;
    }
    return {static_cast<float>(loss), lp == -INFINITY ? 0.f : static_cast<float>(slope)};
}

// The largest of a row and its sum of exponentials, over the CTA.
template <typename T, int VEC> __device__ __forceinline__ MaxSum row_statistics(const T* row, int64_t v, float c, MaxSum* part) {
    MaxSum mine{-INFINITY, 0.f};
    float x[VEC];
    for (int64_t j0 = static_cast<int64_t>(threadIdx.x) * VEC - row_lead<T, VEC>(row); j0 < v; j0 += blockDim.x * VEC) {
        load_slot<T, VEC>(row, j0, v, -INFINITY, x);
        const float m = largest(mine.m, x);
        const Reference r(m, c);
        if (mine.s != 0.f) mine.s *= exp2_fast(r.of_part(mine.m, c));
        mine.m = m;
        exponentials(x, r, c);
#pragma unroll
        for (int k = 0; k < VEC; ++k) mine.s += x[k];
    }
    mine = warp_join(mine, c);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = mine;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_join(lane < (blockDim.x >> 5) ? part[lane] : MaxSum{-INFINITY, 0.f}, c);
}

// g ([c == a] - softmax); g == 0: zeros, whatever the logits.
template <typename T, int VEC> __device__ __forceinline__ void row_gradient(const T* row, T* out, int64_t v, int a, float c, MaxSum all, float g) {
    const Reference r(all.m, c);
    const float factor = g == 0.f ? 0.f : -g / all.s;
    for (int64_t j0 = static_cast<int64_t>(threadIdx.x) * VEC - row_lead<T, VEC>(row); j0 < v; j0 += blockDim.x * VEC) {
        float x[VEC];
        if (g == 0.f) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = 0.f;
        } else {
            load_slot<T, VEC>(row, j0, v, -INFINITY, x);
            exponentials(x, r, c);
            multiply(x, factor);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (j0 + k == a) x[k] += g;
        }
        store_slot<T, VEC>(out, j0, v, x);
    }
}

// One CTA a row.  POLICY: the loss too, and the gradient if it is wanted; otherwise lp and stats alone.
template <typename T, int VEC, bool POLICY> __global__ void __launch_bounds__(512) token_rows_kernel(const __grid_constant__ TokenArgs a, const T* logits, T* dlogits) {
    __shared__ MaxSum part[32];
    __shared__ float slope;
    const int64_t i = blockIdx.x;
    const T* row = logits + i * a.ld;
    const int at = a.index[i];
    const bool there = at >= 0 && at < a.v;
    MaxSum all{-INFINITY, 0.f};
    if (there) all = row_statistics<T, VEC>(row, a.v, a.c, part);
    if (threadIdx.x == 0) {
        float4 st = make_float4(-INFINITY, 0.f, 0.f, __int_as_float(static_cast<int>(i)));
        float lp = 0.f, loss = 0.f;
        if (there) {
            st.x = all.m, st.y = all.s / Reference(all.m, a.c).left_out(a.c);
            const double precise = log_probability(to_f32(row[at]), st.x, st.y, a.inv_t);
            lp = static_cast<float>(precise);
            if (POLICY) {
                const PolicyRow p = policy_row(a, i, precise);
                loss = p.loss, st.z = p.slope;
            }
        }
        if (a.logp != nullptr) a.logp[i] = lp;
        if (POLICY && a.loss != nullptr) a.loss[i] = loss;
        if (a.stats != nullptr) a.stats[i] = st;
        slope = st.z;
    }
    if (!POLICY || dlogits == nullptr) return;
    __syncthreads();
    const float g = slope == 0.f ? 0.f : slope * (a.dloss != nullptr ? a.dloss[i] : 1.f) / a.temperature;
    row_gradient<T, VEC>(row, dlogits + i * a.ld_d, a.v, at, a.c, all, g);
}

// The gradient from given stats.
template <typename T, int VEC> __global__ void __launch_bounds__(512) token_gradient_kernel(const __grid_constant__ TokenArgs a, const T* logits, T* dlogits) {
    const int64_t i = gridDim.x - 1 - blockIdx.x;
    const T* row = logits + i * a.ld;
    const float4 st = a.stats[i];
    const int at = a.index[i];
    const bool there = at >= 0 && at < a.v;
    const float g = st.z == 0.f || !there ? 0.f : st.z * (a.dloss != nullptr ? a.dloss[__float_as_int(st.w)] : 1.f) / a.temperature;
    row_gradient<T, VEC>(row, dlogits + i * a.ld_d, a.v, at, a.c, {st.x, st.y * Reference(st.x, a.c).left_out(a.c)}, g);
}

struct PairArgs {
    const int32_t* starts;
    int64_t m, v, pairs;
    float beta, margin, smoothing;
    int mean;
    float *loss, *reward;
};

// One CTA a pair: the sequences' sums, the loss and each row's slope.
__global__ void __launch_bounds__(256) pair_kernel(const __grid_constant__ TokenArgs a, const __grid_constant__ PairArgs p, const void* logits, int dtype) {
    __shared__ double sums[2][8];
    __shared__ int counts[2][8];
    const int64_t pair = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t from[2], to[2];
    for (int side = 0; side < 2; ++side) {
        const int64_t n = pair + side * p.pairs;
        from[side] = min(max(static_cast<int64_t>(p.starts[n]), int64_t(0)), p.m);
        to[side] = max(from[side], min(static_cast<int64_t>(p.starts[n + 1]), p.m));
        double sum = 0.0;
        int count = 0;
        for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += blockDim.x) {
            const int at = a.index[i];
            if (at < 0 || at >= p.v) continue;
            const int64_t k = i * a.ld + at;
            const float logit = dtype == BZ_F32 ? static_cast<const float*>(logits)[k] : dtype == BZ_F16 ? to_f32(static_cast<const __half*>(logits)[k])
                                                                                                          : to_f32(static_cast<const __nv_bfloat16*>(logits)[k]);
            const float4 st = a.stats[i];
            sum += log_probability(logit, st.x, st.y, a.inv_t) - (a.ref_logp != nullptr ? static_cast<double>(a.ref_logp[i]) : 0.0);
            ++count;
        }
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o), count += __shfl_xor_sync(~0u, count, o);
        if (lane == 0) sums[side][warp] = sum, counts[side][warp] = count;
    }
    __syncthreads();
    double reward[2], share[2];
    for (int side = 0; side < 2; ++side) {
        double sum = 0.0;
        int count = 0;
        for (int w = 0; w < 8; ++w) sum += sums[side][w], count += counts[side][w];
        share[side] = static_cast<double>(p.beta) / (p.mean ? max(count, 1) : 1);
        reward[side] = share[side] * sum;
    }
    const double h = reward[0] - reward[1] - static_cast<double>(p.margin), eps = p.smoothing;
    const double tail = log1p(exp(-fabs(h)));   // -log sigmoid(|h|)
    if (threadIdx.x == 0) {
        // a weight of 0 has no term, whatever its logarithm
        const double up = tail + fmax(-h, 0.0), down = tail + fmax(h, 0.0);
        if (p.loss != nullptr) p.loss[pair] = isnan(h) ? NAN : static_cast<float>((eps != 1.0 ? (1.0 - eps) * up : 0.0) + (eps != 0.0 ? eps * down : 0.0));
        if (p.reward != nullptr) p.reward[pair] = static_cast<float>(reward[0]), p.reward[pair + p.pairs] = static_cast<float>(reward[1]);
    }
    // d loss / d h = sigmoid(h) - (1 - eps); sigmoid(h) = 1 - sigmoid(-h) for the digits of the smaller one
    const double small = exp(-fabs(h)) / (1.0 + exp(-fabs(h)));
    const double dh = h >= 0.0 ? eps - small : h < 0.0 ? small - (1.0 - eps) : NAN;
    for (int side = 0; side < 2; ++side) {
        const float slope = static_cast<float>(side == 0 ? dh * share[0] : -dh * share[1]);
        for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += blockDim.x) {
            const int at = a.index[i];
            float4 st = a.stats[i];
            const float logit = at < 0 || at >= p.v ? -INFINITY : dtype == BZ_F32 ? static_cast<const float*>(logits)[i * a.ld + at]
                                : dtype == BZ_F16 ? to_f32(static_cast<const __half*>(logits)[i * a.ld + at]) : to_f32(static_cast<const __nv_bfloat16*>(logits)[i * a.ld + at]);
            st.z = logit == -INFINITY ? 0.f : slope;
            st.w = __int_as_float(static_cast<int>(pair));
            a.stats[i] = st;
        }
    }
}

// v == 0: rows without a token.
__global__ void token_empty_kernel(int64_t m, float* loss, float* logp, float4* stats) {
    for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < m; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        if (loss != nullptr) loss[i] = 0.f;
        if (logp != nullptr) logp[i] = 0.f;
        if (stats != nullptr) stats[i] = make_float4(-INFINITY, 0.f, 0.f, __int_as_float(static_cast<int>(i)));
    }
}

// ---- host side ----------------------------------------------------------------------------------

enum What { kPolicy, kScore, kGradient };

template <typename T, int VEC> int launch(const TokenArgs& a, int64_t m, const T* logits, T* dlogits, What what, cudaStream_t s) {
    const unsigned rows = static_cast<unsigned>(m);
    if (what == kPolicy)
        token_rows_kernel<T, VEC, true><<<rows, 512, 0, s>>>(a, logits, dlogits);
    else if (what == kScore)
        token_rows_kernel<T, VEC, false><<<rows, 512, 0, s>>>(a, logits, dlogits);
    else
        token_gradient_kernel<T, VEC><<<rows, 512, 0, s>>>(a, logits, dlogits);
    note_launch();
    return check_launch();
}

template <typename T> int dispatch(const TokenArgs& a, int64_t m, const void* logits, void* dlogits, What what, cudaStream_t s) {
    const T* in = static_cast<const T*>(logits);
    T* out = static_cast<T*>(dlogits);
    const uintptr_t apart = reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(dlogits);
    const bool alike = out == nullptr || ((apart & 15) == 0 && (m == 1 || ((a.ld - a.ld_d) * static_cast<int64_t>(sizeof(T))) % 16 == 0));
    return alike ? launch<T, Word<T>::kN>(a, m, in, out, what, s) : launch<T, 1>(a, m, in, out, what, s);
}

int dispatch(const TokenArgs& a, int dtype, int64_t m, const void* logits, void* dlogits, What what, cudaStream_t s) {
    if (dtype == BZ_F32) return dispatch<float>(a, m, logits, dlogits, what, s);
    if (dtype == BZ_F16) return dispatch<__half>(a, m, logits, dlogits, what, s);
    return dispatch<__nv_bfloat16>(a, m, logits, dlogits, what, s);
}

int check(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, float temperature, const void* stats, const void* dlogits, int64_t ld_d) {
    const int bytes = element_bytes(dtype);
    if (bytes == 0 || m < 0 || v < 0 || !(temperature > 0.f) || isinf(temperature) || isinf(kLog2e / temperature) || !aligned16(stats)) return BZ_ERR_INVALID_ARG;
    if (v >= (int64_t(1) << 31) || m >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    if (m == 0) return BZ_OK;
    if (index == nullptr) return BZ_ERR_INVALID_ARG;
    if (v == 0) return BZ_OK;
    if (logits == nullptr || (m > 1 && ld < v) || reinterpret_cast<uintptr_t>(logits) % bytes) return BZ_ERR_INVALID_ARG;
    if (dlogits != nullptr && ((m > 1 && ld_d < v) || reinterpret_cast<uintptr_t>(dlogits) % bytes)) return BZ_ERR_INVALID_ARG;
    if (m > 1 && (ld >= (int64_t(1) << 31) || (dlogits != nullptr && ld_d >= (int64_t(1) << 31)))) return BZ_ERR_UNSUPPORTED;
    return BZ_OK;
}

TokenArgs token_args(int64_t ld, int64_t v, int64_t ld_d, const int32_t* index, float temperature, const float* dloss, float* logp, float* stats) {
    TokenArgs a{};
    a.ld = ld, a.v = v, a.ld_d = ld_d, a.index = index, a.inv_t = 1.0 / static_cast<double>(temperature), a.temperature = temperature, a.c = kLog2e / temperature;
    a.dloss = dloss, a.logp = logp, a.stats = reinterpret_cast<float4*>(stats);
    return a;
}

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" int bz_policy(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, const float* old_logp,
                         const float* ref_logp, const float* advantage, float temperature, float clip_low, float clip_high, float kl,
                         const float* dloss, float* loss, float* logp, float* stats, void* dlogits, int64_t ld_d, void* stream) {
    if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl >= 0.f) || isinf(kl)) return BZ_ERR_INVALID_ARG;
    const int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK || m == 0) return st;
    if (advantage == nullptr || (kl != 0.f && ref_logp == nullptr) || (loss == nullptr && logp == nullptr && stats == nullptr && dlogits == nullptr))
        return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TokenArgs a = token_args(ld, v, ld_d, index, temperature, dloss, logp, stats);
    a.old_logp = old_logp, a.ref_logp = ref_logp, a.advantage = advantage, a.clip_low = clip_low, a.clip_high = clip_high, a.kl = kl, a.loss = loss;
    if (v == 0) {
        token_empty_kernel<<<kNumSMs, 256, 0, s>>>(m, loss, logp, a.stats);
        note_launch();
        return check_launch();
    }
    return dispatch(a, dtype, m, logits, dlogits, kPolicy, s);
}

extern "C" int bz_preference(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, const float* ref_logp,
                             const int32_t* starts, int64_t pairs, float temperature, float beta, float margin, float smoothing, int mean,
                             const float* dloss, float* loss, float* reward, float* logp, float* stats, void* dlogits, int64_t ld_d, void* stream) {
    if (pairs < 0 || !isfinite(beta) || !isfinite(margin) || !(smoothing >= 0.f && smoothing <= 1.f)) return BZ_ERR_INVALID_ARG;
    if (pairs >= (int64_t(1) << 30)) return BZ_ERR_UNSUPPORTED;
    int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK) return st;
    if ((pairs > 0 && starts == nullptr) || (m > 0 && stats == nullptr)) return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TokenArgs a = token_args(ld, v, ld_d, index, temperature, dloss, logp, stats);
    a.ref_logp = ref_logp;
    if (m > 0 && v == 0) {
        token_empty_kernel<<<kNumSMs, 256, 0, s>>>(m, nullptr, logp, a.stats);
        note_launch();
        st = check_launch();
    } else if (m > 0) {
        st = dispatch(a, dtype, m, logits, nullptr, kScore, s);
    }
    if (st != BZ_OK) return st;
    if (pairs > 0) {
        const PairArgs p{starts, m, v, pairs, beta, margin, smoothing, mean, loss, reward};
        pair_kernel<<<static_cast<unsigned>(pairs), 256, 0, s>>>(a, p, logits, dtype);
        note_launch();
        st = check_launch();
        if (st != BZ_OK) return st;
    }
    return m > 0 && v > 0 && dlogits != nullptr ? dispatch(a, dtype, m, logits, dlogits, kGradient, s) : BZ_OK;
}

extern "C" int bz_token_loss_backward(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, float temperature,
                                      const float* stats, const float* dloss, void* dlogits, int64_t ld_d, void* stream) {
    const int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK || m == 0 || v == 0) return st;
    if (stats == nullptr || dlogits == nullptr) return BZ_ERR_INVALID_ARG;
    return dispatch(token_args(ld, v, ld_d, index, temperature, dloss, nullptr, const_cast<float*>(stats)), dtype, m, logits, dlogits, kGradient,
                    static_cast<cudaStream_t>(stream));
}
