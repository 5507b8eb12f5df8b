// Losses that look at one token a position (clipped policy loss with a KL term, paired preference loss) and their gradient.
//
// Both rest on lp = z[a] - log(sum of exp z), z = logits / T, and on one number a row, the slope d loss / d lp:
// dlogits = dloss * slope / T * ([c == a] - softmax(z)[c]).
//
// Exponents are s c - R, one multiply-add: c = log2(e)/T rounded to binary32 and R the largest s c, rounded to binary32 and to a whole number, so that
// the multiply-add's rounding is the only one, and joining two parts of a row is exact.  The rounding of c is a temperature that differs by 2^-24 at
// most; the token's own logit goes by the same c, or the error would have one sign in all lp and a sum over a sequence would collect it.
// The largest's own exponent is what the rounding of R left: half a unit of the largest s c beyond 2^24.  So from 2^30 on (a row of a mask's
// fill, a peak) exponents are (s - largest) c; below, that exponent is 32 at most, and a sum of 2^31 terms fits.
#include <cooperative_groups.h>

#include "worker_common.cuh"

namespace bz {

namespace {

namespace cg = cooperative_groups;

constexpr int kTeam = 512;      // threads of a CTA at most
constexpr int kMostRanks = 8;   // CTAs of a cluster: the portable size

struct TokenArgs {
    int64_t m, ld, v, ld_d;
    const int32_t* index;
    Extent extent;            // of the logits
    float temperature, c;     // c = log2(e) / T
    const float *old_logp, *ref_logp, *advantage;
    float clip_low, clip_high, kl;
    const float* dloss;
    uint32_t places;          // of dloss, for the gradient alone
    float *loss, *logp;
    float4* stats;            // largest logit, sum of e^((s - that)/T) (negative: the token is likely), slope, place in dloss
};

__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }
// What the exponents of a row, or a part of it, are relative to.  A MaxSum here is the largest s and the sum of 2^(s c - R).
struct Base {
    float r, m;     // R; apart: the largest
    bool apart;
    __device__ __forceinline__ Base(const TokenArgs& a, float largest) {
        const float y = largest * a.c;
        m = largest, apart = !(fabsf(y) < 0x1p30f) && largest != -INFINITY;
        r = apart || largest == -INFINITY ? 0.f : rintf(y);
    }
    __device__ __forceinline__ float exponent(const TokenArgs& a, float s) const { return apart ? (s - m) * a.c : fmaf(s, a.c, -r); }
    // of a part's base, relative to this one, which has the larger s.  Where one of the two is apart and the other is not, they are a unit of a
    // number of 2^30 from one another at least, 2^6, and what the part adds is below 2^-64 of the sum.
    __device__ __forceinline__ float of(const TokenArgs& a, const Base& part) const { return !apart && !part.apart ? part.r - r : apart && part.apart ? (part.m - m) * a.c : -INFINITY; }
    // log2 of what the sum is relative to the largest itself
    __device__ __forceinline__ float rest(const TokenArgs& a) const { return apart || m == -INFINITY ? 0.f : fmaf(m, a.c, -r); }
};
__device__ __forceinline__ float2 powers(const TokenArgs& a, float2 s, float2 minus_r) {
    const float2 y = __ffma2_rn(s, pair(a.c), minus_r);
    return make_float2(exp2_fast(y.x), exp2_fast(y.y));
}
// The parts of a warp's lanes as one.
__device__ __forceinline__ MaxSum joined(const TokenArgs& a, const MaxSum& v) {
    const float m = warp_max(v.m);
    return {m, warp_sum(v.s == 0.f ? 0.f : v.s * exp2_fast(Base(a, m).of(a, Base(a, v.m))))};
}
// sum and the elements of x as one.
template <int K, int N> __device__ __forceinline__ void absorb(const TokenArgs& a, MaxSum& sum, const float (&x)[K][N]) {
    float top = sum.m;
#pragma unroll
    for (int j = 0; j < K; ++j) top = largest(top, x[j]);
    const Base base(a, top);
    float2 s0 = make_float2(sum.s == 0.f ? 0.f : sum.s * exp2_fast(base.of(a, Base(a, sum.m))), 0.f), s1 = pair(0.f);
    if (base.apart) {
        rare();
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < N; ++e) s0.x += exp2_fast(base.exponent(a, x[j][e]));
    } else {
        const float2 minus_r = pair(-base.r);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if constexpr (N == 1) {
                s0.x += exp2_fast(base.exponent(a, x[j][0]));
            } else {
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    s0 = __fadd2_rn(s0, powers(a, make_float2(x[j][e], x[j][e + 1]), minus_r));
                    s1 = __fadd2_rn(s1, powers(a, make_float2(x[j][e + 2], x[j][e + 3]), minus_r));
                }
            }
        }
    }
    s0 = __fadd2_rn(s0, s1);
    sum = {top, s0.x + s0.y};
}
// x = f 2^(exponents of x)
template <int N> __device__ __forceinline__ void scaled_powers(const TokenArgs& a, const Base& base, float f, float (&x)[N]) {
    if (base.apart) {
        rare();
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = f * exp2_fast(base.exponent(a, x[e]));
    } else if constexpr (N == 1) {
        x[0] = f * exp2_fast(base.exponent(a, x[0]));
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const float2 y = __fmul2_rn(powers(a, make_float2(x[e], x[e + 1]), pair(-base.r)), pair(f));
            x[e] = y.x, x[e + 1] = y.y;
        }
    }
}

// ex2.approx returns 2.2e-8 too little on average (measured over rows of normal logits: 1.9 to 2.5e-8), which a sum over a sequence would
// collect.
constexpr double kPowers = 1.0 + 2.2e-8;

// lp of a logit in a row of largest m, where the sum relative to 2^(m c + rest) is s.
__device__ __forceinline__ double log_probability(const TokenArgs& a, float logit, float m, double rest, double s) {
    if (logit == -INFINITY) return -INFINITY;
    return (static_cast<double>(logit) - static_cast<double>(m)) * static_cast<double>(a.c) * 0.6931471805599453094 + rest * 0.6931471805599453094 - log(s);
}
// Of a sum relative to R: s c - R = (s - m) c + (m c - R).
__device__ __forceinline__ double exact_rest(const TokenArgs& a, const Base& base) {
    return base.apart || base.m == -INFINITY ? 0.0 : static_cast<double>(base.m) * static_cast<double>(a.c) - static_cast<double>(base.r);
}

__device__ __forceinline__ bool has_token(const TokenArgs& a, int at) { return at >= 0 && at < a.v; }

// What one warp does of a row with a token, all lanes alike: its scalars.
struct RowInputs {
    float logit, old_logp, ref_logp, advantage, dloss;
};
template <bool POLICY> __device__ __forceinline__ RowInputs row_inputs(const TokenArgs& a, int64_t i, float logit) {
    RowInputs r{logit, 0.f, 0.f, 0.f, 1.f};
    if (POLICY) {
        if (a.old_logp != nullptr) r.old_logp = __ldg(a.old_logp + i);
        if (a.ref_logp != nullptr) r.ref_logp = __ldg(a.ref_logp + i);
        r.advantage = __ldg(a.advantage + i);
        if (a.dloss != nullptr) r.dloss = __ldg(a.dloss + i);
    }
    return r;
}
struct RowScalars {
    double lp, sum, rest;
    float loss, slope;
    float own;      // the token's exponential
    bool likely;    // more than half of the sum
    // of the gradient: g times (indicator of the token less softmax)
    __device__ __forceinline__ float factor(const TokenArgs& a, const RowInputs& in) const { return slope == 0.f ? 0.f : slope * in.dloss / a.temperature; }
    // at the token: g (1 - p) by what the sum has beside it, or a rounded p would leave its rounding
    __device__ __forceinline__ float at_token(float g, float sum_) const { return g == 0.f ? 0.f : g * ((sum_ - own) / sum_); }
};
template <bool POLICY> __device__ __forceinline__ RowScalars row_scalars(const TokenArgs& a, const RowInputs& in, const MaxSum& all) {
    const Base base(a, all.m);
    RowScalars s{0.0, static_cast<double>(all.s) * kPowers, exact_rest(a, base), 0.f, 0.f, exp2_fast(base.exponent(a, in.logit)), false};
    // A token that has most of the row goes by its own exponential, which is a term of the sum bit for bit (it is the largest, and its thread's
    // whole number was the row's): sums only grow, so lp is at most 0, and 0 where the others vanish beside it.  The correction is a mean over
    // many terms and has no place there.
    s.likely = in.logit == all.m && s.own > 0.5f * all.s;
    if (s.likely)
        s.lp = 0.0 - log1p((static_cast<double>(all.s) - static_cast<double>(s.own)) / static_cast<double>(s.own));
    else
        s.lp = log_probability(a, in.logit, all.m, s.rest, s.sum);
    if (POLICY) {
        // both exponentials at once: the ratio's on the even lanes, the KL term's on the odd ones
        const double shift = threadIdx.x & 1 ? static_cast<double>(in.ref_logp) - s.lp : s.lp - static_cast<double>(in.old_logp), e = expm1(shift);
        const double ratio = __shfl_sync(~0u, e, 0) + 1.0, back = __shfl_sync(~0u, shift, 1), grown = __shfl_sync(~0u, e, 1);
        const double adv = in.advantage, k = a.kl;
        double loss = 0.0, slope = 0.0;
        if (adv != 0.0) {   // a NaN goes on
            const double r = a.old_logp != nullptr ? ratio : 1.0;
            const double lo = 1.0 - static_cast<double>(a.clip_low), hi = 1.0 + static_cast<double>(a.clip_high);
            const bool held = adv > 0.0 ? r > hi : adv < 0.0 && r < lo;
            loss = -(held ? (adv > 0.0 ? hi : lo) : r) * adv;
            slope = held ? 0.0 : -r * adv;
        }
        if (k != 0.0) {
            loss += k * (isinf(grown) ? grown : grown - back);
            slope -= k * grown;
        }
        s.loss = static_cast<float>(loss), s.slope = s.lp == -INFINITY ? 0.f : static_cast<float>(slope);
    }
    return s;
}
// In the place of that rest: a row without a token.
constexpr float kNoToken = INFINITY;
// One thread.
__device__ __forceinline__ void write_row(const TokenArgs& a, int64_t i, const MaxSum& all, const RowScalars& s, bool policy) {
    if (policy && a.loss != nullptr) a.loss[i] = s.loss;
    // until a pair's slopes are known the last place holds what lp has beyond binary32
    const float lp = static_cast<float>(s.lp), rest = isfinite(lp) ? static_cast<float>(s.lp - static_cast<double>(lp)) : 0.f;
    if (a.logp != nullptr) a.logp[i] = lp;
    // a likely token is the largest itself; the sign tells the gradient's call
    const float sum = s.likely ? -all.s / s.own : static_cast<float>(s.sum * exp2(-s.rest));
    if (a.stats != nullptr) a.stats[i] = make_float4(all.m, sum, s.slope, policy ? __int_as_float(static_cast<int>(i)) : rest);
}
__device__ __forceinline__ void finish_without(const TokenArgs& a, int64_t i, bool policy) {
    if (a.logp != nullptr) a.logp[i] = 0.f;
    if (policy && a.loss != nullptr) a.loss[i] = 0.f;
    if (a.stats != nullptr) a.stats[i] = make_float4(-INFINITY, 0.f, 0.f, policy ? __int_as_float(static_cast<int>(i)) : kNoToken);
}

// ---- a row in a CTA's or a cluster's shared memory -----------------------------------------------
//
// A thread copies its own 16-byte words of the row (cp.async, up to four groups), takes each group into its largest logit and sum as it
// arrives, and with a gradient passes over them again out of shared memory: the row comes from memory once.  The row's maximum and
// sum cost one exchange, the scalars of its loss one warp in binary64.  Nothing of a row overlaps inside its CTA but the loads; three CTAs or
// more on an SM, each at another point of its row, do that.  4096 x 32128 bfloat16 with the gradient: 108 us, 81 at the copy's rate;
// issue slots 52 %, exponentials 61 %, two an element.  Of other forms, rows kept as exponentials in registers with the next one on its way (two
// CTAs an SM) took 148 us, rows through a ring with warps for each part of the work 170 (most of it bookkeeping of sixteen
// warps for rows of four chunks), the row read again out of the L2 129.

constexpr int kShared = 256;     // threads of a CTA at most
constexpr int kBatch = 4;        // words a thread works on at a time
constexpr int kMostWords = 227 * 1024 / 16 - 64;   // of a CTA

// All but the last LEFT groups of copies have arrived.
template <int LEFT> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

__device__ __forceinline__ void copy_word(uint32_t to, const char* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }

struct RowShare {
    int ranks, words;   // CTAs of a row; words of a CTA at most
};

// THREADS: of the CTA, or 0 for whatever it is launched with (the distances of a thread's words are constants in the long rows).
template <typename T, bool POLICY, bool GRADIENT, int THREADS>
__global__ void __launch_bounds__(kShared, 4) token_shared_kernel(const __grid_constant__ TokenArgs a, const RowShare share, const T* logits, T* dlogits) {
    constexpr int N = Word<T>::kN;
    extern __shared__ __align__(16) uint4 held[];
    __shared__ MaxSum part[16], peers[kMostRanks];
    __shared__ float4 outcome;   // the row's largest, the exponentials' factor, the gradient's, its entry at the token
    const int threads = THREADS ? THREADS : blockDim.x, t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const unsigned r = share.ranks == 1 ? blockIdx.x : blockIdx.x / static_cast<unsigned>(share.ranks);
    const int rank = static_cast<int>(blockIdx.x - r * share.ranks);
    const int64_t i = r;
    if (share.ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // every CTA of the cluster has started
    const int at = __ldg(a.index + i);
    const T* row = logits + i * a.ld;
    const int n = static_cast<int>(a.v), lead = row_lead<T, N>(row);
    // this CTA's words [begin, begin + count) of the row's, counted from the 16-byte boundary at or before it; this thread's: t, t + threads, ...
    const int all = (lead + n + N - 1) / N, begin = rank * share.words, count = min(share.words, all - begin);
    // words over an end of the row: places in the CTA, -1: elsewhere
    const int head = lead != 0 && begin == 0 ? 0 : -1, tail = (lead + n) % N != 0 && begin + count == all ? count - 1 : -1;
    // batches, and those without any of these and without words behind the last
    const int batches = (count + kBatch * threads - 1) / (kBatch * threads), stride = threads * 16, plain_from = head >= 0, plain_to = (count - (tail >= 0)) / (kBatch * threads);
    const bool there = has_token(a, at);
    float g = 0.f, f = 0.f, top = 0.f, hot = 0.f;
    if (there) {
        const char* from = reinterpret_cast<const char*>(row - lead) + (begin + t) * int64_t(16);
        uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(held + t));
        for (int b = 0, w = t; b < batches; ++b, w += kBatch * threads, from += kBatch * stride, to += kBatch * stride) {
            if (b >= plain_from && b < plain_to) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) copy_word(to + j * stride, from + j * stride);
            } else {
                rare();
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (const int v = w + j * threads; v < count && v != head && v != tail) copy_word(to + j * stride, from + j * stride);
            }
            if (b < 3 || b + 1 == batches) asm volatile("cp.async.commit_group;" ::: "memory");
        }
        RowInputs in{};
        if (warp == 0) in = row_inputs<POLICY>(a, i, to_f32(row[at]));
        // -inf in what was not copied: words behind the CTA's last, elements that are not the row's
        for (int b = 0; b < batches; ++b) {
            if (b >= plain_from && b < plain_to) continue;
            for (int w = b * kBatch * threads + t, j = 0; j < kBatch; ++j, w += threads) {
                if (w < count && w != head && w != tail) continue;
                float x[N];
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = -INFINITY;
                if (w < count) load_slot<T, N>(row, static_cast<int64_t>(begin + w) * N - lead, n, -INFINITY, x);
                held[w] = Word<T>::pack(x);
            }
        }
        MaxSum sum{-INFINITY, 0.f};
        const char* word = reinterpret_cast<const char*>(held + t);
#pragma unroll 1
        for (int b = 0; b < batches; ++b) {
            // groups: a batch each, the fourth all that are left
            switch (min(batches, 4) - 1 - b) {
                case 3: wait_copies<3>(); break;
                case 2: wait_copies<2>(); break;
                case 1: wait_copies<1>(); break;
                default: wait_copies<0>();
            }
            float x[kBatch][N];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) Word<T>::unpack(*reinterpret_cast<const uint4*>(word + j * stride), x[j]);
            word += kBatch * stride;
            absorb(a, sum, x);
        }
        sum = joined(a, sum);
        if (lane == 0) part[warp] = sum;
        __syncthreads();
        if (share.ranks > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (warp == 0) {
                sum = joined(a, lane < (threads >> 5) ? part[lane] : MaxSum{-INFINITY, 0.f});
                if (lane < share.ranks) *cluster.map_shared_rank(&peers[rank], lane) = sum;
            }
            cluster.sync();
        }
        RowScalars scalars{};
        if (warp == 0) {
            sum = joined(a, share.ranks > 1 ? (lane < share.ranks ? peers[lane] : MaxSum{-INFINITY, 0.f}) : (lane < (threads >> 5) ? part[lane] : MaxSum{-INFINITY, 0.f}));
            scalars = row_scalars<POLICY>(a, in, sum);
            if (GRADIENT) {
                const float got = scalars.factor(a, in);
                if (lane == 0) outcome = make_float4(sum.m, got == 0.f ? 0.f : -got / sum.s, got, scalars.at_token(got, sum.s));
            }
        }
        if (GRADIENT) __syncthreads();
        if (t == 0 && rank == 0) write_row(a, i, sum, scalars, POLICY);
        if (!GRADIENT) return;
        top = outcome.x, f = outcome.y, g = outcome.z, hot = outcome.w;
    } else {
        if (share.ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (t == 0 && rank == 0) finish_without(a, i, POLICY);
        if (!GRADIENT) return;
    }
    const Base base(a, top);
    T* out = dlogits + i * a.ld_d;
    char* to = reinterpret_cast<char*>(out - lead) + (begin + t) * int64_t(16);
    const char* word = reinterpret_cast<const char*>(held + t);
    if (g == 0.f) {
        for (int w = t; w < count; w += threads, to += stride)
            if (w != head && w != tail) *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
    } else {
#pragma unroll 1
        for (int b = 0, w = t; b < batches; ++b, w += kBatch * threads, word += kBatch * stride, to += kBatch * stride) {
            float x[kBatch][N];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) Word<T>::unpack(*reinterpret_cast<const uint4*>(word + j * stride), x[j]);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) scaled_powers(a, base, f, x[j]);
            if (b >= plain_from && b < plain_to) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) *reinterpret_cast<uint4*>(to + j * stride) = Word<T>::pack(x[j]);
            } else {
                rare();
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (const int v = w + j * threads; v < count && v != head && v != tail) *reinterpret_cast<uint4*>(to + j * stride) = Word<T>::pack(x[j]);
            }
        }
    }
    for (int which = 0; which < 2; ++which) {
        const int w = which == 0 ? head : tail == head ? -1 : tail;
        if (w < 0 || w % threads != t) continue;
        float x[N];
        Word<T>::unpack(held[w], x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = g == 0.f ? 0.f : exp2_fast(base.exponent(a, x[e])) * f;
        store_slot<T, N>(out, static_cast<int64_t>(begin + w) * N - lead, n, x);
    }
    if (g != 0.f) {   // the token's place, once more, by the thread that has just written it
        const int w = (at + lead) / N - begin;
        if (w >= 0 && w < count && w % threads == t) out[at] = from_f32<T>(hot);
    }
}

// ---- the loss alone, many rows: one CTA a row, words from memory into registers ------------------
//
// Nothing of the row has to stay, so a row of any length takes one CTA and three of them an SM; a thread has its next four words on their
// way while it takes four in.  1531 x 65537 binary16: 47 us (31 at the copy's rate), 60 through shared memory and clusters; rows of 64 KB and
// less are as fast there (57 us at 4096 x 32128) or faster (8192 x 8000: 33 against 57).

constexpr int kScoreThreads = 256;
template <typename T, bool POLICY> __global__ void __launch_bounds__(kScoreThreads, 3) token_score_kernel(const __grid_constant__ TokenArgs a, const T* logits) {
    constexpr int N = Word<T>::kN;
    __shared__ MaxSum part[kScoreThreads / 32];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int64_t i = blockIdx.x;
    const int at = __ldg(a.index + i);
    if (!has_token(a, at)) {
        if (t == 0) finish_without(a, i, POLICY);
        return;
    }
    const T* row = logits + i * a.ld;
    const int n = static_cast<int>(a.v), lead = row_lead<T, N>(row), all = (lead + n + N - 1) / N;
    const int head = lead != 0 ? 0 : -1, tail = (lead + n) % N != 0 ? all - 1 : -1;   // words over an end of the row
    const int batches = (all + kBatch * kScoreThreads - 1) / (kBatch * kScoreThreads);
    const uint4* from = reinterpret_cast<const uint4*>(row - lead) + t;
    auto plain = [&](int b) { return (b > 0 || head < 0) && (b + 1) * kBatch * kScoreThreads <= all - (tail >= 0); };
    uint4 next[kBatch];
    auto fetch = [&](int b) {
        if (plain(b)) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) next[j] = __ldg(from + (b * kBatch + j) * kScoreThreads);
        } else {
            rare();
            float x[N];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int w = (b * kBatch + j) * kScoreThreads + t;
                if (w < all && w != head && w != tail) {
                    next[j] = __ldg(from + (b * kBatch + j) * kScoreThreads);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) x[e] = -INFINITY;
                    if (w < all) load_slot<T, N>(row, static_cast<int64_t>(w) * N - lead, n, -INFINITY, x);
                    next[j] = Word<T>::pack(x);
                }
            }
        }
    };
    fetch(0);
    RowInputs in{};
    if (warp == 0) in = row_inputs<POLICY>(a, i, to_f32(row[at]));
    MaxSum sum{-INFINITY, 0.f};
#pragma unroll 1
    for (int b = 0; b < batches; ++b) {
        float x[kBatch][N];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) Word<T>::unpack(next[j], x[j]);
        if (b + 1 < batches) fetch(b + 1);
        absorb(a, sum, x);
    }
    sum = joined(a, sum);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (warp != 0) return;
    sum = joined(a, lane < kScoreThreads / 32 ? part[lane] : MaxSum{-INFINITY, 0.f});
    const RowScalars scalars = row_scalars<POLICY>(a, in, sum);
    if (lane == 0) write_row(a, i, sum, scalars, POLICY);
}

// ---- any length and layout: the row is read twice -----------------------------------------------------------

// The largest of a row and its sum of exponentials, over the CTA.
template <typename T, int VEC> __device__ __forceinline__ MaxSum row_statistics(const TokenArgs& a, const T* row, MaxSum* part) {
    MaxSum mine{-INFINITY, 0.f};
    for (int64_t j0 = static_cast<int64_t>(threadIdx.x) * VEC - row_lead<T, VEC>(row); j0 < a.v; j0 += blockDim.x * VEC) {
        float x[1][VEC];
        load_slot<T, VEC>(row, j0, a.v, -INFINITY, x[0]);
        absorb(a, mine, x);
    }
    mine = joined(a, mine);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = mine;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return joined(a, lane < (blockDim.x >> 5) ? part[lane] : MaxSum{-INFINITY, 0.f});
}

// One CTA a row.  POLICY: the loss too, and the gradient if it is wanted; otherwise lp and stats alone.
template <typename T, int VEC, bool POLICY> __global__ void __launch_bounds__(kTeam) token_rows_kernel(const __grid_constant__ TokenArgs a, const T* logits, T* dlogits) {
    __shared__ MaxSum part[32];
    __shared__ float2 factor;   // of the gradient, its entry at the token
    const int64_t i = blockIdx.x;
    const T* row = logits + i * a.ld;
    const int at = a.index[i];
    const bool there = has_token(a, at);
    MaxSum all{-INFINITY, 0.f};
    if (there) all = row_statistics<T, VEC>(a, row, part);
    if (threadIdx.x < 32) {
        float2 g = pair(0.f);
        if (there) {
            const RowInputs in = row_inputs<POLICY>(a, i, to_f32(row[at]));
            const RowScalars scalars = row_scalars<POLICY>(a, in, all);
            g.x = scalars.factor(a, in), g.y = scalars.at_token(g.x, all.s);
            if (threadIdx.x == 0) write_row(a, i, all, scalars, POLICY);
        } else if (threadIdx.x == 0) {
            finish_without(a, i, POLICY);
        }
        if (threadIdx.x == 0) factor = g;
    }
    if (!POLICY || dlogits == nullptr) return;
    __syncthreads();
    const float g = factor.x, hot = factor.y, f = g == 0.f ? 0.f : -g / all.s;
    const Base base(a, all.m);
    T* out = dlogits + i * a.ld_d;
    for (int64_t j0 = static_cast<int64_t>(threadIdx.x) * VEC - row_lead<T, VEC>(row); j0 < a.v; j0 += blockDim.x * VEC) {
        float x[VEC];
        load_slot<T, VEC>(row, j0, a.v, -INFINITY, x);
#pragma unroll
        for (int k = 0; k < VEC; ++k) x[k] = g == 0.f ? 0.f : j0 + k == at ? hot : exp2_fast(base.exponent(a, x[k])) * f;
        store_slot<T, VEC>(out, j0, a.v, x);
    }
}

// ---- the gradient from given stats ---------------------------------------------------------------

// What comes from above for a row whose place in dloss is `place`.
__device__ __forceinline__ float upstream(const TokenArgs& a, float place) {
    const uint32_t k = __float_as_uint(place);
    return a.dloss == nullptr ? 1.f : k < a.places ? a.dloss[k] : NAN;
}

// CTA (row, share): shares of kGradientColumns elements a thread; the last rows first, as far as the L2 still holds them.  4096 x 32128
// bfloat16: 85 us, 96 % of the copy's rate.  (Stores that leave the L2 first, to keep more of the logits there: 95 us.)
constexpr int kGradientThreads = 256, kGradientColumns = 32;
template <typename T, int VEC, int THREADS>
__global__ void __launch_bounds__(kGradientThreads) token_gradient_kernel(const __grid_constant__ TokenArgs a, const T* logits, T* dlogits, int shares) {
    constexpr int kSlots = kGradientColumns / VEC;
    const int threads = THREADS ? THREADS : blockDim.x;
    const unsigned k = gridDim.x - 1 - blockIdx.x, r = shares == 1 ? k : k / static_cast<unsigned>(shares);
    const int64_t i = r;
    const T* row = logits + i * a.ld;
    T* out = dlogits + i * a.ld_d;
    const int n = static_cast<int>(a.v);
    // places of this thread's first elements: below 2^31, as v and a share more are
    const int base = static_cast<int>((k - r * shares) * (threads * kGradientColumns)) + static_cast<int>(threadIdx.x) * VEC - row_lead<T, VEC>(row);
    auto first = [&](int q) { return base + q * threads * VEC; };
    Raw<T, VEC> raw[kSlots];
    const bool safe = a.extent.around(row, a.v);
    auto whole = [&](int j0) { return j0 < n && (safe || (j0 >= 0 && j0 + VEC <= n)); };
#pragma unroll
    for (int q = 0; q < kSlots; ++q) raw[q].fetch(row + first(q), whole(first(q)));
    const float4 st = a.stats[i];
    const int at = a.index[i];
    const float g = st.z == 0.f || !has_token(a, at) ? 0.f : st.z * upstream(a, st.w) / a.temperature, sum = fabsf(st.y);
    const Base reference(a, st.x);
    const float f = g == 0.f ? 0.f : -g / sum * exp2_fast(-reference.rest(a));
#pragma unroll
    for (int q = 0; q < kSlots; ++q) {
        const int j0 = first(q);
        if (j0 >= n) continue;
        float x[VEC];
        raw[q].get(x);
        if (!whole(j0)) read_apart<T, VEC>(row, j0, n, x);
        scaled_powers(a, reference, f, x);
        if (g == 0.f) {
            rare();
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = 0.f;
        }
        if (static_cast<unsigned>(at - j0) < static_cast<unsigned>(VEC)) {
            rare();
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j0 + e == at) x[e] += g;
        }
        store_slot<T, VEC>(out, j0, n, x);
    }
    if (st.y < 0.f && g != 0.f) {   // a likely token's entry once more, by the thread that has just written it
        rare();
        const unsigned from = static_cast<unsigned>(at - base), slot = static_cast<unsigned>(threads * VEC);
        if (from / slot < kSlots && from % slot < VEC) out[at] = from_f32<T>(g * ((sum - 1.f) / sum));
    }
}

struct PairArgs {
    const int32_t* starts;
    int64_t m, pairs;
    float beta, margin, smoothing;
    int mean;
    float *loss, *reward;
};

// One CTA a pair, a half of it each sequence: the sums, the loss and each row's slope.  lp comes as it was stored and what it has beyond
// binary32, so that a row costs two independent loads and no logarithm (forming it anew from the logit took 8 us of a call, now 3).
constexpr int kPairThreads = 1024, kHalf = kPairThreads / 2;
__global__ void __launch_bounds__(kPairThreads) pair_kernel(const __grid_constant__ TokenArgs a, const __grid_constant__ PairArgs p) {
    __shared__ double sums[2][kHalf / 32];
    __shared__ int counts[2][kHalf / 32];
    const int64_t pair = blockIdx.x;
    const int side = threadIdx.x / kHalf, t = threadIdx.x % kHalf, lane = t & 31, warp = t >> 5;
    const int64_t n = pair + side * p.pairs;
    const int64_t from = min(max(static_cast<int64_t>(p.starts[n]), int64_t(0)), p.m), to = max(from, min(static_cast<int64_t>(p.starts[n + 1]), p.m));
    double sum = 0.0;
    int count = 0;
#pragma unroll 4
    for (int64_t i = from + t; i < to; i += kHalf) {
        const float rest = a.stats[i].w, lp = a.logp[i], ref = a.ref_logp != nullptr ? a.ref_logp[i] : 0.f;
        if (rest != kNoToken) sum += static_cast<double>(lp) + static_cast<double>(rest) - static_cast<double>(ref), ++count;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o), count += __shfl_xor_sync(~0u, count, o);
    if (lane == 0) sums[side][warp] = sum, counts[side][warp] = count;
    __syncthreads();
    double reward[2], share[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        sum = 0.0, count = 0;
#pragma unroll
        for (int w = 0; w < kHalf / 32; ++w) sum += sums[k][w], count += counts[k][w];
        share[k] = static_cast<double>(p.beta) / (p.mean ? max(count, 1) : 1);
        reward[k] = share[k] * sum;
    }
    const double h = reward[0] - reward[1] - static_cast<double>(p.margin), eps = p.smoothing;
    const double e = exp(-fabs(h));
    // d loss / d h = sigmoid(h) - (1 - eps); sigmoid(h) = 1 - sigmoid(-h) for the digits of the smaller one
    const double small = e / (1.0 + e);
    const double dh = h >= 0.0 ? eps - small : h < 0.0 ? small - (1.0 - eps) : NAN;
    const float slope = static_cast<float>(side == 0 ? dh * share[0] : -dh * share[1]);
    for (int64_t i = from + t; i < to; i += kHalf) {
        float4* st = a.stats + i;
        const bool takes = st->w != kNoToken && a.logp[i] != -INFINITY;
        reinterpret_cast<float2*>(st)[1] = make_float2(takes ? slope : 0.f, __int_as_float(static_cast<int>(pair)));
    }
    if (threadIdx.x == 0) {
        const double tail = log1p(e);   // -log sigmoid(|h|)
        // a weight of 0 has no term, whatever its logarithm
        const double up = tail + fmax(-h, 0.0), down = tail + fmax(h, 0.0);
        if (p.loss != nullptr) p.loss[pair] = isnan(h) ? NAN : static_cast<float>((eps != 1.0 ? (1.0 - eps) * up : 0.0) + (eps != 0.0 ? eps * down : 0.0));
        if (p.reward != nullptr) p.reward[pair] = static_cast<float>(reward[0]), p.reward[pair + p.pairs] = static_cast<float>(reward[1]);
    }
}

// v == 0: rows without a token.
__global__ void token_empty_kernel(int64_t m, float* loss, float* logp, float4* stats, bool policy) {
    for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < m; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        if (loss != nullptr) loss[i] = 0.f;
        if (logp != nullptr) logp[i] = 0.f;
        if (stats != nullptr) stats[i] = make_float4(-INFINITY, 0.f, 0.f, policy ? __int_as_float(static_cast<int>(i)) : kNoToken);
    }
}

// ---- host side ----------------------------------------------------------------------------------

enum What { kPolicy, kScore, kGradient };

// Threads for a CTA's words: a warp up to 640, 128 threads up to 2048, else 256; where few rows leave SMs idle, four words each.  (Policy
// loss with its gradient, bfloat16: 8192 rows of 2000 with a warp 22.6 us, with two 26.9; of 4096 42, 49; 8192 x 8000 with 128 threads 57, with two
// warps 66, with 256 threads 80.)
int threads_for(int words, bool few) {
    const int quarter = (words + 127) / 128 * 32;
    if (few) return quarter < kShared ? quarter : kShared;
    return words <= 640 ? 32 : words <= 2048 ? 128 : 256;
}
// Words that they take in, those behind the last ones among them.
int in_batches(int words, int threads) { return (words + threads * kBatch - 1) / (threads * kBatch) * (threads * kBatch); }
// CTAs of a long row, parts of 1024 to 2048 words where it has them: what leaves the fewest words behind the last ones, and the more CTAs
// of two like that.  2048 x 50257 bfloat16 in 5 parts of 1257 words 106 us, in 4 of 1571 (2048 with the empty ones) 115, in 7 of 898 113.
int ranks_for(int64_t words) {
    const int64_t most = words <= 2048 * kMostRanks ? 2048 : 4096;
    int best = kMostRanks;
    int64_t least = INT64_MAX;
    for (int r = 2; r <= kMostRanks; ++r) {
        const int64_t part = (words + r - 1) / r;
        if (part < 1024 || part > most) continue;
        const int64_t all = static_cast<int64_t>(r) * in_batches(static_cast<int>(part), threads_for(static_cast<int>(part), false));
        if (all <= least) least = all, best = r;
    }
    return best;
}

template <typename T, bool POLICY, bool GRADIENT> int shared(const TokenArgs& a, const T* logits, T* dlogits, int64_t words, int ranks, cudaStream_t s) {
    const RowShare share{ranks, static_cast<int>((words + ranks - 1) / ranks)};
    const int threads = threads_for(share.words, a.m * ranks <= kNumSMs);
    auto kern = threads == 256 ? token_shared_kernel<T, POLICY, GRADIENT, 256> : threads == 128 ? token_shared_kernel<T, POLICY, GRADIENT, 128> : token_shared_kernel<T, POLICY, GRADIENT, 0>;
    const int smem = in_batches(share.words, threads) * 16;
    cudaError_t e = cudaSuccess;
    // up to 48 KB need no leave; beyond, the limit belongs to the kernel and not to the call: the same one each time
    if (smem > 48 * 1024 - 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostWords * 16);
    if (e != cudaSuccess) return cuda_failed(e);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(a.m * ranks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kern, a, share, logits, dlogits);
    if (e != cudaSuccess) return cuda_failed(e);
    note_launch();
    return check_launch();
}

// Rows, and words of a row, from which the loss alone takes its own kernel.
constexpr int64_t kScoreRows = 2 * kNumSMs, kScoreWords = 4096;

template <typename T, int VEC, bool POLICY> int rows(const TokenArgs& a, const T* logits, T* dlogits, cudaStream_t s) {
    if constexpr (VEC > 1) {
        const int64_t words = (a.v + 2 * (VEC - 1)) / VEC;   // of a row, at most
        const bool score = dlogits == nullptr && a.m >= kScoreRows && words > kScoreWords;
        // a cluster's CTAs hold what they can of the longest rows
        int64_t ranks = words <= 4096 ? 1 : ranks_for(words);
        while (ranks < kMostRanks && a.m * ranks * 2 <= kNumSMs && words > ranks * 256) ranks *= 2;   // few rows: on more SMs
        if (ranks > kMostRanks) ranks = kMostRanks;
        if ((words + ranks - 1) / ranks + kBatch * kShared <= kMostWords && a.m * ranks < (int64_t(1) << 31)) {
            if constexpr (POLICY)
                if (dlogits != nullptr) return shared<T, true, true>(a, logits, dlogits, words, static_cast<int>(ranks), s);
            if (score) {
                token_score_kernel<T, POLICY><<<static_cast<unsigned>(a.m), kScoreThreads, 0, s>>>(a, logits);
                note_launch();
                return check_launch();
            }
            return shared<T, POLICY, false>(a, logits, dlogits, words, static_cast<int>(ranks), s);
        }
    }
    token_rows_kernel<T, VEC, POLICY><<<static_cast<unsigned>(a.m), kTeam, 0, s>>>(a, logits, dlogits);
    note_launch();
    return check_launch();
}

template <typename T, int VEC> int launch(const TokenArgs& a, const T* logits, T* dlogits, What what, cudaStream_t s) {
    if (what == kPolicy) return rows<T, VEC, true>(a, logits, dlogits, s);
    if (what == kScore) return rows<T, VEC, false>(a, logits, dlogits, s);
    const int64_t each = (a.v + (VEC - 1) + kGradientColumns - 1) / kGradientColumns;   // threads for a row
    const int threads = static_cast<int>(each < kGradientThreads ? (each + 31) / 32 * 32 : kGradientThreads);
    const int64_t shares = (each + threads - 1) / threads;
    if (a.m * shares >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    auto kern = threads == kGradientThreads ? token_gradient_kernel<T, VEC, kGradientThreads> : token_gradient_kernel<T, VEC, 0>;
    kern<<<static_cast<unsigned>(a.m * shares), threads, 0, s>>>(a, logits, dlogits, static_cast<int>(shares));
    note_launch();
    return check_launch();
}

template <typename T> int dispatch(const TokenArgs& a, int64_t m, const void* logits, void* dlogits, What what, cudaStream_t s) {
    const T* in = static_cast<const T*>(logits);
    T* out = static_cast<T*>(dlogits);
    const uintptr_t apart = reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(dlogits);
    const bool alike = out == nullptr || ((apart & 15) == 0 && (m == 1 || ((a.ld - a.ld_d) * static_cast<int64_t>(sizeof(T))) % 16 == 0));
    return alike ? launch<T, Word<T>::kN>(a, in, out, what, s) : launch<T, 1>(a, in, out, what, s);
}

int dispatch(const TokenArgs& a, int dtype, int64_t m, const void* logits, void* dlogits, What what, cudaStream_t s) {
    if (dtype == BZ_F32) return dispatch<float>(a, m, logits, dlogits, what, s);
    if (dtype == BZ_F16) return dispatch<__half>(a, m, logits, dlogits, what, s);
    return dispatch<__nv_bfloat16>(a, m, logits, dlogits, what, s);
}

// binary32 and int32 arrays lie on their type's boundary
template <typename... P> bool on_boundary(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 3u) == 0; }

int check(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, float temperature, const void* stats, const void* dlogits, int64_t ld_d) {
    const int bytes = element_bytes(dtype);
    if (bytes == 0 || m < 0 || v < 0 || !(temperature > 0.f) || isinf(temperature) || isinf(kLog2e / temperature) || !aligned16(stats)) return BZ_ERR_INVALID_ARG;
    if (v > (int64_t(1) << 31) - 16384 || m >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    if (m == 0) return BZ_OK;
    if (index == nullptr) return BZ_ERR_INVALID_ARG;
    if (v == 0) return BZ_OK;
    if (logits == nullptr || (m > 1 && ld < v) || reinterpret_cast<uintptr_t>(logits) % bytes) return BZ_ERR_INVALID_ARG;
    if (dlogits != nullptr && ((m > 1 && ld_d < v) || reinterpret_cast<uintptr_t>(dlogits) % bytes)) return BZ_ERR_INVALID_ARG;
    if (m > 1 && (ld >= (int64_t(1) << 31) || (dlogits != nullptr && ld_d >= (int64_t(1) << 31)))) return BZ_ERR_UNSUPPORTED;
    return BZ_OK;
}

TokenArgs token_args(const void* logits, int dtype, int64_t m, int64_t ld, int64_t v, int64_t ld_d, const int32_t* index, float temperature, const float* dloss, float* logp, float* stats) {
    TokenArgs a{};
    a.ld = ld, a.v = v, a.ld_d = ld_d, a.index = index, a.temperature = temperature;
    a.m = m;
    const char* p = static_cast<const char*>(logits);
    a.extent = {p, p + ((m - 1) * ld + v) * element_bytes(dtype)};
    a.c = static_cast<float>(1.4426950408889634 / static_cast<double>(temperature));
    a.dloss = dloss, a.logp = logp, a.stats = reinterpret_cast<float4*>(stats);
    return a;
}

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" int bz_policy(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, const float* old_logp,
                         const float* ref_logp, const float* advantage, float temperature, float clip_low, float clip_high, float kl,
                         const float* dloss, float* loss, float* logp, float* stats, void* dlogits, int64_t ld_d, void* stream) {
    if (!on_boundary(index, old_logp, ref_logp, advantage, dloss, loss, logp) || !(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl >= 0.f) || isinf(kl)) return BZ_ERR_INVALID_ARG;
    const int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK || m == 0) return st;
    if (advantage == nullptr || (kl != 0.f && ref_logp == nullptr) || (loss == nullptr && logp == nullptr && stats == nullptr && dlogits == nullptr))
        return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TokenArgs a = token_args(logits, dtype, m, ld, v, ld_d, index, temperature, dloss, logp, stats);
    a.old_logp = old_logp, a.ref_logp = ref_logp, a.advantage = advantage, a.clip_low = clip_low, a.clip_high = clip_high, a.kl = kl, a.loss = loss;
    if (v == 0) {
        token_empty_kernel<<<kNumSMs, 256, 0, s>>>(m, loss, logp, a.stats, true);
        note_launch();
        return check_launch();
    }
    return dispatch(a, dtype, m, logits, dlogits, kPolicy, s);
}

extern "C" int bz_preference(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, const float* ref_logp,
                             const int32_t* starts, int64_t pairs, float temperature, float beta, float margin, float smoothing, int mean,
                             const float* dloss, float* loss, float* reward, float* logp, float* stats, void* dlogits, int64_t ld_d, void* stream) {
    if (!on_boundary(index, ref_logp, starts, dloss, loss, reward, logp) || pairs < 0 || !isfinite(beta) || !isfinite(margin) || !(smoothing >= 0.f && smoothing <= 1.f)) return BZ_ERR_INVALID_ARG;
    if (pairs >= (int64_t(1) << 30)) return BZ_ERR_UNSUPPORTED;
    int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK) return st;
    if ((pairs > 0 && starts == nullptr) || (m > 0 && (stats == nullptr || logp == nullptr))) return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TokenArgs a = token_args(logits, dtype, m, ld, v, ld_d, index, temperature, dloss, logp, stats);
    a.ref_logp = ref_logp, a.places = static_cast<uint32_t>(pairs);
    if (m > 0 && v == 0) {
        token_empty_kernel<<<kNumSMs, 256, 0, s>>>(m, nullptr, logp, a.stats, false);
        note_launch();
        st = check_launch();
    } else if (m > 0) {
        st = dispatch(a, dtype, m, logits, nullptr, kScore, s);
    }
    if (st != BZ_OK) return st;
    if (pairs > 0) {
        const PairArgs p{starts, m, pairs, beta, margin, smoothing, mean, loss, reward};
        pair_kernel<<<static_cast<unsigned>(pairs), kPairThreads, 0, s>>>(a, p);
        note_launch();
        st = check_launch();
        if (st != BZ_OK) return st;
    }
    return m > 0 && v > 0 && dlogits != nullptr ? dispatch(a, dtype, m, logits, dlogits, kGradient, s) : BZ_OK;
}

extern "C" int bz_token_loss_backward(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const int32_t* index, float temperature,
                                      const float* stats, const float* dloss, int64_t places, void* dlogits, int64_t ld_d, void* stream) {
    if (!on_boundary(index, dloss) || (dloss != nullptr && places < 0)) return BZ_ERR_INVALID_ARG;
    const int st = check(logits, ld, dtype, m, v, index, temperature, stats, dlogits, ld_d);
    if (st != BZ_OK || m == 0 || v == 0) return st;
    if (stats == nullptr || dlogits == nullptr) return BZ_ERR_INVALID_ARG;
    TokenArgs a = token_args(logits, dtype, m, ld, v, ld_d, index, temperature, dloss, nullptr, const_cast<float*>(stats));
    a.places = static_cast<uint32_t>(places < (int64_t(1) << 31) ? places : int64_t(1) << 31);
    return dispatch(a, dtype, m, logits, dlogits, kGradient, static_cast<cudaStream_t>(stream));
}
