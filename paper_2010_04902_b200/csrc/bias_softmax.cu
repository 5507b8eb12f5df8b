// Softmax of attention scores with a learned relative position bias, and its gradient.
//
// Forward: z = scale*s + bias[bucket(j - p)], P = e^(z - M) / S.  One read of the scores, one write of P: bound by memory
// (8 x 16 x 1024 x 1024 bfloat16 in 87 us, 94 % of the copy's rate; causal 2 x 16 x 4096 x 4096 in 380, bound by issue).
// A row lies in the registers of G threads (a warp, then 64 to 512 threads; 32 16-bit elements each, 16 of binary32 or where
// rows are taken element by element), the next row's loads are on their way while this one is worked on, and a warp takes
// its exponentials relative to its own maximum, so that one exchange of (maximum, sum) pairs a row is all that a CTA's
// warps need.  Rows of more than 16 384 keys (8192 at 16 elements a thread; the gradient's kernels, up to 256 threads: 8192
// and 4096) are read twice.
// The bias depends on j - p alone and is constant from max_distance on, so a CTA keeps the head's values for the
// 2*max_distance + 1 distances in shared memory, in copies that make a slot's values whole words (struct Window).
//
// Backward: p from the kept maximum and sum, D = sum p dp, dz = p (dp - D).  The table's gradient needs the sum of dz over
// each diagonal of the scores inside the window and one sum for either side beyond it.  A warp owns a private array
// of diagonals: a row meets each diagonal once, so its lanes add without conflict, row after row, in a fixed order;
// the far sums stay in registers.  CTAs leave one value a bucket and a last kernel adds those in order.  Three transfers an
// element; 176 us at 8 x 16 x 1024 x 1024 (70 % of the copy's rate): 22 instructions an element are what is left to cut.
#include <algorithm>

#include "bucket_rule.h"
#include "worker_common.cuh"

namespace bz {

namespace {

constexpr int kMaxStarts = 128;  // nb - nb/2 with nb up to 256

struct BiasForm {
    const float* table;
    const int32_t *k_len, *q_start;
    float scale;
    int buckets, nb, exact, distance, bidirectional, causal;
    int h;
    int64_t tq, tk;
    int rows_per_cta;
    uint16_t starts[kMaxStarts];  // starts[t]: smallest distance of bucket exact + t
};

template <typename T> struct Rows4 {  // a [b][h][tq][tk] tensor
    T* p;
    int64_t b, h, q;
    Extent extent;
    __device__ T* row(int64_t ib, int64_t ih, int64_t iq) const { return p + ib * b + ih * h + iq * q; }
};

__device__ __forceinline__ int bucket_of(const BiasForm& f, int rel) {
    const int n = f.bidirectional ? abs(rel) : max(-rel, 0);
    int c = n;
    if (n >= f.exact) {
        c = f.exact;
        for (int t = 1; t < f.nb - f.exact; ++t) c += n >= f.starts[t];
    }
    return f.bidirectional && rel > 0 ? c + f.nb : c;
}

// The head's bias by distance in shared memory, for slots of VEC keys.  A slot that begins at relative position rel needs
// the values of distances rel .. rel + VEC - 1; with rel + max_distance = VEC*b + a (0 <= a < VEC) these are VEC consecutive
// values from VEC*b + a on, ends repeated outside.  Copy a of the table is laid out so that they are whole 16-byte words:
// b runs from -2 to `last`, where all VEC values are an end's, so a slot beyond the window is clamped to one of those and
// nothing branches.  The four-value groups of a slot lie in different halves: neighbouring lanes read neighbouring words.
template <int VEC> struct Window {
    static constexpr int kGroups = VEC / 4 > 0 ? VEC / 4 : 1, kIn = VEC / kGroups;
    int slots;   // per copy
    // VEC == 1: rounded up to whole 16-byte words
    __host__ __device__ explicit Window(int distance) : slots(VEC == 1 ? (2 * distance + 6) / 4 * 4 : (2 * distance + VEC - 1) / VEC + 3) {}
    __host__ __device__ int floats() const { return VEC * slots * VEC; }
    // value indices run over [-2*VEC, values() - 2*VEC)
    __host__ __device__ int values() const { return VEC * (slots + 1); }
    __device__ __forceinline__ int at(int a, int slot, int group) const { return ((a * kGroups + group) * slots + slot) * kIn; }
    // copy and slot of relative position rel
    __device__ __forceinline__ void place(int rel, int distance, int& a, int& slot) const {
        const int first = rel + distance;
        a = first & (VEC - 1);
        slot = max(0, min(slots - 1, (first - a) / VEC + 2));
    }
    // value index (a distance plus max_distance, maybe outside [0, 2*max_distance]) of element i
    __device__ __forceinline__ int index(int a, int slot, int i) const { return VEC * (slot - 2) + a + i; }
};
template <int VEC> __device__ __forceinline__ void build_bias(const BiasForm& f, int head, const Window<VEC>& w, float* plain, float* bias) {
    for (int d = threadIdx.x; d <= 2 * f.distance; d += blockDim.x) plain[d] = f.table[bucket_of(f, d - f.distance) * f.h + head];
    __syncthreads();
    constexpr int kGroups = Window<VEC>::kGroups, kIn = Window<VEC>::kIn;
    for (int o = threadIdx.x >> 5; o < VEC * kGroups; o += blockDim.x >> 5) {   // a warp one copy's half
        const int a = o / kGroups, group = o % kGroups;
        for (int slot = threadIdx.x & 31; slot < w.slots; slot += 32)
#pragma unroll
            for (int i = 0; i < kIn; ++i) bias[w.at(a, slot, group) + i] = plain[max(0, min(2 * f.distance, w.index(a, slot, group * kIn + i)))];
    }
}
template <int VEC> __device__ __forceinline__ void window_load(const float* table, const Window<VEC>& w, int a, int slot, float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        x[0] = table[w.at(a, slot, 0)];
    } else {
#pragma unroll
        for (int g = 0; g < VEC / 4; ++g) {
            const float4 v = *reinterpret_cast<const float4*>(table + w.at(a, slot, g));
            x[4 * g] = v.x, x[4 * g + 1] = v.y, x[4 * g + 2] = v.z, x[4 * g + 3] = v.w;
        }
    }
}

// Keys [0, end) are seen by the query at position p.
struct Queries {
    int64_t keys, start;   // this batch entry's
    __device__ Queries(const BiasForm& f, int ib)
        : keys(f.k_len != nullptr ? min(f.tk, static_cast<int64_t>(max(f.k_len[ib], 0))) : f.tk), start(f.q_start != nullptr ? f.q_start[ib] : 0) {}
    __device__ int64_t position(int64_t iq) const { return iq + start; }
    __device__ int64_t end(const BiasForm& f, int64_t iq) const { return f.causal ? min(keys, max(position(iq) + 1, int64_t(0))) : keys; }
};

// A position as the held kernels use it: rows of at most 2^14 keys, so everything beyond +-2^28 is alike.
__device__ __forceinline__ int near_position(int64_t p) { return static_cast<int>(max(int64_t(-1) << 28, min(int64_t(1) << 28, p))); }

// z[i] = scale*s[i] + bias.  rel = j0 - p.
template <int VEC> __device__ __forceinline__ void add_bias(const BiasForm& f, const float* bias, const Window<VEC>& w, int rel, float (&z)[VEC]) {
    float b[VEC];
    int a, slot;
    w.place(rel, f.distance, a, slot);
    window_load<VEC>(bias, w, a, slot, b);
    multiply_add(z, f.scale, b);
}
// `gone` in the place of the keys j0 + i that are not seen.
template <int VEC, typename I> __device__ __forceinline__ void mask(I j0, I end, float gone, float (&z)[VEC]) {
    if (j0 < 0 || j0 + VEC > end) {
        rare();
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (j0 + i < 0 || j0 + i >= end) z[i] = gone;
    }
}
// Of a row's SLOTS steps (G slots of VEC keys each): the first `whole` hold seen keys only, those from `some` on hold none.
// Both are the same for all threads of a row, so the common steps run without a test of their own.
template <int VEC, int G> struct Steps {
    int whole, some;
    __device__ __forceinline__ Steps(int lead, int end) : whole(lead == 0 ? end / (G * VEC) : 0), some((lead + end + G * VEC - 1) / (G * VEC)) {}
};

template <int G> struct Cta {
    static constexpr int kThreads = G > 32 ? G : 128;
    static constexpr int kRows = kThreads / G;    // rows in hand at a time
};

// Joins one part per warp over the G threads of a row (a CTA when G > 32); every lane passes its warp's part.  `part`
// holds two sets of warp results used in turn, so one barrier a call suffices.
template <int G> __device__ __forceinline__ MaxSum group_join(MaxSum v, float c, MaxSum (*part)[16], int turn) {
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) part[turn & 1][threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_join(lane < G / 32 ? part[turn & 1][lane] : MaxSum{-INFINITY, 0.f}, c);
    }
    return v;
}
template <int G> __device__ __forceinline__ float group_sum(float v, float (*part)[16], int turn) {
    v = warp_sum(v);
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) part[turn & 1][threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_sum(lane < G / 32 ? part[turn & 1][lane] : 0.f);
    }
    return v;
}

// SLOTS slots a thread are held in registers, and the next row's are loaded before this row's are used.
// WHOLE: every slot of every row holds seen keys only - no test, no mask.
template <typename T, int VEC, int G, int SLOTS, bool WHOLE>
__global__ void __launch_bounds__(Cta<G>::kThreads, 768 / Cta<G>::kThreads)
    bias_softmax_kernel(const __grid_constant__ BiasForm f, const Rows4<const T> scores, const Rows4<T> probs, MaxSum* stats) {
    extern __shared__ __align__(16) float bias[];
    __shared__ MaxSum part[2][16];
    const Window<VEC> w(f.distance);
    const int t = threadIdx.x % G, ib = blockIdx.z, ih = blockIdx.y, n = static_cast<int>(f.tk);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * f.rows_per_cta + threadIdx.x / G;
    const Queries q(f, ib);
    const int rows = static_cast<int>(min(static_cast<int64_t>(f.rows_per_cta), f.tq - first));   // it < rows: this group's (may be <= 0)
    const T* in = scores.row(ib, ih, first);
    T* out = probs.row(ib, ih, first);
    const int64_t in_step = Cta<G>::kRows * scores.q, out_step = Cta<G>::kRows * probs.q;
    Raw<T, VEC> raw[SLOTS];
    auto fetch = [&](const T* row, int64_t iq) {
        const int lead = WHOLE ? 0 : row_lead<T, VEC>(row), j = t * VEC - lead, end = WHOLE ? n : static_cast<int>(q.end(f, iq));
        const bool safe = WHOLE || scores.extent.around(row, n);
#pragma unroll
        for (int c = 0; c < SLOTS; ++c) {
            const int j0 = j + c * G * VEC;
            raw[c].fetch(row + j0, WHOLE || (j0 < end && (safe || VEC == 1 || (j0 >= 0 && j0 + VEC <= n))));
        }
    };
    if (rows > 0) fetch(in, first);
    build_bias<VEC>(f, ih, w, bias + w.floats(), bias);
    __syncthreads();
    for (int it = 0; it < rows; it += Cta<G>::kRows, in += in_step, out += out_step) {   // G > 32: the whole CTA alike
        const int64_t iq = first + it;
        const int lead = WHOLE ? 0 : row_lead<T, VEC>(in), end = WHOLE ? n : static_cast<int>(q.end(f, iq));
        const Steps<VEC, G> steps(lead, end);
        const int p = near_position(q.position(iq)), j = t * VEC - lead;
        float z[SLOTS][VEC];
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < SLOTS; ++c)
            if (WHOLE || c < steps.some) {
                const int j0 = j + c * G * VEC;
                raw[c].get(z[c]);
                if (!WHOLE && VEC > 1 && c >= steps.whole && (j0 < 0 || j0 + VEC > n) && !scores.extent.around(in, n)) read_apart<T, VEC>(in, j0, n, z[c]);
                add_bias<VEC>(f, bias, w, j0 - p, z[c]);
                if (!WHOLE && c >= steps.whole) mask<VEC>(j0, end, -INFINITY, z[c]);
                top = largest(top, z[c]);
            }
        if (it + Cta<G>::kRows < rows) fetch(in + in_step, iq + Cta<G>::kRows);
        MaxSum v{warp_max(top), 0.f};
        const Reference own(v.m, kLog2e);
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < SLOTS; ++c)
            if (WHOLE || c < steps.some) {
                exponentials(z[c], own, kLog2e);
                add_up(sum, z[c]);
            }
        v.s = warp_sum(sum.x + sum.y);
        const MaxSum all = group_join<G>(v, kLog2e, part, it / Cta<G>::kRows);
        float norm = all.s == 0.f ? 0.f : 1.f / all.s;
        if (G > 32 && v.s != 0.f) norm *= exp2_fast(Reference(all.m, kLog2e).of_part(v.m, kLog2e));
#pragma unroll
        for (int c = 0; c < SLOTS; ++c) {
            const int j0 = j + c * G * VEC;
            if (WHOLE || c < steps.some) {
                multiply(z[c], norm);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) z[c][i] = 0.f;
            }
            if (WHOLE || c < steps.whole)
                store_whole<T, VEC>(out + j0, z[c]);
            else if (j0 < n)
                store_slot<T, VEC>(out, j0, n, z[c]);
        }
        if (t == 0 && stats != nullptr) stats[(static_cast<int64_t>(ib) * f.h + ih) * f.tq + iq] = {all.m, all.s / Reference(all.m, kLog2e).left_out(kLog2e)};
    }
}

// Rows of any length, read twice.
template <typename T, int VEC>
__global__ void __launch_bounds__(512) bias_softmax_long_kernel(const __grid_constant__ BiasForm f, const Rows4<const T> scores, const Rows4<T> probs, MaxSum* stats) {
    constexpr int G = 512;
    extern __shared__ __align__(16) float bias[];
    __shared__ MaxSum part[2][16];
    const Window<VEC> w(f.distance);
    const int t = threadIdx.x, ib = blockIdx.z, ih = blockIdx.y;
    const Queries q(f, ib);
    build_bias<VEC>(f, ih, w, bias + w.floats(), bias);
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * f.rows_per_cta;
    for (int it = 0; it < f.rows_per_cta && first + it < f.tq; ++it) {
        const int64_t iq = first + it, p = q.position(iq), end = q.end(f, iq);
        const T* in = scores.row(ib, ih, iq);
        T* out = probs.row(ib, ih, iq);
        const int lead = row_lead<T, VEC>(in);
        MaxSum v{-INFINITY, 0.f};
        for (int64_t j0 = static_cast<int64_t>(t) * VEC - lead; j0 < end; j0 += G * VEC) {
            float z[VEC];
            load_slot<T, VEC>(in, j0, f.tk, 0.f, z);
            add_bias<VEC>(f, bias, w, near_position(j0 - p), z);
            mask<VEC>(j0, end, -INFINITY, z);
            float m = v.m;
#pragma unroll
            for (int i = 0; i < VEC; ++i) m = fmaxf(m, z[i]);
            const Reference r(m, kLog2e);
            if (v.s != 0.f) v.s *= exp2_fast(r.of_part(v.m, kLog2e));
            v.m = m;
#pragma unroll
            for (int i = 0; i < VEC; ++i) v.s += exp2_fast(r.of(z[i], kLog2e));
        }
        const MaxSum all = group_join<G>(warp_join(v, kLog2e), kLog2e, part, it);
        const Reference r(all.m, kLog2e);
        const float norm = all.s == 0.f ? 0.f : 1.f / all.s;
        for (int64_t j0 = static_cast<int64_t>(t) * VEC - lead; j0 < f.tk; j0 += G * VEC) {
            float z[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) z[i] = 0.f;
            if (j0 < end) {
                load_slot<T, VEC>(in, j0, f.tk, 0.f, z);
                add_bias<VEC>(f, bias, w, near_position(j0 - p), z);
            mask<VEC>(j0, end, -INFINITY, z);
#pragma unroll
                for (int i = 0; i < VEC; ++i) z[i] = exp2_fast(r.of(z[i], kLog2e)) * norm;
            }
            store_slot<T, VEC>(out, j0, f.tk, z);
        }
        if (t == 0 && stats != nullptr) stats[(static_cast<int64_t>(ib) * f.h + ih) * f.tq + iq] = {all.m, all.s / Reference(all.m, kLog2e).left_out(kLog2e)};
    }
}

// One slot of the table's gradient: dz of the keys at distances rel .. rel + VEC - 1 (0 where a key is not seen).  `sums`:
// the warp's window, laid out as the bias.  Lanes whose slot touches the window have slots of their own in it; the first
// and the last slot of a copy stand for either side beyond it and stay in registers.
template <int VEC>
__device__ __forceinline__ void add_diagonals(const BiasForm& f, float* sums, const Window<VEC>& w, int rel, const float (&dz)[VEC], float2& left, float2& right) {
    int a, slot;
    w.place(rel, f.distance, a, slot);
    float2 sum = make_float2(0.f, 0.f);
    add_up(sum, dz);
    left.x += slot == 0 ? sum.x + sum.y : 0.f;
    right.x += slot == w.slots - 1 ? sum.x + sum.y : 0.f;
    if (slot > 0 && slot < w.slots - 1) {
        float x[VEC];
        window_load<VEC>(sums, w, a, slot, x);
        multiply_add(x, 1.f, dz);
        if constexpr (VEC == 1) {
            sums[w.at(a, slot, 0)] = x[0];
        } else {
#pragma unroll
            for (int g = 0; g < VEC / 4; ++g)
                *reinterpret_cast<float4*>(sums + w.at(a, slot, g)) = make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
        }
    }
}

// What the rows of a CTA leave for the table.  Each warp's far sums take the first and last slot of its copy 0; then warps
// and copies are added in order, value index by value index, and a warp a bucket adds its distances (those beyond the
// window belong to the last bucket of their side).
template <int VEC>
__device__ __forceinline__ void leave_buckets(const BiasForm& f, float* all_sums, const Window<VEC>& w, int warps, float2 left2, float2 right2, float* by_value, float* mine) {
    const float left = warp_sum(left2.x + left2.y), right = warp_sum(right2.x + right2.y);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, values = w.values();
    if (lane == 0) {
        float* sums = all_sums + warp * w.floats();
        sums[w.at(0, 0, 0)] = left;
        sums[w.at(0, w.slots - 1, 0)] = right;
    }
    __syncthreads();
    for (int v = threadIdx.x; v < values; v += blockDim.x) {
        float s = 0.f;
#pragma unroll
        for (int a = 0; a < VEC; ++a) {
            const int e = v - a;   // VEC*slot + i
            if (e < 0 || e >= VEC * w.slots) continue;
            const float* sums = all_sums + w.at(a, e / VEC, e % VEC / Window<VEC>::kIn) + e % VEC % Window<VEC>::kIn;
            for (int k = 0; k < warps; ++k) s += sums[k * w.floats()];
        }
        by_value[v] = s;
    }
    __syncthreads();
    const float* at = by_value + 2 * VEC + f.distance;   // at[rel]
    for (int c = warp; c < f.buckets; c += warps) {
        const int k = f.bidirectional && c >= f.nb ? c - f.nb : c;
        const bool last = k == f.nb - 1;
        const int lo = k < f.exact ? k : f.starts[k - f.exact], hi = k < f.exact && !last ? k + 1 : (last ? values : f.starts[k - f.exact + 1]);
        const int most_left = f.distance + 2 * VEC, most_right = values - 1 - most_left;   // largest distances there are
        float s = 0.f;
        if (c != k) {
            for (int n = max(lo, 1) + lane; n < hi && n <= most_right; n += 32) s += at[n];
        } else {
            for (int n = lo + lane; n < hi && n <= most_left; n += 32) s += at[-n];
            if (!f.bidirectional && c == 0)
                for (int n = 1 + lane; n <= most_right; n += 32) s += at[n];
        }
        s = warp_sum(s);
        if (lane == 0) mine[c] = s;
    }
}

// SLOTS slots of scores and of dprobs a thread are held: p in binary32, dprobs as loaded.
template <typename T, int VEC, int G, int SLOTS, bool WHOLE>
__global__ void __launch_bounds__(Cta<G>::kThreads, 512 / Cta<G>::kThreads)
    bias_softmax_backward_kernel(const __grid_constant__ BiasForm f, const Rows4<const T> scores, const Rows4<const T> dprobs,
                                 const Rows4<T> dscores, const MaxSum* __restrict__ stats, float* __restrict__ partial) {
    extern __shared__ __align__(16) float bias[];
    __shared__ float part[2][16];
    constexpr int kWarps = Cta<G>::kThreads / 32;
    const Window<VEC> w(f.distance);
    float* all_sums = bias + w.floats();
    float* sums = all_sums + (threadIdx.x >> 5) * w.floats();
    float* plain = all_sums + (partial != nullptr ? kWarps * w.floats() : 0);
    const int t = threadIdx.x % G, ib = blockIdx.z, ih = blockIdx.y, n = static_cast<int>(f.tk);
    const Queries q(f, ib);
    build_bias<VEC>(f, ih, w, plain, bias);
    if (partial != nullptr)
        for (int i = threadIdx.x; i < kWarps * w.floats() / 4; i += blockDim.x) reinterpret_cast<float4*>(all_sums)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    float2 left = make_float2(0.f, 0.f), right = left;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * f.rows_per_cta + threadIdx.x / G;
    const int rows = static_cast<int>(min(static_cast<int64_t>(f.rows_per_cta), f.tq - first));   // it < rows: this group's
    const T* in = scores.row(ib, ih, first);
    const T* up = dprobs.row(ib, ih, first);
    T* out = dscores.p != nullptr ? dscores.row(ib, ih, first) : nullptr;
    const MaxSum* stat = stats + (static_cast<int64_t>(ib) * f.h + ih) * f.tq + first;
    constexpr int kRows = Cta<G>::kRows;
    Raw<T, VEC> s[SLOTS], dp[SLOTS];
    for (int it = 0; it < rows; it += kRows, in += kRows * scores.q, up += kRows * dprobs.q, out += kRows * dscores.q, stat += kRows) {
        const int lead = WHOLE ? 0 : row_lead<T, VEC>(in), end = WHOLE ? n : static_cast<int>(q.end(f, first + it));
        const Steps<VEC, G> steps(lead, end);
        const int p0 = near_position(q.position(first + it)), j = t * VEC - lead;
        const bool safe = WHOLE || VEC == 1 || (scores.extent.around(in, n) && dprobs.extent.around(up, n));
#pragma unroll
        for (int c = 0; c < SLOTS; ++c) {
            const int j0 = j + c * G * VEC;
            const bool go = WHOLE || (j0 < end && (safe || (j0 >= 0 && j0 + VEC <= n)));
            s[c].fetch(in + j0, go);
            dp[c].fetch(up + j0, go);
        }
        const MaxSum all = *stat;
        const Reference r(all.m, kLog2e);
        const bool empty = all.s == 0.f;   // a row without keys, or none above -inf: all 0
        const float norm = empty ? 0.f : 1.f / (all.s * r.left_out(kLog2e));
        float p[SLOTS][VEC];
        float2 dot2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < SLOTS; ++c)
            if (WHOLE || c < steps.some) {
                const int j0 = j + c * G * VEC;
                float d[VEC];
                s[c].get(p[c]);
                dp[c].get(d);
                if (!WHOLE && c >= steps.whole && !safe && (j0 < 0 || j0 + VEC > n)) {
                    read_apart<T, VEC>(in, j0, n, p[c]);
                    read_apart<T, VEC>(up, j0, n, d);
                }
                add_bias<VEC>(f, bias, w, j0 - p0, p[c]);
                exponentials(p[c], r, kLog2e);
                multiply(p[c], norm);
                if (!WHOLE && c >= steps.whole) {
                    mask<VEC>(j0, end, 0.f, p[c]);
                    mask<VEC>(j0, end, 0.f, d);
                }
                add_products(dot2, p[c], d);
            }
        const float dot = group_sum<G>(dot2.x + dot2.y, part, it / Cta<G>::kRows);
        // a warp's step may meet the window, lie left of it or right
        const int warp_j = j - (t & 31) * VEC - p0;
#pragma unroll
        for (int c = 0; c < SLOTS; ++c) {
            const int j0 = j + c * G * VEC;
            float dz[VEC];
            if ((WHOLE || c < steps.some) && !empty) {
                dp[c].get(dz);
                if (!WHOLE && c >= steps.whole && !safe && (j0 < 0 || j0 + VEC > n)) read_apart<T, VEC>(up, j0, n, dz);
                float less[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) less[i] = -dot;
                multiply_add(dz, 1.f, less);
                multiply_by(dz, p[c]);
                if (!WHOLE && c >= steps.whole) mask<VEC>(j0, end, 0.f, dz);   // whatever dot is
                if (partial != nullptr) {
                    const int at = warp_j + c * G * VEC;   // of the warp's first key
                    if (at + 32 * VEC <= -f.distance)
                        add_up(left, dz);
                    else if (at >= f.distance)
                        add_up(right, dz);
                    else
                        add_diagonals<VEC>(f, sums, w, j0 - p0, dz, left, right);
                }
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) dz[i] = 0.f;
            }
            if (out != nullptr) {
                multiply(dz, f.scale);
                if (WHOLE || c < steps.whole)
                    store_whole<T, VEC>(out + j0, dz);
                else if (j0 < n)
                    store_slot<T, VEC>(out, j0, n, dz);
            }
        }
        __syncwarp();  // the next row meets this row's diagonals through other lanes
    }
    if (partial == nullptr) return;
    leave_buckets<VEC>(f, all_sums, w, kWarps, left, right, plain, partial + ((static_cast<int64_t>(ih) * gridDim.z + ib) * gridDim.x + blockIdx.x) * f.buckets);
}

// Rows of any length, read twice.
template <typename T, int VEC>
__global__ void __launch_bounds__(256)
    bias_softmax_backward_long_kernel(const __grid_constant__ BiasForm f, const Rows4<const T> scores, const Rows4<const T> dprobs,
                                      const Rows4<T> dscores, const MaxSum* __restrict__ stats, float* __restrict__ partial) {
    constexpr int G = 256, kWarps = G / 32;
    extern __shared__ __align__(16) float bias[];
    __shared__ float part[2][16];
    const Window<VEC> w(f.distance);
    float* all_sums = bias + w.floats();
    float* sums = all_sums + (threadIdx.x >> 5) * w.floats();
    float* plain = all_sums + (partial != nullptr ? kWarps * w.floats() : 0);
    const int t = threadIdx.x, ib = blockIdx.z, ih = blockIdx.y;
    const Queries q(f, ib);
    build_bias<VEC>(f, ih, w, plain, bias);
    if (partial != nullptr)
        for (int i = threadIdx.x; i < kWarps * w.floats() / 4; i += blockDim.x) reinterpret_cast<float4*>(all_sums)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    float2 left = make_float2(0.f, 0.f), right = left;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * f.rows_per_cta;
    for (int it = 0; it < f.rows_per_cta && first + it < f.tq; ++it) {
        const int64_t iq = first + it, p0 = q.position(iq);
        const T* in = scores.row(ib, ih, iq);
        const T* up = dprobs.row(ib, ih, iq);
        T* out = dscores.p != nullptr ? dscores.row(ib, ih, iq) : nullptr;
        const int lead = row_lead<T, VEC>(in);
        const MaxSum all = stats[(static_cast<int64_t>(ib) * f.h + ih) * f.tq + iq];
        const int64_t end = all.s == 0.f ? 0 : q.end(f, iq);
        const Reference r(all.m, kLog2e);
        const float norm = 1.f / (all.s * r.left_out(kLog2e));
        float dot = 0.f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int64_t j0 = static_cast<int64_t>(t) * VEC - lead; j0 < (pass ? f.tk : end); j0 += G * VEC) {
                float p[VEC], dp[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) p[i] = dp[i] = 0.f;
                if (j0 < end) {
                    load_slot<T, VEC>(in, j0, f.tk, 0.f, p);
                    load_slot<T, VEC>(up, j0, end, 0.f, dp);
                    add_bias<VEC>(f, bias, w, near_position(j0 - p0), p);
                    mask<VEC>(j0, end, -INFINITY, p);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) p[i] = exp2_fast(r.of(p[i], kLog2e)) * norm;
                }
                if (pass == 0) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) dot = fmaf(p[i], dp[i], dot);
                    continue;
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) p[i] = j0 + i >= 0 && j0 + i < end ? p[i] * (dp[i] - dot) : 0.f;
                if (partial != nullptr && j0 < end) add_diagonals<VEC>(f, sums, w, near_position(j0 - p0), p, left, right);
                if (out != nullptr) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) p[i] *= f.scale;
                    store_slot<T, VEC>(out, j0, f.tk, p);
                }
            }
            if (pass == 0) dot = group_sum<G>(dot, part, it);
        }
        __syncwarp();
    }
    if (partial == nullptr) return;
    leave_buckets<VEC>(f, all_sums, w, kWarps, left, right, plain, partial + ((static_cast<int64_t>(ih) * gridDim.z + ib) * gridDim.x + blockIdx.x) * f.buckets);
}

// dtable[c][head]: the parts of one head added by 32 lanes, then the lanes; one warp a value.
__global__ void __launch_bounds__(256) bias_table_kernel(const float* __restrict__ partial, int64_t parts, int h, int buckets, float* __restrict__ dtable) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (id >= static_cast<int64_t>(h) * buckets) return;
    const int head = static_cast<int>(id / buckets), c = static_cast<int>(id % buckets);
    float s = 0.f;
    for (int64_t i = threadIdx.x & 31; i < parts; i += 32) s += partial[(head * parts + i) * buckets + c];
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) dtable[static_cast<int64_t>(c) * h + head] = s;
}

// ---- host side ----------------------------------------------------------------------------------

// Query rows a CTA takes.  Building the window (and leaving the buckets) costs a CTA what some rows do, so it takes up to
// `most` of them; `resident` CTAs run at a time, and of the counts that fill whole rounds of those the smallest one is taken
// (a part-filled last round leaves the GPU idle).  Small problems spread over one round.  `most` is a multiple of at_a_time.
int rows_for(int64_t heads, int64_t tq, int64_t resident, int at_a_time, int most) {
    const int64_t least = (tq + most - 1) / most;   // chunks a head that keep a CTA to `most` rows
    const int64_t rounds = least < 2 ? 1 : (least * heads + resident - 1) / resident;
    const int64_t chunks = std::max<int64_t>(1, rounds * resident / heads);
    return static_cast<int>(((tq + chunks - 1) / chunks + at_a_time - 1) / at_a_time * at_a_time);
}
// The backward kernels run 512 threads an SM; the smallest groups (64 threads, one row) make the most CTAs.
constexpr int kBackwardMost = 64;
int64_t most_chunks(int64_t heads, int64_t tq) {
    const int rows = rows_for(heads, tq, 8 * kNumSMs, 1, kBackwardMost);
    return (tq + rows - 1) / rows;
}

int check_form(int dtype, int64_t b, int64_t h, int64_t tq, int64_t tk, const float* table, int buckets, int max_distance,
               int bidirectional, float scale) {
    if (element_bytes(dtype) == 0 || b < 0 || h < 0 || tq < 0 || tk < 0) return BZ_ERR_INVALID_ARG;
    if (table == nullptr || buckets < 2 || (bidirectional && (buckets < 4 || buckets % 2)) || !(scale == scale)) return BZ_ERR_INVALID_ARG;
    const int nb = bidirectional ? buckets / 2 : buckets;
    if (max_distance <= nb / 2) return BZ_ERR_INVALID_ARG;
    if (buckets > 256 || max_distance > BZ_MAX_DISTANCE || b > 65535 || h > 65535 || tq >= (int64_t(1) << 31) || tk >= (int64_t(1) << 31))
        return BZ_ERR_UNSUPPORTED;
    return BZ_OK;
}

int check_tensor(const void* p, const int64_t* strides, int dtype) {
    if (p == nullptr || strides == nullptr || reinterpret_cast<uintptr_t>(p) % element_bytes(dtype)) return BZ_ERR_INVALID_ARG;
    return strides[0] < 0 || strides[1] < 0 || strides[2] < 0 ? BZ_ERR_INVALID_ARG : BZ_OK;
}

// An output's: no two rows may share memory.  In order of the strides of the dimensions longer than one, each has to reach over
// all that the ones before it span (so lie slices, permutations and gaps of any tensor).
int check_output(const void* p, const int64_t* strides, int dtype, int64_t b, int64_t h, int64_t tq, int64_t tk) {
    const int st = check_tensor(p, strides, dtype);
    if (st != BZ_OK) return st;
    struct Dim {
        int64_t stride, n;
    } d[3] = {{strides[0], b}, {strides[1], h}, {strides[2], tq}};
    std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    __int128 span = tk;
    for (const Dim& x : d) {
        if (x.n == 1) continue;
        if (x.stride < span) return BZ_ERR_INVALID_ARG;
        span += static_cast<__int128>(x.stride) * (x.n - 1);
    }
    return BZ_OK;
}

// Whether two tensors' rows all sit alike relative to 16-byte boundaries.
bool alike(const void* p, const int64_t* sp, const void* q, const int64_t* sq, int64_t b, int64_t h, int64_t tq, int bytes) {
    if ((reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(q)) & 15) return false;
    const int64_t n[3] = {b, h, tq};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && ((sp[i] - sq[i]) * bytes) & 15) return false;
    return true;
}

BiasForm make_form(int64_t h, int64_t tq, int64_t tk, const float* table, int buckets, int max_distance, int bidirectional, int causal,
                   float scale, const int32_t* k_len, const int32_t* q_start) {
    BiasForm f{};
    f.table = table, f.k_len = k_len, f.q_start = q_start, f.scale = scale;
    f.buckets = buckets, f.nb = bidirectional ? buckets / 2 : buckets, f.exact = f.nb / 2, f.distance = max_distance;
    f.bidirectional = bidirectional != 0, f.causal = causal != 0, f.h = static_cast<int>(h), f.tq = tq, f.tk = tk;
    bucket_starts(f.nb, f.distance, f.starts);
    return f;
}

// The limit belongs to the kernel and not to the call, so every call sets the same one, the most that the kernel can need:
// a smaller one would make another thread's launch fail.
template <typename K> int allow_smem(K kern, size_t bytes, size_t most) {
    if (bytes <= 48 * 1024) return BZ_OK;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
    return e == cudaSuccess ? BZ_OK : cuda_failed(e);
}

// The wide kernels keep eight (or four) copies of the window in shared memory, the backward ones a set for each warp too, so
// there is a distance beyond which one element at a time is faster.  4 x 8 x 1024 x 1024 bfloat16, wide against narrow:
// forward 40 against 86 us at distance 512; backward 87 against 145 at 300, 156 against 152 at 400 (one CTA an SM from 337 on).
constexpr int kWideForward = 512, kWideBackward = 336;

template <int VEC> size_t backward_smem(int distance, int warps, bool table) {
    const Window<VEC> w(distance);
    return (w.floats() * (1 + (table ? warps : 0)) + w.values()) * sizeof(float);
}

template <typename T> Rows4<T> rows4(T* p, const int64_t* s, int64_t b, const BiasForm& f) {
    if (p == nullptr) return {};
    return {p, s[0], s[1], s[2],
            {reinterpret_cast<const char*>(p), reinterpret_cast<const char*>(p + (b - 1) * s[0] + (f.h - 1) * s[1] + (f.tq - 1) * s[2] + f.tk)}};
}

// Whether every query sees every key and the rows fill the group's registers.
template <typename T, int VEC, int G, int SLOTS> bool whole_rows(const BiasForm& f, int64_t n) {
    return VEC > 1 && !f.causal && f.k_len == nullptr && n == f.tk && f.tk == static_cast<int64_t>(G) * SLOTS * VEC;
}

template <typename T, int VEC, int G, int SLOTS>
int launch_forward(BiasForm& f, int64_t n, int64_t b, const Rows4<const T>& in, const Rows4<T>& out, MaxSum* stats, cudaStream_t s) {
    constexpr int kRows = Cta<G>::kRows;
    // causal rows differ in length, so their CTAs are kept small enough for the last ones to even out
    f.rows_per_cta = f.causal ? rows_for(b * f.h, f.tq, 16 * kNumSMs, kRows, kRows * 8)
                              : rows_for(b * f.h, f.tq, SLOTS == 0 ? 4 * kNumSMs : 768 / Cta<G>::kThreads * kNumSMs, kRows, kRows * 16);
    const size_t smem = (Window<VEC>(f.distance).floats() + 2 * f.distance + 1) * sizeof(float);
    const dim3 grid(static_cast<unsigned>((f.tq + f.rows_per_cta - 1) / f.rows_per_cta), f.h, static_cast<unsigned>(b));
    if constexpr (SLOTS == 0) {
        bias_softmax_long_kernel<T, VEC><<<grid, 512, smem, s>>>(f, in, out, stats);
    } else {
        if (VEC > 1 && whole_rows<T, VEC, G, SLOTS>(f, n))
            bias_softmax_kernel<T, VEC, G, SLOTS, (VEC > 1)><<<grid, Cta<G>::kThreads, smem, s>>>(f, in, out, stats);
        else
            bias_softmax_kernel<T, VEC, G, SLOTS, false><<<grid, Cta<G>::kThreads, smem, s>>>(f, in, out, stats);
    }
    note_launch();
    return check_launch();
}

// `n`: elements from the first slot's begin to the row's end.
template <typename T, int VEC>
int dispatch_forward(BiasForm& f, int64_t n, int64_t b, const Rows4<const T>& in, const Rows4<T>& out, MaxSum* stats, cudaStream_t s) {
    constexpr int kFew = VEC == 1 ? 8 : 1, kFull = VEC == 1 ? 16 : 4, kMost = kFull * VEC;   // 64 bytes a thread
    if (n <= kFew * VEC * 32) return launch_forward<T, VEC, 32, kFew>(f, n, b, in, out, stats, s);
    if (n <= kMost * 32) return launch_forward<T, VEC, 32, kFull>(f, n, b, in, out, stats, s);
    if (n <= kMost * 64) return launch_forward<T, VEC, 64, kFull>(f, n, b, in, out, stats, s);
    if (n <= kMost * 128) return launch_forward<T, VEC, 128, kFull>(f, n, b, in, out, stats, s);
    if (n <= kMost * 256) return launch_forward<T, VEC, 256, kFull>(f, n, b, in, out, stats, s);
    if (n <= kMost * 512) return launch_forward<T, VEC, 512, kFull>(f, n, b, in, out, stats, s);
    return launch_forward<T, VEC, 512, 0>(f, n, b, in, out, stats, s);
}

template <typename T, int VEC, int G, int SLOTS>
int launch_backward(BiasForm& f, int64_t n, int64_t b, const Rows4<const T>& in, const Rows4<const T>& up, const Rows4<T>& out, const MaxSum* stats,
                    float* partial, cudaStream_t s) {
    f.rows_per_cta = rows_for(b * f.h, f.tq, 512 / Cta<G>::kThreads * kNumSMs, Cta<G>::kRows, kBackwardMost);
    const int warps = Cta<G>::kThreads / 32;
    const size_t smem = backward_smem<VEC>(f.distance, warps, partial != nullptr), most = backward_smem<VEC>(VEC > 1 ? kWideBackward : BZ_MAX_DISTANCE, warps, true);
    const dim3 grid(static_cast<unsigned>((f.tq + f.rows_per_cta - 1) / f.rows_per_cta), f.h, static_cast<unsigned>(b));
    int st;
    if constexpr (SLOTS == 0) {
        if ((st = allow_smem(bias_softmax_backward_long_kernel<T, VEC>, smem, most)) != BZ_OK) return st;
        bias_softmax_backward_long_kernel<T, VEC><<<grid, 256, smem, s>>>(f, in, up, out, stats, partial);
    } else {
        auto kern = VEC > 1 && whole_rows<T, VEC, G, SLOTS>(f, n) ? bias_softmax_backward_kernel<T, VEC, G, SLOTS, (VEC > 1)>
                                                                  : bias_softmax_backward_kernel<T, VEC, G, SLOTS, false>;
        if ((st = allow_smem(kern, smem, most)) != BZ_OK) return st;
        kern<<<grid, Cta<G>::kThreads, smem, s>>>(f, in, up, out, stats, partial);
    }
    note_launch();
    return check_launch();
}

template <typename T, int VEC>
int dispatch_backward(BiasForm& f, int64_t n, int64_t b, const Rows4<const T>& in, const Rows4<const T>& up, const Rows4<T>& out,
                      const MaxSum* stats, float* partial, cudaStream_t s) {
    constexpr int kFew = VEC == 1 ? 8 : 1, kFull = VEC == 1 ? 16 : 4, kMost = kFull * VEC;
    if (n <= kFew * VEC * 32) return launch_backward<T, VEC, 32, kFew>(f, n, b, in, up, out, stats, partial, s);
    if (n <= kMost * 32) return launch_backward<T, VEC, 32, kFull>(f, n, b, in, up, out, stats, partial, s);
    if (n <= kMost * 64) return launch_backward<T, VEC, 64, kFull>(f, n, b, in, up, out, stats, partial, s);
    if (n <= kMost * 128) return launch_backward<T, VEC, 128, kFull>(f, n, b, in, up, out, stats, partial, s);
    if (n <= kMost * 256) return launch_backward<T, VEC, 256, kFull>(f, n, b, in, up, out, stats, partial, s);
    return launch_backward<T, VEC, 256, 0>(f, n, b, in, up, out, stats, partial, s);
}

// Elements a row takes up from its first slot on: none before it if every row begins on a 16-byte boundary.
int64_t row_span(const void* p, const int64_t* strides, int64_t b, int64_t h, int64_t tq, int64_t tk, int bytes) {
    const int64_t zero[3] = {0, 0, 0};
    return alike(p, strides, nullptr, zero, b, h, tq, bytes) ? tk : tk + 16 / bytes - 1;
}

template <typename T>
int forward(BiasForm& f, int64_t b, const void* scores, const int64_t* ss, void* probs, const int64_t* sp, MaxSum* stats, cudaStream_t s) {
    const auto in = rows4(static_cast<const T*>(scores), ss, b, f);
    const auto out = rows4(static_cast<T*>(probs), sp, b, f);
    if (f.distance <= kWideForward && alike(scores, ss, probs, sp, b, f.h, f.tq, sizeof(T)))
        return dispatch_forward<T, Word<T>::kN>(f, row_span(scores, ss, b, f.h, f.tq, f.tk, sizeof(T)), b, in, out, stats, s);
    return dispatch_forward<T, 1>(f, f.tk, b, in, out, stats, s);
}

template <typename T>
int backward(BiasForm& f, int64_t b, const void* scores, const int64_t* ss, const void* dprobs, const int64_t* sd, void* dscores,
             const int64_t* so, const MaxSum* stats, float* partial, cudaStream_t s) {
    const auto in = rows4(static_cast<const T*>(scores), ss, b, f);
    const auto up = rows4(static_cast<const T*>(dprobs), sd, b, f);
    const auto out = rows4(static_cast<T*>(dscores), so, b, f);
    if (f.distance <= kWideBackward && alike(scores, ss, dprobs, sd, b, f.h, f.tq, sizeof(T)) && (dscores == nullptr || alike(scores, ss, dscores, so, b, f.h, f.tq, sizeof(T))))
        return dispatch_backward<T, Word<T>::kN>(f, row_span(scores, ss, b, f.h, f.tq, f.tk, sizeof(T)), b, in, up, out, stats, partial, s);
    return dispatch_backward<T, 1>(f, f.tk, b, in, up, out, stats, partial, s);
}

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" size_t bz_bias_softmax_workspace_bytes(int64_t b, int64_t h, int64_t tq, int64_t tk, int buckets) {
    if (b < 1 || h < 1 || tq < 1 || tk < 1 || buckets < 2 || buckets > 256 || b > 65535 || h > 65535) return 0;
    if (tq >= (int64_t(1) << 31) || tk >= (int64_t(1) << 31)) return 0;
    const size_t parts = static_cast<size_t>(b) * h * most_chunks(b * h, tq), each = buckets * sizeof(float);   // parts < 2^58
    const size_t most = ~size_t(0) / 256 * 256;
    return parts > most / each ? most : round_up(parts * each, 256);
}

extern "C" int bz_bias_softmax(const void* scores, const int64_t* strides_scores, int dtype, int64_t b, int64_t h, int64_t tq, int64_t tk,
                               const float* table, int buckets, int max_distance, int bidirectional, int causal, float scale,
                               const int32_t* k_len, const int32_t* q_start, void* probs, const int64_t* strides_probs, float* stats,
                               void* stream) {
    int st = check_form(dtype, b, h, tq, tk, table, buckets, max_distance, bidirectional, scale);
    if (st != BZ_OK) return st;
    if (b == 0 || h == 0 || tq == 0 || tk == 0) return BZ_OK;
    if ((st = check_tensor(scores, strides_scores, dtype)) != BZ_OK || (st = check_output(probs, strides_probs, dtype, b, h, tq, tk)) != BZ_OK) return st;
    if (!aligned8(stats)) return BZ_ERR_INVALID_ARG;
    BiasForm f = make_form(h, tq, tk, table, buckets, max_distance, bidirectional, causal, scale, k_len, q_start);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == BZ_F32) return forward<float>(f, b, scores, strides_scores, probs, strides_probs, reinterpret_cast<MaxSum*>(stats), s);
    if (dtype == BZ_F16) return forward<__half>(f, b, scores, strides_scores, probs, strides_probs, reinterpret_cast<MaxSum*>(stats), s);
    return forward<__nv_bfloat16>(f, b, scores, strides_scores, probs, strides_probs, reinterpret_cast<MaxSum*>(stats), s);
}

extern "C" int bz_bias_softmax_backward(const void* scores, const int64_t* strides_scores, int dtype, int64_t b, int64_t h, int64_t tq,
                                        int64_t tk, const float* table, int buckets, int max_distance, int bidirectional, int causal,
                                        float scale, const int32_t* k_len, const int32_t* q_start, const float* stats, const void* dprobs,
                                        const int64_t* strides_dprobs, void* dscores, const int64_t* strides_dscores, float* dtable,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    int st = check_form(dtype, b, h, tq, tk, table, buckets, max_distance, bidirectional, scale);
    if (st != BZ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dscores == nullptr && dtable == nullptr) return BZ_ERR_INVALID_ARG;
    if (b == 0 || h == 0 || tq == 0 || tk == 0) {
        if (dtable == nullptr || h == 0) return BZ_OK;
        const cudaError_t e = cudaMemsetAsync(dtable, 0, sizeof(float) * buckets * h, s);
        return e == cudaSuccess ? BZ_OK : cuda_failed(e);
    }
    if (stats == nullptr || !aligned8(stats)) return BZ_ERR_INVALID_ARG;
    if ((st = check_tensor(scores, strides_scores, dtype)) != BZ_OK || (st = check_tensor(dprobs, strides_dprobs, dtype)) != BZ_OK) return st;
    if (dscores != nullptr && (st = check_output(dscores, strides_dscores, dtype, b, h, tq, tk)) != BZ_OK) return st;
    if (dtable != nullptr &&
        (workspace == nullptr || !aligned256(workspace) || workspace_bytes < bz_bias_softmax_workspace_bytes(b, h, tq, tk, buckets)))
        return BZ_ERR_WORKSPACE;
    BiasForm f = make_form(h, tq, tk, table, buckets, max_distance, bidirectional, causal, scale, k_len, q_start);
    float* partial = dtable != nullptr ? static_cast<float*>(workspace) : nullptr;
    if (dtype == BZ_F32)
        st = backward<float>(f, b, scores, strides_scores, dprobs, strides_dprobs, dscores, strides_dscores, reinterpret_cast<const MaxSum*>(stats), partial, s);
    else if (dtype == BZ_F16)
        st = backward<__half>(f, b, scores, strides_scores, dprobs, strides_dprobs, dscores, strides_dscores, reinterpret_cast<const MaxSum*>(stats), partial, s);
    else
        st = backward<__nv_bfloat16>(f, b, scores, strides_scores, dprobs, strides_dprobs, dscores, strides_dscores, reinterpret_cast<const MaxSum*>(stats), partial, s);
    if (st != BZ_OK || dtable == nullptr) return st;
    const int64_t parts = b * ((tq + f.rows_per_cta - 1) / f.rows_per_cta);
    const int64_t values = h * buckets;
    bias_table_kernel<<<static_cast<unsigned>((values + 7) / 8), 256, 0, s>>>(partial, parts, static_cast<int>(h), buckets, dtable);
    note_launch();
    return check_launch();
}
