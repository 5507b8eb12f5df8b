// The join of a block to its residual stream: norm of the block's output, gate, dropout, residual scale, norm for the next
// block - and its gradient.
#include <cmath>

#include "dropout_rule.h"
#include "philox.cuh"
#include "worker_common.cuh"

namespace bz {

namespace {

constexpr int kWide = 1024;                       // threads of the kernels for any width
constexpr int kWideColumns = BZ_MAX_WIDTH / kWide;

struct JoinArgs {
    int64_t m;
    int n, layer;
    float eps;
    const float *w_post, *gate, *w_pre;
    int64_t group_rows;          // rows that share a gate row
    float residual, scale;       // of the branch: its own times dropout's
    int drop;                    // whether there is dropout
    Dropout dropout;
    float4* stats;
};
template <typename T> struct JoinRows {
    T* p;
    int64_t ld;
    __device__ __forceinline__ T* row(int64_t i) const { return p + i * ld; }
};

// Sum over the CTA; every thread gets it.
__device__ __forceinline__ float cta_sum(float v, float* part) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < (blockDim.x >> 5) ? part[lane] : 0.f);
}

// Mean and 1 / deviation of a row held in `value(column)`.
template <typename F> __device__ __forceinline__ float2 row_norm(const JoinArgs& a, float* part, F value) {
    float mean = 0.f, sum = 0.f;
    if (a.layer) {
        for (int c = threadIdx.x; c < a.n; c += blockDim.x) sum += value(c);
        mean = cta_sum(sum, part) / static_cast<float>(a.n);
        sum = 0.f;
    }
    for (int c = threadIdx.x; c < a.n; c += blockDim.x) {
        const float d = value(c) - mean;
        sum = fmaf(d, d, sum);
    }
    return {mean, 1.f / sqrtf(cta_sum(sum, part) / static_cast<float>(a.n) + a.eps)};
}

// One CTA a row, any width; the row of s in shared memory.
template <typename T> __global__ void __launch_bounds__(kWide) join_wide_kernel(const __grid_constant__ JoinArgs a, JoinRows<const T> x, JoinRows<const T> y, JoinRows<T> s, JoinRows<T> z) {
    extern __shared__ float held[];
    __shared__ float part[32];
    const Keep keep(a.dropout);
    for (int64_t i = blockIdx.x; i < a.m; i += gridDim.x) {
        const T* in = x.row(i);
        const T* block = y.p != nullptr ? y.row(i) : nullptr;
        const float* gate = a.gate != nullptr ? a.gate + i / a.group_rows * a.n : nullptr;
        float2 post = make_float2(0.f, 1.f), pre = make_float2(0.f, 1.f);
        if (a.w_post != nullptr) post = row_norm(a, part, [&](int c) { return to_f32(block[c]); });
        for (int c = threadIdx.x; c < a.n; c += kWide) {
            float v = a.residual * to_f32(in[c]);
            if (block != nullptr) {
                float b = to_f32(block[c]);
                if (a.w_post != nullptr) b = (b - post.x) * post.y * a.w_post[c];
                const float f = gate != nullptr ? a.scale * gate[c] : a.scale;
                if (!a.drop || keep.elements<1>(static_cast<uint64_t>(i) * a.n + c)) v = fmaf(f, b, v);
            }
            held[c] = v;
        }
        if (a.w_pre != nullptr) pre = row_norm(a, part, [&](int c) { return held[c]; });
        for (int c = threadIdx.x; c < a.n; c += kWide) {
            if (s.p != nullptr) s.row(i)[c] = from_f32<T>(held[c]);
            if (z.p != nullptr) z.row(i)[c] = from_f32<T>((held[c] - pre.x) * pre.y * a.w_pre[c]);
        }
        if (a.stats != nullptr && threadIdx.x == 0) a.stats[i] = make_float4(post.x, post.y, pre.x, pre.y);
    }
}

// ---- rows of up to 8192 columns ------------------------------------------------------------------
//
// A thread owns the same columns of every row, SL slots of VEC (a 16-byte word where every tensor's rows begin on 16-byte boundaries, else
// single elements), so what belongs to a column - weights in shared memory, column sums in registers - needs no exchange.  The next
// row's words come by cp.async while a row is worked on; each thread copies what it reads itself, and waits for nobody.

constexpr int kTeam = 512;   // threads of a CTA at most

// Two rows of NT tensors in shared memory, or (VEC = 1) one row in registers.
template <typename T, int VEC, int SL, int NT> struct Staged {
    uint4* room;
    __device__ __forceinline__ explicit Staged(void* smem) : room(static_cast<uint4*>(smem) + threadIdx.x) {}
    __device__ __forceinline__ void fetch(int t, int which, const T* row, int n) {
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            const int c = (q * blockDim.x + threadIdx.x) * VEC;
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(room + ((which * NT + t) * SL + q) * blockDim.x));
            const int left = (n - c) * static_cast<int>(sizeof(T)), bytes = left < 16 ? left : 16;
            if (left > 0) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row + c), "r"(bytes) : "memory");
        }
    }
    __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ static void arrived() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }   // all but the last group
    __device__ __forceinline__ void get(int t, int which, int q, float (&x)[VEC]) const { Word<T>::unpack(room[((which * NT + t) * SL + q) * blockDim.x], x); }
};
template <typename T, int SL, int NT> struct Staged<T, 1, SL, NT> {
    float r[NT][SL];
    __device__ __forceinline__ explicit Staged(void*) {}
    __device__ __forceinline__ void fetch(int t, int, const T* row, int n) {
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            const int c = q * blockDim.x + threadIdx.x;
            r[t][q] = c < n ? to_f32(row[c]) : 0.f;
        }
    }
    __device__ __forceinline__ static void commit() {}
    __device__ __forceinline__ static void arrived() {}
    __device__ __forceinline__ void get(int t, int, int q, float (&x)[1]) const { x[0] = r[t][q]; }
};

// A vector of weights in shared memory, a thread's columns where only it looks.
template <int VEC, int SL> struct Weights {
    static constexpr int kPiece = VEC == 1 ? 1 : 4;
    float* room;
    __device__ __forceinline__ void load(const float* w, int n) const {
#pragma unroll
        for (int q = 0; q < SL; ++q)
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC + k;
                room[((q * (VEC / kPiece) + k / kPiece) * blockDim.x + threadIdx.x) * kPiece + k % kPiece] = c < n ? __ldg(w + c) : 0.f;
            }
    }
    __device__ __forceinline__ void get(int q, float (&x)[VEC]) const {
        if constexpr (VEC == 1) {
            x[0] = room[q * blockDim.x + threadIdx.x];
        } else {
#pragma unroll
            for (int k = 0; k < VEC / 4; ++k) {
                const float4 w = reinterpret_cast<const float4*>(room)[(q * (VEC / 4) + k) * blockDim.x + threadIdx.x];
                x[4 * k] = w.x, x[4 * k + 1] = w.y, x[4 * k + 2] = w.z, x[4 * k + 3] = w.w;
            }
        }
    }
};
inline __host__ __device__ int weight_floats(int threads, int columns) { return threads * columns; }

// Sums over the CTA, one barrier each: two sets of partial sums in turn.
struct Exchange {
    float (*part)[2][16];
    int turn = 0;
    __device__ __forceinline__ explicit Exchange(float (*p)[2][16]) : part(p) {
        if (threadIdx.x < 64) p[threadIdx.x / 32][threadIdx.x / 16 % 2][threadIdx.x % 16] = 0.f;
        if (blockDim.x < 64) p[1][threadIdx.x / 16][threadIdx.x % 16] = 0.f;
        __syncthreads();
    }
    template <int K> __device__ __forceinline__ void sum(float (&v)[K]) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
        const int warps = blockDim.x >> 5;
        if (warps == 1) return;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) part[turn][k][threadIdx.x >> 5] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
            for (int w = 0; w < warps; w += 4) {
                const float4 p = *reinterpret_cast<const float4*>(&part[turn][k][w]);
                v[k] += (p.x + p.y) + (p.z + p.w);
            }
        }
        turn ^= 1;
    }
};

// Mean and 1 / deviation of what the CTA's threads hold.
template <int VEC, int SL> __device__ __forceinline__ float2 held_norm(const JoinArgs& a, Exchange& ex, const float (&v)[SL][VEC], float inv_n) {
    float mean = 0.f, t[1] = {0.f};
    if (a.layer) {
#pragma unroll
        for (int q = 0; q < SL; ++q)
#pragma unroll
            for (int k = 0; k < VEC; ++k) t[0] += v[q][k];   // 0 behind the last column
        ex.sum(t);
        mean = t[0] * inv_n;
        t[0] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < SL; ++q) {
        const int c = (q * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float d = c + k < a.n ? v[q][k] - mean : 0.f;
            t[0] = fmaf(d, d, t[0]);
        }
    }
    ex.sum(t);
    return {mean, 1.f / sqrtf(t[0] * inv_n + a.eps)};
}

// Which of a slot's elements stay.
template <int VEC> __device__ __forceinline__ uint32_t staying(const JoinArgs& a, const Keep& keep, int64_t i, int c) {
    return a.drop && c < a.n ? keep.elements<VEC>(static_cast<uint64_t>(i) * a.n + c) : 0xffffffffu;
}

template <typename T, int VEC> __device__ __forceinline__ void put_slot(T* row, int c, int n, const float (&x)[VEC]) {
    if (c + VEC <= n) {
        store_whole<T, VEC>(row + c, x);
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            if (c + k < n) row[c + k] = from_f32<T>(x[k]);
    }
}

// s of a slot from x, the block's output (normalised if it is) and their factors.
template <int VEC> __device__ __forceinline__ void joined(const JoinArgs& a, bool branch, uint32_t stays, const float (&w_post)[VEC], const float (&gate)[VEC], const float (&b)[VEC], float (&x)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        x[k] *= a.residual;
        if (branch && (stays >> k & 1)) {
            const float v = a.w_post != nullptr ? b[k] * w_post[k] : b[k];
            x[k] = fmaf(a.gate != nullptr ? a.scale * gate[k] : a.scale, v, x[k]);
        }
    }
}

template <typename T, int VEC, int SL>
__global__ void __launch_bounds__(kTeam) join_kernel(const __grid_constant__ JoinArgs a, JoinRows<const T> x, JoinRows<const T> y, JoinRows<T> s, JoinRows<T> z) {
    extern __shared__ __align__(16) float smem[];
    __shared__ __align__(16) float part[2][2][16];
    Exchange ex(part);
    const Keep keep(a.dropout);
    const bool branch = y.p != nullptr, post = a.w_post != nullptr;
    const int floats = weight_floats(blockDim.x, VEC * SL);
    float* room = smem;
    Weights<VEC, SL> w_post{room}, gate{room += post ? floats : 0}, w_pre{room += a.gate != nullptr ? floats : 0};
    Staged<T, VEC, SL, 2> in(room + (a.w_pre != nullptr ? floats : 0));
    const float inv_n = 1.f / static_cast<float>(a.n);
    int64_t i = a.m * blockIdx.x / gridDim.x, group = -1;
    const int64_t last = a.m * (blockIdx.x + 1) / gridDim.x;
    auto fetch = [&](int64_t row, int which) {
        if (row < last) {
            in.fetch(0, which, x.row(row), a.n);
            if (branch) in.fetch(1, which, y.row(row), a.n);
        }
        in.commit();
    };
    if (VEC > 1) fetch(i, 0);
    if (post) w_post.load(a.w_post, a.n);
    if (a.w_pre != nullptr) w_pre.load(a.w_pre, a.n);
    for (int which = 0; i < last; ++i, which ^= 1) {
        if (a.gate != nullptr && i / a.group_rows != group) group = i / a.group_rows, gate.load(a.gate + group * a.n, a.n);
        fetch(VEC > 1 ? i + 1 : i, which ^ 1);
        in.arrived();
        float v[SL][VEC];
        float2 st = make_float2(0.f, 1.f), pre = make_float2(0.f, 1.f);
        if (post) {
#pragma unroll
            for (int q = 0; q < SL; ++q) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[q][k] = 0.f;
                if ((q * blockDim.x + threadIdx.x) * VEC < a.n) in.get(1, which, q, v[q]);
            }
            st = held_norm(a, ex, v, inv_n);
        }
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            const int c = (q * blockDim.x + threadIdx.x) * VEC;
            float b[VEC], wp[VEC], g[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) b[k] = wp[k] = g[k] = 0.f;
            if (c < a.n) {
                if (post) {
                    w_post.get(q, wp);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) b[k] = (v[q][k] - st.x) * st.y;
                } else if (branch) {
                    in.get(1, which, q, b);
                }
                if (a.gate != nullptr) gate.get(q, g);
                in.get(0, which, q, v[q]);
                joined(a, branch, staying<VEC>(a, keep, i, c), wp, g, b, v[q]);
            } else {
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[q][k] = 0.f;
            }
        }
        if (s.p != nullptr) {
#pragma unroll
            for (int q = 0; q < SL; ++q) put_slot(s.row(i), (q * blockDim.x + threadIdx.x) * VEC, a.n, v[q]);
        }
        if (a.w_pre != nullptr) {
            pre = held_norm(a, ex, v, inv_n);
#pragma unroll
            for (int q = 0; q < SL; ++q) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC;
                if (c >= a.n) continue;
                float w[VEC];
                w_pre.get(q, w);
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[q][k] = (v[q][k] - pre.x) * pre.y * w[k];
                put_slot(z.row(i), c, a.n, v[q]);
            }
        }
        if (a.stats != nullptr && threadIdx.x == 0) a.stats[i] = make_float4(st.x, st.y, pre.x, pre.y);
    }
}

// ---- gradient -----------------------------------------------------------------------------------
//
// The rows are cut into parts that lie within a gate's group each; a CTA takes a run of parts and keeps the column sums of
// dw_post and dw_pre over all of them, that of dgate over a part.  The sums of the CTAs and parts go to the workspace and are
// added up in their order by a second kernel.

struct Parts {
    int64_t groups, rows, per_group, count, ctas;   // rows of a group; parts of a group, of all
};
struct Sums {
    float *post, *gate, *pre;   // [ctas][n], [count][n], [ctas][n]; nullptr: not wanted
};

__device__ __forceinline__ int64_t part_begin(const Parts& p, int64_t k) { return k / p.per_group * p.rows + k % p.per_group * p.rows / p.per_group; }
__device__ __forceinline__ int64_t part_end(const Parts& p, int64_t k) { return k / p.per_group * p.rows + (k % p.per_group + 1) * p.rows / p.per_group; }

// Any width: column sums in shared memory, what a row's passes share in registers.
template <typename T>
__global__ void __launch_bounds__(kWide) join_wide_backward_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ Parts parts, const __grid_constant__ Sums out,
                                                                   JoinRows<const T> x, JoinRows<const T> y, JoinRows<const T> ds, JoinRows<const T> dz, JoinRows<T> dx, JoinRows<T> dy) {
    extern __shared__ float sums[];
    __shared__ float part[32];
    float *sum_post = sums, *sum_gate = sums + a.n, *sum_pre = sums + 2 * a.n;
    const Keep keep(a.dropout);
    const bool pre = a.w_pre != nullptr && dz.p != nullptr, post = a.w_post != nullptr, branch = y.p != nullptr;
    const float inv_n = 1.f / static_cast<float>(a.n);
    for (int c = threadIdx.x; c < 3 * a.n; c += kWide) sums[c] = 0.f;
    __syncthreads();
    const int64_t last = parts.count * (blockIdx.x + 1) / parts.ctas;
    for (int64_t k = parts.count * blockIdx.x / parts.ctas; k < last; ++k) {
        for (int64_t i = part_begin(parts, k); i < part_end(parts, k); ++i) {
            const float4 st = a.stats != nullptr ? a.stats[i] : make_float4(0.f, 1.f, 0.f, 1.f);
            const float* gate = a.gate != nullptr ? a.gate + i / a.group_rows * a.n : nullptr;
            uint32_t stays = 0xffffffffu;   // bit q: column q of this thread is not dropped
            float hat[kWideColumns], c0 = 0.f, c1 = 0.f;
#pragma unroll
            for (int q = 0; q < kWideColumns; ++q) {
                const int c = q * kWide + threadIdx.x;
                hat[q] = 0.f;
                if (c >= a.n) continue;
                if (a.drop && !keep.elements<1>(static_cast<uint64_t>(i) * a.n + c)) stays &= ~(1u << q);
                if (!pre) continue;
                float v = a.residual * to_f32(x.row(i)[c]);
                if (branch && (stays >> q & 1)) {
                    float b = to_f32(y.row(i)[c]);
                    if (post) b = (b - st.x) * st.y * a.w_post[c];
                    v = fmaf(gate != nullptr ? a.scale * gate[c] : a.scale, b, v);
                }
                hat[q] = (v - st.z) * st.w;
                const float d = to_f32(dz.row(i)[c]);
                sum_pre[c] = fmaf(d, hat[q], sum_pre[c]);
                c0 = fmaf(d, a.w_pre[c], c0), c1 = fmaf(d * a.w_pre[c], hat[q], c1);
            }
            if (pre) {
                c0 = a.layer ? cta_sum(c0, part) * inv_n : 0.f;
                c1 = cta_sum(c1, part) * inv_n;
            }
            float k0 = 0.f, k1 = 0.f;
            // from here on hat[] is what the block's norm gets; dx is written last, so that it may lie over any input
            float g[kWideColumns];
#pragma unroll
            for (int q = 0; q < kWideColumns; ++q) {
                const int c = q * kWide + threadIdx.x;
                g[q] = 0.f;
                if (c >= a.n) continue;
                g[q] = ds.p != nullptr ? to_f32(ds.row(i)[c]) : 0.f;
                if (pre) g[q] += st.w * (to_f32(dz.row(i)[c]) * a.w_pre[c] - c0 - hat[q] * c1);
                if (!branch) continue;
                float u = stays >> q & 1 ? a.scale * g[q] : 0.f;
                float h = to_f32(y.row(i)[c]);
                if (post) h = (h - st.x) * st.y;
                sum_gate[c] = fmaf(u, post ? h * a.w_post[c] : h, sum_gate[c]);
                if (gate != nullptr) u *= gate[c];
                if (post) {
                    sum_post[c] = fmaf(u, h, sum_post[c]);
                    u *= a.w_post[c];
                    k0 += u, k1 = fmaf(u, h, k1);
                }
                hat[q] = u;
            }
            if (post) {
                k0 = a.layer ? cta_sum(k0, part) * inv_n : 0.f;
                k1 = cta_sum(k1, part) * inv_n;
            }
#pragma unroll
            for (int q = 0; q < kWideColumns; ++q) {
                const int c = q * kWide + threadIdx.x;
                if (c >= a.n) continue;
                const float h = post ? (to_f32(y.row(i)[c]) - st.x) * st.y : 0.f;
                if (dy.p != nullptr) dy.row(i)[c] = from_f32<T>(post ? st.y * (hat[q] - k0 - h * k1) : hat[q]);
                if (dx.p != nullptr) dx.row(i)[c] = from_f32<T>(a.residual * g[q]);
            }
        }
        if (out.gate != nullptr)
            for (int c = threadIdx.x; c < a.n; c += kWide) out.gate[k * a.n + c] = sum_gate[c], sum_gate[c] = 0.f;
    }
    for (int c = threadIdx.x; c < a.n; c += kWide) {
        if (out.post != nullptr) out.post[static_cast<int64_t>(blockIdx.x) * a.n + c] = sum_post[c];
        if (out.pre != nullptr) out.pre[static_cast<int64_t>(blockIdx.x) * a.n + c] = sum_pre[c];
    }
}

// Column sums in registers.
template <typename T, int VEC, int SL>
__global__ void __launch_bounds__(kTeam) join_backward_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ Parts parts, const __grid_constant__ Sums out, JoinRows<const T> x,
                                                              JoinRows<const T> y, JoinRows<const T> ds, JoinRows<const T> dz, JoinRows<T> dx, JoinRows<T> dy) {
    extern __shared__ __align__(16) float smem[];
    __shared__ __align__(16) float part[2][2][16];
    Exchange ex(part);
    const Keep keep(a.dropout);
    const bool branch = y.p != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr && dz.p != nullptr;
    const int floats = weight_floats(blockDim.x, VEC * SL);
    float* room = smem;
    Weights<VEC, SL> w_post{room}, gate{room += post ? floats : 0}, w_pre{room += a.gate != nullptr ? floats : 0};
    Staged<T, VEC, SL, 4> in(room + (pre ? floats : 0));
    const float inv_n = 1.f / static_cast<float>(a.n);
    float sum_post[SL][VEC], sum_gate[SL][VEC], sum_pre[SL][VEC];
#pragma unroll
    for (int q = 0; q < SL; ++q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) sum_post[q][k] = sum_gate[q][k] = sum_pre[q][k] = 0.f;
    if (post) w_post.load(a.w_post, a.n);
    if (pre) w_pre.load(a.w_pre, a.n);
    // the CTA's rows, part after part: parts that follow one another hold rows that do
    int64_t k = parts.count * blockIdx.x / parts.ctas, group = -1;
    const int64_t last_part = parts.count * (blockIdx.x + 1) / parts.ctas, last = part_end(parts, last_part - 1);
    int64_t i = part_begin(parts, k), end = part_end(parts, k);
    auto fetch = [&](int64_t row, int which) {
        if (row < last) {
            if (pre) in.fetch(0, which, x.row(row), a.n), in.fetch(3, which, dz.row(row), a.n);
            if (branch) in.fetch(1, which, y.row(row), a.n);
            if (ds.p != nullptr) in.fetch(2, which, ds.row(row), a.n);
        }
        in.commit();
    };
    if (VEC > 1) fetch(i, 0);
    int which = 0;
    for (; k < last_part; ++k, end = part_end(parts, k)) {
        for (; i < end; ++i, which ^= 1) {
            if (a.gate != nullptr && i / a.group_rows != group) group = i / a.group_rows, gate.load(a.gate + group * a.n, a.n);
            const float4 st = a.stats != nullptr ? a.stats[i] : make_float4(0.f, 1.f, 0.f, 1.f);
            fetch(VEC > 1 ? i + 1 : i, which ^ 1);
            in.arrived();
            uint32_t stays[SL];
            float v[SL][VEC], c01[2] = {0.f, 0.f};
#pragma unroll
            for (int q = 0; q < SL; ++q) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC;
                stays[q] = staying<VEC>(a, keep, i, c);
                if (!pre || c >= a.n) continue;
                float b[VEC], wp[VEC], g[VEC], d[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) b[e] = wp[e] = g[e] = 0.f;
                if (branch) {
                    in.get(1, which, q, b);
                    if (post) {
                        w_post.get(q, wp);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) b[e] = (b[e] - st.x) * st.y;
                    }
                    if (a.gate != nullptr) gate.get(q, g);
                }
                in.get(0, which, q, v[q]);
                joined(a, branch, stays[q], wp, g, b, v[q]);
                in.get(3, which, q, d);
                w_pre.get(q, wp);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[q][e] = c + e < a.n ? (v[q][e] - st.z) * st.w : 0.f;
                    sum_pre[q][e] = fmaf(d[e], v[q][e], sum_pre[q][e]);
                    d[e] *= wp[e];   // 0 behind the last column
                    c01[0] += d[e], c01[1] = fmaf(d[e], v[q][e], c01[1]);
                }
            }
            if (pre) {
                ex.sum(c01);
                c01[0] = a.layer ? c01[0] * inv_n : 0.f, c01[1] *= inv_n;
            }
            float k01[2] = {0.f, 0.f};
#pragma unroll
            for (int q = 0; q < SL; ++q) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC;
                if (c >= a.n) continue;
                float g[VEC], d[VEC], w[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) g[e] = 0.f;
                if (ds.p != nullptr) in.get(2, which, q, g);
                if (pre) {
                    in.get(3, which, q, d);
                    w_pre.get(q, w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) g[e] = fmaf(st.w, fmaf(-v[q][e], c01[1], fmaf(d[e], w[e], -c01[0])), g[e]);
                }
                float h[VEC];
                if (branch) in.get(1, which, q, h);
                if (dx.p != nullptr) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) d[e] = a.residual * g[e];
                    put_slot(dx.row(i), c, a.n, d);
                }
                if (!branch) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    g[e] = (stays[q] >> e & 1) && c + e < a.n ? a.scale * g[e] : 0.f;
                    if (post) h[e] = (h[e] - st.x) * st.y;
                }
                if (a.gate != nullptr) {
                    float wp[VEC];
                    if (post) w_post.get(q, wp);
                    gate.get(q, w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        sum_gate[q][e] = fmaf(g[e], post ? h[e] * wp[e] : h[e], sum_gate[q][e]);
                        g[e] *= w[e];
                    }
                }
                if (post) {
                    w_post.get(q, w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        sum_post[q][e] = fmaf(g[e], h[e], sum_post[q][e]);
                        g[e] *= w[e];
                        k01[0] += g[e], k01[1] = fmaf(g[e], h[e], k01[1]);
                    }
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[q][e] = g[e];
            }
            if (dy.p == nullptr) continue;
            if (post) {
                ex.sum(k01);
                k01[0] = a.layer ? k01[0] * inv_n : 0.f, k01[1] *= inv_n;
            }
#pragma unroll
            for (int q = 0; q < SL; ++q) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC;
                if (c >= a.n) continue;
                if (post) {
                    float h[VEC];
                    in.get(1, which, q, h);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[q][e] = st.y * fmaf(-(h[e] - st.x) * st.y, k01[1], v[q][e] - k01[0]);
                }
                put_slot(dy.row(i), c, a.n, v[q]);
            }
        }
        if (out.gate != nullptr) {
#pragma unroll
            for (int q = 0; q < SL; ++q) {
                const int c = (q * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if (c + e < a.n) out.gate[k * a.n + c + e] = sum_gate[q][e];
                    sum_gate[q][e] = 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int q = 0; q < SL; ++q) {
        const int c = (q * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (out.post != nullptr && c + e < a.n) out.post[static_cast<int64_t>(blockIdx.x) * a.n + c + e] = sum_post[q][e];
            if (out.pre != nullptr && c + e < a.n) out.pre[static_cast<int64_t>(blockIdx.x) * a.n + c + e] = sum_pre[q][e];
        }
    }
}

// to[g][c] = from[g * per][c] + ... + from[g * per + per - 1][c], in that order within eight interleaved sums.
struct Fold {
    const float* from;
    float* to;
    int64_t rows, per;
};
struct Folds {
    Fold f[3];
};
__global__ void __launch_bounds__(256) fold_kernel(const __grid_constant__ Folds folds, int n) {
    __shared__ float part[8][32];
    const Fold f = folds.f[blockIdx.z];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), which = threadIdx.x >> 5;
    for (int64_t g = blockIdx.y; g < f.rows; g += gridDim.y) {
        float sum = 0.f;
        if (c < n)
            for (int64_t k = which; k < f.per; k += 8) sum += f.from[(g * f.per + k) * n + c];
        part[which][threadIdx.x & 31] = sum;
        __syncthreads();
        if (which == 0 && c < n) {
#pragma unroll
            for (int w = 1; w < 8; ++w) sum += part[w][threadIdx.x];
            f.to[g * n + c] = sum;
        }
        __syncthreads();
    }
}

// ---- host side ----------------------------------------------------------------------------------

Parts parts_of(int64_t m, int64_t n, int64_t groups) {
    Parts p;
    p.groups = groups > 0 ? groups : 1;
    p.rows = m / p.groups;
    // CTAs that share an SM, as many as have 32 rows each: fewer would have the column sums' traffic show
    int64_t per_sm = n <= 8 * kTeam ? 8 * kTeam / (n > 256 ? n : 256) : 1;
    if (per_sm > 1 && m < per_sm * kNumSMs * 32) per_sm = m / (kNumSMs * 32) > 1 ? m / (kNumSMs * 32) : 1;
    p.ctas = per_sm * kNumSMs;
    // one group: a part for each CTA; more: four rounds of parts, so that the last round is short
    int64_t per = p.groups == 1 ? p.ctas : (4 * p.ctas + p.groups - 1) / p.groups;
    p.per_group = per < p.rows ? per : (p.rows > 0 ? p.rows : 1);
    p.count = p.groups * p.per_group;
    if (p.ctas > p.count) p.ctas = p.count;
    return p;
}
size_t gate_sums(const Parts& p, int64_t n) { return p.per_group > 1 ? static_cast<size_t>(p.count) * n : 0; }
size_t workspace_of(int64_t m, int64_t n, int64_t groups) {
    const Parts p = parts_of(m, n, groups);
    return round_up((gate_sums(p, n) + 2 * static_cast<size_t>(p.ctas) * n) * sizeof(float), 256);
}

struct JoinTensors {
    const void *a, *b, *c, *d;   // inputs: x, y, -, - or x, y, ds, dz
    int64_t ld_a, ld_b, ld_c, ld_d;
    void *e, *f;                 // outputs: s, z or dx, dy
    int64_t ld_e, ld_f;
};

// Whether the rows of every tensor begin on 16-byte boundaries.
bool in_words(const JoinTensors& t, int64_t m, int bytes) {
    const void* p[6] = {t.a, t.b, t.c, t.d, t.e, t.f};
    const int64_t ld[6] = {t.ld_a, t.ld_b, t.ld_c, t.ld_d, t.ld_e, t.ld_f};
    for (int k = 0; k < 6; ++k)
        if (p[k] != nullptr && (!aligned16(p[k]) || (m > 1 && ld[k] * bytes % 16 != 0))) return false;
    return true;
}
int threads_for(int64_t n, int columns) {
    int t = 32;
    while (t < kTeam && static_cast<int64_t>(t) * columns < n) t *= 2;
    return t;
}

constexpr int kSharedPerSm = 220 * 1024;   // leaves room for the static arrays and what the system takes of each CTA

template <typename T, int VEC, int SL> int forward_fast(const JoinArgs& a, const JoinTensors& t, cudaStream_t s) {
    const int threads = threads_for(a.n, VEC * SL), weights = (a.w_post != nullptr) + (a.gate != nullptr) + (a.w_pre != nullptr);
    const int smem = threads * VEC * SL * (4 * weights + (VEC > 1 ? 2 * 2 * static_cast<int>(sizeof(T)) : 0));
    auto kern = join_kernel<T, VEC, SL>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTeam * VEC * SL * (12 + (VEC > 1 ? 4 * static_cast<int>(sizeof(T)) : 0)));
    if (e != cudaSuccess) return cuda_failed(e);
    int per_sm = 1024 / threads;
    if (per_sm * (smem + 1280) > kSharedPerSm) per_sm = kSharedPerSm / (smem + 1280);
    if (per_sm < 1) per_sm = 1;
    const int64_t grid = a.m < static_cast<int64_t>(per_sm) * kNumSMs ? a.m : static_cast<int64_t>(per_sm) * kNumSMs;
    kern<<<static_cast<unsigned>(grid), threads, smem, s>>>(a, {static_cast<const T*>(t.a), t.ld_a}, {static_cast<const T*>(t.b), t.ld_b}, {static_cast<T*>(t.e), t.ld_e},
                                                            {static_cast<T*>(t.f), t.ld_f});
    note_launch();
    return check_launch();
}

template <typename T> int forward(const JoinArgs& a, const JoinTensors& t, cudaStream_t s) {
    constexpr int N = Word<T>::kN;
    const bool words = in_words(t, a.m, sizeof(T));
    if (a.n <= 8 * 32) return words ? forward_fast<T, N, 8 / N>(a, t, s) : forward_fast<T, 1, 8>(a, t, s);
    if (a.n <= 16 * kTeam) return words ? forward_fast<T, N, 16 / N>(a, t, s) : forward_fast<T, 1, 16>(a, t, s);
    auto kern = join_wide_kernel<T>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, BZ_MAX_WIDTH * sizeof(float));
    if (e != cudaSuccess) return cuda_failed(e);
    kern<<<static_cast<unsigned>(a.m < 2 * kNumSMs ? a.m : 2 * kNumSMs), kWide, static_cast<size_t>(a.n) * sizeof(float), s>>>(
        a, {static_cast<const T*>(t.a), t.ld_a}, {static_cast<const T*>(t.b), t.ld_b}, {static_cast<T*>(t.e), t.ld_e}, {static_cast<T*>(t.f), t.ld_f});
    note_launch();
    return check_launch();
}

template <typename T, int VEC, int SL> int backward_fast(const JoinArgs& a, const JoinTensors& t, const Parts& p, const Sums& sums, cudaStream_t s) {
    const int threads = threads_for(a.n, VEC * SL), weights = (a.w_post != nullptr) + (a.gate != nullptr) + (a.w_pre != nullptr && t.d != nullptr);
    const int smem = threads * VEC * SL * (4 * weights + (VEC > 1 ? 4 * 2 * static_cast<int>(sizeof(T)) : 0));
    auto kern = join_backward_kernel<T, VEC, SL>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTeam * VEC * SL * (12 + (VEC > 1 ? 8 * static_cast<int>(sizeof(T)) : 0)));
    if (e != cudaSuccess) return cuda_failed(e);
    kern<<<static_cast<unsigned>(p.ctas), threads, smem, s>>>(a, p, sums, {static_cast<const T*>(t.a), t.ld_a}, {static_cast<const T*>(t.b), t.ld_b}, {static_cast<const T*>(t.c), t.ld_c},
                                                              {static_cast<const T*>(t.d), t.ld_d}, {static_cast<T*>(t.e), t.ld_e}, {static_cast<T*>(t.f), t.ld_f});
    note_launch();
    return check_launch();
}

template <typename T> int backward(const JoinArgs& a, const JoinTensors& t, const Parts& p, const Sums& sums, cudaStream_t s) {
    constexpr int N = Word<T>::kN;
    const bool words = in_words(t, a.m, sizeof(T));
    if (a.n <= 8 * kTeam) return words ? backward_fast<T, N, 8 / N>(a, t, p, sums, s) : backward_fast<T, 1, 8>(a, t, p, sums, s);
    if constexpr (sizeof(T) == 2)
        if (a.n <= 16 * kTeam && words) return backward_fast<T, N, 16 / N>(a, t, p, sums, s);
    auto kern = join_wide_backward_kernel<T>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * BZ_MAX_WIDTH * sizeof(float));
    if (e != cudaSuccess) return cuda_failed(e);
    kern<<<static_cast<unsigned>(p.ctas), kWide, 3 * static_cast<size_t>(a.n) * sizeof(float), s>>>(
        a, p, sums, {static_cast<const T*>(t.a), t.ld_a}, {static_cast<const T*>(t.b), t.ld_b}, {static_cast<const T*>(t.c), t.ld_c}, {static_cast<const T*>(t.d), t.ld_d},
        {static_cast<T*>(t.e), t.ld_e}, {static_cast<T*>(t.f), t.ld_f});
    note_launch();
    return check_launch();
}

// A row tensor: rows that do not overlap, elements on their type's boundary.
bool good(const void* p, int64_t ld, int64_t m, int64_t n, int bytes) {
    return p == nullptr || ((m <= 1 || ld >= n) && reinterpret_cast<uintptr_t>(p) % bytes == 0);
}
bool far_apart(const JoinTensors& t) {
    const int64_t lim = int64_t(1) << 31;
    return t.ld_a >= lim || t.ld_b >= lim || t.ld_c >= lim || t.ld_d >= lim || t.ld_e >= lim || t.ld_f >= lim;
}
bool words(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// What both calls check of sizes and form; `least` gets the dropout threshold.
int check(int dtype, int64_t m, int64_t n, int norm, float eps, const void* y, const float* w_post, const float* gate, int64_t groups, float residual,
          float branch, double rate, const uint64_t* rng, const float* w_pre, const void* stats, uint32_t* least) {
    if (element_bytes(dtype) == 0 || m < 0 || n < 0 || (norm != BZ_NORM_RMS && norm != BZ_NORM_LAYER) || groups < 0 || !isfinite(residual) || !isfinite(branch) ||
        !(eps >= 0.f) || isinf(eps) || !drop_threshold(rate, least) || !aligned16(stats) || !aligned8(rng) || !words(w_post) || !words(gate) || !words(w_pre))
        return BZ_ERR_INVALID_ARG;
    if (m >= (int64_t(1) << 31) || n > BZ_MAX_WIDTH || groups >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    if ((gate != nullptr) != (groups > 0) || (groups > 0 && m % groups != 0)) return BZ_ERR_INVALID_ARG;
    if (m > 0 && y == nullptr && (w_post != nullptr || gate != nullptr || *least != 0)) return BZ_ERR_INVALID_ARG;
    if (*least != 0 && rng == nullptr) return BZ_ERR_INVALID_ARG;
    return BZ_OK;
}

JoinArgs join_args(int64_t m, int64_t n, int norm, float eps, const float* w_post, const float* gate, int64_t groups, float residual, float branch, uint32_t least,
                   const uint64_t* rng, const float* w_pre, const float* stats) {
    JoinArgs a{};
    a.m = m, a.n = static_cast<int>(n), a.layer = norm == BZ_NORM_LAYER, a.eps = eps, a.w_post = w_post, a.gate = gate, a.w_pre = w_pre;
    a.group_rows = groups > 0 && m > 0 ? m / groups : (m > 0 ? m : 1), a.residual = residual, a.scale = branch * drop_scale(least), a.drop = least != 0;
    a.dropout = {least != 0 ? rng : nullptr, least, drop_scale(least)};
    a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
    return a;
}

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" int bz_join(const void* x, int64_t ld_x, const void* y, int64_t ld_y, int dtype, int64_t m, int64_t n, int norm, float eps,
                       const float* w_post, const float* gate, int64_t groups, float residual_scale, float branch_scale, double rate,
                       const uint64_t* rng, const float* w_pre, void* s, int64_t ld_s, void* z, int64_t ld_z, float* stats, void* stream) {
    uint32_t least;
    const int st = check(dtype, m, n, norm, eps, y, w_post, gate, groups, residual_scale, branch_scale, rate, rng, w_pre, stats, &least);
    if (st != BZ_OK) return st;
    if (m == 0 || n == 0) return BZ_OK;
    const int bytes = element_bytes(dtype);
    const JoinTensors t{x, y, nullptr, nullptr, ld_x, ld_y, 0, 0, s, z, ld_s, ld_z};
    if (x == nullptr || (s == nullptr && z == nullptr) || (z != nullptr) != (w_pre != nullptr) || !good(x, ld_x, m, n, bytes) || !good(y, ld_y, m, n, bytes) ||
        !good(s, ld_s, m, n, bytes) || !good(z, ld_z, m, n, bytes))
        return BZ_ERR_INVALID_ARG;
    if (m > 1 && far_apart(t)) return BZ_ERR_UNSUPPORTED;
    const JoinArgs a = join_args(m, n, norm, eps, w_post, gate, groups, residual_scale, branch_scale, least, rng, w_pre, stats);
    cudaStream_t stream_ = static_cast<cudaStream_t>(stream);
    if (dtype == BZ_F32) return forward<float>(a, t, stream_);
    if (dtype == BZ_F16) return forward<__half>(a, t, stream_);
    return forward<__nv_bfloat16>(a, t, stream_);
}

extern "C" size_t bz_join_workspace_bytes(int64_t m, int64_t n, int64_t groups) {
    if (m < 0 || n < 0 || groups < 0 || m >= (int64_t(1) << 31) || n > BZ_MAX_WIDTH || groups >= (int64_t(1) << 31) || (groups > 0 && m % groups != 0)) return 0;
    return workspace_of(m, n, groups);
}

extern "C" int bz_join_backward(const void* x, int64_t ld_x, const void* y, int64_t ld_y, int dtype, int64_t m, int64_t n, int norm,
                                const float* w_post, const float* gate, int64_t groups, float residual_scale, float branch_scale, double rate,
                                const uint64_t* rng, const float* w_pre, const float* stats, const void* ds, int64_t ld_ds, const void* dz,
                                int64_t ld_dz, void* dx, int64_t ld_dx, void* dy, int64_t ld_dy, float* dw_post, float* dgate, float* dw_pre,
                                void* workspace, size_t workspace_bytes, void* stream) {
    uint32_t least;
    const int st = check(dtype, m, n, norm, 0.f, y, w_post, gate, groups, residual_scale, branch_scale, rate, rng, w_pre, stats, &least);
    if (st != BZ_OK) return st;
    const int bytes = element_bytes(dtype);
    JoinTensors t{x, y, ds, dz, ld_x, ld_y, ld_ds, ld_dz, dx, dy, ld_dx, ld_dy};
    const bool pre = dz != nullptr && w_pre != nullptr, sums = dw_post != nullptr || dgate != nullptr || dw_pre != nullptr;
    if ((dw_post != nullptr && w_post == nullptr) || (dgate != nullptr && gate == nullptr) || (dw_pre != nullptr && w_pre == nullptr) || !words(dw_post) || !words(dgate) ||
        !words(dw_pre))
        return BZ_ERR_INVALID_ARG;
    if (n == 0) return BZ_OK;
    if (dx == nullptr && dy == nullptr && !sums) return m == 0 ? BZ_OK : BZ_ERR_INVALID_ARG;
    if (m == 0 && !sums) return BZ_OK;
    if (m > 0 && ((pre && x == nullptr) || (dz != nullptr && w_pre == nullptr) || ((pre || w_post != nullptr) && stats == nullptr) || (dy != nullptr && y == nullptr) ||
                  !good(x, ld_x, m, n, bytes) || !good(y, ld_y, m, n, bytes) || !good(ds, ld_ds, m, n, bytes) || !good(dz, ld_dz, m, n, bytes) ||
                  !good(dx, ld_dx, m, n, bytes) || !good(dy, ld_dy, m, n, bytes)))
        return BZ_ERR_INVALID_ARG;
    if (m > 1 && far_apart(t)) return BZ_ERR_UNSUPPORTED;
    const Parts p = parts_of(m, n, groups);
    if (sums && (workspace == nullptr || !aligned256(workspace) || workspace_bytes < workspace_of(m, n, groups))) return BZ_ERR_WORKSPACE;
    float* room = static_cast<float*>(workspace);
    Sums partial{};
    Folds folds{};
    int count = 0;
    auto fold = [&](float* to, int64_t rows, int64_t per) {
        float* from = room;
        room += rows * per * n;
        folds.f[count++] = {from, to, rows, per};
        return from;
    };
    if (dw_post != nullptr) partial.post = fold(dw_post, 1, p.ctas);
    if (dw_pre != nullptr) partial.pre = fold(dw_pre, 1, p.ctas);
    if (dgate != nullptr) partial.gate = p.per_group > 1 ? fold(dgate, p.groups, p.per_group) : dgate;
    const JoinArgs a = join_args(m, n, norm, 0.f, w_post, gate, groups, residual_scale, branch_scale, least, rng, w_pre, stats);
    cudaStream_t stream_ = static_cast<cudaStream_t>(stream);
    const int done = dtype == BZ_F32 ? backward<float>(a, t, p, partial, stream_) : dtype == BZ_F16 ? backward<__half>(a, t, p, partial, stream_)
                                                                                              : backward<__nv_bfloat16>(a, t, p, partial, stream_);
    if (done != BZ_OK || count == 0) return done;
    int64_t rows = 1;
    for (int k = 0; k < count; ++k) rows = rows > folds.f[k].rows ? rows : folds.f[k].rows;
    fold_kernel<<<dim3(static_cast<unsigned>((n + 31) / 32), static_cast<unsigned>(rows < 1024 ? rows : 1024), count), 256, 0, stream_>>>(folds, static_cast<int>(n));
    note_launch();
    return check_launch();
}
