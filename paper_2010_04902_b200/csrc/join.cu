// The join of a block to its residual stream: norm of the block's output, gate, dropout, residual scale, norm for the next
// block - and its gradient.
//
// With h = norm(y) (h = y without that norm), w = scale * gate * w_post by column (scale: the branch's times dropout's) and [.] the mask:
//   s = residual * x + [h w],  z = norm(s) w_pre;
//   g = ds + norm'(dz w_pre),  dx = residual * g,  e = [g] w,  dy = norm'(e),
//   P = sum over a group's rows of [g] h:  dgate = scale * w_post * P,  dw_post = sum over the groups of scale * gate * P,
//   dw_pre = sum over rows of dz norm(s).
// One read of x, y and one write of s, z forward; one read of x, y, ds, dz and one write of dx, dy backward.
//
// A thread owns the same columns of every row: COLS of them, in 16-byte words (rows that do not begin on 16-byte boundaries are
// copied in whole words and shifted in shared memory).  So what belongs to a column (w and w_pre in shared memory, the column sums in
// registers) needs no exchange.  A CTA of up to 512 threads holds a row, a cluster of two or four a wider one; the row's
// sums cost one barrier each.  The next row's words come by cp.async while a row is worked on: a thread copies what it reads
// itself, and waits for nobody.
//
// 8192 x 4096 bfloat16 with both norms, a gate and dropout: forward 70 us (42 at the copy's rate; 49 with the second norm alone), backward
// 114 (62; 82).  Bound by instructions and their latencies: 40 and 57 an element (the generator 8 of them each time), issue slots 55 and
// 51 % with 16 warps an SM, which wait for two sums a row.  Sixteen columns a thread carry the bookkeeping of a row better
// than eight (backward 156 us); what takes part in a call known beforehand made the forward call 2 % faster and the backward call
// 4 % slower (registers spilled).
#include <cooperative_groups.h>

#include <cmath>

#include "dropout_rule.h"
#include "philox.cuh"
#include "worker_common.cuh"

namespace bz {

namespace {

namespace cg = cooperative_groups;

constexpr int kTeam = 512;       // threads of a CTA at most
constexpr int kMostRanks = 4;    // CTAs of a cluster

struct JoinArgs {
    int64_t m;
    int n, layer;
    float eps;
    const float *w_post, *gate, *w_pre;
    int64_t group_rows;          // rows that share a gate row
    float residual, scale;       // scale of the branch: its own times dropout's
    int drop;                    // whether there is dropout
    Dropout dropout;
    float4* stats;
};
template <typename T> struct JoinRows {
    T* p;
    int64_t ld;
    T* end;   // behind the tensor's last element
    __device__ __forceinline__ T* row(int64_t i) const { return p + i * ld; }
};

// ---- pairs of elements ---------------------------------------------------------------------------

__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }
template <typename T> __device__ __forceinline__ float2 word_pair(const uint4& w, int k) {   // elements 2k, 2k + 1 of a word
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (sizeof(T) == 4)
        return make_float2(__uint_as_float(u[2 * k]), __uint_as_float(u[2 * k + 1]));
    else
        return unpack2(T(), u[k]);
}

// Threads of the CTA: known beforehand for wide rows (the distances of a thread's words are constants then), or 0.
template <int THREADS> __device__ __forceinline__ int team_threads() { return THREADS ? THREADS : static_cast<int>(blockDim.x); }

// Where a thread's columns lie: element e of COLS.
template <int VEC, int THREADS> struct Columns {
    int first;   // of the CTA
    __device__ __forceinline__ int of(int e) const { return first + static_cast<int>(threadIdx.x) * VEC + e / VEC * team_threads<THREADS>() * VEC + e % VEC; }
};

// NT tensors' elements of a row, as they were loaded.  The next row's are on their way to the other half of the room meanwhile; a half is
// filled again only a whole row after it was read.  SHIFT: rows that do not all begin on 16-byte boundaries.
template <typename T, int COLS, int NT, int THREADS, bool SHIFT> struct Held {
    static constexpr int VEC = Word<T>::kN, kWords = COLS / VEC;
    uint4* room;
    int half = 0;
    int filled[kWords];   // bytes of the row in each word
    __device__ __forceinline__ Held(void* smem, int n, const Columns<VEC, THREADS>& at) : room(static_cast<uint4*>(smem) + threadIdx.x) {
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            filled[q] = min(max((n - at.of(q * VEC)) * static_cast<int>(sizeof(T)), 0), 16);
            if (filled[q] == 0) {   // never copied, and stays zero
#pragma unroll
                for (int t = 0; t < NT; ++t) *place(0, t, q) = *place(1, t, q) = make_uint4(0, 0, 0, 0);
            }
        }
    }
    __device__ __forceinline__ uint4* place(int which, int t, int q) const { return room + which * (NT * kWords * team_threads<THREADS>()) + (t * kWords + q) * team_threads<THREADS>(); }
    __host__ __device__ static int bytes(int threads, int) { return 2 * NT * kWords * threads * 16; }
    // the next row's: fetches, then commit; what a word has behind the row's end is filled with zeros
    __device__ __forceinline__ void fetch(int t, const JoinRows<const T>& from, int64_t i, const Columns<VEC, THREADS>& at) {
        const T* row = from.row(i);
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(place(half, t, q)));
            if (filled[q] > 0) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row + at.of(q * VEC)), "r"(filled[q]) : "memory");
        }
    }
    __device__ __forceinline__ void commit() {
        asm volatile("cp.async.commit_group;" ::: "memory");
        half ^= 1;
    }
    __device__ __forceinline__ static void arrived() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }   // all but the last commit
    __device__ __forceinline__ void get(int t, float2 (&v)[COLS / 2], const Columns<VEC, THREADS>&) const {   // this row's: the half that the next commit will fill
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            const uint4 w = *place(half, t, q);
#pragma unroll
            for (int p = 0; p < VEC / 2; ++p) v[q * (VEC / 2) + p] = word_pair<T>(w, p);
        }
    }
    __device__ __forceinline__ void put(int, T* row, const Columns<VEC, THREADS>& at, const float2 (&v)[COLS / 2]) const {
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            const int c = at.of(q * VEC);
            float x[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = k & 1 ? v[(q * VEC + k) / 2].y : v[(q * VEC + k) / 2].x;
            if (filled[q] == 16) {
                *reinterpret_cast<uint4*>(row + c) = Word<T>::pack(x);
            } else if (filled[q] > 0) {
                rare();
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if ((k + 1) * static_cast<int>(sizeof(T)) <= filled[q]) row[c + k] = from_f32<T>(x[k]);
            }
        }
    }
};
// Rows that do not all begin on 16-byte boundaries.  Whole words are copied, from the boundary at or before the row on, and a thread's elements lie in two
// of them: its own copy and its neighbour's, so a row begins with a barrier.  Outputs go through shared memory in the same way.
template <typename T, int COLS, int NT, int THREADS> struct Held<T, COLS, NT, THREADS, true> {
    static constexpr int N = Word<T>::kN, kWords = COLS / N;
    uint4 *room, *out;
    int half = 0, lead[NT];   // of this row's tensors; the next row's are found anew
    int n, left[NT];
    __device__ __forceinline__ Held(void* smem, int n_, const Columns<N, THREADS>&) : room(static_cast<uint4*>(smem)), n(n_) { out = room + 2 * NT * words(); }
    __device__ __forceinline__ static int words() { return kWords * team_threads<THREADS>() + 1; }
    __host__ __device__ static int bytes(int threads, int outputs) { return (2 * NT + outputs) * (kWords * threads + 1) * 16; }
    __device__ __forceinline__ void fetch(int t, const JoinRows<const T>& from, int64_t i, const Columns<N, THREADS>& at) {
        const T* row = from.row(i);
        left[t] = row_lead<T, N>(row);
        const T* begin = row - left[t] + at.first;
        uint4* to = room + (half * NT + t) * words();
        auto copy = [&](int w) {
            const T* p = begin + w * N;
            if (p >= row + n) return;   // behind the row: its columns are masked
            if (p < from.p) {           // before the tensor: element by element
                rare();
                for (int e = 0; e < N; ++e)
                    if (p + e >= from.p && p + e < from.end) reinterpret_cast<T*>(to + w)[e] = p[e];
                return;
            }
            const int64_t room_left = (from.end - p) * static_cast<int64_t>(sizeof(T));
            const int size = room_left < 16 ? static_cast<int>(room_left) : 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to + w))), "l"(p), "r"(size) : "memory");
        };
#pragma unroll
        for (int q = 0; q < kWords; ++q) copy(q * team_threads<THREADS>() + threadIdx.x);
        if (threadIdx.x == 0) copy(kWords * team_threads<THREADS>());
    }
    __device__ __forceinline__ void commit() {
        asm volatile("cp.async.commit_group;" ::: "memory");
        half ^= 1;
    }
    // this row's words, everyone's
    __device__ __forceinline__ void arrived() {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t) lead[t] = left[t];
    }
    // the four registers from element `by` on of two words
    __device__ __forceinline__ static uint4 shifted(const uint4& a, const uint4& b, int by) {
        uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        const int words = by * static_cast<int>(sizeof(T)) / 4;
        if (words & 2) {
#pragma unroll
            for (int k = 0; k < 6; ++k) u[k] = u[k + 2];
        }
        if (words & 1) {
#pragma unroll
            for (int k = 0; k < 5; ++k) u[k] = u[k + 1];
        }
        if (sizeof(T) == 2 && (by & 1)) {
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = __funnelshift_r(u[k], u[k + 1], 16);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    // after the next row's commit: this row's half is the one that the commit after it will fill
    __device__ __forceinline__ void get(int t, float2 (&v)[COLS / 2], const Columns<N, THREADS>& at) const {
        const uint4* from = room + (half * NT + t) * words();
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            const int w = q * team_threads<THREADS>() + threadIdx.x;
            const uint4 u = shifted(from[w], from[w + 1], lead[t]);
#pragma unroll
            for (int p = 0; p < N / 2; ++p) v[q * (N / 2) + p] = word_pair<T>(u, p);
            const int c = at.of(q * N);
            if (c + N > n) {
                rare();
#pragma unroll
                for (int p = 0; p < N / 2; ++p) {
                    if (c + 2 * p >= n) v[q * (N / 2) + p].x = 0.f;
                    if (c + 2 * p + 1 >= n) v[q * (N / 2) + p].y = 0.f;
                }
            }
        }
    }
    // which: 0 or 1, the output's room; ends behind a barrier
    __device__ __forceinline__ void put(int which, T* row, const Columns<N, THREADS>& at, const float2 (&v)[COLS / 2]) const {
        uint4* mine = out + which * words();
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            float x[N];
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = k & 1 ? v[(q * N + k) / 2].y : v[(q * N + k) / 2].x;
            mine[q * team_threads<THREADS>() + threadIdx.x] = Word<T>::pack(x);
        }
        __syncthreads();
        const int shift = row_lead<T, N>(row), all = kWords * team_threads<THREADS>(), width = all * N;
        T* to = row - shift + at.first;
        auto store = [&](int w) {   // columns w N - shift ... of the CTA's
            const int c = w * N - shift;
            if (c >= width || at.first + c >= n) return;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            const uint4 u = shift == 0 ? mine[w] : shifted(w > 0 ? mine[w - 1] : zero, w < all ? mine[w] : zero, N - shift);
            if (c >= 0 && c + N <= width && at.first + c + N <= n) {
                *reinterpret_cast<uint4*>(to + w * N) = u;
            } else {
                rare();
                const uint32_t r[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c + e >= 0 && c + e < width && at.first + c + e < n) {
                        if constexpr (sizeof(T) == 4)
                            to[w * N + e] = __uint_as_float(r[e]);
                        else
                            reinterpret_cast<uint16_t*>(to)[w * N + e] = static_cast<uint16_t>(r[e / 2] >> (e & 1 ? 16 : 0));
                    }
            }
        };
#pragma unroll
        for (int q = 0; q < kWords; ++q) store(q * team_threads<THREADS>() + threadIdx.x);
        if (threadIdx.x == 0) store(all);
    }
};

// A number for each column in shared memory, where only its thread looks; 0 behind the last column.
template <int VEC, int COLS, int THREADS> struct ByColumn {
    float4* room;
    template <typename F> __device__ __forceinline__ void set(int n, const Columns<VEC, THREADS>& at, F value) const {
#pragma unroll
        for (int k = 0; k < COLS / 4; ++k) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = at.of(4 * k + e) < n ? value(at.of(4 * k + e)) : 0.f;
            room[k * team_threads<THREADS>() + threadIdx.x] = make_float4(x[0], x[1], x[2], x[3]);
        }
    }
    __device__ __forceinline__ void get(int k, float2 (&w)[2]) const {   // pairs 2k, 2k + 1
        const float4 f = room[k * team_threads<THREADS>() + threadIdx.x];
        w[0] = make_float2(f.x, f.y), w[1] = make_float2(f.z, f.w);
    }
};

// Sums over the row's threads, one barrier each; two sets of partial sums in turn.
struct ExchangeRoom {
    float warp[2][2][kTeam / 32];
    float rank[2][2][kMostRanks];
};
template <int THREADS> struct Exchange {
    using Room = ExchangeRoom;
    Room* room;
    int ranks, turn = 0;
    __device__ __forceinline__ Exchange(Room* r, int ranks_) : room(r), ranks(ranks_) {
        for (int k = threadIdx.x; k < kTeam / 8; k += team_threads<THREADS>()) (&r->warp[0][0][0])[k] = 0.f;
        if (ranks > 1)
            cg::this_cluster().sync();
        else
            __syncthreads();
    }
    template <int K> __device__ __forceinline__ void sum(float (&v)[K]) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
        const int warps = team_threads<THREADS>() >> 5;
        if (warps > 1) {
            if ((threadIdx.x & 31) == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) room->warp[turn][k][threadIdx.x >> 5] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int w = 0; w < kTeam / 32; w += 4) {
                    if (w >= warps) break;
                    const float4 p = *reinterpret_cast<const float4*>(&room->warp[turn][k][w]);
                    v[k] += (p.x + p.y) + (p.z + p.w);
                }
            }
        }
        if (ranks > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            if (threadIdx.x < ranks) {
#pragma unroll
                for (int k = 0; k < K; ++k) cluster.map_shared_rank(room, threadIdx.x)->rank[turn][k][cluster.block_rank()] = v[k];
            }
            cluster.sync();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.f;
                for (int r = 0; r < ranks; ++r) v[k] += room->rank[turn][k][r];
            }
        }
        turn ^= 1;
    }
};

// The bits of a row's elements, two halves of a word a pair.  Where the thread's words are whole groups of the generator it makes
// its own; else the CTA makes each group once and leaves the 16-bit numbers in shared memory, two rows' in turn.
template <int VEC, int COLS, int THREADS> struct Mask {
    uint16_t* room;      // [2][width + 16]
    int width, turn = 0;
    bool own;
    __device__ __forceinline__ static int halves(int width) { return width + 16; }
    __device__ __forceinline__ void make(const JoinArgs& a, const Keep& keep, int64_t i, const Columns<VEC, THREADS>& at, uint32_t (&r)[COLS / 2]) {
        const uint64_t first = static_cast<uint64_t>(i) * a.n;
        if constexpr (VEC == 8) {
            if (own) {
#pragma unroll
                for (int q = 0; q < COLS / 8; ++q) {
                    const uint4 w = keep.words((first + at.of(q * 8)) >> 3);
                    r[4 * q] = w.x, r[4 * q + 1] = w.y, r[4 * q + 2] = w.z, r[4 * q + 3] = w.w;
                }
                return;
            }
        }
        const uint64_t begin = first + at.first;
        const int lead = static_cast<int>(begin & 7), used = min(width, a.n - at.first);
        uint16_t* to = room + turn * halves(width);
        for (int g = threadIdx.x; g * 8 < lead + used; g += team_threads<THREADS>()) reinterpret_cast<uint4*>(to)[g] = keep.words((begin >> 3) + g);
        __syncthreads();
        turn ^= 1;
#pragma unroll
        for (int p = 0; p < COLS / 2; ++p) {
            // numbers behind the last column are whatever lies there
            const int c = at.of(2 * p) - at.first + lead, d = at.of(2 * p + 1) - at.first + lead;
            r[p] = static_cast<uint32_t>(to[c]) | static_cast<uint32_t>(to[d]) << 16;
        }
    }
    __device__ __forceinline__ static float2 apply(const Keep& keep, uint32_t r, float2 v) { return make_float2(keep.lower(r) ? v.x : 0.f, keep.upper(r) ? v.y : 0.f); }
};

// Mean and 1 / deviation of what the row's threads hold.
template <int VEC, int COLS, int THREADS> __device__ __forceinline__ float2 held_norm(const JoinArgs& a, Exchange<THREADS>& ex, const Columns<VEC, THREADS>& at, const float2 (&v)[COLS / 2], float inv_n) {
    float mean = 0.f, t[1];
    float2 sum = pair(0.f);
    if (a.layer) {
#pragma unroll
        for (int p = 0; p < COLS / 2; ++p) sum = __fadd2_rn(sum, v[p]);   // 0 behind the last column
        t[0] = sum.x + sum.y;
        ex.sum(t);
        mean = t[0] * inv_n;
        sum = pair(0.f);
    }
    if (mean == 0.f || at.of(COLS - 1) < a.n) {
#pragma unroll
        for (int p = 0; p < COLS / 2; ++p) {
            const float2 d = __fadd2_rn(v[p], pair(-mean));
            sum = __ffma2_rn(d, d, sum);
        }
    } else {
#pragma unroll
        for (int p = 0; p < COLS / 2; ++p) {
            const float x = at.of(2 * p) < a.n ? v[p].x - mean : 0.f, y = at.of(2 * p + 1) < a.n ? v[p].y - mean : 0.f;
            sum.x = fmaf(x, x, sum.x), sum.y = fmaf(y, y, sum.y);
        }
    }
    t[0] = sum.x + sum.y;
    ex.sum(t);
    return {mean, 1.f / sqrtf(t[0] * inv_n + a.eps)};
}

// v[p] = s of the pair, from x[p].
template <int VEC, int COLS, int THREADS>
__device__ __forceinline__ void joined(const JoinArgs& a, const Keep& keep, bool branch, const float2 (&h)[COLS / 2], const uint32_t (&r)[COLS / 2], const ByColumn<VEC, COLS, THREADS>& weight,
                                       float2 (&v)[COLS / 2]) {
    if (branch) {
#pragma unroll
        for (int k = 0; k < COLS / 4; ++k) {
            float2 w[2];
            weight.get(k, w);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int p = 2 * k + e;
                float2 b = __fmul2_rn(h[p], w[e]);
                if (a.drop) b = Mask<VEC, COLS, THREADS>::apply(keep, r[p], b);
                v[p] = __ffma2_rn(v[p], pair(a.residual), b);
            }
        }
    } else {
#pragma unroll
        for (int p = 0; p < COLS / 2; ++p) v[p] = __fmul2_rn(v[p], pair(a.residual));
    }
}

// The weight of a column of the branch.
__device__ __forceinline__ float branch_weight(const JoinArgs& a, int64_t group, int c) {
    const float w = a.gate != nullptr ? a.scale * a.gate[group * a.n + c] : a.scale;
    return a.w_post != nullptr ? w * a.w_post[c] : w;
}

// Threads that an SM holds of the kernel, by its registers; of a CTA without a constant number.
template <typename T, int COLS, bool SHIFT> constexpr int held_threads() { return sizeof(T) == 2 && COLS == 8 && !SHIFT ? 768 : kTeam; }
template <int COLS> constexpr int most_threads() { return COLS == 8 ? 256 : kTeam; }
// 16-bit rows in words of 4096 to 6144 columns (of a CTA): a row's time is its own chain of barriers, 2.3 us, and an SM holds two CTAs of 320
// (96 registers a thread) or 384 (80) threads.  Bfloat16 with both norms and dropout: 8192 x 5120 87 us, one CTA an SM 128; x 6144 101, 131; 4096 x 12288
// in pairs of CTAs 132, 202.  (Three CTAs of 256 threads, for up to 4096 columns: 8192 rows 70 us, as with two; 1024 rows 18.5 for 16.6.)
template <typename T, int COLS, bool SHIFT> constexpr bool two_wide() { return COLS == 16 && sizeof(T) == 2 && !SHIFT; }

template <typename T, int COLS, int THREADS, bool SHIFT>
__global__ void __launch_bounds__(THREADS ? THREADS : most_threads<COLS>(), THREADS == 320 || THREADS == 384 ? 2 : held_threads<T, COLS, SHIFT>() / (THREADS ? THREADS : most_threads<COLS>())) join_kernel(const __grid_constant__ JoinArgs a, int ranks, JoinRows<const T> x, JoinRows<const T> y, JoinRows<T> s, JoinRows<T> z) {
    constexpr int VEC = Word<T>::kN;
    extern __shared__ __align__(16) float4 smem[];
    __shared__ __align__(16) ExchangeRoom room;
    const int width = team_threads<THREADS>() * COLS, rank = blockIdx.x % ranks, team = blockIdx.x / ranks, teams = gridDim.x / ranks;
    const Columns<VEC, THREADS> at{rank * width};
    const ByColumn<VEC, COLS, THREADS> weight{smem}, w_pre{smem + width / 4};
    Held<T, COLS, 2, THREADS, SHIFT> in(smem + width / 2, a.n, at);
    Mask<VEC, COLS, THREADS> mask{reinterpret_cast<uint16_t*>(smem + width / 2 + Held<T, COLS, 2, THREADS, SHIFT>::bytes(team_threads<THREADS>(), 2) / 16), width, 0, VEC == 8 && a.n % 8 == 0};
    const bool branch = y.p != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr;
    const float inv_n = 1.f / static_cast<float>(a.n);
    int64_t i = a.m * team / teams, change = i;   // change: the row at which the next gate row begins
    const int64_t last = a.m * (team + 1) / teams;
    auto fetch = [&](int64_t row) {
        in.fetch(0, x, row, at);
        if (branch) in.fetch(1, y, row, at);
    };
    if (i < last) fetch(i);
    in.commit();
    const Keep keep(a.dropout);
    if (pre) w_pre.set(a.n, at, [&](int c) { return __ldg(a.w_pre + c); });
    Exchange<THREADS> ex(&room, ranks);
    for (; i < last; ++i) {
        if (branch && i == change) {
            const int64_t group = i / a.group_rows;
            change = (group + 1) * a.group_rows;
            weight.set(a.n, at, [&](int c) { return branch_weight(a, group, c); });
        }
        if (SHIFT) in.arrived();
        if (i + 1 < last) fetch(i + 1);
        in.commit();
        if (!SHIFT) in.arrived();
        uint32_t r[COLS / 2];
        if (a.drop) mask.make(a, keep, i, at, r);
        float2 h[COLS / 2], v[COLS / 2], st = make_float2(0.f, 1.f), to = make_float2(0.f, 1.f);
        if (branch) {
            in.get(1, h, at);
            if (post) {
                st = held_norm<VEC, COLS, THREADS>(a, ex, at, h, inv_n);
#pragma unroll
                for (int p = 0; p < COLS / 2; ++p) h[p] = __fmul2_rn(__fadd2_rn(h[p], pair(-st.x)), pair(st.y));
            }
        }
        in.get(0, v, at);
        joined<VEC, COLS, THREADS>(a, keep, branch, h, r, weight, v);
        if (s.p != nullptr) in.put(0, s.row(i), at, v);
        if (pre) {
            to = held_norm<VEC, COLS, THREADS>(a, ex, at, v, inv_n);
#pragma unroll
            for (int k = 0; k < COLS / 4; ++k) {
                float2 w[2];
                w_pre.get(k, w);
#pragma unroll
                for (int e = 0; e < 2; ++e) v[2 * k + e] = __fmul2_rn(__fmul2_rn(__fadd2_rn(v[2 * k + e], pair(-to.x)), pair(to.y)), w[e]);
            }
            in.put(1, z.row(i), at, v);
        }
        if (a.stats != nullptr && threadIdx.x == 0 && rank == 0) a.stats[i] = make_float4(st.x, st.y, to.x, to.y);
    }
}

// ---- gradient -----------------------------------------------------------------------------------
//
// The rows are cut into parts that lie within a gate's group each; a CTA (cluster) takes a run of parts and keeps the column sums of
// dw_post and dw_pre over all of them, that of dgate over a part.  The sums of the CTAs and parts go to the workspace and are
// added up in their order by a second kernel.

// Sums over the row of c0 (0 but for LAYER) and c1.
template <int THREADS> __device__ __forceinline__ float2 row_sums(const JoinArgs& a, Exchange<THREADS>& ex, float2 c0, float2 c1) {
    if (a.layer) {
        float t[2] = {c0.x + c0.y, c1.x + c1.y};
        ex.sum(t);
        return make_float2(t[0], t[1]);
    }
    float t[1] = {c1.x + c1.y};
    ex.sum(t);
    return make_float2(0.f, t[0]);
}

struct Parts {
    int64_t groups, rows, per_group, count, teams;   // rows of a group; parts of a group, of all
};
struct Sums {
    float *post, *gate, *pre;   // [teams][n], [count][n], [teams][n]; nullptr: not wanted
};

__device__ __forceinline__ int64_t part_begin(const Parts& p, int64_t k) { return k / p.per_group * p.rows + k % p.per_group * p.rows / p.per_group; }
__device__ __forceinline__ int64_t part_end(const Parts& p, int64_t k) { return k / p.per_group * p.rows + (k % p.per_group + 1) * p.rows / p.per_group; }

template <typename T, int COLS, int THREADS, bool SHIFT>
__global__ void __launch_bounds__(THREADS ? THREADS : kTeam, 512 / (THREADS ? THREADS : kTeam)) join_backward_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ Parts parts, const __grid_constant__ Sums out, int ranks,
                                                              JoinRows<const T> x, JoinRows<const T> y, JoinRows<const T> ds, JoinRows<const T> dz, JoinRows<T> dx, JoinRows<T> dy) {
    constexpr int VEC = Word<T>::kN;
    extern __shared__ __align__(16) float4 smem[];
    __shared__ __align__(16) ExchangeRoom room;
    const int width = team_threads<THREADS>() * COLS, rank = blockIdx.x % ranks, team = blockIdx.x / ranks;
    const Columns<VEC, THREADS> at{rank * width};
    const ByColumn<VEC, COLS, THREADS> weight{smem}, w_pre{smem + width / 4};
    const ByColumn<VEC, COLS, THREADS> sum_post{smem + width / 2};
    Held<T, COLS, 4, THREADS, SHIFT> in(smem + 3 * width / 4, a.n, at);
    Mask<VEC, COLS, THREADS> mask{reinterpret_cast<uint16_t*>(smem + 3 * width / 4 + Held<T, COLS, 4, THREADS, SHIFT>::bytes(team_threads<THREADS>(), 2) / 16), width, 0, VEC == 8 && a.n % 8 == 0};
    const bool branch = y.p != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr && dz.p != nullptr, stream = ds.p != nullptr;
    const float inv_n = 1.f / static_cast<float>(a.n);
    float2 sum_branch[COLS / 2], sum_pre[COLS / 2];
#pragma unroll
    for (int p = 0; p < COLS / 2; ++p) sum_branch[p] = sum_pre[p] = pair(0.f);
    if (post) sum_post.set(a.n, at, [](int) { return 0.f; });
    // the CTA's rows, part after part: parts that follow one another hold rows that do
    int64_t k = parts.count * team / parts.teams;
    const int64_t last_part = parts.count * (team + 1) / parts.teams, last = part_end(parts, last_part - 1);
    int64_t i = part_begin(parts, k), end = part_end(parts, k);
    auto fetch = [&](int64_t row) {
        if (pre) in.fetch(0, x, row, at), in.fetch(3, dz, row, at);
        if (branch) in.fetch(1, y, row, at);
        if (stream) in.fetch(2, ds, row, at);
    };
    if (i < last) fetch(i);
    in.commit();
    const Keep keep(a.dropout);
    if (pre) w_pre.set(a.n, at, [&](int c) { return __ldg(a.w_pre + c); });
    Exchange<THREADS> ex(&room, ranks);
    for (; k < last_part; ++k, end = part_end(parts, k)) {
        const int64_t group = k / parts.per_group;
        if (branch && i < end) weight.set(a.n, at, [&](int c) { return branch_weight(a, group, c); });
        for (; i < end; ++i) {
            const float4 st = a.stats != nullptr ? a.stats[i] : make_float4(0.f, 1.f, 0.f, 1.f);
            if (SHIFT) in.arrived();
            if (i + 1 < last) fetch(i + 1);
            in.commit();
            if (!SHIFT) in.arrived();
            uint32_t r[COLS / 2];
            if (a.drop) mask.make(a, keep, i, at, r);
            float2 h[COLS / 2], g[COLS / 2];
            if (branch) {
                in.get(1, h, at);
                if (post) {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) h[p] = __fmul2_rn(__fadd2_rn(h[p], pair(-st.x)), pair(st.y));
                }
            }
            if (pre) {
                float2 v[COLS / 2], d[COLS / 2], c0 = pair(0.f), c1 = pair(0.f);
                in.get(0, v, at);
                joined<VEC, COLS, THREADS>(a, keep, branch, h, r, weight, v);
                in.get(3, d, at);
#pragma unroll
                for (int q = 0; q < COLS / 4; ++q) {
                    float2 w[2];
                    w_pre.get(q, w);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int p = 2 * q + e;
                        v[p] = __fmul2_rn(__fadd2_rn(v[p], pair(-st.z)), pair(st.w));
                        sum_pre[p] = __ffma2_rn(d[p], v[p], sum_pre[p]);
                        d[p] = __fmul2_rn(d[p], w[e]);
                        c1 = __ffma2_rn(d[p], v[p], c1);
                    }
                }
                if (a.layer) {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) c0 = __fadd2_rn(c0, d[p]);
                }
                const float2 k01 = row_sums(a, ex, c0, c1);
                const float2 k0 = pair(-st.w * k01.x * inv_n), k1 = pair(-st.w * k01.y * inv_n);
                if (stream) {
                    in.get(2, g, at);
                } else {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) g[p] = pair(0.f);
                }
                if (a.layer) {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) g[p] = __fadd2_rn(g[p], k0);
                }
#pragma unroll
                for (int p = 0; p < COLS / 2; ++p) g[p] = __ffma2_rn(v[p], k1, __ffma2_rn(d[p], pair(st.w), g[p]));
            } else if (stream) {
                in.get(2, g, at);
            } else {
#pragma unroll
                for (int p = 0; p < COLS / 2; ++p) g[p] = pair(0.f);
            }
            if (dx.p != nullptr) {
                float2 v[COLS / 2];
#pragma unroll
                for (int p = 0; p < COLS / 2; ++p) v[p] = __fmul2_rn(g[p], pair(a.residual));
                in.put(0, dx.row(i), at, v);
            }
            if (!branch) continue;
            float2 c0 = pair(0.f), c1 = pair(0.f);
#pragma unroll
            for (int q = 0; q < COLS / 4; ++q) {
                float2 w[2];
                weight.get(q, w);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int p = 2 * q + e;
                    if (a.drop) g[p] = Mask<VEC, COLS, THREADS>::apply(keep, r[p], g[p]);
                    sum_branch[p] = __ffma2_rn(g[p], h[p], sum_branch[p]);
                    g[p] = __fmul2_rn(g[p], w[e]);
                    c1 = __ffma2_rn(g[p], h[p], c1);
                }
            }
            if (dy.p == nullptr) continue;
            if (post) {
                if (a.layer) {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) c0 = __fadd2_rn(c0, g[p]);
                }
                const float2 k01 = row_sums(a, ex, c0, c1);
                const float2 k0 = pair(-k01.x * inv_n), k1 = pair(-k01.y * inv_n);
                if (a.layer) {
#pragma unroll
                    for (int p = 0; p < COLS / 2; ++p) g[p] = __fadd2_rn(g[p], k0);
                }
#pragma unroll
                for (int p = 0; p < COLS / 2; ++p) g[p] = __fmul2_rn(__ffma2_rn(h[p], k1, g[p]), pair(st.y));
            }
            in.put(1, dy.row(i), at, g);
        }
        if (out.gate != nullptr || out.post != nullptr) {
#pragma unroll
            for (int q = 0; q < COLS / 4; ++q) {
                float total[4];
                float2 before[2];
                if (post) sum_post.get(q, before);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = at.of(4 * q + e), p = 2 * q + e / 2;
                    const float sum = a.scale * (e & 1 ? sum_branch[p].y : sum_branch[p].x);
                    total[e] = e & 1 ? before[e / 2].y : before[e / 2].x;
                    if (c >= a.n) continue;
                    if (out.gate != nullptr) out.gate[k * a.n + c] = post ? a.w_post[c] * sum : sum;
                    total[e] = a.gate != nullptr ? fmaf(a.gate[group * a.n + c], sum, total[e]) : total[e] + sum;
                }
                if (post) sum_post.room[q * team_threads<THREADS>() + threadIdx.x] = make_float4(total[0], total[1], total[2], total[3]);
            }
#pragma unroll
            for (int p = 0; p < COLS / 2; ++p) sum_branch[p] = pair(0.f);
        }
    }
#pragma unroll
    for (int q = 0; q < COLS / 4; ++q) {
        float2 total[2];
        if (out.post != nullptr) sum_post.get(q, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = at.of(4 * q + e), p = 2 * q + e / 2;
            if (c >= a.n) continue;
            if (out.post != nullptr) out.post[static_cast<int64_t>(team) * a.n + c] = e & 1 ? total[e / 2].y : total[e / 2].x;
            if (out.pre != nullptr) out.pre[static_cast<int64_t>(team) * a.n + c] = e & 1 ? sum_pre[p].y : sum_pre[p].x;
        }
    }
}

// to[g][c] = sum of from[g * per + k][c] over k < per: 32 interleaved sums a column, then their sum, in an order fixed by `per`.
struct Fold {
    const float* from;
    float* to;
    int64_t rows, per;
};
struct Folds {
    Fold f[3];
};
constexpr int kFoldRows = 32;
__global__ void __launch_bounds__(32 * kFoldRows) fold_kernel(const __grid_constant__ Folds folds, int n) {
    __shared__ float part[kFoldRows][33];
    const Fold f = folds.f[blockIdx.z];
    const int lane = threadIdx.x & 31, which = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    for (int64_t g = blockIdx.y; g < f.rows; g += gridDim.y) {
        float sum = 0.f;
        if (c < n) {
            const float* from = f.from + g * f.per * n + c;
#pragma unroll 8
            for (int64_t k = which; k < f.per; k += kFoldRows) sum += from[k * n];
        }
        part[which][lane] = sum;
        __syncthreads();
        sum = warp_sum(part[lane][which]);   // of column `which`
        const int column = blockIdx.x * 32 + which;
        if (lane == 0 && column < n) f.to[g * n + column] = sum;
        __syncthreads();
    }
}

// ---- host side ----------------------------------------------------------------------------------

// Threads for so many columns, a multiple of 32.  A power of two, whose distances are constants for 256 and 512 threads, but what the row
// needs where an SM, which holds `held` threads, then has another CTA (8192 x 2560 bfloat16, 160 threads for 256: 56 us forward and 89 backward,
// 68 and 121; x 3584, two CTAs either way: 76 and 119 against 68 and 109) and, if `wide`, beyond 256: backward 4096 x 5120 binary32 242 -> 218 us
// (forward 89 -> 94).
int threads_of(int columns, int each, int held, bool wide) {
    int threads = 32;
    while (threads * each < columns) threads *= 2;
    const int needed = (columns + 32 * each - 1) / (32 * each) * 32;
    return (needed > 256 ? wide : held / needed > held / threads) ? needed : threads;
}

// columns: how many a thread of the backward kernel has (16: 16-bit rows in words)
Parts parts_of(int64_t m, int64_t n, int64_t groups, int columns) {
    Parts p;
    p.groups = groups > 0 ? groups : 1;
    p.rows = m / p.groups;
    // As many CTAs as an SM holds (512 threads by their registers, and a little less by the shared memory of small ones), but none of fewer
    // than 16 rows: their sums' traffic would show (few rows take the time of one after the other: two then).  Wider rows take a cluster.
    int64_t per_sm = columns * kTeam / (n > 512 ? n : columns == 16 ? 683 : 512);
    if (n <= 512 * columns) {
        const int fit = kTeam / threads_of(static_cast<int>(n), columns, kTeam, true);
        if (per_sm > fit) per_sm = fit;
    }
    const int64_t least = m * n >= (int64_t(1) << 23) ? 16 : 2;
    if (per_sm > 1 && m < per_sm * kNumSMs * least) per_sm = m / (kNumSMs * least);
    p.teams = per_sm > 1 ? per_sm * kNumSMs : n <= 16 * kTeam ? kNumSMs : kNumSMs / 2;
    // one group: a part for each CTA; more: four rounds of parts, so that the last round is short
    int64_t per = p.groups == 1 ? p.teams : (4 * p.teams + p.groups - 1) / p.groups;
    p.per_group = per < p.rows ? per : (p.rows > 0 ? p.rows : 1);
    p.count = p.groups * p.per_group;
    if (p.teams > p.count) p.teams = p.count;
    return p;
}
size_t gate_sums(const Parts& p, int64_t n) { return p.per_group > 1 ? static_cast<size_t>(p.count) * n : 0; }
size_t workspace_of(int64_t m, int64_t n, int64_t groups) {
    if (n == 0) return 256;   // no columns to cut: nothing is kept, and 0 would be a refusal
    size_t most = 0;
    for (int columns : {8, 16}) {
        const Parts p = parts_of(m, n, groups, columns);
        const size_t bytes = (gate_sums(p, n) + 2 * static_cast<size_t>(p.teams) * n) * sizeof(float);
        if (bytes > most) most = bytes;
    }
    return round_up(most, 256);
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

struct Shape {
    int threads, ranks, smem;
};
// vectors: weights and sums by column in shared memory
template <typename T, int COLS, int NT, bool SHIFT> int smem_of(int threads, int vectors, bool numbers) {
    return threads * COLS * 4 * vectors + Held<T, COLS, NT, 0, SHIFT>::bytes(threads, 2) + (numbers ? 2 * 2 * (threads * COLS + 16) : 0);
}
template <typename T, int COLS, int NT, bool SHIFT> Shape shape_of(int n, int vectors, bool drop) {
    Shape s{32, 1, 0};
    const int held = NT == 2 ? held_threads<T, COLS, SHIFT>() : kTeam;            // by an SM
    const int most = sizeof(T) == 4 && COLS == 16 && SHIFT ? kTeam / 2 : kTeam;   // what shared memory holds of the widest
    while (most * COLS * s.ranks < n) s.ranks *= 2;
    const int part = (n + s.ranks - 1) / s.ranks;   // columns of a CTA
    s.threads = threads_of(part, COLS, held, NT == 4);
    if (NT == 2 && two_wide<T, COLS, SHIFT>() && s.threads == 512 && part <= 384 * COLS) s.threads = part <= 320 * COLS ? 320 : 384;
    s.smem = smem_of<T, COLS, NT, SHIFT>(s.threads, vectors, drop && !(sizeof(T) == 2 && n % 8 == 0));
    return s;
}
// teams: clusters of s.ranks CTAs
template <typename K, typename... A> int start(K kern, const Shape& s, int64_t teams, int most_smem, cudaStream_t stream, A... args) {
    cudaError_t e = cudaSuccess;
    // up to 48 KB need no leave; beyond, the limit belongs to the kernel and not to the call: the same one each time
    if (s.smem > 48 * 1024 - 2048) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem);
    if (e != cudaSuccess) return cuda_failed(e);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(teams * s.ranks));
    cfg.blockDim = dim3(static_cast<unsigned>(s.threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(s.smem);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(s.ranks), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = s.ranks > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kern, args...);
    if (e != cudaSuccess) return cuda_failed(e);
    note_launch();
    return check_launch();
}
template <typename T, int COLS, int NT, bool SHIFT> int most_smem(int vectors) {
    const int all = smem_of<T, COLS, NT, SHIFT>(kTeam, vectors, true), limit = 227 * 1024 - 1024;
    return all < limit ? all : limit;
}
template <typename T> JoinRows<const T> input(const void* p, int64_t ld, const JoinArgs& a) {
    const T* t = static_cast<const T*>(p);
    return {t, ld, t == nullptr ? t : t + (a.m - 1) * ld + a.n};
}
template <typename T> JoinRows<T> output(void* p, int64_t ld) { return {static_cast<T*>(p), ld, nullptr}; }

template <typename T, int COLS, bool SHIFT> int forward_as(const JoinArgs& a, const JoinTensors& t, cudaStream_t s) {
    const Shape shape = shape_of<T, COLS, 2, SHIFT>(a.n, 2, a.drop != 0);
    // as many as an SM holds, by their registers and by their shared memory
    int per_sm = held_threads<T, COLS, SHIFT>() / shape.threads;
    if (two_wide<T, COLS, SHIFT>() && shape.threads > 256 && shape.threads <= 384) per_sm = 2;
    if (per_sm * (shape.smem + 2048) > 220 * 1024) per_sm = 220 * 1024 / (shape.smem + 2048);
    const int64_t most = static_cast<int64_t>(per_sm > 1 ? per_sm : 1) * kNumSMs / shape.ranks;
    auto kern = join_kernel<T, COLS, 0, SHIFT>;
    if (shape.threads == 256) kern = join_kernel<T, COLS, 256, SHIFT>;
    if constexpr (two_wide<T, COLS, SHIFT>()) {
        if (shape.threads == 320) kern = join_kernel<T, COLS, 320, SHIFT>;
        if (shape.threads == 384) kern = join_kernel<T, COLS, 384, SHIFT>;
    }
    if constexpr (COLS == 16 && !(sizeof(T) == 4 && SHIFT))   // eight columns a thread end at 256 threads, and what shared memory holds of these
        if (shape.threads == 512) kern = join_kernel<T, COLS, 512, SHIFT>;
    return start(kern, shape, a.m < most ? a.m : most, most_smem<T, COLS, 2, SHIFT>(2), s, a, shape.ranks, input<T>(t.a, t.ld_a, a), input<T>(t.b, t.ld_b, a), output<T>(t.e, t.ld_e),
                 output<T>(t.f, t.ld_f));
}
template <typename T, int COLS, bool SHIFT> int backward_as(const JoinArgs& a, const JoinTensors& t, const Parts& p, const Sums& sums, cudaStream_t s) {
    const Shape shape = shape_of<T, COLS, 4, SHIFT>(a.n, 3, a.drop != 0);
    auto kern = join_backward_kernel<T, COLS, 0, SHIFT>;
    if (shape.threads == 512) kern = join_backward_kernel<T, COLS, 512, SHIFT>;
    if constexpr (sizeof(T) == 4 || COLS == 16 || SHIFT)   // 16-bit words by eight columns: up to 256 columns, or from 4096 on
        if (shape.threads == 256) kern = join_backward_kernel<T, COLS, 256, SHIFT>;
    return start(kern, shape, p.teams, most_smem<T, COLS, 4, SHIFT>(3), s, a, p, sums, shape.ranks, input<T>(t.a, t.ld_a, a), input<T>(t.b, t.ld_b, a), input<T>(t.c, t.ld_c, a),
                 input<T>(t.d, t.ld_d, a), output<T>(t.e, t.ld_e), output<T>(t.f, t.ld_f));
}

template <typename T> int forward(const JoinArgs& a, const JoinTensors& t, cudaStream_t s) {
    if (!in_words(t, a.m, sizeof(T))) return a.n <= 8 * 256 ? forward_as<T, 8, true>(a, t, s) : forward_as<T, 16, true>(a, t, s);
    return a.n <= 8 * 256 ? forward_as<T, 8, false>(a, t, s) : forward_as<T, 16, false>(a, t, s);
}
// Columns of a thread of the backward kernel.  Sixteen keep two CTAs on an SM at 4096 columns; with random numbers of odd rows beside them
// their shared memory ends at 4096.
int backward_columns(int64_t n, int bytes, bool words, bool drop) { return bytes == 2 && words && n > 256 && (n <= 8 * kTeam || n % 8 == 0 || !drop) ? 16 : 8; }
template <typename T> int backward(const JoinArgs& a, const JoinTensors& t, const Parts& p, const Sums& sums, bool words, int columns, cudaStream_t s) {
    if (!words) return backward_as<T, 8, true>(a, t, p, sums, s);
    if constexpr (sizeof(T) == 2)
        if (columns == 16) return backward_as<T, 16, false>(a, t, p, sums, s);
    return backward_as<T, 8, false>(a, t, p, sums, s);
}

// A row tensor: rows that do not overlap, elements on their type's boundary.
bool good(const void* p, int64_t ld, int64_t m, int64_t n, int bytes) {
    return p == nullptr || ((m <= 1 || ld >= n) && reinterpret_cast<uintptr_t>(p) % bytes == 0);
}
bool far_apart(const JoinTensors& t) {
    const int64_t lim = int64_t(1) << 31;
    return t.ld_a >= lim || t.ld_b >= lim || t.ld_c >= lim || t.ld_d >= lim || t.ld_e >= lim || t.ld_f >= lim;
}
bool on_float(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// What both calls check of sizes and form; `least` gets the dropout threshold.
int check(int dtype, int64_t m, int64_t n, int norm, float eps, const void* y, const float* w_post, const float* gate, int64_t groups, float residual,
          float branch, double rate, const uint64_t* rng, const float* w_pre, const void* stats, uint32_t* least) {
    if (element_bytes(dtype) == 0 || m < 0 || n < 0 || (norm != BZ_NORM_RMS && norm != BZ_NORM_LAYER) || groups < 0 || !isfinite(residual) || !isfinite(branch) ||
        !(eps >= 0.f) || isinf(eps) || !drop_threshold(rate, least) || !aligned16(stats) || !aligned8(rng) || !on_float(w_post) || !on_float(gate) || !on_float(w_pre))
        return BZ_ERR_INVALID_ARG;
    if (m >= (int64_t(1) << 31) || n > BZ_MAX_WIDTH || groups >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    if ((gate != nullptr) != (groups > 0) || (groups > 0 && m % groups != 0)) return BZ_ERR_INVALID_ARG;
    if (m > 0 && n > 0 && y == nullptr && (w_post != nullptr || gate != nullptr || *least != 0)) return BZ_ERR_INVALID_ARG;
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
    if ((dw_post != nullptr && w_post == nullptr) || (dgate != nullptr && gate == nullptr) || (dw_pre != nullptr && w_pre == nullptr) || !on_float(dw_post) || !on_float(dgate) ||
        !on_float(dw_pre))
        return BZ_ERR_INVALID_ARG;
    if (n == 0) return BZ_OK;
    if (dx == nullptr && dy == nullptr && !sums) return m == 0 ? BZ_OK : BZ_ERR_INVALID_ARG;
    if (m == 0 && !sums) return BZ_OK;
    if (m > 0 && ((pre && x == nullptr) || (dz != nullptr && w_pre == nullptr) || ((pre || w_post != nullptr) && stats == nullptr) || (dy != nullptr && y == nullptr) ||
                  !good(x, ld_x, m, n, bytes) || !good(y, ld_y, m, n, bytes) || !good(ds, ld_ds, m, n, bytes) || !good(dz, ld_dz, m, n, bytes) ||
                  !good(dx, ld_dx, m, n, bytes) || !good(dy, ld_dy, m, n, bytes)))
        return BZ_ERR_INVALID_ARG;
    if (m > 1 && far_apart(t)) return BZ_ERR_UNSUPPORTED;
    const bool words = in_words(t, m, bytes);
    const int columns = backward_columns(n, bytes, words, least != 0);
    const Parts p = parts_of(m, n, groups, columns);
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
    if (dw_post != nullptr) partial.post = fold(dw_post, 1, p.teams);
    if (dw_pre != nullptr) partial.pre = fold(dw_pre, 1, p.teams);
    if (dgate != nullptr) partial.gate = p.per_group > 1 ? fold(dgate, p.groups, p.per_group) : dgate;
    const JoinArgs a = join_args(m, n, norm, 0.f, w_post, gate, groups, residual_scale, branch_scale, least, rng, w_pre, stats);
    cudaStream_t stream_ = static_cast<cudaStream_t>(stream);
    const int done = dtype == BZ_F32 ? backward<float>(a, t, p, partial, words, columns, stream_) : dtype == BZ_F16 ? backward<__half>(a, t, p, partial, words, columns, stream_)
                                                                                              : backward<__nv_bfloat16>(a, t, p, partial, words, columns, stream_);
    if (done != BZ_OK || count == 0) return done;
    int64_t rows = 1;
    for (int k = 0; k < count; ++k) rows = rows > folds.f[k].rows ? rows : folds.f[k].rows;
    fold_kernel<<<dim3(static_cast<unsigned>((n + 31) / 32), static_cast<unsigned>(rows < 1024 ? rows : 1024), count), 32 * kFoldRows, 0, stream_>>>(folds, static_cast<int>(n));
    note_launch();
    return check_launch();
}
