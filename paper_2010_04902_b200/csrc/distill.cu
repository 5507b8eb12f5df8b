// Distillation loss against a teacher's top logits, and its gradient.
//
// q = softmax(s/T) runs over the whole vocabulary, the teacher's p over t entries.  Loss and gradient need the same
// maximum and sum of a row, so the fused call reads the row once, keeps its exponentials in registers (32 elements a
// thread) and writes the gradient from there: two transfers a logit (4096 x 32128 bfloat16 in 130 us, 62 % of the copy's rate;
// the loss alone of 2048 x 100003 binary16 in 87 us, 72 %: the exponentials' unit is at 51 and 58 %).  A row that one CTA cannot hold
// is split over a cluster of up to eight; the CTAs exchange their (maximum, sum) pair through distributed shared
// memory, one barrier a row.  Beyond that (more than 131 072 logits) the cluster reads the row twice.
// The t entries: one warp forms p while the row's loads are in flight; after the dense part dlogits = dloss*T*q is
// stored, the threads overwrite the named places, adding up entries that name the same one in their order.  No atomics:
// the same inputs give the same bits.
#include <cooperative_groups.h>

#include "umma.cuh"
#include "worker_common.cuh"

namespace bz {

namespace {

namespace cg = cooperative_groups;

__device__ unsigned int g_timeouts = 0;

constexpr int kHeld = 32;        // logits a thread keeps in registers
constexpr int kMaxThreads = 512, kBestThreads = 256;
constexpr int kMaxCluster = 8;   // portable cluster size

struct DistillArgs {
    int64_t ld, v, ld_d;
    const float* teacher;
    const int32_t* index;
    Extent extent;               // of the logits
    int t;
    float temperature, c;        // c = log2(e) / T
    const float* dloss;
    float* loss;
    MaxSum* stats;               // largest logit and the sum of e^((s - that)/T)
};

struct Entries {  // dynamic shared memory: the teacher's entries of one row
    float *p, *log_p, *s;  // probability, its logarithm, student logit
    int* at;               // -1: not kept
};
__device__ __forceinline__ Entries entries(float* smem, int t) {
    return {smem, smem + t, smem + 2 * t, reinterpret_cast<int*>(smem + 3 * t)};
}

// One warp: p of the row's kept entries; the student's logit at each that lies in [lo, hi).  Returns whether any is kept.
template <typename T>
__device__ __forceinline__ bool teacher_row(const DistillArgs& a, const T* row, int64_t i, const Entries& e, int64_t lo, int64_t hi) {
    constexpr int B = 4;   // entries a lane has on their way at a time
    const int lane = threadIdx.x & 31;
    float top = -INFINITY;
    for (int k0 = lane; k0 < a.t; k0 += 32 * B) {
        int at[B];
        float z[B], x[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int k = k0 + 32 * b;
            at[b] = k < a.t ? __ldg(a.index + i * a.t + k) : -1;
            z[b] = k < a.t ? __ldg(a.teacher + i * a.t + k) : -INFINITY;
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (at[b] < 0 || at[b] >= a.v || z[b] == -INFINITY) at[b] = -1;
            x[b] = at[b] >= 0 && at[b] >= lo && at[b] < hi ? to_f32(row[at[b]]) : 0.f;
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int k = k0 + 32 * b;
            if (k < a.t) e.at[k] = at[b], e.log_p[k] = z[b], e.s[k] = x[b];
            if (at[b] >= 0) top = fmaxf(top, z[b]);
        }
    }
    const Reference r(warp_max(top), a.c);
    float sum = 0.f;
    bool any = false;
    for (int k = lane; k < a.t; k += 32)
        if (e.at[k] >= 0) {
            any = true;
            sum += exp2_fast(r.of(e.log_p[k], a.c));
        }
    sum = warp_sum(sum);
    any = __any_sync(~0u, any);
    const float log_sum = logf(sum), norm = 1.f / sum;
    for (int k = lane; k < a.t; k += 32) {
        const float y = r.of(e.log_p[k], a.c);
        e.p[k] = e.at[k] >= 0 ? exp2_fast(y) * norm : 0.f;
        e.log_p[k] = y * kLn2 - log_sum;
    }
    __syncwarp();
    return any;
}

// One warp: the loss of the row from its maximum and sum.
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Entries& e, const MaxSum& all) {
    const Reference r(all.m, a.c);
    const float log_sum = logf(all.s);
    float sum = 0.f;
    for (int k = threadIdx.x & 31; k < a.t; k += 32) {
        const float p = e.p[k];
        if (p != 0.f) {  // an entry without weight adds nothing, whatever its q
            const float log_q = e.s[k] == -INFINITY ? -INFINITY : r.of(e.s[k], a.c) * kLn2 - log_sum;
            sum += p * (e.log_p[k] - log_q);
        }
    }
    return warp_sum(sum) * (a.temperature * a.temperature);
}

// The gradient at the place that entry k names.
__device__ __forceinline__ float entry_value(const DistillArgs& a, const Entries& e, const Reference& r, const MaxSum& all, float g, int k) {
    const int at = e.at[k];
    float p = 0.f;
#pragma unroll 8
    for (int o = 0; o < a.t; ++o) p += e.at[o] == at ? e.p[o] : 0.f;
    const float q = e.s[k] == -INFINITY ? 0.f : exp2_fast(r.of(e.s[k], a.c)) / all.s;
    return g * (q - p);
}
// All threads: the places of [lo, hi) that the teacher names.
template <typename T>
__device__ __forceinline__ void write_entries(const DistillArgs& a, const Entries& e, const MaxSum& all, float g, int64_t lo, int64_t hi, T* out) {
    const Reference r(all.m, a.c);
    for (int k = threadIdx.x; k < a.t; k += blockDim.x)
        if (e.at[k] >= 0 && e.at[k] >= lo && e.at[k] < hi)   // lo may lie before the row (its first slot's lead)
            out[e.at[k]] = from_f32<T>(entry_value(a, e, r, all, g, k));
}

// Joins one part per warp (each lane passes its warp's) over the CTA.
__device__ __forceinline__ MaxSum cta_join(const MaxSum& v, float c, MaxSum* part) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_join(lane < (blockDim.x >> 5) ? part[lane] : MaxSum{-INFINITY, 0.f}, c);
}

// -inf in the place of what is not the row's.
template <int VEC> __device__ __forceinline__ void outside(int64_t j0, int64_t n, float (&x)[VEC]) {
    if (j0 < 0 || j0 + VEC > n) {
        rare();
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            if (j0 + k < 0 || j0 + k >= n) x[k] = -INFINITY;
    }
}

// Whether a slot of the row can be read whole.
template <int VEC> __device__ __forceinline__ bool fetchable(int64_t j0, int64_t n, bool safe) {
    return j0 < n && (safe || (j0 >= 0 && j0 + VEC <= n));
}

// One cluster a row.  HELD: the row's exponentials stay in registers; otherwise the row is read twice.
template <typename T, int VEC, bool HELD>
__global__ void __launch_bounds__(kMaxThreads) distill_kernel(const __grid_constant__ DistillArgs a, const T* logits, T* dlogits) {
    extern __shared__ float smem[];
    __shared__ MaxSum part[32], peers[kMaxCluster];
    __shared__ int s_any;
    constexpr int kSlots = kHeld / VEC;
    const Entries e = entries(smem, a.t);
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = cluster.block_rank(), ranks = cluster.num_blocks();
    const int64_t i = blockIdx.x / ranks;
    const T* row = logits + i * a.ld;
    const int lead = row_lead<T, VEC>(row), n = static_cast<int>(a.v);
    const int per_cta = blockDim.x * kHeld;          // HELD: elements of one CTA's share
    const int64_t base = (HELD ? static_cast<int64_t>(rank) * per_cta : static_cast<int64_t>(rank) * blockDim.x * VEC) - lead;
    const int step = blockDim.x * VEC * (HELD ? 1 : ranks);
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // every CTA of the cluster has started
    float x[HELD ? kSlots : 1][VEC];
    Raw<T, VEC> raw[HELD ? kSlots : 1];
    const bool safe = a.extent.around(row, a.v);
    MaxSum mine{-INFINITY, 0.f};
    const int at0 = static_cast<int>(base) + threadIdx.x * VEC;   // HELD: at most 8 * 512 * 32
    if constexpr (HELD) {
#pragma unroll
        for (int c = 0; c < kSlots; ++c) raw[c].fetch(row + at0 + c * step, fetchable<VEC>(at0 + c * step, n, safe));
    }
    if (threadIdx.x < 32) {
        const bool any = teacher_row(a, row, i, e, 0, a.v);
        if (threadIdx.x == 0) s_any = any;
    }
    if constexpr (HELD) {
#pragma unroll
        for (int c = 0; c < kSlots; ++c) {
            raw[c].get(x[c]);
            if (at0 + c * step < n && !fetchable<VEC>(at0 + c * step, n, safe)) read_apart<T, VEC>(row, at0 + c * step, n, x[c]);
            outside<VEC>(at0 + c * step, n, x[c]);
            mine.m = largest(mine.m, x[c]);
        }
        mine.m = warp_max(mine.m);
        const Reference own(mine.m, a.c);
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kSlots; ++c) {
            exponentials(x[c], own, a.c);
            add_up(sum, x[c]);
        }
        mine.s = warp_sum(sum.x + sum.y);
    } else {
        for (int64_t j0 = base + static_cast<int64_t>(threadIdx.x) * VEC; j0 < a.v; j0 += step) {
            load_slot<T, VEC>(row, j0, a.v, -INFINITY, x[0]);
            float m = mine.m;
#pragma unroll
            for (int k = 0; k < VEC; ++k) m = fmaxf(m, x[0][k]);
            const Reference r(m, a.c);
            if (mine.s != 0.f) mine.s *= exp2_fast(r.of_part(mine.m, a.c));
            mine.m = m;
            exponentials(x[0], r, a.c);
#pragma unroll
            for (int k = 0; k < VEC; ++k) mine.s += x[0][k];
        }
        mine = warp_join(mine, a.c);
    }
    MaxSum all = cta_join(mine, a.c, part);
    if (ranks > 1) {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (threadIdx.x < ranks) *cluster.map_shared_rank(&peers[rank], threadIdx.x) = all;
        cluster.sync();
        const int lane = threadIdx.x & 31;
        all = warp_join(lane < ranks ? peers[lane] : MaxSum{-INFINITY, 0.f}, a.c);
    }
    const bool any = s_any != 0;
    if (rank == 0 && threadIdx.x < 32) {
        const float loss = row_loss(a, e, all);
        if (threadIdx.x == 0) {
            if (a.loss != nullptr) a.loss[i] = any ? loss : 0.f;
            if (a.stats != nullptr) a.stats[i] = {all.m, all.s / Reference(all.m, a.c).left_out(a.c)};
        }
    }
    if (dlogits == nullptr) return;
    T* out = dlogits + i * a.ld_d;
    const float g = any ? (a.dloss != nullptr ? a.dloss[i] : 1.f) * a.temperature : 0.f;
    const Reference r(all.m, a.c);
    float factor = all.s == 0.f || !any ? 0.f : g / all.s;
    if constexpr (HELD) {
        factor = mine.s == 0.f ? 0.f : factor * exp2_fast(r.of_part(mine.m, a.c));
#pragma unroll
        for (int c = 0; c < kSlots; ++c)
            if (at0 + c * step < n) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[c][k] = any ? x[c][k] * factor : 0.f;
                store_slot<T, VEC>(out, at0 + c * step, n, x[c]);
            }
        __syncthreads();
        if (any) write_entries(a, e, all, g, base, base + per_cta, out);
    } else {
        for (int64_t j0 = base + static_cast<int64_t>(threadIdx.x) * VEC; j0 < a.v; j0 += step) {
            load_slot<T, VEC>(row, j0, a.v, -INFINITY, x[0]);
            exponentials(x[0], r, a.c);
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[0][k] = any ? x[0][k] * factor : 0.f;
            store_slot<T, VEC>(out, j0, a.v, x[0]);
        }
        // the cluster's CTAs share the row slot by slot: the named places wait for all of them
        if (ranks > 1)
            cluster.sync();
        else
            __syncthreads();
        if (any && rank == 0) write_entries(a, e, all, g, 0, a.v, out);
    }
}

// ---- many long rows: two CTAs an SM, rows streamed through a ring --------------------------------
//
// A producer thread copies a row's 16-byte words in chunks of 16 KB (cp.async.bulk) into a ring of six, running ahead
// over rows; eight warps read a chunk from shared memory, four words a thread.  First pass: each thread's largest logit and
// sum.  Second pass (gradient): exponentials again from shared memory if the row is at most four chunks long, so that the
// next row still has some of the ring; longer rows come a second time, out of the L2.  Two further warps take the
// teacher's side of every other row: p while the row before is worked on, the loss once the CTA has joined its sums,
// the named places once every warp has stored its part of the gradient - the eight warps wait for neither.  Two CTAs, because
// one waits at its row's exchange while the other works (one of 16 warps: 0.16 against 0.135 ms at 4096 x 32128 bfloat16).
// Words that reach over an end of the row are read by the thread that owns them, element by element.

constexpr int kStreamCtas = 2;   // an SM
constexpr int kChunkBytes = 16384, kChunkWords = kChunkBytes / 16, kRing = 6, kHoldChunks = 4;
constexpr int kWorkers = 256, kTeachers = 2, kStreamThreads = kWorkers + 32 * kTeachers + 32;

__device__ __forceinline__ void named_sync(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kWorkers + 32) : "memory"); }
__device__ __forceinline__ void named_arrive(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kWorkers + 32) : "memory"); }

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
                 "r"(smem_u32(bar))
                 : "memory");
}

// The row's words: [begin, end) whole ones, counted from the 16-byte boundary at or before the row.
template <typename T> struct RowWords {
    int lead, begin, end, chunks;
    __device__ __forceinline__ RowWords(const T* row, int64_t v) {
        constexpr int N = Word<T>::kN;
        lead = row_lead<T, N>(row);
        begin = lead != 0;
        end = static_cast<int>((lead + v) / N);
        chunks = static_cast<int>(((lead + v + N - 1) / N + kChunkWords - 1) / kChunkWords);
    }
};

template <typename T>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtas) distill_stream_kernel(const __grid_constant__ DistillArgs a, int64_t m, const T* logits, T* dlogits, int hold) {
    constexpr int N = Word<T>::kN, kMine = kChunkWords / kWorkers;
    extern __shared__ __align__(128) unsigned char ring[];
    uint64_t* full = reinterpret_cast<uint64_t*>(ring + kRing * kChunkBytes);
    uint64_t* empty = full + kRing;
    // four sets of warp results in turn: a set is written again only after the teacher that read it has met the workers
    MaxSum(*part)[32] = reinterpret_cast<MaxSum(*)[32]>(empty + kRing);
    float* entry_room = reinterpret_cast<float*>(part + 4);
    __shared__ int dead_word, some[4];   // some: whether the row's teacher keeps an entry
    volatile int* dead = &dead_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        dead_word = 0;
        for (int s = 0; s < kRing; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], kWorkers / 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const bool grad = dlogits != nullptr;
    const int passes = grad && !hold ? 2 : 1;
    RingAt<kRing> at;      // of the loads (producer), of the chunk in hand (workers)
    int filled = 0;        // stages loaded at least once (producer)
    if (warp == kWorkers / 32 + kTeachers) {
        // ---------------------------------------------------------------- loads
        if (lane == 0) {
            bool alive = true;
            for (int64_t i = blockIdx.x; i < m && alive; i += gridDim.x) {
                const T* row = logits + i * a.ld;
                const RowWords<T> w(row, a.v);
                for (int c = 0; c < passes * w.chunks; ++c, at.next()) {
                    const int s = at.stage;
                    if (filled < kRing) {
                        ++filled;
                    } else if (!mbar_wait_live(&empty[s], at.parity ^ 1, dead)) {
                        alive = false;
                        break;
                    }
                    const int base = (c < w.chunks ? c : c - w.chunks) * kChunkWords;
                    const int from = max(base, w.begin), to = min(base + kChunkWords, w.end);
                    if (from < to) {
                        const uint32_t bytes = static_cast<uint32_t>(to - from) * 16;
                        mbar_expect_tx(&full[s], bytes);
                        bulk_load(ring + s * kChunkBytes + (from - base) * 16, row - w.lead + static_cast<int64_t>(from) * N, bytes, &full[s]);
                    } else {
                        mbar_arrive(&full[s]);
                    }
                }
            }
        }
    } else if (warp >= kWorkers / 32) {
        // ---------------------------------------------------------------- the teacher's side of every other row
        const int which = warp - kWorkers / 32;
        const Entries e = entries(entry_room + which * 4 * a.t, a.t);
        int64_t r = which;
        for (int64_t i = blockIdx.x + which * static_cast<int64_t>(gridDim.x); i < m; i += kTeachers * static_cast<int64_t>(gridDim.x), r += kTeachers) {
            const T* row = logits + i * a.ld;
            const bool any = teacher_row(a, row, i, e, 0, a.v);
            const float d = grad && a.dloss != nullptr ? a.dloss[i] : 1.f;
            if (lane == 0) some[r & 3] = any;
            named_sync(1 + which);
            const MaxSum all = warp_join(lane < kWorkers / 32 ? part[r & 3][lane] : MaxSum{-INFINITY, 0.f}, a.c);
            const float loss = row_loss(a, e, all);
            if (lane == 0) {
                if (a.loss != nullptr) a.loss[i] = any ? loss : 0.f;
                if (a.stats != nullptr) a.stats[i] = {all.m, all.s / Reference(all.m, a.c).left_out(a.c)};
            }
            if (grad) {
                // what the named places get is formed before the stores are waited for; it takes the place of log_p
                const Reference ref(all.m, a.c);
                __syncwarp();
                for (int k = lane; k < a.t; k += 32) e.log_p[k] = e.at[k] >= 0 ? entry_value(a, e, ref, all, d * a.temperature, k) : 0.f;
                named_sync(3 + which);
                T* out = dlogits + i * a.ld_d;
                for (int k = lane; k < a.t; k += 32)
                    if (e.at[k] >= 0) out[e.at[k]] = from_f32<T>(e.log_p[k]);
                __syncwarp();
            }
        }
    } else {
        // ---------------------------------------------------------------- the row
        int64_t r = 0;
        for (int64_t i = blockIdx.x; i < m; i += gridDim.x, ++r) {
            const T* row = logits + i * a.ld;
            const RowWords<T> w(row, a.v);
            const int n = static_cast<int>(a.v);
            RingAt<kRing> again = at;   // the row's first chunk
            MaxSum mine{-INFINITY, 0.f};
            // A chunk of whole words takes the straight path, four words a thread (a first word that begins before the row is
            // mended by the thread that owns it); a row's last chunk takes its steps one by one.
            auto whole = [&](int c) { return (c + 1) * kChunkWords <= w.end; };
            auto word_of = [&](int s, int in, float (&x)[N]) { Word<T>::unpack(*reinterpret_cast<const uint4*>(ring + s * kChunkBytes + in * 16), x); };
            auto partial = [&](int word, float (&x)[N]) {   // a word over an end of the row, or behind it
                rare();
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = -INFINITY;
                if (word * N - w.lead < n) load_slot<T, N>(row, word * N - w.lead, n, -INFINITY, x);
            };
            auto absorb = [&](auto& x) {
                float top = mine.m;
                for (auto& v : x) top = largest(top, v);
                const Reference own(top, a.c);
                float2 sum = make_float2(mine.s == 0.f ? 0.f : mine.s * exp2_fast(own.of_part(mine.m, a.c)), 0.f);
                for (auto& v : x) {
                    exponentials(v, own, a.c);
                    add_up(sum, v);
                }
                mine = {top, sum.x + sum.y};
            };
            const int tid = static_cast<int>(threadIdx.x);
            for (int c = 0; c < w.chunks; ++c, at.next()) {
                const int s = at.stage;
                mbar_wait_live(&full[s], at.parity, dead);   // expired: go on with what is there
                if (whole(c)) {
                    float x[kMine][N];
#pragma unroll
                    for (int k = 0; k < kMine; ++k) word_of(s, k * kWorkers + tid, x[k]);
                    if (c == 0 && tid == 0 && w.begin) partial(0, x[0]);
                    absorb(x);
                } else {
#pragma unroll 1
                    for (int in = tid; (c * kChunkWords + in - tid) * N - w.lead < n; in += kWorkers) {
                        const int word = c * kChunkWords + in;
                        if (in >= kChunkWords) break;
                        float x[1][N];
                        if (word >= w.begin && word < w.end)
                            word_of(s, in, x[0]);
                        else
                            partial(word, x[0]);
                        absorb(x);
                    }
                }
                if (!(grad && hold)) release_stage(&empty[s]);
            }
            mine = warp_join(mine, a.c);
            if (lane == 0) part[r & 3][warp] = mine;
            named_sync(1 + static_cast<int>(r & 1));
            if (!grad) continue;
            const MaxSum all = warp_join(lane < kWorkers / 32 ? part[r & 3][lane] : MaxSum{-INFINITY, 0.f}, a.c);
            const Reference ref(all.m, a.c);
            const float g = (a.dloss != nullptr ? a.dloss[i] : 1.f) * a.temperature;
            const float factor = all.s == 0.f ? 0.f : g / all.s;
            const bool any = some[r & 3] != 0;
            T* out = dlogits + i * a.ld_d;
            if (!hold) again = at;
            for (int c = 0; c < w.chunks; ++c, again.next()) {
                const int s = again.stage;
                if (!hold) mbar_wait_live(&full[s], again.parity, dead);
                auto finish = [&](float (&x)[N]) {
                    exponentials(x, ref, a.c);
                    multiply(x, factor);
                    if (!any) {
                        rare();
#pragma unroll
                        for (int e = 0; e < N; ++e) x[e] = 0.f;
                    }
                };
                if (whole(c)) {
                    float x[kMine][N];
#pragma unroll
                    for (int k = 0; k < kMine; ++k) word_of(s, k * kWorkers + tid, x[k]);
                    if (c == 0 && tid == 0 && w.begin) partial(0, x[0]);
                    T* to = out + (static_cast<int64_t>(c) * kChunkWords + tid) * N - w.lead;
#pragma unroll
                    for (int k = 0; k < kMine; ++k) {
                        finish(x[k]);
                        if (k == 0 && c == 0 && tid == 0 && w.begin)
                            store_slot<T, N>(out, -w.lead, n, x[0]);
                        else
                            *reinterpret_cast<uint4*>(to + k * kWorkers * N) = Word<T>::pack(x[k]);
                    }
                } else {
#pragma unroll 1
                    for (int in = tid; (c * kChunkWords + in - tid) * N - w.lead < n; in += kWorkers) {
                        const int word = c * kChunkWords + in;
                        if (in >= kChunkWords) break;
                        float x[N];
                        if (word >= w.begin && word < w.end)
                            word_of(s, in, x);
                        else
                            partial(word, x);
                        finish(x);
                        if (word * N - w.lead < n) store_slot<T, N>(out, word * N - w.lead, n, x);
                    }
                }
                release_stage(&empty[s]);
            }
            if (!hold) at = again;
            named_arrive(3 + static_cast<int>(r & 1));
        }
    }
    __syncthreads();
    if (*dead && warp == kWorkers / 32 + kTeachers && lane == 0) {
        atomicAdd(&g_timeouts, 1u);
        for (int j = 0; j < filled; ++j, at.next()) mbar_wait(&full[filled < kRing ? j : at.stage], filled < kRing ? 0 : at.parity ^ 1);  // loads in flight
    }
}

// The gradient from a given maximum and sum: CTA (x, y) takes share x of row y's columns.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) distill_backward_kernel(const __grid_constant__ DistillArgs a, const T* logits, T* dlogits, int shares) {
    extern __shared__ float smem[];
    __shared__ int s_any;
    constexpr int kSlots = kHeld / VEC;
    const Entries e = entries(smem, a.t);
    const int64_t i = blockIdx.x / shares, share = blockIdx.x % shares;
    const T* row = logits + i * a.ld;
    T* out = dlogits + i * a.ld_d;
    const int64_t base = share * (256 * kHeld) - row_lead<T, VEC>(row);
    Raw<T, VEC> raw[kSlots];
    const bool safe = a.extent.around(row, a.v);
#pragma unroll
    for (int c = 0; c < kSlots; ++c) {
        const int64_t j0 = base + (c * 256 + static_cast<int64_t>(threadIdx.x)) * VEC;
        raw[c].fetch(row + j0, fetchable<VEC>(j0, a.v, safe));
    }
    if (threadIdx.x < 32) {
        const bool any = teacher_row(a, row, i, e, base, base + 256 * kHeld);
        if (threadIdx.x == 0) s_any = any;
    }
    __syncthreads();
    const bool any = s_any != 0;
    MaxSum all = a.stats[i];
    const Reference r(all.m, a.c);
    all.s *= r.left_out(a.c);
    const float g = any ? (a.dloss != nullptr ? a.dloss[i] : 1.f) * a.temperature : 0.f;
    const float factor = all.s == 0.f ? 0.f : g / all.s;
#pragma unroll
    for (int c = 0; c < kSlots; ++c) {
        const int64_t j0 = base + (c * 256 + static_cast<int64_t>(threadIdx.x)) * VEC;
        if (j0 < a.v) {
            float x[VEC];
            raw[c].get(x);
            if (!fetchable<VEC>(j0, a.v, safe)) read_apart<T, VEC>(row, j0, a.v, x);
            exponentials(x, r, a.c);
            multiply(x, factor);
            if (!any) {
                rare();
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[k] = 0.f;
            }
            store_slot<T, VEC>(out, j0, a.v, x);
        }
    }
    __syncthreads();
    if (any) write_entries(a, e, all, g, base, base + 256 * kHeld, out);
}

// v == 0: no logits at all.
__global__ void distill_empty_kernel(int64_t m, float* loss, MaxSum* stats) {
    for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < m; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        if (loss != nullptr) loss[i] = 0.f;
        if (stats != nullptr) stats[i] = {-INFINITY, 0.f};
    }
}

// ---- host side ----------------------------------------------------------------------------------

template <typename T, int VEC> int launch(const DistillArgs& a, int64_t m, const T* logits, T* dlogits, cudaStream_t s) {
    const int64_t slots = (a.v + (VEC > 1 ? VEC - 1 : 0) + VEC - 1) / VEC, per_thread = kHeld / VEC;
    int ranks = 1;
    while (ranks < kMaxCluster && (slots + ranks * per_thread - 1) / (ranks * per_thread) > kBestThreads) ranks *= 2;
    int64_t threads = ((slots + ranks * per_thread - 1) / (ranks * per_thread) + 31) / 32 * 32;
    const bool held = threads <= kMaxThreads;
    if (!held) threads = kMaxThreads;
    if (m * ranks >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(m * ranks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(a.t) * 16;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = held ? cudaLaunchKernelEx(&cfg, distill_kernel<T, VEC, true>, a, logits, dlogits)
                               : cudaLaunchKernelEx(&cfg, distill_kernel<T, VEC, false>, a, logits, dlogits);
    if (e != cudaSuccess) return cuda_failed(e);
    note_launch();
    return check_launch();
}

// Number of rows, and bytes of a row, from which the ring pays.  Loss and gradient, bfloat16, ring against clusters:
// 148 x 8192 5.5 against 6.8 us, 148 x 32768 10.3 against 14.8, 2048 x 8192 27 against 34, 2048 x 32768 64 against 131;
// 2048 x 4000 22 against 14, 600 x 4000 10.1 against 6.9 (many short rows at a time hide the exchange better);
// 32 x 32768 8.8 against 6.9, 32 x 100000 20 against 8.4 (a cluster puts eight SMs on a row).
constexpr int64_t kStreamRows = kNumSMs, kStreamBytes = 16384;

template <typename T> int stream(const DistillArgs& a, int64_t m, const T* logits, T* dlogits, cudaStream_t s) {
    constexpr int kRingSmem = kRing * kChunkBytes + 2 * kRing * 8 + 4 * 32 * static_cast<int>(sizeof(MaxSum)), kEach = kTeachers * 16;
    const int smem = kRingSmem + kEach * a.t;
    auto kern = distill_stream_kernel<T>;
    // the limit belongs to the kernel and not to the call: the same one each time, or another thread's launch could fail
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem + kEach * BZ_MAX_TOP);
    if (e != cudaSuccess) return cuda_failed(e);
    const int hold = a.v + 2 * (Word<T>::kN - 1) <= static_cast<int64_t>(kHoldChunks) * kChunkWords * Word<T>::kN;
    kern<<<static_cast<unsigned>(m < kStreamCtas * kNumSMs ? m : kStreamCtas * kNumSMs), kStreamThreads, smem, s>>>(a, m, logits, dlogits, hold);
    note_launch();
    return check_launch();
}

template <typename T, int VEC> int launch_backward(const DistillArgs& a, int64_t m, const T* logits, T* dlogits, cudaStream_t s) {
    const int64_t shares = (a.v + (VEC > 1 ? VEC - 1 : 0) + 256 * kHeld - 1) / (256 * kHeld);
    if (m * shares >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
    distill_backward_kernel<T, VEC><<<static_cast<unsigned>(m * shares), 256, static_cast<size_t>(a.t) * 16, s>>>(
        a, logits, dlogits, static_cast<int>(shares));
    note_launch();
    return check_launch();
}

template <typename T> int dispatch(const DistillArgs& a, int64_t m, const void* logits, void* dlogits, bool backward, cudaStream_t s) {
    const T* in = static_cast<const T*>(logits);
    T* out = static_cast<T*>(dlogits);
    const uintptr_t apart = reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(dlogits);
    const bool alike = out == nullptr || ((apart & 15) == 0 && (m == 1 || ((a.ld - a.ld_d) * static_cast<int64_t>(sizeof(T))) % 16 == 0));
    if (backward)
        return alike ? launch_backward<T, Word<T>::kN>(a, m, in, out, s) : launch_backward<T, 1>(a, m, in, out, s);
    if (alike && m >= kStreamRows && a.v * static_cast<int64_t>(sizeof(T)) >= kStreamBytes && a.v < (int64_t(1) << 30)) return stream<T>(a, m, in, out, s);
    return alike ? launch<T, Word<T>::kN>(a, m, in, out, s) : launch<T, 1>(a, m, in, out, s);
}

int check(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const float* teacher, const int32_t* index, int t,
          float temperature, const void* dlogits, int64_t ld_d) {
    const int bytes = element_bytes(dtype);
    if (bytes == 0 || m < 0 || v < 0 || t < 1 || !(temperature > 0.f) || isinf(temperature) || isinf(kLog2e / temperature)) return BZ_ERR_INVALID_ARG;
    if (v >= (int64_t(1) << 31) || t > BZ_MAX_TOP) return BZ_ERR_UNSUPPORTED;
    if (m == 0) return BZ_OK;
    if (teacher == nullptr || index == nullptr) return BZ_ERR_INVALID_ARG;
    if (v == 0) return BZ_OK;
    if (logits == nullptr || (m > 1 && ld < v) || reinterpret_cast<uintptr_t>(logits) % bytes) return BZ_ERR_INVALID_ARG;
    if (dlogits != nullptr && ((m > 1 && ld_d < v) || reinterpret_cast<uintptr_t>(dlogits) % bytes)) return BZ_ERR_INVALID_ARG;
    return BZ_OK;
}

Extent extent_of(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v) {
    const char* p = static_cast<const char*>(logits);
    return {p, p + ((m - 1) * ld + v) * element_bytes(dtype)};
}

}  // namespace

int distill_timeouts(unsigned int* count) {
    const cudaError_t e = cudaMemcpyFromSymbol(count, g_timeouts, sizeof(unsigned int));
    return e == cudaSuccess ? BZ_OK : cuda_failed(e);
}

}  // namespace bz

using namespace bz;

extern "C" int bz_distill(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const float* teacher, const int32_t* index,
                          int t, float temperature, const float* dloss, float* loss, float* stats, void* dlogits, int64_t ld_d, void* stream) {
    const int st = check(logits, ld, dtype, m, v, teacher, index, t, temperature, dlogits, ld_d);
    if (st != BZ_OK) return st;
    if (m == 0) return BZ_OK;
    if ((loss == nullptr && stats == nullptr && dlogits == nullptr) || !aligned8(stats)) return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (v == 0) {
        distill_empty_kernel<<<kNumSMs, 256, 0, s>>>(m, loss, reinterpret_cast<MaxSum*>(stats));
        note_launch();
        return check_launch();
    }
    const DistillArgs a{ld, v, ld_d, teacher, index, extent_of(logits, ld, dtype, m, v), t, temperature, kLog2e / temperature, dloss, loss, reinterpret_cast<MaxSum*>(stats)};
    if (dtype == BZ_F32) return dispatch<float>(a, m, logits, dlogits, false, s);
    if (dtype == BZ_F16) return dispatch<__half>(a, m, logits, dlogits, false, s);
    return dispatch<__nv_bfloat16>(a, m, logits, dlogits, false, s);
}

extern "C" int bz_distill_backward(const void* logits, int64_t ld, int dtype, int64_t m, int64_t v, const float* teacher,
                                   const int32_t* index, int t, float temperature, const float* stats, const float* dloss, void* dlogits,
                                   int64_t ld_d, void* stream) {
    const int st = check(logits, ld, dtype, m, v, teacher, index, t, temperature, dlogits, ld_d);
    if (st != BZ_OK) return st;
    if (m == 0 || v == 0) return BZ_OK;
    if (stats == nullptr || !aligned8(stats) || dlogits == nullptr) return BZ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const DistillArgs a{ld, v, ld_d, teacher, index, extent_of(logits, ld, dtype, m, v), t, temperature, kLog2e / temperature, dloss, nullptr, reinterpret_cast<MaxSum*>(const_cast<float*>(stats))};
    if (dtype == BZ_F32) return dispatch<float>(a, m, logits, dlogits, true, s);
    if (dtype == BZ_F16) return dispatch<__half>(a, m, logits, dlogits, true, s);
    return dispatch<__nv_bfloat16>(a, m, logits, dlogits, true, s);
}
