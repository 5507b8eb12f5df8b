// Gated feed-forward block and its gradient: host side, the pass between the products, and operands laid out on the way in.
#include <algorithm>
#include <atomic>

#include "glu_few.cuh"

namespace bz {

namespace {

std::atomic<int> g_glu_stall{0};   // bz_debug_stall_pipeline

constexpr int kClusters = kNumSMs / 2;
constexpr size_t kPartialBytes = static_cast<size_t>(2 * kClusters) * kRowTile * 256 * sizeof(float);  // see plan_backward()

// dgu[0] = dh * u * act'(g), dgu[1] = dh * act(g), each [m][ld], rounded to the operands' type.  14 bytes a hidden unit
// (8 of them preact): bound by memory, 135 us at 8192 x 8192 (0.94 GB: the copy's rate).  V columns a thread.
template <typename T, int ACT, int V>
__global__ void __launch_bounds__(256) glu_dgu_kernel(const float* __restrict__ preact, const T* __restrict__ dh, int64_t ld_dh, int64_t m, int64_t n,
                                                      T* __restrict__ dgu, int64_t ld) {
    const int64_t c = (blockIdx.x * int64_t(256) + threadIdx.x) * V;
    if (c >= n) return;
    for (int64_t r = blockIdx.y; r < m; r += gridDim.y) {
        float g[V], u[V], d[V], a[V], b[V];
        if constexpr (V == 2) {
            const float2 g2 = *reinterpret_cast<const float2*>(preact + r * n + c), u2 = *reinterpret_cast<const float2*>(preact + (m + r) * n + c);
            const float2 d2 = unpack2(T(), *reinterpret_cast<const uint32_t*>(dh + r * ld_dh + c));
            g[0] = g2.x, g[1] = g2.y, u[0] = u2.x, u[1] = u2.y, d[0] = d2.x, d[1] = d2.y;
        } else if constexpr (V == 8) {
            const uint4* pg = reinterpret_cast<const uint4*>(preact + r * n + c);
            const uint4* pu = reinterpret_cast<const uint4*>(preact + (m + r) * n + c);
            const uint4 g0 = pg[0], g1 = pg[1], u0 = pu[0], u1 = pu[1];   // not evict-first: a thread reads the two halves of a sector apart (199 us)
            Word<T>::unpack(*reinterpret_cast<const uint4*>(dh + r * ld_dh + c), d);
            Word<float>::unpack(g0, g), Word<float>::unpack(g1, g + 4), Word<float>::unpack(u0, u), Word<float>::unpack(u1, u + 4);
        } else {
            g[0] = preact[r * n + c], u[0] = preact[(m + r) * n + c], d[0] = to_f32(dh[r * ld_dh + c]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = d[i] * u[i] * act_slope<ACT>(g[i]), b[i] = d[i] * act<ACT>(g[i]);
        if constexpr (V == 2) {
            *reinterpret_cast<uint32_t*>(dgu + r * ld + c) = pack2(T(), a[0], a[1]);
            *reinterpret_cast<uint32_t*>(dgu + (m + r) * ld + c) = pack2(T(), b[0], b[1]);
        } else if constexpr (V == 8) {
            *reinterpret_cast<uint4*>(dgu + r * ld + c) = Word<T>::pack(a);
            *reinterpret_cast<uint4*>(dgu + (m + r) * ld + c) = Word<T>::pack(b);
        } else {
            dgu[r * ld + c] = from_f32<T>(a[0]), dgu[(m + r) * ld + c] = from_f32<T>(b[0]);
        }
    }
}

// Rows of 16-bit elements copied to rows that begin on 16-byte boundaries.
__global__ void __launch_bounds__(256) glu_lay_out_kernel(const uint16_t* __restrict__ from, int64_t ld_from, int64_t rows, int64_t n,
                                                          uint16_t* __restrict__ to, int64_t ld_to) {
    const int64_t c = blockIdx.x * int64_t(256) + threadIdx.x;
    if (c >= n) return;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) to[r * ld_to + c] = from[r * ld_from + c];
}

// A CTA a row (and 256 threads of its columns): 8192 x 8192 in 135 us, 145 with a few rows a CTA in turn.
dim3 row_grid(int64_t rows, int64_t columns_of_threads) {
    return dim3(static_cast<unsigned>((columns_of_threads + 255) / 256), static_cast<unsigned>(rows < 65535 ? rows : 65535));
}

// Whether a tensor map can describe rows like these.
bool laid_out(const void* p, int64_t ld, int64_t rows) { return aligned16(p) && (rows <= 1 || ld % 8 == 0); }

// An operand as the tensor maps describe it: itself, or a copy of it in the workspace that lay_out() makes.  The maps are made
// first, so that nothing has been launched when one is refused.
struct Operand {
    const void* p;
    int64_t ld, rows, n;
    const void* at;      // what the map describes
    int64_t ld_at;
};
Operand place_operand(const void* p, int64_t ld, int64_t rows, int64_t n, char*& room) {
    const int64_t ld_at = (n + 7) / 8 * 8;
    if (laid_out(p, ld, rows)) return {p, ld, rows, n, p, rows > 1 ? ld : ld_at};
    const Operand o{p, ld, rows, n, room, ld_at};
    room += round_up(static_cast<size_t>(rows) * ld_at * 2, 256);
    return o;
}
int lay_out(const Operand& o, cudaStream_t s) {
    if (o.at == o.p) return BZ_OK;
    glu_lay_out_kernel<<<row_grid(o.rows, o.n), 256, 0, s>>>(static_cast<const uint16_t*>(o.p), o.ld, o.rows, o.n,
                                                             static_cast<uint16_t*>(const_cast<void*>(o.at)), o.ld_at);
    note_launch();
    return check_launch();
}

// Tensor map of [z][rows][n] 16-bit elements, boxes of box_columns x box_rows, zeros outside; 128-byte swizzle for the boxes
// of 64 columns that the tensor cores read.
template <typename T>
bool make_map(CUtensorMap* map, const void* p, int64_t n, int64_t rows, int64_t ld, int box_rows, int64_t ld_z, int box_columns = 64) {
    EncodeTiledFn enc = encode_tiled();
    if (enc == nullptr) return false;
    const cuuint32_t rank = ld_z ? 3 : 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(n), static_cast<cuuint64_t>(rows), 2};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld_z) * 2};
    const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_columns), static_cast<cuuint32_t>(box_rows), 1}, elem[3] = {1, 1, 1};
    return enc(map, __is_same(T, __half) ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(p), dims,
               strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               box_columns == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Cycles of a block of the contraction and of a tile's ends, for choosing the width of the tiles: 256 columns a tile fill the
// tensor cores (512 cycles a block); narrower ones are bound by their loads out of the L2, which a block of A shares among
// fewer columns, but part the work more evenly.
double block_cycles(int bn) { return bn == 256 ? 520 : (bn == 128 ? 380 : 320); }
constexpr double kTileCycles = 1500, kSharesCycles = 4000;

int plan_forward(int64_t rows, int64_t cols, int64_t blocks) {
    int best = 256;
    double least = 0;
    for (int bn = 256; bn >= 64; bn /= 2) {
        const int64_t tiles = ceil_div(rows, kRowTile) * ceil_div(cols, bn / 2);
        const double cost = static_cast<double>(ceil_div(tiles, kClusters)) * (blocks * block_cycles(bn) + kTileCycles);
        if (bn == 256 || cost < least) least = cost, best = bn;
    }
    return best;
}

// Sets the two parts' tiles and shares for tiles of bn columns and returns the cycles that it should take.  A contraction
// longer than a cluster's part of the whole work (and than eight blocks) is cut into pieces no longer than that.  Only parts
// of fewer than kClusters tiles can be that long, so there are fewer than 2 * kClusters pieces with sums to keep.
double plan_backward(ProductParams& p, int bn) {
    int64_t work = 0;
    for (ProductPart& o : p.part) {
        if (o.out == nullptr) continue;
        o.row_tiles = (&o == &p.part[kWeight] ? 2 : 1) * ceil_div(o.rows, kRowTile);
        o.col_tiles = ceil_div(o.cols, bn);
        work += o.row_tiles * o.col_tiles * o.blocks;
    }
    const int64_t piece = std::max<int64_t>(8, ceil_div(work, kClusters));
    double cost = 0;
    for (ProductPart& o : p.part)
        if (o.out != nullptr) {
            o.splits = static_cast<int>(ceil_div(o.blocks, piece));
            if (o.splits > 1) cost = kSharesCycles;
        }
    p.weight_first = p.part[kWeight].out != nullptr &&
                     (p.part[kInput].out == nullptr || p.part[kWeight].blocks / p.part[kWeight].splits > p.part[kInput].blocks / p.part[kInput].splits);
    // pieces go round the clusters, longer ones first
    double longest = 0;
    int64_t at = 0, rounds = 0;
    for (int k = 0; k < 2; ++k) {
        const ProductPart& o = p.part[p.weight_first ? 1 - k : k];
        if (o.out == nullptr) continue;
        at += o.tiles();
        const int64_t more = ceil_div(at, kClusters) - rounds;
        longest += more * (static_cast<double>(ceil_div(o.blocks, o.splits)) * block_cycles(bn) + kTileCycles);
        rounds += more;
    }
    return cost + longest;
}

template <typename T, GluProduct P, int BN> int launch_product(const ProductMaps& maps, const ProductParams& p, cudaStream_t s) {
    auto kern = glu_product_kernel<T, P, BN>;
    constexpr int smem = ProductShape<BN>::kSmem;
    // the attribute stays with the kernel: set once per device (bits of the first 64 devices)
    static std::atomic<uint64_t> set{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_failed(e);
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (!(set.load(std::memory_order_relaxed) & bit)) {
        if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return cuda_failed(e);
        set.fetch_or(bit, std::memory_order_relaxed);
    }
    const int64_t tiles = p.part[0].tiles() + p.part[1].tiles();
    kern<<<static_cast<unsigned>(2 * (tiles < kClusters ? tiles : kClusters)), kProductThreads, smem, s>>>(maps, p);
    note_launch();
    const int st = check_launch();
    if constexpr (P == kBackward) {
        int64_t groups = 0;
        for (const ProductPart& o : p.part)
            if (o.splits > 1) groups = std::max(groups, o.row_tiles * o.col_tiles * (256 * BN / 4 / 256));
        if (st != BZ_OK || groups == 0) return st;
        glu_shares_kernel<T, BN><<<static_cast<unsigned>(std::min<int64_t>(groups, 16 * kNumSMs)), 256, 0, s>>>(p);
        note_launch();
        return check_launch();
    }
    return st;
}

int zero(void* p, int64_t ld, int64_t rows, int64_t n, int bytes, cudaStream_t s) {
    if (p == nullptr || rows == 0 || n == 0) return BZ_OK;
    const cudaError_t e = cudaMemset2DAsync(p, static_cast<size_t>(rows > 1 ? ld : n) * bytes, 0, static_cast<size_t>(n) * bytes, rows, s);
    return e == cudaSuccess ? BZ_OK : cuda_failed(e);
}

bool pair_rows(const void* p, int64_t ld, int64_t rows, int bytes) { return reinterpret_cast<uintptr_t>(p) % (2 * bytes) == 0 && (rows <= 1 || ld % 2 == 0); }
bool wide_rows(const void* p, int64_t ld, int64_t rows, int bytes) { return aligned16(p) && (rows <= 1 || ld * bytes % 16 == 0); }

// The ring pays from nine rows on, and for eight and fewer from 16 MB of weights on (out of memory, ring against registers:
// 24 rows, 512 x 2048 4.9 against 5.7 us; one row, 1024 x 2816 7.1 against 5.9; one row, 2048 x 5461 14.2 against 17.6;
// one row, 4096 x 10922 42 against 53; 32 rows of that 70 against 90: there the rows' own traffic out of the L2 is the bound).
constexpr int64_t kFewStreamRows = 9, kFewStreamBytes = int64_t(16) << 20;

template <typename T, int NT> int launch_few(const FewParams& p, bool wide, cudaStream_t s) {
    if (wide && (p.m >= kFewStreamRows || 4 * p.n * p.k >= kFewStreamBytes)) {
        constexpr int smem = few_stream_smem<NT>();
        const cudaError_t e = cudaFuncSetAttribute(glu_few_stream_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_failed(e);
        CUtensorMap gate, up;
        if (!make_map<T>(&gate, p.wg, p.k, p.n, p.n > 1 ? p.ld_w : (p.k + 7) / 8 * 8, kFewUnits, 0, kFewChunk) ||
            !make_map<T>(&up, p.wu, p.k, p.n, p.n > 1 ? p.ld_w : (p.k + 7) / 8 * 8, kFewUnits, 0, kFewChunk))
            return BZ_ERR_UNSUPPORTED;
        const int64_t groups = ceil_div(p.n, kFewUnits);
        glu_few_stream_kernel<T, NT><<<static_cast<unsigned>(std::min<int64_t>(groups, 2 * kNumSMs)), kFewStreamThreads, smem, s>>>(gate, up, p);
        note_launch();
        return check_launch();
    }
    static_assert(kFewStreamRows == 9, "wide operands of more than one group of eight rows take the ring");
    const unsigned grid = static_cast<unsigned>(ceil_div(p.n, kFewUnits));
    if (NT == 1 && wide)
        glu_few_kernel<T, NT, NT == 1><<<grid, 32 * kFewWarps, 0, s>>>(p);
    else
        glu_few_kernel<T, NT, false><<<grid, 32 * kFewWarps, 0, s>>>(p);
    note_launch();
    return check_launch();
}
template <typename T> int few(const FewParams& p, bool wide, cudaStream_t s) {
    if (p.m <= 8) return launch_few<T, 1>(p, wide, s);
    if (p.m <= 16) return launch_few<T, 2>(p, wide, s);
    if (p.m <= 24) return launch_few<T, 3>(p, wide, s);
    return launch_few<T, 4>(p, wide, s);
}

template <typename T>
int forward(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, int64_t m, int64_t n, int64_t k, int act, void* h,
            int64_t ld_h, float* preact, char* ws, cudaStream_t s) {
    int st;
    if (k == 0) {
        if (preact != nullptr && (st = zero(preact, n, 2 * m, n, 4, s)) != BZ_OK) return st;
        return zero(h, ld_h, m, n, 2, s);
    }
    if (m <= kFewMost) {
        const FewParams p{x, wg, wu, ld_x, ld_w, n, k, static_cast<int>(m), act, h, ld_h, preact};
        const bool wide = laid_out(x, ld_x, m) && laid_out(wg, ld_w, n) && laid_out(wu, ld_w, n);
        return few<T>(p, wide, s);
    }
    const Operand ox = place_operand(x, ld_x, m, k, ws), og = place_operand(wg, ld_w, n, k, ws), ou = place_operand(wu, ld_w, n, k, ws);
    ProductParams p{};
    p.stall = g_glu_stall.load(std::memory_order_relaxed);
    ProductPart& o = p.part[0];
    o.rows = m, o.cols = n, o.blocks = ceil_div(k, kBlockK);
    const int bn = plan_forward(m, n, o.blocks);
    o.row_tiles = ceil_div(m, kRowTile), o.col_tiles = ceil_div(n, bn / 2), o.splits = 1;
    o.out = h, o.ld_out = ld_h, o.wide = wide_rows(h, ld_h, m, 2), o.pairs = pair_rows(h, ld_h, m, 2);
    p.act = act, p.preact = preact, p.preact_wide = n % 4 == 0, p.preact_pairs = n % 2 == 0;
    ProductMaps maps;
    if (!make_map<T>(&maps.map[0], ox.at, k, m, ox.ld_at, 128, 0) || !make_map<T>(&maps.map[1], og.at, k, n, og.ld_at, bn / 2, 0) ||
        !make_map<T>(&maps.map[2], ou.at, k, n, ou.ld_at, bn / 2, 0))
        return BZ_ERR_UNSUPPORTED;
    if ((st = lay_out(ox, s)) != BZ_OK || (st = lay_out(og, s)) != BZ_OK || (st = lay_out(ou, s)) != BZ_OK) return st;
    if (bn == 256) return launch_product<T, kForward, 256>(maps, p, s);
    return bn == 128 ? launch_product<T, kForward, 128>(maps, p, s) : launch_product<T, kForward, 64>(maps, p, s);
}

template <typename T, int ACT>
int launch_dgu(const float* preact, const T* dh, int64_t ld_dh, int64_t m, int64_t n, T* dgu, int64_t ld, cudaStream_t s) {
    if (n % 8 == 0 && laid_out(dh, ld_dh, m))
        glu_dgu_kernel<T, ACT, 8><<<row_grid(m, n / 8), 256, 0, s>>>(preact, dh, ld_dh, m, n, dgu, ld);
    else if (n % 2 == 0 && pair_rows(dh, ld_dh, m, 2))
        glu_dgu_kernel<T, ACT, 2><<<row_grid(m, n / 2), 256, 0, s>>>(preact, dh, ld_dh, m, n, dgu, ld);
    else
        glu_dgu_kernel<T, ACT, 1><<<row_grid(m, n), 256, 0, s>>>(preact, dh, ld_dh, m, n, dgu, ld);
    note_launch();
    return check_launch();
}

template <typename T>
int backward(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, const float* preact, const void* dh, int64_t ld_dh,
             int64_t m, int64_t n, int64_t k, int act, void* dx, int64_t ld_dx, void* dwg, void* dwu, int64_t ld_dw, int grad_f32, char* ws,
             cudaStream_t s) {
    int st;
    if (m == 0 || n == 0) {
        if ((st = zero(dx, ld_dx, m, k, 2, s)) != BZ_OK || (st = zero(dwg, ld_dw, n, k, grad_f32 ? 4 : 2, s)) != BZ_OK) return st;
        return zero(dwu, ld_dw, n, k, grad_f32 ? 4 : 2, s);
    }
    const int64_t ld = (n + 7) / 8 * 8;
    T* dgu = reinterpret_cast<T*>(ws);
    float* partial = reinterpret_cast<float*>(ws + round_up(static_cast<size_t>(4) * m * ld, 256));
    char* room = reinterpret_cast<char*>(partial) + kPartialBytes;
    ProductParams p{};
    p.stall = g_glu_stall.load(std::memory_order_relaxed);
    ProductMaps maps;
    Operand og{}, ou{}, ox{};
    if (dx != nullptr) {
        og = place_operand(wg, ld_w, n, k, room), ou = place_operand(wu, ld_w, n, k, room);
        ProductPart& o = p.part[kInput];
        o.rows = m, o.cols = k, o.half_blocks = ceil_div(n, kBlockK), o.blocks = 2 * o.half_blocks;
        o.out = dx, o.ld_out = ld_dx, o.wide = wide_rows(dx, ld_dx, m, 2), o.pairs = pair_rows(dx, ld_dx, m, 2);
        if (!make_map<T>(&maps.map[0], dgu, n, m, ld, 128, m * ld) || !make_map<T>(&maps.map[1], og.at, k, n, og.ld_at, kBlockK, 0) ||
            !make_map<T>(&maps.map[2], ou.at, k, n, ou.ld_at, kBlockK, 0))
            return BZ_ERR_UNSUPPORTED;
    }
    if (dwg != nullptr) {
        ox = place_operand(x, ld_x, m, k, room);
        const int bytes = grad_f32 ? 4 : 2;
        ProductPart& o = p.part[kWeight];
        o.rows = n, o.cols = k, o.blocks = ceil_div(m, kBlockK);
        o.out = dwg, o.out2 = dwu, o.ld_out = ld_dw, o.out_f32 = grad_f32;
        o.wide = wide_rows(dwg, ld_dw, n, bytes) && aligned16(dwu);
        o.pairs = pair_rows(dwg, ld_dw, n, bytes) && pair_rows(dwu, ld_dw, n, bytes);
        if (!make_map<T>(&maps.map[3], dgu, n, m, ld, kBlockK, m * ld) || !make_map<T>(&maps.map[4], ox.at, k, m, ox.ld_at, kBlockK, 0))
            return BZ_ERR_UNSUPPORTED;
    }
    const T* d = static_cast<const T*>(dh);
    switch (act) {
        case BZ_ACT_SILU: st = launch_dgu<T, BZ_ACT_SILU>(preact, d, ld_dh, m, n, dgu, ld, s); break;
        case BZ_ACT_GELU_TANH: st = launch_dgu<T, BZ_ACT_GELU_TANH>(preact, d, ld_dh, m, n, dgu, ld, s); break;
        case BZ_ACT_GELU: st = launch_dgu<T, BZ_ACT_GELU>(preact, d, ld_dh, m, n, dgu, ld, s); break;
        default: st = launch_dgu<T, BZ_ACT_RELU>(preact, d, ld_dh, m, n, dgu, ld, s); break;
    }
    if (st != BZ_OK) return st;
    if ((st = lay_out(og, s)) != BZ_OK || (st = lay_out(ou, s)) != BZ_OK || (st = lay_out(ox, s)) != BZ_OK) return st;
    if (dx == nullptr) maps.map[0] = maps.map[1] = maps.map[2] = maps.map[3];   // prefetched, not used
    if (dwg == nullptr) maps.map[3] = maps.map[4] = maps.map[0];
    const double narrow = plan_backward(p, 128);
    const int bn = plan_backward(p, 256) <= narrow ? 256 : 128;
    if (bn == 128) plan_backward(p, 128);
    float* at = partial;
    for (ProductPart& o : p.part)
        if (o.splits > 1) o.partial = at, at += o.tiles() * kRowTile * bn;
    return bn == 256 ? launch_product<T, kBackward, 256>(maps, p, s) : launch_product<T, kBackward, 128>(maps, p, s);
}

constexpr int64_t kMostExtent = (int64_t(1) << 31) - 512;  // tile coordinates are 32-bit
// Whether a tensor map's stride cannot reach from dg to du.
bool too_far_apart(int64_t m, int64_t n) { return m > 0 && static_cast<int64_t>(round_up(n, 8)) >= (int64_t(1) << 39) / m; }

int check(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, int64_t m, int64_t n, int64_t k, int dtype, int act) {
    if (m < 0 || n < 0 || k < 0 || element_bytes(dtype) == 0 || act < BZ_ACT_SILU || act > BZ_ACT_RELU) return BZ_ERR_INVALID_ARG;
    if (m > kMostExtent || n > kMostExtent || k > kMostExtent || dtype == BZ_F32 || ld_x >= int64_t(1) << 38 || ld_w >= int64_t(1) << 38) return BZ_ERR_UNSUPPORTED;
    if ((m > 1 && ld_x < k) || (n > 1 && ld_w < k)) return BZ_ERR_INVALID_ARG;
    if ((m > 0 && k > 0 && x == nullptr) || (n > 0 && k > 0 && (wg == nullptr || wu == nullptr))) return BZ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(wg) | reinterpret_cast<uintptr_t>(wu)) & 1) return BZ_ERR_INVALID_ARG;
    return BZ_OK;
}

}  // namespace

void glu_stall(int on) { g_glu_stall.store(on == 2 ? 2 : on != 0, std::memory_order_relaxed); }

int glu_timeouts(unsigned int* count) {
    const cudaError_t e = cudaMemcpyFromSymbol(count, g_glu_timeouts, sizeof(unsigned int));
    return e == cudaSuccess ? BZ_OK : cuda_failed(e);
}

}  // namespace bz

using namespace bz;

extern "C" size_t bz_glu_workspace_bytes(int64_t m, int64_t n, int64_t k, int dtype, int backward) {
    if (m < 0 || n < 0 || k < 0 || m > kMostExtent || n > kMostExtent || k > kMostExtent || (dtype != BZ_F16 && dtype != BZ_BF16)) return 0;
    if (backward ? too_far_apart(m, n) : m <= kFewMost) return 0;
    const size_t kp = round_up(k, 8), np = round_up(n, 8);
    const size_t operands = round_up(2 * m * kp, 256) + 2 * round_up(2 * n * kp, 256);
    return backward ? round_up(4 * m * np, 256) + kPartialBytes + operands : operands;
}

extern "C" int bz_glu(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w, int64_t m, int64_t n, int64_t k,
                      int dtype, int act, void* h, int64_t ld_h, float* preact, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = check(x, ld_x, w_gate, w_up, ld_w, m, n, k, dtype, act);
    if (st != BZ_OK) return st;
    if (m == 0 || n == 0) return BZ_OK;
    if (h == nullptr || (m > 1 && ld_h < n) || (reinterpret_cast<uintptr_t>(h) & 1) || !aligned16(preact)) return BZ_ERR_INVALID_ARG;
    if (m > kFewMost && !(laid_out(x, ld_x, m) && laid_out(w_gate, ld_w, n) && laid_out(w_up, ld_w, n)) && k > 0 &&
        (workspace == nullptr || !aligned256(workspace) || workspace_bytes < bz_glu_workspace_bytes(m, n, k, dtype, 0)))
        return BZ_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == BZ_F16 ? forward<__half>(x, ld_x, w_gate, w_up, ld_w, m, n, k, act, h, ld_h, preact, ws, s)
                           : forward<__nv_bfloat16>(x, ld_x, w_gate, w_up, ld_w, m, n, k, act, h, ld_h, preact, ws, s);
}

extern "C" int bz_glu_backward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w, const float* preact,
                               const void* dh, int64_t ld_dh, int64_t m, int64_t n, int64_t k, int dtype, int act, void* dx, int64_t ld_dx,
                               void* dw_gate, void* dw_up, int64_t ld_dw, int grad_dtype, void* workspace, size_t workspace_bytes,
                               void* stream) {
    const int st = check(x, ld_x, w_gate, w_up, ld_w, m, n, k, dtype, act);
    if (st != BZ_OK) return st;
    if ((grad_dtype != dtype && grad_dtype != BZ_F32) || (dw_gate == nullptr) != (dw_up == nullptr)) return BZ_ERR_INVALID_ARG;
    if (too_far_apart(m, n)) return BZ_ERR_UNSUPPORTED;
    if (k == 0 || (m == 0 && n == 0)) return BZ_OK;
    const uintptr_t grads = reinterpret_cast<uintptr_t>(dw_gate) | reinterpret_cast<uintptr_t>(dw_up);
    if (dx == nullptr && dw_gate == nullptr) return BZ_ERR_INVALID_ARG;
    if ((m > 1 && ld_dh < n) || (dx != nullptr && m > 1 && ld_dx < k) || (dw_gate != nullptr && n > 1 && ld_dw < k)) return BZ_ERR_INVALID_ARG;
    if (m > 0 && n > 0 && (preact == nullptr || dh == nullptr)) return BZ_ERR_INVALID_ARG;
    if (!aligned16(preact) || ((reinterpret_cast<uintptr_t>(dh) | reinterpret_cast<uintptr_t>(dx)) & 1) || grads % (grad_dtype == BZ_F32 ? 4 : 2))
        return BZ_ERR_INVALID_ARG;
    if (workspace == nullptr || !aligned256(workspace) || workspace_bytes < bz_glu_workspace_bytes(m, n, k, dtype, 1)) return BZ_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const int f32 = grad_dtype == BZ_F32;
    return dtype == BZ_F16
               ? backward<__half>(x, ld_x, w_gate, w_up, ld_w, preact, dh, ld_dh, m, n, k, act, dx, ld_dx, dw_gate, dw_up, ld_dw, f32, ws, s)
               : backward<__nv_bfloat16>(x, ld_x, w_gate, w_up, ld_w, preact, dh, ld_dh, m, n, k, act, dx, ld_dx, dw_gate, dw_up, ld_dw, f32, ws, s);
}
