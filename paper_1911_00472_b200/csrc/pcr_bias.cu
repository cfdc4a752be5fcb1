// Host side of the learned bias of distances (see include/pcr.h): checks, choice of form, launches.  Nothing is allocated and
// nothing is kept between calls.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/pcr.h"
#include "pcr_bias.cuh"
#include "pcr_launches.h"
#include "pcr_spans.h"

using namespace pcr;

namespace {

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 148;
    }
    return n;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t size_of(int dtype) { return dtype == PCR_F32 ? 4 : 2; }
bool is_dtype(int d) { return d == PCR_F16 || d == PCR_F32 || d == PCR_BF16; }
int finish() { return cudaGetLastError() == cudaSuccess ? PCR_OK : PCR_E_CUDA; }
int64_t pairs(const pcr_bias_args& a) { return a.batch * a.q_tokens * a.k_tokens; }

int check(const pcr_bias_args& a, bool back) {
    if (!is_dtype(a.dtype) || !is_dtype(a.table_dtype) || (!back && a.table_dtype != a.dtype && a.table_dtype != PCR_F32)) return PCR_E_ARG;
    if (a.heads < 1 || a.heads > 4096 || a.axes < 1 || a.axes > kBiasAxes || a.buckets < 1 || a.buckets > kBiasBuckets || a.reach < 0 || a.reach > kBiasReach) return PCR_E_ARG;
    for (int64_t n : {a.batch, a.q_tokens, a.k_tokens}) if (n < 0 || n > 1 << 30) return PCR_E_ARG;
    if ((__int128)a.batch * a.q_tokens * a.k_tokens > (__int128)1 << 48) return PCR_E_ARG;
    if (a.batch > 65535 || (a.q_ids == nullptr) != (a.k_ids == nullptr)) return PCR_E_ARG;
    if (!a.table || !aligned(a.table, size_of(a.table_dtype))) return PCR_E_ARG;
    if (pairs(a) == 0) return PCR_OK;
    if (!a.bucket_of || !a.q_positions || !a.k_positions || !a.bias || !aligned(a.bias, size_of(a.dtype))) return PCR_E_ARG;
    for (const int32_t* p : {a.bucket_of, a.q_positions, a.k_positions, a.q_ids, a.k_ids}) if (!aligned(p, 4)) return PCR_E_ARG;
    return PCR_OK;
}

Span rows_of(const pcr_bias_args& a) { return span_of(a.bias, a.bias_stride, a.batch, a.heads, a.q_tokens, a.k_tokens, size_of(a.dtype)); }

// Whether what is written (and the scratch memory) shares memory with what is read.
bool shares(const pcr_bias_args& a, bool back, const void* scratch, size_t scratch_bytes) {
    const Span rows = rows_of(a), table = span_of(a.table, (size_t)a.axes * a.buckets * a.heads * size_of(a.table_dtype));
    const Span in[] = {span_of(a.bucket_of, (2 * (size_t)a.reach + 1) * 4), span_of(a.q_positions, a.q_stride, a.axes, a.batch, a.q_tokens, 1, 4),
                       span_of(a.k_positions, a.k_stride, a.axes, a.batch, a.k_tokens, 1, 4),
                       span_of(a.q_ids, {a.q_id_stride[0], a.q_id_stride[1], 0}, a.q_ids ? a.batch : 0, a.q_tokens, 1, 1, 4),
                       span_of(a.k_ids, {a.k_id_stride[0], a.k_id_stride[1], 0}, a.k_ids ? a.batch : 0, a.k_tokens, 1, 1, 4)};
    const Span& out = back ? table : rows;
    const Span own = span_of(scratch, scratch ? scratch_bytes : 0);
    if (share_memory(rows, table) || share_memory(own, rows) || share_memory(own, table)) return true;
    return std::any_of(in, in + 5, [&](const Span& s) { return share_memory(out, s) || share_memory(own, s); });
}

bool overlaps_itself(const pcr_bias_args& a) {
    const int64_t size[3] = {a.batch, a.heads, a.q_tokens};
    int order[3] = {0, 1, 2};
    auto far = [&](int i) { return a.bias_stride[i] < 0 ? -a.bias_stride[i] : a.bias_stride[i]; };
    std::sort(order, order + 3, [&](int x, int y) { return far(x) < far(y); });
    __int128 reach = a.k_tokens - 1;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (far(i) <= reach) return true;
        reach += (__int128)(size[i] - 1) * far(i);
    }
    return false;
}

// Rows that are whole vectors of 16 bytes.
bool whole(const pcr_bias_args& a) {
    const int64_t v = 16 / size_of(a.dtype), size[3] = {a.batch, a.heads, a.q_tokens};
    if (!aligned(a.bias, 16) || a.k_tokens % v) return false;
    for (int i = 0; i < 3; ++i) if (size[i] > 1 && a.bias_stride[i] % v) return false;
    return true;
}

BiasArgs args_of(const pcr_bias_args& a) {
    BiasArgs A = {};
    A.table = a.table; A.dtable = a.table; A.bucket_of = a.bucket_of; A.q_pos = a.q_positions; A.k_pos = a.k_positions; A.q_ids = a.q_ids; A.k_ids = a.k_ids;
    for (int i = 0; i < 3; ++i) { A.qs[i] = a.q_stride[i]; A.ks[i] = a.k_stride[i]; A.rs[i] = a.bias_stride[i]; }
    for (int i = 0; i < 2; ++i) { A.qis[i] = a.q_id_stride[i]; A.kis[i] = a.k_id_stride[i]; }
    A.rows = a.bias; A.batch = (int)a.batch; A.nq = (int)a.q_tokens; A.nk = (int)a.k_tokens; A.heads = a.heads; A.axes = a.axes;
    A.buckets = a.buckets; A.reach = a.reach; A.table32 = a.table_dtype == PCR_F32;
    return A;
}

template <typename T, int V, bool kWide>
void launch_axes(const BiasArgs& A, dim3 grid, size_t shared, cudaStream_t st) {
    if (A.axes == 1) bias_kernel<T, V, kWide, 1><<<grid, kBiasThreads, shared, st>>>(A);
    else if (A.axes == 2) bias_kernel<T, V, kWide, 2><<<grid, kBiasThreads, shared, st>>>(A);
    else if (A.axes == 3) bias_kernel<T, V, kWide, 3><<<grid, kBiasThreads, shared, st>>>(A);
    else bias_kernel<T, V, kWide, 4><<<grid, kBiasThreads, shared, st>>>(A);
}

template <typename T>
int launch_bias(BiasArgs& A, bool wide, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    // All combinations of buckets first, where 44 KB hold them for four heads at least and there are more pairs for every CTA than lines.
    int64_t lines = 1;
    for (int a = 0; a < A.axes; ++a) lines *= A.buckets + 1;
    const int64_t map = 2 * (2 * (int64_t)A.reach + 1) + 16;
    A.mapped = map <= 8 * 1024;
    const int64_t most = (46 * 1024 - (A.mapped ? map : 0)) / (4 * (int64_t)sizeof(T) * (lines + 1) + 16 * A.axes * (A.buckets + 1)) * 4;
    if (most >= 4 && (int64_t)A.batch * A.nq < INT32_MAX / 2 && (A.axes == 1 || (int64_t)A.batch * A.nq * A.nk >= lines * 2 * sm_count())) {
        const int64_t columns = A.nk + (!wide && sizeof(T) == 2 ? 1 : 0);         // (a row's first pair of columns may begin before it)
        A.tiles = (int)((columns + 32 * V - 1) / (32 * V));
        A.lines = (int)lines;
        const int64_t ctas = ((int64_t)A.batch * A.nq * A.tiles + 7) / 8, room = 3 * sm_count();
        int group = (int)std::min<int64_t>((A.heads + 3) / 4 * 4, most);
        while (group > 4 && ctas * ((A.heads + group - 1) / group) < 2 * sm_count()) group = (group / 2 + 3) / 4 * 4;
        A.group = group;
        const int groups = (A.heads + group - 1) / group;
        const dim3 grid((unsigned)std::min<int64_t>(ctas, std::max<int64_t>(1, room / groups)), groups);
        const size_t shared = (size_t)group * (lines + 1) * sizeof(T) + 16 + (size_t)group * A.axes * (A.buckets + 1) * sizeof(float) + (A.mapped ? map : 0);
        if (wide) bias_joint_kernel<T, true><<<grid, kBiasThreads, shared, st>>>(A);
        else bias_joint_kernel<T, false><<<grid, kBiasThreads, shared, st>>>(A);
        ++g_launches;
        return finish();
    }
    A.tiles = (A.nk + 32 * V - 1) / (32 * V);
    const int64_t ctas = ((int64_t)A.nq * A.tiles + 7) / 8;
    const int held = A.axes * (A.buckets + 1);
    // Heads of a CTA: as many as 40 KB of table hold, fewer where that leaves SMs without work
    int group = std::max(4, std::min((A.heads + 3) / 4 * 4, 40 * 1024 / (16 * held) * 4));
    while (group > 4 && ctas * A.batch * ((A.heads + group - 1) / group) < 2 * sm_count()) group = (group / 2 + 3) / 4 * 4;
    A.group = group;
    const size_t shared = (size_t)group * held * 4;
    const dim3 grid((unsigned)ctas, (A.heads + group - 1) / group, A.batch);
    if (wide) launch_axes<T, V, true>(A, grid, shared, st);
    else launch_axes<T, V, false>(A, grid, shared, st);
    ++g_launches;
    return finish();
}

// The gradient's form: as products of matrices where at least four heads (or batches' heads) share a look-up and the map fits into shared
// memory; else by lanes' own sums.
struct BackForm { bool products; int ax, tiles, per, slabs, slice, slices, nt, kt, combos, batches, rows, width, col_blocks, row_slabs, each; };

BackForm back_form(const pcr_bias_args& a) {
    BackForm f = {};
    // all batches have the same positions: their heads are further columns of the product
    const bool shared = a.batch > 1 && a.q_stride[1] == 0 && a.k_stride[1] == 0 && (!a.q_ids || (a.q_id_stride[0] == 0 && a.k_id_stride[0] == 0));
    f.batches = shared ? (int)a.batch : 1;
    f.combos = f.batches * a.heads;
    f.rows = (int)((shared ? 1 : a.batch) * a.q_tokens);
    if (f.combos >= 4 && 2 * a.reach + 1 <= kBackMap && (shared ? 1 : a.batch) * a.q_tokens <= INT32_MAX) {
        // axes of a CTA: what is read serves them all, as long as their sums stay in registers
        f.kt = a.buckets <= 16 ? 1 : a.buckets <= 32 ? 2 : 4;
        f.ax = f.kt == 4 ? 1 : a.axes == 3 ? 3 : std::min(a.axes, 2);
        f.slices = (a.buckets + 16 * f.kt - 1) / (16 * f.kt);
        f.nt = f.combos <= 8 ? 1 : f.combos > 16 && f.ax == 1 && a.dtype != PCR_F32 ? 4 : 2;
        // about 3 CTAs an SM, of long rows where there are enough of them: a CTA's beginning and end are a warp's work on some hundred columns
        const int64_t beside = (int64_t)((a.axes + f.ax - 1) / f.ax) * f.slices * ((f.combos + 8 * f.nt - 1) / (8 * f.nt)), room = 3 * sm_count();
        f.width = kBackCols;
        auto blocks = [&] { return (a.k_tokens + f.width - 1) / f.width; };
        while (f.width > 128 && beside * blocks() * (((int64_t)f.rows + 31) / 32) < room) f.width /= 2;
        f.col_blocks = (int)blocks();
        const int64_t want = std::max<int64_t>(1, room / std::max<int64_t>(1, beside * f.col_blocks));
        f.each = (int)std::max<int64_t>(8, (f.rows + want - 1) / want);
        f.row_slabs = (int)std::max<int64_t>(1, ((int64_t)f.rows + f.each - 1) / f.each);
        // (slabs and CTAs are numbered in 31 bits: gradients that many batches share by strides of 0 may have more)
        const int64_t slabs = (int64_t)f.row_slabs * std::max(1, f.col_blocks) * f.batches;
        f.products = slabs <= INT32_MAX / 2 && (__int128)f.row_slabs * f.col_blocks * beside <= INT32_MAX;
        f.slabs = (int)slabs;
        if (f.products) return f;
    }
    const int v = 16 / (int)size_of(a.dtype);
    f.tiles = (int)((a.k_tokens + 32 * v - 1) / (32 * v));
    f.slice = std::min(a.axes * a.buckets, 96);           // 4 warps, 128 bytes a bucket: 48 KB
    f.slices = (a.axes * a.buckets + f.slice - 1) / f.slice;
    const int64_t units = a.batch * a.q_tokens * f.tiles, want = std::max<int64_t>(1, sm_count() * 8 / a.heads);
    f.per = (int)std::min<int64_t>(INT32_MAX, std::max<int64_t>(4, (units + want - 1) / want));
    f.slabs = (int)std::max<int64_t>(1, (units + f.per - 1) / f.per);
    return f;
}

template <typename T, int kAx, int kTiles, int kNt>
int launch_products(const BackArgs& G, dim3 grid, bool wide, cudaStream_t st) {
    constexpr size_t kSums = (size_t)kAx * 16 * kTiles * 8 * kNt * 4;
    const size_t shared = kSums + std::max<size_t>((kAx + (G.a.k_ids ? 1 : 0)) * kBackCols * 4 + (2 * (size_t)G.a.reach + 1) * 2, kSums);
    static_assert(2 * kSums <= 48 * 1024 && kSums + (kAx + 1) * kBackCols * 4 + 2 * kBackMap <= 48 * 1024, "no more than any launch may have");
    if (wide) bias_back_mma_kernel<T, kAx, kTiles, kNt, true><<<grid, 256, shared, st>>>(G);
    else bias_back_mma_kernel<T, kAx, kTiles, kNt, false><<<grid, 256, shared, st>>>(G);
    ++g_launches;
    return finish();
}
template <typename T, int kNt>
int launch_tiles_of(const BackArgs& G, const BackForm& f, dim3 grid, bool wide, cudaStream_t st) {
    if (f.ax == 3) return f.kt == 1 ? launch_products<T, 3, 1, kNt>(G, grid, wide, st) : launch_products<T, 3, 2, kNt>(G, grid, wide, st);
    if (f.ax == 2) return f.kt == 1 ? launch_products<T, 2, 1, kNt>(G, grid, wide, st) : launch_products<T, 2, 2, kNt>(G, grid, wide, st);
    if (f.kt == 1) return launch_products<T, 1, 1, kNt>(G, grid, wide, st);
    if (f.kt == 2) return launch_products<T, 1, 2, kNt>(G, grid, wide, st);
    return launch_products<T, 1, 4, kNt>(G, grid, wide, st);
}
template <typename T>
int launch_back(const BackArgs& G, const BackForm& f, bool wide, cudaStream_t st) {
    const dim3 grid((unsigned)(f.row_slabs * f.col_blocks * ((G.a.axes + f.ax - 1) / f.ax) * f.slices) * ((f.combos + 8 * f.nt - 1) / (8 * f.nt)));
    if (f.nt == 1) return launch_tiles_of<T, 1>(G, f, grid, wide, st);
    if constexpr (sizeof(T) == 2)
        if (f.nt == 4) {
            if (f.kt == 1) return launch_products<T, 1, 1, 4>(G, grid, wide, st);
            if (f.kt == 2) return launch_products<T, 1, 2, 4>(G, grid, wide, st);
            return launch_products<T, 1, 4, 4>(G, grid, wide, st);
        }
    return launch_tiles_of<T, 2>(G, f, grid, wide, st);
}

}  // namespace

extern "C" {

int pcr_relative_bias(const pcr_bias_args* args, void* stream) {
    if (!args) return PCR_E_ARG;
    const pcr_bias_args& a = *args;
    if (int rc = check(a, false)) return rc;
    if (pairs(a) == 0) return PCR_OK;
    if (overlaps_itself(a) || shares(a, false, nullptr, 0)) return PCR_E_ARG;
    BiasArgs A = args_of(a);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.dtype == PCR_F16) return launch_bias<__half>(A, whole(a), st);
    if (a.dtype == PCR_BF16) return launch_bias<__nv_bfloat16>(A, whole(a), st);
    return launch_bias<float>(A, whole(a), st);
}

size_t pcr_relative_bias_scratch_bytes(const pcr_bias_args* args) {
    if (!args || check(*args, true) != PCR_OK) return 0;
    return (size_t)back_form(*args).slabs * args->axes * args->buckets * args->heads * sizeof(float);
}

int pcr_relative_bias_backward(const pcr_bias_args* args, void* scratch, void* stream) {
    if (!args) return PCR_E_ARG;
    const pcr_bias_args& a = *args;
    if (int rc = check(a, true)) return rc;
    if (!scratch || !aligned(scratch, 16) || shares(a, true, scratch, pcr_relative_bias_scratch_bytes(args))) return PCR_E_ARG;
    BiasArgs A = args_of(a);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const BackForm f = back_form(a);
    A.tiles = f.tiles; A.per = f.per; A.slabs = pairs(a) ? f.slabs : 0; A.slice = f.slice;
    A.partial = static_cast<float*>(scratch);
    if (pairs(a) && f.products) {
        BackArgs G = {A, f.combos, f.batches, f.rows, f.col_blocks, f.row_slabs, f.each, f.slices, f.width};
        const bool wide = whole(a);
        if (int rc = a.dtype == PCR_F16 ? launch_back<__half>(G, f, wide, st) : a.dtype == PCR_BF16 ? launch_back<__nv_bfloat16>(G, f, wide, st) : launch_back<float>(G, f, wide, st)) return rc;
    } else if (pairs(a)) {
        const dim3 grid(f.slabs, a.heads, f.slices);
        const size_t shared = (size_t)4 * f.slice * 128;
        const bool wide = whole(a);
        auto launch = [&](auto vectors, auto singly) { if (wide) vectors<<<grid, 128, shared, st>>>(A); else singly<<<grid, 128, shared, st>>>(A); };
        if (a.dtype == PCR_F16) launch(bias_back_kernel<__half, 8, true>, bias_back_kernel<__half, 8, false>);
        else if (a.dtype == PCR_BF16) launch(bias_back_kernel<__nv_bfloat16, 8, true>, bias_back_kernel<__nv_bfloat16, 8, false>);
        else launch(bias_back_kernel<float, 4, true>, bias_back_kernel<float, 4, false>);
        ++g_launches;
    }
    const unsigned grid = (unsigned)(((int64_t)a.axes * a.buckets * a.heads + 31) / 32);
    if (a.table_dtype == PCR_F16) bias_sum_kernel<__half><<<grid, 1024, 0, st>>>(A);
    else if (a.table_dtype == PCR_BF16) bias_sum_kernel<__nv_bfloat16><<<grid, 1024, 0, st>>>(A);
    else bias_sum_kernel<float><<<grid, 1024, 0, st>>>(A);
    ++g_launches;
    return finish();
}

}  // extern "C"
