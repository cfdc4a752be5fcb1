// A learned bias of the distance between two tokens (see include/pcr.h):
//
//   bias[b, h, i, j] = sum over axes a of table[a, bucket(k_pos[a, b, j] - q_pos[a, b, i]), h]
//
// and the gradient of its table, the sum of the bias's gradient over all pairs of a bucket.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace pcr {

constexpr int kBiasAxes = 4, kBiasBuckets = 512, kBiasReach = 1 << 20;
constexpr int kBiasThreads = 256;

struct BiasArgs {
    const void* table;                         // (axes, buckets, heads)
    void* dtable;
    const int32_t* bucket_of;                  // 2 reach + 1
    const int32_t *q_pos, *k_pos;              // axis, batch, token
    int64_t qs[3], ks[3];
    const int32_t *q_ids, *k_ids;              // batch, token; null: all pairs count
    int64_t qis[2], kis[2];
    void* rows;                                // the bias, or its gradient: batch, head, row; a row's elements side by side
    int64_t rs[3];
    float* partial;                            // backward: sums of CTAs, (slab, axis, bucket, head)
    int batch, nq, nk, heads, axes, buckets, reach, table32;
    int group;                                 // forward: heads of a CTA, a multiple of 4
    int lines, mapped;                         // combinations of buckets (and of none) of all axes; whether the map is in shared memory
    int tiles;                                 // spans of a row that warps take
    int per, slabs, slice;                     // backward: (row, span)s of a CTA; CTAs of a head; (axis, bucket)s of a CTA
};

// Place of a distance in the map: distances beyond its ends are taken as the ends.  The difference stops at the ends of 32 bits, which lie beyond.
__device__ __forceinline__ int map_at(int reach, int k, int q) {
    int d;
    asm("sub.sat.s32 %0, %1, %2;" : "=r"(d) : "r"(k), "r"(q));
    return min(max(d, -reach), reach) + reach;
}
// Bucket of a distance; -1: none.
__device__ __forceinline__ int bucket_of(const BiasArgs& A, int k, int q) {
    const int n = __ldg(A.bucket_of + map_at(A.reach, k, q));
    return n >= 0 && n < A.buckets ? n : -1;
}

template <typename T> __device__ __forceinline__ T bias_from(float v) { return (T)v; }
template <> __device__ __forceinline__ __half bias_from<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 bias_from<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A warp has a span of 32 V columns of a row and goes over `group` heads: buckets are looked up once for all of them, values for
// four heads at a time out of the table in shared memory, laid out (heads / 4, axis, bucket, 4).  kWide: a lane's V columns stand
// side by side and are written as one vector; else they are 32 apart, so that a warp writes runs whatever the row's alignment is.
// Instructions bound it: 8 x 16 heads x 729 x 729 pairs of two axes in fp16 take 77.7 us, which is why the form below is there.
template <typename T, int V, bool kWide, int kAxes>
__global__ void __launch_bounds__(kBiasThreads) bias_kernel(const __grid_constant__ BiasArgs A) {
    extern __shared__ float4 table4[];
    const int tid = threadIdx.x, lane = tid & 31, batch = blockIdx.z, h0 = blockIdx.y * A.group;
    const int group = min(A.group, A.heads - h0), fours = (group + 3) / 4, lines = kAxes * (A.buckets + 1);      // the last line of an axis: zeros
    for (int i = tid; i < fours * lines * 4; i += kBiasThreads) {
        const int e = i & 3, line = (i >> 2) % lines, four = (i >> 2) / lines, a = line / (A.buckets + 1), n = line - a * (A.buckets + 1), h = h0 + four * 4 + e;
        float v = 0.f;
        if (n < A.buckets && h < A.heads) {
            const size_t at = ((size_t)a * A.buckets + n) * A.heads + h;
            v = A.table32 ? static_cast<const float*>(A.table)[at] : (float)static_cast<const T*>(A.table)[at];
        }
        reinterpret_cast<float*>(table4)[i] = v;
    }
    __syncthreads();
    const int64_t unit = (int64_t)blockIdx.x * (kBiasThreads / 32) + (tid >> 5);
    if (unit >= (int64_t)A.nq * A.tiles) return;
    const int row = (int)(unit / A.tiles), j0 = (int)(unit - (int64_t)row * A.tiles) * 32 * V + (kWide ? lane * V : lane);
    constexpr int kStep = kWide ? 1 : 32;
    int line[kAxes][V];
#pragma unroll
    for (int a = 0; a < kAxes; ++a) {
        const int q = A.q_pos[a * A.qs[0] + batch * A.qs[1] + row * A.qs[2]];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = j0 + v * kStep;
            const int n = j < A.nk ? bucket_of(A, A.k_pos[a * A.ks[0] + batch * A.ks[1] + j * A.ks[2]], q) : -1;
            line[a][v] = a * (A.buckets + 1) + (n < 0 ? A.buckets : n);
        }
    }
    unsigned masked = 0;
    if (A.q_ids) {
        const int q = A.q_ids[batch * A.qis[0] + row * A.qis[1]];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = j0 + v * kStep;
            if (j < A.nk && A.k_ids[batch * A.kis[0] + j * A.kis[1]] != q) masked |= 1u << v;
        }
    }
    T* out = static_cast<T*>(A.rows) + batch * A.rs[0] + row * A.rs[2];
    for (int f = 0; f < fours; ++f) {
        float got[4][V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float4 s = table4[f * lines + line[0][v]];
#pragma unroll
            for (int a = 1; a < kAxes; ++a) {
                const float4 x = table4[f * lines + line[a][v]];
                s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
            }
            const bool off = masked >> v & 1;
            const float none = -INFINITY;
            got[0][v] = off ? none : s.x; got[1][v] = off ? none : s.y; got[2][v] = off ? none : s.z; got[3][v] = off ? none : s.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int h = h0 + 4 * f + e;
            if (h >= A.heads) break;
            T* to = out + h * A.rs[1];
            if (kWide) {
                if (j0 < A.nk) {                          // (rows are whole vectors)
                    union { T t[V]; uint4 u; uint2 w; } x;
#pragma unroll
                    for (int v = 0; v < V; ++v) x.t[v] = bias_from<T>(got[e][v]);
                    *reinterpret_cast<uint4*>(to + j0) = x.u;
                }
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (j0 + v * kStep < A.nk) to[j0 + v * kStep] = bias_from<T>(got[e][v]);
            }
        }
    }
}

// The same where the buckets of all axes together are few: the sums are worked out first, rounded, for every combination of buckets (a line of
// `joint` for each, one more for minus infinity), in shared memory as (heads / 4, line, 4), and pairs only pick theirs.  A CTA goes over many
// rows with one table.  kWide as above; 16-bit rows that begin anywhere are written two columns at a time, those that share a word: the
// first of them is even or odd by the head's and the row's place, so that a lane looks up three columns for every two.
// What bounds it: instructions (69 % of the issue slots) and shared memory (57 % of the wavefronts).  The same pairs: 51.9 us, 2.6 TB/s written; one row of
// 32768 columns and 32 heads in bf16 3.9 us (3.8 above).
template <typename T> struct Quad;                       // a line's values for four heads
template <> struct Quad<float> { using V = float4; };
template <> struct Quad<__half> { using V = uint2; };
template <> struct Quad<__nv_bfloat16> { using V = uint2; };
template <typename T, bool kWide>
__global__ void __launch_bounds__(kBiasThreads) bias_joint_kernel(const __grid_constant__ BiasArgs A) {
    using Vec = typename Quad<T>::V;
    constexpr int kCols = 16 / sizeof(T);                  // of a lane
    constexpr bool kPairs = !kWide && sizeof(T) == 2;
    constexpr int kLook = kPairs ? 9 : kCols;
    extern __shared__ __align__(16) uint8_t shared[];
    Vec* joint = reinterpret_cast<Vec*>(shared);
    const int tid = threadIdx.x, lane = tid & 31, h0 = blockIdx.y * A.group, group = min(A.group, A.heads - h0), fours = (group + 3) / 4, lines = A.lines + 1, n1 = A.buckets + 1;
    // the table by itself, zeros behind its last bucket and head, then every combination
    float4* own = reinterpret_cast<float4*>(joint + (fours * lines + 1) / 2 * 2);
    for (int i = tid; i < fours * A.axes * n1 * 4; i += kBiasThreads) {
        const int e = i & 3, n = (i >> 2) % n1, rest = (i >> 2) / n1, a = rest % A.axes, h = h0 + 4 * (rest / A.axes) + e;
        float v = 0.f;
        if (n < A.buckets && h < A.heads) {
            const size_t at = ((size_t)a * A.buckets + n) * A.heads + h;
            v = A.table32 ? static_cast<const float*>(A.table)[at] : (float)static_cast<const T*>(A.table)[at];
        }
        reinterpret_cast<float*>(own)[i] = v;
    }
    __syncthreads();
    for (int line = tid; line < lines; line += kBiasThreads) {
        int at[kBiasAxes], rest = line;
        for (int a = A.axes - 1; a >= 0; --a) { at[a] = rest % n1; rest /= n1; }          // (the last axis's bucket counts single lines)
        for (int four = 0; four < fours; ++four) {
            float4 s = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (line < A.lines) {
                s = own[four * A.axes * n1 + at[0]];
                for (int a = 1; a < A.axes; ++a) {                                        // axis after axis
                    const float4 x = own[(four * A.axes + a) * n1 + at[a]];
                    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
                }
            }
            union { T t[4]; Vec v; } x;
            x.t[0] = bias_from<T>(s.x); x.t[1] = bias_from<T>(s.y); x.t[2] = bias_from<T>(s.z); x.t[3] = bias_from<T>(s.w);
            joint[four * lines + line] = x.v;
        }
    }
    uint16_t* map = reinterpret_cast<uint16_t*>(own + fours * A.axes * n1);
    if (A.mapped)
        for (int i = tid; i <= 2 * A.reach; i += kBiasThreads) {
            const int n = __ldg(A.bucket_of + i);
            map[i] = (uint16_t)(n >= 0 && n < A.buckets ? n : A.buckets);
        }
    __syncthreads();
    // (row, span) after (row, span): the next is a fixed number of either on
    const uint32_t all = (uint32_t)A.batch * A.nq, step = gridDim.x * (kBiasThreads / 32), step_rows = step / A.tiles, step_spans = step - step_rows * A.tiles;
    uint32_t line_no = (blockIdx.x * (kBiasThreads / 32) + (tid >> 5)) / A.tiles, span = blockIdx.x * (kBiasThreads / 32) + (tid >> 5) - line_no * A.tiles;
    for (; line_no < all; line_no += step_rows, span += step_spans) {
        if (span >= (uint32_t)A.tiles) { span -= A.tiles; ++line_no; if (line_no >= all) break; }
        const int batch = (int)(line_no / A.nq), row = (int)(line_no - batch * A.nq), j0 = (int)span * 32 * kCols;
        // a lane's columns: side by side; or every 32nd; or two of every 64, and (the last) the one before the span
        auto column = [&](int v) { return kWide ? j0 + lane * kCols + v : kPairs ? (v == 8 ? j0 - 1 : j0 + 64 * (v / 2) + 2 * lane + v % 2) : j0 + 32 * v + lane; };
        int line[kLook] = {};
        for (int a = 0; a < A.axes; ++a) {
            const int q = A.q_pos[a * A.qs[0] + batch * A.qs[1] + (int64_t)row * A.qs[2]];
            const int32_t* k = A.k_pos + a * A.ks[0] + batch * A.ks[1];
            const bool dense = A.ks[2] == 1;
#pragma unroll
            for (int v = 0; v < kLook; ++v) {
                const int j = min(max(column(v), 0), A.nk - 1), at = map_at(A.reach, dense ? k[j] : k[j * A.ks[2]], q);
                if (A.mapped) line[v] = line[v] * n1 + map[at];
                else {
                    const int n = __ldg(A.bucket_of + at);
                    line[v] = line[v] * n1 + (n >= 0 && n < A.buckets ? n : A.buckets);
                }
            }
        }
        if (A.q_ids) {
            const int q = A.q_ids[batch * A.qis[0] + (int64_t)row * A.qis[1]];
#pragma unroll
            for (int v = 0; v < kLook; ++v) {
                const int j = min(max(column(v), 0), A.nk - 1);
                if (A.k_ids[batch * A.kis[0] + (int64_t)j * A.kis[1]] != q) line[v] = A.lines;
            }
        }
        int before[kPairs ? 4 : 1];                        // of the columns before the lane's own two
        if constexpr (kPairs)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                before[v] = __shfl_up_sync(~0u, line[2 * v + 1], 1);
                const int last = v == 0 ? line[8] : __shfl_sync(~0u, line[v == 0 ? 0 : 2 * v - 1], 31);
                if (lane == 0) before[v] = last;
            }
        const bool inside = j0 + 32 * kCols <= A.nk;                                      // (nothing of the span lies behind the row)
        T* out = static_cast<T*>(A.rows) + batch * A.rs[0] + (int64_t)h0 * A.rs[1] + (int64_t)row * A.rs[2];
        for (int f = 0; f < fours; ++f) {
            const Vec* from = joint + f * lines;
            if constexpr (sizeof(T) == 4) {
                float got[4][kCols];
#pragma unroll
                for (int v = 0; v < kCols; ++v) {
                    const float4 x = from[line[v]];
                    got[0][v] = x.x; got[1][v] = x.y; got[2][v] = x.z; got[3][v] = x.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (4 * f + e >= group) break;
                    float* to = reinterpret_cast<float*>(out) + (4 * f + e) * A.rs[1];
                    if (kWide) { if (column(0) < A.nk) *reinterpret_cast<float4*>(to + column(0)) = make_float4(got[e][0], got[e][1], got[e][2], got[e][3]); }
                    else
#pragma unroll
                        for (int v = 0; v < kCols; ++v) if (column(v) < A.nk) to[column(v)] = got[e][v];
                }
            } else {
                uint2 x[8], y[kPairs ? 4 : 1];
#pragma unroll
                for (int v = 0; v < 8; ++v) x[v] = from[line[v]];
                if constexpr (kPairs)
#pragma unroll
                    for (int v = 0; v < 4; ++v) y[v] = from[before[v]];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (4 * f + e >= group) break;
                    uint16_t* to = reinterpret_cast<uint16_t*>(out + (4 * f + e) * A.rs[1]);
                    auto two = [&](const uint2& a, const uint2& b) { return __byte_perm(e < 2 ? a.x : a.y, e < 2 ? b.x : b.y, e & 1 ? 0x7632 : 0x5410); };
                    if constexpr (kWide) {
                        if (column(0) < A.nk) *reinterpret_cast<uint4*>(to + column(0)) = make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
                    } else {
                        const int odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1 & 1);  // (of the whole warp)
                        uint32_t w[4];
                        if (odd) {
#pragma unroll
                            for (int v = 0; v < 4; ++v) w[v] = two(y[v], x[2 * v]);
                        } else {
#pragma unroll
                            for (int v = 0; v < 4; ++v) w[v] = two(x[2 * v], x[2 * v + 1]);
                        }
                        to += j0 + 2 * lane - odd;
                        if (inside && (j0 > 0 || !odd)) {
#pragma unroll
                            for (int v = 0; v < 4; ++v) *reinterpret_cast<uint32_t*>(to + 64 * v) = w[v];
                        } else {
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                const int j = j0 + 64 * v + 2 * lane - odd;
                                if (j >= 0 && j + 1 < A.nk) *reinterpret_cast<uint32_t*>(to + 64 * v) = w[v];
                                else if (j >= 0 && j < A.nk) to[64 * v] = (uint16_t)w[v];
                                else if (j == -1) to[64 * v + 1] = (uint16_t)(w[v] >> 16);
                            }
                        }
                    }
                }
            }
        }
    }
}

// The table's gradient, added up by lanes that have sums of their own for every bucket (in shared memory, a bank each): no two
// threads write to one place, so that the order is always the same.  A CTA has `per` (row, span)s of a head, and `slice` of the
// (axis, bucket)s.  For few heads, or maps that do not fit into shared memory; elsewhere the products below are faster: 8 heads x 1001 x 1001 pairs of
// three axes in 32 bits 50.5 us here, 40.3 there; 2 x 16 heads x 4096 x 4096 of one axis in bf16 1500 and 324.
template <typename T, int V, bool kWide>
__global__ void __launch_bounds__(128) bias_back_kernel(const __grid_constant__ BiasArgs A) {
    extern __shared__ float hist[];                       // (warp, axis and bucket, lane)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, head = blockIdx.y, first = blockIdx.z * A.slice;
    const int mine = min(A.slice, A.axes * A.buckets - first);
    float* own = hist + (size_t)warp * mine * 32 + lane;
    for (int i = 0; i < mine; ++i) own[i * 32] = 0.f;
    constexpr int kStep = kWide ? 1 : 32;
    const int64_t all = (int64_t)A.batch * A.nq * A.tiles, from = (int64_t)blockIdx.x * A.per;
    for (int64_t unit = from + warp; unit < min(from + A.per, all); unit += 4) {
        const int64_t line = unit / A.tiles;
        const int batch = (int)(line / A.nq), row = (int)(line - (int64_t)batch * A.nq), j0 = (int)(unit - line * A.tiles) * 32 * V + (kWide ? lane * V : lane);
        const T* at = static_cast<const T*>(A.rows) + batch * A.rs[0] + head * A.rs[1] + row * A.rs[2];
        float g[V];
        if (kWide) {
            union { T t[V]; uint4 u; } x;
            x.u = j0 < A.nk ? *reinterpret_cast<const uint4*>(at + j0) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int v = 0; v < V; ++v) g[v] = (float)x.t[v];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) g[v] = j0 + v * kStep < A.nk ? (float)at[j0 + v * kStep] : 0.f;
        }
        unsigned counts = 0;
        const int q_id = A.q_ids ? A.q_ids[batch * A.qis[0] + row * A.qis[1]] : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = j0 + v * kStep;
            if (j < A.nk && (!A.q_ids || A.k_ids[batch * A.kis[0] + j * A.kis[1]] == q_id)) counts |= 1u << v;
        }
        for (int a = 0; a < A.axes; ++a) {
            const int q = A.q_pos[a * A.qs[0] + batch * A.qs[1] + row * A.qs[2]];
            int last = -1;
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!(counts >> v & 1)) continue;
                const int n = bucket_of(A, A.k_pos[a * A.ks[0] + batch * A.ks[1] + (j0 + v * kStep) * A.ks[2]], q);
                const int to = n < 0 ? -1 : a * A.buckets + n - first;
                if (to != last) {
                    if (last >= 0 && last < mine) own[last * 32] += sum;
                    last = to; sum = 0.f;
                }
                sum += g[v];
            }
            if (last >= 0 && last < mine) own[last * 32] += sum;
        }
    }
    __syncthreads();
    for (int i = warp; i < mine; i += 4) {
        float s = 0.f;
        for (int w = 0; w < 4; ++w) s += hist[((size_t)w * mine + i) * 32 + lane];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        if (lane == 0) A.partial[((size_t)blockIdx.x * A.axes * A.buckets + first + i) * A.heads + head] = s;
    }
}

// The same as products of matrices: (bucket, pair) times (pair, head), where the first is 1 at a pair's bucket and 0 elsewhere, so that all
// products are exact and the sums are the tensor cores' 32 bits.  A CTA has 16 kTiles buckets of an axis, kNt groups of 8 heads (or
// batches' heads, where all batches have the same positions), a block of columns and a share of the rows; a warp goes along a row, 64 pairs
// at a time, whole lines of 128 bytes of every head.  Which of the 16 pairs of a product stands where is free as long as both operands agree:
// lane l has head l / 4 and, of the 64 columns, 16 (l % 4) .. + 15, four products.  32-bit values are cut into three parts of 8 bits of mantissa each.
// What bounds it: instructions (57 % of the issue slots at 13 warps an SM) and the products' issue; DRAM 38 to 50 %.  A bucket is looked up once
// for all heads of a CTA; the comparison with a bucket's number makes a register of the first operand in one instruction (16-bit numbers hold 0 .. 255).
constexpr int kBackCols = 1024, kBackMap = 8192;       // columns of a CTA; places of the map in shared memory at most

template <typename T> struct OneHot;
template <> struct OneHot<__nv_bfloat16> {
    using Pair = __nv_bfloat162;
    __device__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
    }
};
template <> struct OneHot<__half> {
    using Pair = __half2;
    __device__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
    }
};
template <typename H> __device__ __forceinline__ typename OneHot<H>::Pair both(float v);
template <> __device__ __forceinline__ __nv_bfloat162 both<__nv_bfloat16>(float v) { return __float2bfloat162_rn(v); }
template <> __device__ __forceinline__ __half2 both<__half>(float v) { return __float2half2_rn(v); }
template <typename T> struct BackAs { using Half = T; static constexpr int kParts = 1; };
template <> struct BackAs<float> { using Half = __nv_bfloat16; static constexpr int kParts = 3; };

struct BackArgs {
    BiasArgs a;
    int combos, batches, rows;                 // heads, or all batches' where they share positions; those batches; rows of all batches that do not
    int col_blocks, row_slabs, each;           // blocks of columns; shares of the rows, `each` rows
    int slices;                                // of an axis's buckets
    int width;                                 // of a block
};

// (Two CTAs an SM where their sums leave room: 2048 x 2048, 32 heads, two axes of 32 buckets in bf16 163 us, at one 183; what is added to once a
// row may wait in local memory.  With more sums than that their own loads and stores cost more than the second CTA gives.)
template <typename T, int kAx, int kTiles, int kNt, bool kWide>
__global__ void __launch_bounds__(256, kAx * kTiles * kNt <= (sizeof(T) == 2 ? 8 : 4) ? 2 : 1) bias_back_mma_kernel(const __grid_constant__ BackArgs G) {
    using H = typename BackAs<T>::Half;
    using Pair = typename OneHot<H>::Pair;
    constexpr int kParts = BackAs<T>::kParts;
    extern __shared__ __align__(16) uint8_t shared[];
    const BiasArgs& A = G.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = lane >> 2, quarter = lane & 3;
    // groups of axes and slices of buckets side by side: what one CTA has read, the others find in the second-level cache
    const int sides = (A.axes + kAx - 1) / kAx * G.slices, side = blockIdx.x % sides, all = G.col_blocks * G.row_slabs, share = blockIdx.x / sides % all, axis0 = side / G.slices * kAx, base = side % G.slices * 16 * kTiles;
    const int block = share % G.col_blocks, slab = share / G.col_blocks, j0 = block * G.width, cols = min(G.width, A.nk - j0);
    const int first = (int)(blockIdx.x / sides / all) * 8 * kNt;
    float* extra = reinterpret_cast<float*>(shared);                       // sums of what is not finite
    int32_t* pos = reinterpret_cast<int32_t*>(extra + kAx * 16 * kTiles * 8 * kNt);
    int32_t* ids = pos + kAx * kBackCols;
    H* map = reinterpret_cast<H*>(ids + (A.k_ids ? kBackCols : 0));
    float* sums = reinterpret_cast<float*>(pos);                           // (when all else has been read)
    for (int i = tid; i < kAx * 16 * kTiles * 8 * kNt; i += 256) extra[i] = 0.f;
    for (int i = tid; i <= 2 * A.reach; i += 256) {
        const int n = __ldg(A.bucket_of + i);
        map[i] = (H)(float)(n >= base && n < base + 16 * kTiles && n < A.buckets ? n - base : 255);
    }
    float acc[kAx][kNt][kTiles][4] = {}, total[kAx][kNt][kTiles][4] = {};
    // The tensor cores cut off what their sums have no bits for: single ones would lose half a step with every product, always to the same side.  So they add
    // up a few products only (which values of 16 bits leave exact, or nearly so, for a row), and those sums are rounded.
    auto settle = [&] {
#pragma unroll
        for (int x = 0; x < kAx; ++x)
#pragma unroll
            for (int t = 0; t < kNt; ++t)
#pragma unroll
                for (int m = 0; m < kTiles; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { total[x][t][m][e] += acc[x][t][m][e]; if (kParts == 1) acc[x][t][m][e] = 0.f; }
    };
    int held = -1;                                                         // the batch whose columns' positions are in shared memory
    // (rows are fewer than 2^31, but what lies behind a share or a warp's last row may be more)
    const uint32_t from = (uint32_t)slab * G.each, to = min(from + G.each, (uint32_t)G.rows);
    for (uint32_t line = from; line < to;) {
        const int batch = (int)(line / A.nq);
        const uint32_t until = min(to, (uint32_t)(batch + 1) * A.nq);              // rows of one batch
        if (batch != held) {
            __syncthreads();
            for (int i = tid; i < kBackCols; i += 256) {
#pragma unroll
                for (int x = 0; x < kAx; ++x) pos[x * kBackCols + i] = i < cols && axis0 + x < A.axes ? A.k_pos[(axis0 + x) * A.ks[0] + batch * A.ks[1] + (int64_t)(j0 + i) * A.ks[2]] : 0;
                if (A.k_ids) ids[i] = i < cols ? A.k_ids[batch * A.kis[0] + (int64_t)(j0 + i) * A.kis[1]] : 0;
            }
            held = batch;
            __syncthreads();
        }
        for (uint32_t l = line + warp; l < until; l += 8) {
            const int row = (int)(l - (uint32_t)batch * A.nq);
            int q[kAx];
#pragma unroll
            for (int x = 0; x < kAx; ++x) q[x] = axis0 + x < A.axes ? A.q_pos[(axis0 + x) * A.qs[0] + batch * A.qs[1] + (int64_t)row * A.qs[2]] : 0;
            const int q_id = A.q_ids ? A.q_ids[batch * A.qis[0] + (int64_t)row * A.qis[1]] : 0;
            const T* at[kNt];
            bool has[kNt];
#pragma unroll
            for (int t = 0; t < kNt; ++t) {
                const int combo = first + 8 * t + group, b = G.batches > 1 ? combo / A.heads : 0;
                has[t] = combo < G.combos;
                at[t] = static_cast<const T*>(A.rows) + (int64_t)(batch + b) * A.rs[0] + (int64_t)(combo - b * A.heads) * A.rs[1] + (int64_t)row * A.rs[2] + j0;
            }
            // a lane's eight values of each group, those of the next step on their way
            uint4 raw[2][kNt][kParts == 1 ? 1 : 2];
            auto load = [&](uint4 (&raw)[kNt][kParts == 1 ? 1 : 2], int c) {
#pragma unroll
                for (int t = 0; t < kNt; ++t) {
                    if constexpr (kParts == 1) {
                        raw[t][0] = make_uint4(0, 0, 0, 0);
                        if (kWide) { if (has[t] && c < cols) raw[t][0] = __ldcs(reinterpret_cast<const uint4*>(at[t] + c)); }
                        else {
                            uint32_t e[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) e[i] = has[t] && c + 4 * i < cols ? __ldcs(reinterpret_cast<const unsigned short*>(at[t] + c + 4 * i)) : 0;
                            raw[t][0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            raw[t][i] = make_uint4(0, 0, 0, 0);
                            const uint32_t* p = reinterpret_cast<const uint32_t*>(at[t] + c + (kWide ? 4 : 16) * i);
                            if (kWide) { if (has[t] && c + 4 * i < cols) raw[t][i] = __ldcs(reinterpret_cast<const uint4*>(p)); }
                            else if (has[t]) {
                                if (c + 16 * i < cols) raw[t][i].x = __ldcs(p);
                                if (c + 16 * i + 4 < cols) raw[t][i].y = __ldcs(p + 4);
                                if (c + 16 * i + 8 < cols) raw[t][i].z = __ldcs(p + 8);
                                if (c + 16 * i + 12 < cols) raw[t][i].w = __ldcs(p + 12);
                            }
                        }
                    }
                }
            };
            // (rows that begin anywhere are read value by value: every fourth column is a lane's, so that four lanes read side by side)
            const int lane0 = kWide ? 16 * quarter : quarter, next = kWide ? 8 : 32;
            load(raw[0], lane0);
            load(raw[1], lane0 + next);
#pragma unroll 1
            for (int c0 = 0; c0 < cols; c0 += 64)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int c = c0 + lane0 + next * half;
                uint32_t v[kNt][kParts][4];
                uint32_t counts = 255u;                                    // which of the lane's eight columns count
                if (kWide) counts = c + 8 <= cols ? 255u : c < cols ? (1u << (cols - c)) - 1 : 0u;
                else if (c + 28 >= cols) counts = c < cols ? (2u << ((cols - 1 - c) >> 2)) - 1 : 0u;
                float whole[kParts == 3 ? kNt : 1][8];
#pragma unroll
                for (int t = 0; t < kNt; ++t) {
                    if constexpr (kParts == 1) { v[t][0][0] = raw[half][t][0].x; v[t][0][1] = raw[half][t][0].y; v[t][0][2] = raw[half][t][0].z; v[t][0][3] = raw[half][t][0].w; }
                    else
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            whole[t][4 * i] = __uint_as_float(raw[half][t][i].x); whole[t][4 * i + 1] = __uint_as_float(raw[half][t][i].y);
                            whole[t][4 * i + 2] = __uint_as_float(raw[half][t][i].z); whole[t][4 * i + 3] = __uint_as_float(raw[half][t][i].w);
                        }
                }
                if (c0 + 64 < cols) load(raw[half], c + 64);
                auto eight = [&](int (&x)[8], const int32_t* from) {
                    if (kWide) {
                        const int4 a = *reinterpret_cast<const int4*>(from + c), b = *reinterpret_cast<const int4*>(from + c + 4);
                        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
                    } else
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = from[c + 4 * i];
                };
                if (A.q_ids) {
                    int id[8];
                    eight(id, ids);
#pragma unroll
                    for (int i = 0; i < 8; ++i) counts &= id[i] == q_id ? ~0u : ~(1u << i);
                }
                // buckets of the lane's eight columns
                uint32_t n2[kAx][4];
#pragma unroll
                for (int x = 0; x < kAx; ++x) {
                    int k[8];
                    eight(k, pos + x * kBackCols);
                    const uint16_t* bits = reinterpret_cast<const uint16_t*>(map);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        n2[x][i] = bits[map_at(A.reach, k[2 * i], q[x])] | (uint32_t)bits[map_at(A.reach, k[2 * i + 1], q[x])] << 16;
                }
                if (__any_sync(~0u, counts != 255u)) {                     // what does not count is 0, whatever stands there
#pragma unroll
                    for (int t = 0; t < kNt; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (counts >> i & 1) continue;
                            if constexpr (kParts == 1) v[t][0][i / 2] &= i & 1 ? 0xffffu : 0xffff0000u;
                            else whole[t][i] = 0.f;
                        }
                }
                // A value that is not finite belongs to its own bucket and head alone, where a product with 0 would take it to all: added by itself
                // (in whatever order: what comes of infinities does not depend on it).
                bool odd = false;
                if constexpr (kParts == 1) {
                    Pair z[2] = {};
#pragma unroll
                    for (int t = 0; t < kNt; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[i & 1] = __hfma2(*reinterpret_cast<const Pair*>(&v[t][0][i]), Pair{}, z[i & 1]);
                    z[0] = __hadd2(z[0], z[1]);
                    odd = !(__low2float(z[0]) == 0.f && __high2float(z[0]) == 0.f);
                } else {
                    float z[2] = {};
#pragma unroll
                    for (int t = 0; t < kNt; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[i & 1] = fmaf(whole[t][i], 0.f, z[i & 1]);
                    odd = !(z[0] + z[1] == 0.f);
                }
                if (odd) {
#pragma unroll
                    for (int t = 0; t < kNt; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float x;
                            if constexpr (kParts == 1) { const Pair p = *reinterpret_cast<const Pair*>(&v[t][0][i / 2]); x = i & 1 ? __high2float(p) : __low2float(p); }
                            else x = whole[t][i];
                            if (isfinite(x)) continue;
#pragma unroll
                            for (int y = 0; y < kAx; ++y) {
                                const Pair np = *reinterpret_cast<const Pair*>(&n2[y][i / 2]);
                                const int n = (int)(i & 1 ? __high2float(np) : __low2float(np));
                                if (n < 16 * kTiles) atomicAdd(&extra[(y * 16 * kTiles + n) * 8 * kNt + 8 * t + group], x);
                            }
                            if constexpr (kParts == 1) v[t][0][i / 2] &= i & 1 ? 0xffffu : 0xffff0000u;
                            else whole[t][i] = 0.f;
                        }
                }
                __syncwarp();
                if constexpr (kParts == 3) {
#pragma unroll
                    for (int t = 0; t < kNt; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float x = whole[t][2 * i], y = whole[t][2 * i + 1];
#pragma unroll
                            for (int p = 0; p < 3; ++p) {
                                v[t][p][i] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
                                x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
                                y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
                            }
                        }
                }
#pragma unroll
                for (int m = 0; m < kTiles; ++m) {
                    const Pair lo = both<H>((float)(16 * m + group)), hi = both<H>((float)(16 * m + group + 8));
#pragma unroll
                    for (int x = 0; x < kAx; ++x)
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            uint32_t a[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const Pair one = __heq2(*reinterpret_cast<const Pair*>(&n2[x][2 * s + e / 2]), e & 1 ? hi : lo);
                                a[e] = *reinterpret_cast<const uint32_t*>(&one);
                            }
#pragma unroll
                            for (int t = 0; t < kNt; ++t)
#pragma unroll
                                for (int p = kParts - 1; p >= 0; --p) {
                                    const float none[4] = {};
                                    if (kParts == 3 && half == 0 && s == 0 && p == 2) OneHot<H>::mma(acc[x][t][m], a, v[t][p][2 * s], v[t][p][2 * s + 1], none);
                                    else OneHot<H>::mma(acc[x][t][m], a, v[t][p][2 * s], v[t][p][2 * s + 1], acc[x][t][m]);
                                }
                        }
                }
                if (kParts == 3 && half) settle();
            }
            if (kParts == 1) settle();
        }
        line = until;
    }
    // the warps' sums, one after the other
    __syncthreads();
    for (int w = 0; w < 8; ++w) {
        if (warp == w)
#pragma unroll
            for (int x = 0; x < kAx; ++x)
#pragma unroll
                for (int t = 0; t < kNt; ++t)
#pragma unroll
                    for (int m = 0; m < kTiles; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float& s = sums[((x * kTiles + m) * 16 + group + 8 * (e / 2)) * 8 * kNt + 8 * t + 2 * quarter + (e & 1)];
                            s = w == 0 ? total[x][t][m][e] : s + total[x][t][m][e];
                        }
        __syncthreads();
    }
    for (int i = tid; i < kAx * 16 * kTiles * 8 * kNt; i += 256) {
        const int at = i / (8 * kNt), n = base + at % (16 * kTiles), axis = axis0 + at / (16 * kTiles), combo = first + i % (8 * kNt);
        if (n >= A.buckets || axis >= A.axes || combo >= G.combos) continue;
        const int b = combo / A.heads;
        A.partial[(((size_t)share * G.batches + b) * A.axes * A.buckets + (size_t)axis * A.buckets + n) * A.heads + combo - b * A.heads] = sums[i] + extra[i];
    }
}

// Sums over the slabs, in 64 bits and always in the same order: a CTA has 32 values, a warp every 32nd slab, eight of them on their way at a
// time.
template <typename T>
__global__ void __launch_bounds__(1024) bias_sum_kernel(const __grid_constant__ BiasArgs A) {
    __shared__ double sums[32][33];
    const int64_t n = (int64_t)A.axes * A.buckets * A.heads, e = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int warp = threadIdx.x / 32;
    double s = 0;
    if (e < n)
        for (int i = warp; i < A.slabs; i += 256) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = i + 32 * u < A.slabs ? A.partial[(i + 32 * u) * n + e] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) s += x[u];
        }
    sums[warp][threadIdx.x % 32] = s;
    __syncthreads();
    s = sums[threadIdx.x % 32][warp];                                      // (a warp adds up one value)
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    const int64_t to = (int64_t)blockIdx.x * 32 + warp;
    if (threadIdx.x % 32 == 0 && to < n) static_cast<T*>(A.dtable)[to] = bias_from<T>((float)s);
}

}  // namespace pcr
