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
    int lines;                                 // combinations of buckets (and of none) of all axes
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
template <typename T> struct Quad;                       // a line's values for four heads
template <> struct Quad<float> { using V = float4; };
template <> struct Quad<__half> { using V = uint2; };
template <> struct Quad<__nv_bfloat16> { using V = uint2; };
template <typename T, bool kWide>
__global__ void __launch_bounds__(kBiasThreads) bias_joint_kernel(const __grid_constant__ BiasArgs A) {
    using Vec = typename Quad<T>::V;
    constexpr int kCols = 16 / sizeof(T);                  // of a lane
    constexpr bool kPairs = !kWide && sizeof(T) == 2;
    constexpr int kLook = kPairs ? 12 : kCols;
    extern __shared__ __align__(16) uint8_t shared[];
    Vec* joint = reinterpret_cast<Vec*>(shared);
    const int tid = threadIdx.x, lane = tid & 31, h0 = blockIdx.y * A.group, group = min(A.group, A.heads - h0), fours = (group + 3) / 4, lines = A.lines + 1, n1 = A.buckets + 1;
    for (int i = tid; i < fours * lines; i += kBiasThreads) {
        const int four = i / lines, line = i - four * lines;
        float s[4] = {};
        int rest = line;
        for (int a = A.axes - 1; a >= 0; --a) {            // (the last axis's bucket counts single lines)
            const int n = rest % n1;
            rest /= n1;
            for (int e = 0; e < 4; ++e) {
                const int h = h0 + 4 * four + e;
                if (n >= A.buckets || h >= A.heads) continue;
                const size_t at = ((size_t)a * A.buckets + n) * A.heads + h;
                s[e] += A.table32 ? static_cast<const float*>(A.table)[at] : (float)static_cast<const T*>(A.table)[at];
            }
        }
        union { T t[4]; Vec v; } x;
        for (int e = 0; e < 4; ++e) x.t[e] = bias_from<T>(line == A.lines ? -INFINITY : s[e]);
        joint[i] = x.v;
    }
    __syncthreads();
    const int64_t per = (int64_t)A.nq * A.tiles, all = per * A.batch;
    for (int64_t unit = (int64_t)blockIdx.x * (kBiasThreads / 32) + (tid >> 5); unit < all; unit += (int64_t)gridDim.x * (kBiasThreads / 32)) {
        const int batch = (int)(unit / per), in = (int)(unit - batch * per), row = in / A.tiles, j0 = (in - row * A.tiles) * 32 * kCols;
        // a lane's columns: side by side; or every 32nd; or the three around every 64th even one
        auto column = [&](int v) { return kWide ? j0 + lane * kCols + v : kPairs ? j0 + 64 * (v / 3) + 2 * lane + v % 3 - 1 : j0 + 32 * v + lane; };
        int line[kLook] = {};
        for (int a = 0; a < A.axes; ++a) {
            const int q = A.q_pos[a * A.qs[0] + batch * A.qs[1] + (int64_t)row * A.qs[2]];
            const int32_t* k = A.k_pos + a * A.ks[0] + batch * A.ks[1];
#pragma unroll
            for (int v = 0; v < kLook; ++v) {
                const int j = min(max(column(v), 0), A.nk - 1), n = bucket_of(A, k[j * A.ks[2]], q);
                line[v] = line[v] * n1 + (n < 0 ? A.buckets : n);
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
                uint2 x[kLook];
#pragma unroll
                for (int v = 0; v < kLook; ++v) x[v] = from[line[v]];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (4 * f + e >= group) break;
                    uint16_t* to = reinterpret_cast<uint16_t*>(out + (4 * f + e) * A.rs[1]);
                    auto two = [&](int v, int w) { return __byte_perm(e < 2 ? x[v].x : x[v].y, e < 2 ? x[w].x : x[w].y, e & 1 ? 0x7632 : 0x5410); };
                    if constexpr (kWide) {
                        if (column(0) < A.nk) *reinterpret_cast<uint4*>(to + column(0)) = make_uint4(two(0, 1), two(2, 3), two(4, 5), two(6, 7));
                    } else {
                        const int odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1 & 1);       // (of the whole warp)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const uint32_t y = odd ? two(3 * v, 3 * v + 1) : two(3 * v + 1, 3 * v + 2);
                            const int j = column(3 * v + 1) - odd;
                            if (j >= 0 && j + 1 < A.nk) *reinterpret_cast<uint32_t*>(to + j) = y;
                            else if (j >= 0 && j < A.nk) to[j] = (uint16_t)y;
                            else if (j == -1) to[0] = (uint16_t)(y >> 16);
                        }
                    }
                }
            }
        }
    }
}

// The table's gradient, added up by lanes that have sums of their own for every bucket (in shared memory, a bank each): no two
// threads write to one place, so that the order is always the same.  A CTA has `per` (row, span)s of a head, and `slice` of the
// (axis, bucket)s.
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
// batches' heads, where all batches have the same positions), a block of columns and a share of the rows; a warp goes along a row, 32 pairs
// at a time.  Which of the 16 pairs of a step stands where is free as long as both operands agree: lane l has heads l / 4 and, of the step's 32
// columns, 8 (l % 4) .. + 7, one vector of 16 bits, two steps.  32-bit values are cut into three parts of 8 bits of mantissa each.
// What bounds it: instructions.  A bucket is looked up once for all heads of a CTA; the comparison with a bucket's number makes a
// register of the first operand in one instruction (16-bit numbers hold 0 .. 255).
constexpr int kBackCols = 1024, kBackMap = 16384;       // columns of a CTA; places of the map in shared memory at most

template <typename T> struct OneHot;
template <> struct OneHot<__nv_bfloat16> {
    using Pair = __nv_bfloat162;
    __device__ static void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct OneHot<__half> {
    using Pair = __half2;
    __device__ static void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
};

template <typename T, int kTiles, int kNt, bool kWide>
__global__ void __launch_bounds__(256) bias_back_mma_kernel(const __grid_constant__ BackArgs G) {
    using H = typename BackAs<T>::Half;
    using Pair = typename OneHot<H>::Pair;
    constexpr int kParts = BackAs<T>::kParts;
    extern __shared__ __align__(16) uint8_t shared[];
    const BiasArgs& A = G.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = lane >> 2, quarter = lane & 3;
    // axes and slices of buckets side by side: what one CTA has read, the others find in the second-level cache
    const int sides = A.axes * G.slices, side = blockIdx.x % sides, share = blockIdx.x / sides, axis = side / G.slices, base = (side - axis * G.slices) * 16 * kTiles;
    const int block = share % G.col_blocks, slab = share / G.col_blocks, j0 = block * kBackCols, cols = min(kBackCols, A.nk - j0);
    const int first = blockIdx.y * 8 * kNt;
    float* extra = reinterpret_cast<float*>(shared);                       // sums of what is not finite
    int32_t* pos = reinterpret_cast<int32_t*>(extra + 16 * kTiles * 8 * kNt);
    int32_t* ids = pos + kBackCols;
    H* map = reinterpret_cast<H*>(ids + (A.k_ids ? kBackCols : 0));
    float* sums = reinterpret_cast<float*>(pos);                           // (when all else has been read)
    for (int i = tid; i < 16 * kTiles * 8 * kNt; i += 256) extra[i] = 0.f;
    for (int i = tid; i <= 2 * A.reach; i += 256) {
        const int n = __ldg(A.bucket_of + i) - base;
        map[i] = (H)(float)(n >= 0 && n < 16 * kTiles && n + base < A.buckets ? n : 255);
    }
    float acc[kNt][kTiles][4] = {};
    int held = -1;                                                         // the batch whose columns' positions are in shared memory
    const int from = slab * G.each, to = min(from + G.each, G.rows);
    for (int line = from; line < to;) {
        const int batch = line / A.nq, until = min(to, (batch + 1) * A.nq);       // rows of one batch
        if (batch != held) {
            __syncthreads();
            for (int i = tid; i < kBackCols; i += 256) {
                pos[i] = i < cols ? A.k_pos[axis * A.ks[0] + batch * A.ks[1] + (int64_t)(j0 + i) * A.ks[2]] : 0;
                if (A.k_ids) ids[i] = i < cols ? A.k_ids[batch * A.kis[0] + (int64_t)(j0 + i) * A.kis[1]] : 0;
            }
            held = batch;
            __syncthreads();
        }
        for (int l = line + warp; l < until; l += 8) {
            const int row = l - batch * A.nq;
            const int q = A.q_pos[axis * A.qs[0] + batch * A.qs[1] + (int64_t)row * A.qs[2]], q_id = A.q_ids ? A.q_ids[batch * A.qis[0] + (int64_t)row * A.qis[1]] : 0;
            const T* at[kNt];
            bool has[kNt];
#pragma unroll
            for (int t = 0; t < kNt; ++t) {
                const int combo = first + 8 * t + group, b = G.batches > 1 ? combo / A.heads : 0;
                has[t] = combo < G.combos;
                at[t] = static_cast<const T*>(A.rows) + (int64_t)(batch + b) * A.rs[0] + (int64_t)(combo - b * A.heads) * A.rs[1] + (int64_t)row * A.rs[2] + j0;
            }
            // a lane's eight values of each group, those of the next step on their way
            uint4 raw[kNt][kParts == 1 ? 1 : 2];
            auto load = [&](int c) {
#pragma unroll
                for (int t = 0; t < kNt; ++t) {
                    if constexpr (kParts == 1) {
                        raw[t][0] = make_uint4(0, 0, 0, 0);
                        if (kWide) { if (has[t] && c < cols) raw[t][0] = __ldcs(reinterpret_cast<const uint4*>(at[t] + c)); }
                        else {
                            uint32_t e[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) e[i] = has[t] && c + i < cols ? __ldcs(reinterpret_cast<const unsigned short*>(at[t] + c + i)) : 0;
                            raw[t][0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            raw[t][i] = make_uint4(0, 0, 0, 0);
                            const uint32_t* p = reinterpret_cast<const uint32_t*>(at[t] + c + 4 * i);
                            if (kWide) { if (has[t] && c + 4 * i < cols) raw[t][i] = __ldcs(reinterpret_cast<const uint4*>(p)); }
                            else if (has[t]) {
                                if (c + 4 * i < cols) raw[t][i].x = __ldcs(p);
                                if (c + 4 * i + 1 < cols) raw[t][i].y = __ldcs(p + 1);
                                if (c + 4 * i + 2 < cols) raw[t][i].z = __ldcs(p + 2);
                                if (c + 4 * i + 3 < cols) raw[t][i].w = __ldcs(p + 3);
                            }
                        }
                    }
                }
            };
            load(8 * quarter);
#pragma unroll 1
            for (int c0 = 0; c0 < cols; c0 += 32) {
                const int c = c0 + 8 * quarter;
                uint32_t v[kNt][kParts][4];
                uint32_t counts = c + 8 <= cols ? 255u : c < cols ? (1u << (cols - c)) - 1 : 0u;
                float whole[kParts == 3 ? kNt : 1][8];
#pragma unroll
                for (int t = 0; t < kNt; ++t) {
                    if constexpr (kParts == 1) { v[t][0][0] = raw[t][0].x; v[t][0][1] = raw[t][0].y; v[t][0][2] = raw[t][0].z; v[t][0][3] = raw[t][0].w; }
                    else
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            whole[t][4 * i] = __uint_as_float(raw[t][i].x); whole[t][4 * i + 1] = __uint_as_float(raw[t][i].y);
                            whole[t][4 * i + 2] = __uint_as_float(raw[t][i].z); whole[t][4 * i + 3] = __uint_as_float(raw[t][i].w);
                        }
                }
                if (c0 + 32 < cols) load(c + 32);
                // buckets of the lane's eight columns; pairs that do not count have none
                uint32_t n2[4];
                {
                    const int4 p0 = *reinterpret_cast<const int4*>(pos + c), p1 = *reinterpret_cast<const int4*>(pos + c + 4);
                    const int k[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
                    if (A.q_ids) {
                        const int4 s0 = *reinterpret_cast<const int4*>(ids + c), s1 = *reinterpret_cast<const int4*>(ids + c + 4);
                        const int id[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
                        for (int i = 0; i < 8; ++i) counts &= id[i] == q_id ? ~0u : ~(1u << i);
                    }
                    const uint16_t* bits = reinterpret_cast<const uint16_t*>(map);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        n2[i] = bits[map_at(A.reach, k[2 * i], q)] | (uint32_t)bits[map_at(A.reach, k[2 * i + 1], q)] << 16;
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
                            const Pair np = *reinterpret_cast<const Pair*>(&n2[i / 2]);
                            const int n = (int)(i & 1 ? __high2float(np) : __low2float(np));
                            if (n < 16 * kTiles) atomicAdd(&extra[n * 8 * kNt + 8 * t + group], x);
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
                    for (int s = 0; s < 2; ++s) {
                        uint32_t a[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const Pair one = __heq2(*reinterpret_cast<const Pair*>(&n2[2 * s + e / 2]), e & 1 ? hi : lo);
                            a[e] = *reinterpret_cast<const uint32_t*>(&one);
                        }
#pragma unroll
                        for (int t = 0; t < kNt; ++t)
#pragma unroll
                            for (int p = kParts - 1; p >= 0; --p) OneHot<H>::mma(acc[t][m], a, v[t][p][2 * s], v[t][p][2 * s + 1]);
                    }
                }
            }
        }
        line = until;
    }
    // the warps' sums, one after the other
    __syncthreads();
    for (int w = 0; w < 8; ++w) {
        if (warp == w)
#pragma unroll
            for (int t = 0; t < kNt; ++t)
#pragma unroll
                for (int m = 0; m < kTiles; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& s = sums[(16 * m + group + 8 * (e / 2)) * 8 * kNt + 8 * t + 2 * quarter + (e & 1)];
                        s = w == 0 ? acc[t][m][e] : s + acc[t][m][e];
                    }
        __syncthreads();
    }
    for (int i = tid; i < 16 * kTiles * 8 * kNt; i += 256) {
        const int n = i / (8 * kNt), combo = first + i % (8 * kNt);
        if (base + n >= A.buckets || combo >= G.combos) continue;
        const int b = combo / A.heads;
        A.partial[(((size_t)share * G.batches + b) * A.axes * A.buckets + (size_t)axis * A.buckets + base + n) * A.heads + combo - b * A.heads] = sums[i] + extra[i];
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
