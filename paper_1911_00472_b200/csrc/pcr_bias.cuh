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
    int tiles;                                 // spans of a row that warps take
    int per, slabs, slice;                     // backward: (row, span)s of a CTA; CTAs of a head; (axis, bucket)s of a CTA
};

// Bucket of a distance, from whole numbers: distances beyond the map's ends are taken as the ends.  -1: none.
__device__ __forceinline__ int bucket_of(const BiasArgs& A, int k, int q) {
    const int64_t d = (int64_t)k - q;
    const int at = (int)(d < -A.reach ? -A.reach : d > A.reach ? A.reach : d) + A.reach;
    const int n = __ldg(A.bucket_of + at);
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

// Sums over the slabs, in their order, in 64 bits; a warp a value.
template <typename T>
__global__ void __launch_bounds__(256) bias_sum_kernel(const __grid_constant__ BiasArgs A) {
    const int64_t n = (int64_t)A.axes * A.buckets * A.heads, e = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (e >= n) return;
    double s = 0;
    for (int i = threadIdx.x & 31; i < A.slabs; i += 32) s += A.partial[i * n + e];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if ((threadIdx.x & 31) == 0) static_cast<T*>(A.dtable)[e] = bias_from<T>((float)s);
}

}  // namespace pcr
