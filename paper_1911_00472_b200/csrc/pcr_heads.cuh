// Queries and keys turned by the positions of their tokens, with or without a root-mean-square norm of every head in
// front, and the backward pass of both together.
//
//   angle_i = position[axis_i] * inv_freq_i                    (64 bits: the position may lie millions of turns away)
//   turned: (a, b) -> (a cos - b sin, a sin + b cos) for the pairs (i, i + rot/2) or (2 i, 2 i + 1), i < rot/2
//   forward, norm:  y = turn(w * x * r),  r = 1 / sqrt(mean(x^2) + eps)
//   backward:       d = turn back(g),  u = x * r,  dx = r * (d * w - u * mean(d * w * u)),  dw = sum over rows of d * u
//
// All of it reads every value once and writes every value once with few operations between: HBM bounds it.  A thread
// holds V pairs of a row (two vectors of up to 16 bytes), the lanes of a row stand side by side in one warp (their sums
// meet in shuffles, rows never leave the registers), and a thread goes over several heads of ONE token, so that cosine
// and sine are worked out once for all of them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace pcr {

constexpr int kMaxAxes = 4;
constexpr int kMaxHeadDim = 512;
constexpr int kHeadThreads = 128;

// One of the two operands (queries, keys).  Strides of batch, token and head in elements.
struct HeadBlock {
    const void* x;
    void* y;
    const void* g;
    const void* weight;
    float* partial;               // backward: sums of dw, one row of head_dim per CTA
    int64_t xs[3], ys[3], gs[3];
    int32_t heads, slots;         // slots: shares of the heads, `per` heads each but for the last
};

struct HeadArgs {
    HeadBlock part[2];
    const int32_t* positions;
    int64_t ps[3];                // strides of axis, batch, token
    const void* inv_freq;
    const int32_t* axes;
    uint32_t tokens, seq;         // batch * tokens of a sequence, tokens of a sequence
    int32_t n_axes, freq64, weight32, inverse;
    int32_t dim, rot, chunks, per;
    float eps, inv_dim;
};

template <typename T, int N> struct alignas(sizeof(T) * N) Vec { T v[N]; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// cosine and sine of position * freq: the whole turns are taken off in 64 bits, what is left fits single precision
__device__ __forceinline__ void turn_of(int32_t position, double freq, bool inverse, float& c, float& s) {
    double turns = (double)position * (freq * 0.15915494309189533577);       // 1 / (2 pi)
    turns -= rint(turns);
    sincospif((float)(2.0 * turns), &s, &c);
    if (inverse) s = -s;
}

__device__ __forceinline__ double freq_at(const HeadArgs& A, int i) {
    return A.freq64 ? static_cast<const double*>(A.inv_freq)[i] : (double)static_cast<const float*>(A.inv_freq)[i];
}
template <typename T> __device__ __forceinline__ float weight_of(const HeadArgs& A, const void* w, int i) {
    return A.weight32 ? static_cast<const float*>(w)[i] : to_f(static_cast<const T*>(w)[i]);
}

// A position on an axis that is not there is 0: the pair stays as it is.
__device__ __forceinline__ int32_t on_axis(const int32_t (&p)[kMaxAxes], int axis) {
    int32_t r = 0;
#pragma unroll
    for (int a = 0; a < kMaxAxes; ++a) r = axis == a ? p[a] : r;
    return r;
}
__device__ __forceinline__ void positions_of(const HeadArgs& A, uint32_t b, uint32_t t, int32_t (&p)[kMaxAxes]) {
    const int32_t* at = A.positions + (int64_t)b * A.ps[1] + (int64_t)t * A.ps[2];
#pragma unroll
    for (int a = 0; a < kMaxAxes; ++a) p[a] = a < A.n_axes ? __ldg(at + (int64_t)a * A.ps[0]) : 0;
}

enum { kTurn = 0, kNormTurn = 1, kNormTurnBack = 2 };

// Sum of v over the `n` lanes of a row that begins at lane `first`; every lane of the row gets it.
__device__ __forceinline__ float row_sum(float v, int first, int at, int n) {
    if ((n & (n - 1)) == 0) {
        for (int o = n >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    for (int o = n > 16 ? 16 : n > 8 ? 8 : n > 4 ? 4 : 2; o > 0; o >>= 1) {
        const float w = __shfl_down_sync(0xffffffffu, v, o);
        if (at + o < n) v += w;
    }
    return __shfl_sync(0xffffffffu, v, first);
}

// grid (token groups, slots of queries then keys).  A warp takes 32 / chunks tokens at a time; tokens go round the grid.
template <typename T, int V, int kMode, bool kNext>
__global__ void __launch_bounds__(kHeadThreads) heads_kernel(const __grid_constant__ HeadArgs A) {
    using VT = Vec<T, V>;
    const int which = (int)blockIdx.y >= A.part[0].slots ? 1 : 0;
    const HeadBlock& H = A.part[which];
    const int slot = (int)blockIdx.y - (which ? A.part[0].slots : 0);
    const int h0 = slot * A.per, h1 = min(h0 + A.per, H.heads);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nc = A.chunks, rows = 32 / nc;
    const int sub = lane / nc, chunk = lane - sub * nc, first = sub * nc;
    const bool in_row = sub < rows;
    // where this thread's two vectors lie in a head
    const int turning = A.rot / (2 * V);
    const bool turns = chunk < turning;
    const int pair0 = chunk * V;
    int o1, o2;
    if (kNext) { o1 = 2 * V * chunk; o2 = o1 + V; }
    else if (turns) { o1 = pair0; o2 = pair0 + A.rot / 2; }
    else { o1 = A.rot + 2 * V * (chunk - turning); o2 = o1 + V; }
    float w1[V], w2[V], dw1[V], dw2[V];
    if (kMode != kTurn) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool there = H.weight != nullptr && in_row;
            w1[i] = there ? weight_of<T>(A, H.weight, o1 + i) : 1.f;
            w2[i] = there ? weight_of<T>(A, H.weight, o2 + i) : 1.f;
            dw1[i] = dw2[i] = 0.f;
        }
    }
    constexpr int kWarps = kHeadThreads / 32;
    const uint32_t step = gridDim.x * (uint32_t)(kWarps * rows);
    const uint32_t base0 = (blockIdx.x * kWarps + warp) * (uint32_t)rows;
    for (uint32_t base = base0; base < A.tokens; base += step) {           // (the bound holds for the whole warp: shuffles inside)
        const uint32_t n = base + (uint32_t)sub;
        const bool live = in_row && n < A.tokens;
        const uint32_t b = live ? n / A.seq : 0, t = live ? n - b * A.seq : 0;
        float c[V], s[V];
        {
            int32_t p[kMaxAxes] = {0, 0, 0, 0};
            if (live && turns) positions_of(A, b, t, p);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = 1.f; s[i] = 0.f;
                if (live && turns) turn_of(on_axis(p, __ldg(A.axes + pair0 + i)), freq_at(A, pair0 + i), A.inverse, c[i], s[i]);
            }
        }
        const T* x = static_cast<const T*>(H.x) + (int64_t)b * H.xs[0] + (int64_t)t * H.xs[1];
        T* y = static_cast<T*>(H.y) + (int64_t)b * H.ys[0] + (int64_t)t * H.ys[1];
        const T* g = kMode == kNormTurnBack ? static_cast<const T*>(H.g) + (int64_t)b * H.gs[0] + (int64_t)t * H.gs[1] : nullptr;
        for (int h = h0; h < h1; ++h) {
            VT x1, x2, g1, g2;
#pragma unroll
            for (int i = 0; i < V; ++i) { x1.v[i] = x2.v[i] = from_f<T>(0.f); g1.v[i] = g2.v[i] = from_f<T>(0.f); }
            if (live) {
                const T* xr = x + (int64_t)h * H.xs[2];
                x1 = *reinterpret_cast<const VT*>(xr + o1); x2 = *reinterpret_cast<const VT*>(xr + o2);
                if (kMode == kNormTurnBack) {
                    const T* gr = g + (int64_t)h * H.gs[2];
                    g1 = *reinterpret_cast<const VT*>(gr + o1); g2 = *reinterpret_cast<const VT*>(gr + o2);
                }
            }
            float a1[V], a2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) { a1[i] = to_f(x1.v[i]); a2[i] = to_f(x2.v[i]); }
            // element i of the first and of the second vector are a pair, or 2 i and 2 i + 1 of both together
            auto pairwise = [&](float (&p)[V], float (&q)[V], float sign) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float& a = kNext ? (2 * i < V ? p[(2 * i) % V] : q[(2 * i) % V]) : p[i];
                    float& e = kNext ? (2 * i < V ? p[(2 * i + 1) % V] : q[(2 * i + 1) % V]) : q[i];
                    const float si = sign * s[i], u = a * c[i] - e * si, v = a * si + e * c[i];
                    a = u; e = v;
                }
            };
            float r1[V], r2[V];
            if (kMode == kTurn) {
                pairwise(a1, a2, 1.f);
#pragma unroll
                for (int i = 0; i < V; ++i) { r1[i] = a1[i]; r2[i] = a2[i]; }
            } else {
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) sq += a1[i] * a1[i] + a2[i] * a2[i];
                if (kMode == kNormTurn) {
                    sq = row_sum(sq, first, chunk, nc);
                    const float r = 1.f / sqrtf(sq * A.inv_dim + A.eps);
#pragma unroll
                    for (int i = 0; i < V; ++i) { r1[i] = a1[i] * r * w1[i]; r2[i] = a2[i] * r * w2[i]; }
                    pairwise(r1, r2, 1.f);
                } else {
                    float d1[V], d2[V], dot = 0.f;
#pragma unroll
                    for (int i = 0; i < V; ++i) { d1[i] = to_f(g1.v[i]); d2[i] = to_f(g2.v[i]); }
                    pairwise(d1, d2, -1.f);
#pragma unroll
                    for (int i = 0; i < V; ++i) dot += d1[i] * w1[i] * a1[i] + d2[i] * w2[i] * a2[i];
                    sq = row_sum(sq, first, chunk, nc);
                    dot = row_sum(dot, first, chunk, nc);
                    const float r = live ? 1.f / sqrtf(sq * A.inv_dim + A.eps) : 0.f;
                    const float m = dot * r * A.inv_dim;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float u1 = a1[i] * r, u2 = a2[i] * r;
                        r1[i] = r * (d1[i] * w1[i] - u1 * m); r2[i] = r * (d2[i] * w2[i] - u2 * m);
                        dw1[i] += d1[i] * u1; dw2[i] += d2[i] * u2;
                    }
                }
            }
            if (live) {
                VT y1, y2;
#pragma unroll
                for (int i = 0; i < V; ++i) { y1.v[i] = from_f<T>(r1[i]); y2.v[i] = from_f<T>(r2[i]); }
                T* yr = y + (int64_t)h * H.ys[2];
                *reinterpret_cast<VT*>(yr + o1) = y1; *reinterpret_cast<VT*>(yr + o2) = y2;
            }
        }
    }
    if (kMode == kNormTurnBack) {
        if (H.partial == nullptr) return;                       // (the same for the whole CTA)
        __shared__ float sums[kWarps][kMaxHeadDim];
        // the rows of a warp, in the order of their lanes
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float p = dw1[i], q = dw2[i];
            for (int k = 1; k < rows; ++k) {
                const float pk = __shfl_sync(0xffffffffu, dw1[i], chunk + k * nc), qk = __shfl_sync(0xffffffffu, dw2[i], chunk + k * nc);
                p += pk; q += qk;
            }
            if (sub == 0) { sums[warp][o1 + i] = p; sums[warp][o2 + i] = q; }
        }
        __syncthreads();
        float* out = H.partial + ((size_t)slot * gridDim.x + blockIdx.x) * A.dim;
        for (int j = threadIdx.x; j < A.dim; j += kHeadThreads) {
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) v += sums[k][j];
            out[j] = v;
        }
    }
}

// Heads of any even or odd size, any alignment and any strides: a warp a token, lanes over pairs, then over what is not
// turned, value by value.
template <typename T, int kMode, bool kNext>
__global__ void __launch_bounds__(kHeadThreads) heads_any_kernel(const __grid_constant__ HeadArgs A) {
    constexpr int kWarps = kHeadThreads / 32;
    __shared__ float sums[kMode == kNormTurnBack ? kWarps : 1][kMode == kNormTurnBack ? kMaxHeadDim : 1];
    const int which = (int)blockIdx.y >= A.part[0].slots ? 1 : 0;
    const HeadBlock& H = A.part[which];
    const int slot = (int)blockIdx.y - (which ? A.part[0].slots : 0);
    const int h0 = slot * A.per, h1 = min(h0 + A.per, H.heads);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int half = A.rot / 2;
    if (kMode == kNormTurnBack)
        for (int j = lane; j < A.dim; j += 32) sums[warp][j] = 0.f;          // (a lane keeps to elements of its own, but for this)
    __syncwarp();
    for (uint32_t n = blockIdx.x * kWarps + warp; n < A.tokens; n += gridDim.x * kWarps) {
        const uint32_t b = n / A.seq, t = n - b * A.seq;
        int32_t p[kMaxAxes];
        positions_of(A, b, t, p);
        for (int h = h0; h < h1; ++h) {
            const T* x = static_cast<const T*>(H.x) + (int64_t)b * H.xs[0] + (int64_t)t * H.xs[1] + (int64_t)h * H.xs[2];
            T* y = static_cast<T*>(H.y) + (int64_t)b * H.ys[0] + (int64_t)t * H.ys[1] + (int64_t)h * H.ys[2];
            const T* g = kMode == kNormTurnBack ? static_cast<const T*>(H.g) + (int64_t)b * H.gs[0] + (int64_t)t * H.gs[1] + (int64_t)h * H.gs[2] : nullptr;
            auto weight = [&](int j) { return H.weight ? weight_of<T>(A, H.weight, j) : 1.f; };
            float r = 1.f, m = 0.f;
            if (kMode != kTurn) {
                float sq = 0.f, dot = 0.f;
                for (int j = lane; j < A.dim; j += 32) { const float v = to_f(x[j]); sq += v * v; }
                if (kMode == kNormTurnBack) {
                    for (int i = lane; i < half; i += 32) {
                        const int ja = kNext ? 2 * i : i, jb = kNext ? 2 * i + 1 : i + half;
                        float c, s;
                        turn_of(on_axis(p, A.axes[i]), freq_at(A, i), false, c, s);
                        const float ga = to_f(g[ja]), gb = to_f(g[jb]);
                        dot += (ga * c + gb * s) * weight(ja) * to_f(x[ja]) + (gb * c - ga * s) * weight(jb) * to_f(x[jb]);
                    }
                    for (int j = A.rot + lane; j < A.dim; j += 32) dot += to_f(g[j]) * weight(j) * to_f(x[j]);
                }
                sq = row_sum(sq, 0, lane, 32);
                if (kMode == kNormTurnBack) dot = row_sum(dot, 0, lane, 32);
                r = 1.f / sqrtf(sq * A.inv_dim + A.eps);
                m = dot * r * A.inv_dim;
            }
            for (int i = lane; i < half; i += 32) {
                const int ja = kNext ? 2 * i : i, jb = kNext ? 2 * i + 1 : i + half;
                float c, s;
                turn_of(on_axis(p, A.axes[i]), freq_at(A, i), A.inverse, c, s);
                float a = to_f(x[ja]), e = to_f(x[jb]);
                if (kMode == kNormTurnBack) {
                    const float ga = to_f(g[ja]), gb = to_f(g[jb]), da = ga * c + gb * s, db = gb * c - ga * s;
                    const float ua = a * r, ub = e * r;
                    y[ja] = from_f<T>(r * (da * weight(ja) - ua * m));
                    y[jb] = from_f<T>(r * (db * weight(jb) - ub * m));
                    sums[warp][ja] += da * ua; sums[warp][jb] += db * ub;
                } else {
                    if (kMode == kNormTurn) { a *= r * weight(ja); e *= r * weight(jb); }
                    y[ja] = from_f<T>(a * c - e * s);
                    y[jb] = from_f<T>(a * s + e * c);
                }
            }
            for (int j = A.rot + lane; j < A.dim; j += 32) {
                const float v = to_f(x[j]);
                if (kMode == kNormTurnBack) {
                    const float d = to_f(g[j]);
                    y[j] = from_f<T>(r * (d * weight(j) - v * r * m));
                    sums[warp][j] += d * (v * r);
                } else {
                    y[j] = kMode == kNormTurn ? from_f<T>(v * r * weight(j)) : x[j];
                }
            }
        }
    }
    if (kMode == kNormTurnBack) {
        if (H.partial == nullptr) return;
        __syncthreads();
        float* out = H.partial + ((size_t)slot * gridDim.x + blockIdx.x) * A.dim;
        for (int j = threadIdx.x; j < A.dim; j += kHeadThreads) {
            float v = 0.f;
            for (int k = 0; k < kWarps; ++k) v += sums[k][j];
            out[j] = v;
        }
    }
}

// dw of queries (blockIdx.y 0) and keys (1): the rows of partial sums added up, eight columns a CTA, always in the same order.
struct WeightSums {
    const float* partial[2];
    void* dw[2];
    int32_t rows[2];
    int32_t dim, weight32;
};
constexpr int kSumCols = 8, kSumThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kSumThreads) weight_sums_kernel(const WeightSums S) {
    constexpr int kRows = kSumThreads / kSumCols;
    __shared__ float part[kRows][kSumCols + 1];
    const bool keys = blockIdx.y != 0;
    const float* partial = keys ? S.partial[1] : S.partial[0];
    const int rows = keys ? S.rows[1] : S.rows[0];
    void* const dw = keys ? S.dw[1] : S.dw[0];
    if (dw == nullptr) return;
    const int col = threadIdx.x % kSumCols, row = threadIdx.x / kSumCols, j = blockIdx.x * kSumCols + col;
    float v = 0.f;
    if (j < S.dim)
        for (int r = row; r < rows; r += kRows) v += partial[(size_t)r * S.dim + j];
    part[row][col] = v;
    __syncthreads();
    if (threadIdx.x < kSumCols && j < S.dim) {
        v = 0.f;
        for (int r = 0; r < kRows; ++r) v += part[r][threadIdx.x];
        if (S.weight32) static_cast<float*>(dw)[j] = v;
        else static_cast<T*>(dw)[j] = from_f<T>(v);
    }
}

}  // namespace pcr
