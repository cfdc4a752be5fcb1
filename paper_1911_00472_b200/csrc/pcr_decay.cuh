// Kernels of linear attention with a decay for each head: the plain form of a walk (see pcr_walks.h), what goes on between walks, one
// token of each request.
#pragma once
#include "pcr_walks.h"

namespace pcr {

constexpr int kWalkThreads = 256;
constexpr int kWalkCols = 64;                  // columns of c (and of R) of a CTA of the plain kernel

inline size_t walk_shared(int bd, int rows) {
    const int bdp = (bd + 3) / 4 * 4;
    return sizeof(float) * ((size_t)2 * rows * (bdp + 4) + (size_t)rows * kWalkCols + (size_t)rows * (rows + 4) + (size_t)bdp * kWalkCols + rows + 4);
}

// The plain form of a walk, in single precision from end to end: any sizes, strides and types.  256 threads, 16 x 16; a CTA has
// 64 columns of c, a chunk has kRows tokens (64; 32 where heads of more than 128 would not leave room for them).
// What bounds it: instructions (57 % of the issue slots at two CTAs of 8 warps an SM) and shared memory (54 % of its wavefronts); DRAM 6 %.  3 x 1001
// tokens, 12 heads of 64 in 32 bits, memories given and taken: 36.9 us in each of two launches, 231 with whole sequences in the place of
// segments; gradients of 2 x 257 tokens, 8 + 2 heads of 64: 21.6 us each of two, 70.5 whole.  (With fewer products a load, and a
// chunk's loads one operand after the other, the two calls took 145 and 109 us; now 85 and 57.)
template <typename T, int kRows>
__global__ void __launch_bounds__(kWalkThreads) walk_kernel(const __grid_constant__ WalkArgs A) {
    extern __shared__ float4 shared4[];
    constexpr int kPer = kRows / 16;
    const int slices = gridDim.z / A.kinds, kind = blockIdx.z / slices, slice = blockIdx.z - kind * slices;
    const Walk& W = A.w[kind];
    const int head = blockIdx.y, c0 = slice * kWalkCols;
    if (c0 >= W.cd) return;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, warp = tid >> 5, lane = tid & 31;
    if (!A.states && slice == 0) zero_tail(A, W, W.y32 ? 4 : (int)sizeof(T), blockIdx.x, gridDim.x, head, tid, kWalkThreads);
    Item it;
    if (!item_of(A, W.rev, blockIdx.x, it)) return;
    if (A.states && it.last) return;

    const int bd = W.bd, bdp = (bd + 3) / 4 * 4, ld = bdp + 4, cols = min(kWalkCols, W.cd - c0);
    float* As = reinterpret_cast<float*>(shared4);
    float* Bs = As + kRows * ld;
    float* Cs = Bs + kRows * ld;
    float* Ps = Cs + kRows * kWalkCols;
    float* Rs = Ps + kRows * (kRows + 4);
    float* pw = Rs + bdp * kWalkCols;                     // powers of the factor, 0 .. kRows
    const float rate = rate_of(A.log_decay, head);
    for (int i = tid; i <= kRows; i += kWalkThreads) pw[i] = power(rate, i);
    {
        const size_t of = (size_t)bd * W.cd;
        const float* from = nullptr;
        int64_t fi = 0, fj = 0;
        float age = 1.f;
        if (!A.states) {
            if (it.m > 0) { from = W.slots + ((size_t)(it.slot - 1) * A.heads + head) * of; fi = W.si; fj = W.sj; }
            else if (W.first) { from = W.first + ((size_t)it.seq * A.heads + head) * of; fi = W.fi; fj = W.fj; age = W.rev ? 1.f : power(rate, 1); }
        }
        for (int i = warp; i < bdp; i += 8)
            for (int j = lane; j < kWalkCols; j += 32) Rs[i * kWalkCols + j] = from && i < bd && j < cols ? age * from[i * fi + (c0 + j) * fj] : 0.f;
    }
    const T* a = static_cast<const T*>(W.a.at) + (int64_t)it.batch * W.a.st[0] + (int64_t)(head / W.a.group) * W.a.st[2];
    const T* b = static_cast<const T*>(W.b.at) + (int64_t)it.batch * W.b.st[0] + (int64_t)(head / W.b.group) * W.b.st[2];
    const T* c = static_cast<const T*>(W.c.at) + (int64_t)it.batch * W.c.st[0] + (int64_t)(head / W.c.group) * W.c.st[2] + c0;
    const int64_t y0 = (int64_t)it.batch * W.ys[0] + (int64_t)head * W.ys[2] + c0;

    for (int at = it.from; at < it.from + it.n; at += kRows) {
        const int n = min(kRows, it.from + it.n - at);
        const int64_t t0 = it.begin + (W.rev ? it.len - at - n : at);
        const bool final = it.last && at + n >= it.len && !W.rev;         // forward, the memory that is given out is not aged
        __syncthreads();                                                   // the chunk before is done with
        // 32 columns of every eighth row a warp, all three operands' on their way before the first is needed
        for (int d0 = 0; d0 < max(bdp, kWalkCols); d0 += 32) {
            constexpr int kEach = kRows / 8;
            const int d = d0 + lane;
            const bool ab = d < bd, cc = d < cols;
            T x[3][kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = warp + 8 * i;
                const bool in = r < n;
                const T none = from_float<T>(0.f);
                x[0][i] = !A.states && in && ab ? a[(t0 + r) * W.a.st[1] + d] : none;
                x[1][i] = in && ab ? b[(t0 + r) * W.b.st[1] + d] : none;
                x[2][i] = in && cc ? c[(t0 + r) * W.c.st[1] + d] : none;
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = warp + 8 * i;
                if (d < bdp) { As[r * ld + d] = to_float(x[0][i]); Bs[r * ld + d] = to_float(x[1][i]); }
                if (d < kWalkCols) Cs[r * kWalkCols + d] = to_float(x[2][i]);
            }
        }
        __syncthreads();
        if (!A.states) {
            float s[kPer][kPer] = {};
            for (int d = 0; d < bdp; d += 4) {
                float4 x[kPer], z[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) x[i] = *reinterpret_cast<const float4*>(As + (ty + 16 * i) * ld + d);
#pragma unroll
                for (int j = 0; j < kPer; ++j) z[j] = *reinterpret_cast<const float4*>(Bs + (tx + 16 * j) * ld + d);
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) s[i][j] += x[i].x * z[j].x + x[i].y * z[j].y + x[i].z * z[j].z + x[i].w * z[j].w;
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = ty + 16 * i, q = tx + 16 * j, far = W.rev ? q - r : r - q;
                    Ps[r * (kRows + 4) + q] = far >= 0 ? s[i][j] * pw[far] : 0.f;
                }
            // four rows by four columns a thread, four steps of the sum at a time: eight loads of 16 bytes for 64 products
            float o[kPer][4] = {};
            auto add = [&](const float* rows, int ld_rows, const float* with, int steps) {
#pragma unroll 2
                for (int d = 0; d < steps; d += 4) {
                    float4 m[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) m[e] = *reinterpret_cast<const float4*>(with + (d + e) * kWalkCols + 4 * tx);
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const float4 x = *reinterpret_cast<const float4*>(rows + (ty + 16 * i) * ld_rows + d);
                        o[i][0] += x.x * m[0].x + x.y * m[1].x + x.z * m[2].x + x.w * m[3].x;
                        o[i][1] += x.x * m[0].y + x.y * m[1].y + x.z * m[2].y + x.w * m[3].y;
                        o[i][2] += x.x * m[0].z + x.y * m[1].z + x.z * m[2].z + x.w * m[3].z;
                        o[i][3] += x.x * m[0].w + x.y * m[1].w + x.z * m[2].w + x.w * m[3].w;
                    }
                }
            };
            add(As, ld, Rs, bdp);
            float past[kPer][4];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = ty + 16 * i, far = W.rev ? n - 1 - r : r;
#pragma unroll
                for (int e = 0; e < 4; ++e) past[i][e] = o[i][e] = o[i][e] * (r < n ? pw[far] : 0.f);
            }
            __syncthreads();
            add(Ps, kRows + 4, Cs, kRows);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = ty + 16 * i;
                if (r >= n) continue;
                const int64_t to = y0 + (t0 + r) * W.ys[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (4 * tx + e >= cols) continue;
                    float v = o[i][e];
                    if (!isfinite(v)) {                   // a masked token that is not finite leaves no trace: 0 * inf is none
                        v = past[i][e];
                        for (int q = W.rev ? r : 0; q <= (W.rev ? n - 1 : r); ++q) v += Ps[r * (kRows + 4) + q] * Cs[q * kWalkCols + 4 * tx + e];
                    }
                    if (W.y32) static_cast<float*>(W.y)[to + 4 * tx + e] = v;
                    else static_cast<T*>(W.y)[to + 4 * tx + e] = from_float<T>(v);
                }
            }
        }
        // the memory: rows of B times their factors, then four rows by four columns of it a thread
        __syncthreads();
        for (int i = tid; i < kRows * (bdp / 4); i += kWalkThreads) {
            const int r = i / (bdp / 4);
            float4* x = reinterpret_cast<float4*>(Bs + r * ld) + (i - r * (bdp / 4));
            const float f = r < n ? pw[(W.rev ? r + 1 : n - r) - (final ? 1 : 0)] : 0.f;
            *x = make_float4(x->x * f, x->y * f, x->z * f, x->w * f);
        }
        __syncthreads();
        const float keep = power(rate, final ? n - 1 : n);
        for (int i = 4 * ty; i < bdp; i += 64) {
            float m[4][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 x = *reinterpret_cast<const float4*>(Rs + (i + e) * kWalkCols + 4 * tx);
                m[e][0] = x.x * keep; m[e][1] = x.y * keep; m[e][2] = x.z * keep; m[e][3] = x.w * keep;
            }
#pragma unroll 4
            for (int r = 0; r < n; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(Bs + r * ld + i), v = *reinterpret_cast<const float4*>(Cs + r * kWalkCols + 4 * tx);
                m[0][0] += x.x * v.x; m[0][1] += x.x * v.y; m[0][2] += x.x * v.z; m[0][3] += x.x * v.w;
                m[1][0] += x.y * v.x; m[1][1] += x.y * v.y; m[1][2] += x.y * v.z; m[1][3] += x.y * v.w;
                m[2][0] += x.z * v.x; m[2][1] += x.z * v.y; m[2][2] += x.z * v.z; m[2][3] += x.z * v.w;
                m[3][0] += x.w * v.x; m[3][1] += x.w * v.y; m[3][2] += x.w * v.z; m[3][3] += x.w * v.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) *reinterpret_cast<float4*>(Rs + (i + e) * kWalkCols + 4 * tx) = make_float4(m[e][0], m[e][1], m[e][2], m[e][3]);
        }
    }
    __syncthreads();
    float* out = nullptr;
    int64_t oi = 0, oj = 0;
    float age = 1.f;
    const size_t of = (size_t)bd * W.cd;
    if (A.states) { out = W.slots + ((size_t)it.slot * A.heads + head) * of; oi = W.si; oj = W.sj; }
    else if (it.last && W.last) {
        out = W.last + ((size_t)it.seq * A.heads + head) * of; oi = W.li; oj = W.lj;
        if (it.len == 0) {                                // the memory as it came
            for (int i = warp; i < bd; i += 8)
                for (int j = lane; j < cols; j += 32)
                    out[i * oi + (c0 + j) * oj] = W.first ? W.first[((size_t)it.seq * A.heads + head) * of + i * W.fi + (c0 + j) * W.fj] : 0.f;
            return;
        }
    }
    if (out)
        for (int i = warp; i < bd; i += 8)
            for (int j = lane; j < cols; j += 32) out[i * oi + (c0 + j) * oj] = age * Rs[i * kWalkCols + j];
}

// Along every sequence of more than one segment: what the segments add becomes the memory with which the next one begins.  A thread
// goes along with V elements of a memory, eight segments' on their way at a time.
template <int V>
__global__ void __launch_bounds__(256) walk_scan_kernel(const __grid_constant__ WalkArgs A) {
    const int blocks = gridDim.z / A.kinds, kind = blockIdx.z / blocks, block = blockIdx.z - kind * blocks, seg = (int)A.seg;
    const Walk& W = A.w[kind];
    int64_t slot = (int64_t)blockIdx.x * ((A.tokens + A.seg - 1) / A.seg - 1), len = A.tokens;
    if (A.starts) {                                        // (as item_of has it, for a sequence's first segment)
        const uint32_t i = W.rev ? A.sequences - 1 - blockIdx.x : blockIdx.x;
        const int64_t b = start_of(A, W.rev, i);
        len = start_of(A, W.rev, i + 1) - b;
        slot = b / seg;
    }
    if (len <= seg) return;
    const int more = (int)((len - 1) / seg), of = W.bd * W.cd;         // segments that have one behind them
    for (int head = blockIdx.y; head < A.heads; head += gridDim.y) {
        const float rate = rate_of(A.log_decay, head), keep = power(rate, seg), age = W.rev ? 1.f : power(rate, 1);
        const size_t step = (size_t)A.heads * of;
        const float* first = W.first ? W.first + ((size_t)blockIdx.x * A.heads + head) * of : nullptr;
        for (int e = (block * 256 + threadIdx.x) * V; e < of; e += blocks * 256 * V) {
            float* p = W.slots + ((size_t)slot * A.heads + head) * of + e;
            float m[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = W.si >= W.sj ? (e + v) / W.cd : (e + v) % W.bd, j = W.si >= W.sj ? (e + v) % W.cd : (e + v) / W.bd;
                m[v] = first ? age * first[i * W.fi + j * W.fj] : 0.f;
            }
            for (int k = 0; k < more; k += 8) {
                float x[8][V];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (k + u < more) {
                        if constexpr (V == 4) *reinterpret_cast<float4*>(x[u]) = *reinterpret_cast<const float4*>(p + (k + u) * step);
                        else x[u][0] = p[(k + u) * step];
                    }
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (k + u < more) {
#pragma unroll
                        for (int v = 0; v < V; ++v) m[v] = keep * m[v] + x[u][v];
                        if constexpr (V == 4) *reinterpret_cast<float4*>(p + (k + u) * step) = *reinterpret_cast<const float4*>(m);
                        else p[(k + u) * step] = m[0];
                    }
            }
        }
    }
}

// Gradients of keys and values that several heads share: the heads' sums, in the order of the heads.
struct GroupSum { const float* from; void* to; int64_t ts[3]; int64_t tokens, rows; int heads, group, dim; };
template <typename T>
__global__ void __launch_bounds__(256) group_sum_kernel(const __grid_constant__ GroupSum G0, const __grid_constant__ GroupSum G1, const int32_t* starts, int sequences, int zero) {
    const GroupSum& G = blockIdx.y ? G1 : G0;
    int64_t from = 0, to = G.tokens;
    if (starts) {                                          // rows of no sequence were not written
        from = min(max((int64_t)starts[0], (int64_t)0), G.tokens);
        to = max(from, min((int64_t)starts[sequences], G.tokens));
    }
    const int64_t n = G.rows * (G.heads / G.group) * G.dim;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int d = (int)(e % G.dim);
        const int64_t rest = e / G.dim;
        const int h = (int)(rest % (G.heads / G.group));
        const int64_t row = rest / (G.heads / G.group), b = row / G.tokens, t = row - b * G.tokens;
        const bool in = t >= from && t < to;
        if (!in && !zero) continue;
        float sum = 0.f;
        if (in)
            for (int g = 0; g < G.group; ++g) sum += G.from[(row * G.heads + h * G.group + g) * G.dim + d];
        static_cast<T*>(G.to)[b * G.ts[0] + t * G.ts[1] + h * G.ts[2] + d] = from_float<T>(sum);
    }
}

// ---- one token of each request ---------------------------------------------------------------------------------------------

struct StepArgs {
    const void *q, *k, *v;
    void* out;
    int64_t qs[2], ks[2], vs[2], os[2];        // row, head
    float* state;
    const int32_t* slots;                      // rows, or null: row i has memory i
    const float* log_decay;
    int rows, n_slots, q_heads, group, kd, vd, cols, splits;    // a memory's columns go to `splits` CTAs, `cols` to each
};
constexpr int kStepThreads = 256;
constexpr int kStepAhead = 4;                  // rows of the memory on their way to a thread

// A CTA has `cols` columns of a memory; a thread V of them in every (threads / lanes)-th row.  Reading and writing the memory is all
// there is to it: 8 bytes an element at the rate of the DRAM.  200 requests, 32 heads of 128 x 128: 134 us, 6.3 TB/s, 96 % of the copy rate (rows on
// their way 2: 150, 3: 142, 8: 149, 16: 207); one request's 16 heads of 64 x 64 3.1 us.
template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads) step_kernel(const __grid_constant__ StepArgs A) {
    __shared__ float qs[kMaxDecayDim], ks[kMaxDecayDim], sums[kStepThreads * V];
    __shared__ int next;
    const int row0 = blockIdx.x / A.splits, head = blockIdx.y, c0 = (blockIdx.x - row0 * A.splits) * A.cols, tid = threadIdx.x;
    const int cols = min(A.cols, A.vd - c0), lanes = A.cols / V, stripes = kStepThreads / lanes;
    const int lane = tid % lanes, stripe = tid / lanes, c = lane * V;
    const bool on = stripe < stripes && c < cols;
    const float factor = exp2f(rate_of(A.log_decay, head));
    int slot = row0, row = row0;
    if (A.slots) {
        slot = A.slots[row0];
        if (slot < 0 || slot >= A.n_slots) {              // no memory: zeros
            for (int i = tid; i < cols; i += kStepThreads) static_cast<T*>(A.out)[row0 * A.os[0] + head * A.os[1] + c0 + i] = from_float<T>(0.f);
            return;
        }
        bool earlier = false;                              // rows of one memory: the first one's CTA takes them all, one after the other
        for (int i = tid; i < row0; i += kStepThreads) earlier |= A.slots[i] == slot;
        if (__syncthreads_or(earlier)) return;
    }
    float* S = A.state + ((size_t)slot * A.q_heads + head) * A.kd * A.vd + c0;
    while (true) {
        const T* q = static_cast<const T*>(A.q) + row * A.qs[0] + head * A.qs[1];
        const T* k = static_cast<const T*>(A.k) + row * A.ks[0] + head / A.group * A.ks[1];
        const T* v = static_cast<const T*>(A.v) + row * A.vs[0] + head / A.group * A.vs[1] + c0;
        for (int i = tid; i < A.kd; i += kStepThreads) { qs[i] = to_float(q[i]); ks[i] = to_float(k[i]); }
        if (tid == 0) next = A.rows;
        float val[V], sum[V] = {};
#pragma unroll
        for (int e = 0; e < V; ++e) val[e] = on ? to_float(v[c + e]) : 0.f;
        __syncthreads();
        if (on)
            for (int i0 = stripe; i0 < A.kd; i0 += kStepAhead * stripes) {
                float m[kStepAhead][V];
#pragma unroll
                for (int u = 0; u < kStepAhead; ++u) {
                    const int i = i0 + u * stripes;
                    if (i < A.kd) {
                        if constexpr (V == 4) *reinterpret_cast<float4*>(m[u]) = *reinterpret_cast<const float4*>(S + (size_t)i * A.vd + c);
                        else m[u][0] = S[(size_t)i * A.vd + c];
                    }
                }
#pragma unroll
                for (int u = 0; u < kStepAhead; ++u) {
                    const int i = i0 + u * stripes;
                    if (i >= A.kd) continue;
#pragma unroll
                    for (int e = 0; e < V; ++e) { m[u][e] = factor * m[u][e] + ks[i] * val[e]; sum[e] += qs[i] * m[u][e]; }
                    if constexpr (V == 4) *reinterpret_cast<float4*>(S + (size_t)i * A.vd + c) = *reinterpret_cast<const float4*>(m[u]);
                    else S[(size_t)i * A.vd + c] = m[u][0];
                }
            }
        if (on)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[stripe * A.cols + c + e] = sum[e];
        if (A.slots)
            for (int i = row + 1 + tid; i < A.rows; i += kStepThreads)
                if (A.slots[i] == slot) { atomicMin(&next, i); break; }
        __syncthreads();
        for (int i = tid; i < cols; i += kStepThreads) {
            float total = 0.f;
            for (int s = 0; s < stripes; ++s) total += sums[s * A.cols + i];
            static_cast<T*>(A.out)[row * A.os[0] + head * A.os[1] + c0 + i] = from_float<T>(total);
        }
        if (!A.slots || next >= A.rows) return;
        row = next;
        __syncthreads();
    }
}

}  // namespace pcr
