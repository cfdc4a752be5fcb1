// Queries and keys turned by the positions of their tokens, with or without a root-mean-square norm of every head in
// front, and the backward pass of both together.
//
//   angle_i = position[axis_i] * inv_freq_i                    (whole turns go in 64 bits: the position may lie millions of them away)
//   turned: (a, b) -> (a cos - b sin, a sin + b cos) for the pairs (i, i + rot/2) or (2 i, 2 i + 1), i < rot/2
//   forward, norm:  y = turn(w * x * r),  r = 1 / sqrt(mean(x^2) + eps)
//   backward:       d = turn back(g),  u = x * r,  dx = r * (d * w - u * mean(d * w * u)),  dw = sum over rows of d * u
//
// All of it reads every value once and writes every value once with few operations between.  A thread holds V pairs of a row
// (two vectors of up to 16 bytes), the lanes of a row stand side by side in one warp (their sums meet in shuffles, forward
// rows never leave the registers), and a thread goes over several heads of ONE token, so that cosine and sine are worked out
// once for all of them.
//
// Measured on a B200 (6567 GB/s copied): norm and rotation of 32768 tokens, 32 + 8 heads of 128, bf16: 117 us, 5.7 TB/s, 88 % of
// the copy rate; rotation of 8191 tokens out of a packed projection, fp16: 34 us, 4.9 TB/s (1.7 rounds of CTAs, the rest is
// their end); rotation of 12003 tokens, 32 heads of 80, fp32: 43 us, 5.7 TB/s.  Backward of 8192 tokens, 40 heads of 128, bf16:
// 50 us, 5.1 TB/s, fp32: 84 us, 6.0 TB/s; of 16384 tokens, 32 heads of 72, bf16: 56.5 us, 4.0 TB/s.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stddef.h>
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
    int32_t heads, slots;         // value by value: shares of `per` heads; backward by vectors: CTAs that take this operand
};

struct HeadArgs {
    HeadBlock part[2];
    const int32_t* positions;
    int64_t ps[3];                // strides of axis, batch, token
    const void* inv_freq;
    const int32_t* axes;
    uint32_t tokens, seq;         // batch * tokens of a sequence, tokens of a sequence
    int32_t n_axes, freq64, weight32, inverse;
    int32_t dim, rot, lanes, per;   // lanes: of a row
    float eps, inv_dim;
};

// N elements as 32-bit words: two 16-bit elements are taken apart and put together in one or two instructions.
template <typename T, int N> struct alignas(sizeof(T) * N) Vec { uint32_t w[N * sizeof(T) / 4]; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void two_of(uint32_t w, float& a, float& b, __nv_bfloat16) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void two_of(uint32_t w, float& a, float& b, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x; b = f.y;
}
__device__ __forceinline__ uint32_t word_of(float a, float b, __nv_bfloat16) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ uint32_t word_of(float a, float b, __half) { const __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&v); }
template <typename T, int N> __device__ __forceinline__ void floats_of(const Vec<T, N>& v, float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __uint_as_float(v.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) two_of(v.w[i / 2], f[i], f[i + 1], T());
    }
}
template <typename T, int N> __device__ __forceinline__ Vec<T, N> vec_of(const float (&f)[N]) {
    Vec<T, N> v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) v.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) v.w[i / 2] = word_of(f[i], f[i + 1], T());
    }
    return v;
}

// 1 / (2 pi) in two parts: a product with the first alone is off by 2^-53 of its turns, and times 2^31 positions by more than
// single precision is.
constexpr double kTurns = 0x1.45f306dc9c883p-3, kTurnsRest = -0x1.6b01ec5417056p-57;

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

// The kernel that adds the weights' sums up is launched while this one runs and waits for its end.
__device__ __forceinline__ void sums_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void sums_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

enum { kTurn = 0, kNormTurn = 1, kNormTurnBack = 2 };

// How the `n` lanes of a row add up.  Where n is no power of two, sums of 1, 2, 4, ... lanes going round the row are made,
// and those that n's bits name added up: as few shuffles as for the next larger power of two, and no condition on the lane.
// `twice` and `rest` hold the lanes to take from, six bits a step.  n is the same for all lanes.
struct RowLanes {
    int n;
    bool power;
    uint32_t twice, rest;
    __device__ __forceinline__ RowLanes(int n_, int first, int at) : n(n_), power((n_ & (n_ - 1)) == 0), twice(0), rest(0) {
        auto round = [&](int o) { const int l = at + o; return (uint32_t)(first + (l < n ? l : l - n)); };
        int have = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int o = 1 << i;
            if (o < n) twice |= round(o) << (6 * i);
            if (n & o) { if (have < n) rest |= round(have) << (6 * i); have += o; }
        }
    }
};
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], const RowLanes& L) {
    if (L.power) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            if (o >= L.n) return;
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        return;
    }
    float all[N];
    bool none = true;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        if (L.n >> i & 1) {
#pragma unroll
            for (int k = 0; k < N; ++k) all[k] = none ? v[k] : all[k] + __shfl_sync(0xffffffffu, v[k], (int)(L.rest >> (6 * i)));
            none = false;
        }
        if (L.n >> (i + 1) == 0) break;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_sync(0xffffffffu, v[k], (int)(L.twice >> (6 * i)));
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = all[k];
}

// The same with the number of steps known (the backward pass, which instructions bound: 16384 tokens, heads of 72, 9 lanes: 63.6 ->
// 55.7 us; heads of 256, 16 lanes: 59.5 -> 51.4; of 128, 8 lanes: 54.7 -> 53.0; of 64, 4 lanes: 55.4 -> 53.5; 48 heads of 72 of which
// 36 are turned, 18 lanes: 109 -> 84; forward passes wait for memory and gain nothing).
// kSteps > 0: rows of 2^kSteps lanes.  kSteps < 0: of any other number below 2^-kSteps; step i adds the sum that begins 2^i
// lanes further on, which ends with the row, and the first lane's sum goes round.  32 is no multiple of such a number, so
// that the warp's last lane is free to hold 0 for what lies behind a row.  0: any number (above).
template <int kSteps> struct RowSums {
    uint32_t from;                 // lanes to take from, five bits a step
    int first;
    bool spare;
    __device__ __forceinline__ RowSums(int n, int first_, int at) : from(0), first(first_), spare((threadIdx.x & 31) == 31) {
#pragma unroll
        for (int i = 0; i < -kSteps; ++i) from |= (uint32_t)(!spare && at + (1 << i) < n ? (first + at + (1 << i)) & 31 : 31) << (5 * i);
    }
    template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) const {
        if constexpr (kSteps > 0) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], 1 << i);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = spare ? 0.f : v[k];
#pragma unroll
            for (int i = 0; i < -kSteps; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] += __shfl_sync(0xffffffffu, v[k], (int)(from >> (5 * i)));
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, v[k], first);
        }
    }
};
template <> struct RowSums<0> {
    RowLanes lanes;
    __device__ __forceinline__ RowSums(int n, int first, int at) : lanes(n, first, at) {}
    template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) const { row_sums<N>(v, lanes); }
};
// (rows of 1 and 2 lanes, heads of 4 to 32 elements, have no steps to save)
inline int steps_of(int lanes) {
    if ((lanes & (lanes - 1)) == 0) return lanes == 4 ? 2 : lanes == 8 ? 3 : lanes == 16 ? 4 : lanes == 32 ? 5 : 0;
    return lanes < 8 ? -3 : lanes < 16 ? -4 : -5;
}

// A frequency as the turns of one position, a fraction of 2^64, modulo whole turns: the product and what its rounding left out
// each lose 2^-65 (half a turn, 2^63 itself, saturates to just below).
__device__ __forceinline__ uint2 fraction_of(double freq) {
    const double t = freq * kTurns, rest = fma(freq, kTurnsRest, fma(freq, kTurns, -t));
    const unsigned long long f = (unsigned long long)__double2ll_rn((t - rint(t)) * 18446744073709551616.0) +
                                 (unsigned long long)__double2ll_rn((rest - rint(rest)) * 18446744073709551616.0);
    return make_uint2((uint32_t)f, (uint32_t)(f >> 32));
}

// What a CTA keeps for its tokens: every pair's turn for one position as a fraction of 2^64, its axis, and the weights of both
// norms, which are read as vectors of up to eight.
template <int kParts> struct alignas(32) HeadTables {          // 0 parts: no weights, 1: of one operand, 2: of both
    uint2 turn[kMaxHeadDim / 2];
    int32_t axis[kMaxHeadDim / 2];
    float w[kParts > 0 ? kParts : 1][kParts > 0 ? kMaxHeadDim : 1];
};
static_assert(alignof(HeadTables<2>) % alignof(Vec<float, 8>) == 0 && offsetof(HeadTables<2>, w) % alignof(Vec<float, 8>) == 0, "weights are read as whole vectors");

template <typename T, int kParts>
__device__ __forceinline__ void fill_tables(const HeadArgs& A, HeadTables<kParts>& S, int first) {
    for (int j = threadIdx.x; j < A.rot / 2; j += kHeadThreads) {
        S.turn[j] = fraction_of(freq_at(A, j));
        S.axis[j] = A.axes[j];
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const void* w = A.part[first + k].weight;
        for (int j = threadIdx.x; j < A.dim; j += kHeadThreads) S.w[k][j] = w != nullptr ? weight_of<T>(A, w, j) : 1.f;
    }
}

// cosine and sine of a position's turn.  The product of the position and the 64-bit fraction is taken modulo 2^64, that is
// modulo whole turns: exact but for the fraction's own rounding (2^-64 turns a position for frequencies up to 2^40), however far
// the position.  The upper 32 bits are kept (2^-32 turns: 1.5e-9 of an angle).  16-bit results take the hardware's sine and cosine, off by
// 2^-21.19 at most, where the result itself is rounded to 2^-8 or 2^-11 of its value: 5 instructions in the place of about 40.
template <typename T>
__device__ __forceinline__ void turn_by(int32_t position, uint2 turn, bool inverse, float& c, float& s) {
    const uint32_t p = (uint32_t)position;
    uint32_t hi = __umulhi(p, turn.x) + p * turn.y;
    if (position < 0) hi -= turn.x;                                          // p is position + 2^32 there
    const float half_turns = (float)(int32_t)hi * 4.656612873077393e-10f;    // 2^-31
    if (sizeof(T) == 2) __sincosf(half_turns * 3.14159265358979f, &s, &c);
    else sincospif(half_turns, &s, &c);
    if (inverse) s = -s;
}

// Where the lanes of a warp stand: number `at` of a row, which of the warp's rows, and where the lane's two vectors of V
// elements begin in a head (`gap` elements apart).
template <int V, bool kNext> struct Place {
    int rows, sub, at, o1, gap, pair;
    bool in_row, turns;
    __device__ __forceinline__ explicit Place(const HeadArgs& A) {
        const int lane = threadIdx.x & 31, turning = A.rot / (2 * V);
        rows = 32 / A.lanes; sub = lane / A.lanes; at = lane - sub * A.lanes;
        in_row = sub < rows; turns = at < turning; pair = at * V;
        o1 = kNext ? 2 * V * at : turns ? pair : A.rot + 2 * V * (at - turning);
        gap = kNext || !turns ? V : A.rot / 2;
    }
    template <typename Sums> __device__ __forceinline__ Sums row_sums_of(const HeadArgs& A) const { return Sums(A.lanes, sub * A.lanes, at); }
};

// The elements that make pair i: of the first and of the second vector, or 2 i and 2 i + 1 of both together.
template <int V, bool kNext> __device__ __forceinline__ float& one(float (&p)[V], float (&q)[V], int i) {
    return kNext ? (2 * i < V ? p[(2 * i) % V] : q[(2 * i) % V]) : p[i];
}
template <int V, bool kNext> __device__ __forceinline__ float& two(float (&p)[V], float (&q)[V], int i) {
    return kNext ? (2 * i < V ? p[(2 * i + 1) % V] : q[(2 * i + 1) % V]) : q[i];
}

// Two single-precision numbers in one register pair; the operations below take both in one instruction.
using F2 = unsigned long long;
__device__ __forceinline__ F2 pack2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(F2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// A lane's part of a row: as it lies in memory, and as pairs two by two, first elements in a, second ones in b.
template <typename T, int V> struct Row { Vec<T, V> a, b; };
template <int V> struct Pairs { F2 a[V / 2], b[V / 2]; };

template <typename T, int V>
__device__ __forceinline__ Row<T, V> load_row(const T* x, int gap) {
    return {*reinterpret_cast<const Vec<T, V>*>(x), *reinterpret_cast<const Vec<T, V>*>(x + gap)};
}
template <typename T, int V>
__device__ __forceinline__ void store_row(T* y, int gap, const Row<T, V>& r) {
    *reinterpret_cast<Vec<T, V>*>(y) = r.a;
    *reinterpret_cast<Vec<T, V>*>(y + gap) = r.b;
}
template <typename T, int V, bool kNext>
__device__ __forceinline__ Pairs<V> pairs_of(const Row<T, V>& row) {
    float f[V], g[V];
    floats_of(row.a, f);
    floats_of(row.b, g);
    Pairs<V> r;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        r.a[i / 2] = pack2(one<V, kNext>(f, g, i), one<V, kNext>(f, g, i + 1));
        r.b[i / 2] = pack2(two<V, kNext>(f, g, i), two<V, kNext>(f, g, i + 1));
    }
    return r;
}
template <typename T, int V, bool kNext>
__device__ __forceinline__ Row<T, V> row_of(const Pairs<V>& p) {
    float f[V], g[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        unpack2(p.a[i / 2], one<V, kNext>(f, g, i), one<V, kNext>(f, g, i + 1));
        unpack2(p.b[i / 2], two<V, kNext>(f, g, i), two<V, kNext>(f, g, i + 1));
    }
    return {vec_of<T, V>(f), vec_of<T, V>(g)};
}
template <int V, bool kNext>
__device__ __forceinline__ Pairs<V> weights_of(const float* w, const Place<V, kNext>& at) {
    return pairs_of<float, V, kNext>(load_row<float, V>(w + at.o1, at.gap));
}
// cosine and sine of the lane's pairs at a token's positions
template <typename T, int V, bool kNext, int kParts>
__device__ __forceinline__ void turns_of(const HeadArgs& A, const HeadTables<kParts>& S, const int32_t (&p)[kMaxAxes], const Place<V, kNext>& at, F2 (&c)[V / 2], F2 (&s)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        float fc[2] = {1.f, 1.f}, fs[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (at.turns) turn_by<T>(on_axis(p, S.axis[at.pair + i + j]), S.turn[at.pair + i + j], A.inverse, fc[j], fs[j]);
        c[i / 2] = pack2(fc[0], fc[1]); s[i / 2] = pack2(fs[0], fs[1]);
    }
}
__device__ __forceinline__ F2 negative(F2 v) { return v ^ 0x8000000080000000ull; }
__device__ __forceinline__ void soon(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }

constexpr int kRowsAhead = 4;
// Forward: grid (token groups, shares of `per` heads of queries and keys in a row).  A warp takes 32 / lanes tokens, a
// thread `per` heads of its token, kAhead of them at a time.  Lanes without a token go along with the last one's data and
// store nothing: no shuffle and no load stands in a branch.
// HBM bounds it (32768 tokens, 40 heads of 128, bf16: DRAM 72 % busy, instructions issued in 36 % of the cycles, 7.8 of 12 stalled
// warps wait for loads).  Four rows ahead and five CTAs an SM: two ahead take 123 us in the place of 116, six CTAs 127; rows handed
// on in registers while the next are on their way 128 to 160; a loop over tokens in a CTA, whose tables then serve longer, 140.
// With 16-byte vectors registers are spilled all the same: 228 bytes a thread at five CTAs with the norm in 16 bits (12 to 72 in
// 32), 64 to 72 at the rotation's six (20 to 48 in 32); shorter vectors spill nothing.
template <typename T, int V, bool kNorm, bool kNext>
__global__ void __launch_bounds__(kHeadThreads, kNorm ? 5 : 6) heads_kernel(const __grid_constant__ HeadArgs A) {
    constexpr int kWarps = kHeadThreads / 32, kAhead = kRowsAhead, N = V / 2;
    __shared__ HeadTables<kNorm ? 2 : 0> S;
    const Place<V, kNext> at(A);
    const uint32_t n0 = (blockIdx.x * kWarps + (threadIdx.x >> 5)) * (uint32_t)at.rows + (uint32_t)at.sub;
    const bool live = at.in_row && n0 < A.tokens;
    const uint32_t n = min(n0, A.tokens - 1), b = n / A.seq, t = n - b * A.seq;
    const int from = (int)blockIdx.y * A.per, to = from + A.per;
    int which = from < A.part[0].heads ? 0 : 1;
    {   // the first row is on its way while the tables are filled
        const HeadBlock& H = A.part[which];
        const T* x = static_cast<const T*>(H.x) + (int64_t)b * H.xs[0] + (int64_t)t * H.xs[1] + (int64_t)(from - (which ? A.part[0].heads : 0)) * H.xs[2] + at.o1;
        soon(x); soon(x + at.gap);
    }
    int32_t p[kMaxAxes];
    positions_of(A, b, t, p);
    fill_tables<T>(A, S, 0);
    __syncthreads();
    const auto lanes = at.template row_sums_of<RowLanes>(A);
    F2 c[N], s[N];
    turns_of<T, V, kNext>(A, S, p, at, c, s);
#pragma unroll 1
    for (; which < 2; ++which) {
        const HeadBlock& H = A.part[which];
        const int base = which ? A.part[0].heads : 0;
        const int h0 = max(from - base, 0), h1 = min(to - base, H.heads);
        if (h0 >= h1) continue;
        // a' = a wa c + b (-wb s), b' = a wa s + b wb c: four factors a pair, the same for all heads
        F2 ac[N], as[N], bc[N], bs[N];
        {
            Pairs<V> w;
            if (kNorm) w = weights_of<V, kNext>(S.w[kNorm ? which : 0], at);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ac[i] = kNorm ? mul2(w.a[i], c[i]) : c[i]; as[i] = kNorm ? mul2(w.a[i], s[i]) : s[i];
                bc[i] = kNorm ? mul2(w.b[i], c[i]) : c[i]; bs[i] = negative(kNorm ? mul2(w.b[i], s[i]) : s[i]);
            }
        }
        const int64_t xs = H.xs[2], ys = H.ys[2];
        const T* x = static_cast<const T*>(H.x) + (int64_t)b * H.xs[0] + (int64_t)t * H.xs[1] + h0 * xs + at.o1;
        T* y = static_cast<T*>(H.y) + (int64_t)b * H.ys[0] + (int64_t)t * H.ys[1] + h0 * ys + at.o1;
        auto work = [&](const Row<T, V>& row) {
            Pairs<V> v = pairs_of<T, V, kNext>(row);
            if (kNorm) {
                F2 sq = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) { sq = fma2(v.a[i], v.a[i], sq); sq = fma2(v.b[i], v.b[i], sq); }
                float sum[1], other;
                unpack2(sq, sum[0], other);
                sum[0] += other;
                row_sums<1>(sum, lanes);
                const float r = rsqrtf(sum[0] * A.inv_dim + A.eps);
                const F2 r2 = pack2(r, r);
#pragma unroll
                for (int i = 0; i < N; ++i) { v.a[i] = mul2(v.a[i], r2); v.b[i] = mul2(v.b[i], r2); }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const F2 u = fma2(v.b[i], bs[i], mul2(v.a[i], ac[i])), e = fma2(v.b[i], bc[i], mul2(v.a[i], as[i]));
                v.a[i] = u; v.b[i] = e;
            }
            if (live) store_row<T, V>(y, at.gap, row_of<T, V, kNext>(v));
            y += ys;
        };
        int h = h0;
#pragma unroll 1
        for (; h + kAhead <= h1; h += kAhead) {
            Row<T, V> rows[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k, x += xs) rows[k] = load_row<T, V>(x, at.gap);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) work(rows[k]);
        }
        if (h < h1) {                              // (the bounds are the same for the whole CTA)
            Row<T, V> rows[kAhead - 1];
#pragma unroll
            for (int k = 0; k < kAhead - 1; ++k, x += xs)
                if (h + k < h1) rows[k] = load_row<T, V>(x, at.gap);
#pragma unroll
            for (int k = 0; k < kAhead - 1; ++k)
                if (h + k < h1) work(rows[k]);
        }
    }
}

// Copies of N bytes to shared memory that the thread does not wait for, and the wait for all but the newest `kLeft` groups.
template <int N> __device__ __forceinline__ void copy_soon(uint32_t to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(N) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Backward: the first part[0].slots CTAs take the queries, the others the keys, in turn each share of `per` heads; a warp
// goes round the tokens and over its heads of each, so that the sums for the weights stay in registers to the end.
//   q = d a, dot = sum of q w, dw += q r, dx = r (d w - a r^2 dot / dim)
// Two operands, their factors and the sums leave no registers for rows on their way.  So every lane has a ring of kStages
// groups of rows in shared memory that it alone fills and reads: no barrier, and kStages - 1 groups are always on their way
// (three stages in the place of four: 57.5 us in the place of 52 for 8192 tokens, 40 heads of 128).
// With vectors of 16 bytes three CTAs an SM keep everything in registers (four: 59.5 us in the place of 52), with shorter ones
// four (16384 tokens, 32 heads of 72: 55.5 us, three 59.5, five 66).  What bounds it there: the lines that rows of odd sizes touch
// in L1 and the sums' shuffles (77 % busy) and instructions (56 % of the issue slots, 15 warps an SM whose rows are chains of
// dependent steps), not HBM (43 %).  Lanes with three chunks of a row each (105 us in the place of 64 at the time) and whole
// tokens copied to shared memory first (68 to 84) were slower.
__host__ __device__ constexpr int kBackCtas(int vector_bytes) { return vector_bytes >= 16 ? 3 : 4; }      // of an SM: what the registers leave room for
template <typename T, int V, bool kNext, int kSteps>
__global__ void __launch_bounds__(kHeadThreads, kBackCtas(V * sizeof(T))) heads_back_kernel(const __grid_constant__ HeadArgs A) {
    constexpr int kWarps = kHeadThreads / 32, kBytes = V * (int)sizeof(T), kGroup = kBytes >= 16 ? 1 : 2, kStages = 4, N = V / 2;
    using VT = Vec<T, V>;
    struct Stage { VT rows[kGroup][4][32]; int32_t positions[kMaxAxes][32]; };
    __shared__ HeadTables<1> S;
    __shared__ union { Stage ring[kWarps][kStages]; float sums[kWarps][kMaxHeadDim]; } U;
    const int which = (int)blockIdx.x >= A.part[0].slots ? 1 : 0, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const HeadBlock& H = A.part[which];
    const uint32_t mine = blockIdx.x - (which ? (uint32_t)A.part[0].slots : 0u);
    const Place<V, kNext> at(A);
    const uint32_t shares = (uint32_t)(H.heads + A.per - 1) / (uint32_t)A.per, group = mine / shares;
    const int h0 = (int)(mine - group * shares) * A.per, heads = min(A.per, H.heads - h0);
    const int64_t xs = H.xs[2], gs = H.gs[2], ys = H.ys[2];
    const uint32_t step = (uint32_t)H.slots / shares * (uint32_t)(kWarps * at.rows), begin = (group * kWarps + warp) * (uint32_t)at.rows;     // (sums of tokens and steps fit)
    auto token_of = [&](uint32_t base, uint32_t& b, uint32_t& t) {        // lanes without one go along with the last
        const uint32_t n = min(base + at.sub, A.tokens - 1);
        b = n / A.seq; t = n - b * A.seq;
    };

    // the side that fills
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(&U.ring[warp][0]) + lane * kBytes, ring_end = ring + kStages * (uint32_t)sizeof(Stage);
    uint32_t fbase = begin, fat = ring;
    int fhead = 0;
    const T *fx = nullptr, *fg = nullptr;
    auto fill = [&]() {
        if (fbase < A.tokens) {
            if (fhead == 0) {
                uint32_t b, t;
                token_of(fbase, b, t);
                fx = static_cast<const T*>(H.x) + (int64_t)b * H.xs[0] + (int64_t)t * H.xs[1] + h0 * xs + at.o1;
                fg = static_cast<const T*>(H.g) + (int64_t)b * H.gs[0] + (int64_t)t * H.gs[1] + h0 * gs + at.o1;
                const int32_t* p = A.positions + (int64_t)b * A.ps[1] + (int64_t)t * A.ps[2];
                const uint32_t to = fat + (uint32_t)offsetof(Stage, positions) + lane * (4 - kBytes);
#pragma unroll
                for (int a = 0; a < kMaxAxes; ++a)
                    if (a < A.n_axes) copy_soon<4>(to + a * 128, p + (int64_t)a * A.ps[0]);
            }
#pragma unroll
            for (int m = 0; m < kGroup; ++m, fx += xs, fg += gs)
                if (m == 0 || fhead + m < heads) {
                    const uint32_t to = fat + m * 4 * 32 * kBytes;
                    copy_soon<kBytes>(to, fx); copy_soon<kBytes>(to + 32 * kBytes, fx + at.gap);
                    copy_soon<kBytes>(to + 64 * kBytes, fg); copy_soon<kBytes>(to + 96 * kBytes, fg + at.gap);
                }
            fhead += kGroup;
            if (fhead >= heads) { fhead = 0; fbase += step; }
        }
        fat += (uint32_t)sizeof(Stage);
        if (fat == ring_end) fat = ring;
        copies_close();
    };
#pragma unroll 1
    for (int k = 0; k < kStages - 1; ++k) fill();
    fill_tables<T>(A, S, which);
    __syncthreads();
    const auto add_up = at.template row_sums_of<RowSums<kSteps>>(A);
    const Pairs<V> w = weights_of<V, kNext>(S.w[0], at);
    Pairs<V> dw;
#pragma unroll
    for (int i = 0; i < N; ++i) dw.a[i] = dw.b[i] = 0;
    int stage = 0;
#pragma unroll 1
    for (uint32_t base = begin; base < A.tokens; base += step) {
        const bool live = at.in_row && base + at.sub < A.tokens;
        uint32_t b, t;
        token_of(base, b, t);
        T* y = static_cast<T*>(H.y) + (int64_t)b * H.ys[0] + (int64_t)t * H.ys[1] + h0 * ys + at.o1;
        F2 c[N], s[N];
#pragma unroll 1
        for (int h = 0; h < heads; h += kGroup) {
            copies_wait<kStages - 2>();
            const Stage& from = U.ring[warp][stage];
            if (h == 0) {
                int32_t p[kMaxAxes];
#pragma unroll
                for (int a = 0; a < kMaxAxes; ++a) p[a] = a < A.n_axes ? from.positions[a][lane] : 0;
                turns_of<T, V, kNext>(A, S, p, at, c, s);
            }
            auto work = [&](int m) {
                const Pairs<V> x2 = pairs_of<T, V, kNext>(Row<T, V>{from.rows[m][0][lane], from.rows[m][1][lane]});
                Pairs<V> d = pairs_of<T, V, kNext>(Row<T, V>{from.rows[m][2][lane], from.rows[m][3][lane]}), q;
                const F2 minus = pack2(-1.f, -1.f);
                F2 sq = 0, dot = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const F2 u = fma2(d.b[i], s[i], mul2(d.a[i], c[i])), v = fma2(mul2(d.a[i], s[i]), minus, mul2(d.b[i], c[i]));
                    q.a[i] = mul2(u, x2.a[i]); q.b[i] = mul2(v, x2.b[i]);
                    sq = fma2(x2.a[i], x2.a[i], sq); sq = fma2(x2.b[i], x2.b[i], sq);
                    dot = fma2(q.a[i], w.a[i], dot); dot = fma2(q.b[i], w.b[i], dot);
                    d.a[i] = mul2(u, w.a[i]); d.b[i] = mul2(v, w.b[i]);
                }
                float sum[2], other[2];
                unpack2(sq, sum[0], other[0]); unpack2(dot, sum[1], other[1]);
                sum[0] += other[0]; sum[1] += other[1];
                add_up(sum);
                const float r = rsqrtf(sum[0] * A.inv_dim + A.eps), m1 = -(sum[1] * r * A.inv_dim * r);
                const F2 r2 = pack2(r, r), m2 = pack2(m1, m1);
#pragma unroll
                for (int i = 0; i < N; ++i) { d.a[i] = mul2(fma2(x2.a[i], m2, d.a[i]), r2); d.b[i] = mul2(fma2(x2.b[i], m2, d.b[i]), r2); }
                if (live) {
#pragma unroll
                    for (int i = 0; i < N; ++i) { dw.a[i] = fma2(q.a[i], r2, dw.a[i]); dw.b[i] = fma2(q.b[i], r2, dw.b[i]); }
                    store_row<T, V>(y, at.gap, row_of<T, V, kNext>(d));
                }
                y += ys;
            };
            if (kGroup == 2 && h + 2 <= heads) { work(0); work(kGroup - 1); }
            else work(0);
            stage = stage + 1 == kStages ? 0 : stage + 1;
            fill();
        }
    }
    copies_wait<0>();
    sums_may_start();
    if (H.partial == nullptr) return;                           // (the same for the whole CTA)
    __syncthreads();                                            // the rings make room for the sums
    // the rows of a warp in the order of their lanes, then the warps in theirs
    const Row<float, V> row_dw = row_of<float, V, kNext>(dw);
    float dw1[V], dw2[V];
    floats_of(row_dw.a, dw1);
    floats_of(row_dw.b, dw2);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float p = dw1[i], q = dw2[i];
        for (int m = 1; m < at.rows; ++m) {
            const int from = at.at + m * A.lanes;
            p += __shfl_sync(0xffffffffu, dw1[i], from); q += __shfl_sync(0xffffffffu, dw2[i], from);
        }
        if (at.sub == 0) { U.sums[warp][at.o1 + i] = p; U.sums[warp][at.o1 + at.gap + i] = q; }
    }
    __syncthreads();
    float* out = H.partial + (size_t)mine * A.dim;
    for (int j = threadIdx.x; j < A.dim; j += kHeadThreads) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) v += U.sums[k][j];
        out[j] = v;
    }
}

// Heads of any even or odd size, any alignment and any strides: a warp a token, lanes over pairs, then over what is not
// turned, value by value.  Bound by its instructions and single loads: 8192 tokens, 40 heads of 128, bf16, off by one element, take
// 97 us (rotation), 127 (norm), 384 (backward), where whole vectors take 29, 32 and 51.  Turns are the vector kernels', out of a
// table (worked out in 64-bit floating point for every pair, with what its roundings left out: 110, 137 and 438).
template <typename T, int kMode, bool kNext>
__global__ void __launch_bounds__(kHeadThreads) heads_any_kernel(const __grid_constant__ HeadArgs A) {
    constexpr int kWarps = kHeadThreads / 32;
    __shared__ HeadTables<0> S;
    __shared__ float sums[kMode == kNormTurnBack ? kWarps : 1][kMode == kNormTurnBack ? kMaxHeadDim : 1];
    const int which = (int)blockIdx.y >= A.part[0].slots ? 1 : 0;
    const HeadBlock& H = A.part[which];
    const int slot = (int)blockIdx.y - (which ? A.part[0].slots : 0);
    const int h0 = slot * A.per, h1 = min(h0 + A.per, H.heads);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int half = A.rot / 2;
    fill_tables<T>(A, S, 0);
    if (kMode == kNormTurnBack)
        for (int j = lane; j < A.dim; j += 32) sums[warp][j] = 0.f;          // (a lane keeps to elements of its own, but for this)
    __syncthreads();
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
                        turn_by<float>(on_axis(p, S.axis[i]), S.turn[i], false, c, s);
                        const float ga = to_f(g[ja]), gb = to_f(g[jb]);
                        dot += (ga * c + gb * s) * weight(ja) * to_f(x[ja]) + (gb * c - ga * s) * weight(jb) * to_f(x[jb]);
                    }
                    for (int j = A.rot + lane; j < A.dim; j += 32) dot += to_f(g[j]) * weight(j) * to_f(x[j]);
                }
                float sum[2] = {sq, dot};
                row_sums<2>(sum, RowLanes(32, 0, lane));
                r = rsqrtf(sum[0] * A.inv_dim + A.eps);
                m = sum[1] * r * A.inv_dim;
            }
            for (int i = lane; i < half; i += 32) {
                const int ja = kNext ? 2 * i : i, jb = kNext ? 2 * i + 1 : i + half;
                float c, s;
                turn_by<float>(on_axis(p, S.axis[i]), S.turn[i], A.inverse, c, s);
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

// dw of queries (blockIdx.y 0) and keys (1): the rows of partial sums (one a CTA of the backward pass: some hundred kilobytes, out
// of L2) added up, eight columns a CTA, always in the same order.  Nothing but latency: it is launched while the backward
// pass still runs.
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
    sums_wait();
    if (dw == nullptr) return;
    const int col = threadIdx.x % kSumCols, row = threadIdx.x / kSumCols, j = blockIdx.x * kSumCols + col;
    float v = 0.f;
    if (j < S.dim) {
#pragma unroll 8
        for (int r = row; r < rows; r += kRows) v += partial[(size_t)r * S.dim + j];
    }
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
