// Linear attention whose memory fades at a rate of each head's own (see include/pcr.h).
//
//   S_t = f S_(t-1) + k_t v_t^T,   o_t = S_t^T q_t,   f = exp(log_decay)
//
// written out: o_t = sum over j <= t of f^(t-j) (q_t . k_j) v_j.  All three gradients are sums of the same form over other
// operands, so that one kernel, a walk, does the forward and the backward pass:
//
//   y_t = sum over j of f^|t-j| (a_t . b_j) c_j      j <= t: out (a, b, c = q, k, v), dq (dout, v, k)
//                                                    j >= t: dk (v, dout, q), dv (k, q, dout)
//
// A walk goes over a sequence in chunks.  Within a chunk the sum is a product of two matrices, (A B^T, faded and masked) C; what
// lies before comes out of the memory R = sum f^(...) b_j c_j^T, which every chunk brings up to date.  Long sequences are cut into
// segments that CTAs take side by side: a first launch works out what each segment adds to the memory (`states`), a
// second adds those up along the sequence, and the walk proper begins each segment with the memory before it.
//
// "Before" and "along" are meant in the direction of the walk (`rev`: from the last token to the first); segments are cut from
// the end at which it begins, so that all but a sequence's last one are whole.  R is kept aged: what R holds counts with f^0 for the
// nearest token of the next chunk.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace pcr {

constexpr int kMaxDecayDim = 256;              // of a head, keys and values
constexpr uint32_t kPatience = 2000000000u;    // nanoseconds that a wait goes on at most

struct WalkRows { const void* at; int64_t st[3]; int group; };       // batch, token, head; `group` heads of the walk share one of these

struct Walk {
    WalkRows a, b, c;
    void* y;
    int64_t ys[3];
    const float* first;                        // the memory before: element (i, j) of (sequence, head) at (...) bd cd + i fi + j fj
    float* last;                               // the memory behind the last token
    float* slots;                              // memories of segments: element (i, j) of (slot, head) at (...) bd cd + i si + j sj
    int64_t fi, fj, li, lj, si, sj;
    int bd, cd;                                // size of a's and b's heads, and of c's and y's
    int rev, y32, wide, zero_tail;             // y32: y is in 32 bits whatever the operands are; wide: 16-bit rows of y begin at 32 bytes
};

struct WalkArgs {
    Walk w[3];
    const float* log_decay;
    const int32_t* starts;                     // sequences + 1, or null: every batch is one of `tokens`
    uint32_t sequences, tokens, seg;           // tokens of a segment: a multiple of the chunk
    int heads, kinds, states;                  // states: only what segments add
    uint32_t limit, stop;                      // nanoseconds of a wait; chunks after which a CTA's copies of tiles stop (for tests of waits that run out)
};

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v) { return (T)v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// log2 of a head's factor; one of 0 (log_decay of minus infinity) is taken as 2^-15000, so that its power 0 is 1
__device__ __forceinline__ float rate_of(const float* log_decay, int head) {
    const float r = log_decay[head] * 1.4426950408889634f;
    return r < -15000.f ? -15000.f : r;
}
__device__ __forceinline__ float power(float rate, int n) { return exp2f(rate * (float)n); }

// What a CTA is to do: segment m of a sequence.  `begin`, `len`: the sequence in memory; `from`, `n`: the segment, counted from where
// the walk begins.
struct Item { int batch, seq, m, begin, len, from, n, slot; bool last; };

// Where sequence i of those in the walk's order begins, counted in its direction.  Values outside 0 .. tokens are taken as the nearest.
__device__ __forceinline__ int64_t start_of(const WalkArgs& A, int rev, uint32_t i) {
    const int32_t v = __ldg(A.starts + (rev ? A.sequences - i : i));
    const int64_t t = min(max((int64_t)v, (int64_t)0), (int64_t)A.tokens);
    return rev ? (int64_t)A.tokens - t : t;
}

// Segments are numbered without gaps that could not be found again: segment m of sequence s, which begins at b, has the key
// s + floor((b + m seg) / seg) = s + floor(b / seg) + m, and keys grow from each segment to the next.  Called by whole warps.
__device__ __forceinline__ bool item_of(const WalkArgs& A, int rev, uint32_t key, Item& it) {
    const int seg = (int)A.seg;
    if (!A.starts) {
        const uint32_t per = max(1u, (A.tokens + A.seg - 1) / A.seg);
        it.batch = it.seq = (int)(key / per);
        it.m = (int)(key - (uint32_t)it.seq * per);
        it.begin = 0; it.len = (int)A.tokens;
        it.slot = it.seq * (int)(per - 1) + it.m;
    } else {
        if (A.sequences == 0) return false;
        // the last sequence whose first key is not beyond `key`: 32 tries at a time
        const int lane = threadIdx.x & 31;
        uint32_t lo = 0, count = A.sequences;
        while (count > 1) {
            const uint32_t step = (count + 31) / 32, at = min((uint32_t)lane * step, count - 1);
            const bool below = (uint32_t)(lo + at) + (uint64_t)start_of(A, rev, lo + at) / A.seg <= key;
            const int n = max(1, __popc(__ballot_sync(~0u, below)));         // (lane 0 holds lo itself)
            const uint32_t skip = min((uint32_t)(n - 1) * step, count - 1);
            lo += skip; count = min(step, count - skip);
        }
        const int64_t b = start_of(A, rev, lo), e = start_of(A, rev, lo + 1);
        const int64_t m = (int64_t)key - lo - b / seg;
        it.len = (int)max(e - b, (int64_t)0);
        if (m < 0 || (m > 0 && m * seg >= it.len)) return false;
        it.m = (int)m;
        it.seq = (int)(rev ? A.sequences - 1 - lo : lo);
        it.batch = 0;
        it.begin = (int)(rev ? (int64_t)A.tokens - b - it.len : b);
        it.slot = (int)((b + m * seg) / seg);
    }
    it.from = it.m * seg;
    it.n = min(seg, it.len - it.from);
    it.last = it.from + it.n >= it.len;
    return true;
}

// Rows that no sequence holds, in an output that has to be whole: zeros.
__device__ __forceinline__ void zero_tail(const WalkArgs& A, const Walk& W, int es, uint32_t cta, uint32_t ctas, int head, int thread, int threads) {
    if (!A.starts || !W.zero_tail) return;
    const int64_t from = min(max((int64_t)__ldg(A.starts), (int64_t)0), (int64_t)A.tokens);
    const int64_t to = max(from, min((int64_t)__ldg(A.starts + A.sequences), (int64_t)A.tokens));
    const int64_t rows = from + (int64_t)A.tokens - to;
    for (int64_t r = cta; r < rows; r += ctas) {
        const int64_t at = (r < from ? r : r - from + to) * W.ys[1] + (int64_t)head * W.ys[2];
        for (int c = thread; c < W.cd; c += threads) {
            if (es == 4) static_cast<float*>(W.y)[at + c] = 0.f;
            else static_cast<uint16_t*>(W.y)[at + c] = 0;
        }
    }
}

}  // namespace pcr
