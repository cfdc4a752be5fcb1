// From decoded pixels to the tokens of a sequence model: patches of images at their own sizes, and the positions of
// packed sequences of text and image or clip grids.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "pcr_heads.cuh"

namespace pcr {

constexpr int kMaxPatch = 32;
constexpr int kPatchWarps = 4;
constexpr int64_t kMaxSide = 1 << 20;         // pixels of an image's side and of a resampled side

// A row of the image table; ten 64-bit integers.
struct PatchImage { int64_t offset, width, height, x0, y0, w, h, rows, cols, flip; };

struct PatchArgs {
    const uint8_t* rgb;
    const PatchImage* images;
    const int2* index;             // (image, patch inside it) of every token
    void* out;
    uint64_t rgb_bytes;
    uint32_t n_tokens;
    int32_t n_images, patch, merge;
    float scale[3], shift[3];      // (v / 255 - mean) / std = v * scale + shift
};

// Bilinear taps with half-pixel centres: the source coordinate (o + 1/2) side / out - 1/2 as a whole number over 2 out,
// so that where it falls between pixels is exact whatever the sizes.
struct Tap { int32_t lo; float f; };
__device__ __forceinline__ Tap tap_of(int32_t o, int32_t out, int32_t side) {
    Tap t;
    if ((int64_t)out * side < (1 << 29)) {
        const int32_t den = 2 * out;
        const int32_t num = min(max((2 * o + 1) * side - out, 0), (side - 1) * den);
        t.lo = (int32_t)((uint32_t)num / (uint32_t)den);
        t.f = __fdividef((float)(num - t.lo * den), (float)den);         // (off by 2 units in the last place at most)
    } else {
        const int64_t den = 2 * (int64_t)out;
        const int64_t num = min(max((2 * (int64_t)o + 1) * side - out, (int64_t)0), (side - 1) * den);
        t.lo = (int32_t)(num / den);
        t.f = __fdividef((float)(num - t.lo * den), (float)den);
    }
    return t;
}

// Whether a token's entry stands for a patch of pixels that are there.
__device__ __forceinline__ bool patch_ok(const PatchArgs& A, const PatchImage& m, int32_t local) {
    const int64_t most = kMaxSide / A.patch;
    if (m.width < 1 || m.width > kMaxSide || m.height < 1 || m.height > kMaxSide || m.offset < 0 || m.rows < 1 || m.cols < 1 || m.rows > most || m.cols > most) return false;
    const int32_t rows = (int32_t)m.rows, cols = (int32_t)m.cols;
    return (uint64_t)m.offset <= A.rgb_bytes && (uint64_t)(3 * m.width * m.height) <= A.rgb_bytes - (uint64_t)m.offset &&
           m.x0 >= 0 && m.y0 >= 0 && m.w >= 1 && m.h >= 1 && m.w <= m.width && m.h <= m.height && m.x0 <= m.width - m.w &&
           m.y0 <= m.height - m.h && rows % A.merge == 0 && cols % A.merge == 0 && (m.flip == 0 || m.flip == 1) && local >= 0 &&
           local < m.rows * m.cols;
}

// Bytes become floats as 2^23 + byte, exactly; differences need no more, what is added to has the 2^23 taken off.
__device__ __forceinline__ float byte_up(uint32_t word, int i) { return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440u | (uint32_t)i)); }
constexpr float kUp = 8388608.f;

struct Rgb { F2 rg; float b; };

// The pixel whose bytes are the lowest three of `lo` mixed with the next one (fourth byte of `lo`, two of `hi`).
__device__ __forceinline__ Rgb mix_bytes(uint32_t lo, uint32_t hi, float f) {
    const F2 a = pack2(byte_up(lo, 0), byte_up(lo, 1)), e = pack2(byte_up(lo, 3), byte_up(hi, 0));
    const float ab = byte_up(lo, 2), eb = byte_up(hi, 1);
    return {fma2(pack2(f, f), fma2(a, pack2(-1.f, -1.f), e), fma2(a, pack2(1.f, 1.f), pack2(-kUp, -kUp))), fmaf(f, eb - ab, ab - kUp)};
}
// ... read as aligned words, which have to lie inside the buffer
__device__ __forceinline__ Rgb mix_words(const uint8_t* at, float f) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)3);
    const uint32_t sh = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 3) * 8, w0 = __ldg(p), w1 = __ldg(p + 1);
    uint32_t w2 = 0;
    if (sh == 24) w2 = __ldg(p + 2);
    return mix_bytes(__funnelshift_r(w0, w1, sh), __funnelshift_r(w1, w2, sh), f);
}
// ... byte by byte, the next pixel only where it counts: it may lie behind the last one
__device__ __forceinline__ Rgb mix_single(const uint8_t* at, float f) {
    uint32_t lo = at[0] | (uint32_t)at[1] << 8 | (uint32_t)at[2] << 16, hi = 0;
    if (f != 0.f) { lo |= (uint32_t)at[3] << 24; hi = at[4] | (uint32_t)at[5] << 8; }
    return mix_bytes(lo, hi, f);
}

// A lane a column of a patch, walking down its rows: a source row that serves two output rows is read and mixed once.
// A warp takes 32 / patch tokens; their values meet in shared memory and leave as whole vectors.  Every lane asks for one
// of the source rows before the walk begins, so that the rows arrive together and not one after the other.
template <typename T>
__global__ void __launch_bounds__(32 * kPatchWarps) patch_tokens_kernel(const __grid_constant__ PatchArgs A) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    __shared__ float2 s_rows[kPatchWarps][32];                    // (first byte of the upper source row as bits, weight of the lower)
    const int p = A.patch, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = 32 / p, area = p * p, values = 3 * area;
    const int sub = lane / p, px = lane - sub * p;
    const uint32_t own = ((uint32_t)(each * values) * (uint32_t)sizeof(T) + 15) / 16 * 16;
    T* const buf = reinterpret_cast<T*>(s_raw + warp * own);
    const uint64_t first = ((uint64_t)blockIdx.x * (blockDim.x >> 5) + warp) * (uint64_t)each;
    if (first >= A.n_tokens) return;
    const int count = (int)min((uint64_t)each, A.n_tokens - first);
    const bool here = sub < count;
    bool ok = false, words = false;
    const uint8_t* base = nullptr;        // the rectangle's first row at this lane's column
    int64_t pitch = 0;
    float fx = 0.f;
    if (here) {
        const int2 at = A.index[first + sub];
        if (at.x >= 0 && at.x < A.n_images) {
            const PatchImage m = A.images[at.x];
            ok = patch_ok(A, m, at.y);
            if (ok) {
                const int32_t cols = (int32_t)m.cols, mg = A.merge, band = mg * cols;
                const int32_t block = at.y / band, rest = at.y - block * band, square = mg * mg;
                const int32_t side = rest / square, in = rest - side * square;
                const int32_t row = block * mg + in / mg, col = side * mg + in % mg;
                int32_t ox = col * p + px;
                if (m.flip) ox = cols * p - 1 - ox;
                const Tap tx = tap_of(ox, cols * p, (int32_t)m.w), ty = tap_of(row * p + px, (int32_t)m.rows * p, (int32_t)m.h);
                pitch = 3 * m.width;
                fx = tx.f;
                const int64_t corner = m.offset + m.y0 * pitch + 3 * m.x0;
                base = A.rgb + corner + 3 * (int64_t)tx.lo;
                // rows are counted in bytes from the first, 32 bits; words are read where none can end behind the buffer
                words = m.h * pitch < (int64_t)1 << 31 && (uint64_t)(corner + (m.h - 1) * pitch + 3 * m.w + 12) <= A.rgb_bytes;
                const uint32_t off = words ? (uint32_t)ty.lo * (uint32_t)pitch : (uint32_t)ty.lo;
                s_rows[warp][lane] = make_float2(__uint_as_float(off), ty.f);
                if (words) {
                    const uint8_t* row0 = base - 3 * (int64_t)px + off;       // about where the patch's part of this row begins: no more than a hint
                    if (row0 >= A.rgb && row0 + 3 * p < A.rgb + A.rgb_bytes) { soon(row0); soon(row0 + 3 * p); }
                }
            }
        }
    }
    __syncwarp();
    if (here) {
        T* o = buf + sub * values + px;
        const F2 scale = pack2(A.scale[0], A.scale[1]), shift = pack2(A.shift[0], A.shift[1]), minus = pack2(-1.f, -1.f);
        auto put = [&](const Rgb& top, const Rgb& low, float fy) {
            const F2 rg = fma2(fma2(pack2(fy, fy), fma2(top.rg, minus, low.rg), top.rg), scale, shift);
            float r, g;
            unpack2(rg, r, g);
            o[0] = from_f<T>(r); o[area] = from_f<T>(g); o[2 * area] = from_f<T>(fmaf(fmaf(fy, low.b - top.b, top.b), A.scale[2], A.shift[2]));
            o += p;
        };
        const float2* rows = &s_rows[warp][sub * p];
        if (words) {
            Rgb top = {0, 0.f}, low = {0, 0.f};
            uint32_t top_at = ~0u, low_at = ~0u;
            const uint32_t down = (uint32_t)pitch;
            for (int dy = 0; dy < p; ++dy) {
                const float2 r = rows[dy];
                const uint32_t a = __float_as_uint(r.x), e = r.y != 0.f ? a + down : a;     // (weight 0: the row below may not be there)
                if (a != top_at) {
                    if (a == low_at) top = low; else top = mix_words(base + a, fx);
                    top_at = a;
                }
                if (e != low_at) {
                    if (e == top_at) low = top; else low = mix_words(base + e, fx);
                    low_at = e;
                }
                put(top, low, r.y);
            }
        } else if (ok) {
            for (int dy = 0; dy < p; ++dy) {
                const float2 r = rows[dy];
                const uint8_t* a = base + (int64_t)__float_as_uint(r.x) * pitch;
                const Rgb top = mix_single(a, fx), low = r.y != 0.f ? mix_single(a + pitch, fx) : top;
                put(top, low, r.y);
            }
        } else {
            for (int dy = 0; dy < p; ++dy, o += p) o[0] = o[area] = o[2 * area] = from_f<T>(0.f);
        }
    }
    __syncwarp();
    const uint32_t bytes = (uint32_t)(count * values * (int)sizeof(T));
    unsigned char* out = static_cast<unsigned char*>(A.out) + first * (uint64_t)values * sizeof(T);
    const unsigned char* src = reinterpret_cast<const unsigned char*>(buf);
    const uint32_t align = (uint32_t)(reinterpret_cast<uintptr_t>(out) | bytes);
    if ((align & 15u) == 0) {
        for (uint32_t i = lane * 16; i < bytes; i += 512) *reinterpret_cast<uint4*>(out + i) = *reinterpret_cast<const uint4*>(src + i);
    } else if ((align & 3u) == 0) {
        for (uint32_t i = lane * 4; i < bytes; i += 128) *reinterpret_cast<uint32_t*>(out + i) = *reinterpret_cast<const uint32_t*>(src + i);
    } else {
        for (uint32_t i = lane * 2; i < bytes; i += 64) *reinterpret_cast<uint16_t*>(out + i) = *reinterpret_cast<const uint16_t*>(src + i);
    }
}

// ---- positions of packed sequences ------------------------------------------------------------------------------------
//
// A segment is (t, h, w, sequence): t tokens of text where h or w is 0, else a grid of t x h x w tokens.  Sums over the
// segments before give a segment's first token and, inside its sequence, its first position.
struct PositionArgs {
    const int4* segments;
    int64_t* starts;               // first token of every segment, and one behind the last
    int32_t* bases;                // first position of every segment
    int32_t* positions;
    int32_t* next;
    int64_t stride;                // of the axes of `positions`
    uint32_t n_tokens, run;        // run: tokens of a CTA
    int32_t n_segments, n_sequences, merge, time_step, restart, zero_tail;
};

__device__ __forceinline__ void segment_sizes(const PositionArgs& A, const int4& s, int64_t& count, int64_t& extent) {
    const int32_t t = max(s.x, 0);
    if (s.y <= 0 || s.z <= 0) { count = extent = t; return; }
    const uint64_t plane = (uint64_t)(uint32_t)s.y * (uint32_t)s.z, most = (uint64_t)1 << 32;
    count = t == 0 ? 0 : (int64_t)min(min(plane, most) * (uint32_t)t, most);       // (more than any output holds)
    extent = t == 0 ? 0 : max((int64_t)(t - 1) * A.time_step, (int64_t)max(s.y, s.z) - 1) + 1;
}

// Positions of token number l of a segment that begins at position `base`.
__device__ __forceinline__ void position_in(const PositionArgs& A, const int4& s, int32_t base, uint32_t l, int32_t& pt, int32_t& ph, int32_t& pw) {
    if (s.y <= 0 || s.z <= 0) { pt = ph = pw = base + (int32_t)l; return; }
    const uint64_t plane = (uint64_t)(uint32_t)s.y * (uint32_t)s.z;
    uint32_t f = 0, rest = l, row, col;
    if ((plane >> 32) == 0) { f = l / (uint32_t)plane; rest = l - f * (uint32_t)plane; }
    const uint32_t m = (uint32_t)A.merge;
    if (m > 1 && s.y % A.merge == 0 && s.z % A.merge == 0) {
        const uint64_t band = (uint64_t)m * (uint32_t)s.z;
        const uint32_t block = band >> 32 ? 0 : rest / (uint32_t)band, in = rest - block * (uint32_t)band, q = in % (m * m);
        row = block * m + q / m; col = in / (m * m) * m + q % m;
    } else {
        row = rest / (uint32_t)s.z; col = rest - row * (uint32_t)s.z;
    }
    pt = base + (int32_t)f * A.time_step; ph = base + (int32_t)row; pw = base + (int32_t)col;
}

// Sums over the threads before this one, of kScanThreads threads: tokens, and positions since the last begin of a sequence
// (`first`: whether one lies in this thread's share).  In: the thread's own; out: those before it.  `total`: all tokens.
constexpr int kScanThreads = 1024;
__device__ __forceinline__ void sums_before(int64_t& tokens, int64_t& extent, bool first, int64_t& total) {
    __shared__ int64_t s_tokens[32], s_extent[32];
    __shared__ int32_t s_first[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto scan = [&](int64_t& t, int64_t& e, int32_t& f) {                // inclusive, over a warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t2 = __shfl_up_sync(0xffffffffu, t, o), e2 = __shfl_up_sync(0xffffffffu, e, o);
            const int32_t f2 = __shfl_up_sync(0xffffffffu, f, o);
            if (lane >= o) { t += t2; if (!f) e += e2; f |= f2; }
        }
    };
    int64_t t = tokens, e = extent;
    int32_t f = first;
    scan(t, e, f);
    if (lane == 31) { s_tokens[warp] = t; s_extent[warp] = e; s_first[warp] = f; }
    __syncthreads();
    int64_t wt = s_tokens[lane], we = s_extent[lane];
    int32_t wf = s_first[lane];
    scan(wt, we, wf);
    total = __shfl_sync(0xffffffffu, wt, 31);
    // the warps before, then the lanes before
    const int64_t bt = __shfl_sync(0xffffffffu, wt, max(warp - 1, 0)), be = __shfl_sync(0xffffffffu, we, max(warp - 1, 0));
    const int64_t lt = __shfl_up_sync(0xffffffffu, t, 1), le = __shfl_up_sync(0xffffffffu, e, 1);
    const int32_t lf = __shfl_up_sync(0xffffffffu, f, 1);
    tokens = (warp ? bt : 0) + (lane ? lt : 0);
    extent = (lane ? le : 0) + (warp && !(lane && lf) ? be : 0);
    __syncthreads();                                                      // the arrays may be used again
}

// Goes over this thread's share of the segments; put(i, first token, first position) is called for each.  A sequence's end
// is written to A.next where `ends` is set.
template <typename Put>
__device__ __forceinline__ int64_t walk_segments(const PositionArgs& A, bool ends, Put put) {
    const int tid = threadIdx.x, n = A.n_segments, each = (int)(((int64_t)n + kScanThreads - 1) / kScanThreads);
    const int a = (int)min((int64_t)tid * each, (int64_t)n), b = (int)min((int64_t)a + each, (int64_t)n);
    const int32_t before = a > 0 && a < n ? A.segments[a - 1].w : -1;
    if (ends)
        for (int i = tid; i < A.n_sequences; i += kScanThreads) A.next[i] = 0;
    int64_t tokens = 0, extent = 0, total;
    bool first = false;
    for (int i = a, seq = before; i < b; ++i) {
        const int4 s = A.segments[i];
        int64_t c, e;
        segment_sizes(A, s, c, e);
        if (s.w != seq || A.restart) { first = true; extent = 0; }
        seq = s.w;
        tokens += c; extent += e;
    }
    sums_before(tokens, extent, first, total);
    for (int i = a, seq = before; i < b; ++i) {
        const int4 s = A.segments[i];
        int64_t c, e;
        segment_sizes(A, s, c, e);
        if (s.w != seq || A.restart) extent = 0;
        seq = s.w;
        put(i, tokens, (int32_t)extent);
        tokens += c; extent += e;
        if (ends && (i + 1 == n || A.segments[i + 1].w != s.w) && s.w >= 0 && s.w < A.n_sequences) A.next[s.w] = (int32_t)extent;
    }
    return total;
}

// Up to kFewSegments segments: every CTA works out where all of them begin, keeps that in shared memory and writes its own
// run of tokens.  One launch; the segments are read by every CTA, 16 bytes each, out of L2.
constexpr int kFewSegments = 16384, kRunTokens = 1024;
__global__ void __launch_bounds__(kScanThreads) positions_kernel(const __grid_constant__ PositionArgs A) {
    extern __shared__ uint2 s_begin[];                                    // (first token, first position)
    const int64_t total = walk_segments(A, blockIdx.x == 0, [&](int i, int64_t token, int32_t position) {
        s_begin[i] = make_uint2((uint32_t)min(token, (int64_t)0xffffffff), (uint32_t)position);
    });
    __syncthreads();
    const uint32_t t0 = (uint32_t)min((uint64_t)blockIdx.x * A.run, (uint64_t)A.n_tokens), t1 = (uint32_t)min((uint64_t)t0 + A.run, (uint64_t)A.n_tokens);
    for (uint64_t tok = (uint64_t)t0 + threadIdx.x; tok < t1; tok += kScanThreads) {
        const uint32_t token = (uint32_t)tok;
        int32_t pt = 0, ph = 0, pw = 0;
        if ((int64_t)token < total) {
            int lo = 0, hi = A.n_segments;                                // the last segment that begins at or before the token
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_begin[mid].x <= token) lo = mid; else hi = mid;
            }
            position_in(A, A.segments[lo], (int32_t)s_begin[lo].y, token - s_begin[lo].x, pt, ph, pw);
        } else if (!A.zero_tail) {
            break;
        }
        A.positions[token] = pt; A.positions[A.stride + token] = ph; A.positions[2 * A.stride + token] = pw;
    }
}

// More segments: one CTA writes where each begins to device memory, then a thread a token looks its segment up there.
__global__ void __launch_bounds__(kScanThreads) position_scan_kernel(const __grid_constant__ PositionArgs A) {
    const int64_t total = walk_segments(A, true, [&](int i, int64_t token, int32_t position) { A.starts[i] = token; A.bases[i] = position; });
    if (threadIdx.x == 0) A.starts[A.n_segments] = total;
}

constexpr int kFillThreads = 256;
__global__ void __launch_bounds__(kFillThreads) position_fill_kernel(const __grid_constant__ PositionArgs A) {
    const uint64_t tok = (uint64_t)blockIdx.x * kFillThreads + threadIdx.x;
    if (tok >= A.n_tokens) return;
    const uint32_t token = (uint32_t)tok;
    int32_t pt = 0, ph = 0, pw = 0;
    if ((int64_t)token < A.starts[A.n_segments]) {
        int lo = 0, hi = A.n_segments;
        while (hi - lo > 1) {
            const int mid = lo + ((hi - lo) >> 1);
            if (A.starts[mid] <= (int64_t)token) lo = mid; else hi = mid;
        }
        position_in(A, A.segments[lo], A.bases[lo], (uint32_t)((int64_t)token - A.starts[lo]), pt, ph, pw);
    } else if (!A.zero_tail) {
        return;
    }
    A.positions[token] = pt; A.positions[A.stride + token] = ph; A.positions[2 * A.stride + token] = pw;
}

}  // namespace pcr
