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
        t.f = (float)(num - t.lo * den) / (float)den;
    } else {
        const int64_t den = 2 * (int64_t)out;
        const int64_t num = min(max((2 * (int64_t)o + 1) * side - out, (int64_t)0), (side - 1) * den);
        t.lo = (int32_t)(num / den);
        t.f = (float)(num - t.lo * den) / (float)den;
    }
    return t;
}

// Whether a token's entry stands for a patch of pixels that are there.
__device__ __forceinline__ bool patch_ok(const PatchArgs& A, const PatchImage& m, int32_t local) {
    const int64_t p = A.patch;
    return m.width >= 1 && m.width <= kMaxSide && m.height >= 1 && m.height <= kMaxSide && m.offset >= 0 &&
           (uint64_t)m.offset <= A.rgb_bytes && (uint64_t)(3 * m.width * m.height) <= A.rgb_bytes - (uint64_t)m.offset &&
           m.x0 >= 0 && m.y0 >= 0 && m.w >= 1 && m.h >= 1 && m.w <= m.width && m.h <= m.height && m.x0 <= m.width - m.w &&
           m.y0 <= m.height - m.h && m.rows >= 1 && m.cols >= 1 && m.rows <= kMaxSide / p && m.cols <= kMaxSide / p &&
           m.rows % A.merge == 0 && m.cols % A.merge == 0 && (m.flip == 0 || m.flip == 1) && local >= 0 && local < m.rows * m.cols;
}

__device__ __forceinline__ float byte_f(uint32_t word, int i) {          // byte i of a word: exact through 2^23 + byte
    return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440u | (uint32_t)i)) - 8388608.f;
}

// The two pixels from byte `at` of the buffer on, mixed: aligned words where they lie inside the buffer.
__device__ __forceinline__ void mix_pixels(const PatchArgs& A, uint64_t at, float f, float (&v)[3]) {
    uint32_t lo, hi;
    const uint64_t word = at & ~3ull;
    if (word + 12 <= A.rgb_bytes) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(A.rgb + word);
        const uint32_t sh = (uint32_t)(at & 3) * 8, w0 = __ldg(p), w1 = __ldg(p + 1), w2 = sh == 24 ? __ldg(p + 2) : 0;
        lo = __funnelshift_r(w0, w1, sh);
        hi = __funnelshift_r(w1, w2, sh);
    } else {                                                             // (a tap of weight 0 may lie behind the last pixel)
        lo = A.rgb[at] | (uint32_t)A.rgb[at + 1] << 8 | (uint32_t)A.rgb[at + 2] << 16;
        hi = 0;
        if (f != 0.f) {
            lo |= (uint32_t)A.rgb[at + 3] << 24;
            hi = A.rgb[at + 4] | (uint32_t)A.rgb[at + 5] << 8;
        }
    }
    const float r0 = byte_f(lo, 0), g0 = byte_f(lo, 1), b0 = byte_f(lo, 2), r1 = byte_f(lo, 3), g1 = byte_f(hi, 0), b1 = byte_f(hi, 1);
    v[0] = r0 + f * (r1 - r0); v[1] = g0 + f * (g1 - g0); v[2] = b0 + f * (b1 - b0);
}

// A lane a column of a patch, walking down its rows: a source row that serves two output rows is read and mixed once.
// A warp takes 32 / patch tokens; their values meet in shared memory and leave as whole vectors.
template <typename T>
__global__ void __launch_bounds__(32 * kPatchWarps) patch_tokens_kernel(const __grid_constant__ PatchArgs A) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    const int p = A.patch, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = 32 / p, area = p * p, values = 3 * area;
    const int sub = lane / p, px = lane - sub * p;
    const size_t own = ((size_t)each * values * sizeof(T) + 15) / 16 * 16;
    T* const buf = reinterpret_cast<T*>(s_raw + warp * own);
    const uint64_t first = ((uint64_t)blockIdx.x * kPatchWarps + warp) * (uint64_t)each;
    if (first >= A.n_tokens) return;
    const int count = (int)min((uint64_t)each, A.n_tokens - first);
    const bool here = sub < count;
    bool ok = false;
    int64_t corner = 0, pitch = 0;        // first byte of the rectangle, bytes of a row
    Tap tx = {0, 0.f}, ty = {0, 0.f};     // this lane's column; the row that has this lane's number
    int32_t h = 1;
    if (here) {
        const int2 at = A.index[first + sub];
        if (at.x >= 0 && at.x < A.n_images) {
            const PatchImage m = A.images[at.x];
            ok = patch_ok(A, m, at.y);
            if (ok) {
                const int32_t cols = (int32_t)m.cols, mg = A.merge, band = mg * cols;
                const int32_t block = at.y / band, rest = at.y - block * band;
                const int32_t in = rest % (mg * mg);
                const int32_t row = block * mg + in / mg, col = rest / (mg * mg) * mg + in % mg;
                int32_t ox = col * p + px;
                if (m.flip) ox = cols * p - 1 - ox;
                tx = tap_of(ox, cols * p, (int32_t)m.w);
                ty = tap_of(row * p + px, (int32_t)m.rows * p, (int32_t)m.h);
                pitch = 3 * m.width;
                corner = m.offset + m.y0 * pitch + 3 * m.x0;
                h = (int32_t)m.h;
            }
        }
    }
    const int64_t left = corner + 3 * (int64_t)tx.lo;
    T* o = buf + (here ? sub * values + px : 0);
    float top[3] = {0.f, 0.f, 0.f}, low[3] = {0.f, 0.f, 0.f};
    int32_t top_row = -1, low_row = -1;
    for (int dy = 0; dy < p; ++dy, o += p) {
        const int from = min(sub * p + dy, 31);
        const int32_t ya = __shfl_sync(0xffffffffu, ty.lo, from);
        const float fy = __shfl_sync(0xffffffffu, ty.f, from);
        if (!here) continue;
        float v[3] = {0.f, 0.f, 0.f};
        if (ok) {
            const int32_t yb = min(ya + 1, h - 1);
            if (ya != top_row) {
                if (ya == low_row) { top[0] = low[0]; top[1] = low[1]; top[2] = low[2]; }
                else mix_pixels(A, (uint64_t)(left + ya * pitch), tx.f, top);
                top_row = ya;
            }
            if (yb != low_row) { mix_pixels(A, (uint64_t)(left + yb * pitch), tx.f, low); low_row = yb; }
#pragma unroll
            for (int c = 0; c < 3; ++c) v[c] = (top[c] + fy * (low[c] - top[c])) * A.scale[c] + A.shift[c];
        }
        o[0] = from_f<T>(v[0]); o[area] = from_f<T>(v[1]); o[2 * area] = from_f<T>(v[2]);
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
    uint32_t n_tokens;
    int32_t n_segments, n_sequences, merge, time_step, restart, zero_tail;
};

__device__ __forceinline__ void segment_sizes(const PositionArgs& A, const int4& s, int64_t& count, int64_t& extent) {
    if (s.y <= 0 || s.z <= 0) { count = extent = max(s.x, 0); return; }
    const int64_t t = max(s.x, 0);
    const unsigned __int128 all = (unsigned __int128)t * (uint64_t)s.y * (uint64_t)s.z;
    count = all > ((uint64_t)1 << 32) ? (int64_t)1 << 32 : (int64_t)all;       // (more than any output holds)
    extent = t == 0 ? 0 : max((t - 1) * A.time_step, (int64_t)max(s.y, s.z) - 1) + 1;
}

// One CTA: every thread sums a run of segments, the runs' sums meet in shared memory, every thread goes over its run again.
constexpr int kScanThreads = 1024;
__global__ void __launch_bounds__(kScanThreads) position_scan_kernel(const __grid_constant__ PositionArgs A) {
    __shared__ int64_t s_tokens[kScanThreads], s_extent[kScanThreads];
    __shared__ int32_t s_first[kScanThreads];       // whether a sequence begins inside the run
    const int tid = threadIdx.x, n = A.n_segments, each = (int)(((int64_t)n + kScanThreads - 1) / kScanThreads);
    const int a = (int)min((int64_t)tid * each, (int64_t)n), b = (int)min((int64_t)a + each, (int64_t)n);
    for (int i = tid; i < A.n_sequences; i += kScanThreads) A.next[i] = 0;
    int64_t tokens = 0, extent = 0;
    bool first = false;
    const int32_t before = a > 0 && a < n ? A.segments[a - 1].w : -1;
    for (int i = a, seq = before; i < b; ++i) {
        const int4 s = A.segments[i];
        int64_t c, e;
        segment_sizes(A, s, c, e);
        if (s.w != seq || A.restart) { first = true; extent = 0; }
        seq = s.w;
        tokens += c; extent += e;
    }
    s_tokens[tid] = tokens; s_extent[tid] = extent; s_first[tid] = first;
    __syncthreads();
    for (int o = 1; o < kScanThreads; o <<= 1) {      // inclusive sums; positions stop at a sequence's begin
        int64_t t = 0, e = 0;
        int32_t f = 0;
        if (tid >= o) { t = s_tokens[tid - o]; e = s_extent[tid - o]; f = s_first[tid - o]; }
        __syncthreads();
        s_tokens[tid] += t;
        if (!s_first[tid]) { s_extent[tid] += e; s_first[tid] = f; }
        __syncthreads();
    }
    tokens = tid ? s_tokens[tid - 1] : 0;
    extent = tid ? s_extent[tid - 1] : 0;
    for (int i = a, seq = before; i < b; ++i) {
        const int4 s = A.segments[i];
        int64_t c, e;
        segment_sizes(A, s, c, e);
        if (s.w != seq || A.restart) extent = 0;
        seq = s.w;
        A.starts[i] = tokens; A.bases[i] = (int32_t)extent;
        tokens += c; extent += e;
        const bool last = i + 1 == n || A.segments[i + 1].w != s.w;
        if (last && s.w >= 0 && s.w < A.n_sequences) A.next[s.w] = (int32_t)extent;
    }
    if (tid == kScanThreads - 1) A.starts[n] = s_tokens[tid];
}

constexpr int kFillThreads = 256;
__global__ void __launch_bounds__(kFillThreads) position_fill_kernel(const __grid_constant__ PositionArgs A) {
    const uint64_t tok = (uint64_t)blockIdx.x * kFillThreads + threadIdx.x;
    if (tok >= A.n_tokens) return;
    const uint32_t token = (uint32_t)tok;
    int32_t pt = 0, ph = 0, pw = 0;
    if ((int64_t)token < A.starts[A.n_segments]) {
        int lo = 0, hi = A.n_segments;                // the last segment that begins at or before the token
        while (hi - lo > 1) {
            const int mid = lo + ((hi - lo) >> 1);
            if (A.starts[mid] <= (int64_t)token) lo = mid; else hi = mid;
        }
        const int4 s = A.segments[lo];
        const int32_t base = A.bases[lo];
        const uint32_t l = (uint32_t)((int64_t)token - A.starts[lo]);
        if (s.y <= 0 || s.z <= 0) { pt = ph = pw = base + (int32_t)l; }
        else {
            const uint64_t plane = (uint64_t)s.y * (uint64_t)s.z;
            uint32_t f, rest;
            if (plane >> 32) { f = 0; rest = l; } else { f = l / (uint32_t)plane; rest = l - f * (uint32_t)plane; }
            uint32_t row, col;
            const uint32_t m = (uint32_t)A.merge;
            if (m > 1 && s.y % A.merge == 0 && s.z % A.merge == 0) {
                const uint64_t band = (uint64_t)m * (uint32_t)s.z;
                const uint32_t block = (uint32_t)(rest / band), in = (uint32_t)(rest - block * band), q = in % (m * m);
                row = block * m + q / m; col = in / (m * m) * m + q % m;
            } else {
                row = rest / (uint32_t)s.z; col = rest - row * (uint32_t)s.z;
            }
            pt = base + (int32_t)f * A.time_step; ph = base + (int32_t)row; pw = base + (int32_t)col;
        }
    } else if (!A.zero_tail) {
        return;
    }
    A.positions[token] = pt; A.positions[A.stride + token] = ph; A.positions[2 * A.stride + token] = pw;
}

}  // namespace pcr
