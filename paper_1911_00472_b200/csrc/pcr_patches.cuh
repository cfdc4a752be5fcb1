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
    int32_t n_images, patch, merge, each;        // each: tokens of a warp
    uint32_t by_lanes, by_merge;   // lane / lanes of a patch = lane * by_lanes >> 16, i / merge = i * by_merge >> 20 (i < merge^2)
    float scale[3], shift[3];      // (v / 255 - mean) / std = v * scale + shift
};

// Bilinear taps with half-pixel centres: the source coordinate (o + 1/2) side / out - 1/2 as a whole number over 2 out,
// so that where it falls between pixels is exact whatever the sizes.
struct Tap { int32_t lo; float f; };
struct Axis { int32_t out, side; float inv; bool small; };               // resampled and source pixels, 1 / (2 out)
__device__ __forceinline__ Axis axis_of(int32_t out, int32_t side) {
    return {out, side, __fdividef(1.f, 2.f * (float)out), (int64_t)out * side < (1 << 29)};
}
__device__ __forceinline__ Tap tap_of(int32_t o, const Axis& x) {
    Tap t;
    if (x.small) {
        // below 2^30, and the quotient below 2^20: with the approximate reciprocal it is off by one at most
        const int32_t den = 2 * x.out;
        const int32_t num = min(max((2 * o + 1) * x.side - x.out, 0), (x.side - 1) * den);
        t.lo = (int32_t)((float)num * x.inv);
        int32_t rest = num - t.lo * den;
        if (rest < 0) { --t.lo; rest += den; }
        if (rest >= den) { ++t.lo; rest -= den; }
        t.f = (float)rest * x.inv;                                       // (off by 3 roundings)
    } else {
        const int64_t den = 2 * (int64_t)x.out;
        const int64_t num = min(max((2 * (int64_t)o + 1) * x.side - x.out, (int64_t)0), (x.side - 1) * den);
        t.lo = (int32_t)(num / den);
        t.f = (float)(num - t.lo * den) / (float)den;
    }
    return t;
}

// a / b where a < 2^22: one unit off at most before it is put right
__device__ __forceinline__ uint32_t quotient(uint32_t a, uint32_t b) {
    if ((a | b) >= 1u << 22) return a / b;
    uint32_t q = (uint32_t)__fdividef((float)a, (float)b);
    const int32_t rest = (int32_t)(a - q * b);
    return rest < 0 ? q - 1 : rest >= (int32_t)b ? q + 1 : q;
}

// A token's patch: whether there is one, and where.
struct Patch {
    bool ok, near, words, flip;    // near: rows may be counted in 32 bits; words: and every row is followed by 16 bytes of the buffer
    int32_t row, col;
    int64_t pitch;
    const uint8_t* corner;         // the rectangle's first byte
    Axis x, y;
};
__device__ __forceinline__ void look_up(const PatchArgs& A, int2 token, Patch& r) {
    r.ok = r.near = r.words = false;
    const int32_t image = token.x;
    if (image < 0 || image >= A.n_images) return;
    const longlong2* from = reinterpret_cast<const longlong2*>(A.images + image);
    const longlong2 m0 = __ldg(from), m1 = __ldg(from + 1), m2 = __ldg(from + 2), m3 = __ldg(from + 3), m4 = __ldg(from + 4);
    const PatchImage m = {m0.x, m0.y, m1.x, m1.y, m2.x, m2.y, m3.x, m3.y, m4.x, m4.y};
    // (a negative number has its upper bits set)
    if (((uint64_t)(m.width | m.height | m.x0 | m.y0 | m.w | m.h | m.rows | m.cols | m.flip) >> 21) != 0 || m.offset < 0) return;
    const int32_t width = (int32_t)m.width, height = (int32_t)m.height, w = (int32_t)m.w, h = (int32_t)m.h, rows = (int32_t)m.rows, cols = (int32_t)m.cols;
    const uint32_t odd = (uint32_t)(A.merge - 1);
    const bool whole = (A.merge & odd) == 0 ? ((rows | cols) & odd) == 0 : rows % A.merge == 0 && cols % A.merge == 0;
    const uint64_t room = A.rgb_bytes - (uint64_t)m.offset;
    r.ok = width >= 1 && width <= kMaxSide && height >= 1 && height <= kMaxSide && (uint64_t)m.offset <= A.rgb_bytes &&
           3 * (uint64_t)width * (uint64_t)height <= room && w >= 1 && h >= 1 && (int32_t)m.x0 + w <= width && (int32_t)m.y0 + h <= height &&
           rows >= 1 && cols >= 1 && rows * A.patch <= kMaxSide && cols * A.patch <= kMaxSide && whole && m.flip <= 1;
    if (!r.ok || token.y < 0 || token.y >= (int64_t)rows * cols) { r.ok = false; return; }
    const uint32_t mg = (uint32_t)A.merge, band = mg * (uint32_t)cols, block = quotient((uint32_t)token.y, band), rest = (uint32_t)token.y - block * band;
    const uint32_t side = mg == 1 ? rest : quotient(rest, mg * mg), in = rest - side * (mg * mg), down = in * A.by_merge >> 20;
    r.row = (int32_t)(block * mg + down); r.col = (int32_t)(side * mg + in - down * mg);
    r.flip = m.flip != 0;
    r.pitch = 3 * (int64_t)width;
    const int64_t corner = m.y0 * r.pitch + 3 * m.x0, behind = corner + (h - 1) * r.pitch + 3 * w + 16;
    r.near = h * r.pitch < (int64_t)1 << 31;
    r.words = r.near && (uint64_t)behind <= room;
    r.corner = A.rgb + m.offset + corner;
    r.x = axis_of(cols * A.patch, w);
    r.y = axis_of(rows * A.patch, h);
}

// Bytes become floats as 2^23 + byte, exactly; differences need no more, what is added to has the 2^23 taken off.
__device__ __forceinline__ float byte_up(uint32_t word, int i) { return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440u | (uint32_t)i)); }
constexpr float kUp = 8388608.f;

// The pixel whose bytes are the lowest three of `lo` mixed with the next one (fourth byte of `lo`, two of `hi`).
struct Rgb { float r, g, b; };
__device__ __forceinline__ Rgb mix_bytes(uint32_t lo, uint32_t hi, float f) {
    const float r = byte_up(lo, 0), g = byte_up(lo, 1), b = byte_up(lo, 2);
    return {fmaf(f, byte_up(lo, 3) - r, r - kUp), fmaf(f, byte_up(hi, 0) - g, g - kUp), fmaf(f, byte_up(hi, 1) - b, b - kUp)};
}
// ... read as aligned words, which have to lie inside the buffer
__device__ __forceinline__ Rgb mix_words(const uint8_t* at, float f) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)3);
    const uint32_t sh = (uint32_t)reinterpret_cast<uintptr_t>(at) << 3, w0 = __ldg(p), w1 = __ldg(p + 1);        // (shifts count modulo 32)
    uint32_t w2 = 0;
    if ((sh & 31) == 24) w2 = __ldg(p + 2);
    return mix_bytes(__funnelshift_r(w0, w1, sh), __funnelshift_r(w1, w2, sh), f);
}
// ... byte by byte, the next pixel only where it counts: it may lie behind the last one
__device__ __forceinline__ Rgb mix_single(const uint8_t* at, float f) {
    uint32_t lo = at[0] | (uint32_t)at[1] << 8 | (uint32_t)at[2] << 16, hi = 0;
    if (f != 0.f) { lo |= (uint32_t)at[3] << 24; hi = at[4] | (uint32_t)at[5] << 8; }
    return mix_bytes(lo, hi, f);
}

// How a walk reads its words.  kPlain: from addresses of whole words on (their shift is the lane's own), and no column two
// pixels on; kFree: from any address; kEnd: and none beyond the end of the buffer.
enum { kPlain, kFree, kEnd };
template <int kHow> struct How { static constexpr int value = kHow; };

// Two columns of a source row, mixed; both in every instruction.
struct Mixed { F2 c[3]; };

// The words that two neighbouring columns lie in: the left one's six bytes begin at `sh` bits into the first, the right
// one's 0, 3 or 6 bytes further on.
struct Words { uint32_t w0, w1, w2, w3, sh; };
// The end of a buffer of at least four bytes: its last whole word, and the bytes behind that.
struct End { const uint32_t* last; uint32_t rest; };
__device__ __forceinline__ End end_of(const uint8_t* from, size_t bytes) {
    const uint8_t* b = from + (bytes & ~(size_t)3);
    const int n = (int)(bytes & 3);
    return {reinterpret_cast<const uint32_t*>(b) - 1, (n > 0 ? b[0] : 0u) | (n > 1 ? (uint32_t)b[1] << 8 : 0u) | (n > 2 ? (uint32_t)b[2] << 16 : 0u)};
}
template <int kHow>
__device__ __forceinline__ Words words_at(const uint8_t* at, bool wide, const End& end) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(kHow == kPlain ? reinterpret_cast<uintptr_t>(at) : reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)3);
    Words r = {0, 0, 0, 0, (uint32_t)reinterpret_cast<uintptr_t>(at) << 3};
    if (kHow == kEnd) {                       // (what lies behind the last bytes has no weight: any number does)
        auto word = [&](int i) { const uint32_t v = __ldg(p + i <= end.last ? p + i : end.last); return p + i <= end.last ? v : end.rest; };
        r.w0 = word(0); r.w1 = word(1); r.w2 = word(2); r.w3 = word(3);
        return r;
    }
    r.w0 = __ldg(p); r.w1 = __ldg(p + 1); r.w2 = __ldg(p + 2);
    if (kHow != kPlain && wide) r.w3 = __ldg(p + 3);
    return r;
}
template <int kHow>
__device__ __forceinline__ Mixed mix_words(const Words& w, uint32_t own, bool wide, uint32_t shift, F2 f) {
    const uint32_t sh = kHow == kPlain ? own : w.sh;
    const uint32_t x0 = __funnelshift_r(w.w0, w.w1, sh), x1 = __funnelshift_r(w.w1, w.w2, sh), x2 = __funnelshift_r(w.w2, w.w3, sh);
    const uint32_t a = kHow != kPlain && wide ? x1 : x0, b = kHow != kPlain && wide ? x2 : x1, y0 = __funnelshift_r(a, b, shift), y1 = __funnelshift_r(b, x2, shift);
    const F2 one = pack2(1.f, 1.f), minus = pack2(-1.f, -1.f), down = pack2(-kUp, -kUp);
    Mixed r;
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        const F2 left = pack2(byte_up(x0, c), byte_up(y0, c)), right = c == 0 ? pack2(byte_up(x0, 3), byte_up(y0, 3)) : pack2(byte_up(x1, c - 1), byte_up(y1, c - 1));
        r.c[c] = fma2(f, fma2(left, minus, right), fma2(left, one, down));
    }
    return r;
}

// Values of one or two columns side by side.
__device__ __forceinline__ void put_two(float* to, float a, float b, bool swap) { *reinterpret_cast<float2*>(to) = swap ? make_float2(b, a) : make_float2(a, b); }
__device__ __forceinline__ void put_two(__half* to, float a, float b, bool swap) {
    __half2 v = __floats2half2_rn(a, b);
    if (swap) v = __lowhigh2highlow(v);
    *reinterpret_cast<__half2*>(to) = v;
}
__device__ __forceinline__ void put_two(__nv_bfloat16* to, float a, float b, bool swap) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    if (swap) v = __lowhigh2highlow(v);
    *reinterpret_cast<__nv_bfloat162*>(to) = v;
}

// A lane kCols neighbouring columns of a patch, walking down its rows: a source row that serves two output rows is read and
// mixed once, and its words are asked for one row ahead.  A warp takes 32 / lanes-of-a-patch tokens, whose values meet in
// shared memory and leave as whole vectors, or (kDirect) are written as they come.
// What bounds it: instructions, not HBM (192 images to patches of 14, 16 bits: issued in 70 % of the cycles, four of ten
// instructions on the integer pipe that takes bytes apart, L1 71 %, DRAM 28 %).  So two columns go to a lane (they share the walk's addresses, words
// and conditions, and go two to an instruction: 568 -> 405 us for 1024 images; patches of odd size have one column a lane), and
// what a token costs once (its entry, image and taps: a third of the instructions at patches of 14) is kept in 32 bits and
// without divisions.  Looking up 32 tokens at once in shared memory (457 us) or keeping an image for several rounds of a warp
// (560 to 620 in the place of 568) was slower: fewer warps fit.
// Measured: 1024 images of 256 to 496 pixels a side to patches of 14, 16 bits: 398 us, 3.4 TB/s of what has to move; of 16: 334 us, in
// 32 bits 360 (6.0 TB/s); of 13, 15 and 17 (one column a lane): 730, 616 and 1016 us.  96 crops of images of 600 x 450 to patches
// of 16, 32 bits: 41.5 us, 4.8 TB/s; 768 patches of 4 small images: 6 us.
template <typename T, int kCols, bool kDirect>
__global__ void __launch_bounds__(32 * kPatchWarps, 8) patch_tokens_kernel(const __grid_constant__ PatchArgs A) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    __shared__ uint4 s_rows[kPatchWarps][kMaxPatch * kCols];      // first bytes of the upper and the lower source row, weight of the lower
    const int p = A.patch, across = p / kCols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = A.each, area = p * p, values = 3 * area;
    const int sub = (int)(lane * A.by_lanes >> 16), px = (lane - sub * across) * kCols;
    const uint32_t own = ((uint32_t)(each * values) * (uint32_t)sizeof(T) + 15) / 16 * 16;
    T* const buf = reinterpret_cast<T*>(s_raw + warp * own);
    const uint64_t first = ((uint64_t)blockIdx.x * (blockDim.x >> 5) + warp) * (uint64_t)each;
    if (first >= A.n_tokens) return;
    const int count = (int)min((uint64_t)each, A.n_tokens - first);
    const bool here = sub < count;
    Patch m;
    m.ok = m.near = m.words = false;
    const uint8_t *base = nullptr, *other = nullptr;        // the rectangle's first row at the left column, at the right one
    float fl = 0.f, fr = 0.f;
    uint4* const rows0 = &s_rows[warp][here ? sub * p : 0];
    if (here) {
        look_up(A, A.index[first + sub], m);
        if (m.ok) {
            // the columns of a mirrored patch run to the left: its second is the left one
            const int32_t ox = m.flip ? m.x.out - kCols - (m.col * p + px) : m.col * p + px;
            const Tap tl = tap_of(ox, m.x), tr = kCols == 2 ? tap_of(ox + 1, m.x) : tl;
            fl = tl.f; fr = tr.f;
            base = m.corner + 3 * tl.lo; other = m.corner + 3 * tr.lo;
            const uint32_t pitch = m.near ? (uint32_t)m.pitch : 1u;
#pragma unroll
            for (int k = 0; k < kCols; ++k) {
                const Tap ty = tap_of(m.row * p + px + k, m.y);
                const uint32_t off = (uint32_t)ty.lo * pitch;
                rows0[px + k] = make_uint4(off, ty.f != 0.f ? off + pitch : off, __float_as_uint(ty.f), 0);       // (weight 0: the row below may not be there)
                if (m.near) soon(base + off);                // the patch's diagonal: its rows arrive together
            }
        }
    }
    // As a rule a warp's rows begin at whole words, are not mirrored, and its neighbouring columns at most a pixel apart:
    // a third of the walk's shifts, selects and address arithmetic is then left out (they bound it).
    const bool plain = kCols == 2 && __all_sync(0xffffffffu, !here || (m.words && !m.flip && (m.pitch & 3) == 0 && other - base <= 3));
    __syncwarp();
    // A patch whose last row (the lowest: its entry stands last) is the buffer's may have fewer than the four words that a lane
    // reads: its warp looks at every word's place.
    const bool at_end = !plain && __any_sync(0xffffffffu, here && m.near && !m.words && other + rows0[p - 1].y + 16 > A.rgb + A.rgb_bytes);
    if (here) {
        T* o = (kDirect ? static_cast<T*>(A.out) + (first + sub) * (uint64_t)values : buf + sub * values) + px;
        const uint4* rows = rows0;
        const bool swap = m.flip && m.ok;
        auto value = [&](int c, float top, float low, float fy) { return fmaf(fmaf(fy, low - top, top), A.scale[c], A.shift[c]); };
        if (kCols == 2 && m.near && other - base <= 6 && A.rgb_bytes >= 4) {
            const F2 f = pack2(fl, fr), minus = pack2(-1.f, -1.f);
            // On entry `top` holds the mixed row at low_at and `low` the one at top_at (the last output row's, roles swapped): as
            // a rule an output row's upper source row is the last one's lower, and one row is mixed.
            auto walk = [&](auto how, const uint8_t* from, uint32_t own_shift, bool wide, uint32_t shift, bool mirror, const End& end) {
                constexpr int kHow = decltype(how)::value;
                uint32_t top_at = ~0u, low_at = ~0u;
                auto step = [&](Mixed& top, Mixed& low, const Words& now, Words& next, T* to, const uint4& r, const uint4& after) {
                    next = words_at<kHow>(from + after.y, wide, end);
                    if (r.x != low_at) top = r.x == top_at ? low : mix_words<kHow>(words_at<kHow>(from + r.x, wide, end), own_shift, wide, shift, f);
                    low = mix_words<kHow>(now, own_shift, wide, shift, f);
                    top_at = r.x; low_at = r.y;
                    const float fy = __uint_as_float(r.z);
                    const F2 fy2 = pack2(fy, fy);
#pragma unroll
                    for (int c = 0; c < 3; ++c) {
                        const F2 v = fma2(fma2(fy2, fma2(top.c[c], minus, low.c[c]), top.c[c]), pack2(A.scale[c], A.scale[c]), pack2(A.shift[c], A.shift[c]));
                        float a, b;
                        unpack2(v, a, b);
                        put_two(to + c * area, a, b, kHow != kPlain && mirror);
                    }
                };
                Mixed u = {}, v = {};
                Words even = words_at<kHow>(from + rows[0].y, wide, end), odd;
#pragma unroll 1
                for (int dy = 0; dy < p; dy += 2, o += 2 * p, rows += 2) {
                    const uint4 r0 = rows[0], r1 = rows[1], r2 = rows[dy + 2 < p ? 2 : 1];
                    step(u, v, even, odd, o, r0, r1);
                    step(v, u, odd, even, o + p, r1, r2);
                }
            };
            const uint32_t sh = (uint32_t)reinterpret_cast<uintptr_t>(base) << 3;
            const bool wide = other - base == 6;
            const uint32_t shift = wide ? 16 : other != base ? 24 : 0;
            if (plain) walk(How<kPlain>(), base - (reinterpret_cast<uintptr_t>(base) & 3), sh, false, shift, false, End());
            else if (!at_end) walk(How<kFree>(), base, sh, wide, shift, swap, End());
            else walk(How<kEnd>(), base, sh, wide, shift, swap, end_of(A.rgb, A.rgb_bytes));
        } else if (m.near && !at_end) {
            Rgb top[kCols], low[kCols];
            const float f[2] = {fl, fr};
            const uint8_t* const from[2] = {base, other};
            uint32_t top_at = ~0u, low_at = ~0u;
            for (int dy = 0; dy < p; ++dy, o += p) {
                const uint4 r = rows[dy];
#pragma unroll
                for (int k = 0; k < kCols; ++k) {
                    if (r.x != top_at) { if (r.x == low_at) top[k] = low[k]; else top[k] = mix_words(from[k] + r.x, f[k]); }
                    if (r.y != low_at) low[k] = mix_words(from[k] + r.y, f[k]);
                    const float fy = __uint_as_float(r.z);
                    T* to = o + (swap ? kCols - 1 - k : k);
                    to[0] = from_f<T>(value(0, top[k].r, low[k].r, fy)); to[area] = from_f<T>(value(1, top[k].g, low[k].g, fy)); to[2 * area] = from_f<T>(value(2, top[k].b, low[k].b, fy));
                }
                top_at = r.x; low_at = r.y;
            }
        } else if (m.ok) {
            const int64_t pitch = m.near ? 1 : m.pitch;        // (of what stands in s_rows)
            for (int dy = 0; dy < p; ++dy, o += p) {
                const uint4 r = rows[dy];
                for (int k = 0; k < kCols; ++k) {
                    const uint8_t* at = k ? other : base;
                    const Rgb top = mix_single(at + r.x * pitch, k ? fr : fl), low = mix_single(at + r.y * pitch, k ? fr : fl);
                    const float fy = __uint_as_float(r.z);
                    T* to = o + (swap ? kCols - 1 - k : k);
                    to[0] = from_f<T>(value(0, top.r, low.r, fy)); to[area] = from_f<T>(value(1, top.g, low.g, fy)); to[2 * area] = from_f<T>(value(2, top.b, low.b, fy));
                }
            }
        } else {
            for (int dy = 0; dy < p; ++dy, o += p)
                for (int k = 0; k < kCols; ++k) o[k] = o[k + area] = o[k + 2 * area] = from_f<T>(0.f);
        }
    }
    if (kDirect) return;
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
    if ((t | s.y | s.z | A.time_step) < 1 << 10) {          // as a rule: in 32 bits
        count = t * s.y * s.z;
        extent = t == 0 ? 0 : max((t - 1) * A.time_step, max(s.y, s.z) - 1) + 1;
        return;
    }
    const uint64_t plane = (uint64_t)(uint32_t)s.y * (uint32_t)s.z, most = (uint64_t)1 << 32;
    count = t == 0 ? 0 : (int64_t)min(min(plane, most) * (uint32_t)t, most);       // (more than any output holds)
    extent = t == 0 ? 0 : max((int64_t)(t - 1) * A.time_step, (int64_t)max(s.y, s.z) - 1) + 1;
}

// Positions of token number l of a segment that begins at position `base`.
__device__ __forceinline__ void position_in(const PositionArgs& A, const int4& s, int32_t base, uint32_t l, int32_t& pt, int32_t& ph, int32_t& pw) {
    if (s.y <= 0 || s.z <= 0) { pt = ph = pw = base + (int32_t)l; return; }
    const uint64_t plane = (uint64_t)(uint32_t)s.y * (uint32_t)s.z;
    uint32_t f = 0, rest = l, row, col;
    if (s.x > 1 && (plane >> 32) == 0) { f = quotient(l, (uint32_t)plane); rest = l - f * (uint32_t)plane; }
    const uint32_t m = (uint32_t)A.merge;
    if (m > 1 && s.y % A.merge == 0 && s.z % A.merge == 0) {
        const uint64_t band = (uint64_t)m * (uint32_t)s.z;
        const uint32_t block = band >> 32 ? 0 : quotient(rest, (uint32_t)band), in = rest - block * (uint32_t)band, side = quotient(in, m * m), q = in - side * (m * m);
        const uint32_t down = quotient(q, m);
        row = block * m + down; col = side * m + q - down * m;
    } else {
        row = quotient(rest, (uint32_t)s.z); col = rest - row * (uint32_t)s.z;
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

// Goes over this thread's share of the segments; put(i, first token, first position) is called for each.  Sequences' ends are
// written to A.next.
template <typename Put>
__device__ __forceinline__ int64_t walk_segments(const PositionArgs& A, Put put) {
    const int tid = threadIdx.x, n = A.n_segments, each = (int)(((int64_t)n + kScanThreads - 1) / kScanThreads);
    const int a = (int)min((int64_t)tid * each, (int64_t)n), b = (int)min((int64_t)a + each, (int64_t)n);
    const int32_t before = a > 0 && a < n ? A.segments[a - 1].w : -1;
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
        if ((i + 1 == n || A.segments[i + 1].w != s.w) && s.w >= 0 && s.w < A.n_sequences) A.next[s.w] = (int32_t)extent;
    }
    return total;
}

// Up to kFewSegments segments: every CTA works out where all of them begin, keeps that in shared memory and writes its own
// run of tokens.  One launch; the segments are read by every CTA, 16 bytes each, out of L2.  A thread finds its first token's
// segment by bisection and goes on from there.
// Latency and the sums that every CTA repeats bound it: 8704 segments of 1.4 million tokens 16 us, 72 segments 6 us; 16384 segments
// of 5 tokens 14 us, one more, by the two launches below, 39.
constexpr int kFewSegments = 16384, kRunTokens = 1024;
__global__ void __launch_bounds__(kScanThreads) positions_kernel(const __grid_constant__ PositionArgs A) {
    extern __shared__ uint2 s_begin[];                                    // (first token, first position)
    const int n = A.n_segments, tid = threadIdx.x;
    const bool ends = blockIdx.x + 1 == gridDim.x;                        // (the last CTA, behind all runs, writes the sequences' ends)
    if (ends)
        for (int i = tid; i < A.n_sequences; i += kScanThreads) A.next[i] = 0;
    for (int i0 = tid; i0 < n; i0 += 4 * kScanThreads) {                  // first: (tokens, and a mark where a sequence begins; positions)
        int4 s[4];
        int32_t before[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {                                     // (four on their way at a time)
            const int i = i0 + k * kScanThreads;
            if (i < n) { s[k] = A.segments[i]; before[k] = i > 0 ? A.segments[i - 1].w : ~s[k].w; }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * kScanThreads;
            if (i >= n) break;
            int64_t c, e;
            segment_sizes(A, s[k], c, e);
            const bool first = A.restart || before[k] != s[k].w;
            s_begin[i] = make_uint2((uint32_t)min(c, (int64_t)0x7fffffff) | (first ? 0x80000000u : 0u), (uint32_t)e);      // (no output has more tokens)
        }
    }
    __syncthreads();
    const int each = (n + kScanThreads - 1) / kScanThreads | 1, a = min(tid * each, n), b = min(a + each, n);       // (odd: no two lanes in one bank)
    int64_t tokens = 0, extent = 0, total;
    bool first = false;
    for (int i = a; i < b; ++i) {
        const uint2 s = s_begin[i];
        if (s.x >> 31) { first = true; extent = 0; }
        tokens += s.x & 0x7fffffffu; extent += s.y;
    }
    sums_before(tokens, extent, first, total);
    for (int i = a; i < b; ++i) {
        const uint2 s = s_begin[i];
        if (s.x >> 31) extent = 0;
        s_begin[i] = make_uint2((uint32_t)min(tokens, (int64_t)0xffffffff), (uint32_t)extent);
        tokens += s.x & 0x7fffffffu; extent += s.y;
    }
    __syncthreads();
    if (ends) {
#pragma unroll 4
        for (int i = tid; i < n; i += kScanThreads) {
            const int4 s = A.segments[i];
            const int32_t after = i + 1 < n ? A.segments[i + 1].w : ~s.w;
            int64_t c, e;
            segment_sizes(A, s, c, e);
            if (after != s.w && s.w >= 0 && s.w < A.n_sequences) A.next[s.w] = (int32_t)(s_begin[i].y + (uint32_t)e);
        }
    }
    // a warp a stretch of the run: its tokens are in one segment after the other
    const uint64_t stretch = A.run / (kScanThreads / 32), t0 = (uint64_t)blockIdx.x * A.run + (tid >> 5) * stretch, t1 = min(t0 + stretch, (uint64_t)A.n_tokens);
    int at = 0;                                                           // the segment at hand
    int4 s = make_int4(0, 0, 0, 0);
    uint2 from = make_uint2(0, 0);
    uint32_t behind = 0;                                                  // the first token behind it
    bool any = false;
    for (uint64_t tok = t0 + (tid & 31); tok < t1; tok += 32) {
        const uint32_t token = (uint32_t)tok;
        int32_t pt = 0, ph = 0, pw = 0;
        if ((int64_t)token < total) {
            if (!any || token >= behind) {
                int lo = at, hi = n;                                      // the last segment that begins at or before the token
                for (int near = 0; any && near < 4 && lo + 1 < hi; ++near) {
                    if (s_begin[lo + 1].x > token) { hi = lo + 1; break; }
                    ++lo;
                }
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_begin[mid].x <= token) lo = mid; else hi = mid;
                }
                at = lo; any = true;
                s = A.segments[at]; from = s_begin[at];
                behind = at + 1 < n ? s_begin[at + 1].x : 0xffffffffu;
            }
            position_in(A, s, (int32_t)from.y, token - from.x, pt, ph, pw);
        } else if (!A.zero_tail) {
            break;
        }
        A.positions[token] = pt; A.positions[A.stride + token] = ph; A.positions[2 * A.stride + token] = pw;
    }
}

// More segments: one CTA writes where each begins to device memory, then a thread a token looks its segment up there.  The one
// CTA's walk over the segments bounds it (most of 39 us for 16385 segments of 5 tokens, 45 of 50; 285 us for 100000); so many
// segments in one call are rare.
__global__ void __launch_bounds__(kScanThreads) position_scan_kernel(const __grid_constant__ PositionArgs A) {
    const int64_t total = walk_segments(A, [&](int i, int64_t token, int32_t position) { A.starts[i] = token; A.bases[i] = position; });
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
