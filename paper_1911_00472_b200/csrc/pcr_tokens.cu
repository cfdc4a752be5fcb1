// Host side of the operators between decoded pixels and a sequence model (see include/pcr.h): patch tokens, token
// positions, queries and keys turned by positions.  Every call checks its arguments, enqueues kernels on the caller's
// stream and returns; nothing is allocated and nothing is kept between calls.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>

#include "../../include/pcr.h"
#include "pcr_heads.cuh"
#include "pcr_launches.h"
#include "pcr_patches.cuh"
#include "pcr_spans.h"

using namespace pcr;

namespace {

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 148;
    }
    return n;
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t size_of(int dtype) { return dtype == PCR_F32 ? 4 : 2; }

int finish() { return cudaGetLastError() == cudaSuccess ? PCR_OK : PCR_E_CUDA; }

// Whether two elements of a strided output can be one and the same: sizes and strides sorted, each stride has to step
// over all that the smaller ones reach.
bool overlaps_itself(const int64_t (&stride)[3], int64_t batch, int64_t tokens, int64_t heads, int64_t dim) {
    const int64_t size[3] = {batch, tokens, heads};
    auto far = [&](int i) { const __int128 s = stride[i]; return s < 0 ? -s : s; };
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return far(a) < far(b); });
    __int128 reach = dim - 1;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (far(i) <= reach) return true;
        reach += (size[i] - 1) * far(i);
    }
    return false;
}

int check_heads(const pcr_turn_args& a, bool norm, bool back) {
    if (a.dtype != PCR_F16 && a.dtype != PCR_F32 && a.dtype != PCR_BF16) return PCR_E_ARG;
    if (a.batch < 0 || a.tokens < 0 || a.batch > INT32_MAX || a.tokens > INT32_MAX || a.batch * a.tokens > INT32_MAX) return PCR_E_ARG;
    if (a.head_dim < 1 || a.head_dim > kMaxHeadDim || a.rot_dim < 0 || a.rot_dim > a.head_dim || a.rot_dim % 2) return PCR_E_ARG;
    if (a.n_axes < 1 || a.n_axes > kMaxAxes || (a.interleaved & ~1) || (a.inverse & ~1)) return PCR_E_ARG;
    if (a.freq_dtype != PCR_F32 && a.freq_dtype != PCR_F64) return PCR_E_ARG;
    if (norm && (!(a.eps >= 0.f) || isinf(a.eps) || a.inverse || (a.weight_dtype != PCR_F32 && a.weight_dtype != a.dtype))) return PCR_E_ARG;
    if (a.q.heads < 0 || a.k.heads < 0 || a.q.heads > 65535 || a.k.heads > 65535 || a.q.heads + a.k.heads > 65535) return PCR_E_ARG;
    const size_t es = size_of(a.dtype), ws = size_of(a.weight_dtype);
    const bool any = a.batch * a.tokens > 0;
    if (any && (!a.positions || !aligned(a.positions, 4))) return PCR_E_ARG;
    if (any && a.rot_dim > 0 && (!a.inv_freq || !a.axes || !aligned(a.inv_freq, a.freq_dtype == PCR_F64 ? 8 : 4) || !aligned(a.axes, 4))) return PCR_E_ARG;
    for (const pcr_heads* h : {&a.q, &a.k}) {
        if (norm && (!aligned(h->weight, ws) || (back && (!aligned(h->dweight, ws) || (h->dweight && !h->weight))))) return PCR_E_ARG;
        if (!any || h->heads == 0) continue;
        if (!h->x || !h->y || !aligned(h->x, es) || !aligned(h->y, es) || (back && (!h->dy || !aligned(h->dy, es)))) return PCR_E_ARG;
        if (overlaps_itself(h->y_stride, a.batch, a.tokens, h->heads, a.head_dim)) return PCR_E_ARG;
    }
    return PCR_OK;
}

// Vectors of `v` elements: whether every row starts on one and the pairs fall into whole ones.
bool fits(const pcr_turn_args& a, bool back, int v) {
    if (a.head_dim % (2 * v) || a.rot_dim % (2 * v) || a.head_dim / (2 * v) > 32) return false;
    const size_t bytes = v * size_of(a.dtype);
    for (const pcr_heads* h : {&a.q, &a.k}) {
        if (h->heads == 0) continue;
        if (!aligned(h->x, bytes) || !aligned(h->y, bytes) || (back && !aligned(h->dy, bytes))) return false;
        const int64_t size[3] = {a.batch, a.tokens, h->heads};
        for (int i = 0; i < 3; ++i) {
            if (size[i] <= 1) continue;
            if (h->x_stride[i] % v || h->y_stride[i] % v || (back && h->dy_stride[i] % v)) return false;
        }
    }
    return true;
}

// How a call is cut: vectors of `v` pairs (0: value by value), lanes of a row, `per` heads of a token to a thread, the grid,
// and how many rows of partial sums each operand's weights get.
struct Cut { int v, lanes, per, slots[2], rows[2]; unsigned x, y; };

Cut cut_of(const pcr_turn_args& a, bool back) {
    Cut c = {};
    // the longest vectors that fit: 8192 tokens, 40 heads of 128, bf16, by 16 / 8 / 4 bytes and value by value: rotation 29, 31, 33 and 97 us,
    // norm 32, 39, 56 and 127, backward 50, 54, 69 and 385.  A row has 32 lanes of two vectors at most, so that heads of 32 bits
    // beyond 256 elements go value by value: 4096 tokens, 40 heads of 256: 55, 57 and 83 us, of 264: 119, 126 and 427.
    for (int v : {8, 4, 2})
        if (c.v == 0 && v * size_of(a.dtype) <= 16 && fits(a, back, v)) c.v = v;
    c.lanes = c.v ? a.head_dim / (2 * c.v) : 32;
    constexpr int kWarps = kHeadThreads / 32;
    const int64_t n = a.batch * a.tokens, heads = a.q.heads + a.k.heads, sms = sm_count();
    const int rows = 32 / c.lanes;       // tokens of a warp
    const int64_t warps = (n + rows - 1) / rows, groups = (warps + kWarps - 1) / kWarps;
    // Heads are shared out while that gives the SMs warps that they lack (forward 32 an SM: 8191 tokens, 40 heads, rotation: 16
    // an SM 36 us, 32 and 64 32 to 33; 16384 tokens of 5 heads, norm: 32 20.5 us, 64 22.6; backward 4: 514 tokens, 16 heads: 9.0 us,
    // all heads in one share 12.4), forward whole batches of rows to a share (8192 tokens, 40 heads of 128, norm: 39.0 -> 35.6 us)
    const int64_t want = sms * (back ? 4 : 32), shares = std::min<int64_t>((want + warps - 1) / warps, heads);
    c.per = (int)((heads + shares - 1) / shares);
    if (!back && c.v && c.per > kRowsAhead) c.per = (c.per + kRowsAhead - 1) / kRowsAhead * kRowsAhead;
    if (back && c.v) {
        // CTAs by the operands' heads: those of both end at about the same time
        const int ctas = kBackCtas(c.v * (int)size_of(a.dtype));
        const int64_t of[2] = {a.q.heads, a.k.heads};
        for (int i = 0; i < 2; ++i) {
            const int64_t cuts = (of[i] + c.per - 1) / c.per;           // shares of this operand; whole rounds of them
            c.slots[i] = cuts == 0 ? 0 : (int)(cuts * std::min(groups, std::max<int64_t>(1, (sms * ctas * of[i] + heads * cuts / 2) / (heads * cuts))));
        }
        c.x = c.slots[0] + c.slots[1]; c.y = 1;
        c.rows[0] = c.slots[0]; c.rows[1] = c.slots[1];
    } else {
        c.slots[0] = (a.q.heads + c.per - 1) / c.per;
        c.slots[1] = (a.k.heads + c.per - 1) / c.per;
        c.y = c.v ? (unsigned)((heads + c.per - 1) / c.per) : (unsigned)(c.slots[0] + c.slots[1]);
        c.x = (unsigned)(back ? std::min<int64_t>(groups, std::max<int64_t>(sms * 8 / c.y, 1)) : groups);
        c.rows[0] = c.slots[0] * c.x; c.rows[1] = c.slots[1] * c.x;
    }
    return c;
}

void fill(HeadArgs& A, const pcr_turn_args& a, const Cut& c) {
    const pcr_heads* from[2] = {&a.q, &a.k};
    for (int i = 0; i < 2; ++i) {
        HeadBlock& H = A.part[i];
        const pcr_heads& h = *from[i];
        H.x = h.x; H.y = h.y; H.g = h.dy; H.weight = h.weight; H.partial = nullptr;
        for (int j = 0; j < 3; ++j) { H.xs[j] = h.x_stride[j]; H.ys[j] = h.y_stride[j]; H.gs[j] = h.dy_stride[j]; A.ps[j] = a.position_stride[j]; }
        H.heads = h.heads; H.slots = c.slots[i];
    }
    A.positions = a.positions; A.inv_freq = a.inv_freq; A.axes = a.axes;
    A.tokens = (uint32_t)(a.batch * a.tokens); A.seq = (uint32_t)std::max<int64_t>(a.tokens, 1);
    A.n_axes = a.n_axes; A.freq64 = a.freq_dtype == PCR_F64; A.weight32 = a.weight_dtype == PCR_F32; A.inverse = a.inverse;
    A.dim = a.head_dim; A.rot = a.rot_dim; A.lanes = c.lanes; A.per = c.per;
    A.eps = a.eps; A.inv_dim = 1.f / (float)a.head_dim;
}

template <typename T, int V, int kMode, bool kNext>
void launch_vectors(const HeadArgs& A, dim3 grid, cudaStream_t st) {
    if constexpr (kMode == kNormTurnBack) {
        const int steps = steps_of(A.lanes);
        auto with = [&](auto kernel) { kernel<<<grid, kHeadThreads, 0, st>>>(A); };
        if (steps == 2) return with(heads_back_kernel<T, V, kNext, 2>);
        if (steps == 3) return with(heads_back_kernel<T, V, kNext, 3>);
        if (steps == 4) return with(heads_back_kernel<T, V, kNext, 4>);
        if (steps == 5) return with(heads_back_kernel<T, V, kNext, 5>);
        if (steps == -3) return with(heads_back_kernel<T, V, kNext, -3>);
        if (steps == -4) return with(heads_back_kernel<T, V, kNext, -4>);
        if (steps == -5) return with(heads_back_kernel<T, V, kNext, -5>);
        with(heads_back_kernel<T, V, kNext, 0>);
    } else heads_kernel<T, V, kMode == kNormTurn, kNext><<<grid, kHeadThreads, 0, st>>>(A);
}

template <typename T, int kMode, bool kNext>
void launch(const HeadArgs& A, const Cut& c, cudaStream_t st) {
    const dim3 grid(c.x, c.y);
    if (sizeof(T) == 2 && c.v == 8) launch_vectors<T, sizeof(T) == 2 ? 8 : 4, kMode, kNext>(A, grid, st);
    else if (c.v == 4) launch_vectors<T, 4, kMode, kNext>(A, grid, st);
    else if (c.v == 2) launch_vectors<T, 2, kMode, kNext>(A, grid, st);
    else heads_any_kernel<T, kMode, kNext><<<grid, kHeadThreads, 0, st>>>(A);
    ++g_launches;
}

template <int kMode>
void launch_mode(const HeadArgs& A, const Cut& c, int dtype, bool next, cudaStream_t st) {
    if (dtype == PCR_F16) { if (next) launch<__half, kMode, true>(A, c, st); else launch<__half, kMode, false>(A, c, st); }
    else if (dtype == PCR_BF16) { if (next) launch<__nv_bfloat16, kMode, true>(A, c, st); else launch<__nv_bfloat16, kMode, false>(A, c, st); }
    else { if (next) launch<float, kMode, true>(A, c, st); else launch<float, kMode, false>(A, c, st); }
}

template <typename T>
void launch_patches(const PatchArgs& A, bool pairs, bool direct, unsigned grid, int warps, size_t own, cudaStream_t st) {
    if (direct) patch_tokens_kernel<T, 2, true><<<grid, 32 * warps, 0, st>>>(A);
    else if (pairs) patch_tokens_kernel<T, 2, false><<<grid, 32 * warps, own * warps, st>>>(A);
    else patch_tokens_kernel<T, 1, false><<<grid, 32 * warps, own * warps, st>>>(A);
}

size_t scratch_bytes_of(const pcr_turn_args& a, const Cut& c) { return ((size_t)c.rows[0] + c.rows[1]) * a.head_dim * sizeof(float); }
bool nothing(const pcr_turn_args& a) { return a.batch * a.tokens == 0 || a.q.heads + a.k.heads == 0; }

// Whether an output shares memory with another output or with an operand, other than an operand's own output that lies just
// where it (or its gradient) does: kernels read and write in no order that a caller could count on.  A weight's gradient may
// lie on what is read: it is written when all of that is done.
bool outputs_shared(const pcr_turn_args& a, bool norm, bool back, const void* scratch, size_t scratch_bytes) {
    const size_t es = size_of(a.dtype), ws = size_of(a.weight_dtype);
    const pcr_heads* of[2] = {&a.q, &a.k};
    const int reads = back ? 2 : 1;
    Span y[2], x[2][2], held[5], late[2];                            // outputs; operands and gradients; what else is read; weights' gradients
    int n_held = 0, n_late = 0;
    for (int i = 0; i < 2; ++i) {
        const pcr_heads& h = *of[i];
        auto heads = [&](const void* p, const int64_t (&stride)[3]) { return span_of(p, stride, a.batch, a.tokens, h.heads, a.head_dim, es); };
        y[i] = heads(h.y, h.y_stride);
        x[i][0] = heads(h.x, h.x_stride);
        x[i][1] = heads(h.dy, h.dy_stride);
        if (norm && h.weight) held[n_held++] = span_of(h.weight, a.head_dim * ws);
        if (back && h.dweight) late[n_late++] = span_of(h.dweight, a.head_dim * ws);
    }
    held[n_held++] = span_of(a.positions, a.position_stride, a.n_axes, a.batch, a.tokens, 1, sizeof(int32_t));
    held[n_held++] = span_of(a.inv_freq, a.rot_dim / 2 * (a.freq_dtype == PCR_F64 ? 8 : 4));
    held[n_held++] = span_of(a.axes, a.rot_dim / 2 * sizeof(int32_t));
    auto same = [](const Span& s, const Span& t) {
        for (int i = 0; i < 3; ++i)
            if (s.n[i] > 1 && s.step[i] != t.step[i]) return false;
        return s.at == t.at;
    };
    auto any = [](const Span& s, const Span* t, int n) { return std::any_of(t, t + n, [&](const Span& u) { return share_memory(s, u); }); };
    for (int i = 0; i < 2; ++i) {
        for (int j = 0; j < 2; ++j)
            for (int r = 0; r < reads; ++r)
                if (!(i == j && same(y[i], x[j][r])) && share_memory(y[i], x[j][r])) return true;
        if (any(y[i], held, n_held) || any(y[i], late, n_late)) return true;
    }
    if (share_memory(y[0], y[1]) || (n_late == 2 && share_memory(late[0], late[1]))) return true;
    if (n_late == 0) return false;
    const Span s = span_of(scratch, scratch_bytes);
    return any(s, y, 2) || any(s, x[0], 2) || any(s, x[1], 2) || any(s, held, n_held) || any(s, late, n_late);
}

}  // namespace

extern "C" {

int pcr_rotate(const pcr_turn_args* args, void* stream) {
    if (!args) return PCR_E_ARG;
    if (int rc = check_heads(*args, false, false)) return rc;
    if (nothing(*args)) return PCR_OK;
    if (outputs_shared(*args, false, false, nullptr, 0)) return PCR_E_ARG;
    const Cut c = cut_of(*args, false);
    HeadArgs A;
    fill(A, *args, c);
    launch_mode<kTurn>(A, c, args->dtype, args->interleaved != 0, static_cast<cudaStream_t>(stream));
    return finish();
}

int pcr_norm_rotate(const pcr_turn_args* args, void* stream) {
    if (!args) return PCR_E_ARG;
    if (int rc = check_heads(*args, true, false)) return rc;
    if (nothing(*args)) return PCR_OK;
    if (outputs_shared(*args, true, false, nullptr, 0)) return PCR_E_ARG;
    const Cut c = cut_of(*args, false);
    HeadArgs A;
    fill(A, *args, c);
    launch_mode<kNormTurn>(A, c, args->dtype, args->interleaved != 0, static_cast<cudaStream_t>(stream));
    return finish();
}

size_t pcr_norm_rotate_scratch_bytes(const pcr_turn_args* args) {
    if (!args || check_heads(*args, true, true) != PCR_OK || nothing(*args)) return 0;
    return scratch_bytes_of(*args, cut_of(*args, true));
}

int pcr_norm_rotate_backward(const pcr_turn_args* args, void* scratch, void* stream) {
    if (!args) return PCR_E_ARG;
    if (int rc = check_heads(*args, true, true)) return rc;
    const bool sums = args->q.dweight || args->k.dweight;
    if (sums && !nothing(*args) && (!scratch || !aligned(scratch, 4))) return PCR_E_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    WeightSums S = {{nullptr, nullptr}, {args->q.dweight, args->k.dweight}, {0, 0}, args->head_dim, args->weight_dtype == PCR_F32};
    if (!nothing(*args)) {
        const Cut c = cut_of(*args, true);
        if (outputs_shared(*args, true, true, scratch, scratch_bytes_of(*args, c))) return PCR_E_ARG;
        HeadArgs A;
        fill(A, *args, c);
        float* at = static_cast<float*>(scratch);
        for (int i = 0; i < 2; ++i) {
            if (S.dw[i]) { A.part[i].partial = at; S.partial[i] = at; S.rows[i] = c.rows[i]; }
            if (at) at += (size_t)c.rows[i] * args->head_dim;
        }
        launch_mode<kNormTurnBack>(A, c, args->dtype, args->interleaved != 0, st);
    }
    if (sums) {
        const dim3 grid((unsigned)((args->head_dim + kSumCols - 1) / kSumCols), 2);
        cudaLaunchConfig_t config = {};
        config.gridDim = grid; config.blockDim = dim3(kSumThreads); config.stream = st;
        cudaLaunchAttribute early;
        early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        early.val.programmaticStreamSerializationAllowed = 1;
        config.attrs = &early; config.numAttrs = nothing(*args) ? 0 : 1;
        if (args->dtype == PCR_F16) cudaLaunchKernelEx(&config, weight_sums_kernel<__half>, S);
        else if (args->dtype == PCR_BF16) cudaLaunchKernelEx(&config, weight_sums_kernel<__nv_bfloat16>, S);
        else cudaLaunchKernelEx(&config, weight_sums_kernel<float>, S);
        ++g_launches;
    }
    return finish();
}

int pcr_patch_tokens(const void* rgb, size_t rgb_bytes, const pcr_patch_image* images, int n_images, const int32_t* index,
                     int64_t n_tokens, int patch, int merge, const float* mean, const float* std_, int dtype, void* tokens, void* stream) {
    static_assert(sizeof(pcr_patch_image) == sizeof(PatchImage), "pcr_patch_image and PatchImage have the same layout");
    if (n_images < 0 || n_tokens < 0 || n_tokens > INT32_MAX || patch < 1 || patch > kMaxPatch || merge < 1 || merge > 64) return PCR_E_ARG;
    if (!mean || !std_ || (dtype != PCR_F16 && dtype != PCR_F32 && dtype != PCR_BF16)) return PCR_E_ARG;
    for (int c = 0; c < 3; ++c)
        if (!(std_[c] > 0.f) || !(fabsf(mean[c]) <= 3.0e38f) || !isnormal(1.f / (255.f * std_[c]))) return PCR_E_ARG;
    if (n_tokens == 0) return PCR_OK;
    if ((n_images > 0 && (!rgb || !images)) || !index || !tokens) return PCR_E_ARG;
    if (!aligned(rgb, 4) || !aligned(images, 16) || !aligned(index, 8) || !aligned(tokens, size_of(dtype))) return PCR_E_ARG;
    const Span rows = span_of(tokens, (size_t)n_tokens * 3 * patch * patch * size_of(dtype));
    if (share_memory(rows, span_of(rgb, rgb_bytes)) || share_memory(rows, span_of(images, (size_t)n_images * sizeof(PatchImage))) ||
        share_memory(rows, span_of(index, (size_t)n_tokens * sizeof(int2)))) return PCR_E_ARG;
    PatchArgs A;
    A.rgb = static_cast<const uint8_t*>(rgb); A.images = reinterpret_cast<const PatchImage*>(images);
    A.index = reinterpret_cast<const int2*>(index); A.out = tokens; A.rgb_bytes = rgb_bytes;
    A.n_tokens = (uint32_t)n_tokens; A.n_images = n_images; A.patch = patch; A.merge = merge;
    for (int c = 0; c < 3; ++c) { A.scale[c] = 1.f / (255.f * std_[c]); A.shift[c] = -mean[c] / std_[c]; }
    const bool pairs = patch % 2 == 0;                         // two columns to a lane
    // Lanes write their values as they come, or through shared memory as whole vectors.  As they come where a patch's rows are
    // whole sectors of 32 bytes (400 images, patches of 16, 16 bits: 155 us, through shared memory 178; 96 images, of 16, 32
    // bits: 43 and 60); 16 bits also beyond patches of 16, whose values would leave shared memory for few warps (300 images,
    // of 28: 103 and 130).  Else rows share sectors, and shared memory makes up for it (1024 images, of 14, 16 bits: 431 and
    // 405; 300 images, of 14, 32 bits: 211 and 164).
    const bool direct = pairs && aligned(tokens, 32) && (patch * size_of(dtype) % 32 == 0 || (dtype != PCR_F32 && patch > 16));
    const int lanes = pairs ? patch / 2 : patch;
    A.each = 32 / lanes; A.by_lanes = (65536u + lanes - 1) / lanes; A.by_merge = ((1u << 20) + merge - 1) / merge;
    const size_t own = ((size_t)A.each * 3 * patch * patch * size_of(dtype) + 15) / 16 * 16;
    const int64_t warps = (n_tokens + A.each - 1) / A.each;
    int in_cta = kPatchWarps;                                  // fewer where their values would not fit into shared memory
    while (!direct && in_cta > 1 && own * in_cta > 32 * 1024) in_cta /= 2;
    const unsigned grid = (unsigned)((warps + in_cta - 1) / in_cta);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == PCR_F16) launch_patches<__half>(A, pairs, direct, grid, in_cta, own, st);
    else if (dtype == PCR_BF16) launch_patches<__nv_bfloat16>(A, pairs, direct, grid, in_cta, own, st);
    else launch_patches<float>(A, pairs, direct, grid, in_cta, own, st);
    ++g_launches;
    return finish();
}

size_t pcr_token_positions_scratch_bytes(int n_segments) { return n_segments <= kFewSegments ? 0 : ((size_t)n_segments + 1) * 12 + 16; }

int pcr_token_positions(const int32_t* segments, int n_segments, int64_t n_tokens, int n_sequences, int merge, int time_step,
                        int flags, int32_t* positions, int64_t axis_stride, int32_t* next, void* scratch, void* stream) {
    if (n_segments < 0 || n_sequences < 0 || n_tokens < 0 || n_tokens > INT32_MAX || merge < 1 || merge > 64) return PCR_E_ARG;
    if (time_step < 0 || time_step > (1 << 20) || (flags & ~(PCR_POSITIONS_RESTART | PCR_POSITIONS_ZERO_TAIL))) return PCR_E_ARG;
    if ((n_segments > 0 && !segments) || (n_tokens > 0 && !positions) || (n_sequences > 0 && !next) || (n_segments > kFewSegments && !scratch)) return PCR_E_ARG;
    if (!aligned(segments, 16) || !aligned(positions, 4) || !aligned(next, 4) || !aligned(scratch, 8)) return PCR_E_ARG;
    if (n_tokens > 0 && axis_stride < n_tokens) return PCR_E_ARG;
    const Span read = span_of(segments, (size_t)n_segments * sizeof(int4)), ends = span_of(next, (size_t)n_sequences * 4),
               rows = span_of(positions, {axis_stride, 0, 0}, 3, 1, 1, n_tokens, 4), own = span_of(scratch, n_segments > kFewSegments ? pcr_token_positions_scratch_bytes(n_segments) : 0);
    if (share_memory(rows, read) || share_memory(ends, read) || share_memory(rows, ends) || share_memory(own, read) || share_memory(own, ends) || share_memory(own, rows)) return PCR_E_ARG;
    PositionArgs A;
    A.segments = reinterpret_cast<const int4*>(segments);
    A.starts = static_cast<int64_t*>(scratch);
    A.bases = reinterpret_cast<int32_t*>(A.starts + n_segments + 1);
    A.positions = positions; A.next = next; A.stride = axis_stride; A.n_tokens = (uint32_t)n_tokens; A.run = 0;
    A.n_segments = n_segments; A.n_sequences = n_sequences; A.merge = merge; A.time_step = time_step;
    A.restart = (flags & PCR_POSITIONS_RESTART) != 0; A.zero_tail = (flags & PCR_POSITIONS_ZERO_TAIL) != 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_segments <= kFewSegments) {
        const size_t shared = (size_t)n_segments * sizeof(uint2);
        // a CTA an SM, as each adds all segments up (4000 segments of 1.04 million tokens: 10.3 us, two CTAs an SM 14.4; 300 of 290914: 6.2, 8.3)
        const int64_t runs = std::min<int64_t>(std::max<int64_t>((n_tokens + kRunTokens - 1) / kRunTokens, 1), std::max(sm_count() - 1, 1));
        A.run = (uint32_t)(((n_tokens + runs - 1) / runs + kScanThreads - 1) / kScanThreads * kScanThreads);      // whole rounds of every warp
        // (always the same limit: calls from several host threads set it side by side)
        if (shared > 40 * 1024 && cudaFuncSetAttribute(positions_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSegments * (int)sizeof(uint2)) != cudaSuccess) {
            cudaGetLastError();
            return PCR_E_CUDA;
        }
        positions_kernel<<<(unsigned)runs + 1, kScanThreads, shared, st>>>(A);
        ++g_launches;
        return finish();
    }
    position_scan_kernel<<<1, kScanThreads, 0, st>>>(A);
    ++g_launches;
    if (n_tokens > 0) {
        position_fill_kernel<<<(unsigned)((n_tokens + kFillThreads - 1) / kFillThreads), kFillThreads, 0, st>>>(A);
        ++g_launches;
    }
    return finish();
}

}  // extern "C"
