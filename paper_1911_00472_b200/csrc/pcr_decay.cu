// Host side of linear attention with a decay for each head (see include/pcr.h): checks, choice of form, launches.  Nothing is
// allocated and nothing is kept between calls.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/pcr.h"
#include "pcr_decay.cuh"
#include "pcr_decay_tiles.h"
#include "pcr_launches.h"
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

// Whether two elements of a strided output can be one and the same: sizes and strides sorted, each stride has to step over all
// that the smaller ones reach.
bool overlaps_itself(const int64_t* stride, std::initializer_list<int64_t> sizes, int64_t dim) {
    int64_t size[3], far[3];
    int n = 0;
    for (int64_t s : sizes) {
        if (s > 1) { size[n] = s; far[n++] = *stride < 0 ? -*stride : *stride; }
        ++stride;
    }
    __int128 reach = dim - 1;
    for (int done = 0; done < n; ++done) {
        const int least = (int)(std::min_element(far + done, far + n) - far);
        std::swap(far[done], far[least]); std::swap(size[done], size[least]);
        if (far[done] <= reach) return true;
        reach += (__int128)(size[done] - 1) * far[done];
    }
    return false;
}

bool heads_fit(int q_heads, int k_heads, int k_dim, int v_dim, int dtype) {
    return q_heads >= 1 && k_heads >= 1 && q_heads <= 65535 && q_heads % k_heads == 0 && k_dim >= 1 && v_dim >= 1 && k_dim <= kMaxDecayDim &&
           v_dim <= kMaxDecayDim && (dtype == PCR_F16 || dtype == PCR_F32 || dtype == PCR_BF16);
}

constexpr uint32_t kNever = UINT32_MAX, kTestPatience = 1000000;           // (nanoseconds, where waits are to run out)

struct Form {
    bool tiles;                                 // on the tensor cores
    int chunk, parts;                           // tokens of a chunk; 16-bit parts of what goes into a memory
    uint32_t seg, keys, slots;                  // tokens of a segment; segments to look for; memories of segments to keep
    bool split;                                 // whether a sequence may have several segments
    size_t slot_bytes, shared_bytes;            // of one direction's memories; of the gradients that heads share
};

// (rows of no sequence may have to become 0 all the same)
bool nothing(const pcr_decay_args& a) { return a.sequences == 0 && !(a.starts && a.tokens > 0 && (a.flags & PCR_DECAY_ZERO_TAIL)); }

Form form_of(const pcr_decay_args& a, bool back) {
    Form f = {};
    const int most = std::max(a.k_dim, a.v_dim);
    // (on the tensor cores wherever operands allow it: four prompts of 61 tokens 8.0 us for 31.9, 32768 tokens 465 for 8760)
    f.tiles = a.sequences > 0 && tiles_fit(a, back);
    f.chunk = f.tiles ? 128 : most > 128 ? 32 : 64;
    // two parts of bf16 hold 16 bits of a value, which an output of 16 bits does not show; a memory that is given out would
    f.parts = a.dtype == PCR_BF16 && (a.state_after || a.dstate) ? 3 : 2;
    // Segments of equal length, as many of a sequence as end first by this count, in halves of a chunk's time: rounds of CTAs times their
    // chunks and a CTA's beginning and end (a chunk; two where chunks are short, on the tensor cores), and for several segments half as much again
    // and two more launches (a chunk of the plain kernel takes 14 us, one on the tensor cores 3.5).  Packed sequences are taken to be of
    // equal length.  (Two CTAs an SM of the plain kernel: heads of 104 to 128 and of 200 and more ask for 113 KB of shared memory and more each, so
    // that one fits, and their rounds are too few here; not measured.)
    const int64_t wide = (int64_t)a.q_heads * (back ? 3 : 1) * (f.tiles ? 1 : (most + kWalkCols - 1) / kWalkCols) * a.sequences;
    const int64_t room = (int64_t)sm_count() * (f.tiles ? 1 : 2), mean = std::max<int64_t>(1, a.batch * a.tokens / std::max<int64_t>(1, a.sequences)), whole = (mean + f.chunk - 1) / f.chunk;
    int64_t best = 1, least = INT64_MAX;
    for (int64_t per = 1; per <= std::min<int64_t>(whole, 64); ++per) {
        const int64_t chunks = (whole + per - 1) / per, ends = f.tiles ? 2 : 1, rounds = (wide * per + room - 1) / room, less = (wide * (per - 1) + room - 1) / room;
        const int64_t cost = 2 * rounds * (chunks + ends) + (per > 1 ? less * (chunks + ends) + (f.tiles ? 8 : 2) : 0);
        if (cost < least) { least = cost; best = per; }
    }
    int64_t seg = (whole + best - 1) / best * f.chunk;
    // a sequence much longer than the others is cut all the same, but for four chunks not at all
    if (a.starts) seg = std::max<int64_t>({seg, ((wide * whole / room + 1) / 2) * f.chunk, (int64_t)4 * f.chunk});
    seg = std::min<int64_t>(seg, std::max<int64_t>((a.tokens + f.chunk - 1) / f.chunk, 1) * f.chunk);
    f.seg = (uint32_t)seg;
    f.split = a.tokens > seg;
    if (a.starts) { f.keys = (uint32_t)std::max<int64_t>(1, a.sequences + a.tokens / seg); f.slots = f.split ? (uint32_t)(a.tokens / seg) : 0; }
    else {
        const int64_t per = std::max<int64_t>((a.tokens + seg - 1) / seg, 1);
        f.keys = (uint32_t)(a.batch * per); f.slots = (uint32_t)(a.batch * (per - 1));
    }
    f.slot_bytes = (size_t)f.slots * a.q_heads * a.k_dim * a.v_dim * sizeof(float);
    f.shared_bytes = back && a.q_heads != a.k_heads ? (size_t)a.batch * a.tokens * a.q_heads * (a.k_dim + a.v_dim) * sizeof(float) : 0;
    return f;
}
size_t scratch_of(const Form& f, bool back) { return f.slot_bytes * (back ? 2 : 1) + f.shared_bytes; }

int check(const pcr_decay_args& a, bool back) {
    if (!heads_fit(a.q_heads, a.k_heads, a.k_dim, a.v_dim, a.dtype) || (a.flags & ~PCR_DECAY_ZERO_TAIL)) return PCR_E_ARG;
    if (a.batch < 0 || a.tokens < 0 || a.batch > INT32_MAX || a.tokens > INT32_MAX || a.batch * a.tokens > INT32_MAX) return PCR_E_ARG;
    if (a.sequences < 0 || a.sequences >= 1 << 24 || (a.starts ? a.batch != 1 : a.sequences != a.batch)) return PCR_E_ARG;
    if (nothing(a)) return PCR_OK;
    if (!a.log_decay || !aligned(a.log_decay, 4) || !aligned(a.starts, 4) || !aligned(a.state, 4) || !aligned(a.state_after, 4) ||
        !aligned(a.dstate_after, 4) || !aligned(a.dstate, 4)) return PCR_E_ARG;
    const size_t es = size_of(a.dtype);
    if (a.batch * a.tokens > 0) {
        for (const pcr_rows* r : {&a.q, &a.k, &a.v, &a.out}) if (!r->at || !aligned(r->at, es)) return PCR_E_ARG;
        if (back) for (const pcr_rows* r : {&a.dq, &a.dk, &a.dv}) if (!r->at || !aligned(r->at, es)) return PCR_E_ARG;
        if (!back && overlaps_itself(a.out.stride, {a.batch, a.tokens, a.q_heads}, a.v_dim)) return PCR_E_ARG;
        if (back && (overlaps_itself(a.dq.stride, {a.batch, a.tokens, a.q_heads}, a.k_dim) || overlaps_itself(a.dk.stride, {a.batch, a.tokens, a.k_heads}, a.k_dim) ||
                     overlaps_itself(a.dv.stride, {a.batch, a.tokens, a.k_heads}, a.v_dim))) return PCR_E_ARG;
    }
    return PCR_OK;
}

// Whether an output (or the scratch memory) shares memory with anything else.
bool shares(const pcr_decay_args& a, bool back, const void* scratch, size_t scratch_bytes) {
    const size_t es = size_of(a.dtype), state = (size_t)a.sequences * a.q_heads * a.k_dim * a.v_dim * sizeof(float);
    Span in[8], out[5];
    int n_in = 0, n_out = 0;
    auto rows = [&](const pcr_rows& r, int heads, int dim) { return span_of(r.at, r.stride, a.batch, a.tokens, heads, dim, es); };
    auto plain = [&](const void* p, size_t bytes) { return span_of(p, p ? bytes : 0); };
    in[n_in++] = rows(a.q, a.q_heads, a.k_dim);
    in[n_in++] = rows(a.k, a.k_heads, a.k_dim);
    in[n_in++] = rows(a.v, a.k_heads, a.v_dim);
    in[n_in++] = plain(a.log_decay, a.q_heads * sizeof(float));
    in[n_in++] = plain(a.starts, (a.sequences + 1) * sizeof(int32_t));
    in[n_in++] = plain(a.state, state);
    if (back) {
        in[n_in++] = rows(a.out, a.q_heads, a.v_dim);
        in[n_in++] = plain(a.dstate_after, state);
        out[n_out++] = rows(a.dq, a.q_heads, a.k_dim);
        out[n_out++] = rows(a.dk, a.k_heads, a.k_dim);
        out[n_out++] = rows(a.dv, a.k_heads, a.v_dim);
        out[n_out++] = plain(a.dstate, state);
    } else {
        out[n_out++] = rows(a.out, a.q_heads, a.v_dim);
        out[n_out++] = plain(a.state_after, state);
    }
    out[n_out++] = plain(scratch, scratch_bytes);
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < i; ++j) if (share_memory(out[i], out[j])) return true;
        for (int j = 0; j < n_in; ++j) if (share_memory(out[i], in[j])) return true;
    }
    return false;
}

WalkRows walk_rows(const pcr_rows& r, int group) {
    WalkRows w = {r.at, {r.stride[0], r.stride[1], r.stride[2]}, group};
    return w;
}
void walk_out(Walk& w, const pcr_rows& r) {
    w.y = const_cast<void*>(r.at);
    for (int i = 0; i < 3; ++i) w.ys[i] = r.stride[i];
}

template <typename T, int kRows>
int launch_walk(const WalkArgs& A, unsigned keys, cudaStream_t st) {
    int bd = 0, cd = 0;
    for (int i = 0; i < A.kinds; ++i) { bd = std::max(bd, A.w[i].bd); cd = std::max(cd, A.w[i].cd); }
    const size_t shared = walk_shared(bd, kRows);
    if (shared > 48 * 1024 &&                   // (always the same limit: calls from several host threads set it side by side)
        cudaFuncSetAttribute(walk_kernel<T, kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)walk_shared(kRows == 64 ? 128 : kMaxDecayDim, kRows)) != cudaSuccess) {
        cudaGetLastError();
        return PCR_E_CUDA;
    }
    const dim3 grid(keys, A.heads, A.kinds * ((cd + kWalkCols - 1) / kWalkCols));
    walk_kernel<T, kRows><<<grid, kWalkThreads, shared, st>>>(A);
    ++g_launches;
    return finish();
}
template <typename T>
int launch_rows(const WalkArgs& A, const Form& f, cudaStream_t st) {
    return f.chunk == 64 ? launch_walk<T, 64>(A, f.keys, st) : launch_walk<T, 32>(A, f.keys, st);
}
int launch_any(const WalkArgs& A, const Form& f, int dtype, cudaStream_t st) {
    if (dtype == PCR_F16) return launch_rows<__half>(A, f, st);
    if (dtype == PCR_BF16) return launch_rows<__nv_bfloat16>(A, f, st);
    return launch_rows<float>(A, f, st);
}

// What segments add, the memories before them, and the walks themselves.  `of`: which of q, k, v, out are a, b, c of each.
int run(WalkArgs& states, const int (*states_of)[3], WalkArgs& walks, const int (*walks_of)[3], const Form& f, const pcr_decay_args& a, cudaStream_t st) {
    if (f.split) {
        states.states = 1;
        if (int rc = f.tiles ? launch_tiles(states, states_of, a, f.keys, f.parts, sm_count(), st) : launch_any(states, f, a.dtype, st)) return rc;
        int of = 0;
        for (int i = 0; i < states.kinds; ++i) of = std::max(of, states.w[i].bd * states.w[i].cd);
        // (memories begin at 16 bytes where they are whole vectors; several heads to a CTA where sequences alone give CTAs enough)
        const int blocks = (of + 1023) / 1024;
        const unsigned heads = (unsigned)std::min<int64_t>(states.heads, std::max<int64_t>(1, 8 * sm_count() / ((int64_t)states.sequences * blocks)));
        const dim3 grid(states.sequences, heads, states.kinds * blocks);
        if (of % 4 == 0) walk_scan_kernel<4><<<grid, 256, 0, st>>>(states);
        else walk_scan_kernel<1><<<grid, 256, 0, st>>>(states);
        ++g_launches;
        if (int rc = finish()) return rc;
    }
    walks.states = 0;
    return f.tiles ? launch_tiles(walks, walks_of, a, f.keys, f.parts, sm_count(), st) : launch_any(walks, f, a.dtype, st);
}

// `stop`: chunks after which the copies of tiles of a CTA stop, so that its waits run out; kNever
WalkArgs common(const pcr_decay_args& a, const Form& f, uint32_t stop) {
    WalkArgs A = {};
    A.log_decay = a.log_decay; A.starts = a.starts; A.sequences = (uint32_t)a.sequences; A.tokens = (uint32_t)a.tokens;
    A.seg = f.seg; A.heads = a.q_heads; A.limit = stop == kNever ? kPatience : kTestPatience; A.stop = stop;
    return A;
}

int forward(const pcr_decay_args& a, void* scratch, void* stream, uint32_t stop) {
    if (int rc = check(a, false)) return rc;
    if (nothing(a)) return PCR_OK;
    const Form f = form_of(a, false);
    const size_t need = scratch_of(f, false);
    if ((need && !scratch) || !aligned(scratch, 16) || shares(a, false, scratch, need)) return PCR_E_ARG;
    const int group = a.q_heads / a.k_heads;
    if (stop != kNever && !f.tiles) return PCR_E_ARG;
    WalkArgs A = common(a, f, stop);
    Walk& w = A.w[0];
    A.kinds = 1;
    w.a = walk_rows(a.q, 1); w.b = walk_rows(a.k, group); w.c = walk_rows(a.v, group);
    walk_out(w, a.out);
    w.bd = a.k_dim; w.cd = a.v_dim; w.zero_tail = (a.flags & PCR_DECAY_ZERO_TAIL) != 0;
    w.first = a.state; w.last = a.state_after; w.slots = static_cast<float*>(scratch);
    w.fi = w.li = w.si = a.v_dim; w.fj = w.lj = w.sj = 1;
    WalkArgs S = A;
    const int of[3][3] = {{0, 1, 2}};
    return run(S, of, A, of, f, a, static_cast<cudaStream_t>(stream));
}

int backward(const pcr_decay_args& a, void* scratch, void* stream, uint32_t stop) {
    if (int rc = check(a, true)) return rc;
    if (nothing(a)) return PCR_OK;
    const Form f = form_of(a, true);
    const size_t need = scratch_of(f, true);
    if ((need && !scratch) || !aligned(scratch, 16) || shares(a, true, scratch, need)) return PCR_E_ARG;
    const int group = a.q_heads / a.k_heads, zero = (a.flags & PCR_DECAY_ZERO_TAIL) != 0;
    float* const slots = static_cast<float*>(scratch);
    float* const slots_back = slots + f.slot_bytes / sizeof(float);
    float* const dk32 = slots_back + f.slot_bytes / sizeof(float);
    float* const dv32 = dk32 + (size_t)a.batch * a.tokens * a.q_heads * a.k_dim;
    const WalkRows q = walk_rows(a.q, 1), k = walk_rows(a.k, group), v = walk_rows(a.v, group), g = walk_rows(a.out, 1);

    if (stop != kNever && !f.tiles) return PCR_E_ARG;
    WalkArgs S = common(a, f, stop), A = S;
    S.kinds = 2;                                // the memories from either end, as (k_dim, v_dim)
    S.w[0].b = k; S.w[0].c = v; S.w[0].first = a.state; S.w[0].slots = slots;
    S.w[1].b = q; S.w[1].c = g; S.w[1].first = a.dstate_after; S.w[1].slots = slots_back; S.w[1].rev = 1;
    for (int i = 0; i < 2; ++i) {
        Walk& w = S.w[i];
        w.a = w.b; w.bd = a.k_dim; w.cd = a.v_dim; w.fi = w.si = a.v_dim; w.fj = w.sj = 1;
    }
    A.kinds = 3;
    Walk &dq = A.w[0], &dk = A.w[1], &dv = A.w[2];
    dq.a = g; dq.b = v; dq.c = k; dq.first = a.state; dq.slots = slots;
    dk.a = v; dk.b = g; dk.c = q; dk.first = a.dstate_after; dk.slots = slots_back;
    dv.a = k; dv.b = q; dv.c = g; dv.first = a.dstate_after; dv.slots = slots_back; dv.last = a.dstate;
    dk.rev = dv.rev = 1;
    dq.bd = dk.bd = a.v_dim; dq.cd = dk.cd = a.k_dim; dv.bd = a.k_dim; dv.cd = a.v_dim;
    for (Walk* w : {&dq, &dk}) { w->fi = w->si = 1; w->fj = w->sj = a.v_dim; }          // (b's and c's sizes change places)
    dv.fi = dv.si = dv.li = a.v_dim; dv.fj = dv.sj = dv.lj = 1;
    walk_out(dq, a.dq); walk_out(dk, a.dk); walk_out(dv, a.dv);
    dq.zero_tail = dk.zero_tail = dv.zero_tail = zero;
    if (group > 1) {
        const int dims[2] = {a.k_dim, a.v_dim};
        Walk* of[2] = {&dk, &dv};
        for (int i = 0; i < 2; ++i) {
            of[i]->y = i ? dv32 : dk32; of[i]->y32 = 1; of[i]->zero_tail = 0;
            of[i]->ys[2] = dims[i]; of[i]->ys[1] = (int64_t)a.q_heads * dims[i]; of[i]->ys[0] = a.tokens * of[i]->ys[1];
        }
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int states_of[3][3] = {{1, 1, 2}, {0, 0, 3}}, walks_of[3][3] = {{3, 2, 1}, {2, 3, 0}, {1, 0, 3}};
    if (int rc = run(S, states_of, A, walks_of, f, a, st)) return rc;
    if (group > 1 && a.batch * a.tokens > 0) {
        GroupSum G[2];
        int64_t most = 0;
        for (int i = 0; i < 2; ++i) {
            const pcr_rows& r = i ? a.dv : a.dk;
            G[i] = {i ? dv32 : dk32, const_cast<void*>(r.at), {r.stride[0], r.stride[1], r.stride[2]}, a.tokens, a.batch * a.tokens, a.q_heads, group, i ? a.v_dim : a.k_dim};
            most = std::max<int64_t>(most, a.batch * a.tokens * a.k_heads * G[i].dim);
        }
        const dim3 grid((unsigned)std::min<int64_t>((most + 255) / 256, (int64_t)sm_count() * 32), 2);
        const int n = (int)a.sequences;
        if (a.dtype == PCR_F16) group_sum_kernel<__half><<<grid, 256, 0, st>>>(G[0], G[1], a.starts, n, zero);
        else if (a.dtype == PCR_BF16) group_sum_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(G[0], G[1], a.starts, n, zero);
        else group_sum_kernel<float><<<grid, 256, 0, st>>>(G[0], G[1], a.starts, n, zero);
        ++g_launches;
    }
    return finish();
}

}  // namespace

extern "C" {

size_t pcr_decay_scratch_bytes(const pcr_decay_args* args, int backward) {
    if (!args || check(*args, backward != 0) != PCR_OK || nothing(*args)) return 0;
    return scratch_of(form_of(*args, backward != 0), backward != 0);
}

int pcr_decay_attention(const pcr_decay_args* args, void* scratch, void* stream) { return args ? forward(*args, scratch, stream, kNever) : PCR_E_ARG; }

int pcr_decay_attention_backward(const pcr_decay_args* args, void* scratch, void* stream) { return args ? backward(*args, scratch, stream, kNever) : PCR_E_ARG; }

int pcr_selftest_decay_waits(const pcr_decay_args* args, int back, void* scratch, uint32_t after, void* stream) {
    if (!args || after == kNever) return PCR_E_ARG;
    return back ? backward(*args, scratch, stream, after) : forward(*args, scratch, stream, after);
}

int pcr_decay_step(const pcr_decay_step_args* args, void* stream) {
    if (!args) return PCR_E_ARG;
    const pcr_decay_step_args& a = *args;
    if (!heads_fit(a.q_heads, a.k_heads, a.k_dim, a.v_dim, a.dtype) || a.rows < 0 || a.rows >= 1 << 24 || a.n_slots < 0 || a.n_slots > INT32_MAX) return PCR_E_ARG;
    if (!a.slots && a.n_slots < a.rows) return PCR_E_ARG;
    if (a.rows == 0) return PCR_OK;
    const size_t es = size_of(a.dtype);
    if (!a.q || !a.k || !a.v || !a.out || !a.log_decay || (!a.state && a.n_slots > 0)) return PCR_E_ARG;
    if (!aligned(a.q, es) || !aligned(a.k, es) || !aligned(a.v, es) || !aligned(a.out, es) || !aligned(a.log_decay, 4) || !aligned(a.state, 4) || !aligned(a.slots, 4)) return PCR_E_ARG;
    if (overlaps_itself(a.out_stride, {a.rows, a.q_heads}, a.v_dim)) return PCR_E_ARG;
    auto rows = [&](const void* p, const int64_t (&s)[2], int heads, int dim) { return span_of(p, {s[0], s[1], 0}, a.rows, heads, 1, dim, es); };
    const Span out = rows(a.out, a.out_stride, a.q_heads, a.v_dim), state = span_of(a.state, (size_t)a.n_slots * a.q_heads * a.k_dim * a.v_dim * sizeof(float));
    const Span in[] = {rows(a.q, a.q_stride, a.q_heads, a.k_dim), rows(a.k, a.k_stride, a.k_heads, a.k_dim), rows(a.v, a.v_stride, a.k_heads, a.v_dim),
                       span_of(a.log_decay, a.q_heads * sizeof(float)), span_of(a.slots, a.slots ? a.rows * sizeof(int32_t) : 0)};
    if (share_memory(out, state)) return PCR_E_ARG;
    for (const Span& s : in) if (share_memory(out, s) || share_memory(state, s)) return PCR_E_ARG;
    StepArgs A = {};
    A.q = a.q; A.k = a.k; A.v = a.v; A.out = a.out;
    for (int i = 0; i < 2; ++i) { A.qs[i] = a.q_stride[i]; A.ks[i] = a.k_stride[i]; A.vs[i] = a.v_stride[i]; A.os[i] = a.out_stride[i]; }
    A.state = a.state; A.slots = a.slots; A.log_decay = a.log_decay;
    A.rows = (int)a.rows; A.n_slots = (int)a.n_slots; A.q_heads = a.q_heads; A.group = a.q_heads / a.k_heads; A.kd = a.k_dim; A.vd = a.v_dim;
    const bool four = a.v_dim % 4 == 0 && aligned(a.state, 16);
    // Columns of a CTA: all, fewer where that leaves SMs idle, as long as 16 KB of memory are left for each (one request, 4 heads of 256: 8.6 us whole,
    // 3.1 cut; 8 requests, 32 heads of 64, 16 KB each: 4.6 whole, 6.8 cut).
    int cols = four ? (a.v_dim + 31) / 32 * 32 : a.v_dim;
    while (cols > 32 && a.k_dim * cols > 8191 && a.rows * a.q_heads * ((a.v_dim + cols - 1) / cols) < 4 * sm_count()) cols = four ? (cols / 2 + 3) / 4 * 4 : (cols + 1) / 2;
    A.cols = cols;
    A.splits = (a.v_dim + cols - 1) / cols;
    const dim3 grid((unsigned)(a.rows * A.splits), a.q_heads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto four_at_once, auto one) { if (four) four_at_once<<<grid, kStepThreads, 0, st>>>(A); else one<<<grid, kStepThreads, 0, st>>>(A); };
    if (a.dtype == PCR_F16) launch(step_kernel<__half, 4>, step_kernel<__half, 1>);
    else if (a.dtype == PCR_BF16) launch(step_kernel<__nv_bfloat16, 4>, step_kernel<__nv_bfloat16, 1>);
    else launch(step_kernel<float, 4>, step_kernel<float, 1>);
    ++g_launches;
    return finish();
}

}  // extern "C"
