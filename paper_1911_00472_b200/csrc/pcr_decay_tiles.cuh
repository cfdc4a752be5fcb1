// Walks of 16-bit operands on the tensor cores (see pcr_walks.h for what a walk is).
//
// A CTA takes a segment of a sequence and a head, 128 tokens at a time, with the tiles A, B, C of a chunk in shared memory and
// all products in tensor memory:
//
//   S = A B^T                       128 x 128     masked and faded on the way to P, which goes back to tensor memory in 16 bits
//   O = P C                         128 x cd      what the chunk's own tokens add
//   I = A R                         128 x cd      what the memory adds; y = O + f^(distance) I
//   D = C^T B'                      cd x bd       what the chunk adds to the memory: B' = rows of B times their factors
//
// The memory itself stays in the registers of one warpgroup, in 32 bits, a column of it (an element of c) to a thread; its 16-bit image
// is the other operand of I.  B' is kept in two parts, x = hi + lo, three where the memory is given out in 32 bits and 16 bits of each
// would show; they take the places of B, A and of the memory's image, which S and I are done with by then.  So the roundings
// to 16 bits are P's, the image's and the output's, each half a step at most.  fp16 has few exponents: rows of P and of
// the image are brought to about 2^14 by a power of two, which is taken off again behind the product.
//
// 10 warps: four turn S into P and write y (a thread a row), four make B' and keep the memory, one asks for tiles (TMA), one issues
// the products.  What bounds it: DRAM, 4 tiles of 32 KB a chunk at 1/148 of the copy rate are 2.9 us; the products are 3072 cycles, the
// warps' work about as much, side by side.
#pragma once
#include <cuda.h>

#include "pcr_walks.h"

namespace pcr {

constexpr int kTileThreads = 320;
constexpr int kTile = 128;                     // tokens of a chunk
constexpr int kHalf = 16384;                   // bytes of 128 rows of 64 elements

struct TileMaps { CUtensorMap q, k, v, g; };   // (element, head, token, batch): boxes of 64 elements, 128 tokens
struct TileArgs {
    TileMaps maps;
    WalkArgs walks;
    int of[3][3];                              // which map is a, b, c of a walk
    int parts;                                 // of B'
};

// Shared memory of a CTA, from a boundary of 1024 bytes on.
template <int DB> struct TileShared {
    static constexpr int kSide = DB / 64 * kHalf;              // A, B, the image of the memory
    static constexpr int kStage = 2 * kSide + 2 * kHalf;
    static constexpr int kStages = DB == 64 ? 3 : 2;
    static constexpr int kImage = kStages * kStage;
    static constexpr int kRest = kImage + kSide;
    static constexpr int kBytes = kRest + 2048 + 1024;         // (and what the boundary may take)
};

struct TileBars { uint64_t full[3], empty[3], s, i, p, k, o, d, e, r, end; };

__device__ __forceinline__ uint32_t at_shared(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(at_shared(b)), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(at_shared(b)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(at_shared(b)), "r"(bytes) : "memory");
}
// Waits for the phase of that parity to end, for two seconds at most: false if it gave up, or if another thread did before.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* dead) {
    uint64_t begin = 0;
    for (uint32_t tries = 1;; ++tries) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(at_shared(b)), "r"(parity) : "memory");
        if (done) return true;
        if (tries % 256) continue;
        uint64_t now;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
        if (!begin) begin = now;
        if (*dead) return false;
        if (now - begin > 2000000000ull) { *dead = 1; return false; }
    }
}
// The same for a whole warp: all of its lanes go on, together, or none.
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t parity, volatile int* dead) { return __all_sync(~0u, bar_wait(b, parity, dead)); }
__device__ __forceinline__ void tile_load(void* to, const CUtensorMap* map, uint64_t* bar, int x, int head, int token, int batch) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(at_shared(to)),
                 "l"(map), "r"(at_shared(bar)), "r"(x), "r"(head), "r"(token), "r"(batch) : "memory");
}
// Descriptors of tiles in rows of 128 bytes whose 16-byte pieces are turned by the row's number modulo 8.  Rows along the tile's own
// dimension (M or N), 64 elements of the summed one in a row: groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t at) { return (uint64_t)((at & 0x3ffff) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61; }
// Rows along the summed dimension, 64 elements of M or N in a row: groups of 8 rows 1024 bytes apart, the next 64 elements kHalf.
__device__ __forceinline__ uint64_t desc_cols(uint32_t at) { return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)(kHalf >> 4) << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61; }
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t how, bool add) {       // A in tensor memory
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(at_shared(b)) : "memory");
}
__device__ __forceinline__ void order_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void order_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void order_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }   // own writes, before products read them
__device__ __forceinline__ void tensor_load32(float (&v)[32], uint32_t at) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
                 "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tensor_load16(float (&v)[16], uint32_t at) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tensor_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tensor_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> {
    static constexpr uint32_t kHow = 1u << 4 | 1u << 7 | 1u << 10;             // 32-bit sums of bf16
    __device__ static uint32_t pack(float a, float b) { __nv_bfloat162 x = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&x); }
    __device__ static float2 open(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&w)); }
};
template <> struct Two<__half> {
    static constexpr uint32_t kHow = 1u << 4;
    __device__ static uint32_t pack(float a, float b) { __half2 x = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&x); }
    __device__ static float2 open(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
};
// 2^14 / a power of two about as large as `most`, and what takes it off again
__device__ __forceinline__ float2 to_middle(float most) {
    const int e = min(max((int)(__float_as_uint(most) >> 23 & 255), 15), 250);
    return {__uint_as_float((uint32_t)(127 + 14 + 127 - e) << 23), __uint_as_float((uint32_t)(e - 14) << 23)};
}

// Outputs of a chunk's rows in which some value is not finite, once more: masked tokens leave no trace (0 * inf is none), so what is not
// finite is added up again over the tokens that a row sees.  Rare, and slow.
template <typename T>
__device__ __noinline__ void careful(const WalkArgs& A, const Walk& W, const Item& it, int head, int64_t t0, int n, int r, float rate, float age, uint32_t O, uint32_t I,
                                     float off, const float* cs, int64_t to) {
    const T* a = static_cast<const T*>(W.a.at) + (int64_t)it.batch * W.a.st[0] + (t0 + r) * W.a.st[1] + (int64_t)(head / W.a.group) * W.a.st[2];
    const T* b = static_cast<const T*>(W.b.at) + (int64_t)it.batch * W.b.st[0] + t0 * W.b.st[1] + (int64_t)(head / W.b.group) * W.b.st[2];
    const T* c = static_cast<const T*>(W.c.at) + (int64_t)it.batch * W.c.st[0] + t0 * W.c.st[1] + (int64_t)(head / W.c.group) * W.c.st[2];
    for (int j0 = 0; j0 < W.cd; j0 += 16) {
        float o[16], m[16];
        tensor_load16(o, O + j0);
        tensor_load16(m, I + j0);
        tensor_load_wait();
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            m[j] *= (cs ? cs[j0 + j] : 1.f) * age;
            if (j0 + j < W.cd && r < n && !isfinite(o[j] * off + m[j])) odd |= 1u << j;
        }
        for (int q = W.rev ? r : 0; odd && q <= (W.rev ? n - 1 : r); ++q) {
            float s = 0.f;
            for (int d = 0; d < W.bd; ++d) s += to_float(a[d]) * to_float(b[q * W.b.st[1] + d]);
            s *= power(rate, W.rev ? q - r : r - q);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (odd >> j & 1) m[j] += s * to_float(c[q * W.c.st[1] + j0 + j]);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (odd >> j & 1) {
                if (W.y32) static_cast<float*>(W.y)[to + j0 + j] = m[j];
                else static_cast<T*>(W.y)[to + j0 + j] = from_float<T>(m[j]);
            }
        __syncwarp();
    }
}

template <typename T, int DB, bool kStates>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(const __grid_constant__ TileArgs G) {
    extern __shared__ uint8_t raw[];
    using L = TileShared<DB>;
    constexpr int kStages = L::kStages;
    constexpr bool kHalfs = sizeof(T) == 2 && Two<T>::kHow == 1u << 4;
    const WalkArgs& A = G.walks;
    const int kind = blockIdx.z, head = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Walk& W = A.w[kind];
    if (!kStates) zero_tail(A, W, W.y32 ? 4 : 2, blockIdx.x, gridDim.x, head);
    Item it;
    if (!item_of(A, W.rev, blockIdx.x, it)) return;
    if (kStates && it.last) return;
    const int bd = W.bd, cd = W.cd;
    const size_t of = (size_t)bd * cd;
    if (it.len == 0) {                                                     // the memory as it came
        if (!kStates && W.last)
            for (int e = tid; e < (int)of; e += kTileThreads) {
                const int i = e / cd, j = e % cd;
                W.last[((size_t)it.seq * A.heads + head) * of + i * W.li + j * W.lj] = W.first ? W.first[((size_t)it.seq * A.heads + head) * of + i * W.fi + j * W.fj] : 0.f;
            }
        return;
    }
    uint8_t* sm = raw + (-at_shared(raw) & 1023);
    float* pw = reinterpret_cast<float*>(sm + L::kRest);                   // powers of the factor, 0 .. 128
    float* cs = pw + 132;                                                  // fp16: what the image's columns were brought up by, two chunks
    TileBars* bars = reinterpret_cast<TileBars*>(cs + 256);
    uint32_t* tensor = reinterpret_cast<uint32_t*>(bars + 1);
    volatile int* dead = reinterpret_cast<volatile int*>(tensor + 1);
    const float rate = rate_of(A.log_decay, head);
    const int chunks = (it.n + kTile - 1) / kTile;

    for (int i = tid; i <= kTile; i += kTileThreads) pw[i] = power(rate, i);
    if (cd <= 64)                                                          // columns that no copy writes
        for (int s = 0; s < kStages; ++s)
            for (int i = tid; i < kHalf / 16; i += kTileThreads) reinterpret_cast<uint4*>(sm + s * L::kStage + 2 * L::kSide + kHalf)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { bar_init(&bars->full[s], 1); bar_init(&bars->empty[s], 1); }
        for (uint64_t* b : {&bars->s, &bars->i, &bars->o, &bars->d, &bars->end}) bar_init(b, 1);
        for (uint64_t* b : {&bars->p, &bars->k, &bars->e, &bars->r}) bar_init(b, 128);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at_shared(tensor)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    order_shared();
    order_before();
    __syncthreads();
    order_after();
    const uint32_t tm = *tensor, S = tm, O = tm + 128, I = tm + 256, D = tm + 384, mine = (uint32_t)(warp & 3) << 21;       // (a warp's 32 lanes)
    // the chunk's first token and its tokens
    auto chunk = [&](int c, int64_t& t0, int& n) {
        const int at = it.from + c * kTile;
        n = min(kTile, it.from + it.n - at);
        t0 = it.begin + (W.rev ? it.len - at - n : at);
    };

    if (warp == 8) {
        if (lane == 0) {
            const CUtensorMap* all = &G.maps.q;
            const CUtensorMap *ma = all + G.of[kind][0], *mb = all + G.of[kind][1], *mc = all + G.of[kind][2];
            const int ha = head / W.a.group, hb = head / W.b.group, hc = head / W.c.group;
            const uint32_t bytes = (kStates ? 1 : 2) * L::kSide + (cd > 64 ? 2 : 1) * kHalf;
            int c = 0;
            for (; c < chunks; ++c) {
                const int s = c % kStages;
                if (c >= kStages && !bar_wait(&bars->empty[s], (c / kStages - 1) & 1, dead)) break;
                int64_t t0;
                int n;
                chunk(c, t0, n);
                uint8_t* to = sm + s * L::kStage;
                bar_expect(&bars->full[s], bytes);
#pragma unroll
                for (int h = 0; h < DB / 64; ++h) {
                    if (!kStates) tile_load(to + h * kHalf, ma, &bars->full[s], 64 * h, ha, (int)t0, it.batch);
                    tile_load(to + L::kSide + h * kHalf, mb, &bars->full[s], 64 * h, hb, (int)t0, it.batch);
                }
                for (int h = 0; h < (cd > 64 ? 2 : 1); ++h) tile_load(to + 2 * L::kSide + h * kHalf, mc, &bars->full[s], 64 * h, hc, (int)t0, it.batch);
            }
            volatile int again = 0;                                        // copies still under way write here: none may be left
            for (int i = max(0, c - kStages); i < c; ++i) bar_wait(&bars->full[i % kStages], (i / kStages) & 1, &again);
        }
    } else if (warp == 9) {
        if (lane == 0) {
            const uint32_t how = Two<T>::kHow, m128 = 8u << 24, cd16 = (uint32_t)(cd + 15) / 16, bd16 = (uint32_t)(bd + 15) / 16;
            const uint32_t how_s = how | m128 | 16u << 17, how_i = how | m128 | 2 * cd16 << 17, how_o = how_i | 1u << 16, how_d = how | m128 | 1u << 15 | 1u << 16 | 2 * bd16 << 17;
            for (int c = 0; c < chunks; ++c) {
                const int s = c % kStages, ph = c & 1;
                int64_t t0;
                int n;
                chunk(c, t0, n);
                const uint32_t a = at_shared(sm + s * L::kStage), b = a + L::kSide, v = a + 2 * L::kSide, image = at_shared(sm + L::kImage);
                const uint32_t steps = (uint32_t)(n + 15) / 16;            // of the chunk's tokens
                auto part = [&](uint32_t k) { return (k >> 2) * kHalf + (k & 3) * 32; };        // 16 elements on along a row
                if (!bar_wait(&bars->full[s], (c / kStages) & 1, dead)) break;
                if (!kStates) {
                    if (c > 0 && !bar_wait(&bars->o, ph ^ 1, dead)) break;                     // (P lies where S goes)
                    for (uint32_t k = 0; k < bd16; ++k) mma(S, desc_rows(a + part(k)), desc_rows(b + part(k)), how_s, k > 0);
                    mma_commit(&bars->s);
                    if (!bar_wait(&bars->r, ph, dead) || (c > 0 && !bar_wait(&bars->e, ph ^ 1, dead))) break;
                    order_after();
                    for (uint32_t k = 0; k < bd16; ++k) mma(I, desc_rows(a + part(k)), desc_rows(image + part(k)), how_i, k > 0);
                    mma_commit(&bars->i);
                    if (n < kTile && !bar_wait(&bars->k, ph, dead)) break;                     // (rows behind the last token are cleared by then)
                    if (!bar_wait(&bars->p, ph, dead)) break;
                    order_after();
                    for (uint32_t k = 0; k < steps; ++k) mma_tensor(O, S + 8 * k, desc_cols(v + 2048 * k), how_o, k > 0);
                    mma_commit(&bars->o);
                } else if (!bar_wait(&bars->r, ph, dead)) break;                               // (D of the chunk before has been read)
                if (!bar_wait(&bars->k, ph, dead)) break;
                order_after();
                const uint32_t from[3] = {b, a, image};
                for (int p = G.parts - 1; p >= 0; --p)                     // the small parts first
                    for (uint32_t k = 0; k < steps; ++k) mma(D, desc_cols(v + 2048 * k), desc_cols(from[p] + 2048 * k), how_d, p < G.parts - 1 || k > 0);
                mma_commit(&bars->d);
                mma_commit(&bars->empty[s]);
            }
            volatile int again = 0;
            mma_commit(&bars->end);
            bar_wait(&bars->end, 0, &again);
        }
    } else if (warp < 4) {
        if (!kStates) {
            const int r = tid;
            for (int c = 0; c < chunks; ++c) {
                const int ph = c & 1;
                int64_t t0;
                int n;
                chunk(c, t0, n);
                if (!warp_wait(&bars->s, ph, dead)) break;
                order_after();
                float off = 1.f;                                           // fp16: what brings the row of O back
                // Group g of 32 columns of S becomes 16 words of P, which lie where group g / 2 was: in this order none is lost.
                auto faded = [&](float (&p)[32], int g) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int q = 32 * g + j, far = W.rev ? q - r : r - q;
                        p[j] = far >= 0 && q < n ? p[j] * pw[far < 0 ? 0 : far] : 0.f;
                    }
                };
                float on = 1.f;
                if (kHalfs) {
                    float most = 0.f;
#pragma unroll 1
                    for (int g = 0; g < 4; ++g) {
                        if (W.rev ? g < warp : g > warp) continue;         // (a warp's rows see no group beyond their own)
                        float p[32];
                        tensor_load32(p, S + mine + 32 * g);
                        tensor_load_wait();
                        faded(p, g);
#pragma unroll
                        for (int j = 0; j < 32; ++j) most = fmaxf(most, fabsf(p[j]));
                    }
                    const float2 f = to_middle(most);
                    on = f.x; off = f.y;
                }
#pragma unroll 1
                for (int g = 0; g < 4; ++g) {
                    uint32_t w[16] = {};
                    if (W.rev ? g >= warp : g <= warp) {
                        float p[32];
                        tensor_load32(p, S + mine + 32 * g);
                        tensor_load_wait();
                        faded(p, g);
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = kHalfs ? Two<T>::pack(on * p[2 * j], on * p[2 * j + 1]) : Two<T>::pack(p[2 * j], p[2 * j + 1]);
                    }
                    tensor_store16(S + mine + 16 * g, w);
                }
                tensor_store_wait();
                order_before();
                if (kHalfs && !warp_wait(&bars->r, ph, dead)) break;           // (before D can be asked for, which r's next phase comes after)
                bar_arrive(&bars->p);
                if (!warp_wait(&bars->o, ph, dead)) break;
                order_after();
                const float age = r < n ? pw[W.rev ? n - 1 - r : r] : 0.f;
                const int64_t to = (int64_t)it.batch * W.ys[0] + (t0 + r) * W.ys[1] + (int64_t)head * W.ys[2];
                bool odd = false;
                for (int j0 = 0; j0 < cd; j0 += 16) {
                    float o[16], m[16];
                    tensor_load16(o, O + mine + j0);
                    tensor_load16(m, I + mine + j0);
                    tensor_load_wait();
                    if (kHalfs) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) { o[j] *= off; m[j] *= cs[ph * 128 + j0 + j]; }
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        o[j] += age * m[j];
                        odd |= !isfinite(o[j]);
                    }
                    if (r < n) {
                        if (W.y32) {
                            float4* y = reinterpret_cast<float4*>(static_cast<float*>(W.y) + to + j0);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (j0 + 4 * e < cd) y[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        } else {
                            uint4* y = reinterpret_cast<uint4*>(static_cast<T*>(W.y) + to + j0);
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (j0 + 8 * e < cd)
                                    y[e] = make_uint4(Two<T>::pack(o[8 * e], o[8 * e + 1]), Two<T>::pack(o[8 * e + 2], o[8 * e + 3]), Two<T>::pack(o[8 * e + 4], o[8 * e + 5]), Two<T>::pack(o[8 * e + 6], o[8 * e + 7]));
                        }
                    }
                }
                if (__any_sync(~0u, odd && r < n)) careful<T>(A, W, it, head, t0, n, r, rate, age, O + mine, I + mine, off, kHalfs ? cs + ph * 128 : nullptr, to);
                order_before();
                bar_arrive(&bars->e);
            }
        }
    } else {
        const int r = tid - 128;                                           // an element of c; a token of B'
        const bool on = r < cd;
        float R[DB];
        {
            const float* from = nullptr;
            int64_t fi = 0, fj = 0;
            float age = 1.f;
            if (!kStates && on) {
                if (it.m > 0) { from = W.slots + ((size_t)(it.slot - 1) * A.heads + head) * of; fi = W.si; fj = W.sj; }
                else if (W.first) { from = W.first + ((size_t)it.seq * A.heads + head) * of; fi = W.fi; fj = W.fj; age = W.rev ? 1.f : power(rate, 1); }
            }
#pragma unroll
            for (int i = 0; i < DB; ++i) R[i] = from && i < bd ? age * from[i * fi + r * fj] : 0.f;
        }
        uint8_t* image = sm + L::kImage;
        auto write_image = [&](int ph) {
            float up = 1.f;
            if (kHalfs) {
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < DB; ++i) most = fmaxf(most, fabsf(R[i]));
                const float2 f = to_middle(most);
                up = f.x;
                cs[ph * 128 + r] = f.y;
            }
#pragma unroll
            for (int i = 0; i < DB; i += 8) {
                uint4 w;
                w.x = Two<T>::pack(up * R[i], up * R[i + 1]); w.y = Two<T>::pack(up * R[i + 2], up * R[i + 3]);
                w.z = Two<T>::pack(up * R[i + 4], up * R[i + 5]); w.w = Two<T>::pack(up * R[i + 6], up * R[i + 7]);
                *reinterpret_cast<uint4*>(image + (i >> 6) * kHalf + r * 128 + (((i >> 3) & 7) ^ (r & 7)) * 16) = w;
            }
            order_shared();
        };
        if (!kStates) write_image(0);
        bar_arrive(&bars->r);
        int c = 0;
        for (; c < chunks; ++c) {
            const int s = c % kStages, ph = c & 1;
            int64_t t0;
            int n;
            chunk(c, t0, n);
            const bool final = !kStates && it.last && c == chunks - 1 && !W.rev;       // forward, the memory that is given out is not aged
            if (!warp_wait(&bars->full[s], (c / kStages) & 1, dead) || (!kStates && !warp_wait(&bars->i, ph, dead))) break;
            uint8_t *a = sm + s * L::kStage, *b = a + L::kSide, *v = a + 2 * L::kSide;
            const bool in = r < n;
            const float w = in ? pw[(W.rev ? r + 1 : n - r) - (final ? 1 : 0)] : 0.f;
#pragma unroll 4
            for (int i = 0; i < DB; i += 8) {
                const int at = (i >> 6) * kHalf + r * 128 + (((i >> 3) & 7) ^ (r & 7)) * 16;
                uint4 x = *reinterpret_cast<const uint4*>(b + at), hi, lo, last;
                uint32_t *px = &x.x, *ph_ = &hi.x, *pl = &lo.x, *pt = &last.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float2 f = Two<T>::open(px[e]);
                    f.x = in ? f.x * w : 0.f;
                    f.y = in ? f.y * w : 0.f;
                    ph_[e] = Two<T>::pack(f.x, f.y);
                    float2 g = Two<T>::open(ph_[e]);
                    f.x -= g.x; f.y -= g.y;
                    pl[e] = Two<T>::pack(f.x, f.y);
                    g = Two<T>::open(pl[e]);
                    pt[e] = Two<T>::pack(f.x - g.x, f.y - g.y);
                }
                *reinterpret_cast<uint4*>(b + at) = hi;
                if (G.parts > 1) *reinterpret_cast<uint4*>(a + at) = lo;
                if (G.parts > 2) *reinterpret_cast<uint4*>(image + at) = last;
            }
            if (!in)
                for (int i = 0; i < 16; ++i) *reinterpret_cast<uint4*>(v + (i >> 3) * kHalf + r * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
            order_shared();
            bar_arrive(&bars->k);
            if (!warp_wait(&bars->d, ph, dead)) break;
            order_after();
            const float keep = pw[final ? n - 1 : n];
#pragma unroll
            for (int i = 0; i < DB; i += 16) {
                if (i >= bd) continue;                                     // (nothing was put there)
                float x[16];
                tensor_load16(x, D + mine + i);
                tensor_load_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) R[i + j] = keep * R[i + j] + x[j];
            }
            if (!kStates && c + 1 < chunks) write_image((c + 1) & 1);
            order_before();
            bar_arrive(&bars->r);
        }
        float* out = nullptr;
        int64_t oi = 0, oj = 0;
        if (kStates) { out = W.slots + ((size_t)it.slot * A.heads + head) * of; oi = W.si; oj = W.sj; }
        else if (it.last && W.last) { out = W.last + ((size_t)it.seq * A.heads + head) * of; oi = W.li; oj = W.lj; }
        if (out && on) {
#pragma unroll
            for (int i = 0; i < DB; ++i)
                if (i < bd) out[i * oi + r * oj] = c == chunks ? R[i] : __int_as_float(0x7fc00000);
        }
    }
    __syncwarp();
    order_before();
    __syncthreads();
    order_after();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
    if (!kStates && *dead && warp < 4)                                     // a wait that ran out does not go unnoticed
        for (int t = tid; t < it.n; t += 128) {
            const int64_t row = it.begin + (W.rev ? it.len - it.from - it.n : it.from) + t, to = (int64_t)it.batch * W.ys[0] + row * W.ys[1] + (int64_t)head * W.ys[2];
            for (int j = 0; j < cd; ++j) {
                if (W.y32) static_cast<float*>(W.y)[to + j] = __int_as_float(0x7fc00000);
                else static_cast<uint16_t*>(W.y)[to + j] = 0x7fff;
            }
        }
}

}  // namespace pcr
