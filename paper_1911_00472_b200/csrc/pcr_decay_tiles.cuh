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
// would show; hi takes B's place, which S is done with by then, a third the image's.  So the roundings to 16 bits are P's, the image's
// and the output's, each half a step at most.  fp16 has few exponents: rows of P, of the image and all of a chunk's B' are brought to about 2^14 by a
// power of two, which is taken off again behind the product.
//
// 16 warps: four turn S into P and write y (a thread a row), four keep the memory, four make B', one asks for tiles (TMA), one issues the
// products, one asks for work: a CTA that is done with a segment takes the next one that no CTA has begun (the launch's own queue; what
// segments add is dealt out), so that copies of its first tiles go on under the end of the one before.  Tiles lie in a ring, each is
// given back by itself.  From one chunk to the next there are two chains: B' and D; and the memory's sum, its image and I.  P, O and the
// next S go beside them.
// Code is kept short and in loops where it can be: the roles' code runs side by side on every scheduler, and what is unrolled comes out of
// the instruction caches at 4 to 8 cycles an instruction.
//
// What bounds it, heads of 128, cycles a chunk: DRAM, 4 tiles of 32 KB at 1/148 of the copy rate, 5500; shared memory (operands of
// products 2250, copies 770, the warps' loads and stores 1300) 4300; the products 2560.  A chunk takes 6500 to 7000: the chain of B', D, the
// memory's sum, its image and I, each waiting for the one before.  Rows of y are written by the lane that has them, 53 cycles a store; warps
// of their own for y (257 us for the gradients below, 407 for the images) and y through shared memory (245, 413) were not faster.
//
// Measured: 32768 tokens, 32 heads of 128, bf16, memories given and taken: 174 us what segments add, 277 the walk (1.07 GB: 164 at the copy rate);
// whole sequences in the place of segments 1456, the plain kernel 8740.  Gradients of 4 x 4096 tokens, 16 heads of 128, 240 us (floor 72; plain 5680),
// in fp16 302.  96 packed images of 729 tokens, 16 heads of 72 in fp16, 419 us (floor 98; plain 2170).  Four prompts of 61 tokens 8.0 us (plain 31.9).
// Of these, exactness costs 2 % in bf16 (looking for what is not finite in what a chunk adds) and, in fp16, 26 us of the images (the largest product of
// a chunk's B' and of a row of P as it is faded); products by twos (f32x2) took 20 of them back.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "pcr_walks.h"

namespace pcr {

constexpr int kTileThreads = 512;
constexpr int kTile = 128;                     // tokens of a chunk
constexpr int kHalf = 16384;                   // bytes of 128 rows of 64 elements

struct TileMaps { CUtensorMap q, k, v, g; };   // (element, head, token, batch): boxes of 64 elements, 128 tokens
struct TileArgs {
    TileMaps maps;
    WalkArgs walks;
    int of[3][3];                              // which map is a, b, c of a walk
    int parts;                                 // of B'
    uint32_t items;                            // segments (of every head and walk) to look at
};

// Shared memory of a CTA, from a boundary of 1024 bytes on: a ring of tiles, the memory's image, lo.  A chunk's tiles are A, B and C, one
// place each; sizes up to 64: A and B share a place; without an S: B and C.
template <int DB, bool kStates> struct TileShared {
    static constexpr int kSide = DB / 64 * kHalf;              // of A, B, the image and lo
    static constexpr int kPlaces = DB == 64 ? 6 : 5, kPer = DB == 64 || kStates ? 2 : 3, kB = kPer == 3 ? 1 : 0;
    static constexpr int kInA = DB == 64 && !kStates ? kHalf : 0;          // where B lies in a place that it shares
    static constexpr int kImage = kPlaces * 2 * kHalf, kLow = kImage + kSide, kRest = kLow + kSide, kBytes = kRest + 3 * 1024;
};

constexpr int kQueue = 3;                      // segments at work in a CTA or asked for ahead
struct Job { int kind, head, key, chunks, tail; float rate; Item it; };      // kind < 0: there is none left; chunks 0: nothing to walk over; tail: rows of no sequence
struct Patience { int dead; uint32_t limit; };     // whether some wait of the CTA ran out; nanoseconds
struct alignas(16) TileBars {
    uint32_t won[4];                           // the launch's answer
    uint64_t full[6], empty[6], s[2], i[2], z[2], p, k, o, d, e, r, t, end, got[kQueue], taken[kQueue], answer;
    Job jobs[kQueue], held;                    // held: one that was taken and could not be put among them
    uint32_t tops[2][8];                       // fp16: bits of the largest key times factor that a warp has, two chunks
    float down[2];                             // what takes D back to size
    uint32_t odd[2];                           // 1 + the last of every other chunk in which a key is not finite
    Patience patience;
    int undone, posted;                        // after a wait that ran out: the first segment that may not be whole; segments put among `jobs`
    uint32_t rest;                             // and (dealt out) the first that nobody has looked at
    uint32_t tensor;
};

__device__ __forceinline__ uint32_t at_shared(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(at_shared(b)), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t* b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(at_shared(b)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(at_shared(b)), "r"(bytes) : "memory");
}
// Waits for the phase of that parity to end, for some time at most: false if it gave up, or if another thread did before.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile Patience* dead) {
    uint64_t begin = 0;
    for (uint32_t tries = 1;; ++tries) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(at_shared(b)), "r"(parity) : "memory");
        if (done) return true;
        if (tries % 1024) continue;
        uint64_t now;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
        if (!begin) begin = now;
        if (now - begin > dead->limit) dead->dead = 1;
        if (dead->dead) return false;
    }
}
// Whether that phase has ended.
__device__ __forceinline__ bool bar_there(uint64_t* b, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(at_shared(b)), "r"(parity) : "memory");
    return done;
}
// The same for a whole warp: all of its lanes go on, together, or none.
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t parity, volatile Patience* dead) { return __all_sync(~0u, bar_wait(b, parity, dead)); }
__device__ __forceinline__ void tile_load(void* to, const CUtensorMap* map, uint64_t* bar, int x, int head, int token, int batch) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(at_shared(to)),
                 "l"(map), "r"(at_shared(bar)), "r"(x), "r"(head), "r"(token), "r"(batch) : "memory");
}
// Descriptors of tiles in rows of 128 bytes whose 16-byte pieces are turned by the row's number modulo 8.  Rows along the tile's own
// dimension (M or N), 64 elements of the summed one in a row: groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t at) { return (uint64_t)((at & 0x3ffff) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61; }
// Rows along the summed dimension, 64 elements of M or N in a row: groups of 8 rows 1024 bytes apart, the next 64 elements kHalf.
__device__ __forceinline__ uint64_t desc_cols(uint32_t at) { return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)(kHalf >> 4) << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61; }
// One thread of a warp, always the same: what it issues has operands that the compiler knows to be the warp's.
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t how, bool add) {       // A in tensor memory
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
// A whole product, step by step of 16 of the summed dimension, unrolled: issued one by one with operands worked out in a loop a step took
// 110 cycles, so 65, the tensor cores' own time for 128 columns.
template <int kSteps> __device__ __forceinline__ void mma_rows(uint32_t d, uint64_t a, uint64_t b, uint32_t how, uint32_t steps) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const uint64_t part = ((k >> 2) * kHalf + (k & 3) * 32) / 16;      // 16 elements on along a row
        if (k < steps) mma(d, a + part, b + part, how, k > 0);
    }
}
__device__ __forceinline__ void mma_cols(uint32_t d, uint64_t a, uint64_t b, uint32_t how, bool add) {
#pragma unroll
    for (int k = 0; k < 8; ++k) mma(d, a + 128 * k, b + 128 * k, how, add || k > 0);
}
__device__ __forceinline__ void mma_tensor_cols(uint32_t d, uint32_t a, uint64_t b, uint32_t how) {
#pragma unroll
    for (int k = 0; k < 8; ++k) mma_tensor(d, a + 8 * k, b + 128 * k, how, k > 0);
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

// Two products, or sums of products, by one instruction.
__device__ __forceinline__ void mul2(float& a, float& b, float f, float g) {                      // a times f, b times g
    asm("{\n.reg .b64 x, y;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nmul.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}" : "+f"(a), "+f"(b) : "f"(f), "f"(g));
}
__device__ __forceinline__ void fma2(float& a, float& b, float f, float c, float d) {              // a, b times f, plus c, d
    asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %2};\nmov.b64 z, {%3, %4};\nfma.rn.f32x2 x, x, y, z;\nmov.b64 {%0, %1}, x;\n}" : "+f"(a), "+f"(b) : "f"(f), "f"(c), "f"(d));
}

// Pairs of 16-bit values in a word.
template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> {
    using Pair = __nv_bfloat162;
    static constexpr uint32_t kHow = 1u << 4 | 1u << 7 | 1u << 10;             // 32-bit sums of bf16
    __device__ static uint32_t pack(float a, float b) { Pair x = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&x); }
    __device__ static Pair twice(float v) { return __float2bfloat162_rn(v); }
    __device__ static float one(Pair v) { return __low2float(v); }
};
template <> struct Two<__half> {
    using Pair = __half2;
    static constexpr uint32_t kHow = 1u << 4;
    __device__ static uint32_t pack(float a, float b) { Pair x = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&x); }
    __device__ static Pair twice(float v) { return __float2half2_rn(v); }
    __device__ static float one(Pair v) { return __low2float(v); }
};
// 2^14 / a power of two about as large as `most`; the exponent of what takes it off again
__device__ __forceinline__ float to_middle(float most, uint8_t& back) {
    const int e = min(max((int)(__float_as_uint(most) >> 23 & 255), 15), 254);
    back = (uint8_t)(e - 14);
    return __uint_as_float((uint32_t)(127 + 14 + 127 - e) << 23);
}
__device__ __forceinline__ float from_middle(uint8_t back) { return __uint_as_float((uint32_t)back << 23); }

// A factor in 16-bit parts, and products of pairs with it in parts, by 16-bit arithmetic: a product's rounding error is a 16-bit number, which a
// fused multiply-add gives exactly.  hi = (x f0) rounded, lo = what that left + x f1; three parts: the error of lo's sum is found the
// same way (Knuth's two-sum) and joins x f2.  fp16 has bits for that where products are large: those of a chunk are brought to 2^14 at most by
// a power of two, which is taken off D again, so that hi + lo resolves 2^-39 of the chunk's largest product whatever its size.  That power
// goes into the factor, of which a row of small keys would ask for too large a one: such a row is lifted first (exactly) by 2^12 or 2^24.
template <typename T> struct Factor {
    using Pair = typename Two<T>::Pair;
    Pair f0, f1, f2, lift[2];
    bool lifts = false;                        // (of a whole warp)
    // for a row whose largest element is `most`, in a chunk that is brought up by `up`: f up most is 2^15 at most
    __device__ Factor(float f, float most, float up) : Factor(most > 0.f ? f * up * (f * up >= 0x1p15f ? 0x1p-12f : 1.f) * (f * up >= 0x1p27f ? 0x1p-12f : 1.f) : 0.f) {
        lift[0] = Two<T>::twice(f * up >= 0x1p15f ? 4096.f : 1.f);
        lift[1] = Two<T>::twice(f * up >= 0x1p27f ? 4096.f : 1.f);
        lifts = __any_sync(~0u, most > 0.f && f * up >= 0x1p15f);
    }
    __device__ explicit Factor(float f) {
        f0 = Two<T>::twice(f);
        f -= Two<T>::one(f0);
        f1 = Two<T>::twice(f);
        f2 = Two<T>::twice(f - Two<T>::one(f1));
    }
    __device__ uint32_t lifted(uint32_t x) const {
        const Pair v = __hmul2_rn(__hmul2_rn(*reinterpret_cast<Pair*>(&x), lift[0]), lift[1]);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    __device__ void two(uint32_t& x, uint32_t& lo) const {
        const Pair v = *reinterpret_cast<Pair*>(&x), hi = __hmul2_rn(v, f0), left = __hfma2(v, f0, __hneg2(hi)), l = __hfma2(v, f1, left);
        x = *reinterpret_cast<const uint32_t*>(&hi);
        lo = *reinterpret_cast<const uint32_t*>(&l);
    }
    __device__ void three(uint32_t& x, uint32_t& lo, uint32_t& last) const {
        const Pair v = *reinterpret_cast<Pair*>(&x), hi = __hmul2_rn(v, f0), left = __hfma2(v, f0, __hneg2(hi)), next = __hmul2_rn(v, f1), left2 = __hfma2(v, f1, __hneg2(next));
        const Pair l = __hadd2_rn(left, next), b = __hsub2_rn(l, left), off = __hadd2_rn(__hsub2_rn(left, __hsub2_rn(l, b)), __hsub2_rn(next, b));
        const Pair e = __hfma2(v, f2, __hadd2_rn(off, left2));
        x = *reinterpret_cast<const uint32_t*>(&hi);
        lo = *reinterpret_cast<const uint32_t*>(&l);
        last = *reinterpret_cast<const uint32_t*>(&e);
    }
};

// The largest element of pieces `from` .. `end` of a row, those that are not finite left out; row_most: infinity where there are some.  (fp16)
template <typename T>
__device__ __noinline__ float finite_most(const uint8_t* b, int r, int from, int end) {
    float most = 0.f;
    for (int i = from; i < end; ++i) {
        const T* x = reinterpret_cast<const T*>(b + (i >> 3) * kHalf + ((i & 7) ^ (r & 7)) * 16);
        for (int e = 0; e < 8; ++e) {
            const float v = fabsf(to_float(x[e]));
            if (isfinite(v)) most = fmaxf(most, v);
        }
    }
    return most;
}
template <typename T>
__device__ __forceinline__ float row_most(const uint8_t* b, int r, int from, int end) {
    uint32_t most[2] = {};                     // (signs do not count)
#pragma unroll 4
    for (int i = from; i < end; ++i) {
        const uint4 q = *reinterpret_cast<const uint4*>(b + (i >> 3) * kHalf + ((i & 7) ^ (r & 7)) * 16);
        const uint32_t* x = &q.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) asm("max.NaN.xorsign.abs.f16x2 %0, %0, %1;" : "+r"(most[e & 1]) : "r"(x[e]));
    }
    asm("max.NaN.xorsign.abs.f16x2 %0, %0, %1;" : "+r"(most[0]) : "r"(most[1]));
    most[0] &= 0x7fff7fff;
    const float m = __low2float(*reinterpret_cast<__half2*>(most)), other = __high2float(*reinterpret_cast<__half2*>(most));
    return m < INFINITY && other < INFINITY ? fmaxf(m, other) : INFINITY;
}

// Outputs of a chunk's rows in which some value is not finite, once more: masked tokens leave no trace (0 * inf is none), so what is not
// finite is added up again over the tokens that a row sees.  Rare, and slow.
template <typename T>
__device__ __noinline__ void careful(const Walk& W, int batch, int head, int64_t t0, int n, int r, float rate, float age, uint32_t O, uint32_t I, float off, const uint8_t* cs, int64_t to) {
    const T* a = static_cast<const T*>(W.a.at) + (int64_t)batch * W.a.st[0] + (t0 + r) * W.a.st[1] + (int64_t)(head / W.a.group) * W.a.st[2];
    const T* b = static_cast<const T*>(W.b.at) + (int64_t)batch * W.b.st[0] + t0 * W.b.st[1] + (int64_t)(head / W.b.group) * W.b.st[2];
    const T* c = static_cast<const T*>(W.c.at) + (int64_t)batch * W.c.st[0] + t0 * W.c.st[1] + (int64_t)(head / W.c.group) * W.c.st[2];
    for (int j0 = 0; j0 < W.cd; j0 += 16) {
        float o[16], m[16];
        tensor_load16(o, O + j0);
        tensor_load16(m, I + j0);
        tensor_load_wait();
        uint32_t odd = 0, open = 0;                                        // open: not settled by the memory, which is no number from a token like that on
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            m[j] *= (cs ? from_middle(cs[j0 + j]) : 1.f) * age;
            if (j0 + j < W.cd && r < n && !isfinite(o[j] * off + m[j])) { odd |= 1u << j; open |= (uint32_t)!isnan(m[j]) << j; }
        }
        for (int q = W.rev ? r : 0; open && q <= (W.rev ? n - 1 : r); ++q) {
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

// What a chunk adds to a column of the memory (r of c), once more where it is not finite: an infinity in parts is none (inf - inf, 0 * inf), so the
// sum is that of the factors themselves.  It goes to where D has it.  Rare, and slow, but for what is no number at once.
template <typename T>
__device__ __noinline__ void careful_sum(const Walk& W, int batch, int head, int64_t t0, int n, int r, float rate, int near, float up, uint32_t D) {
    const T* b = static_cast<const T*>(W.b.at) + (int64_t)batch * W.b.st[0] + t0 * W.b.st[1] + (int64_t)(head / W.b.group) * W.b.st[2];
    const T* c = static_cast<const T*>(W.c.at) + (int64_t)batch * W.c.st[0] + t0 * W.c.st[1] + (int64_t)(head / W.c.group) * W.c.st[2];
    const bool on = r < W.cd;
    for (int i = 0; i < W.bd; i += 16) {
        float x[16], zero = 0.f;
        tensor_load16(x, D + i);
        tensor_load_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) zero = fmaf(x[e], 0.f, zero);
        if (!__any_sync(~0u, !(zero == 0.f))) continue;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
        for (int t = 0; t < n; ++t) {
            const float v = on ? to_float(c[t * W.c.st[1] + r]) : 0.f, f = power(rate, (W.rev ? t + 1 : n - t) - near);
            bool open = false;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (on && i + e < W.bd) {
                    x[e] += to_float(b[t * W.b.st[1] + i + e]) * f * v;
                    open |= !isnan(x[e]);
                }
            if (!__any_sync(~0u, open)) break;
        }
        uint32_t y[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(x[e] * up);
        tensor_store16(D + i, y);
        tensor_store_wait();
    }
}

template <int kRegs> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }
__device__ __forceinline__ void store32(void* to, const uint32_t (&w)[8]) {       // 32 bytes, aligned
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// What a role of the CTA works on: segment after segment, as the queue gives them, and the chunks of each.  `g` counts chunks over all
// of them: it gives every barrier's phase.
struct Work {
    TileBars* bars;
    uint32_t g = 0;
    int at = -1;
    const volatile Job* job = nullptr;

    // On to the next segment, the one before is given back; false: there is none.  Called by whole warps.
    __device__ __forceinline__ bool next() {
        if (at >= 0) {
            __syncwarp();
            if ((threadIdx.x & 31) == 0) bar_arrive(&bars->taken[at % kQueue]);
        }
        ++at;
        if (!warp_wait(&bars->got[at % kQueue], (at / kQueue) & 1, &bars->patience)) return false;
        job = bars->jobs + at % kQueue;
        return job->kind >= 0;
    }
    // Whether next() would not wait.
    __device__ __forceinline__ bool ready() const { return __all_sync(~0u, bar_there(&bars->got[(at + 1) % kQueue], ((at + 1) / kQueue) & 1)); }
    // A chunk's first token and its tokens.
    __device__ __forceinline__ int tokens(int c) const { return min(kTile, job->it.n - c * kTile); }
    __device__ __forceinline__ int begin(int c, bool rev) const {
        const int at = job->it.from + c * kTile;
        return job->it.begin + (rev ? job->it.len - at - tokens(c) : at);
    }
};

// Rare or once a segment: kept out of the walk's own code, which has to stay near the warps that run it.
__device__ __noinline__ void tile_tail(const WalkArgs& A, const Walk& W, const volatile Job* job, int segments) {
    zero_tail(A, W, W.y32 ? 4 : 2, job->key, segments, job->head, threadIdx.x & 127, 128);
}
// A wait that ran out does not go unnoticed: what the CTA has taken on and not brought to an end becomes no numbers, rows and memories alike.  A
// segment that nobody has taken goes to another CTA.
constexpr int kLosers = 256;                   // threads (those whose registers are as many as at the launch)
template <bool kStates>
__device__ __forceinline__ void lose(const WalkArgs& A, const volatile Job* job, int segments, int thread) {
    if (job->kind < 0) return;
    const Walk& W = A.w[job->kind];
    const size_t of = (size_t)W.bd * W.cd;
    if (job->tail) zero_tail(A, W, W.y32 ? 4 : 2, job->key, segments, job->head, thread, kLosers);
    if (job->it.len < 0) return;
    float* memory = nullptr;
    if (kStates) { if (!job->it.last) memory = W.slots + ((size_t)job->it.slot * A.heads + job->head) * of; }
    else if (job->it.last && W.last) memory = W.last + ((size_t)job->it.seq * A.heads + job->head) * of;
    if (memory)
        for (size_t i = thread; i < of; i += kLosers) memory[i] = __int_as_float(0x7fc00000);
    if (kStates) return;
    const int64_t first = job->it.begin + (W.rev ? job->it.len - job->it.from - job->it.n : job->it.from);
    for (int64_t i = thread; i < (int64_t)job->it.n * W.cd; i += kLosers) {
        const int64_t to = (int64_t)job->it.batch * W.ys[0] + (first + i / W.cd) * W.ys[1] + (int64_t)job->head * W.ys[2] + i % W.cd;
        if (W.y32) static_cast<float*>(W.y)[to] = __int_as_float(0x7fc00000);
        else static_cast<uint16_t*>(W.y)[to] = 0x7fff;
    }
}
// The segment of number x, by a whole warp.
template <bool kStates> __device__ __forceinline__ Job job_of(const WalkArgs& A, uint32_t x, bool tail) {
    Job j = {-1, 0, 0, 0, tail, 0.f, {}};
    const int rest = (int)x / A.kinds;
    j.kind = (int)x - rest * A.kinds;
    j.key = rest / A.heads;
    j.head = rest - j.key * A.heads;
    j.rate = rate_of(A.log_decay, j.head);
    const bool is = item_of(A, A.w[j.kind].rev, j.key, j.it);
    if (!is) j.it.len = -1;
    j.chunks = is && !(kStates && j.it.last) ? (j.it.n + kTile - 1) / kTile : 0;
    return j;
}
template <bool kStates> __device__ __noinline__ void lose_all(const TileArgs& G, const TileBars* bars, int thread) {
    const int segments = kStates ? 0 : gridDim.x / (G.walks.heads * G.walks.kinds);
    for (int i = bars->undone; i < bars->posted; ++i) lose<kStates>(G.walks, bars->jobs + i % kQueue, segments, thread);
    lose<kStates>(G.walks, &bars->held, segments, thread);
    for (uint32_t x = bars->rest; x < G.items; x += gridDim.x) {
        const Job j = job_of<kStates>(G.walks, x, false);
        lose<kStates>(G.walks, &j, segments, thread);
    }
}

// The largest of a row's products, faded.  (fp16)
__device__ __noinline__ float faded_most(uint32_t S, uint32_t powers, int first, int end, int r, int n, bool rev) {
    float most = 0.f;
#pragma unroll 1
    for (int j = first; j < end; ++j) {
        float p[32], x[32];
        tensor_load32(p, S + 32 * j);
#pragma unroll
        for (int e = 0; e < 32; ++e) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[e]) : "r"(powers - 4 * (32 * j + e)));       // (what is not seen may lie beside the table)
        tensor_load_wait();
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const int q = 32 * j + e;
            most = fmaxf(most, q < n && (rev ? q >= r : q <= r) ? fabsf(p[e] * x[e]) : 0.f);
        }
    }
    return most;
}

template <typename T, int DB, bool kStates>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(const __grid_constant__ TileArgs G) {
    extern __shared__ __align__(1024) uint8_t sm[];
    using L = TileShared<DB, kStates>;
    constexpr bool kHalfs = Two<T>::kHow == 1u << 4;
    const WalkArgs& A = G.walks;
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    float* powers = reinterpret_cast<float*>(sm + L::kRest);               // of the factor, 0 .. 128, of two segments
    uint8_t* cs = reinterpret_cast<uint8_t*>(powers + 2 * 132);            // fp16: what the image's columns were brought up by, two chunks
    TileBars* bars = reinterpret_cast<TileBars*>(cs + 256);
    static_assert(2 * 132 * 4 % 16 == 0 && 2 * 132 * 4 + 256 + sizeof(TileBars) <= L::kBytes - L::kRest, "all of it fits, where it has to lie");
    volatile Patience* dead = &bars->patience;
    // Packed sequences, whose lengths the host does not know: often none of them is longer than a segment (looked up by as many threads as there are, up to
    // some number that takes about a microsecond).
    if (kStates && A.starts && A.sequences <= 16 * kTileThreads) {
        bool longer = false;
        for (uint32_t i = tid; i < A.sequences; i += kTileThreads) longer |= start_of(A, 0, i + 1) - start_of(A, 0, i) > A.seg;
        if (!__syncthreads_or(longer)) return;
    }

    if (tid == 0) {
        for (int s = 0; s < L::kPlaces; ++s) { bar_init(&bars->full[s], 1); bar_init(&bars->empty[s], 1); }
        for (uint64_t* b : {&bars->s[0], &bars->s[1], &bars->i[0], &bars->i[1], &bars->o, &bars->d, &bars->end, &bars->answer}) bar_init(b, 1);
        for (uint64_t* b : {&bars->p, &bars->e, &bars->r, &bars->z[0], &bars->z[1]}) bar_init(b, 128);
        bar_init(&bars->k, kStates ? 256 : 128);
        bar_init(&bars->t, kStates ? 8 : 4);
        for (int s = 0; s < kQueue; ++s) { bar_init(&bars->got[s], 1); bar_init(&bars->taken[s], 14); }
        bars->patience = {0, A.limit};
        bars->held.kind = -1;
        bars->undone = INT32_MAX;
        bars->posted = 0;
        bars->rest = ~0u;
        bars->odd[0] = bars->odd[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at_shared(&bars->tensor)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    order_shared();
    order_before();
    __syncthreads();
    order_after();
    const uint32_t tm = bars->tensor, S = tm, O = tm + 128, I = tm + 256, D = tm + 384, mine = (uint32_t)(warp & 3) << 21;       // (a warp's 32 lanes)
    Work w{bars};

    // Tile `which` (0: A, kB: B, kPer - 1: C) of chunk g: its place, and its barriers' phase.
    auto place = [](uint32_t g, int which) { return (g * L::kPer + which) % L::kPlaces; };
    auto turn = [](uint32_t g, int which) { return (g * L::kPer + which) / L::kPlaces & 1; };
    auto has = [&](uint32_t g, int which) { return warp_wait(&bars->full[place(g, which)], turn(g, which), dead); };
    constexpr int kC = L::kPer - 1;

    // B' by the threads of a warpgroup, a token each; where two have a chunk, half of its elements.
    auto make_parts = [&](int r, int which) {
        uint8_t *image = sm + L::kImage + r * 128, *low = sm + L::kLow + r * 128;
        uint32_t g = 0, tops = 0, tails = 0;                               // (tops: chunks whose largest product was looked for; tails: of fewer tokens)
        bool ok = true;
        while (ok && w.next()) {
            const int chunks = w.job->chunks;
            const Walk& W = A.w[w.job->kind];
            const float rate = w.job->rate;
            const bool rev = W.rev, given = kStates || (w.job->it.last && W.last), three = !kHalfs && given && G.parts > 2;
            const int adding = given ? chunks : chunks - 1, pieces = (W.bd + 15) / 16 * 2;
            const int from = kStates && which ? pieces / 2 : 0, end = kStates && !which ? pieces / 2 : pieces;
            for (int c = 0; c < chunks; ++c, ++g) {
                const int n = w.tokens(c);
                const bool in = r < n;
                ok = has(g, L::kB) && (n == kTile || has(g, kC));
                if (!ok) break;
                uint8_t *b = sm + place(g, L::kB) * 2 * kHalf + L::kInA + r * 128, *v = sm + place(g, kC) * 2 * kHalf + r * 128;
                if (n < kTile && which == 0) {                             // rows of C behind the last token, which P's zeros might not stop
                    if (!in)
#pragma unroll 1
                        for (int i = 0; i < 16; ++i) *reinterpret_cast<uint4*>(v + (i >> 3) * kHalf + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
                    order_shared();
                    // (of two chunks in turn: the next one's rows may be cleared before the warp that issues products has looked for this one's)
                    if (!kStates) bar_arrive(&bars->z[tails++ & 1]);
                }
                const float fade = c < adding && in ? power(rate, (rev ? r + 1 : n - r) - (!kStates && given && c + 1 == chunks && !rev ? 1 : 0)) : 0.f;
                float most = 0.f, up = 1.f;
                bool odd = false;                                          // (fp16) an element is not finite
                uint8_t down = 127;
                if (kHalfs && c < adding) {                                // the largest product of the chunk: of the row, of the warp
                    if (in) {
                        most = row_most<T>(b, r, from, end);
                        if (!(most < INFINITY)) { odd = true; most = finite_most<T>(b, r, from, end); }
                    }
                    const uint32_t top = __reduce_max_sync(~0u, __float_as_uint(most * fade));
                    if ((threadIdx.x & 31) == 0) {
                        bars->tops[tops & 1][which * 4 + (r >> 5)] = top;
                        bar_arrive(&bars->t);
                    }
                    ok = warp_wait(&bars->t, tops & 1, dead);
                    if (!ok) break;
                    uint32_t all = 0;
#pragma unroll
                    for (int i = 0; i < (kStates ? 8 : 4); ++i) all = max(all, ((volatile uint32_t*)bars->tops[tops & 1])[i]);
                    if (all) up = to_middle(__uint_as_float(all), down);
                    ++tops;
                }
                const Factor<T> f = kHalfs ? Factor<T>(fade, most, up) : Factor<T>(fade);
                // the parts' places: B's is free when S is done, lo's when the D before is, the image's when I is (or where there is none, that D)
                ok = (g == 0 || warp_wait(&bars->d, (g - 1) & 1, dead)) && (kStates || (warp_wait(&bars->s[g & 1], g >> 1 & 1, dead) && (!three || warp_wait(&bars->i[g & 1], g >> 1 & 1, dead))));
                if (!ok) break;
                if (c < adding) {
                    if (kHalfs && which == 0 && r == 0) bars->down[g & 1] = from_middle(down);         // (the one two chunks ago has been used: D has, since)
                    typename Two<T>::Pair zero = Two<T>::twice(0.f);       // 0 times all of lo, which is no number where the element is not finite
                    // pieces of 8 elements, a few at a time: a piece is a load, a dozen dependent steps and two or three stores
                    auto all = [&](auto how) {
#pragma unroll decltype(how)::value ? 2 : 4
                        for (int i = from; i < end; ++i) {
                            const int at = (i >> 3) * kHalf + ((i & 7) ^ (r & 7)) * 16;
                            uint4 q = *reinterpret_cast<const uint4*>(b + at), lo, last;
                            uint32_t *pq = &q.x, *pl = &lo.x, *pt = &last.x;
                            if (kHalfs && f.lifts)
#pragma unroll
                                for (int e = 0; e < 4; ++e) pq[e] = f.lifted(pq[e]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (decltype(how)::value) f.three(pq[e], pl[e], pt[e]);
                                else f.two(pq[e], pl[e]);
                                if (!kHalfs) zero = __hfma2(*reinterpret_cast<const typename Two<T>::Pair*>(pl + e), Two<T>::twice(0.f), zero);
                            }
                            *reinterpret_cast<uint4*>(b + at) = q;
                            *reinterpret_cast<uint4*>(low + at) = lo;
                            if (decltype(how)::value) *reinterpret_cast<uint4*>(image + at) = last;
                        }
                    };
                    if (!in)                                               // (no product with 0: what stands there might be anything)
#pragma unroll 1
                        for (int i = from; i < end; ++i) *reinterpret_cast<uint4*>(b + (i >> 3) * kHalf + ((i & 7) ^ (r & 7)) * 16) = make_uint4(0, 0, 0, 0);
                    if (three) all(std::true_type());
                    else all(std::false_type());
                    if (kHalfs ? odd : in && !(__low2float(zero) == 0.f && __high2float(zero) == 0.f)) bars->odd[g & 1] = g + 1;
                }
                order_shared();
                bar_arrive(&bars->k);
            }
        }
    };

    if (warp >= 12) {
        fewer_registers<56>();
        if (warp == 12) {                                                  // copies of tiles
            const CUtensorMap* all = &G.maps.q;
            uint32_t issued = 0;                                           // tiles
            bool ok = true;
            while (ok && w.next()) {
                const Walk& W = A.w[w.job->kind];
                const int *of = G.of[w.job->kind], head = w.job->head, batch = w.job->it.batch, chunks = w.job->chunks;
                const CUtensorMap *ma = all + of[0], *mb = all + of[1], *mc = all + of[2];
                const int ha = head / W.a.group, hb = head / W.b.group, hc = head / W.c.group, halves = W.cd > 64 ? 2 : 1;
                for (int c = 0; c < chunks; ++c, ++w.g) {
                    ok = w.g != A.stop;
                    if (!ok) break;
                    const int t0 = w.begin(c, W.rev);
#pragma unroll 1
                    for (int which = 0; which < L::kPer; ++which) {
                        const uint32_t at = w.g * L::kPer + which, s = at % L::kPlaces;
                        ok = at < L::kPlaces || warp_wait(&bars->empty[s], (at / L::kPlaces - 1) & 1, dead);
                        if (!ok) break;
                        uint8_t* to = sm + s * 2 * kHalf;
                        if (elected()) {
                            const bool is_c = which == kC, is_b = which == L::kB && !is_c, is_a = !kStates && which == 0;
                            const CUtensorMap* m = is_c ? mc : is_a ? ma : mb;
                            const int h = is_c ? hc : is_a ? ha : hb, n = is_c ? halves : DB / 64;
                            bar_expect(&bars->full[s], (uint32_t)(n + (DB == 64 && is_a ? 1 : 0)) * kHalf);
                            for (int i = 0; i < n; ++i) tile_load(to + i * kHalf, m, &bars->full[s], 64 * i, h, t0, batch);
                            if (DB == 64 && is_a && is_b) tile_load(to + L::kInA, mb, &bars->full[s], 0, hb, t0, batch);
                        }
                        issued = at + 1;
                        __syncwarp();
                    }
                    if (!ok) break;
                }
            }
            volatile Patience again = {0, kPatience};                     // copies still under way write here: none may be left
            for (uint32_t i = issued > L::kPlaces ? issued - L::kPlaces : 0; i < issued; ++i) bar_wait(&bars->full[i % L::kPlaces], (i / L::kPlaces) & 1, &again);
        } else if (warp == 13) {                                           // products
            const uint32_t how = Two<T>::kHow | 8u << 24;
            const uint64_t rows0 = desc_rows(at_shared(sm)), cols0 = desc_cols(at_shared(sm)), image_rows = rows0 + L::kImage / 16;
            auto rows_at = [&](uint32_t g, int which, int off) { return rows0 + (uint64_t)(place(g, which) * 2 * kHalf + off) / 16; };
            auto cols_at = [&](uint32_t g, int which, int off) { return cols0 + (uint64_t)(place(g, which) * 2 * kHalf + off) / 16; };
            // The chunk that comes next, of whatever segment; 0: not known yet (asked for without waiting), -1: none.
            struct { uint32_t how_i, how_d, bd16; int n, parts; bool adds; } next = {}, now = {};
            int c = -1, chunks = 0, adding = 0;
            auto advance = [&](bool wait) {
                while (++c >= chunks) {
                    --c;
                    if (!wait && !w.ready()) return 0;
                    if (!w.next()) return -1;
                    const Walk& W = A.w[w.job->kind];
                    const bool given = kStates || (w.job->it.last && W.last);
                    c = -1; chunks = w.job->chunks; adding = given ? chunks : chunks - 1;
                    next.bd16 = (uint32_t)(W.bd + 15) / 16;
                    next.how_i = how | 2 * ((uint32_t)(W.cd + 15) / 16) << 17;
                    next.how_d = how | 1u << 15 | 1u << 16 | 2 * next.bd16 << 17;
                    next.parts = given ? G.parts : 2;
                }
                next.n = w.tokens(c);
                next.adds = c < adding;
                return 1;
            };
            auto issue_s = [&](uint32_t g) {
                order_after();
                if (elected()) {
                    mma_rows<DB / 16>(S, rows_at(g, 0, 0), rows_at(g, L::kB, L::kInA), how | 16u << 17, next.bd16);
                    mma_commit(&bars->s[g & 1]);
                }
                __syncwarp();
            };
            bool ok = true, ahead = false;                                 // ahead: S has been issued
            int more = advance(true);
            uint32_t tails = 0;
            while (ok && more > 0) {
                const uint32_t g = w.g, ph = g & 1;
                if (!kStates && !ahead) {                                  // (P lies where S goes, and has been read when O is done)
                    ok = has(g, 0) && has(g, L::kB) && (g == 0 || warp_wait(&bars->o, ph ^ 1, dead));
                    if (!ok) break;
                    issue_s(g);
                }
                now = next;
                ahead = false;
                more = 0;
                ok = has(g, kC);
                if (!kStates) {
                    // rows of C behind the last token have been cleared; P is there; O's and I's places have been read
                    if (now.n < kTile) { ok = ok && warp_wait(&bars->z[tails & 1], tails >> 1 & 1, dead); ++tails; }
                    ok = ok && warp_wait(&bars->p, ph, dead) && (g == 0 || warp_wait(&bars->e, ph ^ 1, dead));
                    if (!ok) break;
                    order_after();
                    if (elected()) {
                        mma_tensor_cols(O, S, cols_at(g, kC, 0), now.how_i | 1u << 16);
                        mma_commit(&bars->o);
                    }
                    __syncwarp();
                    // S of the next chunk, where that is known and its tiles are there.  Nothing is waited for here that might wait for this chunk's D.
                    more = advance(false);
                    if (more > 0 && __all_sync(~0u, bar_there(&bars->full[place(g + 1, 0)], turn(g + 1, 0)) && bar_there(&bars->full[place(g + 1, L::kB)], turn(g + 1, L::kB)))) {
                        ok = warp_wait(&bars->o, ph, dead);
                        if (!ok) break;
                        issue_s(g + 1);
                        ahead = true;
                    }
                }
                ok = ok && warp_wait(&bars->r, ph, dead);                  // (the image is there, D's place has been read)
                if (!ok) break;
                order_after();
                if (!kStates && elected()) {
                    mma_rows<DB / 16>(I, rows_at(g, 0, 0), image_rows, now.how_i, now.bd16);
                    mma_commit(&bars->i[ph]);
                    if (L::kB) mma_commit(&bars->empty[place(g, 0)]);
                }
                __syncwarp();
                ok = warp_wait(&bars->k, ph, dead);
                if (!ok) break;
                order_after();
                if (elected()) {
                    if (now.adds)
#pragma unroll 1
                        for (int p = now.parts - 1; p >= 0; --p)           // the small parts first
                            mma_cols(D, cols_at(g, kC, 0), p == 0 ? cols_at(g, L::kB, L::kInA) : cols0 + (p == 1 ? L::kLow : L::kImage) / 16, now.how_d, p < now.parts - 1);
                    mma_commit(&bars->d);
                    mma_commit(&bars->empty[place(g, L::kB)]);
                    mma_commit(&bars->empty[place(g, kC)]);
                }
                __syncwarp();
                ++w.g;
                if (more == 0) more = advance(true);
            }
            volatile Patience again = {0, kPatience};
            if (elected()) mma_commit(&bars->end);
            __syncwarp();
            bar_wait(&bars->end, 0, &again);
        } else if (warp == 14) {                                           // segments
            const bool tail = !kStates && A.starts && (A.w[0].zero_tail || A.w[1].zero_tail || A.w[2].zero_tail) &&
                              (__ldg(A.starts) > 0 || __ldg(A.starts + A.sequences) < (int64_t)A.tokens);          // rows of no sequence that become 0
            int x = blockIdx.x, i = 0;
            bool late = false;
            for (uint32_t asked = 0;; ++asked) {
                Job j = {-1, 0, 0, 0, tail, 0.f, {}};
                if (x >= 0) j = job_of<kStates>(A, x, tail);
                // (a key of no segment, or one that there is nothing to do for, is passed over)
                if (x < 0 || tail || j.chunks > 0 || (!kStates && j.it.len == 0 && A.w[j.kind].last)) {
                    const int slot = i % kQueue;
                    if (late || (i >= kQueue && !warp_wait(&bars->taken[slot], (i / kQueue - 1) & 1, dead))) {
                        if (lane == 0) {
                            bars->held = j;
                            if (kStates && x >= 0) bars->rest = (uint32_t)x + gridDim.x;
                        }
                        break;
                    }
                    if (lane == 0) {
                        bars->jobs[slot] = j;
                        bar_arrive(&bars->got[slot]);
                    }
                    ++i;
                }
                __syncwarp();
                if (x < 0) break;
                if (kStates) {                                             // all of a length, and many none: dealt out
                    x = (uint32_t)x + gridDim.x < G.items ? (int)(x + gridDim.x) : -1;
                    continue;
                }
                if (lane == 0) {
                    order_shared();
                    bar_expect(&bars->answer, 16);
                    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(at_shared(bars->won)), "r"(at_shared(&bars->answer)) : "memory");
                }
                __syncwarp();
                // (an answer that is late is waited for all the same: it may be a segment, and is written to this CTA's memory)
                late = !warp_wait(&bars->answer, asked & 1, dead);
                if (late) {
                    volatile Patience again = {0, kPatience};
                    if (!warp_wait(&bars->answer, asked & 1, &again)) break;
                }
                uint32_t is, to;
                asm volatile("{\n.reg .b128 h;\n.reg .pred p;\n.reg .b64 lo, hi;\nld.shared.v2.b64 {lo, hi}, [%2];\nmov.b128 h, {lo, hi};\n"
                             "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
                             "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n}" : "=r"(is), "=r"(to) : "r"(at_shared(bars->won)) : "memory");
                x = is ? (int)to : -1;
                __syncwarp();
            }
            if (lane == 0) bars->posted = i;
        }
    } else if (warp < 4) {
        const int r = tid;
        if (kStates) make_parts(r, 0);
        int walked = 0;
        bool ok = !kStates;
        while (ok && w.next()) {
            const Walk& W = A.w[w.job->kind];
            if (w.job->tail) tile_tail(A, W, w.job, gridDim.x / (A.heads * A.kinds));
            const int chunks = w.job->chunks, head = w.job->head, batch = w.job->it.batch, cd = W.cd;
            if (chunks == 0) continue;
            const bool rev = W.rev, y32 = W.y32, wide = W.wide;
            const float rate = w.job->rate;
            // Powers 0 .. 128 of the factor, the other way round where the walk is, so that a row finds those of its columns in one order.
            // Every warp writes the table, all the same values; others may still be at the segment before, none at one before that.
            float* pw = powers + (walked++ & 1) * 132;
            for (int i = lane; i <= kTile; i += 32) pw[rev ? kTile - i : i] = power(rate, i);
            __syncwarp();
            const int first = rev ? warp : 0, end = rev ? 4 : warp + 1;
            float off = 1.f;                                               // fp16: what brings a row of O back
            // P of chunk g, the segment's c-th.  Group j of 32 columns of S becomes 16 words of P, which lie where group j / 2 was: in this order
            // none is lost.  A warp's rows see groups up to (or from) their own; what a row does not see is replaced, not multiplied by 0.
            auto make_p = [&](uint32_t g, int c) {
                if (!warp_wait(&bars->s[g & 1], g >> 1 & 1, dead)) return false;
                order_after();
                const int n = w.tokens(c);
                auto seen_of = [&](int j) {
                    uint32_t seen = ~0u;
                    if (j == warp) seen = rev ? ~0u << lane : (2u << lane) - 1;
                    if (32 * j + 32 > n) seen &= n > 32 * j ? (1u << (n - 32 * j)) - 1 : 0u;
                    return seen;
                };
                float p[32], on = 1.f;
                if (kHalfs) {
                    // The row's largest product, faded; where 15 tokens fade to no less than 2^-18, a bound of it within that: the largest of 16 tokens times
                    // the factor of the nearest, which leaves the largest at 2^-4 and the last bit at 2^-20 of it; where all of a chunk's do, the largest.
                    float most = 0.f;
                    const bool even = rate > -18.f / 127;
                    if (rate < -18.f / 15) most = faded_most(S + mine, at_shared(pw + (rev ? kTile : 0) + r), first, end, r, n, rev);
                    else
#pragma unroll 1
                    for (int j = first; j < end; ++j) {
                        tensor_load32(p, S + mine + 32 * j);
                        const uint32_t seen = seen_of(j);
                        tensor_load_wait();
                        if (j == warp || 32 * j + 32 > n) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) p[e] = seen >> e & 1 ? p[e] : 0.f;
                        }
                        float low = 0.f, high = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) { low = fmaxf(low, fabsf(p[e])); high = fmaxf(high, fabsf(p[e + 16])); }
                        if (!even) {
                            low *= pw[rev ? kTile - max(32 * j - r, 0) : max(r - 32 * j - 15, 0)];
                            high *= pw[rev ? kTile - max(32 * j + 16 - r, 0) : max(r - 32 * j - 31, 0)];
                        }
                        most = fmaxf(most, fmaxf(low, high));
                    }
                    uint8_t back;
                    on = to_middle(most, back);
                    off = from_middle(back);
                }
#pragma unroll 1
                for (int j = 0; j < 4; ++j) {
                    uint32_t y[16] = {};
                    if (j >= first && j < end) {
                        tensor_load32(p, S + mine + 32 * j);
                        const uint32_t f = at_shared(pw + (rev ? kTile : 0) + r - 32 * j);     // (what is not seen may lie beside the table: in shared memory all the same)
                        float x[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[e]) : "r"(f - 4 * e));       // (asm: a load that depends on a bit of `seen` waits for the one before)
                        tensor_load_wait();
#pragma unroll
                        for (int e = 0; e < 32; e += 2) mul2(p[e], p[e + 1], x[e], x[e + 1]);
                        if (kHalfs)
#pragma unroll
                            for (int e = 0; e < 32; e += 2) mul2(p[e], p[e + 1], on, on);
                        if (j == warp || 32 * j + 32 > n) {
                            const uint32_t seen = seen_of(j);
#pragma unroll
                            for (int e = 0; e < 32; ++e) p[e] = seen >> e & 1 ? p[e] : 0.f;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = Two<T>::pack(p[2 * e], p[2 * e + 1]);
                    }
                    tensor_store16(S + mine + 16 * j, y);
                }
                tensor_store_wait();
                order_before();
                bar_arrive(&bars->p);
                return true;
            };
            if (!make_p(w.g, 0)) ok = false;
            for (int c = 0; c < chunks && ok; ++c, ++w.g) {
                const int ph = w.g & 1, n = w.tokens(c);
                const float back = off;
                // the next chunk's P first: its O, and S after that, need not wait for this one's y
                ok = (c + 1 >= chunks || make_p(w.g + 1, c + 1)) && warp_wait(&bars->i[ph], w.g >> 1 & 1, dead);
                if (!ok) break;
                order_after();
                const float age = r < n ? pw[rev ? kTile - (n - 1 - r) : r] : 0.f;
                const int64_t to = (int64_t)batch * W.ys[0] + (int64_t)(w.begin(c, rev) + r) * W.ys[1] + (int64_t)head * W.ys[2];
                typename Two<T>::Pair odd[2] = {Two<T>::twice(0.f), Two<T>::twice(0.f)};     // 0 times all, 0 where all are finite
#pragma unroll 1
                for (int j0 = 0; j0 < cd; j0 += 32) {
                    float x[32], m[32];
                    tensor_load32(x, O + mine + j0);
                    tensor_load32(m, I + mine + j0);
                    tensor_load_wait();
                    if (kHalfs)
#pragma unroll
                        for (int j = 0; j < 32; j += 16) {
                            const uint4 up = *reinterpret_cast<const uint4*>(cs + ph * 128 + j0 + j);
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                mul2(x[j + e], x[j + e + 1], back, back);
                                mul2(m[j + e], m[j + e + 1], from_middle((&up.x)[e / 4] >> 8 * (e % 4) & 255), from_middle((&up.x)[e / 4] >> 8 * (e % 4 + 1) & 255));
                            }
                        }
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        fma2(m[j], m[j + 1], age, x[j], x[j + 1]);
                        x[j] = m[j]; x[j + 1] = m[j + 1];
                    }
                    if (y32) {
                        float4* y = reinterpret_cast<float4*>(static_cast<float*>(W.y) + to + j0);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (r < n && j0 + 4 * e < cd) y[e] = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
                    }
                    uint32_t v[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = Two<T>::pack(x[2 * j], x[2 * j + 1]);
                    if (j0 + 32 > cd)                                      // (what lies behind the head is none of y's)
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = j0 + 2 * j < cd ? v[j] : 0u;
#pragma unroll
                    for (int j = 0; j < 16; ++j) odd[j & 1] = __hfma2(*reinterpret_cast<const typename Two<T>::Pair*>(&v[j]), Two<T>::twice(0.f), odd[j & 1]);
                    if (!y32 && r < n) {
                        T* y = static_cast<T*>(W.y) + to + j0;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t (&u)[8] = *reinterpret_cast<uint32_t (*)[8]>(v + 8 * e);
                            if (wide && j0 + 16 * e + 16 <= cd) store32(y + 16 * e, u);
                            else {
                                if (j0 + 16 * e < cd) reinterpret_cast<uint4*>(y)[2 * e] = make_uint4(u[0], u[1], u[2], u[3]);
                                if (j0 + 16 * e + 8 < cd) reinterpret_cast<uint4*>(y)[2 * e + 1] = make_uint4(u[4], u[5], u[6], u[7]);
                            }
                        }
                    }
                    __syncwarp();
                }
                odd[0] = __hadd2(odd[0], odd[1]);
                if (__any_sync(~0u, !(__low2float(odd[0]) == 0.f && __high2float(odd[0]) == 0.f) && r < n))
                    careful<T>(W, batch, head, w.begin(c, rev), n, r, rate, age, O + mine, I + mine, back, kHalfs ? cs + ph * 128 : nullptr, to);
                order_before();
                bar_arrive(&bars->e);
            }
        }
    } else if (warp < 8) {
        more_registers<184>();
        const int r = tid - 128;                                           // an element of c
        uint8_t* image = sm + L::kImage;
        bool ok = true;
        while (ok && w.next()) {
            const volatile Job& j = *w.job;
            const Walk& W = A.w[j.kind];
            if (j.it.len < 0 || (kStates && j.it.last)) continue;
            const int bd = W.bd, chunks = j.chunks, head = j.head;
            const bool on = r < W.cd, last = j.it.last, rev = W.rev;
            const size_t of = (size_t)bd * W.cd;
            const float rate = w.job->rate;
            float R[DB];
            {
                const float* from = nullptr;
                int64_t fi = 0;
                float age = 1.f;
                if (!kStates && on) {
                    if (j.it.m > 0) { from = W.slots + ((size_t)(j.it.slot - 1) * A.heads + head) * of + r * W.sj; fi = W.si; }
                    else if (W.first) { from = W.first + ((size_t)j.it.seq * A.heads + head) * of + r * W.fj; fi = W.fi; age = rev || j.it.len == 0 ? 1.f : power(rate, 1); }
                }
#pragma unroll
                for (int i = 0; i < DB; ++i) R[i] = 0.f;
                if (!kStates && (j.it.m > 0 || W.first))
#pragma unroll
                for (int i = 0; i < DB; i += 8) {
                    const bool there = from && i < bd;                     // (sizes are multiples of 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (there) { R[i + e] = age * *from; from += fi; }
                    }
                }
            }
            const int adding = chunks - (kStates || (last && W.last) ? 0 : 1);
            for (int c = 0; c <= chunks && chunks > 0; ++c) {
                // the memory behind chunk c - 1, and its image for chunk c
                const bool adds = c > 0 && c <= adding, shows = !kStates && c < chunks;
                float keep = 1.f, ahead[16];
                if (c > 0) {
                    ok = warp_wait(&bars->d, w.g & 1, dead);
                    if (!ok) break;
                    ++w.g;
                    if (adds) {
                        order_after();
                        const int n = w.tokens(c - 1);
                        const int near = !kStates && last && c == chunks && !rev ? 1 : 0;
                        keep = power(rate, n - near);                      // forward, the memory that is given out is not aged
                        // a key that is not finite makes all columns so, a value its own column from end to end
                        tensor_load16(ahead, D + mine);
                        tensor_load_wait();
                        if (((volatile uint32_t*)bars->odd)[(w.g - 1) & 1] == w.g || __any_sync(~0u, !isfinite(ahead[0]))) {
                            careful_sum<T>(W, j.it.batch, head, w.begin(c - 1, rev), n, r, rate, near, kHalfs ? 1.f / ((volatile float*)bars->down)[(w.g - 1) & 1] : 1.f, D + mine);
                            tensor_load16(ahead, D + mine);
                            tensor_load_wait();
                        }
                    }
                }
                float up = 1.f;
                const float down = kHalfs && adds ? ((volatile float*)bars->down)[(w.g - 1) & 1] : 1.f;
                if (kHalfs && adds)
#pragma unroll
                    for (int i = 0; i < DB; i += 16) {
                        if (i >= bd) continue;                             // (nothing was put there)
                        float x[16];
                        if (i) {
                            tensor_load16(x, D + mine + i);
                            tensor_load_wait();
                        }
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            float (&d)[16] = i ? x : ahead;
                            mul2(d[e], d[e + 1], down, down);
                            fma2(R[i + e], R[i + e + 1], keep, d[e], d[e + 1]);
                        }
                    }
                if (kHalfs && shows) {
                    float most = 0.f;
#pragma unroll
                    for (int i = 0; i < DB; ++i) most = fmaxf(most, fabsf(R[i]));
                    up = to_middle(most, cs[(w.g & 1) * 128 + r]);
                }
#pragma unroll
                for (int i = 0; i < DB; i += 16) {
                    if (i >= bd) continue;
                    if (!kHalfs && adds) {
                        float x[16];
                        if (i) tensor_load_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = ahead[e];
                        if (i + 16 < DB && i + 16 < bd) tensor_load16(ahead, D + mine + i + 16);
#pragma unroll
                        for (int e = 0; e < 16; ++e) R[i + e] = keep * R[i + e] + x[e];
                    }
                    if (shows)
#pragma unroll
                        for (int e = 0; e < 16; e += 8) {
                            uint4 x;
                            float m[8];
#pragma unroll
                            for (int u = 0; u < 8; u += 2) {
                                m[u] = R[i + e + u]; m[u + 1] = R[i + e + u + 1];
                                if (kHalfs) mul2(m[u], m[u + 1], up, up);
                            }
                            x.x = Two<T>::pack(m[0], m[1]); x.y = Two<T>::pack(m[2], m[3]); x.z = Two<T>::pack(m[4], m[5]); x.w = Two<T>::pack(m[6], m[7]);
                            *reinterpret_cast<uint4*>(image + (i >> 6) * kHalf + r * 128 + ((((i + e) >> 3) & 7) ^ (r & 7)) * 16) = x;
                        }
                }
                if (c == chunks) break;
                order_shared();
                order_before();
                bar_arrive(&bars->r);
            }
            float* out = nullptr;
            int64_t oi = 0;
            if (kStates) { out = W.slots + ((size_t)j.it.slot * A.heads + head) * of + r * W.sj; oi = W.si; }
            else if (last && W.last) { out = W.last + ((size_t)j.it.seq * A.heads + head) * of + r * W.lj; oi = W.li; }
            if (!ok)
#pragma unroll
                for (int i = 0; i < DB; ++i) R[i] = __int_as_float(0x7fc00000);
            if (out && on) {
                volatile float* to = out;                                  // (volatile: one address after the other, not all at once)
#pragma unroll
                for (int i = 0; i < DB; i += 8)
                    if (i < bd)
#pragma unroll
                        for (int e = 0; e < 8; ++e) { *to = R[i + e]; to += oi; }
            }
        }
    } else make_parts(tid - 256, kStates ? 1 : 0);
    __syncwarp();
    if (lane == 0 && warp < 8 && (!kStates || warp >= 4)) atomicMin(&bars->undone, w.at);        // (y or memory are whole up to here)
    order_before();
    __syncthreads();
    order_after();
    if (dead->dead && (warp < 4 || (warp >= 8 && warp < 12))) lose_all<kStates>(G, bars, warp < 4 ? tid : tid - 128);
    if (warp == 13) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

}  // namespace pcr
