// Host side of the walks on the tensor cores: maps of the operands for copies of tiles, and the launch.
#include "pcr_decay_tiles.h"

#include <cudaTypedefs.h>
#include <stdint.h>

#include <algorithm>

#include "pcr_decay_tiles.cuh"
#include "pcr_launches.h"

namespace pcr {

namespace {

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static const PFN_cuTensorMapEncodeTiled_v12000 f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return f;
}

// Rows that copies of tiles and vectors of 16 bytes can take.
bool fits(const pcr_rows& r, int64_t batch, int64_t tokens, int heads) {
    const int64_t size[3] = {batch, tokens, heads};
    if (reinterpret_cast<uintptr_t>(r.at) % 16) return false;
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (r.stride[i] <= 0 || r.stride[i] % 8 || r.stride[i] >= (int64_t)1 << 38)) return false;
    return true;
}

bool map_of(CUtensorMap* m, const pcr_rows& r, const pcr_decay_args& a, int heads, int dim) {
    const cuuint64_t size[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)a.tokens, (cuuint64_t)a.batch};
    const int64_t st[3] = {r.stride[2], r.stride[1], r.stride[0]};
    cuuint64_t step[3];
    for (int i = 0; i < 3; ++i) step[i] = size[i + 1] > 1 ? (cuuint64_t)st[i] * 2 : 256;       // (a single one has no step)
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)kTile, 1}, each[4] = {1, 1, 1, 1};
    return encoder()(m, a.dtype == PCR_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(r.at), size, step, box, each,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DB, bool kStates>
int launch(TileArgs& G, unsigned keys, int sms, cudaStream_t st) {
    constexpr int kShared = TileShared<DB, kStates>::kBytes;
    if (cudaFuncSetAttribute(tile_kernel<T, DB, kStates>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared) != cudaSuccess) {
        cudaGetLastError();
        return PCR_E_CUDA;
    }
    G.items = keys * G.walks.heads * G.walks.kinds;
    tile_kernel<T, DB, kStates><<<kStates ? std::min(G.items, (unsigned)sms) : G.items, kTileThreads, kShared, st>>>(G);
    ++g_launches;
    return cudaGetLastError() == cudaSuccess ? PCR_OK : PCR_E_CUDA;
}
template <typename T>
int launch_sizes(TileArgs& G, unsigned keys, int sms, cudaStream_t st) {
    int bd = 0;
    for (int i = 0; i < G.walks.kinds; ++i) bd = std::max(bd, G.walks.w[i].bd);
    if (G.walks.states) return bd <= 64 ? launch<T, 64, true>(G, keys, sms, st) : launch<T, 128, true>(G, keys, sms, st);
    return bd <= 64 ? launch<T, 64, false>(G, keys, sms, st) : launch<T, 128, false>(G, keys, sms, st);
}

}  // namespace

bool tiles_fit(const pcr_decay_args& a, bool back) {
    if (a.dtype == PCR_F32 || a.k_dim > 128 || a.v_dim > 128 || a.k_dim % 8 || a.v_dim % 8 || a.batch * a.tokens == 0 || !encoder()) return false;
    // (one CTA for every segment, head and gradient, numbered in 31 bits)
    if ((a.sequences + a.batch * (a.tokens / kTile + 1)) * a.q_heads * (back ? 3 : 1) > INT32_MAX) return false;
    const bool in = fits(a.q, a.batch, a.tokens, a.q_heads) && fits(a.k, a.batch, a.tokens, a.k_heads) && fits(a.v, a.batch, a.tokens, a.k_heads) && fits(a.out, a.batch, a.tokens, a.q_heads);
    if (!in || !back) return in;
    return fits(a.dq, a.batch, a.tokens, a.q_heads) && fits(a.dk, a.batch, a.tokens, a.k_heads) && fits(a.dv, a.batch, a.tokens, a.k_heads);
}

int launch_tiles(const WalkArgs& walks, const int (*of)[3], const pcr_decay_args& a, unsigned keys, int parts, int sms, cudaStream_t st) {
    TileArgs G;
    G.walks = walks;
    G.parts = parts;
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 3; ++j) G.of[i][j] = of[i][j];
        Walk& w = G.walks.w[i];
        w.wide = reinterpret_cast<uintptr_t>(w.y) % 32 == 0 && w.ys[0] % 16 == 0 && w.ys[1] % 16 == 0 && w.ys[2] % 16 == 0;
    }
    if (!map_of(&G.maps.q, a.q, a, a.q_heads, a.k_dim) || !map_of(&G.maps.k, a.k, a, a.k_heads, a.k_dim) || !map_of(&G.maps.v, a.v, a, a.k_heads, a.v_dim) ||
        !map_of(&G.maps.g, a.out, a, a.q_heads, a.v_dim)) return PCR_E_CUDA;
    return a.dtype == PCR_F16 ? launch_sizes<__half>(G, keys, sms, st) : launch_sizes<__nv_bfloat16>(G, keys, sms, st);
}

}  // namespace pcr
