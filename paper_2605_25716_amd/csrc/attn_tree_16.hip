// Attention over a paged cache in 16-bit storage for rows with masks of their own (fedrag_paged_tree_attn).
#include "attn_paged_chunk.h"
#include "attn_tree.h"

namespace fedrag {

// Requests of at most 16 NQ SUBS rows.
template <class T, int D, int NQ, int SUBS>
FEDRAG_KERNEL __launch_bounds__(kTreeWaves * kWave, 2) void tree_16_kernel(const PagedArgs a, uint32_t shares) {
    if (SUBS > 1 && tree_index<SUBS>(blockIdx.x).share >= shares) return;  // (what makes the grid a whole number of XCDs)
    constexpr int SLOT = kDecTile * D * 2;
    __shared__ __attribute__((aligned(16))) char ks[kTreeWaves * SLOT], vs[kTreeWaves * SLOT];
    __shared__ TreeSmall<NQ> sm;
    struct Slots {
        char* p;
        __device__ __forceinline__ char* operator()(int w) const { return p + w * SLOT; }
    };
    tree_body<T, D, NQ, SUBS, 0>(a, blockIdx.x, Slots{ks}, Slots{vs}, sm);
}

// Requests of many rows (a), and with FEW of at most 32 (d): `first` workgroups of many, one to a compute unit; then all of few; then the rest.
template <class T, int D, bool FEW>
FEDRAG_KERNEL __launch_bounds__(kTreeWaves * kWave, 2) void tree_many_16_kernel(const PagedArgs a, const PagedArgs d, int chunks, int first) {
    __shared__ __attribute__((aligned(16))) char ks0[kPreK * D * 2], ks1[kPreK * D * 2], vs0[kPreK * D * 2], vs1[kPreK * D * 2];
    if constexpr (!FEW) {
        __shared__ int flags[kTreeWaves + 1];
        paged_chunk_body<T, D, kTreeWaves, 0, 2, true>(a, blockIdx.x, ks0, ks1, vs0, vs1, flags);
    } else {
        static_assert(2 * kDecTile == kPreK, "both forms share a launch, and its slots");
        __shared__ TreeSmall<2> sm;
        struct Slots {
            char *p, *q;
            __device__ __forceinline__ char* operator()(int w) const { return (w < 2 ? p : q) + w % 2 * (kDecTile * D * 2); }
        };
        const int i = (int)blockIdx.x, few = (int)gridDim.x - chunks;
        if (i >= first && i < first + few)
            tree_body<T, D, 2, 1, 1>(d, (uint32_t)(i - first), Slots{ks0, ks1}, Slots{vs0, vs1}, sm);
        else
            paged_chunk_body<T, D, kTreeWaves, 0, 1, true>(a, (uint32_t)(i < first ? i : i - few), ks0, ks1, vs0, vs1, (int*)&sm);
    }
}

template <class T, int D>
static hipError_t launch_tree_16_t(const PagedArgs& a, int64_t many, const PagedArgs& d, int64_t few, hipStream_t stream) {
    if (many > 0) {
        const int64_t cus = attn_target_wgs();
        const auto kernel = few > 0 ? tree_many_16_kernel<T, D, true> : tree_many_16_kernel<T, D, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(many + few)), dim3(kTreeWaves * kWave), 0, stream, a, d, (int)many,
                           (int)(many < cus ? many : cus));
    } else {
        const auto kernel = d.cut.tile_shift == 4 ? tree_16_kernel<T, D, 1, 1> : d.cut.tile_shift == 5 ? tree_16_kernel<T, D, 2, 1> : tree_16_kernel<T, D, 2, 2>;
        const int64_t grid = d.cut.tile_shift == 6 ? (few + 7) / 8 * 16 : few;  // (tree_index)
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kTreeWaves * kWave), 0, stream, d, (uint32_t)few);
    }
    return hipGetLastError();
}
hipError_t launch_tree_16(const PagedArgs& a, int64_t many, const PagedArgs& d, int64_t few, int D, int dtype, hipStream_t stream) {
    if (dtype == FEDRAG_BF16) return D == 128 ? launch_tree_16_t<BF16, 128>(a, many, d, few, stream) : launch_tree_16_t<BF16, 64>(a, many, d, few, stream);
    return D == 128 ? launch_tree_16_t<F16, 128>(a, many, d, few, stream) : launch_tree_16_t<F16, 64>(a, many, d, few, stream);
}

}  // namespace fedrag
