// Attention over a paged cache in 16-bit storage for rows with masks of their own (fedrag_paged_tree_attn).
#include "attn_paged_chunk.h"
#include "attn_paged_decode.h"

namespace fedrag {

constexpr int kTree16Waves = 4;

// KIND: 1 requests of few rows, 2 of many, 3 both
template <class T, int D, int KIND>
FEDRAG_KERNEL __launch_bounds__(kTree16Waves * kWave, 2) void tree_16_kernel(const PagedArgs a, const PagedArgs d, int chunks, int first) {
    __shared__ __attribute__((aligned(16))) char ks0[kPreK * D * 2], ks1[kPreK * D * 2], vs0[kPreK * D * 2], vs1[kPreK * D * 2];
    __shared__ PagedSmall<D> sm;
    if constexpr (KIND == 1) {
        paged_decode_body<T, D, 1, true>(d, blockIdx.x, ks0, ks1, vs0, vs1, sm);
    } else if constexpr (KIND == 2) {
        paged_chunk_body<T, D, kTree16Waves, 0, 2, true>(a, blockIdx.x, ks0, ks1, vs0, vs1, (int*)&sm);
    } else {
        const int i = (int)blockIdx.x, decodes = (int)gridDim.x - chunks;
        if (i >= first && i < first + decodes)
            paged_decode_body<T, D, 1, true>(d, (uint32_t)(i - first), ks0, ks1, vs0, vs1, sm);
        else
            paged_chunk_body<T, D, kTree16Waves, 0, 1, true>(a, (uint32_t)(i < first ? i : i - decodes), ks0, ks1, vs0, vs1, (int*)&sm);
    }
}

template <class T, int D>
static hipError_t launch_tree_16_t(const PagedArgs& a, int64_t chunks, const PagedArgs& d, int64_t decodes, hipStream_t stream) {
    const int64_t cus = attn_target_wgs();
    const auto kernel = chunks == 0 ? tree_16_kernel<T, D, 1> : decodes == 0 ? tree_16_kernel<T, D, 2> : tree_16_kernel<T, D, 3>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks + decodes)), dim3(kTree16Waves * kWave), 0, stream, a, d, (int)chunks,
                       (int)(chunks < cus ? chunks : cus));
    return hipGetLastError();
}
hipError_t launch_tree_16(const PagedArgs& a, int64_t chunks, const PagedArgs& d, int64_t decodes, int D, int dtype, hipStream_t stream) {
    if (dtype == FEDRAG_BF16)
        return D == 128 ? launch_tree_16_t<BF16, 128>(a, chunks, d, decodes, stream) : launch_tree_16_t<BF16, 64>(a, chunks, d, decodes, stream);
    return D == 128 ? launch_tree_16_t<F16, 128>(a, chunks, d, decodes, stream) : launch_tree_16_t<F16, 64>(a, chunks, d, decodes, stream);
}

}  // namespace fedrag
