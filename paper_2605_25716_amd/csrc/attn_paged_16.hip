// The kernels of attention over a paged cache in 16-bit storage: requests of few rows (attn_paged_decode.h), of many
// (attn_paged_chunk.h), and both in one launch.  A step of a serving node mostly has both, the one bound by HBM and the other by
// the matrix pipe: side by side they take little more than the longer of the two (24 decoding requests beside chunks of 512, 777 and
// 2048 tokens 159 us, one after the other 45 and 143).
#include "attn_paged_chunk.h"
#include "attn_paged_decode.h"

namespace fedrag {

constexpr int kPaged16Waves = 4;
static_assert(kPaged16Waves == kDecWaves, "both forms share a launch");

// KIND: 1 requests of few rows, 2 of many, 3 both
template <class T, int D, int KIND>
FEDRAG_KERNEL __launch_bounds__(kPaged16Waves * kWave, 2) void paged_16_kernel(const PagedArgs a, const PagedArgs d, int chunks, int first) {
    __shared__ __attribute__((aligned(16))) char ks0[kPreK * D * 2], ks1[kPreK * D * 2], vs0[kPreK * D * 2], vs1[kPreK * D * 2];
    __shared__ PagedSmall<D> sm;
    if constexpr (KIND == 1) {
        paged_decode_body<T, D, 1>(d, blockIdx.x, ks0, ks1, vs0, vs1, sm);
    } else if constexpr (KIND == 2) {
        paged_chunk_body<T, D, kPaged16Waves, 0, 3>(a, blockIdx.x, ks0, ks1, vs0, vs1, (int*)&sm);
    } else {
        // `first` workgroups of many rows, one to a compute unit; then all of few rows; then the rest
        const int i = (int)blockIdx.x, decodes = (int)gridDim.x - chunks;
        if (i >= first && i < first + decodes)
            paged_decode_body<T, D, 1>(d, (uint32_t)(i - first), ks0, ks1, vs0, vs1, sm);
        else
            paged_chunk_body<T, D, kPaged16Waves, 0, 2>(a, (uint32_t)(i < first ? i : i - decodes), ks0, ks1, vs0, vs1, (int*)&sm);
    }
}

template <class T, int D>
static hipError_t launch_paged_16_t(const PagedArgs& a, int64_t chunks, const PagedArgs& d, int64_t decodes, hipStream_t stream) {
    const int64_t cus = attn_target_wgs();
    const auto kernel = chunks == 0 ? paged_16_kernel<T, D, 1> : decodes == 0 ? paged_16_kernel<T, D, 2> : paged_16_kernel<T, D, 3>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks + decodes)), dim3(kPaged16Waves * kWave), 0, stream, a, d, (int)chunks,
                       (int)(chunks < cus ? chunks : cus));
    return hipGetLastError();
}
hipError_t launch_paged_16(const PagedArgs& a, int64_t chunks, const PagedArgs& d, int64_t decodes, int D, int dtype, hipStream_t stream) {
    if (dtype == FEDRAG_BF16)
        return D == 128 ? launch_paged_16_t<BF16, 128>(a, chunks, d, decodes, stream) : launch_paged_16_t<BF16, 64>(a, chunks, d, decodes, stream);
    return D == 128 ? launch_paged_16_t<F16, 128>(a, chunks, d, decodes, stream) : launch_paged_16_t<F16, 64>(a, chunks, d, decodes, stream);
}

}  // namespace fedrag
