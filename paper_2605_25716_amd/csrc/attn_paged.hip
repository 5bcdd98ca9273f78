// Attention of a ragged step over a paged cache (fedrag_paged_attn).
#include "fedrag_device.h"
#include "fedrag_host.h"

namespace fedrag {

// The plainest form: one wave per row and query head, 64 keys at a time.  Lane = key in the first product, = D / 64 channels in
// the second; running maximum and sum.
template <class E, int D>
FEDRAG_KERNEL __launch_bounds__(64) void paged_attn_rows_kernel(PagedAttnProblem p, int n_tokens) {
    constexpr int DC = D / 64;
    __shared__ float q[D];
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x;
    const int h = blockIdx.y, g = h / (p.Hq / p.Hkv);
    // the last request that starts at or before t
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (p.q_start[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int64_t begin = p.q_start[lo], end = p.q_start[lo + 1];
    if (t < begin || t >= end) return;
    int64_t L = p.kv_lens[lo] < 0 ? 0 : p.kv_lens[lo];
    if (p.causal) {
        L = L - (end - begin) + (t - begin) + 1;
        L = L < 0 ? 0 : L;
    }
    const int64_t room = p.max_pages << p.pages.shift;
    L = L < room ? L : room;
    const E* Q = (const E*)(p.Q + h * p.q_head_stride + t * p.q_token_stride);
    for (int c = lane; c < D; c += 64) q[c] = (float)Q[c];
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[DC] = {};
    auto row_of = [&](const char* base, int64_t key, uint32_t id) {
        return (const E*)(base + id * p.pages.page_bytes) + (((int64_t)g << p.pages.shift) + (key & (n_tokens - 1))) * D;
    };
    for (int64_t k0 = 0; k0 < L; k0 += 64) {
        const int64_t key = k0 + lane;
        uint32_t id = 0xffffffffu;
        if (key < L) id = (uint32_t)p.table[lo * p.max_pages + (key >> p.pages.shift)];
        float s = -INFINITY;
        if (id < p.pages.n_pages) {
            const E* K = row_of(p.pages.K, key, id);
            float x = 0.f;
            for (int c = 0; c < D; ++c) x = __builtin_fmaf((float)K[c], q[c], x);
            s = x * p.scale;
        }
        float top = s;
        for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float m_new = fmaxf(m, top);
        if (m_new == -INFINITY) continue;
        const float alpha = m == -INFINITY ? 0.f : expf(m - m_new);
        const float w = s == -INFINITY ? 0.f : expf(s - m_new);
        float sum = w;
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
        l = l * alpha + sum;
        m = m_new;
        for (int c = 0; c < DC; ++c) acc[c] *= alpha;
        for (int k = 0; k < 64; ++k) {
            const uint32_t kid = __shfl(id, k);
            const float wk = __shfl(w, k);
            if (kid >= p.pages.n_pages) continue;
            const E* V = row_of(p.pages.V, k0 + k, kid);
            for (int c = 0; c < DC; ++c) acc[c] = __builtin_fmaf(wk, (float)V[lane * DC + c], acc[c]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    float* O = p.O + ((int64_t)h * p.T + t) * D + lane * DC;
    for (int c = 0; c < DC; ++c) O[c] = l > 0.f || l != l ? acc[c] * inv : 0.f;
    if (lane == 0) p.lse[(int64_t)h * p.T + t] = l > 0.f || l != l ? m + logf(l) : -INFINITY;
}

size_t paged_attn_workspace_bytes(int, int, int, int, int, int64_t, int64_t, int, int64_t) { return 0; }

hipError_t launch_paged_attn(const PagedAttnProblem& p, hipStream_t stream) {
    if (p.Hq > 65535 || !grid_fits(p.T * p.Hq, 64)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)p.T, (unsigned)p.Hq);
#define FEDRAG_ROWS(E) (p.D == 128 ? paged_attn_rows_kernel<E, 128> : paged_attn_rows_kernel<E, 64>)
    const auto kernel = p.dtype == FEDRAG_F32 ? FEDRAG_ROWS(float) : p.dtype == FEDRAG_BF16 ? FEDRAG_ROWS(__bf16) : FEDRAG_ROWS(_Float16);
#undef FEDRAG_ROWS
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, stream, p, 1 << p.pages.shift);
    return hipGetLastError();
}

}  // namespace fedrag
