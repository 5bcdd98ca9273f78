// Attention over a paged cache in fp32 storage: the accuracy path.  Products and sums are fp32 on the fp32 matrix cores
// (v_mfma_f32_16x16x4_f32), exponentials and logarithms the accurate library ones.
//
// One workgroup = 16 NQ flattened rows of one request and KV head x one run of keys; its four waves take 16-key tiles in turn
// and are folded at the end.  Sixteen keys lie in one page, so a tile's rows have one buffer descriptor, which ends with the
// request's tokens (empty where the table names no page): what it does not cover arrives as zeros.
// Lane l of a wave: lr = l % 16, lq = l / 16.
//   S^T (16 keys x 16 rows) = K . Q^T, four channels an instruction: lane (lr, lq) supplies channels 16 j + 4 lq + e of key lr and of
//   row lr, and ends up with row lr and keys 4 lq + r.
//   O^T (d x 16) += V^T . P^T, four keys an instruction: in instruction r lane group lq contracts key 4 lq + r, whose probability it
//   holds; channels are assigned d = DCH i + t (tile t, row i), so that lane (i = lr) needs DCH contiguous ones of each key.
// Bound by the matrix pipe (64 NQ instructions of 32 cycles per 16 KiB of K, V at 128 columns): 1024 rows of 32 heads over 4096 keys
// 571 to 604 us, 105 TFLOP/s, where a library product of fp32 reaches 150 (every step of 16 keys rescales all outputs, a multiplication
// for every two matrix instructions at 128 columns); single tokens by HBM (64 over 1000 keys 93 us, 5.6 TB/s).
// Rows with masks of their own: 32 requests of 1000 to 32768 tokens, 8 KV heads of 128, 2.46 GB: 16 rows a KV head 433 us (5.7 TB/s), 64 rows 832 (94
// TFLOP/s; each of two tiles reads the keys, 5.9 TB/s if both did so from HBM: which of the two bounds it was not told apart).
#include "attn_paged.h"

namespace fedrag {

__device__ __forceinline__ f32x4_t paged_mfma_f32(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// TREE: rows have masks of their own.
template <int D, int NQ, bool TREE>
__device__ __forceinline__ void paged_f32_body(const PagedArgs& a) {
    constexpr int W = 4;
    constexpr int kKeys = 16;    // keys per wave step
    constexpr int DCH = D / 16;  // channels per lane and key of V (= 16-row tiles of O^T)
    constexpr int KJ = D / 16;   // 16-byte reads per lane of a K or Q row
    constexpr int ROWB = D * 4;
    constexpr int LDO = D + 4;
    __shared__ float sm_m[W][NQ * 16], sm_l[W][NQ * 16];
    __shared__ int sm_lim[NQ * 16];
    __shared__ __attribute__((aligned(16))) float sm_o[W][NQ * 16][LDO];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave;
    const int lr = lane % 16, lq = lane / 16;
    const PagedPiece p = paged_piece<false>(a, blockIdx.x);
    if (p.b < 0) return;
    const PagedRequest& rq = p.req;
    const int row0 = p.tile * (NQ * 16);
    const int last = (row0 + NQ * 16 < rq.R ? row0 + NQ * 16 : rq.R) - 1;
    const int base = TREE ? paged_base(rq, (int)a.by_g.div((uint32_t)rq.R)) : 0;
    const int lim_min = TREE ? (base < 0 ? 0 : (base < rq.keys ? base : rq.keys)) : paged_limit(a, rq, row0);
    const int lim_max = TREE ? rq.keys : paged_limit(a, rq, last);
    const int k_begin = (int)((int64_t)p.run * p.per << a.cut.unit_shift);
    const int64_t run_end = (int64_t)k_begin + ((int64_t)p.per << a.cut.unit_shift);
    const int k_end = run_end < lim_max ? (int)run_end : lim_max;
    if (p.run > 0 && k_end <= k_begin) return;  // a run behind what the tile sees: its partial is not asked for

    f32x4_t q[NQ][KJ];
    int lim[NQ];
    f32x4_t acc[NQ][DCH];
    float m_run[NQ], l_run[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = row0 + n * 16 + lr < rq.R ? row0 + n * 16 + lr : rq.R - 1;  // (rows that are not there: a real one, not written)
        const uint32_t t = a.by_g.div((uint32_t)row), g = (uint32_t)row - t * a.by_g.d;
        const char* Q = a.Q + ((int64_t)p.head * a.G + g) * a.q_head_stride + ((int64_t)rq.begin + t) * a.q_token_stride + 16 * lq;
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[n][j] = *(const f32x4_t*)(Q + 64 * j);
        const int own = TREE ? rq.keys : paged_limit(a, rq, row);
        lim[n] = own < k_end ? own : k_end;
        m_run[n] = -__FLT_MAX__;  // not -inf: a row may see nothing of a tile, and -inf - m has to be -inf then
        l_run[n] = 0.f;
#pragma unroll
        for (int t2 = 0; t2 < DCH; ++t2) acc[n][t2] = zero_vec<f32x4_t>();
    }

    const int64_t table0 = (int64_t)p.b * a.max_pages;
    const int shift = a.pages.shift;
    const int n_tiles = (k_end - k_begin + kKeys - 1) / kKeys;
    const int n_mine = n_tiles > wave ? (n_tiles - wave + W - 1) / W : 0;
    int ids = -1;  // lane l: page of this wave's tile l of the 64 at hand; -1: none
    auto load_ids = [&](int i) {
        const int64_t key = (int64_t)k_begin + ((int64_t)wave + (int64_t)(i + lane) * W) * kKeys;
        int id = -1;
        if (key < k_end) id = a.table[table0 + (key >> shift)];
        return (uint32_t)id < a.pages.n_pages ? id : -1;
    };
    auto rows_of = [&](const char* base, int id, int key) {
        const char* page = base + (int64_t)(id < 0 ? 0 : id) * a.pages.page_bytes + (((int64_t)p.head << shift) + (key & ((1 << shift) - 1))) * ROWB;
        const int left = k_end - key < kKeys ? k_end - key : kKeys;
        return __builtin_amdgcn_make_buffer_rsrc((void*)page, 0, id < 0 ? 0 : left * ROWB, 0x00020000);
    };
    auto load_k = [&](int i, f32x4_t (&k)[KJ]) {
        const __amdgpu_buffer_rsrc_t r = rows_of(a.pages.K, __builtin_amdgcn_readlane(ids, i % 64), k_begin + (wave + i * W) * kKeys);
#pragma unroll
        for (int j = 0; j < KJ; ++j)
            k[j] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, lr * ROWB + 16 * lq + 64 * j, 0, 0));
    };
    f32x4_t k[KJ];
    if (n_mine > 0) {
        ids = load_ids(0);
        load_k(0, k);
    }
    for (int i = 0; i < n_mine; ++i) {
        const int key0 = k_begin + (wave + i * W) * kKeys;
        const int id = __builtin_amdgcn_readlane(ids, i % 64);
        const __amdgpu_buffer_rsrc_t rv = rows_of(a.pages.V, id, key0);
        f32x4_t v[4][DCH / 4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < DCH / 4; ++c)
                v[r][c] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rv, (4 * lq + r) * ROWB + DCH * 4 * lr + 16 * c, 0, 0));
        f32x4_t s[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            f32x4_t part[2] = {zero_vec<f32x4_t>(), zero_vec<f32x4_t>()};  // two chains: no wait for the last result
#pragma unroll
            for (int j = 0; j < KJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e % 2] = paged_mfma_f32(k[j][e], q[n][j][e], part[e % 2]);
            s[n] = part[0] + part[1];
        }
        if (i + 1 < n_mine) {
            if (i % 64 == 63) ids = load_ids(i + 1);
            load_k(i + 1, k);
        }
        const bool whole = id >= 0 && key0 + kKeys <= lim_min && key0 + kKeys <= k_end;  // wave-uniform
        uint32_t seen[NQ];  // of the tile's keys, by the rows' masks
        if constexpr (TREE)
            if (!whole) {
                const PagedArgsLate& z = late_args<0>();
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const int row = row0 + n * 16 + lr < rq.R ? row0 + n * 16 + lr : rq.R - 1;
                    seen[n] = (uint32_t)paged_tree_bits(z, rq, base, (int)FastDiv::div_by(z.by_g.m, z.by_g.s, (uint32_t)row), key0);
                }
            }
        if (!whole && lim_min != lim_max) {
            // Some rows see a token that others do not.  Where its V is not finite, a product with the probability 0 would bring it to
            // them: such values are taken out, and added by themselves for the rows that see them.
            bool odd = false;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int t = 0; t < DCH; ++t) odd |= !__builtin_isfinite(v[r][t / 4][t % 4]);
            if (__builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int t = 0; t < DCH; ++t)
                        if (!__builtin_isfinite(v[r][t / 4][t % 4])) v[r][t / 4][t % 4] = 0.f;
                for (int key = 0; key < kKeys; ++key)
#pragma unroll
                    for (int t = 0; t < DCH; ++t) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float x = __builtin_bit_cast(
                                float, __builtin_amdgcn_raw_buffer_load_b32(rv, key * ROWB + (DCH * (4 * lq + r) + t) * 4, 0, 0));
#pragma unroll
                            for (int n = 0; n < NQ; ++n)
                                if (!__builtin_isfinite(x) && key0 + key < lim[n] && (!TREE || (seen[n] >> key & 1))) acc[n][t][r] += x;
                        }
                        __builtin_amdgcn_sched_barrier(0);  // (more of these loads in flight would take registers from the loop)
                    }
            }
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[n][r] *= a.scale;
                if (!whole && (id < 0 || key0 + 4 * lq + r >= lim[n] || (TREE && !(seen[n] >> (4 * lq + r) & 1)))) s[n][r] = -INFINITY;
                mx = fmaxf(mx, s[n][r]);
            }
            mx = xor32_max(xor16_max(mx));
            const float m_new = fmaxf(m_run[n], mx);
            const float alpha = expf(m_run[n] - m_new);
            float pr[4], sum = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pr[r] = expf(s[n][r] - m_new);
                sum += pr[r];
            }
            l_run[n] = l_run[n] * alpha + sum;
            m_run[n] = m_new;
#pragma unroll
            for (int t = 0; t < DCH; ++t) acc[n][t] *= alpha;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int t = 0; t < DCH; ++t) acc[n][t] = paged_mfma_f32(v[r][t / 4][t % 4], pr[r], acc[n][t]);
        }
    }

    // fold the waves (Section 4.1 aggregation); a thread finishes 4 columns of a row
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l_tot = xor32_sum(xor16_sum(l_run[n]));
        if (lq == 0) {
            sm_m[wave][n * 16 + lr] = m_run[n];
            sm_l[wave][n * 16 + lr] = l_tot;
            if (wave == 0) sm_lim[n * 16 + lr] = lim[n];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int t = 0; t < DCH; t += 4) {
                f32x4_t o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = acc[n][t + e][r];
                *(f32x4_t*)&sm_o[wave][n * 16 + lr][DCH * (4 * lq + r) + t] = o;
            }
    }
    __syncthreads();
    for (int idx = tid; idx < (last - row0 + 1) * (D / 4); idx += W * kWave) {
        const int n = idx / (D / 4), c = idx % (D / 4) * 4;
        float M = sm_m[0][n];
#pragma unroll
        for (int w = 1; w < W; ++w) M = fmaxf(M, sm_m[w][n]);
        f32x4_t num = zero_vec<f32x4_t>();
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = expf(sm_m[w][n] - M);
            const f32x4_t o = *(const f32x4_t*)&sm_o[w][n][c];
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] = __builtin_fmaf(f, o[e], num[e]);
            den = __builtin_fmaf(f, sm_l[w][n], den);
        }
        const bool any = den != 0.f;  // (not a number where a score was not)
        const float inv = 1.0f / den;
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] = any ? num[e] * inv : 0.f;
        if (!all_finite(num) && __builtin_isfinite(den)) {
            if constexpr (TREE)
                num = paged_with_odd(num, paged_odd_tree_values<float, D>(late_args<0>(), rq, base, (int)a.by_g.div((uint32_t)(row0 + n)), p.b, p.head, k_begin,
                                                                          sm_lim[n], c));
            else
                num = paged_with_odd(num, paged_odd_values<float, D>(late_args<0>(), p.b, p.head, k_begin, sm_lim[n], c));
        }
        const uint32_t t = a.by_g.div((uint32_t)(row0 + n)), g = (uint32_t)(row0 + n) - t * a.by_g.d;
        const int64_t at = p.runs > 1 ? ((int64_t)p.slot << a.cut.tile_shift) + n : ((int64_t)p.head * a.G + g) * a.T + rq.begin + t;
        *(f32x4_t*)((p.runs > 1 ? a.part_O : a.O) + at * D + c) = num;
        if (c == 0) (p.runs > 1 ? a.part_lse : a.lse)[at] = any ? M + logf(den) : -INFINITY;
    }
}

template <int D, int NQ>
FEDRAG_KERNEL __launch_bounds__(256, 2) void paged_f32_kernel(const PagedArgs a) {
    paged_f32_body<D, NQ, false>(a);
}
template <int D, int NQ>
FEDRAG_KERNEL __launch_bounds__(256, 2) void tree_f32_kernel(const PagedArgs a) {
    paged_f32_body<D, NQ, true>(a);
}

hipError_t launch_paged_f32(const PagedArgs& a, int64_t grid, int D, hipStream_t stream) {
    const bool wide = a.cut.tile_shift == 5;
    const auto kernel = D == 128 ? (wide ? paged_f32_kernel<128, 2> : paged_f32_kernel<128, 1>)
                                 : (wide ? paged_f32_kernel<64, 2> : paged_f32_kernel<64, 1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, stream, a);
    return hipGetLastError();
}
hipError_t launch_tree_f32(const PagedArgs& a, int64_t grid, int D, hipStream_t stream) {
    const bool wide = a.cut.tile_shift == 5;
    const auto kernel = D == 128 ? (wide ? tree_f32_kernel<128, 2> : tree_f32_kernel<128, 1>)
                                 : (wide ? tree_f32_kernel<64, 2> : tree_f32_kernel<64, 1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace fedrag
