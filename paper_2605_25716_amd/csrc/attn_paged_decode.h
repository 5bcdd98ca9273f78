// Attention over a paged cache for requests of few rows (at most 16 to a KV head with its group's heads: a decoded token,
// a few tokens), 16-bit storage.  Bound by HBM: every K, V byte is read once (64 tokens over 1000 to 32768 keys, 32 heads of 128, 8 KV
// heads: 2.42 GB in 371 us, 6.5 TB/s, where a read-only stream reaches 7.1), and one request by the chain of its trips (192 keys 7.3 us).
//
// One workgroup = an even share of all KV heads' keys of all requests (attn_paged.h), one span of a head's keys after the other; its
// waves take 32-key tiles in turn.  A tile goes
// from its pages to LDS in whole rows, 1 KiB of them a load, into slots that belong to one wave and need no barrier; K's slot is
// filled again after the first product, V's after the second, so that two tiles' worth of loads fly behind every step, and two
// workgroups share a compute unit: 128 KiB in flight at 128 columns.  A load's rows lie in one page (16 tokens at least), so
// its buffer descriptor is that page's head: it begins at the row and ends with the request's tokens, or is empty where the
// table names no page, and what it does not cover arrives as zeros.  Page ids come 64 half tiles at a time, one a lane.
// Lane l of a wave: lr = l % 16, lq = l / 16.
//   S^T (32 keys x 16 rows) = K (32 x d) . Q^T (d x 16): two 16-key MFMA tiles; this lane holds row lr and keys 16 mt + 4 lq + r,
//   which are also its contraction slice of O^T (d x 16) += V^T (d x 32) . P^T (32 x 16), whose V^T operands come through
//   the transposing LDS read.
// Probabilities enter the second product as two storage-type terms (about 16 significant bits): outputs are fp32.
#pragma once
#include "attn_paged.h"

namespace fedrag {

// What a workgroup has in LDS beside its tiles of K and of V, which are arrays of the kernel (one for every two waves' slots, shared
// with the other form): the waves' maxima and sums of the rows, the keys that a row sees, and the requests that lanes have looked up.
template <int D>
struct PagedSmall {
    float m[kDecWaves][16], l[kDecWaves][16];
    int lim[16];
    PagedLanes lanes;
};
// Wave w's slot of two arrays (by value: a choice between variables that a lambda holds puts them in scratch memory).
__device__ __forceinline__ char* paged_slot(char* first, char* second, int w, int bytes) { return (w < 2 ? first : second) + w % 2 * bytes; }
// ARGS: which of the kernel's arguments `a` is.
template <class T, int D, int ARGS>
__device__ __forceinline__ void paged_decode_body(const PagedArgs& a, uint32_t index, char* ks0, char* ks1, char* vs0, char* vs1, PagedSmall<D>& sm) {
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    constexpr int KS = D / 32;   // contraction steps of the first product
    constexpr int DCH = D / 16;  // 16-row tiles of O^T
    constexpr int ROWB = D * 2;
    constexpr int SLOT = kDecTile * ROWB;
    constexpr int WAVES = kDecWaves;
    constexpr int OROW = (D + 4) * 4;
    static_assert(SLOT >= 8 * OROW, "eight rows of outputs fit a slot");
    const float scale_log2 = a.scale * kLog2e;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave;
    const int lr = lane % 16, lq = lane / 16;
    const PagedShares<PagedArgsLate> shares(late_args<ARGS>(), sm.lanes);
    // `p`: the tile; units u0 .. u0 + take of its n
    auto span = [&](const PagedSpan& p, uint32_t u0, uint32_t take) {
    const PagedRequest& q = p.req;
    const int row0 = p.tile << a.cut.tile_shift;                                  // the tile's first flattened row
    const int R = q.R - row0 < 16 ? q.R - row0 : 16;
    const int row = row0 + (lr < R ? lr : R - 1);
    const int lim = paged_limit(a, q, row);                                // this lane's row sees keys < lim
    const int lim_min = __builtin_amdgcn_readlane(lim, 0), lim_max = __builtin_amdgcn_readlane(lim, 15);
    const int k_begin = (int)((int64_t)u0 << a.cut.unit_shift);            // below the request's keys: 31 bits
    const int64_t span_end = ((int64_t)u0 + take) << a.cut.unit_shift;
    const int k_end = span_end < lim_max ? (int)span_end : lim_max;        // (may lie before k_begin: nothing to see)

    // Q^T operands: column lr, channels 32 ks + 8 lq; rows that are not there are zeros
    const uint32_t tok = a.by_g.div((uint32_t)row), hg = (uint32_t)row - tok * a.by_g.d;
    const char* Qr = a.Q + ((int64_t)p.head * a.G + hg) * a.q_head_stride + ((int64_t)q.begin + tok) * a.q_token_stride;
    vec8 qop[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) qop[i] = *(const vec8*)(Qr + (i * 32 + lq * 8) * 2);

    f32x4_t acc[DCH];
#pragma unroll
    for (int i = 0; i < DCH; ++i) acc[i] = zero_vec<f32x4_t>();
    // the lowest finite value, not -inf: a row may see nothing of a tile, and -inf - m has to be -inf then
    float m_run = -__FLT_MAX__, l_run = 0.f;

    constexpr int CH = D / 8;           // 16-byte chunks per row
    constexpr int RPW = kWave / CH;     // rows per load
    constexpr int HL = 16 / RPW;        // loads per half tile
    constexpr int KL = 2 * HL;
    auto swz_k = [&](int r) { return D == 128 ? r % 16 : r / 2 % 8; };
    auto swz_v = [&](int r) { return D == 128 ? r % 4 * 4 + r / 4 % 2 * 2 : r / 2 % 4 * 2; };
    const int64_t table0 = (int64_t)p.b * a.max_pages;
    const int shift = a.pages.shift;
    const int n_tiles = (k_end - k_begin + kDecTile - 1) / kDecTile;
    const int n_mine = n_tiles > wave ? (n_tiles - wave + WAVES - 1) / WAVES : 0;
    // lane l: bytes from K's or V's first page to half tile l of this wave's 32 tiles from the i-th on; < 0: there are no rows, or no
    // page for them
    auto offsets = [&](int i) {
        const int64_t key = (int64_t)k_begin + ((int64_t)wave + (int64_t)(i + lane / 2) * WAVES) * kDecTile + lane % 2 * 16;
        int id = -1;
        if (key < k_end) id = a.table[table0 + (key >> shift)];
        return (uint32_t)id < a.pages.n_pages
                   ? (int64_t)id * a.pages.page_bytes + (((int64_t)p.head << shift) + ((int)key & ((1 << shift) - 1))) * ROWB : (int64_t)-1;
    };
    int64_t offset = -1;
    auto offset_of = [&](int half) {
        return ((int64_t)__builtin_amdgcn_readlane((int)(offset >> 32), half) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)offset, half);
    };
    auto fill = [&](int i, char* slot, bool is_k) {  // the wave's i-th tile, i within the 32 whose offsets are here
        const int left = k_end - k_begin - (wave + i * WAVES) * kDecTile;  // rows from its first one on
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t off = offset_of(2 * (i % 32) + h);
            const int bytes = off < 0 ? 0 : (left - 16 * h < 16 ? left - 16 * h : 16) * ROWB;
            const __amdgpu_buffer_rsrc_t rs =
                __builtin_amdgcn_make_buffer_rsrc((void*)((is_k ? a.pages.K : a.pages.V) + (off < 0 ? 0 : off)), 0, bytes, 0x00020000);
#pragma unroll
            for (int j = 0; j < HL; ++j) {
                const int r = lane / CH + j * RPW;
                const int at = r * ROWB + (((lane % CH) ^ (is_k ? swz_k(r) : swz_v(r))) << 4);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rs, (void __attribute__((address_space(3)))*)(slot + (h * HL + j) * (kWave * 16)), 16, at, 0, 0, 2);
            }
        }
    };
    auto wait_loads = [&](auto n) {  // all loads done but the N asked for last
        constexpr int N = decltype(n)::value;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
        __builtin_amdgcn_sched_barrier(0);
    };
    char *const kslot = paged_slot(ks0, ks1, wave, SLOT), *const vslot = paged_slot(vs0, vs1, wave, SLOT);

    // One tile; MORE: the next one's loads are asked for as its slots come free.
    auto step = [&](int i, auto more) {
        constexpr bool MORE = decltype(more)::value;
        const int key0 = k_begin + (wave + i * WAVES) * kDecTile;
        const int id0 = __builtin_amdgcn_readlane((int)(offset >> 32), 2 * (i % 32)), id1 = __builtin_amdgcn_readlane((int)(offset >> 32), 2 * (i % 32) + 1);
        const bool masked = key0 + kDecTile > (lim_min < k_end ? lim_min : k_end) || (id0 | id1) < 0;
        if (MORE && i % 32 == 31) offset = offsets(i + 1);
        wait_loads(std::integral_constant<int, KL>{});  // K's (V's are younger)
        f32x4_t s[2];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            s[mt] = zero_vec<f32x4_t>();
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                const vec8 kop = *(const vec8*)(kslot + (mt * 16 + lr) * ROWB + (((4 * j + lq) ^ swz_k(lr)) << 4));
                s[mt] = T::mfma16(kop, qop[j], s[mt]);
            }
        }
        if constexpr (MORE) {
            __builtin_amdgcn_sched_barrier(0);
            fill(i + 1, kslot, true);
            __builtin_amdgcn_sched_barrier(0);
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e / 4][e % 4] * scale_log2;
        if (masked) {
            const int left = (lim < k_end ? lim : k_end) - key0 - lq * 4;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((e / 4) * 16 + e % 4 >= left || (e < 4 ? id0 : id1) < 0) x[e] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e]);
        mx = xor32_max(xor16_max(mx));
        const float m_new = fmaxf(m_run, paged_reference<T>(mx));
        const float alpha = fast_exp2(m_run - m_new);
        if (masked) {  // a key alone has a power of two
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= m_new;
        } else {  // one rounding of the exponent's argument
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(s[e / 4][e % 4], scale_log2, -m_new);
        }
        float sum = 0.f;
        vec8 ph, pl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float pe = fast_exp2(x[e]);
            sum += pe;
            ph[e] = T::from_float(pe);
            pl[e] = T::from_float(pe - T::to_float(ph[e]));
        }
        l_run = l_run * alpha + sum;
        m_run = m_new;
        wait_loads(std::integral_constant<int, MORE ? KL : 0>{});
        u32x4_t vt[DCH];
#pragma unroll
        for (int t = 0; t < DCH; ++t)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const int r = mt * 16 + lq * 4 + lr / 4;
                const u32x2_t w = lds_read_tr16(vslot + r * ROWB + (((2 * t + lr % 4 / 2) ^ swz_v(r)) << 4) + lr % 2 * 8);
                vt[t][2 * mt] = w[0];
                vt[t][2 * mt + 1] = w[1];
            }
#pragma unroll
        for (int t = 0; t < DCH; ++t) acc[t] *= alpha;
        if (masked && lim_min != lim_max) {
            // Some rows see a token that others do not.  Where its V is not finite, a product with the probability 0 would bring it to
            // them: such values are taken out, and added by themselves for the rows that see them.
            constexpr uint32_t kExp = std::is_same<T, BF16>::value ? 0x7f80u : 0x7c00u;
            bool odd = false;
#pragma unroll
            for (int t = 0; t < DCH; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool lo = (vt[t][w] & kExp) == kExp, up = (vt[t][w] >> 16 & kExp) == kExp;
                    odd |= lo || up;
                }
            if (__builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll
                for (int t = 0; t < DCH; ++t)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t v = vt[t][w];
                        if ((v & kExp) == kExp) v &= 0xffff0000u;
                        if ((v >> 16 & kExp) == kExp) v &= 0xffffu;
                        vt[t][w] = v;
                    }
                const int seen = (lim < k_end ? lim : k_end) - key0;
                for (int key = 0; key < kDecTile && key < seen; ++key)
#pragma unroll
                    for (int t = 0; t < DCH; ++t) {
                        // acc[t] holds channels 16 t + 4 lq + 0..3: half of a 16-byte chunk
                        const u32x2_t w = *(const u32x2_t*)(vslot + key * ROWB + (((2 * t + lq / 2) ^ swz_v(key)) << 4) + lq % 2 * 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t v = (e < 2 ? w[0] : w[1]) >> (e % 2 * 16) & 0xffffu;
                            if ((v & kExp) == kExp) acc[t][e] += T::to_float(__builtin_bit_cast(elem, (uint16_t)v));
                        }
                    }
            }
        }
#pragma unroll
        for (int t = 0; t < DCH; ++t) {
            const vec8 vop = __builtin_bit_cast(vec8, vt[t]);
            acc[t] = T::mfma16(vop, ph, acc[t]);
            acc[t] = T::mfma16(vop, pl, acc[t]);
        }
        if constexpr (MORE) {
            __builtin_amdgcn_sched_barrier(0);
            fill(i + 1, vslot, false);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (n_mine > 0) {
        offset = offsets(0);
        fill(0, kslot, true);
        fill(0, vslot, false);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < KS; ++i) {  // waited for here: ahead of a loop the compiler waits for all in flight
            u32x4_t w = __builtin_bit_cast(u32x4_t, qop[i]);
            pin_here(w);
            qop[i] = __builtin_bit_cast(vec8, w);
        }
        for (int i = 0; i + 1 < n_mine; ++i) step(i, std::true_type{});
        step(n_mine - 1, std::false_type{});
    }

    // fold the waves (Section 4.1 aggregation, in base 2); a thread finishes 4 columns of a row
    const float l_tot = xor32_sum(xor16_sum(l_run));
    if (lq == 0) {
        sm.m[wave][lr] = m_run;
        sm.l[wave][lr] = l_tot;
        if (wave == 0) sm.lim[lr] = lim < k_end ? lim : k_end;
    }
    if (lr < R) {
#pragma unroll
        for (int t = 0; t < DCH; ++t) *(f32x4_t*)((lr < 8 ? kslot : vslot) + lr % 8 * OROW + (16 * t + 4 * lq) * 4) = acc[t];
    }
    __syncthreads();
    const PagedArgsLate& z = late_args<ARGS>();
    const bool part = take < p.n;
    const int64_t slot = 2 * (int64_t)index + (u0 == 0 ? 1 : 0);
    for (int idx = tid; idx < R * (D / 4); idx += kDecThreads) {
        const int n = idx / (D / 4), c = idx % (D / 4) * 4;
        float M = sm.m[0][n];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm.m[w][n]);
        f32x4_t num = zero_vec<f32x4_t>();
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = fast_exp2(sm.m[w][n] - M);
            const f32x4_t o = *(const f32x4_t*)((n < 8 ? paged_slot(ks0, ks1, w, SLOT) : paged_slot(vs0, vs1, w, SLOT)) + n % 8 * OROW + c * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] = __builtin_fmaf(f, o[e], num[e]);
            den = __builtin_fmaf(f, sm.l[w][n], den);
        }
        const bool any = den != 0.f;  // (not a number where a score was not)
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] = any ? num[e] / den : 0.f;
        const float lse = any ? paged_log2_sum<T>(M, den) * kLn2 : -INFINITY;
        if (!all_finite(num) && __builtin_isfinite(den)) {
            num = paged_with_odd(num, paged_odd_values<elem, D>(z, p.b, p.head, k_begin, sm.lim[n], c));
        }
        const uint32_t t = FastDiv::div_by(z.by_g.m, z.by_g.s, (uint32_t)(row0 + n)), g = (uint32_t)(row0 + n) - t * z.by_g.d;
        const int64_t at = part ? (slot << z.cut.tile_shift) + n : ((int64_t)p.head * z.G + g) * z.T + q.begin + t;
        *(f32x4_t*)((part ? z.part_O : z.O) + at * D + c) = num;
        if (c == 0) (part ? z.part_lse : z.lse)[at] = lse;
    }
    };
    uint32_t pos = index * shares.share;
    const uint32_t end = pos + shares.share;
    for (bool first = true;; first = false) {
        const PagedSpan p = shares.find(late_args<ARGS>(), pos);
        if (p.b < 0) return;
        uint32_t take = p.begin + p.n - pos;
        if (p.n <= shares.whole) {
            // not cut: the share before has it, if it began there
            if (first && pos != p.begin) take |= 0x80000000u;
        } else if (end - pos < take) {
            take = end - pos;
        }
        if (!(take >> 31)) {
            if (!first) __syncthreads();  // the slots have been read by all, and are filled again
            span(p, pos - p.begin, take);
        }
        pos += take & 0x7fffffff;
        if (pos >= end) return;
    }
}

}  // namespace fedrag
