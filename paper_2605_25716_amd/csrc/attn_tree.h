// Attention over a paged cache for rows with masks of their own: the drafted tokens of a step, 16-bit storage.
//
// One workgroup = an even share of all KV heads' keys of all requests (attn_paged.h), for tiles of 16 NQ flattened rows; its waves take
// 32-key tiles in turn, each for all rows, and are folded at the end.  A key tile goes from its pages to LDS in whole rows, into a slot
// that belongs to one wave and needs no barrier; K's half is filled again after the first product, V's after the second, so that
// two tiles' worth of loads fly behind every step, and two workgroups share a compute unit: 128 KiB in flight at 128 columns.
// Bound by reading: 32 requests of 1000 to 32768 tokens, 8 KV heads of 128 in bf16, 1.24 GB: 16 rows a KV head 212 us (5.9 TB/s), 32 rows 224 (5.6).
// SUBS = 2: a tile's rows are two workgroups', which take the same keys at the same time on one XCD: what the one has read is in L2 for
// the other.  64 rows over the same keys 265 to 280 us (4.5 TB/s): 150 with all of them in L2, 200 by HBM, and the two hardly overlap.  (All 64 rows
// in each of four waves, one to a SIMD: 343; eight waves, two to a key tile behind a barrier 265, but half as long again for short requests.)
// Lane l of a wave: lr = l % 16, lq = l / 16.  For each 16 rows g:
//   S^T (32 keys x 16 rows) = K (32 x d) . Q^T (d x 16): two 16-key MFMA tiles; this lane holds row lr and keys 16 mt + 4 lq + r,
//   which are also its contraction slice of O^T (d x 16) += V^T (d x 32) . P^T (32 x 16), whose V^T operands come through
//   the transposing LDS read.  An operand of K or V is read once for all of a wave's rows.
// Probabilities enter the second product as two storage-type terms in fp16 (22 significant bits) and three in bf16 (24; of two workgroups a
// tile two, 16: there the third would cost 3 to 10 %, 64 rows of 64 columns 162 -> 177 us, up to 32 rows 0 to 1.5 %; outputs of drafts behind
// short requests are 2e-7 to 4e-7 off with it, 6e-7 to 1e-6 without).  They are relative to the largest score so far: in a masked
// tile its own probability is a power of two and exact, elsewhere off by what its rounding took; outputs are rescaled only where it moves.
// (Leaving it until it is 2^8 off takes 1 % off the time and doubles the error of rows whose weight sits on few tokens.)
// Only the key tiles that hold drafted tokens are masked, by bits of the rows' words.
// The way of the keys (pages, descriptors, LDS, its swizzles), the walk along a share and the fold of the waves are attn_paged_decode.h's, written
// again for several groups of rows: what is mended in the one has to be looked at in the other.
#pragma once
#include "attn_paged.h"

namespace fedrag {

constexpr int kTreeWaves = 4;

// What a workgroup has in LDS beside its tiles of K and of V, which are arrays of the kernel (one for every two waves' slots, so that a
// launch can share them with the form for many rows): the waves' maxima and sums of the rows, the rows' first words, and the requests
// that lanes have looked up.
template <int NQ>
struct TreeSmall {
    float m[kTreeWaves][16 * NQ], l[kTreeWaves][16 * NQ];
    uint64_t mask[16 * NQ];
    PagedLanes lanes;
};

// A workgroup's share, and which of its tiles' rows.
struct TreeIndex {
    uint32_t share;
    int sub;
};
template <int SUBS>
__device__ __forceinline__ TreeIndex tree_index(uint32_t wg) {
    static_assert(SUBS == 1 || SUBS == 2, "");
    return SUBS == 1 ? TreeIndex{wg, 0} : TreeIndex{wg / 16 * 8 + wg % 8, (int)(wg / 8 % 2)};  // (eight apart: the same XCD)
}

// k_slot_of, v_slot_of: a wave's slot, of 32 rows.  ARGS: which of the kernel's arguments `a` is.
template <class T, int D, int NQ, int SUBS, int ARGS, class Slots>
__device__ __forceinline__ void tree_body(const PagedArgs& a, uint32_t wg, Slots k_slot_of, Slots v_slot_of, TreeSmall<NQ>& sm) {
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    constexpr int KS = D / 32;   // contraction steps of the first product
    constexpr int DCH = D / 16;  // 16-row tiles of O^T
    constexpr int ROWB = D * 2;
    constexpr int SLOT = kDecTile * ROWB;
    constexpr int WAVES = kTreeWaves;
    constexpr int ROWS = 16 * NQ;
    constexpr int PCH = D / 4;  // 16-byte chunks of a row of O
    constexpr bool kThree = std::is_same<T, BF16>::value && SUBS == 1;
    const float scale_log2 = a.scale * kLog2e;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave;
    const int lr = lane % 16, lq = lane / 16;
    const TreeIndex index = tree_index<SUBS>(wg);
    char* const kslot = k_slot_of(wave);
    char* const vslot = v_slot_of(wave);
    const PagedShares<PagedArgsLate> shares(late_args<ARGS>(), sm.lanes);
    // `p`: the tile; units u0 .. u0 + take of its n
    auto span = [&](const PagedSpan& p, uint32_t u0, uint32_t take) {
        const PagedRequest& rq = p.req;
        const int row0 = (p.tile * SUBS + index.sub) * ROWS;                   // the first flattened row
        const int R = rq.R - row0 < ROWS ? rq.R - row0 : ROWS;
        if (SUBS > 1 && R <= 0) return;
        const PagedArgsLate& z0 = late_args<ARGS>();
        const FastDiv by_g{z0.by_g.m, z0.by_g.s, z0.by_g.d};
        const int base = paged_base(rq, (int)by_g.div((uint32_t)rq.R));
        // (a tile's first units stand for what it costs beside its keys)
        const uint32_t extra = shares.extra, from = u0 > extra ? u0 - extra : 0, to = u0 + take > extra ? u0 + take - extra : 0;
        const int k_begin = (int)((int64_t)from << a.cut.unit_shift);          // below the request's keys: 31 bits
        const int64_t span_end = (int64_t)to << a.cut.unit_shift;
        const int k_end = span_end < rq.keys ? (int)span_end : rq.keys;        // (may lie before k_begin: nothing to see)
        const int shared = base < k_end ? base : k_end;                        // keys before it are seen by all rows
        auto token_of = [&](int r, uint32_t* g) {  // of the tile's row r, and its head of the group; rows that are not there are some real one
            const uint32_t row = (uint32_t)(row0 + (r < R ? r : R - 1)), t = by_g.div(row);
            *g = row - t * by_g.d;
            return t;
        };
        auto query = [&](int r) {
            uint32_t g;
            const uint32_t t = token_of(r, &g);
            return z0.Q + ((int64_t)p.head * z0.G + g) * z0.q_head_stride + ((int64_t)rq.begin + t) * z0.q_token_stride;
        };

        constexpr int CH = D / 8;           // 16-byte chunks per row
        auto swz_k = [&](int r) { return D == 128 ? r % 16 : r / 2 % 8; };
        auto swz_v = [&](int r) { return D == 128 ? r % 4 * 4 + r / 4 % 2 * 2 : r / 2 % 4 * 2; };
        // Where this lane's pieces of a tile lie in LDS, and in its rows.  The others are one exclusive or with a constant away, and made anew
        // in each step (the compiler would keep some thirty registers of them).
        const int op_at = lr * ROWB + ((lq ^ swz_k(lr)) << 4);                    // operand of K or Q, channels 32 i + 8 lq: op_at ^ 64 i
        const int v_at = (lq * 4 + lr / 4) * ROWB + (((lr % 4 / 2) ^ swz_v(lq * 4 + lr / 4)) << 4) + lr % 2 * 8;  // of V, channels 16 t ..: ^ 32 t

        f32x4_t acc[NQ][DCH];
        // the lowest finite value, not -inf: a row may see nothing of a tile, and -inf - m has to be -inf then
        float m_run[NQ], l_run[NQ];
#pragma unroll
        for (int g = 0; g < NQ; ++g) {
            m_run[g] = -__FLT_MAX__;
            l_run[g] = 0.f;
#pragma unroll
            for (int i = 0; i < DCH; ++i) acc[g][i] = zero_vec<f32x4_t>();
        }

        constexpr int RPW = kWave / CH;     // rows per load: 1 KiB
        const int k_from = lane / CH * ROWB + (((lane % CH) ^ swz_k(lane / CH)) << 4), v_from = lane / CH * ROWB + (((lane % CH) ^ swz_v(lane / CH)) << 4);
        constexpr int HL = 16 / RPW;        // loads per half tile
        constexpr int KL = 2 * HL;
        const int n_tiles = (k_end - k_begin + kDecTile - 1) / kDecTile;
        const int n_mine = n_tiles > wave ? (n_tiles - wave + WAVES - 1) / WAVES : 0;
        auto key_of = [&](int i) { return k_begin + (wave + i * WAVES) * kDecTile; };  // the first key of the wave's i-th tile
        // lane l: bytes from K's or V's first page to half tile l of this wave's 32 tiles from the i-th on; < 0: there are no rows, or no
        // page for them
        auto offsets = [&](int i) {
            const int64_t key = (int64_t)k_begin + ((int64_t)wave + (int64_t)(i + lane / 2) * WAVES) * kDecTile + lane % 2 * 16;
            int id = -1;
            const PagedArgsLate& z = late_args<ARGS>();
            const int shift = z.pages.shift;
            if (key < k_end) id = z.table[(int64_t)p.b * z.max_pages + (key >> shift)];
            return (uint32_t)id < z.pages.n_pages
                       ? (int64_t)id * z.pages.page_bytes + (((int64_t)p.head << shift) + ((int)key & ((1 << shift) - 1))) * ROWB : (int64_t)-1;
        };
        int64_t offset = -1;
        vec8 q_regs[NQ][KS];  // Q^T operands: column lr, channels 32 i + 8 lq
        // The wave's i-th tile, i within the 32 whose offsets are here; behind the last tile there is nothing to load, and no loads
        // are left out, so that the counts of those in flight are the same in every step.
        auto fill = [&](int i, char* slot, bool is_k) {
            int from = is_k ? k_from : v_from;
            pin_here(from);
            const int left = k_end - key_of(i);  // rows from its first one on
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int up = __builtin_amdgcn_readlane((int)(offset >> 32), 2 * (i % 32) + h);
                const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)offset, 2 * (i % 32) + h);
                const int there = up < 0 || left < 16 * h ? 0 : left - 16 * h;
                const int bytes = __builtin_amdgcn_readfirstlane((there < 16 ? there : 16) * ROWB);
                // (where nothing is read the address does not count)
                const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                    (void*)((is_k ? a.pages.K : a.pages.V) + (((int64_t)(up & 0x7fffffff) << 32) | low)), 0, bytes, 0x00020000);
#pragma unroll
                for (int j = 0; j < HL; ++j) {
                    const int at = from ^ (j * 1024 + (is_k ? j * 64 : D == 128 ? j % 2 * 32 : 0));
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rs, (void __attribute__((address_space(3)))*)(slot + (h * HL + j) * (kWave * 16)), 16, at, 0, 0, SUBS == 1 ? 2 : 0);
                }
            }
        };
        auto wait_loads = [&](auto n) {  // all loads done but the N asked for last
            constexpr int N = decltype(n)::value;
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
            __builtin_amdgcn_sched_barrier(0);
        };
        // which of a tile's halves have no page, or no rows: two bits
        auto gone_of = [&](int i) {
            return (__builtin_amdgcn_readlane((int)(offset >> 32), 2 * (i % 32)) < 0 ? 1 : 0) |
                   (__builtin_amdgcn_readlane((int)(offset >> 32), 2 * (i % 32) + 1) < 0 ? 2 : 0);
        };
        int gone = 0;

        // One tile; MASKED: some row may not see all of it.
        auto step = [&](int i, auto with_mask) {
            constexpr bool masked = decltype(with_mask)::value;
            const int key0 = key_of(i);
            const int gone_here = gone;
            if ((i + 1) % 32 == 0) offset = offsets(i + 1);
            gone = gone_of(i + 1);
            uint32_t seen[NQ];  // of the tile's keys, by the rows' masks
            if constexpr (masked) {
                const PagedArgsLate& z = late_args<ARGS>();
                const int words = z.tree_words;
#pragma unroll
                for (int g = 0; g < NQ; ++g) {
                    if (words == 1) {
                        const uint64_t mask = sm.mask[16 * g + lr];
                        const int first = key0 - base;  // node of the tile's first key
                        seen[g] = first >= 64 ? 0u : first >= 0 ? (uint32_t)(mask >> first) : first > -32 ? (uint32_t)mask << -first | ~(~0u << -first) : ~0u;
                    } else {
                        const int r = row0 + (16 * g + lr < R ? 16 * g + lr : R - 1);
                        seen[g] = (uint32_t)paged_tree_bits(z, rq, base, (int)FastDiv::div_by(z.by_g.m, z.by_g.s, (uint32_t)r), key0);
                    }
                    const int left = k_end - key0;
                    if (left < 32) seen[g] &= left > 0 ? ~(~0u << left) : 0u;
                    if (gone_here & 1) seen[g] &= 0xffff0000u;
                    if (gone_here & 2) seen[g] &= 0x0000ffffu;
                }
            }
            wait_loads(std::integral_constant<int, KL>{});  // K's of this tile
            f32x4_t s[NQ][2];
            constexpr int NOPS = 2 * KS, KA = 3;  // K operands, and how many are read ahead
            vec8 kop[NOPS];
            int at = op_at;
            pin_here(at);
            auto read_k = [&](int k) { kop[k] = *(const vec8*)(kslot + k % 2 * 16 * ROWB + (at ^ (k / 2 * 64))); };
#pragma unroll
            for (int k = 0; k < KA; ++k) read_k(k);
#pragma unroll
            for (int g = 0; g < NQ; ++g) s[g][0] = s[g][1] = zero_vec<f32x4_t>();
#pragma unroll
            for (int k = 0; k < NOPS; ++k) {
                if (k + KA < NOPS) read_k(k + KA);
#pragma unroll
                for (int g = 0; g < NQ; ++g) s[g][k % 2] = T::mfma16(kop[k], q_regs[g][k / 2], s[g][k % 2]);
                __builtin_amdgcn_sched_barrier(0);
            }
            fill(i + 1, kslot, true);
            __builtin_amdgcn_sched_barrier(0);
            vec8 ph[NQ], pl[NQ], pr[NQ];
#pragma unroll
            for (int g = 0; g < NQ; ++g) {
                if constexpr (masked) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(seen[g] >> (lq * 4) >> ((e / 4) * 16 + e % 4) & 1)) s[g][e / 4][e % 4] = -INFINITY;
                }
                float mx = s[g][0][0];
#pragma unroll
                for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[g][e / 4][e % 4]);
                mx = xor32_max(xor16_max(mx));
                const float top = paged_reference<T>(mx * scale_log2);
                if (__builtin_amdgcn_ballot_w64(top > m_run[g]) != 0) {
                    const float m_new = fmaxf(m_run[g], top);
                    const float alpha = fast_exp2(m_run[g] - m_new);
                    l_run[g] *= alpha;
                    m_run[g] = m_new;
#pragma unroll
                    for (int t = 0; t < DCH; ++t) acc[g][t] *= alpha;
                }
                float x[8];
                if constexpr (masked) {
                    // A key alone has a power of two: the product is rounded as the maximum's was.  (Contracted to one operation, the probability
                    // is 2^(what that rounding took off): in two bf16 terms a lone key's V came back 7e-6 off at scores of 3 * 10^5, in fp16 2.4e-7.)
#pragma clang fp contract(off)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float product = s[g][e / 4][e % 4] * scale_log2;
                        x[e] = product - m_run[g];
                    }
                } else {  // one rounding of the exponent's argument
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(s[g][e / 4][e % 4], scale_log2, -m_run[g]);
                }
                u32x4_t hi, lo, rest;
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float p0 = fast_exp2(x[2 * w]), p1 = fast_exp2(x[2 * w + 1]);
                    sum += p0 + p1;
                    hi[w] = T::pack(p0, p1);
                    const float l0 = p0 - T::low(hi[w]), l1 = p1 - T::high(hi[w]);
                    lo[w] = T::pack(l0, l1);
                    if constexpr (kThree) rest[w] = T::pack(l0 - T::low(lo[w]), l1 - T::high(lo[w]));
                }
                l_run[g] += sum;
                ph[g] = __builtin_bit_cast(vec8, hi);
                pl[g] = __builtin_bit_cast(vec8, lo);
                if constexpr (kThree) pr[g] = __builtin_bit_cast(vec8, rest);
            }
            wait_loads(std::integral_constant<int, KL>{});  // V's
            int vt_at = v_at;
            pin_here(vt_at);
            auto vop_of = [&](int t) {
                u32x4_t vt;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const u32x2_t w = lds_read_tr16(vslot + mt * 16 * ROWB + (vt_at ^ (t * 32)));
                    vt[2 * mt] = w[0];
                    vt[2 * mt + 1] = w[1];
                }
                return vt;
            };
            // Some rows see a token that others do not.  Where its V is not finite, a product with the probability 0 would bring it to
            // them: such values are taken out, and added by themselves for the rows that see them.
            constexpr uint32_t kExp = std::is_same<T, BF16>::value ? 0x7f80u : 0x7c00u;
            bool odd = false;
            if constexpr (masked) {
                bool bad = false;
                if (key0 + kDecTile > shared) {
#pragma unroll 4
                    for (int t = 0; t < DCH; ++t) {
                        const u32x4_t vt = vop_of(t);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const bool lo = (vt[w] & kExp) == kExp, up = (vt[w] >> 16 & kExp) == kExp;
                            bad |= lo || up;
                        }
                    }
                }
                odd = __builtin_amdgcn_ballot_w64(bad) != 0;
                if (odd) {
#pragma unroll 1
                    for (int key = 0; key < kDecTile && key0 + key < k_end; ++key)
#pragma unroll
                        for (int t = 0; t < DCH; ++t) {
                            // acc[g][t] holds channels 16 t + 4 lq + 0..3: half of a 16-byte chunk
                            const u32x2_t w = *(const u32x2_t*)(vslot + key * ROWB + (((2 * t + lq / 2) ^ swz_v(key)) << 4) + lq % 2 * 8);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t v = (e < 2 ? w[0] : w[1]) >> (e % 2 * 16) & 0xffffu;
                                if ((v & kExp) == kExp)
#pragma unroll
                                    for (int g = 0; g < NQ; ++g)
                                        if (seen[g] >> key & 1) acc[g][t][e] += T::to_float(__builtin_bit_cast(elem, (uint16_t)v));
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                }
            }
            constexpr int VA = 2;  // V operands read ahead
            u32x4_t vts[DCH];
#pragma unroll
            for (int t = 0; t < VA; ++t) vts[t] = vop_of(t);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < DCH; ++t) {
                if (t + VA < DCH) vts[t + VA] = vop_of(t + VA);
                u32x4_t vt = vts[t];
                if (odd) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        if ((vt[w] & kExp) == kExp) vt[w] &= 0xffff0000u;
                        if ((vt[w] >> 16 & kExp) == kExp) vt[w] &= 0xffffu;
                    }
                }
                const vec8 vop = __builtin_bit_cast(vec8, vt);
#pragma unroll
                for (int g = 0; g < NQ; ++g) acc[g][t] = T::mfma16(vop, ph[g], acc[g][t]);
#pragma unroll
                for (int g = 0; g < NQ; ++g) acc[g][t] = T::mfma16(vop, pl[g], acc[g][t]);
                if constexpr (kThree)
#pragma unroll
                    for (int g = 0; g < NQ; ++g) acc[g][t] = T::mfma16(vop, pr[g], acc[g][t]);
                __builtin_amdgcn_sched_barrier(0);
            }
            fill(i + 1, vslot, false);
            __builtin_amdgcn_sched_barrier(0);
        };
        // The table's trip, and beside it the queries'; then the first tile's.
        uint64_t mask_word = 0;
#pragma unroll
        for (int g = 0; g < NQ; ++g) {
            const char* Qr = query(16 * g + lr);
#pragma unroll
            for (int i = 0; i < KS; ++i) q_regs[g][i] = *(const vec8*)(Qr + (i * 32 + lq * 8) * 2);
        }
        if (tid < ROWS) {
            uint32_t g;
            mask_word = z0.tree[((int64_t)rq.begin + token_of(tid, &g)) * z0.tree_words];
        }
        if (n_mine > 0) {
            offset = offsets(0);
            gone = gone_of(0);
            fill(0, kslot, true);
            fill(0, vslot, false);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < NQ; ++g)
#pragma unroll
            for (int i = 0; i < KS; ++i) {  // waited for here: ahead of a loop the compiler waits for all in flight
                u32x4_t w = __builtin_bit_cast(u32x4_t, q_regs[g][i]);
                pin_here(w);
                q_regs[g][i] = __builtin_bit_cast(vec8, w);
            }
        if (tid < ROWS) sm.mask[tid] = mask_word;
        __syncthreads();
        if (n_mine > 0) {
            // up to the first tile that is masked, and from there on
            int i = 0;
#pragma unroll 1
            for (; i < n_mine && key_of(i) + kDecTile <= shared && gone == 0; ++i) step(i, std::false_type{});
#pragma unroll 1
            for (; i < n_mine; ++i) step(i, std::true_type{});
            wait_loads(std::integral_constant<int, 0>{});  // (those of nothing write zeros)
        }

        // fold the waves (Section 4.1 aggregation, in base 2); a thread finishes 4 columns of a row
#pragma unroll
        for (int g = 0; g < NQ; ++g) {
            const float l_tot = xor32_sum(xor16_sum(l_run[g]));
            if (lq == 0) {
                sm.m[wave][16 * g + lr] = m_run[g];
                sm.l[wave][16 * g + lr] = l_tot;
            }
        }
        static_assert(NQ <= 2 && 16 * D * 4 <= SLOT, "16 rows of O fit a slot, those of a wave K's and V's");
#pragma unroll
        for (int g = 0; g < NQ; ++g)
            if (16 * g + lr < R) {
#pragma unroll
                for (int t = 0; t < DCH; ++t) *(f32x4_t*)((g ? vslot : kslot) + lr * (D * 4) + (((4 * t + lq) ^ lr) << 4)) = acc[g][t];
            }
        __syncthreads();
        const PagedArgsLate& z = late_args<ARGS>();
        const bool part = take < p.n;
        const int64_t slot = 2 * (int64_t)index.share + (u0 == 0 ? 1 : 0);
        for (int idx = tid; idx < R * PCH; idx += WAVES * kWave) {
            const int n = idx / PCH, c = idx % PCH * 4;
            float M = sm.m[0][n];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm.m[w][n]);
            f32x4_t num = zero_vec<f32x4_t>();
            float den = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = fast_exp2(sm.m[w][n] - M);
                const f32x4_t o = *(const f32x4_t*)((n < 16 ? k_slot_of(w) : v_slot_of(w)) + n % 16 * (D * 4) + (((c / 4) ^ (n % 16)) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) num[e] = __builtin_fmaf(f, o[e], num[e]);
                den = __builtin_fmaf(f, sm.l[w][n], den);
            }
            const bool any = den != 0.f;  // (not a number where a score was not)
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] = any ? num[e] / den : 0.f;
            const float lse = any ? paged_log2_sum<T>(M, den) * kLn2 : -INFINITY;
            const uint32_t t = FastDiv::div_by(z.by_g.m, z.by_g.s, (uint32_t)(row0 + n)), g = (uint32_t)(row0 + n) - t * z.by_g.d;
            if (!all_finite(num) && __builtin_isfinite(den))
                num = paged_with_odd(num, paged_odd_tree_values<elem, D>(z, rq, base, (int)t, p.b, p.head, k_begin, k_end, c));
            const int64_t at = part ? (slot << z.cut.tile_shift) + index.sub * ROWS + n : ((int64_t)p.head * z.G + g) * z.T + rq.begin + t;
            *(f32x4_t*)((part ? z.part_O : z.O) + at * D + c) = num;
            if (c == 0) (part ? z.part_lse : z.lse)[at] = lse;
        }
    };
    uint32_t pos = index.share * shares.share;
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
