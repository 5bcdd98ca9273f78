// Attention over a paged cache for requests of many rows (a chunk of a prompt), 16-bit storage.  Bound by the matrix pipe, which
// the two-term probabilities give half as much again to do, and by the vector work that does not hide behind it: 1024 rows of 32 heads
// of 128 over 16384 keys take 356 to 381 us with the fold, by the card, 0.70 to 0.75 PFLOP/s of the visible pairs and half as much again
// issued (a library product of bf16 reaches 1.39); 268 us with the matrix instructions alone, 199 with the vector ones.  In fp16, whose
// terms have more bits set, 387.
//
// One workgroup = 4 waves x 32 flattened rows (token r / G, head r % G: all heads of a KV head's group share its keys, and a
// tile spans few tokens, so that little of it lies above the diagonal) of one request and KV head x one run of keys.
//   * K, V tiles of 64 keys are shared by the waves through LDS, two slots each, filled by LDS-direct loads one iteration ahead.
//     A load covers rows of one page (it is 4 or 8 of them): its buffer descriptor begins at those rows and ends with what the
//     tile sees of the request, or is empty where the table names no page, and what it does not cover arrives as zeros.  Page ids
//     come 64 loads at a time, one a lane, asked for that long ahead.
//   * S^T = K Q^T and O^T += V^T P^T (32x32x16 MFMA): the scores already sit in the lanes in which the second product wants the
//     probabilities.  V^T operands come through the transposing LDS read.  Slots are swizzled against bank conflicts.
//   * A wave works on two tiles at a time, so that vector work has matrix instructions to hide behind: iteration t issues
//       A(t):   S^T(t) = K(t) Q^T       with B2(t-1): probabilities of keys 32..63 of tile t-1, whose maximum is known;
//       C(t-1): O^T += V(t-1)^T P^T     with B1(t):   maximum, rescale factor and probabilities of keys 0..31 of tile t.
//     The further a wave is in its iteration, the higher its priority over the one that it shares its SIMD with, which belongs to
//     another workgroup: the two stay apart by half an iteration, and a barrier's last waves are not kept (without it 1024 rows over
//     16384 keys take 3.0 % longer and 4096 over 4096 5.5 %; one step in place of three 1.1 and 1.0, the other way round 2.5 and 4.5).
//   * Tiles are visited from the last to the first: those that some row does not see whole (the diagonal, the end of the request)
//     come first and are finished one by one, up to the last of them, with which the pipeline starts.
#pragma once
#include "attn_paged.h"

namespace fedrag {

// ks0 .. vs1: an array each per tile slot, so that the compiler sees that the loads filling one do not alias the reads of another.
// AHEAD: V operands are read from LDS so many before they are used; K operands four.  (Three of V take the registers that are left
// at 128 columns; the other form beside it takes two more for its scalars.)
template <class T, int D, int NW, int ARGS, int AHEAD>
__device__ __forceinline__ void paged_chunk_body(const PagedArgs& a, uint32_t index, char* ks0, char* ks1, char* vs0, char* vs1, int* flags) {
    typedef typename T::elem elem;
    typedef typename T::vec8 vec8;
    constexpr int kThreads = NW * kWave;
    constexpr int ROWB = D * 2;
    constexpr int SLOT = kPreK * ROWB;
    constexpr int KS = D / 16;              // contraction steps of S^T
    constexpr int MT = D / 32;              // 32-row tiles of O^T
    constexpr int CH = D / 8;               // 16-byte chunks per row
    constexpr int RPW = kWave / CH;         // rows per load of a wave
    constexpr int LPT = kPreK / (NW * RPW); // loads per wave and tile
    constexpr int IDT = kWave / LPT;        // tiles whose page ids a wave holds
    const float scale_log2 = a.scale * kLog2e;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lane = tid % kWave;
    const int li = lane % 32, lh = lane / 32;
    const PagedPiece p = paged_piece<false>(a, index);
    if (p.b < 0) return;
    const PagedRequest& rq = p.req;
    const int row0 = p.tile * (NW * kPreQ);
    const int last = (row0 + NW * kPreQ < rq.R ? row0 + NW * kPreQ : rq.R) - 1;
    const int lim_min = paged_limit(a, rq, row0), lim_max = paged_limit(a, rq, last);
    const int k_begin = (int)((int64_t)p.run * p.per << a.cut.unit_shift);
    const int64_t run_end = (int64_t)k_begin + ((int64_t)p.per << a.cut.unit_shift);
    const int L = (run_end < lim_max ? (int)run_end : lim_max) - k_begin;  // keys to visit
    if (p.run > 0 && L <= 0) return;  // a run behind what the tile sees: its partial is not asked for

    const int row_w = row0 + wave * kPreQ;            // this wave's first row
    const int row = row_w + li < rq.R ? row_w + li : rq.R - 1;
    const uint32_t tok = a.by_g.div((uint32_t)row), hg = (uint32_t)row - tok * a.by_g.d;
    if (L <= 0) {  // no keys (workgroup-uniform, before any barrier); other tiles of the request may see several runs
        if (row_w + li < rq.R) {
            const int64_t at = p.runs > 1 ? ((int64_t)p.slot << a.cut.tile_shift) + row - row0 : ((int64_t)p.head * a.G + hg) * a.T + rq.begin + tok;
            float* const O = p.runs > 1 ? a.part_O : a.O;
            for (int c = lh * (D / 2); c < (lh + 1) * (D / 2); c += 4) *(f32x4_t*)(O + at * D + c) = zero_vec<f32x4_t>();
            if (lh == 0) (p.runs > 1 ? a.part_lse : a.lse)[at] = -INFINITY;
        }
        return;
    }
    const int n_tiles = (L + kPreK - 1) / kPreK;
    const int whole = lim_min - k_begin < L ? lim_min - k_begin : L;  // keys that every row sees
    int t_mask0 = whole > 0 ? whole / kPreK : 0;                      // first tile that some row does not see whole
    const int own = paged_limit(a, rq, row) - k_begin;
    const int key_lim = own < L ? own : L;                            // this lane's row sees keys < key_lim

    vec8 qop[KS];  // Q^T operands: column li, channels 16 i + 8 lh
    const char* Qr = a.Q + ((int64_t)p.head * a.G + hg) * a.q_head_stride + ((int64_t)rq.begin + tok) * a.q_token_stride;
#pragma unroll
    for (int i = 0; i < KS; ++i) qop[i] = *(const vec8*)(Qr + (i * 16 + lh * 8) * 2);

    // ---- where this wave's loads begin, lane l: load l % LPT of the tile l / LPT below `top`
    const int64_t table0 = (int64_t)p.b * a.max_pages;
    const int shift = a.pages.shift;
    auto key_of = [&](int top) { return (top - lane / LPT) * kPreK + (lane % LPT * NW + wave) * RPW; };
    auto ask_ids = [&](int top) {
        const int key = key_of(top);
        int id = -1;
        if (key >= 0 && key < L) id = a.table[table0 + ((k_begin + key) >> shift)];
        return id;
    };
    auto valid = [&](int id) { return (uint32_t)id < a.pages.n_pages ? id : -1; };
    // bytes from K's or V's first page to the load's rows; < 0: there are none, or no page
    auto offset_of = [&](int id, int top) {
        return valid(id) < 0 ? (int64_t)-1 : (int64_t)id * a.pages.page_bytes + (((int64_t)p.head << shift) + ((k_begin + key_of(top)) & ((1 << shift) - 1))) * ROWB;
    };
    // whether the table names a page for all keys of the run; if not, every tile is masked, key by key
    bool hole = false;
    for (int64_t key = (int64_t)tid << shift; key < L + ((int64_t)1 << shift); key += (int64_t)kThreads << shift) {
        const int64_t at = (k_begin >> shift) + (key >> shift);  // (a run may begin inside a page)
        if ((at << shift) < (int64_t)k_begin + L && valid(a.table[table0 + at]) < 0) hole = true;
    }
    int top = n_tiles - 1;  // `offset` is of this tile and the IDT - 1 below
    const int ids = ask_ids(top);
    int ids_next = ask_ids(top - IDT);
    int64_t offset = offset_of(ids, top);

    f32x16_t acc_o[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc_o[i] = zero_vec<f32x16_t>();
    // the lowest finite value, not -inf: a row may see nothing of a tile, and -inf - m has to be -inf then
    float m_run = -__FLT_MAX__, l_run = 0.f;

    // ---- pages -> LDS.  LDS slot p of row r holds chunk p ^ swz(r): K swz(r) = r % CH, V (4 (r % 4)) % CH.
    const int ld_r = lane / CH, ld_p = lane % CH;
    const int tile_r = wave * RPW + ld_r;  // row in the tile, but for multiples of NW * RPW
    static_assert((NW * RPW) % 16 == 0, "swizzle must not depend on the load index");
    const int ld_k = ld_r * ROWB + ((ld_p ^ (tile_r % CH)) << 4);
    const int ld_v = ld_r * ROWB + ((ld_p ^ ((4 * (tile_r % 4)) % CH)) << 4);
    int full_tiles = 0;  // tiles whose rows are all there, once it is known that no pages are missing (before, the first tile is asked for)
    auto load_rows = [&](const char* base, char* slot, int tile, int voff) {
        auto begin = [&](int j) {
            const int at = (top - tile) * LPT + j;
            return ((int64_t)__builtin_amdgcn_readlane((int)(offset >> 32), at) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)offset, at);
        };
        auto to = [&](int j) { return slot + (j * NW + wave) * (RPW * ROWB); };
        if ((unsigned)tile < (unsigned)full_tiles) {
            // all rows are there: no descriptors, whose scalar instructions a wave issues one at a time like any others
#pragma unroll
            for (int j = 0; j < LPT; ++j)
                copy_to_lds(base + begin(j) + (uint32_t)voff, to(j));
        } else if (tile >= 0) {
#pragma unroll
            for (int j = 0; j < LPT; ++j) {
                const int left = L - (tile * kPreK + (j * NW + wave) * RPW);
                const int64_t off = begin(j);
                const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                    (void*)(base + (off < 0 ? 0 : off)), 0, left <= 0 || off < 0 ? 0 : (left < RPW ? left : RPW) * ROWB, 0x00020000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (void __attribute__((address_space(3)))*)to(j), 16, voff, 0, 0, 0);
            }
        }
    };
    auto load_k = [&](int tile, char* slot) {  // tile by tile downwards; a tile's V is asked for before the next one's K
        if (top - tile == IDT) {
            top -= IDT;
            offset = offset_of(ids_next, top);
            ids_next = ask_ids(top - IDT);
        }
        load_rows(a.pages.K, slot, tile, ld_k);
    };
    auto load_v = [&](int tile, char* slot) { load_rows(a.pages.V, slot, tile, ld_v); };

    // ---- per-lane LDS read offsets (as the operands of the two products want them)
    const int k_base = li * ROWB + ((lh ^ (li % CH)) << 4);  // channels 16 i + 8 lh of row li: k_base ^ 32 i
    const int s16 = lane % 16, gq = lane / 16;
    int v_off[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int chunk = 4 * i + 2 * (gq % 2) + (s16 % 4) / 2;
        v_off[i] = (4 * lh + s16 / 4) * ROWB + (((chunk % CH) ^ ((4 * ((s16 / 4) % 4)) % CH)) << 4) + 8 * ((s16 % 4) % 2);
    }

    int tile = n_tiles - 1;
    load_k(tile, ks0);
    load_v(tile, vs0);
    // flags: a wave's `hole` each, and whether `mend` has found something
    const bool wave_hole = __builtin_amdgcn_ballot_w64(hole) != 0;
    if (lane == 0) flags[wave] = wave_hole;
    if (tid == 0) flags[NW] = 0;
    f32x16_t S0;                // S^T of the current tile, keys 0..31
    f32x16_t S1[2];             // S1[t & 1]: keys 32..63 of tile t, kept one iteration longer; then their probabilities
    uint32_t P[2][4][4];        // [t & 1]: P^T operands of tile t, one per 16 keys, in words of two,
    uint32_t Plo[2][4][4];      //          and what their narrowing left
    float alph[2];              // [t & 1]: rescale factor of the output that goes with P(t)
    auto operand = [&](const uint32_t (&w)[4]) -> vec8 {
        u32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[e];
        return __builtin_bit_cast(vec8, v);
    };
    // register r (even) of a half's scores and the next one <-> word r % 8 / 2 of the operand of 16 keys r / 8 (+ 2 for the second half)
    auto put_hi = [&](int par, int kk, int w, float x, float y) {
        P[par][kk][w] = T::pack(x, y);
        pin_here(P[par][kk][w]);  // in its slice, not behind the phase
    };
    auto put_lo = [&](int par, int kk, int w, float x, float y) {
        Plo[par][kk][w] = T::pack(x - T::low(P[par][kk][w]), y - T::high(P[par][kk][w]));
        pin_here(Plo[par][kk][w]);
    };
    auto put = [&](int par, int kk, int w, float x, float y) {
        put_hi(par, kk, w, x, y);
        put_lo(par, kk, w, x, y);
    };
    auto read_vop = [&](const char* vt, int kk, int i) -> vec8 {
        const char* at = vt + kk * 16 * ROWB + v_off[i];
        const u32x2_t lo = lds_read_tr16(at), hi = lds_read_tr16(at + 8 * ROWB);
        u32x4_t w;
        w[0] = lo[0]; w[1] = lo[1]; w[2] = hi[0]; w[3] = hi[1];
        return __builtin_bit_cast(vec8, w);
    };

    // par: t & 1 as a constant, so that the double sets are addressed statically.  kFirst: A and B1 of a tile (masked if need be);
    // kLast: B2 and C of the one before; kSteady: all, on tiles that every row sees whole.
    enum { kFirst, kSteady, kLast };
    auto iteration = [&](int tile, int next, auto par, auto stage, bool ld_next, bool ld_v = true) {
        constexpr int c = decltype(par)::value;
        constexpr int o = 1 - c;
        constexpr int kind = decltype(stage)::value;
        constexpr bool doC = kind != kFirst;
        constexpr bool doAB = kind != kLast;
        constexpr int NM = 4 * MT;
        if (doAB && ld_v) load_v(tile, c ? vs1 : vs0);     // slot last read by C(t-2)
        if (ld_next) load_k(next, o ? ks1 : ks0);          // slot last read by A(t-1)

        // lane: row li and, per 32-key half, keys 8 (r / 4) + 4 lh + r % 4, r = 0..15
        const char* kt = c ? ks1 : ks0;
        if constexpr (doAB) {
            constexpr int NA = 2 * KS;
            vec8 kop[NA];
            int k_off[KS];  // (made anew for each tile: eight instructions, and not eight registers in the other phase)
            int kb = k_base;
            pin_here(kb);
#pragma unroll
            for (int i = 0; i < KS; ++i) k_off[i] = kb ^ (32 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) kop[j] = *(const vec8*)(kt + (j % 2) * 32 * ROWB + k_off[j / 2]);
            S0 = zero_vec<f32x16_t>();
            S1[c] = zero_vec<f32x16_t>();
            float psum = 0.f;
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int j = 0; j < NA; ++j) {
                if (j + 4 < NA)
                    kop[j + 4] = *(const vec8*)(kt + ((j + 4) % 2) * 32 * ROWB + k_off[(j + 4) / 2]);
                if (j == NA / 2) __builtin_amdgcn_s_setprio(1);
                if (j % 2 == 0) S0 = T::mfma32(kop[j], qop[j / 2], S0);
                else S1[c] = T::mfma32(kop[j], qop[j / 2], S1[c]);
                if constexpr (doC) {
#pragma unroll
                    for (int r = (j * 16) / NA; r < ((j + 1) * 16) / NA; ++r) {
                        const float pe = fast_exp2(__builtin_fmaf(S1[o][r], scale_log2, -m_run));
                        psum += pe;
                        S1[o][r] = pe;
                        if (r % 2) put(o, 2 + r / 8, r % 8 / 2, S1[o][r - 1], pe);
                    }
                    pin_here(psum);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            l_run += psum;
            if (kind == kFirst && tile >= t_mask0) {
                const int key0 = tile * kPreK + 4 * lh;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = key0 + 8 * (r / 4) + (r % 4);
                    if (key >= key_lim) S0[r] = -INFINITY;
                    if (key + 32 >= key_lim) S1[c][r] = -INFINITY;
                }
                if (t_mask0 < 0) {  // pages are missing: 16 keys lie in one
                    bool gone[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = tile * kPreK + 16 * i;
                        gone[i] = key < L && valid(a.table[table0 + ((k_begin + key) >> shift)]) < 0;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (gone[r / 8]) S0[r] = -INFINITY;
                        if (gone[2 + r / 8]) S1[c][r] = -INFINITY;
                    }
                }
            }
        } else {
            float psum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float pe = fast_exp2(__builtin_fmaf(S1[o][r], scale_log2, -m_run));
                psum += pe;
                S1[o][r] = pe;
                if (r % 2) put(o, 2 + r / 8, r % 8 / 2, S1[o][r - 1], pe);
            }
            l_run += psum;
        }
        __builtin_amdgcn_sched_barrier(0);
        const char* vt = o ? vs1 : vs0;
        if constexpr (doC) {
            if (__builtin_amdgcn_ballot_w64(alph[o] != 1.0f) != 0) {
#pragma unroll
                for (int i = 0; i < MT; ++i) acc_o[i] *= alph[o];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        {
            // One matrix instruction a slice, with its share of the vector work, some six instructions a step: four steps of the row
            // maximum, one of the new maximum and the factor, and three for each pair of probabilities of keys 0..31.  An output tile's two instructions are two apart: the second waits for the first, and a
            // wave that waits issues no vector work either.
            constexpr int NJ = 2 * NM;
            constexpr int kSteps = 4 + 1 + 24;
            vec8 vop[NM];
            if constexpr (doC) {
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) vop[j] = read_vop(vt, j / MT, j % MT);
            }
            __builtin_amdgcn_s_setprio(2);
            float mx = -INFINITY;
            float m_new = 0.f, psum = 0.f;
            auto step = [&](int s) {
                if (s < 4) {
                    if constexpr (doAB) {
#pragma unroll
                        for (int r = 4 * s; r < 4 * s + 4; ++r) mx = fmaxf(fmaxf(mx, S0[r]), S1[c][r]);
                        pin_here(mx);
                    }
                } else if (s == 4) {
                    if constexpr (doAB) {
                        mx = xor32_max(mx);
                        m_new = fmaxf(m_run, paged_reference<T>(mx * scale_log2));
                        alph[c] = fast_exp2(m_run - m_new);
                    }
                } else {
                    if constexpr (doAB) {
                        const int r = (s - 5) / 3 * 2, part = (s - 5) % 3;
                        if (part < 2) {
                            S0[r + part] = fast_exp2(__builtin_fmaf(S0[r + part], scale_log2, -m_new));
                            psum += S0[r + part];
                            pin_here(psum);
                            if (part == 1) put_hi(c, r / 8, r % 8 / 2, S0[r], S0[r + 1]);
                        } else {
                            put_lo(c, r / 8, r % 8 / 2, S0[r], S0[r + 1]);
                        }
                    }
                }
            };
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if constexpr (doC) {
                    // of each four: tiles i, i + 1 with the first terms, then with the second
                    const int at = j / 4 * 2 + j % 2, kk = at / MT, i = at % MT;
                    if (j % 4 < 2 && at + AHEAD < NM) vop[at + AHEAD] = read_vop(vt, (at + AHEAD) / MT, (at + AHEAD) % MT);
                    acc_o[i] = T::mfma32(vop[at], operand(j % 4 < 2 ? P[o][kk] : Plo[o][kk]), acc_o[i]);
                }
#pragma unroll
                for (int s = j * kSteps / NJ; s < (j + 1) * kSteps / NJ; ++s) step(s);
                if constexpr (doC) __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (doAB) {
                l_run = l_run * alph[c] + psum;
                m_run = m_new;
            }
        }
        if constexpr (doAB) pin_here(l_run);  // above the barrier that follows
        __builtin_amdgcn_sched_barrier(0);
    };
    std::integral_constant<int, 0> even;
    std::integral_constant<int, 1> odd;
    std::integral_constant<int, kFirst> first;
    std::integral_constant<int, kSteady> steady;
    std::integral_constant<int, kLast> last_stage;
    auto tile_barrier = [&]() {  // a wave's own LDS-direct loads, then everyone's
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
    };

    // Some rows see a token of this tile that others do not (its scores are computed, its V lies in vs0, nothing has used it yet).
    // Where its V is not finite, a product with the probability 0 would bring it to them: such values are taken out of the tile,
    // and added by themselves for the rows that see them.
    constexpr uint32_t kExp = std::is_same<T, BF16>::value ? 0x7f80u : 0x7c00u;
    auto mend = [&](int tile) {
        int tid = threadIdx.x;  // anew: what is rarely used is not kept in registers through the loops
        pin_here(tid);
        const int lane = tid % kWave, lh = lane / 32;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < SLOT / 16 / kThreads; ++j) {
            const u32x4_t v = *(const u32x4_t*)(vs0 + (j * kThreads + tid) * 16);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const bool lo = (v[w] & kExp) == kExp, up = (v[w] >> 16 & kExp) == kExp;
                bad |= lo || up;
            }
        }
        if (__builtin_amdgcn_ballot_w64(bad) != 0 && lane == 0) flags[NW] = 1;
        __syncthreads();
        if (flags[NW] == 0) return;  // workgroup-uniform
#pragma unroll
        for (int i = 0; i < MT; ++i) acc_o[i] *= alph[0];
        alph[0] = 1.0f;
        for (int k = 0; k < kPreK && tile * kPreK + k < key_lim; ++k)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {  // channels 32 i + 8 r4 + 4 lh + 0..3: half of a 16-byte chunk
                    const u32x2_t v = *(const u32x2_t*)(vs0 + k * ROWB + (((4 * i + r4) ^ ((4 * (k % 4)) % CH)) << 4) + lh * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t x = (e < 2 ? v[0] : v[1]) >> (e % 2 * 16) & 0xffffu;
                        if ((x & kExp) == kExp) acc_o[i][4 * r4 + e] += T::to_float(__builtin_bit_cast(elem, (uint16_t)x));
                    }
                    __builtin_amdgcn_sched_barrier(0);  // (more of these reads in flight would take registers from the loops)
                }
        __syncthreads();
#pragma unroll 1
        for (int j = 0; j < SLOT / 16 / kThreads; ++j) {
            u32x4_t* at = (u32x4_t*)(vs0 + (j * kThreads + tid) * 16);
            u32x4_t v = *at;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t x = v[w];
                if ((x & kExp) == kExp) x &= 0xffff0000u;
                if ((x >> 16 & kExp) == kExp) x &= 0xffffu;
                v[w] = x;
            }
            *at = v;
        }
        if (tid == 0) flags[NW] = 0;
        __syncthreads();
    };
    const bool differ = lim_min != lim_max;

    alph[0] = alph[1] = 1.0f;
    tile_barrier();
    int holes = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) holes |= flags[w];
    if (__builtin_amdgcn_readfirstlane(holes) != 0) t_mask0 = -1;
    else full_tiles = L / kPreK;
    while (tile >= 0 && (tile > t_mask0 || (tile & 1))) {
        iteration(tile, 0, even, first, false, tile != n_tiles - 1);
        tile_barrier();
        if (differ && tile >= t_mask0) mend(tile);
        --tile;
        load_k(tile, ks0);
        iteration(0, 0, odd, last_stage, false);
        tile_barrier();
    }
    if (tile >= 0) {
        iteration(tile, tile - 1, even, first, true, tile != n_tiles - 1);
        tile_barrier();
        if (differ && tile >= t_mask0) mend(tile);
        for (; tile > 0; tile -= 2) {
            iteration(tile - 1, tile - 2, odd, steady, true);
            tile_barrier();
            iteration(tile - 2, tile - 3, even, steady, true);
            tile_barrier();
        }
        iteration(0, 0, odd, last_stage, false);
    }

    // The rows go out through LDS (the tiles are dead; every wave has its share), so that a store covers whole lines.
    const float l_tot = xor32_sum(l_run);
    __syncthreads();
    constexpr int WB = 4 * SLOT / NW;
    static_assert(WB == kPreQ * D * 4, "a wave's rows fit its share");
    constexpr int PCH = D / 4;  // 16-byte chunks per row
    int l = threadIdx.x % kWave;  // anew, as above
    pin_here(l);
    auto finish = [&](const int lane) {
        const int li = lane % 32, lh = lane / 32;
        const int slot_w = wave * 4 / NW;
        char* mine = (slot_w == 0 ? ks0 : slot_w == 1 ? ks1 : slot_w == 2 ? vs0 : vs1) + (wave % (NW / 4)) * WB;
        const PagedArgsLate& z = late_args<ARGS>();
        const int r_in = row_w - row0 + li;  // this lane's row in the tile
        const bool real = row_w + li < rq.R;
        // its partial's place, or its own in O and lse: row t / G of head t % G
        const uint32_t t = FastDiv::div_by(z.by_g.m, z.by_g.s, (uint32_t)(row_w + li)), g = (uint32_t)(row_w + li) - t * z.by_g.d;
        const int64_t at = p.runs > 1 ? ((int64_t)p.slot << z.cut.tile_shift) + r_in : ((int64_t)p.head * z.G + g) * z.T + rq.begin + t;
        float* const O = p.runs > 1 ? z.part_O : z.O;
        const float inv = l_tot != 0.f ? 1.0f / l_tot : 0.f;  // (not a number where a score was not)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                f32x4_t o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = l_tot != 0.f ? acc_o[i][4 * r4 + r] * inv : 0.f;
                *(f32x4_t*)(mine + li * (D * 4) + (((8 * i + 2 * r4 + lh) ^ (li % PCH)) << 4)) = o;
            }
        if (lh == 0 && real) (p.runs > 1 ? z.part_lse : z.lse)[at] = l_tot != 0.f ? paged_log2_sum<T>(m_run, l_tot) * kLn2 : -INFINITY;
        wave_lds_fence();
        // a store covers whole rows; where a row goes is with the lane of its number
        bool odd = false;
#pragma unroll
        for (int u = 0; u < kPreQ * PCH / kWave; ++u) {
            const int r = (u * kWave + lane) / PCH, chunk = lane % PCH;
            const f32x4_t o = *(const f32x4_t*)(mine + r * (D * 4) + ((chunk ^ (r % PCH)) << 4));
            const int64_t to = ((int64_t)__shfl((int)(at >> 32), r) << 32) | (uint32_t)__shfl((int)at, r);
            if (row_w + r < rq.R) *(f32x4_t*)(O + to * D + chunk * 4) = o;
            odd |= !all_finite(o);
        }
        if (__builtin_amdgcn_ballot_w64(odd) == 0) return;
        // What all rows see of this lane's channels once, and for each row what it sees beyond.
        const int chunk = lane % PCH, shared = lim_min < k_begin + L ? lim_min : k_begin + L;
        const f32x4_t all = paged_odd_values<elem, D>(z, p.b, p.head, k_begin, shared, chunk * 4);
#pragma unroll 1
        for (int u = 0; u < kPreQ * PCH / kWave; ++u) {
            const int r = (u * kWave + lane) / PCH;
            const f32x4_t o = *(const f32x4_t*)(mine + r * (D * 4) + ((chunk ^ (r % PCH)) << 4));
            const int64_t to = ((int64_t)__shfl((int)(at >> 32), r) << 32) | (uint32_t)__shfl((int)at, r);
            const float sum = __shfl(l_tot, r);
            if (row_w + r >= rq.R || all_finite(o) || !__builtin_isfinite(sum)) continue;
            const int own = paged_limit(z, rq, row_w + r), end = own < k_begin + L ? own : k_begin + L;
            const f32x4_t more = paged_odd_values<elem, D>(z, p.b, p.head, shared > k_begin ? shared : k_begin, end, chunk * 4);
            *(f32x4_t*)(O + to * D + chunk * 4) = paged_with_odd(o, all + more);
        }
    };
    finish(l);
}

}  // namespace fedrag
