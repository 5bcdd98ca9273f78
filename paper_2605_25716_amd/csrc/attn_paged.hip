// Attention of a ragged step over a paged cache (fedrag_paged_attn).
#include "attn_paged.h"

namespace fedrag {

// The aggregation (Section 4.1) of the tiles whose keys are in several partials: a workgroup takes `rows` rows of one of them, part
// `part`, a thread 4 columns of a row at a time.  Beyond four partials the lanes of a row share out the weights, 16 at a time.
// Which tile: SHARES: the one that workgroup index + 1's share begins inside of, if no share before does; else the index-th of
// those in several runs.
constexpr int kPagedMergeThreads = 256;
template <int D, bool SHARES>
__device__ __forceinline__ void paged_merge(const PagedArgs& a, uint32_t index, int part, int rows) {
    constexpr int TPR = D / 4;
    PagedRequest req;
    int tile, head, S = 0;
    int64_t slot, step, first = 0;  // partial i lies in slot + i * step, partial 0 in `first` if SHARES
    if constexpr (SHARES) {
        __shared__ PagedLanes lanes;
        const PagedShares<const PagedArgs> shares(a, lanes);
        const uint32_t w = index + 1, pos = w * shares.share;
        const PagedSpan p = shares.find(a, pos);
        if (p.b < 0 || pos == p.begin || p.n <= shares.whole) return;
        const uint32_t w0 = p.begin / shares.share;
        if (w0 + 1 != w) return;
        req = p.req;
        tile = p.tile;
        head = p.head;
        S = (int)((p.begin + p.n - 1) / shares.share - w0) + 1;
        if (2 * (w0 + (uint32_t)S) > a.slots) return;  // (where q_start decreases)
        slot = 2 * (int64_t)w0;
        step = 2;
        first = slot + 1;
    } else {
        const PagedPiece p = paged_piece<true>(a, index);
        if (p.b < 0 || p.slot + (uint32_t)(p.runs - 1) * (uint32_t)a.Hkv >= a.slots) return;  // (the latter where q_start decreases)
        req = p.req;
        tile = p.tile;
        head = p.head;
        slot = first = p.slot;
        step = a.Hkv;
        S = p.per;  // units of a run, for now
    }
    const int row0 = tile << a.cut.tile_shift, last = (row0 + (1 << a.cut.tile_shift) < req.R ? row0 + (1 << a.cut.tile_shift) : req.R) - 1;
    if constexpr (!SHARES) {  // runs that hold keys which some row of the tile sees
        const int64_t run_keys = (int64_t)S << a.cut.unit_shift, seen = paged_limit(a, req, last);
        S = seen > 0 ? (int)((seen + run_keys - 1) / run_keys) : 1;
    }
    const int c = threadIdx.x % TPR, k = c % 16, group = threadIdx.x % kWave & 48;
    auto place = [&](int i, int n) { return ((i == 0 ? first : slot + i * step) << a.cut.tile_shift) + n; };
    auto put = [&](int n, f32x4_t acc, float den, float M) {
        const bool any = den != 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = any ? acc[e] / den : 0.f;
        const uint32_t t = a.by_g.div((uint32_t)(row0 + n)), g = (uint32_t)(row0 + n) - t * a.by_g.d;
        const int64_t at = ((int64_t)head * a.G + g) * a.T + req.begin + t;
        *(f32x4_t*)(a.O + at * D + c * 4) = acc;
        if (c == 0) a.lse[at] = any ? M + logf(den) : -INFINITY;
    };
    // a partial's weight: never 0 where it has any, so that what of its outputs is not finite stays (elsewhere the term is rounded off)
    auto weight = [](float l, float M) { return l == -INFINITY ? 0.f : expf(l - M) + __FLT_DENORM_MIN__; };
    auto add = [&](float w, f32x4_t o, f32x4_t& acc, float& den) {  // (a partial of no weight takes no part, whatever it holds)
        den += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(w, w != 0.f ? o[e] : 0.f, acc[e]);
    };
    for (int n0 = part * rows + threadIdx.x / TPR; n0 < (part + 1) * rows && row0 + n0 <= last; n0 += 2 * (kPagedMergeThreads / TPR)) {
        // two rows at a time; the second may not be there
        const int n1 = n0 + kPagedMergeThreads / TPR, n[2] = {n0, n1 < (part + 1) * rows && row0 + n1 <= last ? n1 : n0};
        if (S <= 4) {  // a row's threads read its log-sum-exps all of them, and everything is in flight at once
            float l[2][4];
            f32x4_t o[2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t at = place(i < S ? i : S - 1, n[r]);
                    l[r][i] = a.part_lse[at];
                    o[r][i] = *(const f32x4_t*)(a.part_O + at * D + c * 4);
                }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float M = -INFINITY, den = 0.f;
                f32x4_t acc = zero_vec<f32x4_t>();
#pragma unroll
                for (int i = 0; i < 4; ++i) M = fmaxf(M, i < S ? l[r][i] : -INFINITY);
#pragma unroll
                for (int i = 0; i < 4; ++i) add(i < S ? weight(l[r][i], M) : 0.f, o[r][i], acc, den);
                if (r == 0 || n[1] != n0) put(n[r], acc, den, M);
            }
            continue;
        }
#pragma unroll 1
        for (int row = n0; row <= n[1]; row += kPagedMergeThreads / TPR) {
            constexpr int NB = 16;
            f32x4_t o[NB];
            auto load_o = [&](int i0) {
#pragma unroll
                for (int u = 0; u < NB; ++u) o[u] = *(const f32x4_t*)(a.part_O + place(i0 + u < S ? i0 + u : S - 1, row) * D + c * 4);
            };
            load_o(0);
            float M = -INFINITY;
            for (int i = k; i < S; i += 16) M = fmaxf(M, a.part_lse[place(i, row)]);
            M = group_max<16>(M);
            f32x4_t acc = zero_vec<f32x4_t>();
            float den = 0.f;
            for (int i0 = 0; i0 < S; i0 += NB) {
                if (i0) load_o(i0);
                const float l = i0 + k < S ? a.part_lse[place(i0 + k, row)] : -INFINITY;
                const float mine = weight(l, M);
#pragma unroll
                for (int u = 0; u < NB; ++u) add(__shfl(mine, group + u), o[u], acc, den);
            }
            put(row, acc, den, M);
        }
    }
}

// Tiles in runs (a), then tiles cut by shares (d), each in several workgroups: first every tile's first rows, and so on, so that
// with 8 KV heads a workgroup runs on the XCD that wrote its partials (the tiles' own order has the heads innermost, too).
// KIND: 1 shares, 2 runs, 3 both (which of the two comes first is another trip to the arguments: 0.7 us of a short call).
template <int D, int KIND>
FEDRAG_KERNEL __launch_bounds__(kPagedMergeThreads) void paged_merge_kernel(const PagedArgs a, const PagedArgs d, uint32_t a_wgs, FastDiv tiles_a,
                                                                            FastDiv tiles_d, int rows_a, int rows_d) {
    const uint32_t i = blockIdx.x;
    if (KIND == 2 || (KIND == 3 && i < a_wgs)) {
        const uint32_t part = tiles_a.div(i);
        paged_merge<D, false>(a, i - part * tiles_a.d, (int)part, rows_a);
    } else {
        const uint32_t part = tiles_d.div(i - a_wgs);
        paged_merge<D, true>(d, i - a_wgs - part * tiles_d.d, (int)part, rows_d);
    }
}

// ------------------------------------------------------------------------------------------------ the launches
// What a form of the work may need, from the sizes the host knows.
struct PagedLaunch {
    PagedCut cut;
    int64_t grid;    // at least the pieces; 0: this form is not launched
    int64_t slots;   // at least the partials
    int64_t merges;  // at least the tiles in several partials
    size_t bytes(int D) const { return (((size_t)slots << cut.tile_shift) * (D + 1) * 4 + 15) / 16 * 16; }
    // Rows of a tile that a workgroup of the aggregation takes: those that its threads hold at once, while there are few workgroups
    // (117 rows over 4001 keys: 30.2 us, 35.7 with four times the rows each); else twice or four times that, as most of them, for
    // tiles that might be in several partials, only search (1024 over 16384 keys 2.3 % longer without, 512 over 2048 7 %).
    int merge_rows(int D) const {
        int rows = kPagedMergeThreads / (D / 4);
        const int most = cut.tile_shift >= 7 ? 4 * rows : 2 * rows;
        while (rows < most && 2 * rows <= 1 << cut.tile_shift && (merges << cut.tile_shift) / rows > (cut.tile_shift >= 7 ? 1024 : 512)) rows *= 2;
        return rows < 1 << cut.tile_shift ? rows : 1 << cut.tile_shift;
    }
    int64_t merge_groups(int D) const { return ((int64_t)1 << cut.tile_shift) / merge_rows(D); }
};
constexpr int kPagedDecodeRows = 16;  // a tile of the kernel for few rows

// tiles: at least the tiles of all requests and heads; keys: at most a request's.
static int64_t paged_units_of(PagedCut& cut, int64_t tiles, int64_t keys) {
    int64_t units = 1;
    do {
        units = keys > 0 ? ((keys - 1) >> cut.unit_shift) + 1 : 1;
    } while (tiles > INT32_MAX / units && ++cut.unit_shift < 31);
    return units;
}
static PagedLaunch paged_runs(PagedCut cut, int64_t tiles, int64_t keys) {
    const int64_t target = (int64_t)1 << cut.target_shift;
    const int64_t units = paged_units_of(cut, tiles, keys);
    const int64_t most_runs = units >= cut.least + cut.gain && (units + cut.least / 2) / cut.least > 1 ? (units + cut.least / 2) / cut.least : 1;
    PagedLaunch l{};
    l.cut = cut;
    l.grid = target + tiles < tiles * most_runs ? target + tiles : tiles * most_runs;
    l.slots = most_runs == 1 ? 0 : (l.grid < 2 * target ? l.grid : 2 * target);
    l.merges = most_runs == 1 ? 0 : (tiles < target ? tiles : target);
    return l;
}
static PagedLaunch paged_shares(PagedCut cut, int64_t tiles, int64_t keys) {
    const int64_t target = (int64_t)1 << cut.target_shift;
    const int64_t units = paged_units_of(cut, tiles, keys);
    const int64_t total = tiles * units;
    PagedLaunch l{};
    l.cut = cut;
    l.grid = (total + cut.least - 1) / cut.least < target ? (total + cut.least - 1) / cut.least : target;
    l.slots = units <= cut.least ? 0 : 2 * l.grid;
    l.merges = units <= cut.least ? 0 : l.grid - 1;
    return l;
}

// The forms of a call.  16-bit storage: requests of many rows (in runs), of few (in shares), or both, where the host cannot know that
// there are none; fp32: one form for all, of 16 or 32 rows, in runs.
struct PagedPlan {
    PagedLaunch runs, shares;
    size_t bytes(int D) const { return runs.bytes(D) + shares.bytes(D); }
};
static PagedPlan paged_plan(int B, int Hq, int Hkv, int dtype, int64_t T, int64_t keys, int64_t max_q_len) {
    const int64_t G = Hq / Hkv, some = B < T ? B : T;
    // at least the tiles that T rows of B requests come to
    auto tiles = [&](int tile_shift) { return ((T * G >> tile_shift) + some) * Hkv; };
    const int64_t most = max_q_len > 0 && max_q_len < T ? max_q_len : T;
    const int cus = 63 - __builtin_clzll((uint64_t)attn_target_wgs());  // compute units, rounded down to a power of two
    const bool many = most * G > kPagedDecodeRows, few = !many || B > 1;
    PagedPlan p{};
    if (dtype == FEDRAG_F32) {
        // A unit of keys is a step of each wave: as for 16 bits below, runs have one at least, two from a quarter of the compute units
        // on, four from half of them (least 1, 2, 4, of 32 heads: 33, 1 and 70 rows of 8 heads over 500, 1025 and 70 keys 18.1, 19.2,
        // 24.0 us; 64 over 512 23.6, 19.6, 24.6; 300 over 300 41.8, 41.5, 26.1).
        const int tile = many ? 5 : 4;
        const int64_t t = tiles(tile), full = (int64_t)1 << cus;
        p.runs = paged_runs(PagedCut{tile, 6, 4 * t < full ? 1 : 2 * t < full ? 2 : 4, cus + 1, 0, 1, INT32_MAX}, t, keys);
        return p;
    }
    if (many) {
        // Runs have four tiles of keys at least, but twice or four times that where the tiles alone occupy much of the device, as then
        // the aggregation costs more than shorter runs save (32 heads of 128, least 4 and by this rule: 512 rows over 512 keys 27.2 and
        // 22.8 us, 1000 over 1000 44.0 and 34.1; 64 over 1000 21.1, and 26.3 with 8), and one where there are hardly any (64 over 1000
        // 19.0, 20 over 500 19.2 and 15.6, 569 and 57 of 2 heads over as many 20.6 and 16.7; with 32 tiles 117 over 4001 30.1 and 31.2).
        // A cut has to save 6 units, 4 of few tiles (300 over 500 24.2 us without, 22.4 so; 64 over 300 17.1, and 18.3 with 6).
        // (t: beside the other form a request of this one has more than its rows)
        const int64_t by_rows = T * G / (kPagedDecodeRows + 1) * Hkv;
        const int64_t t = few && by_rows < tiles(7) ? by_rows : tiles(7), full = (int64_t)3 << cus >> 2;
        const int least = 8 * t <= full ? 1 : 2 * t < full ? 4 : t < full ? 8 : 16, gain = least == 1 ? 4 : 6;
        p.runs = paged_runs(PagedCut{7, 6, least, cus + 1, gain, few ? kPagedDecodeRows + 1 : 1, INT32_MAX}, t, keys);
    }
    // beside requests of many rows: one workgroup to a compute unit, for as long as the others take
    if (few)
        p.shares = paged_shares(PagedCut{4, 8, 1, many ? cus : cus + 1, 0, 1, many ? kPagedDecodeRows : INT32_MAX}, many ? some * Hkv : tiles(4), keys);
    return p;
}

bool paged_attn_fits(int B, int Hq, int Hkv, int D, int dtype, int64_t T, int64_t max_pages, int page_tokens, int64_t max_q_len, size_t* bytes) {
    *bytes = 0;
    if (T == 0 || B == 0) return true;
    const int64_t rows = T * (Hq / Hkv);
    if (rows > INT32_MAX || ((rows >> 4) + (B < T ? B : T)) * Hkv > INT32_MAX) return false;  // (tiles of 16 rows, the finest)
    const PagedPlan plan = paged_plan(B, Hq, Hkv, dtype, T, max_pages * page_tokens, max_q_len);
    if (!grid_fits(plan.runs.grid + plan.shares.grid, 256)) return false;  // (the aggregation's is below 2^14)
    *bytes = plan.bytes(D);
    return true;
}

hipError_t launch_paged_attn(const PagedAttnProblem& p, hipStream_t stream) {
    const int G = p.Hq / p.Hkv;
    PagedArgs a{};
    a.Q = p.Q;
    a.q_head_stride = p.q_head_stride;
    a.q_token_stride = p.q_token_stride;
    a.pages = p.pages;
    a.table = p.table;
    a.q_start = p.q_start;
    a.kv_lens = p.kv_lens;
    a.max_pages = p.max_pages;
    a.B = p.B;
    a.T = (int)p.T;
    a.G = G;
    a.Hkv = p.Hkv;
    a.causal = p.causal ? 1 : 0;
    a.by_g = FastDiv(G);
    a.by_hkv = FastDiv(p.Hkv);
    a.scale = p.scale;
    a.O = p.O;
    a.lse = p.lse;
    const PagedPlan plan = paged_plan(p.B, p.Hq, p.Hkv, p.dtype, p.T, p.max_pages << p.pages.shift, p.max_q_len);
    auto with = [&](const PagedLaunch& l, char* scratch) {
        PagedArgs x = a;
        x.cut = l.cut;
        x.slots = (uint32_t)l.slots;
        x.part_O = (float*)scratch;
        x.part_lse = x.part_O + (l.slots << l.cut.tile_shift) * p.D;
        return x;
    };
    const PagedArgs runs = with(plan.runs, (char*)p.workspace), shares = with(plan.shares, (char*)p.workspace + plan.runs.bytes(p.D));
    const int64_t wgs_r = plan.runs.merges * plan.runs.merge_groups(p.D), wgs_s = plan.shares.merges * plan.shares.merge_groups(p.D);
    const hipError_t e = p.dtype == FEDRAG_F32 ? launch_paged_f32(runs, plan.runs.grid, p.D, stream)
                                               : launch_paged_16(runs, plan.runs.grid, shares, plan.shares.grid, p.D, p.dtype, stream);
    if (e != hipSuccess || wgs_r + wgs_s == 0) return e;
#define FEDRAG_MERGE(KIND) (p.D == 128 ? paged_merge_kernel<128, KIND> : paged_merge_kernel<64, KIND>)
    const auto merge = wgs_r == 0 ? FEDRAG_MERGE(1) : wgs_s == 0 ? FEDRAG_MERGE(2) : FEDRAG_MERGE(3);
#undef FEDRAG_MERGE
    hipLaunchKernelGGL(merge, dim3((unsigned)(wgs_r + wgs_s)), dim3(kPagedMergeThreads), 0,
                       stream, runs, shares, (uint32_t)wgs_r, FastDiv(plan.runs.merges > 0 ? plan.runs.merges : 1),
                       FastDiv(plan.shares.merges > 0 ? plan.shares.merges : 1), plan.runs.merge_rows(p.D), plan.shares.merge_rows(p.D));
    return hipGetLastError();
}

}  // namespace fedrag
