// Attention of a ragged step over a paged cache (fedrag_paged_attn).
#include "attn_paged.h"

namespace fedrag {

// The aggregation (Section 4.1) of the tiles whose keys are in several partials: a workgroup takes 8 or 16 rows of one of them, a
// thread 4 columns of a row.  The lanes of a row share out the weights, 16 partials at a time.
// Which tile: SHARES: the one that workgroup blockIdx.x + 1's share begins inside of, if no share before does; else the
// blockIdx.x-th of those in several runs.
constexpr int kPagedMergeThreads = 256;
template <int D, bool SHARES>
FEDRAG_KERNEL __launch_bounds__(kPagedMergeThreads) void paged_merge_kernel(const PagedArgs a) {
    constexpr int TPR = D / 4;
    PagedRequest req;
    int tile, head, S = 0;
    int64_t slot, step, first = 0;  // partial i lies in slot + i * step, partial 0 in `first` if SHARES
    if constexpr (SHARES) {
        __shared__ PagedLanes lanes;
        const PagedShares<const PagedArgs> shares(a, lanes);
        const uint32_t w = blockIdx.x + 1, pos = w * shares.share;
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
        const PagedPiece p = paged_piece<true>(a, blockIdx.x);
        if (p.b < 0 || p.slot + (uint32_t)(p.runs - 1) * (uint32_t)a.Hkv >= a.slots) return;  // (the latter where q_start decreases)
        req = p.req;
        tile = p.tile;
        head = p.head;
        slot = first = p.slot;
        step = a.Hkv;
        S = p.per;  // units of a run, for now
    }
    const int row0 = tile << a.cut.tile_shift, n = blockIdx.y * (kPagedMergeThreads / TPR) + threadIdx.x / TPR;
    const int c = threadIdx.x % TPR, k = c % 16, group = threadIdx.x % kWave & 48;
    const int last = (row0 + (1 << a.cut.tile_shift) < req.R ? row0 + (1 << a.cut.tile_shift) : req.R) - 1;
    if (row0 + n > last) return;
    if constexpr (!SHARES) {  // runs that hold keys which some row of the tile sees
        const int64_t run_keys = (int64_t)S << a.cut.unit_shift, seen = paged_limit(a, req, last);
        S = seen > 0 ? (int)((seen + run_keys - 1) / run_keys) : 1;
    }
    auto place = [&](int i) { return ((i == 0 ? first : slot + i * step) << a.cut.tile_shift) + n; };
    constexpr int NB = 16;
    f32x4_t o[NB];
    auto load_o = [&](int i0) {
#pragma unroll
        for (int u = 0; u < NB; ++u) o[u] = *(const f32x4_t*)(a.part_O + place(i0 + u < S ? i0 + u : S - 1) * D + c * 4);
    };
    load_o(0);
    float M = -INFINITY;
    for (int i = k; i < S; i += 16) M = fmaxf(M, a.part_lse[place(i)]);
    M = group_max<16>(M);
    f32x4_t acc = zero_vec<f32x4_t>();
    float den = 0.f;
    for (int i0 = 0; i0 < S; i0 += NB) {
        if (i0) load_o(i0);
        const float l = i0 + k < S ? a.part_lse[place(i0 + k)] : -INFINITY;
        const float mine = l == -INFINITY ? 0.f : expf(l - M);
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const float w = __shfl(mine, group + u);
            den += w;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(w, w != 0.f ? o[u][e] : 0.f, acc[e]);
        }
    }
    const bool any = den != 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = any ? acc[e] / den : 0.f;
    const uint32_t t = a.by_g.div((uint32_t)(row0 + n)), g = (uint32_t)(row0 + n) - t * a.by_g.d;
    const int64_t at = ((int64_t)head * a.G + g) * a.T + req.begin + t;
    *(f32x4_t*)(a.O + at * D + c * 4) = acc;
    if (c == 0) a.lse[at] = any ? M + logf(den) : -INFINITY;
}

// ------------------------------------------------------------------------------------------------ the launches
// What a launch may need, from the sizes the host knows.
struct PagedLaunch {
    PagedCut cut;
    int64_t grid;    // at least the pieces
    int64_t slots;   // at least the split pieces
    int64_t merges;  // at least the split tiles
    bool shares;
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
    const int64_t most_runs = units > cut.least ? (units + cut.least - 1) / cut.least : 1;
    PagedLaunch l;
    l.cut = cut;
    l.grid = target + tiles < tiles * most_runs ? target + tiles : tiles * most_runs;
    l.slots = most_runs == 1 ? 0 : (l.grid < 2 * target ? l.grid : 2 * target);
    l.merges = most_runs == 1 ? 0 : (tiles < target ? tiles : target);
    l.shares = false;
    return l;
}
static PagedLaunch paged_shares(PagedCut cut, int64_t tiles, int64_t keys) {
    const int64_t target = (int64_t)1 << cut.target_shift;
    const int64_t units = paged_units_of(cut, tiles, keys);
    const int64_t total = tiles * units;
    PagedLaunch l;
    l.cut = cut;
    l.grid = (total + cut.least - 1) / cut.least < target ? (total + cut.least - 1) / cut.least : target;
    l.slots = units <= cut.least ? 0 : 2 * l.grid;
    l.merges = units <= cut.least ? 0 : l.grid - 1;
    l.shares = true;
    return l;
}
static size_t paged_bytes(const PagedLaunch& l, int D) { return (((size_t)l.slots << l.cut.tile_shift) * (D + 1) * 4 + 15) / 16 * 16; }

// The launches of a call.  16-bit storage: requests of few rows, of many, or both, where the host cannot know that there are
// none; fp32: one form for all, of 16 or 32 rows.
struct PagedPlan {
    int n;
    PagedLaunch l[2];
    hipError_t (*kernel[2])(const PagedArgs&, int, int, int64_t, hipStream_t);
    size_t bytes(int D) const { return (n > 0 ? paged_bytes(l[0], D) : 0) + (n > 1 ? paged_bytes(l[1], D) : 0); }
};
static PagedPlan paged_plan(int B, int Hq, int Hkv, int dtype, int64_t T, int64_t keys, int64_t max_q_len) {
    const int64_t G = Hq / Hkv, some = B < T ? B : T;
    // at least the tiles that T rows of B requests come to
    auto tiles = [&](int tile_shift) { return ((T * G >> tile_shift) + some) * Hkv; };
    const int64_t most = max_q_len > 0 && max_q_len < T ? max_q_len : T;
    const int shift = 63 - __builtin_clzll(2 * (uint64_t)attn_target_wgs());  // two workgroups to a compute unit, rounded down
    const bool many = most * G > kPagedDecodeRows, few = !many || B > 1;
    PagedPlan p{};
    auto add = [&](auto kernel, auto how, int tile_shift, int unit_shift, int least, int from, int to, int64_t most_tiles) {
        p.l[p.n] = how(PagedCut{tile_shift, unit_shift, least, shift, from, to}, most_tiles, keys);
        p.kernel[p.n++] = kernel;
    };
    if (dtype == FEDRAG_F32) {
        const int tile = many ? 5 : 4;
        add(launch_paged_f32, paged_runs, tile, 6, 4, 1, INT32_MAX, tiles(tile));
        return p;
    }
    if (many) add(launch_paged_chunk, paged_runs, 7, 6, 4, few ? kPagedDecodeRows + 1 : 1, INT32_MAX, tiles(7));
    if (few)
        add(launch_paged_decode, paged_shares, 4, 8, 1, 1, many ? kPagedDecodeRows : INT32_MAX, many ? some * Hkv : tiles(4));
    return p;
}

size_t paged_attn_workspace_bytes(int B, int Hq, int Hkv, int D, int dtype, int64_t T, int64_t max_pages, int page_tokens,
                                  int64_t max_q_len) {
    if (T == 0 || B == 0) return 0;
    return paged_plan(B, Hq, Hkv, dtype, T, max_pages * page_tokens, max_q_len).bytes(D);
}

static hipError_t launch_paged_merge(const PagedArgs& a, const PagedLaunch& l, int D, hipStream_t stream) {
    const int64_t groups = ((D / 4 << l.cut.tile_shift) + kPagedMergeThreads - 1) / kPagedMergeThreads;
    if (!grid_fits(l.merges * groups, kPagedMergeThreads)) return hipErrorInvalidValue;
    const auto kernel = l.shares ? (D == 128 ? paged_merge_kernel<128, true> : paged_merge_kernel<64, true>)
                                 : (D == 128 ? paged_merge_kernel<128, false> : paged_merge_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)l.merges, (unsigned)groups),
                       dim3(kPagedMergeThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnProblem& p, hipStream_t stream) {
    const int G = p.Hq / p.Hkv;
    if (p.T * G > INT32_MAX) return hipErrorInvalidValue;
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
    char* scratch = (char*)p.workspace;
    for (int i = 0; i < plan.n; ++i) {
        const PagedLaunch& l = plan.l[i];
        a.cut = l.cut;
        a.slots = (uint32_t)l.slots;
        a.part_O = (float*)scratch;
        a.part_lse = a.part_O + (l.slots << l.cut.tile_shift) * p.D;
        scratch += paged_bytes(l, p.D);
        hipError_t e = plan.kernel[i](a, p.D, p.dtype, l.grid, stream);
        if (e == hipSuccess && l.merges > 0) e = launch_paged_merge(a, l, p.D, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace fedrag
