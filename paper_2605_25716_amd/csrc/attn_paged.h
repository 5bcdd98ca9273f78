// What the kernels of attention over a paged cache share: the step as they see it, and how they find their piece of it.
#pragma once
#include <type_traits>

#include "fedrag_device.h"
#include "fedrag_host.h"

namespace fedrag {

// The work of a launch, cut up on the device: the host knows no lengths.  Request b has R = rows * G flattened query rows per
// KV head (row r = token r / G, head r % G of the group), in tiles of `tile` rows, and n = ceil(keys / unit) units of keys for each
// of them.  Runs of at most `per` units, per = max(least, ceil(sum of tiles * n * Hkv / target)), are a workgroup's piece; so
//   pieces       <= target + tiles of all requests and heads   (the grid),
//   split pieces <= 2 target                                   (a tile in two or more runs has n > per: their partials),
//   split tiles  <= target                                     (what the aggregation has to visit).
// `target` is a power of two: no division of the 64-bit sum.
struct PagedCut {
    int tile, unit_shift, least, target_shift;
    int few, many;  // only requests with few <= R <= many are this launch's
};

struct PagedArgs {
    const char* Q;
    int64_t q_head_stride, q_token_stride;  // bytes
    Pages pages;
    const int32_t *table, *q_start, *kv_lens;
    int64_t max_pages;
    int B, T, G, Hkv, causal;
    FastDiv by_g, by_hkv;
    float scale;
    float *O, *lse;
    float *part_O, *part_lse;  // [slot][tile][D], [slot][tile]
    uint32_t slots;
    PagedCut cut;
};

struct PagedRequest {
    int begin, rows, R;  // its first row, how many, times G
    int kv;              // keys the request has
    int keys;            // those that its table has columns for
    int tiles, n;        // tiles of query rows, units of keys
};

__device__ __forceinline__ PagedRequest paged_request(const PagedArgs& a, int b) {
    int s = a.q_start[b], e = a.q_start[b + 1], kv = a.kv_lens[b];
    s = s < 0 ? 0 : (s < a.T ? s : a.T);
    e = e < 0 ? 0 : (e < a.T ? e : a.T);
    PagedRequest r;
    r.begin = s;
    r.rows = e > s ? e - s : 0;
    r.kv = kv < 0 ? 0 : kv;
    const int64_t room = a.max_pages << a.pages.shift;
    r.keys = r.kv < room ? r.kv : (int)room;
    const int64_t R = (int64_t)r.rows * a.G;
    r.R = (int)R;  // below 2^31: checked by the host
    const bool mine = r.R >= a.cut.few && r.R <= a.cut.many;
    r.tiles = mine ? (r.R + a.cut.tile - 1) / a.cut.tile : 0;
    r.n = (int)(((int64_t)r.keys + (1 << a.cut.unit_shift) - 1) >> a.cut.unit_shift);
    return r;
}

__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ uint32_t wave_total(uint32_t x) { return lane_value(wave_scan(x), kWave - 1); }

// Units of keys of the longest run, from each lane's share of the work.  (Held below 2^49 a lane, where it already comes to runs
// of any length.)
__device__ __forceinline__ uint32_t paged_per(const PagedArgs& a, uint64_t cost) {
    cost = cost < ((uint64_t)1 << 49) ? cost : (uint64_t)1 << 49;
    const uint64_t sum = ((uint64_t)wave_total((uint32_t)(cost >> 24)) << 24) + wave_total((uint32_t)cost & 0xffffff);
    const uint64_t per = (sum + ((uint64_t)1 << a.cut.target_shift) - 1) >> a.cut.target_shift;
    const uint32_t p = per > 0x7fffffff ? 0x7fffffff : (uint32_t)per;
    return p > (uint32_t)a.cut.least ? p : (uint32_t)a.cut.least;
}
__device__ __forceinline__ uint32_t paged_runs(const PagedRequest& r, uint32_t per) {
    return (uint32_t)r.n <= per ? 1 : ((uint32_t)r.n + per - 1) / per;
}

// A piece of the work, uniform over the wave.
struct PagedPiece {
    int b;             // request; < 0: there is no such piece
    PagedRequest req;
    int tile, head, run, runs, per;  // tile of rows, KV head, run of keys of `per` units
    uint32_t slot;     // of its partial, if runs > 1; for SPLIT that of run 0
};

// Piece `index` of the launch, or (SPLIT) of its split tiles: each wave finds it by itself, a lane per ceil(B / 64) requests that
// follow each other.  One trip to memory up to 64 requests.  The pieces of a request: tile by tile, the last one first (with a
// mask the longest), run by run, the heads innermost: workgroups are dealt to the XCDs in turn, so with 8 KV heads the pieces that
// read the same keys share an L2.
template <bool SPLIT>
__device__ __forceinline__ PagedPiece paged_piece(const PagedArgs& a, uint32_t index) {
    const int lane = threadIdx.x % kWave;
    const int k = (a.B + kWave - 1) / kWave;  // requests per lane
    const int64_t b0 = (int64_t)lane * k;
    PagedRequest one{};
    uint64_t cost = 0;
    auto add_cost = [&](const PagedRequest& r) { cost += (uint64_t)((uint32_t)r.tiles * (uint32_t)a.Hkv) * (uint32_t)r.n; };
    PagedPiece p{};
    p.b = -1;
    uint32_t pieces = 0, split = 0;
    auto count = [&](const PagedRequest& r, uint32_t per) {
        const uint32_t runs = paged_runs(r, per), n = (uint32_t)r.tiles * (uint32_t)a.Hkv;
        split += runs > 1 ? n * runs : 0;
        pieces += SPLIT ? (runs > 1 ? n : 0) : n * runs;
    };
    uint32_t per;
    if (k == 1) {
        if (b0 < a.B) one = paged_request(a, (int)b0);
        add_cost(one);
        per = paged_per(a, cost);
        count(one, per);
    } else {
        for (int i = 0; i < k; ++i)
            if (b0 + i < a.B) add_cost(paged_request(a, (int)(b0 + i)));
        per = paged_per(a, cost);
        for (int i = 0; i < k; ++i)
            if (b0 + i < a.B) count(paged_request(a, (int)(b0 + i)), per);
    }
    uint32_t pieces_to = wave_scan(pieces), split_to = wave_scan(split);
    const uint64_t past = __builtin_amdgcn_ballot_w64(pieces_to <= index);
    int at = __builtin_popcountll(past);
    if (at == kWave) return p;
    uint32_t base = at ? lane_value(pieces_to, at - 1) : 0, slot = at ? lane_value(split_to, at - 1) : 0;
    int b = at;
    if (k > 1) {  // among that lane's requests, 64 at a time
        for (int i0 = 0;; i0 += kWave) {
            const int64_t c = (int64_t)at * k + i0 + lane;
            const bool is = i0 + lane < k && c < a.B;
            one = PagedRequest{};
            if (is) one = paged_request(a, (int)c);
            pieces = split = 0;
            if (is) count(one, per);
            pieces_to = wave_scan(pieces);
            split_to = wave_scan(split);
            const int in = __builtin_popcountll(__builtin_amdgcn_ballot_w64(base + pieces_to <= index));
            if (in < kWave || i0 + kWave >= k) {  // (there is one: the lane's sum said so)
                const int j = in < kWave ? in : kWave - 1;
                b = at * k + i0 + j;
                if (j) {
                    slot += lane_value(split_to, j - 1);
                    base += lane_value(pieces_to, j - 1);
                }
                at = j;
                break;
            }
            base += lane_value(pieces_to, kWave - 1);
            slot += lane_value(split_to, kWave - 1);
        }
    }
    p.b = b;
    p.req.begin = (int)lane_value((uint32_t)one.begin, at);
    p.req.rows = (int)lane_value((uint32_t)one.rows, at);
    p.req.R = (int)lane_value((uint32_t)one.R, at);
    p.req.kv = (int)lane_value((uint32_t)one.kv, at);
    p.req.keys = (int)lane_value((uint32_t)one.keys, at);
    p.req.tiles = (int)lane_value((uint32_t)one.tiles, at);
    p.req.n = (int)lane_value((uint32_t)one.n, at);
    const uint32_t runs = paged_runs(p.req, per), i = index - base;
    const uint32_t rest = a.by_hkv.div(i);
    p.head = (int)(i - rest * a.by_hkv.d);
    const uint32_t tile = SPLIT || runs == 1 ? rest : rest / runs;
    p.run = SPLIT || runs == 1 ? 0 : (int)(rest - tile * runs);
    p.tile = p.req.tiles - 1 - (int)tile;
    p.runs = (int)runs;
    p.per = (int)(((uint32_t)p.req.n + runs - 1) / runs);
    p.slot = slot + (SPLIT ? (tile * runs) * (uint32_t)a.Hkv + (uint32_t)p.head : i);  // run r's: r * Hkv further
    return p;
}

// Keys that a flattened row sees: row r of the request is token r / G.
__device__ __forceinline__ int paged_limit(const PagedArgs& a, const PagedRequest& q, int r) {
    if (!a.causal) return q.keys;
    const int64_t own = (int64_t)q.kv - q.rows + (int)a.by_g.div((uint32_t)r) + 1;
    return own < 0 ? 0 : (own < q.keys ? (int)own : q.keys);
}

hipError_t launch_paged_decode(const PagedArgs& a, int D, int dtype, int64_t grid, hipStream_t stream);
hipError_t launch_paged_f32(const PagedArgs& a, int D, int dtype, int64_t grid, hipStream_t stream);
hipError_t launch_paged_chunk(const PagedArgs& a, int D, int dtype, int64_t grid, hipStream_t stream);

}  // namespace fedrag
