// What the kernels of attention over a paged cache share: the step as they see it, and how they find their part of it.
#pragma once
#include <type_traits>

#include "fedrag_device.h"
#include "fedrag_host.h"

namespace fedrag {

// The work of a launch is cut up on the device: the host knows no lengths.  Request b has R = rows * G flattened query rows per
// KV head (row r = token r / G, head r % G of the group), in tiles of 2^tile_shift rows, and n = ceil(keys / unit) units of keys (at least
// one: a row without keys has an output all the same) for each of them.  All units together are below 2^31, which the host sees
// to by way of `unit_shift`.  There are two ways to cut:
//   runs    a tile's keys in equal runs of about `per` = ceil(units of all / target) units (those that the mask
//           hides among them), as many as n / per rounds to; a workgroup takes one.  The target is one workgroup to a compute unit while that makes runs of up to eight units, and two
//           from 16 on (two that share it work at half the rate, and write twice the partials: 64 rows of 28 heads of 64 over 6000 keys,
//           6 units, 24.1 us with two, 20.5 with one; 128 of 32 heads of 128 over 16384, 16 units, 67.1 and 68.8).  In between runs stay
//           at eight units, and some compute units get two and some one, which was not looked at more closely.  `least` is the least.
//           A tile is not cut where that saves less than `gain` units, or if it has at most 48 units and no more than a compute unit's
//           part of the work and a third (1200 rows of 32 heads over 1800 keys cut 82.8 us, whole 62.4, 1000 over 1500 53.0 and 48.9;
//           700 over 1500, one and a half times the part, 41.3 and 44.3; 1024 over 16384, 256 units, cut 7 % less than whole, as two workgroups
//           that share a compute unit get 8 % more out of it); not so tiles of fewer rows (377 fp32 rows beside twelve single ones 42 and 56).
//           With a least of 1 a run has c sqrt(n) units, c = 2 / 5 for tiles of 128 rows and 1 / 5 for less: of few tiles of many keys the time to
//           fold n / per partials grows as the time of a run falls (20 rows of 4 heads over 30000 keys, 117 runs 31.8 us, so 59 31.9,
//           469 47.6; 3 of 14 over 6856 27, 27, 108 runs 18.0, 18.9, 25.3; one fp32 row over 30000 40.1, 31.3 by c = 1 / 5).
//             runs         <= target + tiles of all requests and heads   (the grid),
//             split runs   <= 4 / 3 target                               (a tile in two or more has n >= 1.5 per: their partials),
//             split tiles  <= 2 / 3 target                               (what the aggregation has to visit);
//   shares  the units of all tiles in a row, and an even share of them to each workgroup, wherever in a tile it begins and ends:
//           all workgroups end together, whatever the lengths.  For kernels whose partials are small.
// `target` is a power of two.
constexpr uint32_t kPagedShortRun = 8, kPagedWhole = 48;
struct PagedCut {
    int tile_shift, unit_shift, least, target_shift;
    int gain;       // runs: a tile is cut only if they are shorter than the whole by so many units
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
    float *part_O, *part_lse;  // [slot][rows of a tile][D], [slot][rows of a tile]
    uint32_t slots;
    PagedCut cut;
};

// Arguments number N of a kernel, all of this type, read again from memory from here on: what is needed between inner loops would
// otherwise sit in scalar registers throughout, and those that do not fit in lanes of vector registers or in scratch memory.
typedef const __attribute__((address_space(4))) PagedArgs PagedArgsLate;
template <int N>
__device__ __forceinline__ PagedArgsLate& late_args() {
    PagedArgsLate* p = (PagedArgsLate*)__builtin_amdgcn_kernarg_segment_ptr() + N;
    asm volatile("" : "+s"(p));
    return *p;
}

struct PagedRequest {
    int begin, R;  // its first row, and the flattened ones
    int kv;        // keys the request has
    int keys;      // those that its table has columns for
};

// Request b, in two steps: the loads, which many requests have in flight at once, and the rest.
struct PagedLens {
    int s, e, kv;
};
template <class Args>
__device__ __forceinline__ PagedLens paged_lens(Args& a, int b) { return PagedLens{a.q_start[b], a.q_start[b + 1], a.kv_lens[b]}; }
template <class Args>
__device__ __forceinline__ PagedRequest paged_request(Args& a, PagedLens l) {
    const int s = l.s < 0 ? 0 : (l.s < a.T ? l.s : a.T), e = l.e < 0 ? 0 : (l.e < a.T ? l.e : a.T);
    const int64_t room = a.max_pages << a.pages.shift;
    PagedRequest r;
    r.begin = s;
    r.R = e > s ? (e - s) * a.G : 0;  // below 2^31: checked by the host
    r.kv = l.kv < 0 ? 0 : l.kv;
    r.keys = r.kv < room ? r.kv : (int)room;
    return r;
}
template <class Args>
__device__ __forceinline__ uint32_t paged_tiles(Args& a, const PagedRequest& r) {
    return r.R >= a.cut.few && r.R <= a.cut.many ? ((uint32_t)r.R + (1u << a.cut.tile_shift) - 1) >> a.cut.tile_shift : 0;
}
template <class Args>
__device__ __forceinline__ uint32_t paged_units(Args& a, const PagedRequest& r) {
    return r.keys > 0 ? ((uint32_t)(r.keys - 1) >> a.cut.unit_shift) + 1 : 1;
}

__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ __forceinline__ PagedRequest lane_request(const PagedRequest& r, int lane) {
    return PagedRequest{(int)lane_value((uint32_t)r.begin, lane), (int)lane_value((uint32_t)r.R, lane), (int)lane_value((uint32_t)r.kv, lane),
                        (int)lane_value((uint32_t)r.keys, lane)};
}

// A lane's requests, k = ceil(B / 64) that follow each other: f(request, there is one) for each, the loads of four at a time in
// flight together.
template <class Args, class F>
__device__ __forceinline__ void paged_each(Args& a, F f) {
    const int k = (a.B + kWave - 1) / kWave, b0 = threadIdx.x % kWave * k;
    if (k == 1) {
        f(paged_request(a, paged_lens(a, b0 < a.B ? b0 : a.B - 1)), b0 < a.B);
        return;
    }
    for (int i = 0; i < k; i += 4) {
        PagedLens l[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) l[u] = paged_lens(a, b0 + i + u < a.B ? b0 + i + u : a.B - 1);
#pragma unroll
        for (int u = 0; u < 4; ++u) f(paged_request(a, l[u]), i + u < k && b0 + i + u < a.B);
    }
}

// The request that holds number `x` of something that every request has some of, given the sums up to each lane's last request
// (`to`; some lane's is above x), what a lane's one request is (k == 1), and what a request has of it.  base: the sum of the
// requests before.
template <class Args, class Count>
__device__ __forceinline__ PagedRequest paged_find(Args& a, uint32_t x, uint32_t to, PagedRequest one, Count count, int* b, uint32_t* base) {
    const int k = (a.B + kWave - 1) / kWave, lane = threadIdx.x % kWave;
    int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(to <= x));
    *base = at ? lane_value(to, at - 1) : 0;
    *b = at;
    if (k > 1) {  // among that lane's requests, 64 at a time
        const int first = at * k;
        for (int i0 = 0; i0 < k; i0 += kWave) {
            const bool is = i0 + lane < k && first + i0 + lane < a.B;
            one = paged_request(a, paged_lens(a, is ? first + i0 + lane : a.B - 1));
            const uint32_t sums = *base + wave_scan(is ? count(one) : 0);
            at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(sums <= x));
            *b = first + i0 + at;
            if (at < kWave) {
                if (at) *base = lane_value(sums, at - 1);
                break;
            }
            *base = lane_value(sums, kWave - 1);
        }
        at &= kWave - 1;
    }
    return lane_request(one, at);
}

// ---- runs
struct PagedPiece {
    int b;                     // request; < 0: there is no such piece
    PagedRequest req;
    int tile, head, run, runs, per;  // tile of rows, KV head, run of keys of `per` units
    uint32_t slot;             // of its partial, if runs > 1; SPLIT: of run 0
};

// Piece `index` of the launch, or (SPLIT) of its split tiles; each wave finds it by itself.  The pieces of a request: tile by
// tile, the last one first (with a mask the longest), run by run, the heads innermost: workgroups are dealt to the XCDs in turn, so
// with 8 KV heads the pieces that read the same keys share an L2.  Up to 64 requests go side by side, so that long pieces start
// early: the order is that of the pieces' lengths, which with a mask fall from tile to tile (4 x 1000 tokens of 32 heads of 128 one
// request after the other 88 us, 80).
template <bool SPLIT, class Args>
__device__ __forceinline__ PagedPiece paged_piece(Args& a, uint32_t index) {
    PagedRequest one{};
    uint32_t cost = 0;
    paged_each(a, [&](const PagedRequest& r, bool is) {
        one = r;
        cost += is ? paged_tiles(a, r) * (uint32_t)a.Hkv * paged_units(a, r) : 0;
    });
    const uint32_t sum = lane_value(wave_scan(cost), kWave - 1);
    PagedPiece p{};
    p.b = -1;
    if (sum == 0) return p;  // (no requests of this form: the grid was for those that there might be)
    auto evenly = [&](uint64_t units) { return (uint32_t)((units + ((uint64_t)1 << a.cut.target_shift) - 1) >> a.cut.target_shift); };
    const uint32_t unit = evenly((uint64_t)sum * 2);  // of a compute unit
    const uint32_t whole = unit + unit / 3 < kPagedWhole ? unit + unit / 3 : kPagedWhole;
    uint32_t per = unit < kPagedShortRun ? unit : kPagedShortRun;
    per = per > evenly(sum) ? per : evenly(sum);
    per = per > (uint32_t)a.cut.least ? per : (uint32_t)a.cut.least;
    auto runs_of = [&](const PagedRequest& r) {
        const uint32_t n = paged_units(a, r);
        uint32_t len = per;
        if (a.cut.least == 1) {
            const uint32_t fold = (uint32_t)(__builtin_amdgcn_sqrtf((float)n) * (a.cut.tile_shift >= 7 ? 0.4f : 0.2f));
            len = len > fold ? len : fold;
        }
        return 2 * n < 3 * len || n < len + (uint32_t)a.cut.gain || (a.cut.tile_shift >= 7 && n <= whole) ? 1 : (n + len / 2) / len;
    };
    auto pieces_of = [&](const PagedRequest& r) {
        const uint32_t runs = runs_of(r), n = paged_tiles(a, r) * (uint32_t)a.Hkv;
        return SPLIT ? (runs > 1 ? n : 0) : n * runs;
    };
    auto split_of = [&](const PagedRequest& r) {
        const uint32_t runs = runs_of(r);
        return runs > 1 ? paged_tiles(a, r) * (uint32_t)a.Hkv * runs : 0;
    };
    uint32_t pieces = 0, split = 0;
    paged_each(a, [&](const PagedRequest& r, bool is) {
        pieces += is ? pieces_of(r) : 0;
        split += is ? split_of(r) : 0;
    });
    const uint32_t to = wave_scan(pieces), split_to = wave_scan(split);
    if (lane_value(to, kWave - 1) <= index) return p;
    const int k = (a.B + kWave - 1) / kWave;
    uint32_t group = FastDiv::div_by(a.by_hkv.m, a.by_hkv.s, index);  // a tile and run of a request
    uint32_t slot, before;                                            // before: tiles of the request that come before it
    p.head = (int)(index - group * a.by_hkv.d);
    if (!SPLIT && k == 1) {
        // Where all pieces start at once, i and i + compute units on the same one, the second half's go in reverse: the longest beside
        // the shortest (1500 tokens 55.5 us without, 51.7 so; 2000 72.4, 67.6; 512 in fp32 42.8, 37.0).  Not beside the form for few rows,
        // whose workgroups come in between.
        const uint32_t groups = FastDiv::div_by(a.by_hkv.m, a.by_hkv.s, lane_value(to, kWave - 1));
        const uint32_t half = FastDiv::div_by(a.by_hkv.m, a.by_hkv.s, 1u << (a.cut.target_shift - 1));
        if (a.cut.few <= 1 && group >= half && groups <= 2 * half) group = groups - 1 - (group - half);
        const uint32_t tiles = (int)threadIdx.x % kWave < a.B ? paged_tiles(a, one) : 0, runs = runs_of(one);
        // a piece's place in the order: its length behind the longest's in key units, as tiles, and with a mask also its tile
        const uint32_t len = tiles ? (paged_units(a, one) + runs - 1) / runs : 0;
        const uint32_t ahead = (uint32_t)((uint64_t)(wave_max(len) - len) * (uint32_t)a.G << a.cut.unit_shift >> a.cut.tile_shift);
        auto before_level = [&](uint32_t level) {  // groups of this lane's request before it
            const uint32_t v = level > ahead ? level - ahead : 0;
            return (!a.causal && v > 0) || v > tiles ? tiles * runs : v * runs;
        };
        auto below = [&](uint32_t level) { return lane_value(wave_scan(before_level(level)), kWave - 1); };
        uint32_t level = 0;  // the most whose groups all lie before this one
        for (uint32_t bit = (uint32_t)1 << (31 - __builtin_clz(wave_max(tiles ? tiles + ahead : 0) | 1)); bit; bit >>= 1)
            if (below(level + bit) <= group) level += bit;
        const uint32_t here = wave_scan(before_level(level + 1) - before_level(level));
        group -= below(level);
        p.b = __builtin_popcountll(__builtin_amdgcn_ballot_w64(here <= group));
        if (p.b >= kWave) {  // (only by a q_start that decreases)
            p.b = -1;
            return p;
        }
        group -= p.b ? lane_value(here, p.b - 1) : 0;
        p.req = lane_request(one, p.b);
        slot = p.b ? lane_value(split_to, p.b - 1) : 0;
        const uint32_t n_runs = runs_of(p.req);
        before = a.causal ? level - lane_value(ahead, p.b) : group / n_runs;
        p.run = (int)(a.causal ? group : group - before * n_runs);
    } else {
        const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(to <= group * (uint32_t)a.Hkv));
        uint32_t base;
        p.req = paged_find(a, group * (uint32_t)a.Hkv, to, one, pieces_of, &p.b, &base);
        slot = at ? lane_value(split_to, at - 1) : 0;
        for (int b = at * k; b < p.b; ++b) slot += split_of(paged_request(a, paged_lens(a, b)));
        const uint32_t runs = SPLIT ? 1 : runs_of(p.req), rest = group - FastDiv::div_by(a.by_hkv.m, a.by_hkv.s, base);
        before = runs == 1 ? rest : rest / runs;
        p.run = (int)(rest - before * runs);
    }
    const uint32_t runs = runs_of(p.req), n = paged_units(a, p.req), tiles = paged_tiles(a, p.req);
    p.tile = (int)(tiles - 1 - before);
    p.runs = (int)runs;
    p.per = (int)((n + runs - 1) / runs);
    p.slot = slot + (before * runs + (uint32_t)p.run) * (uint32_t)a.Hkv + (uint32_t)p.head;  // SPLIT: run 0's; run r's is r * Hkv further
    // (only sums beyond 32 bits, by a q_start that decreases, lead here)
    if (before >= tiles || p.b >= a.B || (!SPLIT && runs > 1 && p.slot >= a.slots)) p.b = -1;
    return p;
}

// ---- shares
// A share is ceil(units of all / target) units, or `least`.  A tile of few units (at most `least`, or an eighth of a share) is not
// cut: it belongs as a whole to the share in which it begins.  Partials: workgroup w's of a tile that another began in slot 2 w, of one that it begins and does
// not end in slot 2 w + 1.
struct PagedSpan {
    PagedRequest req;
    int b, tile, head;  // b < 0: behind the last
    uint32_t begin, n;  // where the tile begins in the row of units, and its units
};
// What each lane has found out about its requests, in LDS: a search costs no trip to memory, and no registers in between.
struct PagedLanes {
    uint32_t to[kWave];       // units up to the lane's last request
    PagedRequest one[kWave];  // its request, where it has one
};
template <class Args>
struct PagedShares {
    PagedLanes& lanes;
    uint32_t total, share, whole;  // a tile of no more than `whole` units is not cut

    static __device__ __forceinline__ uint32_t cost(Args& a, const PagedRequest& r) {
        return paged_tiles(a, r) * (uint32_t)a.Hkv * paged_units(a, r);
    }
    // By all threads: the first wave counts, the others wait for it.
    __device__ __forceinline__ PagedShares(Args& a, PagedLanes& found) : lanes(found) {
        const int lane = threadIdx.x % kWave;
        if (threadIdx.x < kWave) {
            PagedRequest one{};
            uint32_t mine = 0;
            paged_each(a, [&](const PagedRequest& r, bool is) {
                one = r;
                mine += is ? cost(a, r) : 0;
            });
            lanes.to[lane] = wave_scan(mine);
            lanes.one[lane] = one;
        }
        __syncthreads();
        total = lane_value(lanes.to[kWave - 1], 0);
        share = (uint32_t)(((uint64_t)total + ((uint64_t)1 << a.cut.target_shift) - 1) >> a.cut.target_shift);
        share = share > (uint32_t)a.cut.least ? share : (uint32_t)a.cut.least;
        whole = share / 8 > (uint32_t)a.cut.least ? share / 8 : (uint32_t)a.cut.least;
    }
    // The tile that unit `pos` belongs to.
    __device__ __forceinline__ PagedSpan find(Args& a, uint32_t pos) const {
        PagedSpan s{};
        s.b = -1;
        if (pos >= total) return s;
        uint32_t base;
        const int lane = threadIdx.x % kWave;
        s.req = paged_find(a, pos, lanes.to[lane], lanes.one[lane], [&](const PagedRequest& r) { return cost(a, r); }, &s.b, &base);
        s.n = paged_units(a, s.req);
        const uint32_t i = (pos - base) / s.n, tile = FastDiv::div_by(a.by_hkv.m, a.by_hkv.s, i);
        s.begin = base + i * s.n;
        s.head = (int)(i - tile * a.by_hkv.d);
        const uint32_t tiles = paged_tiles(a, s.req);
        s.tile = (int)(tiles - 1 - tile);
        if (tile >= tiles || s.b >= a.B) s.b = -1;  // (only sums beyond 32 bits, by a q_start that decreases, lead here)
        return s;
    }
};

// Keys that a flattened row sees: row r of the request is token r / G, and rows / G the last.
template <class Args>
__device__ __forceinline__ int paged_limit(Args& a, const PagedRequest& q, int r) {
    if (!a.causal) return q.keys;
    auto token = [&](int row) { return (int)FastDiv::div_by(a.by_g.m, a.by_g.s, (uint32_t)row); };
    const int64_t own = (int64_t)q.kv - token(q.R) + token(r) + 1;
    return own < 0 ? 0 : (own < q.keys ? (int)own : q.keys);
}

// V that is not finite, of a token that a row sees: that channel of the row's output is the sum of such values, an infinity or not a
// number, however small their probabilities.  The products do not keep to that: an infinity times a probability, factor or second
// term that is 0 or negative comes out as not a number.  But they never lose that there was something: where a row's output is not
// finite and its sum is a number, the kernels take the values of these channels (c .. c + 3, keys first .. last - 1 of a KV head)
// once more and by themselves.  It costs a look at the output (calls got 0 to 1.4 % longer), and a pass over V only then
// (with such a value in every page 64 tokens over 1000 to 32768 keys 379 -> 4620 us, 1024 rows over 16384 388 -> 1109).
template <class E>
__device__ __forceinline__ f32x4_t paged_four(const char* at) {
    if constexpr (std::is_same<E, float>::value) return *(const f32x4_t*)at;
    else {
        typedef E vec4 __attribute__((ext_vector_type(4)));
        return __builtin_convertvector(*(const vec4*)at, f32x4_t);
    }
}
__device__ __forceinline__ bool all_finite(f32x4_t v) {
    return __builtin_isfinite(v[0]) && __builtin_isfinite(v[1]) && __builtin_isfinite(v[2]) && __builtin_isfinite(v[3]);
}
// The sums of those values; 0 where there are none.  E: the storage type's elements.
template <class E, int D, class Args>
__device__ __forceinline__ f32x4_t paged_odd_values(Args& a, int b, int head, int first, int last, int c) {
    constexpr int ROWB = D * (int)sizeof(E);
    const int shift = a.pages.shift;
    const uint32_t n_pages = a.pages.n_pages;
    const int64_t page_bytes = a.pages.page_bytes;
    const char* const V = a.pages.V + ((int64_t)head << shift) * ROWB + c * (int)sizeof(E);
    const int32_t* const table = a.table + (int64_t)b * a.max_pages;
    f32x4_t sum = zero_vec<f32x4_t>();
#pragma unroll 1
    for (int key = first; key < last;) {
        const int in_page = key & ((1 << shift) - 1), left = last - key, to_end = (1 << shift) - in_page;
        const int n = left < to_end ? left : to_end;  // keys of this page
        const uint32_t id = (uint32_t)table[key >> shift];
        key += n;
        if (id >= n_pages) continue;
        const char* const page = V + (int64_t)id * page_bytes + in_page * ROWB;
        for (int i = 0; i < n; i += 8) {
            f32x4_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = paged_four<E>(page + (i + u < n ? i + u : n - 1) * ROWB);  // (twice the last changes no sum)
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += __builtin_isfinite(v[u][e]) ? 0.f : v[u][e];
        }
    }
    return sum;
}
// An output with its channels that hold such values.
__device__ __forceinline__ f32x4_t paged_with_odd(f32x4_t o, f32x4_t odd) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_isfinite(odd[e]) ? o[e] : odd[e];
    return o;
}

// What a row's scores (in units of a factor of two) are taken relative to, from their maximum: probabilities are 2^(x - reference), in
// the products and in the sum that they are divided by alike.  bf16: the maximum, probabilities of 1 and less.  fp16: 15 less, up to
// 2^15, as its second term ends at 2^-24.  Relative to a largest probability of 1 tens of thousands of small ones would lose bits, or
// all of them (131072 keys 17.5 below another came to nothing); so it ends at 2^-39 of the largest.  (The bits cost clock, and no instruction that
// could be measured: 1024 rows of 32 heads of 128 over 16384 keys 373 us without, 387.)  A maximum of 2^20 and more is taken as it is:
// its last place, by which an exponent may be off, has to stay far below the factor of 2 that fp16 has above 2^15.
template <class T>
__device__ __forceinline__ float paged_reference(float x) {
    if constexpr (std::is_same<T, F16>::value) return x - (__builtin_fabsf(x) < 1048576.0f ? 15.0f : 0.0f);
    return x;
}
// The log-sum-exp in those units, from the reference and the sum.
template <class T>
__device__ __forceinline__ float paged_log2_sum(float reference, float sum) {
    if constexpr (std::is_same<T, F16>::value) return (reference + 15.0f) + fast_log2(sum * 0x1p-15f);  // (the sum of either as small as may be)
    return reference + fast_log2(sum);
}

// 16-bit storage: workgroups for requests of many rows (a, unless `chunks` is 0) and for those of few (d, unless `decodes` is 0).
hipError_t launch_paged_16(const PagedArgs& a, int64_t chunks, const PagedArgs& d, int64_t decodes, int D, int dtype, hipStream_t stream);
hipError_t launch_paged_f32(const PagedArgs& a, int64_t grid, int D, hipStream_t stream);

}  // namespace fedrag
