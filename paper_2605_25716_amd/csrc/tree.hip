// A drafted step's trees: masks and positions from the nodes' parents (fedrag_tree_map), and the walk that verifies the drafts
// (fedrag_tree_verify).
#include "fedrag_device.h"
#include "fedrag_host.h"

namespace fedrag {

// ------------------------------------------------------------------------------------------------ map
// A wave per request takes its nodes 64 at a time, a node a lane.  mask[i] = bit i | mask[parent[i]], and so for the number of nodes on
// the way up: within the 64, each lane's way doubles in length from step to step, six at most, until it ends or leaves the 64; what
// lies above is the finished mask of the node where it left, read back.  Bound by its chain of trips (starts, parents, masks written):
// 2.0 us on the device for one request, 3.5 for 256 of up to 64 nodes; a call's other 5 us are the host's.
constexpr int kTreeMapThreads = 256;

struct TreeMapJob {
    int batch, n_rows, words;
    const int32_t *q_start, *kv_lens, *parents;
    uint64_t* mask;
    int32_t *positions, *flags;
};

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x < hi ? x : hi); }

FEDRAG_KERNEL __launch_bounds__(kTreeMapThreads) void tree_map_kernel(TreeMapJob j, int request_wgs) {
    const int lane = threadIdx.x % kWave;
    const int words = j.words;
    if ((int)blockIdx.x >= request_wgs) {  // padding rows
        const int64_t t = (int64_t)(blockIdx.x - request_wgs) * kTreeMapThreads + threadIdx.x;
        const int end = j.batch > 0 ? clamped(j.q_start[j.batch], 0, j.n_rows) : 0;
        if (t < end || t >= j.n_rows) return;
        for (int w = 0; w < words; ++w) j.mask[t * words + w] = 0;
        if (j.positions) j.positions[t] = -1;
        return;
    }
    const int64_t b = (int64_t)blockIdx.x * (kTreeMapThreads / kWave) + threadIdx.x / kWave;
    if (b >= j.batch) return;
    const int s = clamped(j.q_start[b], 0, j.n_rows), e = clamped(j.q_start[b + 1], 0, j.n_rows), kv = j.kv_lens[b];
    const int n = e > s ? e - s : 0, base = (kv < 0 ? 0 : kv) - n;
    int bad = n > (int64_t)64 * words ? FEDRAG_TREE_NO_WORDS : 0;
    for (int i0 = 0; i0 < n; i0 += kWave) {
        const int i = i0 + lane;
        int up = i < n ? j.parents[s + i] : -1;
        if (up < -1 || up >= i) {
            if (i < n) bad |= FEDRAG_TREE_BAD_PARENT;
            up = -1;
        }
        int inside = up - i0, outside = up;  // the next on the way up: a lane, or (inside < 0) a node before these, or none
        uint64_t bits = (uint64_t)1 << lane;
        int count = 1;
#pragma unroll 1
        for (int step = 0; step < 6 && __builtin_amdgcn_ballot_w64(inside >= 0) != 0; ++step) {
            const int from = inside < 0 ? lane : inside;
            const uint64_t more = __shfl((unsigned long long)bits, from);
            const int n_more = __shfl(count, from), in = __shfl(inside, from), out = __shfl(outside, from);
            if (inside >= 0) {
                bits |= more;
                count += n_more;
                inside = in;
                outside = out;
            }
        }
        if (i < n) {
            uint64_t* const mine = j.mask + (int64_t)(s + i) * words;
            const uint64_t* const above = j.mask + (int64_t)(s + outside) * words;  // (read only where there is such a node)
            for (int w = 0; w < words; ++w) mine[w] = w == i0 / kWave ? bits : (outside >= 0 && w < i0 / kWave ? above[w] : 0);
            if (j.positions) j.positions[s + i] = outside >= 0 ? j.positions[s + outside] + count : base + count - 1;
        }
        if (i0 + kWave < n) __threadfence_block();  // the next nodes read what this wave has stored
    }
    const uint64_t any1 = __builtin_amdgcn_ballot_w64((bad & 1) != 0), any2 = __builtin_amdgcn_ballot_w64((bad & 2) != 0);
    if (lane == 0) j.flags[b] = (any1 ? 1 : 0) | (any2 ? 2 : 0);
}

static int64_t tree_map_wgs(int batch, int64_t n_rows) {
    return ((int64_t)batch + kTreeMapThreads / kWave - 1) / (kTreeMapThreads / kWave) + (n_rows + kTreeMapThreads - 1) / kTreeMapThreads;
}
bool tree_map_fits(int batch, int64_t n_rows) { return tree_map_wgs(batch, n_rows) == 0 || grid_fits(tree_map_wgs(batch, n_rows), kTreeMapThreads); }

hipError_t launch_tree_map(int batch, int64_t n_rows, int words, const int32_t* q_start, const int32_t* kv_lens, const int32_t* parents,
                           uint64_t* mask, int32_t* positions, int32_t* flags, hipStream_t stream) {
    const int64_t wgs = tree_map_wgs(batch, n_rows);
    if (wgs == 0) return hipSuccess;
    const int requests = (batch + kTreeMapThreads / kWave - 1) / (kTreeMapThreads / kWave);
    hipLaunchKernelGGL(tree_map_kernel, dim3((unsigned)wgs), dim3(kTreeMapThreads), 0, stream,
                       TreeMapJob{batch, (int)n_rows, words, q_start, kv_lens, parents, mask, positions, flags}, requests);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ verify
// A request's walk is a chain: what a rejection leaves of the target's probabilities has to be summed before the next sibling is
// tried.  The walk itself costs two trips to memory for 64 nodes: a lane has a node, and fetches both of its probabilities ahead of the
// walk.  A sum is over whole numbers of units, so that neither the cut nor the form shows in the result.
//
// Rows of up to 128 KiB: one workgroup to a request, with the rows in its registers (tree_verify_whole_kernel, below).
// Longer ones: the launches are rounds.  In each, kPart tokens of the vocabulary are a workgroup's, for every request; it goes on with
// the request's walk by itself, from the state and the sums of the round before, until a sum over the vocabulary is needed, and adds up
// its part of it.  The state is the same in all of a request's workgroups, and the first one writes it down.  No workgroup waits for
// another.  What the last round finds unfinished, the request's first workgroup finishes alone.  Bound by reading the rows while all requests
// are at it (64 requests of 16 nodes and 128000 tokens in fp32, under the profiler: 15.4 and 11.2 us for the first two rounds, 66 MB at most each), later by a
// round's chain of a launch, state, nodes, part and sums, 7 to 9 us.  Without drafts' rows it is one sum, and 11.9 and 8.8 us.
constexpr int kVerifyThreads = 256;                  // (512: 28.5 us for 20.6 where 64 requests of 128000 tokens only draw)
constexpr int kPart = 4096;                          // tokens of a workgroup
constexpr int kEach = kPart / kVerifyThreads;        // and of a thread
constexpr int kMostParts = (1 << 20) / kPart;
static_assert(kMostParts <= kVerifyThreads, "a thread per part finds the part of a threshold");
constexpr double kUnits = 8796093022208.0;           // 2^43
constexpr uint64_t kUnit = (uint64_t)1 << 43;
constexpr uint64_t kMostUnits = (uint64_t)1 << 63;

enum : int { kVerifyDone = 0, kVerifyMass = 1, kVerifyDraw = 2 };
struct VerifyState {
    int need;          // what the sums of this round are for
    int node, last;    // where the walk is, and the child tried last (or the node)
    int n_kept;
    uint64_t taken;    // C
};

__device__ __forceinline__ float verify_value(float x) { return __builtin_amdgcn_fmed3f(x, 0.f, 1.f); }  // (not a number: 0, the least of the others)
__device__ __forceinline__ double verify_random(double u) { return fmin(fmax(u, 0.0), 0x1.fffffffffffffp-1); }
// r in units, and kUnitsBias: adding 2^52 rounds to a whole number, which is then the low bits.
constexpr uint64_t kUnitsBias = 0x4330000000000000;
__device__ __forceinline__ uint64_t verify_units_biased(double r) { return __builtin_bit_cast(uint64_t, __builtin_fma(r, kUnits, 0x1p52)); }
__device__ __forceinline__ uint64_t verify_units(double r) { return verify_units_biased(r) - kUnitsBias; }
__device__ __forceinline__ double verify_left_of(double p, double q, double taken) {
#pragma clang fp contract(off)
    const double product = taken * q;
    return fmax(p - product, 0.0);
}
__device__ __forceinline__ double verify_left(float p, float q, double taken) { return verify_left_of((double)p, (double)q, taken); }

template <class E, bool DRAFT>
struct Verify {
    const TreeVerifyJob& j;
    int b, s, n, parts;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint64_t (*scratch)[2];                              // LDS, a pair for each wave
    uint64_t (*row_sums)[kVerifyThreads / kWave];        // and a number for each part and wave
    bool target_only = false;  // weights are p's
    double next = 0.0;         // the request's u_next

    __device__ __forceinline__ const E* row_p(int node) const { return (const E*)j.target + (int64_t)(s + node) * j.target_stride; }
    __device__ __forceinline__ const E* row_q(int node) const { return (const E*)j.draft + (int64_t)(s + node) * j.draft_stride; }

    // ---- the nodes, 64 at a time
    int at;  // the first of them; < 0: none yet
    int parent, token;
    float p, q;
    double u;
    __device__ __forceinline__ void window(int i0) {
        if (i0 == at) return;
        at = i0;
        const int i = i0 + lane;
        parent = -1;
        token = -1;
        p = q = 0.f;
        u = 0.0;
        if (i < n) {
            parent = j.parents[s + i];
            token = j.tokens[s + i];
            u = verify_random(j.u[s + i]);
            if (parent >= i || token >= j.vocab) parent = -1;
            if (token < 0) parent = -1;
            if (parent >= 0) {
                p = verify_value((float)row_p(parent)[token]);
                if constexpr (DRAFT) q = verify_value((float)row_q(parent)[token]);
            }
        }
    }
    static __device__ __forceinline__ float lane_float(float x, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l)); }
    static __device__ __forceinline__ double lane_double(double x, int l) {
        return __builtin_bit_cast(double, of_lane(__builtin_bit_cast(uint64_t, x), l));
    }
    // Whether a child of `node` before child i has its token x.
    __device__ __forceinline__ bool repeated(int node, int i, int x) {
        bool found = __builtin_amdgcn_ballot_w64(parent == node && at + lane < i && token == x) != 0;
        for (int k = (node + 1) & ~(kWave - 1); k < at && !found; k += kWave) {
            const int c = k + lane;
            found = __builtin_amdgcn_ballot_w64(c > node && j.parents[s + c] == node && j.tokens[s + c] == x) != 0;
        }
        return found;
    }
    // f(child, token) for each child of the node up to child `last`, in order
    template <class F>
    __device__ __forceinline__ void rejected(const VerifyState& st, F f) {
        if (st.last <= st.node) return;
        for (int k = (st.node + 1) & ~(kWave - 1); k <= st.last; k += kWave) {
            window(k);
            uint64_t m = __builtin_amdgcn_ballot_w64(parent == st.node && k + lane <= st.last);
            for (; m; m &= m - 1) {
                const int l = __builtin_ctzll(m);
                f(k + l, __builtin_amdgcn_readlane(token, l));
            }
        }
    }

    // Goes on from `st`, whose M is known, until a sum is needed.  first: whether this workgroup writes what is accepted.
    __device__ __forceinline__ void walk(VerifyState& st, uint64_t mass, bool first) {
        bool known = true;
        st.need = kVerifyDraw;
        if (st.n_kept >= j.max_kept) return;
        int i0 = (st.last + 1) & ~(kWave - 1);
        while (i0 < n) {
            window(i0);
            const uint64_t m = __builtin_amdgcn_ballot_w64(parent == st.node && i0 + lane > st.last);
            if (m == 0) {
                i0 += kWave;
                continue;
            }
            if (!known) {
                st.need = kVerifyMass;
                return;
            }
            const int l = __builtin_ctzll(m), child = i0 + l;
            const float pc = lane_float(p, l);
            const double uc = lane_double(u, l);
            bool yes;
            uint64_t gone = 0;
            if constexpr (DRAFT) {
#pragma clang fp contract(off)
                const float qc = lane_float(q, l);
                const double low = uc * (double)qc * (double)mass;
                yes = low < verify_left(pc, qc, (double)st.taken / kUnits) * kUnits;
            } else {
                const double left = repeated(st.node, child, __builtin_amdgcn_readlane(token, l)) ? 0.0 : (double)pc;
                yes = uc * (double)mass < left * kUnits;
                gone = verify_units(left);
            }
            st.last = child;
            if (yes) {
                st.node = child;
                if (first && threadIdx.x == 0) j.kept[b * j.max_kept + st.n_kept] = child;
                ++st.n_kept;
                st.taken = 0;
                mass = kUnit;
                if (st.n_kept >= j.max_kept) return;
            } else if constexpr (DRAFT) {
                st.taken = mass < kMostUnits - st.taken ? st.taken + mass : kMostUnits;
                known = false;
            } else {
                mass = mass > gone ? mass - gone : 0;
            }
        }
    }

    // ---- sums over the vocabulary.  Where nothing was rejected, r is p and q is not read.
    __device__ __forceinline__ bool with_draft(const VerifyState& st) const { return DRAFT && st.taken != 0 && !target_only; }
    // A token's weight and kUnitsBias.  WITH: 0 r is p, 1 C is one (no product to round), 2 any C.
    template <int WITH>
    static __device__ __forceinline__ uint64_t weight(float pv, float qv, double taken) {
        const float x = verify_value(pv);
        if constexpr (WITH == 0) return verify_units_biased((double)x);
        if constexpr (WITH == 1) return verify_units_biased(fmax((double)x - (double)verify_value(qv), 0.0));
        return verify_units_biased(verify_left(x, verify_value(qv), taken));
    }
    // This thread's share of the sums of N parts; every token of a part is some thread's.
    template <int WITH, int N>
    __device__ __forceinline__ void part_sums_of(const E* pr, const E* qr, double taken, int part, uint64_t (&sum)[N]) const {
        const int begin = part * kPart, end = begin + N * kPart < j.vocab ? begin + N * kPart : j.vocab;
        constexpr int VEC = 16 / (int)sizeof(E);
        typedef E vec __attribute__((ext_vector_type(VEC)));
        typedef vec vec_any __attribute__((aligned(sizeof(E))));
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0;
        if (end - begin == N * kPart) {
            vec pv[N][kEach / VEC], qv[N][kEach / VEC];
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < kEach / VEC; ++i) {
                    const int at = begin + k * kPart + (i * kVerifyThreads + (int)threadIdx.x) * VEC;
                    pv[k][i] = *(const vec_any*)(pr + at);
                    if constexpr (WITH != 0) qv[k][i] = *(const vec_any*)(qr + at);
                }
#pragma unroll
            for (int k = 0; k < N; ++k) {
#pragma unroll
                for (int i = 0; i < kEach / VEC; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[k] += weight<WITH>((float)pv[k][i][e], WITH ? (float)qv[k][i][e] : 0.f, taken);
                sum[k] -= kEach * kUnitsBias;
            }
            return;
        }
        // (the row's end, by single values; what is not there has no weight)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            E pv[kEach], qv[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int v = begin + k * kPart + i * kVerifyThreads + (int)threadIdx.x;
                pv[i] = v < end ? pr[v] : (E)0.f;
                if constexpr (WITH != 0) qv[i] = v < end ? qr[v] : (E)0.f;
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) sum[k] += weight<WITH>((float)pv[i], WITH ? (float)qv[i] : 0.f, taken);
            sum[k] -= kEach * kUnitsBias;
        }
    }
    template <int N>
    __device__ __forceinline__ void part_sums(const VerifyState& st, int part, uint64_t (&sum)[N]) const {
        const E* const pr = row_p(st.node);
        if constexpr (DRAFT) {
            if (with_draft(st)) {
                if (N == 1 && st.taken == kUnit) return part_sums_of<1>(pr, row_q(st.node), 1.0, part, sum);
                return part_sums_of<2>(pr, row_q(st.node), (double)st.taken / kUnits, part, sum);
            }
        }
        return part_sums_of<0>(pr, pr, 0.0, part, sum);
    }
    static __device__ __forceinline__ uint64_t of_lane(uint64_t x, int l) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l);
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | lo;
    }
    // Over a wave's lanes.
    static __device__ __forceinline__ uint64_t wave_add(uint64_t x) {
        x += dpp_move64<0xb1>(x);   // the neighbour, in pairs
        x += dpp_move64<0x4e>(x);   // the other pair of four
        x += dpp_move64<0x141>(x);  // the other four of eight
        x += dpp_move64<0x140>(x);  // the other eight of sixteen
        return of_lane(x, 0) + of_lane(x, 16) + of_lane(x, 32) + of_lane(x, 48);
    }
    __device__ __forceinline__ uint64_t total(uint64_t x) const {
        x = wave_add(x);
        __syncthreads();
        if (lane == 0) scratch[wave][0] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < kVerifyThreads / kWave; ++w) x += scratch[w][0];
        return x;
    }
    // A part's sum, in every thread.
    __device__ __forceinline__ uint64_t part_total(const VerifyState& st, int part) {
        uint64_t sum[1];
        part_sums(st, part, sum);
        uint64_t x = total(sum[0]);
        if constexpr (!DRAFT) {
            if (!target_only)
                rejected(st, [&](int child, int v) {
                    if (v / kPart == part && !repeated(st.node, child, v)) x -= verify_units((double)verify_value((float)row_p(st.node)[v]));
                });
        }
        return x;
    }
    // Of numbers x, one a thread: the first thread whose inclusive sum is above `t` (kVerifyThreads: none), and the sum before it.
    __device__ __forceinline__ int first_beyond(uint64_t x, uint64_t t, uint64_t* before) const {
        uint64_t to = x;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const uint64_t y = __shfl_up((unsigned long long)to, o);
            if (lane >= o) to += y;
        }
        __syncthreads();
        if (lane == kWave - 1) scratch[wave][0] = to;
        __syncthreads();
        uint64_t base = 0;
        int found = kVerifyThreads;
        *before = 0;
#pragma unroll
        for (int w = 0; w < kVerifyThreads / kWave; ++w) {
            const uint64_t sum = scratch[w][0];
            if (found == kVerifyThreads && base + sum > t) {
                found = w;
                *before = base;
            }
            base += sum;
        }
        if (found == kVerifyThreads) return found;
        const int in = found;
        __syncthreads();
        if (wave == in) {
            const int l = __builtin_popcountll(__builtin_amdgcn_ballot_w64(*before + to <= t));
            if (lane == l) {
                scratch[0][0] = *before + to - x;
                scratch[0][1] = (uint64_t)l;
            }
        }
        __syncthreads();
        *before = scratch[0][0];
        return in * kWave + (int)scratch[0][1];
    }
    // The sums of all parts, a thread each, by this workgroup alone.
    __device__ __forceinline__ uint64_t all_parts(const VerifyState& st) {
        constexpr int N = 2;  // parts on their way at once (one: 49 us where one of two requests needs a sum more than there are rounds, so 39)
        __syncthreads();
        for (int i = 0; i < parts; i += N) {
            uint64_t sum[N];
            part_sums(st, i, sum);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const uint64_t x = wave_add(sum[k]);
                if (lane == 0 && i + k < parts) row_sums[i + k][wave] = x;
            }
        }
        __syncthreads();
        uint64_t mine = 0;
        if ((int)threadIdx.x < parts) {
#pragma unroll
            for (int w = 0; w < kVerifyThreads / kWave; ++w) mine += row_sums[threadIdx.x][w];
        }
        if constexpr (!DRAFT) {
            if (!target_only)
                rejected(st, [&](int child, int v) {
                    if (!repeated(st.node, child, v) && v / kPart == (int)threadIdx.x) mine -= verify_units((double)verify_value((float)row_p(st.node)[v]));
                });
        }
        return mine;
    }
    // The token, from the sums of the parts, a thread each.  only: the workgroup's part, or -1: whichever it is.
    __device__ __forceinline__ void draw(const VerifyState& st, uint64_t mine, int only) {
        uint64_t all = total(mine);
        if (all == 0) {  // nothing is left of r: p, by one workgroup
            if (only > 0) return;
            only = -1;
            target_only = true;
            mine = all_parts(st);
            all = total(mine);
            if (all == 0) {
                if (threadIdx.x == 0) j.next_token[b] = -1;
                return;
            }
        }
        const double x = next * (double)all;
        uint64_t t = (uint64_t)x;
        t = t < all ? t : all - 1;
        uint64_t before;
        const int part = first_beyond(mine, t, &before);
        if (only >= 0 && part != only) return;
        const E* const pr = row_p(st.node);
        const E* const qr = DRAFT ? row_q(st.node) : pr;
        const bool with = with_draft(st);
        const double taken = with ? (double)st.taken / kUnits : 0.0;  // (of p with q = 0: p)
        const int v0 = part * kPart + (int)threadIdx.x * kEach;
        uint64_t w[kEach], here = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            w[e] = v0 + e < j.vocab ? weight<2>((float)pr[v0 + e], with ? (float)qr[v0 + e] : 0.f, taken) - kUnitsBias : 0;
        if constexpr (!DRAFT) {
            if (!target_only)
                rejected(st, [&](int, int v) {
#pragma unroll
                    for (int e = 0; e < kEach; ++e) w[e] = v0 + e == v ? 0 : w[e];
                });
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) here += w[e];
        const uint64_t t_part = t - before;
        uint64_t in_part;
        const int thread = first_beyond(here, t_part, &in_part);
        if ((int)threadIdx.x == thread) {
            int v = v0;
            uint64_t to = in_part;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                to += w[e];
                if (to <= t_part) v = v0 + e + 1;
            }
            j.next_token[b] = v;
        }
    }
};

template <class E, bool DRAFT>
FEDRAG_KERNEL __launch_bounds__(kVerifyThreads) void tree_verify_kernel(TreeVerifyJob j, int parts, int round, int last_round) {
    __shared__ uint64_t scratch[kVerifyThreads / kWave][2], row_sums[kMostParts][kVerifyThreads / kWave];
    const int part = (int)blockIdx.x, b = (int)blockIdx.y;
    VerifyState* const states = (VerifyState*)j.workspace;  // [2][batch], then the sums [2][batch][parts]
    uint64_t* const sums = (uint64_t*)(states + 2 * (int64_t)j.batch);
    const int now = round & 1, before = 1 - now;
    const int s = clamped(j.q_start[b], 0, j.n_rows), e = clamped(j.q_start[b + 1], 0, j.n_rows);
    Verify<E, DRAFT> v{j, b, s, e > s ? e - s : 0, parts};
    v.scratch = scratch;
    v.row_sums = row_sums;
    v.at = -1;
    VerifyState st{kVerifyDone, 0, 0, 1, 0};
    // (what the round may need of the one before, in one trip to memory)
    uint64_t own_sum = 0;
    v.next = verify_random(j.u_next[b]);
    if (round > 0) {
        st = states[(int64_t)before * j.batch + b];
        if ((int)threadIdx.x < parts) own_sum = sums[((int64_t)before * j.batch + b) * parts + threadIdx.x];
        pin_here(own_sum);
    }
    if (round == 0) {
        if (v.n > 0) {
            if (part == 0 && threadIdx.x == 0) j.kept[b * j.max_kept] = 0;
            v.walk(st, kUnit, part == 0);
        } else if (part == 0) {
            for (int64_t i = threadIdx.x; i < j.max_kept; i += kVerifyThreads) j.kept[b * j.max_kept + i] = 0;
            if (threadIdx.x == 0) {
                j.n_kept[b] = 0;
                j.next_token[b] = -1;
            }
        }
    } else {
        if (st.need == kVerifyDraw) {
            v.draw(st, own_sum, part);
            st.need = kVerifyDone;
        } else if (st.need == kVerifyMass) {
            v.walk(st, v.total(own_sum), part == 0);
        }
    }
    auto finish_kept = [&]() {  // the path is complete
        if (part != 0) return;
        for (int64_t i = st.n_kept + threadIdx.x; i < j.max_kept; i += kVerifyThreads) j.kept[b * j.max_kept + i] = 0;
        if (threadIdx.x == 0) j.n_kept[b] = st.n_kept;
    };
    if (round < last_round) {
        if (part == 0 && threadIdx.x == 0) states[(int64_t)now * j.batch + b] = st;
        if (st.need == kVerifyDone) return;
        if (st.need == kVerifyDraw) finish_kept();
        const uint64_t sum = v.part_total(st, part);
        if (threadIdx.x == 0) sums[((int64_t)now * j.batch + b) * parts + part] = sum;
        return;
    }
    if (st.need == kVerifyDone || part != 0) return;
    uint64_t mine = v.all_parts(st);
    while (st.need == kVerifyMass) {  // (each time around a child has been tried)
        v.walk(st, v.total(mine), true);
        mine = v.all_parts(st);
    }
    finish_kept();
    v.draw(st, mine, -1);
}

// Rows of up to 128 KiB (32768 tokens in fp32, 65536 in 16 bits): one workgroup to a request, whose threads have the row of p and that of q
// in registers, so that a sum after the first at a node costs no trip to memory, and one launch does.  Bound by that workgroup's 64-bit
// arithmetic (8 instructions a token and sum) and by what it can read (256 KB in some 4 us): 13.3 us on the device for 8 nodes of 32000 tokens in
// fp32, 6.0 for 64 tokens, both under the profiler.
// Against rounds it is ahead everywhere (calls, without it): 1 request of 32000 tokens 11.7 us (17.4 by rounds), 64 23 (35), 200 27 (60), 1000 of 4 nodes 59
// (104); 128 of 16000 in bf16 21 (50); 8 of 65001 in fp16 26 (31); without drafts 1000 of 32000 45 (64).
constexpr int kWholeThreads = 1024;
constexpr int kWholeWaves = kWholeThreads / kWave;
constexpr int kWholeSteps = 8;  // 16-byte pieces of a row in a thread's registers: 32 of its 128 registers, and as many for q
constexpr int kWholeBytes = kWholeThreads * kWholeSteps * 16;
static_assert(kWholeWaves * kWholeSteps == 2 * kWave, "two sums a lane");

template <class E, bool DRAFT>
FEDRAG_KERNEL __launch_bounds__(kWholeThreads) void tree_verify_whole_kernel(TreeVerifyJob j) {
    constexpr int VEC = 16 / (int)sizeof(E);
    constexpr int kStep = kWholeThreads * VEC;  // tokens of a step: a wave's in their order, the waves' in theirs
    typedef E vec __attribute__((ext_vector_type(VEC)));
    typedef vec vec_any __attribute__((aligned(sizeof(E))));
    __shared__ __attribute__((aligned(16))) uint64_t sums[2][kWholeSteps * kWholeWaves][kWave / 16];
    __shared__ VerifyState walked;
    const int b = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave, vocab = j.vocab;
    const int s = clamped(j.q_start[b], 0, j.n_rows), e = clamped(j.q_start[b + 1], 0, j.n_rows);
    Verify<E, DRAFT> v{j, b, s, e > s ? e - s : 0, 0};
    v.at = -1;
    v.next = verify_random(j.u_next[b]);
    VerifyState st{kVerifyDone, 0, 0, 1, 0};
    if (v.n == 0) {
        for (int64_t i = tid; i < j.max_kept; i += kWholeThreads) j.kept[b * j.max_kept + i] = 0;
        if (tid == 0) {
            j.n_kept[b] = 0;
            j.next_token[b] = -1;
        }
        return;
    }
    if (tid == 0) j.kept[b * j.max_kept] = 0;
    // A thread's piece of a step: VEC tokens from `own` on.  The row's last piece is read so that it ends with the row, and what
    // belongs to the piece before is 0 in it.
    vec p[kWholeSteps], q[kWholeSteps];
    auto own = [&](int i) { return i * kStep + tid * VEC; };
    auto any = [&](int i) { return i * kStep + wave * kWave * VEC < vocab; };  // (of the wave's)
    auto from = [&](int i) { return own(i) + VEC <= vocab ? own(i) : vocab - VEC; };
    auto load = [&](const E* row, vec (&x)[kWholeSteps]) __attribute__((always_inline)) {
        uint32_t first = (uint32_t)(tid * VEC);
        pin_here(first);  // (the steps' places are not kept)
#pragma unroll
        for (int i = 0; i < kWholeSteps; ++i) {
            const uint32_t at = first + i * kStep, last = (uint32_t)(vocab - VEC);
            x[i] = zero_vec<vec>();
            if (at < (uint32_t)vocab) x[i] = *(const vec_any*)(row + (at < last ? at : last));
        }
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int i = 0; i < kWholeSteps; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[i][k] = verify_value(x[i][k]);
        }
    };
    double taken = 0.0;
    auto value = [&](E x) __attribute__((always_inline)) { return sizeof(E) == 4 ? (float)x : verify_value((float)x); };
    auto weight = [&](int i, int k) __attribute__((always_inline)) {
        const double x = (double)value(p[i][k]);
        return verify_units(DRAFT ? verify_left_of(x, (double)value(q[i][k]), taken) : x);
    };
    auto step_sum = [&](int i) __attribute__((always_inline)) {
        uint64_t x = 0;
        if (any(i)) {
            pin_here(p[i]);  // (one step's values in 64 bits at a time)
            if constexpr (DRAFT) pin_here(q[i]);
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                x += weight(i, k);
                if (k % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        return x;
    };
    // Sums by step and wave, which is the tokens' order, until it is the next token that they are for.
    int node = -1;  // whose p is here
    bool target_only = false;
    uint64_t two[2], all = kUnit;
    for (int turn = 0;; turn ^= 1) {
        if (!target_only) {
            if constexpr (DRAFT) {  // by one wave (without drafts' rows all need to know the children that were rejected)
                if (wave == 0) {
                    v.walk(st, all, true);
                    if (lane == 0) walked = st;
                }
                __syncthreads();
                st = walked;
            } else {
                v.walk(st, all, true);
            }
            if (st.need == kVerifyDraw) {
                for (int64_t i = st.n_kept + tid; i < j.max_kept; i += kWholeThreads) j.kept[b * j.max_kept + i] = 0;
                if (tid == 0) j.n_kept[b] = st.n_kept;
            }
        }
        if (node != st.node || target_only) {
            const int here = __builtin_amdgcn_readfirstlane(st.node);
            load(v.row_p(here), p);
            const int end = (vocab - 1) / kStep;  // the step of the row's last piece
            vec cut = zero_vec<vec>();
#pragma unroll
            for (int i = 0; i < kWholeSteps; ++i) cut = i == end ? p[i] : cut;
            if (own(end) + VEC > vocab && own(end) < vocab) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) cut[k] = from(end) + k < own(end) ? (E)0.f : cut[k];
            }
#pragma unroll
            for (int i = 0; i < kWholeSteps; ++i) p[i] = i == end ? cut : p[i];
            if constexpr (DRAFT) {
                // (where nothing was rejected at the node it is not read: of p with q = 0)
#pragma unroll
                for (int i = 0; i < kWholeSteps; ++i) q[i] = zero_vec<vec>();
                if (st.taken != 0 && !target_only) load(v.row_q(here), q);
            }
            node = st.node;
        }
        taken = target_only ? 0.0 : (double)st.taken / kUnits;
        if constexpr (!DRAFT) {
            if (!target_only)
                v.rejected(st, [&](int, int x) {
                    const int i = x / kStep, k = x - (x % kStep / VEC == tid ? from(i) : x + 1);
#pragma unroll
                    for (int i1 = 0; i1 < kWholeSteps; ++i1) {
                        if (k >= 0 && i1 == i) {
#pragma unroll
                            for (int k1 = 0; k1 < VEC; ++k1) p[i1][k1] = k1 == k ? (E)0.f : p[i1][k1];
                        }
                    }
                });
        }
        // Over the lanes: of each two one takes the first four steps, and of each four one takes two of these; then over the fours of 16.
        constexpr int kHalf = kWholeSteps / 2;
        uint64_t x[kHalf];
        auto mine = [&](uint64_t lower, uint64_t upper, bool up, auto move) __attribute__((always_inline)) {
            return (up ? upper : lower) + move(up ? lower : upper);
        };
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            const uint64_t lower = step_sum(i), upper = step_sum(kHalf + i);
            x[i] = mine(lower, upper, lane & 1, dpp_move64<0xb1>);
            pin_here(x[i]);
        }
        if (st.need == kVerifyMass) {
            uint64_t sum = x[0] + x[1] + x[2] + x[3];
            sum = Verify<E, DRAFT>::wave_add(sum);
            if (lane == 0) sums[turn][wave][0] = sum;
            __syncthreads();
            all = Verify<E, DRAFT>::wave_add(lane < kWholeWaves ? sums[turn][lane][0] : 0);
            continue;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = mine(x[i], x[2 + i], lane & 2, dpp_move64<0x4e>);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[i] += dpp_move64<0x128>(x[i]);
            x[i] += dpp_move64<0x124>(x[i]);
            if (lane % 16 < 4) sums[turn][((lane & 1) * 4 + (lane & 2) + i) * kWholeWaves + wave][lane / 16] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto& s4 = sums[turn][2 * lane + i];
            two[i] = s4[0] + s4[1] + s4[2] + s4[3];
        }
        all = Verify<E, DRAFT>::wave_add(two[0] + two[1]);
        if (all != 0 || target_only) break;
        target_only = true;  // nothing is left of r: p
    }
    if (all == 0) {
        if (tid == 0) j.next_token[b] = -1;
        return;
    }
    uint64_t t = (uint64_t)(v.next * (double)all);
    t = t < all ? t : all - 1;
    auto up_to = [&](uint64_t x) {  // inclusive, over lanes
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const uint64_t y = __shfl_up((unsigned long long)x, o);
            if (lane >= o) x += y;
        }
        return x;
    };
    const uint64_t to = up_to(two[0] + two[1]);
    const int l = __builtin_popcountll(__builtin_amdgcn_ballot_w64(to <= t));
    const bool second = t >= to - two[1];
    const int found = __builtin_amdgcn_readlane(2 * lane + (second ? 1 : 0), l);
    const uint64_t before = __shfl((unsigned long long)(to - two[1] - (second ? 0 : two[0])), l);
    if (found % kWholeWaves != wave) return;
    const int step = found / kWholeWaves;
#pragma unroll
    for (int i = 1; i < kWholeSteps; ++i)
        if (i == step) {
            p[0] = p[i];
            if constexpr (DRAFT) q[0] = q[i];
        }
    uint64_t w[VEC], mine = 0;
#pragma unroll
    for (int k = 0; k < VEC; ++k) mine += w[k] = weight(0, k);
    const uint64_t sum = before + up_to(mine);
    if (lane != __builtin_popcountll(__builtin_amdgcn_ballot_w64(sum <= t))) return;
    uint64_t x = sum - mine;
    int token = from(step);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        x += w[k];
        token += x <= t ? 1 : 0;
    }
    j.next_token[b] = token;
}

static int verify_parts(int vocab) { return (vocab + kPart - 1) / kPart; }
// Rows that one workgroup has in registers, none shorter than a load of a lane.
static bool verify_whole(int vocab, int dtype) {
    const size_t bytes = (size_t)vocab * (dtype == FEDRAG_F32 ? 4 : 2);
    return bytes >= 16 && bytes <= kWholeBytes;
}
size_t tree_verify_workspace(int batch, int vocab, int dtype) {
    if (verify_whole(vocab, dtype)) return 0;
    return 2 * (size_t)batch * (sizeof(VerifyState) + (size_t)verify_parts(vocab) * sizeof(uint64_t));
}

template <class E>
static hipError_t launch_tree_verify_t(const TreeVerifyJob& job, hipStream_t stream) {
    if (verify_whole(job.vocab, job.dtype)) {
        hipLaunchKernelGGL((job.draft ? tree_verify_whole_kernel<E, true> : tree_verify_whole_kernel<E, false>), dim3((unsigned)job.batch),
                           dim3(kWholeThreads), 0, stream, job);
        return hipGetLastError();
    }
    const int parts = verify_parts(job.vocab);
    // Rounds after the first: without drafts one, to draw; with drafts as many as most requests need, and of many requests some need more
    // (1 request of 32000 tokens, when it went by rounds, 2: 18.7 us, 3: 21.1; 16 requests 3: 25.8, 2: 35.5; 64 of 16 nodes and 128000 tokens
    // 4: 47.9, 3: 69.6, 5: 51).
    const int last = !job.draft ? 1 : job.batch < 4 ? 2 : job.batch < 32 ? 3 : 4;
    const auto kernel = job.draft ? tree_verify_kernel<E, true> : tree_verify_kernel<E, false>;
    for (int round = 0; round <= last; ++round)
        hipLaunchKernelGGL(kernel, dim3((unsigned)parts, (unsigned)job.batch), dim3(kVerifyThreads), 0, stream, job, parts, round, last);
    return hipGetLastError();
}
hipError_t launch_tree_verify(const TreeVerifyJob& job, hipStream_t stream) {
    switch (job.dtype) {
        case FEDRAG_F32: return launch_tree_verify_t<float>(job, stream);
        case FEDRAG_BF16: return launch_tree_verify_t<__bf16>(job, stream);
        default: return launch_tree_verify_t<_Float16>(job, stream);
    }
}

}  // namespace fedrag
