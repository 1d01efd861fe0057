// Log probabilities of given labels under the soft-max of all scores, its entropy and its top labels; and the gradient of the first two.
//   logp_v = (x_v - m) / T - log S,  S = sum exp((x_v - m) / T),  H = log S - sum exp((x_v - m) / T) (x_v - m) / T / S
//   dX_v = (sum of dlogp over v's places in the list - p_v (G + dH (logp_v + H))) / T,  G the sum of dlogp
#include "xc_softmax.h"

namespace xc {

constexpr int kTopKeys = 1024;           // candidates that a workgroup holds

struct LogprobArgs {
    const void* X;
    const int32_t* labels;
    float *logp, *entropy, *norm;
    int32_t* top;
    float* top_logp;
    float4* parts;                       // [B][segments]: sums of a segment
    uint64_t* keys;                      // [B][segments][k]: its best labels, best first; ~0 behind them
    int64_t B, V, ld, segments, length;
    float T, c;
    int n, k, blocks;
};

struct Norm { float m, ls; };            // largest score; log of the sum (-inf: no label is there)
__device__ __forceinline__ Norm norm_of(const Sums& s) { return Norm{s.m, logf(s.s)}; }
__device__ __forceinline__ float logp_of(float x, const Norm& z, float T) { return z.ls == kNone ? kNone : (x - z.m) / T - z.ls; }

// What a row's sums answer: norm, entropy, given labels.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t b, const Sums& s) {
    const Norm z = norm_of(s);
    if (threadIdx.x == 0) {
        a.norm[2 * b] = z.m;
        a.norm[2 * b + 1] = z.ls;
        a.entropy[b] = z.ls == kNone ? 0.0f : z.ls - 0.6931471805599453f * (s.h / s.s);
    }
    for (int j = threadIdx.x; j < a.n; j += static_cast<int>(blockDim.x)) {
        const int32_t v = a.labels[b * a.n + j];
        a.logp[b * a.n + j] = v >= 0 && v < a.V ? logp_of(Elem<T>::get(static_cast<const T*>(a.X) + b * a.ld + v), z, a.T) : 0.0f;
    }
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t b, int rank, uint64_t key, const Norm& z) {
    const bool there = key != kKeySentinel;
    a.top[b * a.k + rank] = there ? key_id(key) : -1;
    a.top_logp[b * a.k + rank] = there ? logp_of(key_score(key), z, a.T) : kNone;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t larger_of_lanes(uint32_t x) {
    const uint32_t t = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, ROWS, 0xf, false));
    return t > x ? t : x;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = larger_of_lanes<0x111, 0xf>(v);                      // row_shr 1, 2, 4, 8
    v = larger_of_lanes<0x112, 0xf>(v);
    v = larger_of_lanes<0x114, 0xf>(v);
    v = larger_of_lanes<0x118, 0xf>(v);
    v = larger_of_lanes<0x142, 0xa>(v);                      // row_bcast 15, 31
    v = larger_of_lanes<0x143, 0xc>(v);
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), kWave - 1));
}

constexpr uint32_t kLowest = 0x00800000u;        // ordered image of the lowest number above -inf

// Of n values, 64 G at most (ordered images of scores; value(i) reads one): one that at least k of them reach, if as many lie above -inf, and
// that few others do; found by halving the range, by one wave, which holds them (read from LDS every time: 1024 x 131072 bf16 with 128 labels
// 73 us against 67).  Equal values can make these many.
template <int G, typename V>
__device__ __forceinline__ uint32_t reached_by(int n, int k, V value) {
    uint32_t lo = ~0u, hi = 0u, o[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        o[g] = 0u;
        if (g * kWave >= n) continue;                        // uniform
        const int i = g * kWave + lane_id();
        if (i < n) {
            o[g] = value(i);
            lo = o[g] < lo ? o[g] : lo;
            hi = o[g] > hi ? o[g] : hi;
        }
    }
    lo = ~wave_max_u32(~lo);
    hi = wave_max_u32(hi) + 1u;
    auto count = [&](uint32_t t) __attribute__((always_inline)) {
        int c = 0;
#pragma unroll
        for (int g = 0; g < G; ++g) if (g * kWave < n) c += __popcll(__ballot(o[g] >= t));           // (t is never 0)
        return c;
    };
    if (lo < kLowest) lo = kLowest;
    bool enough = false;                                     // (does `lo` leave more than k?)
    while (hi > lo && hi - lo > 1u) {
        const uint32_t mid = enough ? lo + (hi - lo) / 2u : lo;
        const int c = count(mid);
        if (!enough) {
            if (c <= k) return lo;
            enough = true;
        } else if (c >= k) {
            lo = mid;
            if (c <= k + k / 4 + 3) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// How many of n keys are better than this one (the keys behind them, up to a multiple of four, are ~0); of LANES neighbouring lanes with the
// same key each counts its share of them.
template <int LANES = 1>
__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t* keys, int n) {
    static_assert(LANES == 1 || LANES == 4, "");
    int rank = 0;
#pragma unroll 2
    for (int j = LANES == 1 ? 0 : (lane_id() & (LANES - 1)) * 4; j < n; j += 4 * LANES) {
        uint64_t k[4];
        __builtin_memcpy(k, __builtin_assume_aligned(keys + j, 16), 32);
        rank += (k[0] < key ? 1 : 0) + (k[1] < key ? 1 : 0) + (k[2] < key ? 1 : 0) + (k[3] < key ? 1 : 0);
    }
    if constexpr (LANES == 4) {
        rank += __builtin_amdgcn_update_dpp(0, rank, 0xB1, 0xf, 0xf, false);           // quad_perm 1 0 3 2
        rank += __builtin_amdgcn_update_dpp(0, rank, 0x4E, 0xf, 0xf, false);           // quad_perm 2 3 0 1
    }
    return rank;
}
// n places of a counter in LDS to each lane.
__device__ __forceinline__ int take_room(int* counter, int n) {
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) int*)counter));
    int before;
    asm volatile("ds_add_rtn_u32 %0, %1, %2\n\ts_waitcnt lgkmcnt(0)" : "=&v"(before) : "v"(at), "v"(n) : "memory");
    return before;
}
// Behind n keys, for the function above; before a barrier.
__device__ __forceinline__ void end_keys(uint64_t* keys, int n) {
    if (threadIdx.x < 3) keys[n + threadIdx.x] = kKeySentinel;
}

// Of a stretch of blocks in which more labels score `least` or more than a workgroup holds (`room` or more of them): the k best, or up to `room`
// that reach a score which k of them reach; to `keys`, kept[0] of them.  That is where many scores are equal, or grow along the row.  The stretch
// is read again a few times, so that this takes few registers from what always runs.  `least`, or a score that k of the threads' largest ones
// reach, is mostly the answer, or more than k labels share it: of equal labels the first ones are taken in their order, by counting.  Else the
// range above it is halved, 32 times at most.  (2048 x 131072 bf16 with 64 top labels: 112 to 116 us for normal scores, 128 to 141 for rows of one
// value, of three, or masked with the type's lowest value but for three labels, where halving keys of score and label and looking at every
// stretch took 18 ms; 507 for rows that grow from end to end.)  `range`, `counts` and `largest` [kRowThreads] are free again after the caller's next barrier.
template <typename T>
__device__ __forceinline__ void best_of_stretch(const PiecedRow<T>& row, int first, int end, int edge, int k, int room, uint32_t least, uint32_t* largest,
                                                uint32_t (&range)[2], int2 (&counts)[2][kRowWaves], uint64_t* keys, int* kept) {
    constexpr int N = PiecedRow<T>::N;
    const int wave = threadIdx.x >> 6;
    uint32_t lo = least, hi = 0u, mid = least;               // k labels or more reach lo, fewer reach hi (0: not known yet)
    int turn = 0, want = 0;                                  // (one buffer of the counts is read while the other is written)
    bool done = false;
    if (threadIdx.x == 0) *kept = 0;
    for (;;) {
        const float t = ordered_to_float(mid), next = ordered_to_float(mid + 1u);            // (behind +infinity: not a number, which nothing reaches)
        float most = kNone;
        int n = 0, above = 0, taken = 0;
        // the row's edges before its pieces, the pieces, the edges behind them
#pragma unroll 1
        for (int at0 = first - kRowThreads;; at0 += kRowThreads) {
            const int at = at0 + static_cast<int>(threadIdx.x);
            const bool inside = at0 >= first && at0 < end;   // uniform
            int id = edge;
            uint4 v = Elem<T>::none();
            float x0 = kNone;
            if (inside) {
                id = static_cast<int>(row.first(at));
                if (at < end) v = row.template load<false>(at);
                x0 = Elem<T>::value(v, 0);
            } else if (edge >= 0 && (at0 < first) == (edge < row.head)) {
                x0 = Elem<T>::get(row.p + edge);
            }
            uint32_t which = x0 >= t ? 1u : 0u, over = x0 >= next ? 1u : 0u;
            most = fmaxf(most, x0);
#pragma unroll
            for (int e = 1; e < N; ++e) {
                const float x = Elem<T>::value(v, e);
                which |= x >= t ? 1u << e : 0u;
                over |= x >= next ? 1u << e : 0u;
                most = fmaxf(most, x);
            }
            n += __popc(which);
            above += __popc(over);
            if (done) {                                      // uniform, as all that follows but the labels themselves
                int at_tie = want;                           // of the thread's labels that score t, the first one's place among all
                if (taken < want) {
                    const int own = __popc(which & ~over), upto = wave_incl_scan(own);
                    turn ^= 1;
                    if (lane_id() == kWave - 1) counts[turn][wave].x = upto;
                    __syncthreads();
                    at_tie = taken + upto - own;
#pragma unroll
                    for (int w = 0; w < kRowWaves; ++w) {
                        const int c = counts[turn][w].x;
                        if (w < wave) at_tie += c;
                        taken += c;
                    }
                }
                if (want == 0) which = over;
#pragma unroll 1
                for (; which != 0u; which &= which - 1u) {
                    const int e = __ffs(static_cast<int>(which)) - 1;
                    const float x = Elem<T>::get(row.p + id + e);
                    if (x >= next || at_tie++ < want) keys[atomicAdd(kept, 1)] = make_key(x + 0.0f, id + e);
                }
            }
            if (at0 >= end) break;
        }
        if (done) return;
        turn ^= 1;
#pragma unroll
        for (int off = kWave / 2; off > 0; off >>= 1) {
            n += __shfl_xor(n, off, kWave);
            above += __shfl_xor(above, off, kWave);
        }
        if (lane_id() == 0) counts[turn][wave] = make_int2(n, above);
        if (hi == 0u) largest[threadIdx.x] = float_to_ordered(most + 0.0f);
        __syncthreads();
        n = above = 0;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
            n += counts[turn][w].x;
            above += counts[turn][w].y;
        }
        if (n >= k && (above < k || n <= room)) {
            done = true;
            want = n <= room ? 0 : k - above;                // of the labels that score t, the first ones
            if (n <= room) --mid;                            // (all that reach t: those above the number before it)
        } else if (hi == 0u) {
            if (threadIdx.x < kWave) {
                uint32_t top = 0u;
#pragma unroll
                for (int g = 0; g < kRowWaves; ++g) top = largest[g * kWave + lane_id()] > top ? largest[g * kWave + lane_id()] : top;
                top = wave_max_u32(top);
                const uint32_t r = reached_by<kRowWaves>(kRowThreads, k, [&](int i) __attribute__((always_inline)) { return largest[i]; });
                if (threadIdx.x == 0) {
                    range[0] = r > least ? r : least + 1u;
                    range[1] = top + 1u;
                }
            }
            __syncthreads();
            mid = lo = range[0];
            hi = range[1];
        } else {
            if (n >= k) lo = mid + 1u;
            else hi = mid;
            mid = lo + (hi - lo) / 2u;
        }
    }
}

// A segment of a row by one workgroup: its sums, and its k best labels.
// The labels: of the first block each thread's largest score is known, and a score that k of the threads reach is reached by all k best
// labels of the block and by few others.  These, and what reaches the same score in the blocks behind, are collected in LDS; behind 1, 4,
// 16, 64, .. blocks a higher threshold is found among them and the others are dropped, so that as many labels are collected in each of these
// stretches (behind 1, 2, 4, 8, ..: 4000 x 32000 bf16 with 64 labels 90.9 us against 86.7).  In the end the few that are left are ranked by counting.
// A piece with such a label is noted in a list of its wave, 64 of them are looked at together: most blocks have a few, and a wave would
// spend as much on these as on 64.
// Bound: 1024 x 131072 bf16 without top labels 44 to 50 us, one read at 5.4 to 6.1 TB/s; 2048 rows with 64 of them 113 us, 4.8 TB/s: vector
// instructions are under way for 0.7 to 0.8 of the time (the exponential, the sums, the largest of every piece against the threshold).
// (C <= 2: five waves to a SIMD, which what runs for crowded stretches alone would take a register too many for.)
template <typename T, int C>
__global__ __launch_bounds__(kRowThreads, C <= 2 ? 5 : 4)
void logprobs_kernel(const LogprobArgs a) {
    constexpr int N = PiecedRow<T>::N, E = C * N;
    __shared__ Sums sums[kRowWaves];
    __shared__ uint32_t largest[kRowThreads];
    __shared__ __align__(16) uint64_t lists[2][kTopKeys + 4];
    __shared__ int noted[kRowWaves][kWave + kWave * C];      // pieces, counted from the segment's first
    __shared__ uint32_t reach, range[2];
    __shared__ int2 counts[2][kRowWaves];
    __shared__ int found, kept;
    const int64_t b = blockIdx.x / static_cast<uint32_t>(a.segments), seg = blockIdx.x - b * a.segments;
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    const int64_t begin = seg * a.length, end = begin + a.length < row.pieces ? begin + a.length : row.pieces;
    Block<T, C> block;
    // Pieces with candidates for the top labels are read again, most of them in the first block: with the hint where these are few (bf16, k = 16,
    // 2048 x 131072 97.8 us with it and 103.1 without; k = 128, 838 x 32249 35.1 and 33.0; fp32, k = 64, 1024 x 131072 95.8 and 102.6).
    const bool seldom = 2 * a.k <= a.blocks * C;
    auto load = [&](int64_t first) __attribute__((always_inline)) {
        if (a.k == 0 || (first != begin && seldom)) block.template load<true>(row, first, end, kRowThreads);
        else block.template load<false>(row, first, end, kRowThreads);
    };
    load(begin);
    const int64_t edge = seg == 0 && static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    float more = edge >= 0 ? Elem<T>::get(row.p + edge) : kNone;
    if (threadIdx.x == 0) found = 0;
    Running run;
    uint64_t* keys = lists[0];
    int have = 0;                                            // keys from the blocks before
    // the threshold among the keys, and what reaches it, in the other list; by the whole workgroup
    auto thin = [&]() __attribute__((always_inline)) {
        __syncthreads();                                     // (`kept` and `range` have been read)
        if (threadIdx.x < kWave) {
            const uint32_t* words = reinterpret_cast<const uint32_t*>(keys);
            auto value = [&](int i) __attribute__((always_inline)) { return ~words[2 * i + 1]; };
            const uint32_t r = have <= 4 * kWave ? reached_by<4>(have, a.k, value) : reached_by<kTopKeys / kWave>(have, a.k, value);
            if (threadIdx.x == 0) {
                range[0] = r;                                // (may be below `reach`, see the end of a stretch)
                if (r > reach) reach = r;
                kept = 0;
            }
        }
        __syncthreads();
        uint64_t* other = keys == lists[0] ? lists[1] : lists[0];
        const uint32_t r = range[0];
        for (int i = threadIdx.x; i < have; i += kRowThreads)
            if (~static_cast<uint32_t>(keys[i] >> 32) >= r) other[atomicAdd(&kept, 1)] = keys[i];
        __syncthreads();
        keys = other;
        have = kept;
    };
    // the k best of the keys alone, in the other list
    auto cut = [&]() __attribute__((always_inline)) {
        end_keys(keys, have);
        __syncthreads();
        uint64_t* other = keys == lists[0] ? lists[1] : lists[0];
        for (int i = threadIdx.x; i < have; i += kRowThreads) {
            const int rank = rank_of(keys[i], keys, have);
            if (rank < a.k) other[rank] = keys[i];
        }
        __syncthreads();                                     // (the keys as well have been read)
        keys = other;
        have = have < a.k ? have : a.k;
    };
    int* notes = noted[threadIdx.x >> 6];
    int n_notes = 0;
    int64_t since = begin;                                   // where the present stretch of blocks began
    // up to 64 of the noted pieces, the last ones; room is taken by a lane for all of a piece's labels at once, by the instruction itself (the
    // compiler would add the lanes' numbers up first)
    auto look = [&](float least) __attribute__((always_inline)) {
        const int take = n_notes < kWave ? n_notes : kWave;
        n_notes -= take;
        if (lane_id() < take) {
            const T* p = row.p + row.first(begin + notes[n_notes + lane_id()]);
            float x[N];
            Elem<T>::values(*reinterpret_cast<const uint4*>(p), x);
            uint32_t which = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) which |= x[e] >= least ? 1u << e : 0u;
            int at = have + take_room(&found, __popc(which));
            const int32_t id = static_cast<int32_t>(p - row.p);
#pragma unroll 1
            for (; which != 0u && at < kTopKeys; which &= which - 1u, ++at) {
                const int e = __ffs(static_cast<int>(which)) - 1;
                keys[at] = make_key(Elem<T>::get(p + e) + 0.0f, id + e);       // (-0 and 0 are equal)
            }
        }
    };
    float least = kNone;
    for (int n = 0; n < a.blocks; ++n) {                     // (a.blocks: of a whole segment; the row may end before)
        const int64_t first = begin + static_cast<int64_t>(n) * (kRowThreads * C), stop = first + kRowThreads * C < end ? first + kRowThreads * C : end;
        float most = kNone, piece[C];
        {
            float f[E];
            block.values(f);
            if (n + 1 < a.blocks) load(first + kRowThreads * C);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                piece[i] = largest_of<N>(f, i * N);
                most = fmaxf(most, piece[i]);
            }
            run.template add<true>(f, most, a.c);
        }
        if (a.k == 0) continue;                              // uniform
        if (n == 0) {
            largest[threadIdx.x] = float_to_ordered(fmaxf(most, more) + 0.0f);
            __syncthreads();
            if (threadIdx.x < kWave) {
                const uint32_t r = reached_by<kRowThreads / kWave>(kRowThreads, a.k, [&](int i) __attribute__((always_inline)) { return largest[i]; });
                if (threadIdx.x == 0) reach = r;
            }
            __syncthreads();
        }
        if (n == 0) least = ordered_to_float(reach);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const bool here = piece[i] >= least;
            const uint64_t all = __ballot(here);
            if (all == 0ull) continue;                       // uniform
            if (here) notes[n_notes + __popcll(all & lanemask_lt())] = static_cast<int>(first - begin) + i * kRowThreads + static_cast<int>(threadIdx.x);
            n_notes += __popcll(all);
        }
        const bool last = n + 1 == a.blocks, ends = last || ((n & (n + 1)) == 0 && (__popc(n) & 1) == 0);      // uniform
        while (n_notes >= kWave || (ends && n_notes > 0)) look(least);
        if (n == 0 && more >= least) {
            const int at = have + take_room(&found, 1);
            if (at < kTopKeys) keys[at] = make_key(more + 0.0f, static_cast<int32_t>(edge));
        }
        if (!ends) continue;
        __syncthreads();
        const int now = found;
        const bool crowded = have + now > kTopKeys;          // uniform, as all of these
        if (__builtin_expect(crowded, 0)) {
            best_of_stretch<T>(row, static_cast<int>(since), static_cast<int>(stop), n == 0 ? static_cast<int>(edge) : -1, a.k, kTopKeys - have, reach,
                               largest, range, counts, keys + have, &kept);
            __syncthreads();
            have += kept;
        } else {
            have += now;
        }
        if (have > a.k + a.k / 2 + 8) thin();
        if (last || crowded || have > kTopKeys / 2) cut();
        __syncthreads();                                     // (everyone has read `found`)
        if (threadIdx.x == 0) {
            found = 0;
            // What scores as the k-th best label does and lies behind it is worse: where scores are equal, no label of the blocks to come is
            // looked at again.  (The elements behind the row's last piece were looked at with the first block.)
            if (crowded && have == a.k) {
                const uint32_t o = ~static_cast<uint32_t>(keys[have - 1] >> 32) + (key_id(keys[have - 1]) < row.first(row.pieces) ? 1u : 0u);
                if (o > reach) reach = o;
            }
        }
        __syncthreads();
        least = ordered_to_float(reach);
        since = stop;
    }
    run.add_one(more, a.c);
    __syncthreads();
    const Sums s = block_sums<kRowWaves>(run.sums(a.c), a.c, sums);
    const bool alone = a.segments == 1;
    if (alone) write_row<T>(a, b, s);
    else if (threadIdx.x == 0) a.parts[b * a.segments + seg] = make_float4(s.m, s.s, s.h, 0.0f);
    if (a.k == 0) return;
    const Norm z = norm_of(s);
    uint64_t* out = a.keys + (b * a.segments + seg) * a.k;
    for (int i = threadIdx.x; i < a.k; i += kRowThreads) {
        const uint64_t key = i < have ? keys[i] : kKeySentinel;
        if (alone) write_top(a, b, i, key, z);
        else out[i] = key;
    }
}

// The segments of a row joined, by a workgroup per row, four lanes to a key that is ranked (67 rows of 15 segments, 128 labels: a thread to
// a key 17.3 us).  The best labels, of up to kJoinAtOnce segments at a time and the best of those
// before them: of the first r of each segment (2 k labels or a few more in all) the k-th best is found by ranking; whatever is worse than
// that is left out, and the few others are ranked.
constexpr int kJoinWaves = 16, kJoinAtOnce = 128;
constexpr int kJoinFirst = 2 * XC_MAX_TOP + kJoinAtOnce;     // labels of the first ranking at most
template <typename T>
__global__ __launch_bounds__(kJoinWaves * kWave)
void logprobs_join_kernel(const LogprobArgs a) {
    __shared__ Sums sums[kJoinWaves];
    __shared__ __align__(16) uint64_t keys[kJoinKeys + XC_MAX_TOP + 4], best[XC_MAX_TOP];
    __shared__ uint64_t bound;
    __shared__ int found;
    static_assert(kJoinFirst <= kJoinKeys, "");
    constexpr int kThreads = kJoinWaves * kWave;
    const int64_t b = blockIdx.x;
    Sums t{kNone, 0.0f, 0.0f};
    for (int64_t i = threadIdx.x; i < a.segments; i += kThreads) {
        const float4 p = a.parts[b * a.segments + i];
        const Sums q{p.x, p.y, p.z};
        const float m = fmaxf(t.m, q.m);
        const Sums u = joined(t, m, a.c), w = joined(q, m, a.c);
        t = Sums{m, u.s + w.s, u.h + w.h};
    }
    const Sums s = block_sums<kJoinWaves>(t, a.c, sums);
    write_row<T>(a, b, s);
    if (a.k == 0) return;
    const Norm z = norm_of(s);
    int have = 0;
    const int at_once = kJoinKeys / a.k < kJoinAtOnce ? kJoinKeys / a.k : kJoinAtOnce;
    for (int64_t s0 = 0; s0 < a.segments; s0 += at_once) {
        const int g = static_cast<int>(a.segments - s0 < at_once ? a.segments - s0 : at_once);
        const uint64_t* in = a.keys + (b * a.segments + s0) * a.k;
        const int want = (2 * a.k + g - 1) / g, r = want < a.k ? want : a.k, first = g * r;
        __syncthreads();                                     // (the round before has read its keys)
        for (int i = threadIdx.x; i < first; i += kThreads) {
            const int seg = i / r;
            keys[i] = in[seg * a.k + (i - seg * r)];
        }
        end_keys(keys, first);
        if (threadIdx.x == 0) {
            bound = kKeySentinel;
            found = have;
        }
        __syncthreads();
        // (labels that are not there have the same key: where they reach the k-th place, `bound` stays what it is, theirs)
        for (int i = threadIdx.x >> 2; i < first; i += kThreads / 4) {
            const uint64_t key = keys[i];
            if (rank_of<4>(key, keys, first) == a.k - 1 && key != kKeySentinel) bound = key;
        }
        __syncthreads();
        const uint64_t limit = bound;
        for (int i = threadIdx.x; i < have; i += kThreads) keys[i] = best[i];
        for (int i = threadIdx.x; i < g * a.k; i += kThreads) {
            const uint64_t x = in[i];
            if (x <= limit && x != kKeySentinel) keys[atomicAdd(&found, 1)] = x;
        }
        __syncthreads();
        const int n = found;
        end_keys(keys, n);
        __syncthreads();
        for (int i = threadIdx.x >> 2; i < n; i += kThreads / 4) {
            const uint64_t key = keys[i];
            const int rank = rank_of<4>(key, keys, n);
            if (rank < a.k) best[rank] = key;
        }
        have = n < a.k ? n : a.k;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.k; i += kThreads) write_top(a, b, i, i < have ? best[i] : kKeySentinel, z);
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
struct LogprobGradArgs {
    const void* X;
    const int32_t* labels;
    const float *dlogp, *norm, *entropy, *dentropy;
    void* dX;
    int64_t B, V, ld, ldd, chunks;
    float T, c;
    int n;
};
constexpr int kGradThreads = 256, kGradEach = 4, kGradPieces = kGradThreads * kGradEach;       // pieces of a workgroup

// Bound: memory.  1024 x 131072 bf16 84 to 86 us, 6.3 TB/s read and written.
// A chunk of a row per workgroup, element by element; then the given labels that lie in the chunk, once each, whose sums of dlogp are
// formed in the order of the list.  (Their scores are read before anything is stored: dX may be X.)
template <typename T, typename TO>
__global__ __launch_bounds__(kGradThreads)
void logprobs_grad_kernel(const LogprobGradArgs a) {
    constexpr int N = PiecedRow<T>::N;
    const int64_t b = blockIdx.x / static_cast<uint32_t>(a.chunks), chunk = blockIdx.x - b * a.chunks;
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    TO* out = static_cast<TO*>(a.dX) + b * a.ldd;
    const int64_t first = chunk * kGradPieces, end = first + kGradPieces < row.pieces ? first + kGradPieces : row.pieces;
    uint4 v[kGradEach];
#pragma unroll
    for (int i = 0; i < kGradEach; ++i) {
        const int64_t at = first + i * kGradThreads + threadIdx.x;
        v[i] = at < end ? row.template load<true>(at) : make_uint4(0, 0, 0, 0);
    }
    const int64_t edge = chunk == 0 && static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    const float more = edge >= 0 ? Elem<T>::get(row.p + edge) : 0.0f;

    // G, by every wave: the lanes' labels in the order of the list
    float g = 0.0f;
    for (int j = lane_id(); j < a.n; j += kWave) {
        const int32_t l = a.labels[b * a.n + j];
        if (l >= 0 && l < a.V) g += a.dlogp[b * a.n + j];
    }
    g = wave_sum(g);
    const float m = a.norm[2 * b], ls = a.norm[2 * b + 1];
    const bool none = ls == kNone;                           // no label is there: nothing to learn from the row
    const float dh = a.dentropy != nullptr ? a.dentropy[b] : 0.0f, H = a.dentropy != nullptr ? a.entropy[b] : 0.0f;
    // logp = ln2 l with l = (x - m) c - ls / ln2; -p (G + dH (logp + H)) / T = 2^l (k0 + k1 l)
    const float ls2 = ls * 1.4426950408889634f, k0 = (ls == ls ? -fmaf(dh, H, g) : ls) / a.T, k1 = -dh * (0.6931471805599453f / a.T);
    auto value = [&](float x) __attribute__((always_inline)) {
        const float l = fmaxf(fmaf(x - m, a.c, -ls2), kFloor);
        const float d = __builtin_amdgcn_exp2f(l) * fmaf(k1, l, k0);
        return none ? 0.0f : d;
    };
    // the thread's place in the list (there are as many threads as places at most)
    static_assert(XC_MAX_GIVEN <= kGradThreads, "a thread per given label");
    int64_t given = -1;
    float dgiven = 0.0f;
    if (static_cast<int>(threadIdx.x) < a.n) {
        const int32_t l = a.labels[b * a.n + threadIdx.x];
        const int64_t piece = l < row.head ? -1 : (l - row.head) / N;
        const bool mine = l >= 0 && l < a.V && (l < row.head || piece >= row.pieces ? chunk == 0 : piece >= first && piece < end);
        if (mine) {
            given = l;
            for (int j = 0; j < a.n; ++j) {
                if (a.labels[b * a.n + j] != l) continue;
                if (j < static_cast<int>(threadIdx.x)) { given = -1; break; }
                dgiven += a.dlogp[b * a.n + j];
            }
            if (given >= 0) dgiven = none ? 0.0f : fmaf(dgiven, 1.0f / a.T, value(Elem<T>::get(row.p + l)));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kGradEach; ++i) {
        const int64_t at = first + i * kGradThreads + threadIdx.x;
        if (at < end) {
            float x[N];
            Elem<T>::values(v[i], x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = value(x[e]);
            put_elements<N>(out + row.first(at), x);
        }
    }
    if (edge >= 0) Elem<TO>::put(out + edge, value(more));
    __syncthreads();                                         // (waits for the stores as well)
    if (given >= 0) Elem<TO>::put(out + given, dgiven);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static size_t logprobs_bytes(int64_t B, int64_t V, int k, xc_dtype t) {
    const RowCut cut = cut_rows(B, V, t == XC_F32 ? 4 : 2, k);
    if (cut.segments == 1) return 16;
    return static_cast<size_t>(B) * cut.segments * (sizeof(float4) + static_cast<size_t>(k) * sizeof(uint64_t));
}

template <typename T>
static void launch_logprobs(const LogprobArgs& all, const RowCut& cut, hipStream_t st) {
    int64_t rows = kSoftmaxGrid / cut.segments;
    if (rows < 1) rows = 1;
    for (int64_t b0 = 0; b0 < all.B; b0 += rows) {
        LogprobArgs a = all;
        const int64_t nb = all.B - b0 < rows ? all.B - b0 : rows;
        a.X = static_cast<const T*>(all.X) + b0 * all.ld;
        a.labels += b0 * all.n;
        a.logp += b0 * all.n;
        a.entropy += b0;
        a.norm += 2 * b0;
        a.top += b0 * all.k;
        a.top_logp += b0 * all.k;
        a.parts += b0 * cut.segments;
        a.keys += b0 * cut.segments * all.k;
        const unsigned grid = static_cast<unsigned>(nb * cut.segments);
        constexpr int kSmall = small_block(sizeof(T)), kLarge = large_block(sizeof(T));
        if (cut.each == kSmall) XC_LAUNCH(K_LOGPROBS, st, (logprobs_kernel<T, kSmall><<<grid, kRowThreads, 0, st>>>(a)));
        else XC_LAUNCH(K_LOGPROBS, st, (logprobs_kernel<T, kLarge><<<grid, kRowThreads, 0, st>>>(a)));
        if (cut.segments > 1)
            XC_LAUNCH(K_LOGPROBS_JOIN, st, (logprobs_join_kernel<T><<<static_cast<unsigned>(nb), kJoinWaves * kWave, 0, st>>>(a)));
    }
}

template <typename T, typename TO>
static void launch_logprobs_grad(const LogprobGradArgs& all, hipStream_t st) {
    int64_t rows = kSoftmaxGrid / all.chunks;
    if (rows < 1) rows = 1;
    for (int64_t b0 = 0; b0 < all.B; b0 += rows) {
        LogprobGradArgs a = all;
        const int64_t nb = all.B - b0 < rows ? all.B - b0 : rows;
        a.X = static_cast<const T*>(all.X) + b0 * all.ld;
        a.dX = static_cast<TO*>(all.dX) + b0 * all.ldd;
        a.labels += b0 * all.n;
        a.dlogp += b0 * all.n;
        a.norm += 2 * b0;
        if (all.dentropy != nullptr) {
            a.entropy += b0;
            a.dentropy += b0;
        }
        XC_LAUNCH(K_LOGPROBS_GRAD, st, (logprobs_grad_kernel<T, TO><<<static_cast<unsigned>(nb * all.chunks), kGradThreads, 0, st>>>(a)));
    }
}

}  // namespace xc

extern "C" int xc_label_logprobs_workspace(int64_t B, int64_t V, int k, xc_dtype t, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (!softmax_shape(B, V, V) || k < 0 || k > XC_MAX_TOP || k > V) return XC_ESHAPE;
    *bytes = logprobs_bytes(B, V, k, t);
    return XC_OK;
}

extern "C" int xc_label_logprobs(const void* X, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature, const int32_t* labels, int n, int k,
                                 float* logp, float* entropy, float* norm, int32_t* top, float* top_logp, void* ws, size_t ws_bytes, void* stream) {
    using namespace xc;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (!softmax_shape(B, V, ld) || n < 0 || n > XC_MAX_GIVEN || k < 0 || k > XC_MAX_TOP || k > V) return XC_ESHAPE;
    if (!softmax_temperature(temperature)) return XC_EINVAL;
    if (!X || (n > 0 && (!labels || !logp)) || !entropy || !norm || (k > 0 && (!top || !top_logp)) || !ws) return XC_EINVAL;
    for (const void* p : {X, static_cast<const void*>(labels), static_cast<const void*>(logp), static_cast<const void*>(entropy), static_cast<const void*>(norm),
                          static_cast<const void*>(top), static_cast<const void*>(top_logp), static_cast<const void*>(ws)})
        if (!aligned16(p)) return XC_EINVAL;
    const size_t need = logprobs_bytes(B, V, k, t);
    if (ws_bytes < need) return XC_EWORKSPACE;
    const size_t per = static_cast<size_t>(B) * 4;
    if (overlap({Span(logp, per * n), Span(entropy, per), Span(norm, per * 2), Span(top, per * k), Span(top_logp, per * k), Span(ws, need)},
                {Span(X, rows_span(B, V, ld, t)), Span(labels, per * n)}))
        return XC_EINVAL;
    const RowCut cut = cut_rows(B, V, t == XC_F32 ? 4 : 2, k);
    float4* parts = static_cast<float4*>(ws);
    const LogprobArgs a{X, labels, logp, entropy, norm, top, top_logp, parts, reinterpret_cast<uint64_t*>(parts + B * cut.segments), B, V, ld, cut.segments,
                        cut.length, temperature, softmax_scale(temperature), n, k, cut.blocks};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (t == XC_F32) launch_logprobs<float>(a, cut, st);
    else launch_logprobs<bf16_t>(a, cut, st);
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

extern "C" int xc_label_logprobs_grad(const void* X, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature, const int32_t* labels, int n,
                                      const float* dlogp, const float* norm, const float* entropy, const float* dentropy, void* dX, int64_t ldd,
                                      xc_dtype out_t, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (!softmax_shape(B, V, ld) || !softmax_shape(B, V, ldd) || n < 0 || n > XC_MAX_GIVEN) return XC_ESHAPE;
    if (!softmax_temperature(temperature)) return XC_EINVAL;
    if (!X || (n > 0 && (!labels || !dlogp)) || !norm || !dX || (dentropy != nullptr && !entropy)) return XC_EINVAL;
    for (const void* p : {X, static_cast<const void*>(labels), static_cast<const void*>(dlogp), static_cast<const void*>(norm), static_cast<const void*>(entropy),
                          static_cast<const void*>(dentropy), static_cast<const void*>(dX)})
        if (!aligned16(p)) return XC_EINVAL;
    const size_t per = static_cast<size_t>(B) * 4;
    const Span x(X, rows_span(B, V, ld, t)), d(dX, rows_span(B, V, ldd, out_t));
    const bool in_place = dX == X && t == out_t && ld == ldd;
    if ((!in_place && d.meets(x)) || overlap({d}, {Span(labels, per * n), Span(dlogp, per * n), Span(norm, per * 2), Span(dentropy != nullptr ? entropy : nullptr, per), Span(dentropy, per)}))
        return XC_EINVAL;
    const int64_t pieces = V / (t == XC_F32 ? 4 : 8), chunks = pieces > kGradPieces ? (pieces + kGradPieces - 1) / kGradPieces : 1;
    const LogprobGradArgs a{X, labels, dlogp, norm, entropy, dentropy, dX, B, V, ld, ldd, chunks, temperature, softmax_scale(temperature), n};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (t == XC_F32 && out_t == XC_F32) launch_logprobs_grad<float, float>(a, st);
    else if (t == XC_F32) launch_logprobs_grad<float, bf16_t>(a, st);
    else if (out_t == XC_F32) launch_logprobs_grad<bf16_t, float>(a, st);
    else launch_logprobs_grad<bf16_t, bf16_t>(a, st);
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
