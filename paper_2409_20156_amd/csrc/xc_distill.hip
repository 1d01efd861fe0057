// The loss against a teacher's distribution, of which its top labels are given, and its gradient.  Per row, with y = x / T:
//   p = soft-max(y), q_k the teacher's probability of its k-th label, with a tail q_r = 1 - sum q_k for the labels that are not listed
//   loss = w T^2 (sum q_k (log q_k - log p_k) + q_r (log q_r - log p_r)),  p_r the sum of p over these
//   dX_v = w T (Q p_v - q_v) for a listed label, w T (Q p_r - q_r) r_v for any other one; Q = sum q_k + q_r, r the soft-max over the others.
// With a tail the row's sums leave the listed labels out, and the sum over all labels is put together from these and the listed ones in
// 64 bits: what the others' sum errs by leaves log p_r and log p_k - log p_r nearly alone, and p_r may be as small as it likes.
#include "xc_softmax.h"

namespace xc {

struct DistillArgs {
    const void* X;
    const int32_t* labels;
    const float *teacher, *weight;
    float* loss;
    void* dX;                            // or null
    float4* parts;                       // [B][segments]: sums of a segment (with a tail: of the labels that are not listed)
    struct RowTerms* terms;              // [B]
    int64_t B, V, ld, ldd, segments, length;
    float T, c;
    int K, blocks;
    bool tail;
};

// What a row's gradient is formed from.
struct RowTerms {
    // (powers of two are taken out as whole ones: the rest is in the factor, so that no large exponent is rounded)
    float other;                         // factor of 2^((x - m) c - l): w T (Q p_r - q_r), without a tail w T
    float m, l;                          // largest score of these labels, log2 of their sum
    float factor, mass;                  // w T; Q
    float m_all, l_all;                  // listed labels: Q p = mass 2^((x - m_all) c - l_all)
    float t, t_log;                      // q = exp(teacher - t - t_log)
    float live;                          // 0: the row counts for nothing
    float pad[2];
};

template <int CTRL, int ROWS>
__device__ __forceinline__ double lanes_from(double x) {     // 0 where there is no such lane
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x));
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
__device__ __forceinline__ double wave_sum(double x) {
    x += lanes_from<0x111, 0xf>(x);
    x += lanes_from<0x112, 0xf>(x);
    x += lanes_from<0x114, 0xf>(x);
    x += lanes_from<0x118, 0xf>(x);
    x += lanes_from<0x142, 0xa>(x);
    x += lanes_from<0x143, 0xc>(x);
    return __shfl(x, kWave - 1, kWave);
}
__device__ __forceinline__ bool is_label(int32_t v, int64_t V) { return v >= 0 && v < V; }

// The list of a row in LDS: its labels, and what one wave has made of each place.
struct Place { double q; float t, x; float q_all; bool once; };           // q_all: of all places with the label, at the first of them (once)
struct List {
    int32_t labels[XC_MAX_TEACHER];      // (read 16 bytes at a time)
    Place places[XC_MAX_TEACHER];
};
// Whether the label of place k is in the list before it, or behind it (16 bytes aligned, -1 behind the last place up to a multiple of 4).
struct Elsewhere { bool before, behind; };
__device__ __forceinline__ Elsewhere listed_elsewhere(const int32_t* list, int K, int k, int32_t id) {
    Elsewhere r{false, false};
#pragma unroll 4
    for (int j = 0; j < K; j += 4) {
        const int4 l = *reinterpret_cast<const int4*>(list + j);
        const int n = (l.x == id ? 1 : 0) | (l.y == id ? 2 : 0) | (l.z == id ? 4 : 0) | (l.w == id ? 8 : 0);
        const int below = k - j >= 4 ? 15 : k > j ? (1 << (k - j)) - 1 : 0, at = k >= j && k - j < 4 ? 1 << (k - j) : 0;
        r.before |= (n & below) != 0;
        r.behind |= (n & ~(below | at)) != 0;
    }
    return r;
}

// What does not depend on the row's sums, by one wave (a lane has every 64th place), while the row is on its way: the teacher's
// probabilities, in 64 bits as all that is formed from the sums.  labels are in the list.
// These two functions are a chain of dependent steps, not work: logarithms that are needed together are taken by neighbouring lanes at
// once, quotients of sums stand where differences of their logarithms would (200 x 131072 fp32: 11.8 us with a logarithm, an exponential
// after the other and a loop over the list for each place).
struct Teacher {
    double sum, weighted;                // of the list: sum of q = exp(t - t0), of q log q over its labels, q of all places of a label together
    float t0, x_max;
    bool any;
};
template <typename T>
__device__ __forceinline__ Teacher teacher_of(const DistillArgs& a, int64_t b, List& list) {
    constexpr int kGroups = XC_MAX_TEACHER / kWave;
    const T* x = static_cast<const T*>(a.X) + b * a.ld;
    const int groups = (a.K + kWave - 1) / kWave;
    Teacher r;
    int32_t ids[kGroups];
    float t_max = kNone;
    r.x_max = kNone;
    bool some = false;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        ids[g] = -1;
        if (g >= groups) continue;                           // uniform
        const int k = g * kWave + lane_id();
        if (k < a.K) {
            ids[g] = list.labels[k];
            Place p{0.0, 0.0f, 0.0f, 0.0f, false};
            if (is_label(ids[g], a.V)) {
                p.t = a.teacher[b * a.K + k];
                p.x = Elem<T>::get(x + ids[g]);
                t_max = fmaxf(t_max, p.t);
                r.x_max = fmaxf(r.x_max, p.x);
                some |= a.tail || p.t != kNone;              // (without a tail a list of probabilities 0 is no distribution)
            }
            list.places[k] = p;
        }
    }
    // places whose label occurs before them
    uint64_t again[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) again[g] = 0ull;
#pragma unroll
    for (int h = 0; h < kGroups; ++h) {
        if (h >= groups) continue;
        const int n = a.K - h * kWave < kWave ? a.K - h * kWave : kWave;
        for (int j = 0; j < n; ++j) {
            const int32_t id = __builtin_amdgcn_readlane(ids[h], j);
            again[h] |= __ballot(ids[h] == id) & (~1ull << j);
#pragma unroll
            for (int g = h + 1; g < kGroups; ++g) if (g < groups) again[g] |= __ballot(ids[g] == id);
        }
    }
    r.any = __ballot(some) != 0ull;
    t_max = wave_max(t_max);
    r.x_max = wave_max(r.x_max);
    r.t0 = a.tail || t_max == kNone ? 0.0f : t_max;
    r.sum = r.weighted = 0.0;
    bool twice = false;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
        if (g < groups && is_label(ids[g], a.V)) {
            const bool once = ((again[g] >> lane_id()) & 1ull) == 0ull;
            list.places[g * kWave + lane_id()].once = once;
            twice |= !once;
        }
    const bool dup = __ballot(twice) != 0ull;
    // (one exponential in the code for all places: a kernel that runs once per row waits for its own instructions as well)
#pragma unroll 1
    for (int k = lane_id(); k < a.K; k += kWave) {
        if (!is_label(list.labels[k], a.V)) continue;
        const double d = static_cast<double>(list.places[k].t) - static_cast<double>(r.t0), q = exp(d);
        list.places[k].q = q;
        r.sum += q;
        if (!dup && !(q == 0.0)) r.weighted += q * d;
    }
    r.sum = wave_sum(r.sum);
    const double scale = a.tail ? 1.0 : 1.0 / r.sum;
#pragma unroll 1
    for (int k = lane_id(); k < a.K; k += kWave) {
        double q = list.places[k].q;
        if (dup && list.places[k].once) {
            const int32_t id = list.labels[k];
            for (int j = k + 1; j < a.K; ++j) if (list.labels[j] == id) q += list.places[j].q;
            if (!(q == 0.0)) r.weighted += q * log(q);
        }
        list.places[k].q_all = static_cast<float>(q * scale);
    }
    r.weighted = wave_sum(r.weighted);
    return r;
}
// 2^n of the size of x (or 1), by which factors are kept from being rounded in an exponent.
__device__ __forceinline__ int size_of(double x) { return x > 0.0 && x < static_cast<double>(INFINITY) ? ilogb(x) : 0; }

// Loss and terms of a row from its sums, by the same wave.  A place whose label occurs before it does not count to the student's sum again.
template <typename T>
__device__ __forceinline__ RowTerms row_terms(const DistillArgs& a, int64_t b, const Sums& s, float weight, const Teacher& t, const List& list) {
    RowTerms r{};
    r.factor = weight * a.T;
    r.live = t.any ? 1.0f : 0.0f;
    if (!t.any) {
        if (lane_id() == 0 && a.loss != nullptr) a.loss[b] = 0.0f;
        return r;
    }
    // (the student's scores relative to the largest one: that may be huge)
    const double invT = 1.0 / static_cast<double>(a.T), none = -static_cast<double>(INFINITY);
    const float m_all = fmaxf(s.m, t.x_max);
    const double ref = m_all == kNone ? 0.0 : static_cast<double>(m_all);
    // sums relative to the largest score: of the listed labels, of those that s is about (as one more place, where that score is another)
    const double below = s.s == 0.0f || s.m == m_all ? 0.0 : (static_cast<double>(s.m) - ref) * invT;
    double listed = 0.0, cross = 0.0, rest = below != 0.0 ? 0.0 : static_cast<double>(s.s);
    const int n = a.tail ? a.K + (below != 0.0 ? 1 : 0) : a.K;
#pragma unroll 1
    for (int k = lane_id(); k < n; k += kWave) {
        const bool place = k < a.K;
        if (place && !is_label(list.labels[k], a.V)) continue;
        const double y = place ? (static_cast<double>(list.places[k].x) - ref) * invT : below;
        const double e = a.tail ? exp(y) : 0.0;
        if (!place) {
            rest = static_cast<double>(s.s) * e;
        } else {
            if (list.places[k].once) listed += e;
            const double q = list.places[k].q;
            if (!(q == 0.0)) cross += q * y;
        }
    }
    cross = wave_sum(cross);
    if (below != 0.0) rest = __shfl(rest, a.K & (kWave - 1), kWave);       // uniform (without a tail the largest score is s's)
    double all = rest;
    if (a.tail) all += wave_sum(listed);
    const double p_r = a.tail ? (s.s == 0.0f ? 0.0 : rest / all) : 1.0;
    double q_r = 0.0;
    if (a.tail && s.s != 0.0f) {                             // (no label but the listed ones: nothing to compare)
        q_r = 1.0 - t.sum;
        if (q_r < 0.0) q_r = 0.0;
    }
    // log of the sum over all, of q_r / p_r, of the teacher's sum
    const double logs = log(lane_id() == 0 ? all : lane_id() == 1 ? q_r / p_r : t.sum);
    const double lse = __shfl(logs, 0, kWave), t_log = a.tail ? 0.0 : __shfl(logs, 2, kWave);
    double ratio = __shfl(logs, 1, kWave);
    if (p_r == 0.0 && q_r != 0.0) ratio = log(q_r) - (log(static_cast<double>(s.s)) + below - lse);          // (beyond what 64 bits hold)
    const double scale = a.tail ? 1.0 : 1.0 / t.sum, q_sum = a.tail ? t.sum : t.sum == t.sum ? 1.0 : t.sum, mass = q_sum + q_r;
    double loss = 0.0;
    if (lse == none) loss = q_sum == 0.0 ? 0.0 : q_sum == q_sum ? -none : q_sum;               // no label at all
    else if (!(q_sum == 0.0)) loss = (t.weighted - cross) * scale + q_sum * (lse - t_log);
    if (!(q_r == 0.0)) loss += q_r * ratio;
    const double T2 = static_cast<double>(a.T) * static_cast<double>(a.T);
    if (lane_id() == 0 && a.loss != nullptr) a.loss[b] = static_cast<float>(static_cast<double>(weight) * T2 * loss);
    r.m = s.m == kNone ? 0.0f : s.m;
    const int l = size_of(static_cast<double>(s.s)), l_all = size_of(all);
    r.l = static_cast<float>(l);
    r.m_all = m_all == kNone ? 0.0f : m_all;
    r.l_all = lse == none ? kNone : static_cast<float>(l_all);
    r.mass = static_cast<float>(lse == none ? mass : mass * (ldexp(1.0, l_all) / all));
    r.t = t.t0;
    r.t_log = a.tail ? 0.0f : static_cast<float>(t_log);
    const double factor = static_cast<double>(weight) * static_cast<double>(a.T);
    r.other = s.s == 0.0f ? 0.0f : static_cast<float>(factor * (mass * p_r - q_r) * (ldexp(1.0, l) / static_cast<double>(s.s)));
    return r;
}

__device__ __forceinline__ float q_of(const RowTerms& r, float t) {
    return __builtin_amdgcn_exp2f(((t - r.t) - r.t_log) * 1.4426950408889634f);
}
__device__ __forceinline__ float other_gradient(const RowTerms& r, float x, float c) {
    return r.other * __builtin_amdgcn_exp2f(fmaf(x - r.m, c, -r.l));
}
// Of a listed label with score x, q the teacher's probability.
__device__ __forceinline__ float listed_gradient(const DistillArgs& a, const RowTerms& r, float x, float q) {
    const float p = r.l_all == kNone ? 0.0f : __builtin_amdgcn_exp2f(fmaf(x - r.m_all, a.c, -r.l_all));
    return r.factor * fmaf(r.mass, p, -q);
}

// Bound: one read.  The loss alone, by this and the next kernel, 64 labels and a tail: 1024 x 131072 bf16 53 us (5.0 TB/s), fp32 89 (6.0), 2048 x
// 131072 bf16 100 (5.3), 2048 x 32000 bf16 38 (3.5: one block to a workgroup).  Sums of a segment.  With a tail the listed labels of a block are marked, a bit each, before its elements are looked at.
template <typename T, int C>
__global__ __launch_bounds__(kRowThreads)
void distill_sums_kernel(const DistillArgs a) {
    constexpr int N = PiecedRow<T>::N, E = C * N, kMarks = kRowThreads * C / 4;
    __shared__ Sums sums[kRowWaves];
    // A byte per piece; the edges.  Block n + 1's are set while block n is summed, block n's cleared behind the barrier that follows: of
    // three, so that the next barrier lies between this and the block that has them next (of two, a fast wave's n + 2 would meet it).
    __shared__ uint32_t marks[3][kMarks + 1];
    const int64_t b = blockIdx.x / static_cast<uint32_t>(a.segments), seg = blockIdx.x - b * a.segments;
    if (a.weight != nullptr && a.weight[b] == 0.0f) return;  // uniform
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    const int64_t begin = seg * a.length, end = begin + a.length < row.pieces ? begin + a.length : row.pieces;
    Block<T, C> block;
    block.template load<true>(row, begin, end, kRowThreads);
    const int64_t edge = seg == 0 && static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    float more = edge >= 0 ? Elem<T>::get(row.p + edge) : kNone;
    Running run;
    static_assert(XC_MAX_TEACHER <= kRowThreads, "a thread per listed label");
    int32_t id = -1;
    int64_t piece = -1;
    if (a.tail) {
        if (static_cast<int>(threadIdx.x) < a.K) id = a.labels[b * a.K + threadIdx.x];
        if (!is_label(id, a.V)) id = -1;
        piece = id < row.head ? -1 : (id - row.head) / N;
        for (int i = threadIdx.x; i <= kMarks; i += kRowThreads) marks[0][i] = marks[1][i] = marks[2][i] = 0;
        __syncthreads();
        if (id >= 0 && (piece < 0 || piece >= row.pieces))
            atomicOr(&marks[0][kMarks], 1u << (id < row.head ? id : static_cast<int>(id - row.pieces * N)));
    }
    auto mark = [&](int n, uint32_t* of, bool on) __attribute__((always_inline)) {        // the thread's listed label, if it lies in block n
        const int64_t at = piece - (begin + static_cast<int64_t>(n) * (kRowThreads * C));
        if (id >= 0 && piece >= 0 && piece < end && at >= 0 && at < kRowThreads * C) {
            uint32_t* w = of + (at >> 2);
            if (on) atomicOr(w, 1u << (static_cast<int>(at & 3) * 8 + static_cast<int>(id - row.first(piece))));
            else *w = 0;
        }
    };
    if (a.tail) {
        mark(0, marks[0], true);
        __syncthreads();
        if (edge >= 0 && ((marks[0][kMarks] >> threadIdx.x) & 1u) != 0u) more = kNone;
    }
    for (int n = 0, at = 0; n < a.blocks; ++n) {             // (at: n % 3)
        const int64_t first = begin + static_cast<int64_t>(n) * (kRowThreads * C);
        const int next = at == 2 ? 0 : at + 1;
        float f[E];
        block.values(f);
        if (n + 1 < a.blocks) block.template load<true>(row, first + kRowThreads * C, end, kRowThreads);
        if (a.tail) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const uint32_t m = reinterpret_cast<const unsigned char*>(marks[at])[i * kRowThreads + threadIdx.x];
                if (__ballot(m != 0u) == 0ull) continue;
#pragma unroll
                for (int e = 0; e < N; ++e) if ((m >> e) & 1u) f[i * N + e] = kNone;
            }
            mark(n + 1, marks[next], true);
        }
        run.template add<false>(f, largest_of<E>(f, 0), a.c);
        if (a.tail && n + 1 < a.blocks) {
            __syncthreads();                                 // (block n's marks have been read, those of n + 1 are set)
            mark(n, marks[at], false);
        }
        at = next;
    }
    run.add_one(more, a.c);
    const Sums s = block_sums<kRowWaves>(run.sums(a.c), a.c, sums);
    if (threadIdx.x == 0) a.parts[b * a.segments + seg] = make_float4(s.m, s.s, 0.0f, 0.0f);
}

// A row's segments joined, by a wave.
__device__ __forceinline__ float4 first_part(const DistillArgs& a, int64_t b) {       // asked for before the teacher's part, which does not need it
    return lane_id() < a.segments ? a.parts[b * a.segments + lane_id()] : make_float4(kNone, 0.0f, 0.0f, 0.0f);
}
__device__ __forceinline__ Sums joined_segments(const DistillArgs& a, int64_t b, const float4& first) {
    Sums t{kNone, 0.0f, 0.0f};
    for (int64_t i = lane_id(); i < a.segments; i += kWave) {
        const float4 p = i < kWave ? first : a.parts[b * a.segments + i];
        const Sums q{p.x, p.y, 0.0f};
        const float m = fmaxf(t.m, q.m);
        const Sums u = joined(t, m, a.c), w = joined(q, m, a.c);
        t = Sums{m, u.s + w.s, 0.0f};
    }
    return wave_sums(t, a.c);
}

// A wave per row: its segments joined, its loss and terms.
constexpr int kTermWaves = 4;
template <typename T>
__global__ __launch_bounds__(kTermWaves * kWave)
void distill_terms_kernel(const DistillArgs a) {
    __shared__ __align__(16) List lists[kTermWaves];
    const int64_t b = static_cast<int64_t>(blockIdx.x) * kTermWaves + (threadIdx.x >> 6);
    List& list = lists[threadIdx.x >> 6];
    if (b < a.B) for (int k = lane_id(); k < a.K; k += kWave) list.labels[k] = a.labels[b * a.K + k];
    __syncthreads();
    if (b >= a.B) return;
    const float weight = a.weight != nullptr ? a.weight[b] : 1.0f;
    RowTerms r{};
    if (weight == 0.0f) {                                    // counts for nothing, whatever it holds
        if (lane_id() == 0) a.loss[b] = 0.0f;
    } else {
        const float4 part = first_part(a, b);
        const Teacher teacher = teacher_of<T>(a, b, list);
        r = row_terms<T>(a, b, joined_segments(a, b, part), weight, teacher, list);
    }
    if (lane_id() == 0) a.terms[b] = r;
}

// The gradient of a chunk of a row, then that of the listed labels in it (their scores are read before anything is stored: dX may be X).
// INLINE: every workgroup makes the row's terms for itself from the segments' sums, while its chunk is on its way, and the first one the
// loss: a launch less, where few rows leave the device idle anyway (kInlineGrid).  Not in place: the list's scores lie
// in other workgroups' chunks.
constexpr int kDistillThreads = 256, kDistillEach = 4, kDistillPieces = kDistillThreads * kDistillEach;
template <typename T, typename TO, bool INLINE>
__global__ __launch_bounds__(kDistillThreads)
void distill_grad_kernel(const DistillArgs a, int64_t chunks) {
    constexpr int N = PiecedRow<T>::N;
    const int64_t b = blockIdx.x / static_cast<uint32_t>(chunks), chunk = blockIdx.x - b * chunks;
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    TO* out = static_cast<TO*>(a.dX) + b * a.ldd;
    const int64_t first = chunk * kDistillPieces, end = first + kDistillPieces < row.pieces ? first + kDistillPieces : row.pieces;
    __shared__ __align__(16) List list;
    __shared__ RowTerms terms;
    Block<T, kDistillEach> block;
    block.template load<true>(row, first, end, kDistillThreads);
    const int64_t edge = chunk == 0 && static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    const float more = edge >= 0 ? Elem<T>::get(row.p + edge) : 0.0f;
    static_assert(XC_MAX_TEACHER <= kDistillThreads, "a thread per listed label");
    const int32_t id = static_cast<int>(threadIdx.x) < a.K ? a.labels[b * a.K + threadIdx.x] : -1;
    list.labels[threadIdx.x] = id;
    if constexpr (!INLINE) { if (threadIdx.x == 0) terms = a.terms[b]; }
    __syncthreads();
    if constexpr (INLINE) {
        const float weight = a.weight != nullptr ? a.weight[b] : 1.0f;
        if (threadIdx.x < kWave) {
            RowTerms r{};
            DistillArgs mine = a;
            if (chunk != 0) mine.loss = nullptr;
            if (weight != 0.0f) {
                const float4 part = first_part(a, b);
                const Teacher teacher = teacher_of<T>(a, b, list);
                r = row_terms<T>(mine, b, joined_segments(a, b, part), weight, teacher, list);
            } else if (threadIdx.x == 0 && chunk == 0) {
                a.loss[b] = 0.0f;
            }
            if (threadIdx.x == 0) terms = r;
        }
        __syncthreads();
    }
    const RowTerms r = terms;
    const bool live = r.live != 0.0f;                        // uniform
    int64_t listed = -1;
    float value = 0.0f;
    if (live && is_label(id, a.V)) {
        const int64_t piece = id < row.head ? -1 : (id - row.head) / N;
        if (id < row.head || piece >= row.pieces ? chunk == 0 : piece >= first && piece < end) {
            float q = 0.0f;                                  // (all places of the label count, at the first of them)
            if constexpr (INLINE) {
                if (list.places[threadIdx.x].once) listed = id;
                q = list.places[threadIdx.x].q_all;
            } else {
                const Elsewhere e = listed_elsewhere(list.labels, a.K, threadIdx.x, id);
                if (!e.before) listed = id;
                q = q_of(r, a.teacher[b * a.K + threadIdx.x]);
                if (e.behind) for (int j = threadIdx.x + 1; j < a.K; ++j) if (list.labels[j] == id) q += q_of(r, a.teacher[b * a.K + j]);
            }
            if (listed >= 0) value = listed_gradient(a, r, Elem<T>::get(row.p + id), q);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kDistillEach; ++i) {
        const int64_t at = first + i * kDistillThreads + threadIdx.x;
        if (at < end) {
            float x[N];
            Elem<T>::values(block.v[i], x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = live ? other_gradient(r, x[e], a.c) : 0.0f;
            put_elements<N>(out + row.first(at), x);
        }
    }
    if (edge >= 0) Elem<TO>::put(out + edge, live ? other_gradient(r, more, a.c) : 0.0f);
    __syncthreads();                                         // (waits for the stores as well)
    if (listed >= 0) Elem<TO>::put(out + listed, value);
}

// ---- a row by one workgroup, which holds it in registers: read once, its sums, its loss and terms by one wave, its gradient.
// Listed labels are taken out of the sums by a mark each, a bit in a byte per piece.
// Bound: memory, and what a compute unit's one or two rows leave idle between their reads and stores.  1024 x 131072 bf16 125 to 131 us (537 MB,
// 4.2 TB/s; 152 in three launches that read the row twice), 300 x 50021 fp32 39 (two rounds on 256 compute units; 44.5), 4096 x 20000 bf16 75
// (4.4 TB/s).
template <typename T, typename TO, int W, int C>
__global__ __launch_bounds__(W * kWave, C == 16 ? 4 : 1)
void distill_row_kernel(const DistillArgs a) {
    constexpr int N = PiecedRow<T>::N, kThreads = W * kWave, kMarks = kThreads * C / 4;
    __shared__ Sums sums[W];
    __shared__ uint32_t marks[kMarks + 1];                   // a byte per piece; the edges
    __shared__ __align__(16) List list;
    __shared__ RowTerms terms;
    static_assert(XC_MAX_TEACHER <= kThreads, "a thread per listed label");
    const int64_t b = blockIdx.x;
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    TO* out = static_cast<TO*>(a.dX) + b * a.ldd;
    const float weight = a.weight != nullptr ? a.weight[b] : 1.0f;
    const int32_t id = static_cast<int>(threadIdx.x) < a.K ? a.labels[b * a.K + threadIdx.x] : -1;
    const bool there = is_label(id, a.V);
    const int64_t edge = static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    const int pieces = static_cast<int>(row.pieces);
    uint4 v[C];
    if (weight != 0.0f) {                                    // uniform
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int at = i * kThreads + static_cast<int>(threadIdx.x);
            v[i] = at < pieces ? row.template load<true>(at) : Elem<T>::none();
        }
    }
    float more = edge >= 0 && weight != 0.0f ? Elem<T>::get(row.p + edge) : kNone;
    const float edge_score = more;
    if (static_cast<int>(threadIdx.x) < XC_MAX_TEACHER) list.labels[threadIdx.x] = id;
    if (a.tail) {
        for (int i = threadIdx.x; i <= kMarks; i += kThreads) marks[i] = 0;
        __syncthreads();
        if (there) {
            const int64_t piece = id < row.head ? -1 : (id - row.head) / N;
            if (piece >= 0 && piece < row.pieces) atomicOr(&marks[piece >> 2], 1u << (static_cast<int>(piece & 3) * 8 + static_cast<int>(id - row.first(piece))));
            else atomicOr(&marks[kMarks], 1u << (id < row.head ? id : static_cast<int>(id - row.pieces * N)));
        }
    }
    __syncthreads();
    if (weight != 0.0f) {
        Teacher teacher{};
        if (threadIdx.x < kWave) teacher = teacher_of<T>(a, b, list);      // (while the row's pieces are under way)
        if (a.tail && edge >= 0 && ((marks[kMarks] >> threadIdx.x) & 1u) != 0u) more = kNone;
        Running run;
        // groups of 8 elements at least, unpacked one after the other
        constexpr int G = 8 / N > 1 ? 8 / N : C % 2 == 0 ? 2 : 1, E = G * N;
#pragma unroll
        for (int i0 = 0; i0 < C; i0 += G) {
            if (i0 * kThreads >= pieces) break;              // uniform: the row ends before
            float f[E];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float x[N];
                Elem<T>::values(v[i0 + i], x);
#pragma unroll
                for (int e = 0; e < N; ++e) f[i * N + e] = x[e];
                if (a.tail) {
                    const uint32_t m = reinterpret_cast<const unsigned char*>(marks)[(i0 + i) * kThreads + threadIdx.x];
                    if (__ballot(m != 0u) == 0ull) continue;
#pragma unroll
                    for (int e = 0; e < N; ++e) if ((m >> e) & 1u) f[i * N + e] = kNone;
                }
            }
            run.template add<false>(f, largest_of<E>(f, 0), a.c);
            __builtin_amdgcn_sched_barrier(0);
        }
        run.add_one(more, a.c);
        const Sums s = block_sums<W>(run.sums(a.c), a.c, sums);
        if (threadIdx.x < kWave) {
            const RowTerms r = row_terms<T>(a, b, s, weight, teacher, list);
            if (threadIdx.x == 0) terms = r;
        }
    } else if (threadIdx.x == 0) {                           // counts for nothing, whatever it holds
        terms = RowTerms{};
        a.loss[b] = 0.0f;
    }
    __syncthreads();                                         // (the row's scores have all been read: dX may be X)
    const RowTerms r = terms;
    const bool live = r.live != 0.0f;                        // uniform
    const bool listed = live && there && list.places[threadIdx.x].once;
    const float value = listed ? listed_gradient(a, r, list.places[threadIdx.x].x, list.places[threadIdx.x].q_all) : 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int at = i * kThreads + static_cast<int>(threadIdx.x);
        if (at < pieces) {
            float x[N];
            if (live) {
                Elem<T>::values(v[i], x);
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = other_gradient(r, x[e], a.c);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = 0.0f;
            }
            put_elements<N>(out + row.first(at), x);
        }
    }
    if (edge >= 0) Elem<TO>::put(out + edge, live ? other_gradient(r, edge_score, a.c) : 0.0f);
    __syncthreads();                                         // (waits for the stores as well)
    if (listed) Elem<TO>::put(out + id, value);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static size_t distill_bytes(int64_t B, int64_t V, xc_dtype t) {
    return static_cast<size_t>(B) * (sizeof(RowTerms) + static_cast<size_t>(cut_rows(B, V, t == XC_F32 ? 4 : 2).segments) * sizeof(float4));
}

// Up to as many workgroups make the row's terms themselves (K = 64, a tail; with a launch for the terms and without: 16 x 131072
// bf16, 256 workgroups, 19.4 us and 15.5; 60 x 65536, 480, 22.8 and 18.7; 64 x 100000 fp32, 1600, 29.3 and 32.8).
constexpr unsigned kInlineGrid = 1024;
// Whether a row is one workgroup's, which holds it (0: it is not): read once.  As few waves as hold it with 4 pieces to a thread, or 16 where
// there are more rows than compute units: two rows at a time on one (16 waves with 4 and 4 with 16: 300 x 32000 bf16 28.1 us and 21.8, 400 x
// 20000 26.0 and 18.7, 2048 x 32000 117 and 64; 257 x 32000 20.4 and 20.8).  Long rows only where they keep the device busy: in two or three
// launches and held, 16 x 131072 bf16 15.5 us and 19.9, 64 x 131072 20.8 and 25.0, 80 x 131072 30.9 and 25.2, 1024 x 131072 152 and 131; the
// shorter rows: 16 x 32768 14.2 and 12.3.
struct Held { int waves, pieces; };
static Held distill_whole(int64_t B, int64_t V, size_t element) {
    const int64_t pieces = V / static_cast<int64_t>(16 / element);
    if (pieces <= 4 * kWave * 4) return {4, 4};
    if (pieces <= 16 * kWave * 4) return B > 256 ? Held{4, 16} : Held{16, 4};
    if (B < 72) return {0, 0};
    if (pieces <= 8 * kWave * 16) return {8, 16};
    return pieces <= 16 * kWave * 16 ? Held{16, 16} : Held{0, 0};
}

template <typename T, typename TO>
static void launch_distill(const DistillArgs& all, const RowCut& cut, hipStream_t st) {
    const Held held = all.dX != nullptr ? distill_whole(all.B, all.V, sizeof(T)) : Held{0, 0};
    if (held.waves != 0) {
        for (int64_t b0 = 0; b0 < all.B; b0 += kSoftmaxGrid) {
            DistillArgs a = all;
            a.B = all.B - b0 < kSoftmaxGrid ? all.B - b0 : kSoftmaxGrid;
            a.X = static_cast<const T*>(all.X) + b0 * all.ld;
            a.dX = static_cast<TO*>(all.dX) + b0 * all.ldd;
            a.labels += b0 * all.K;
            a.teacher += b0 * all.K;
            if (all.weight != nullptr) a.weight += b0;
            a.loss += b0;
            const unsigned grid = static_cast<unsigned>(a.B);
            if (held.waves == 4 && held.pieces == 4) XC_LAUNCH(K_DISTILL_GRAD, st, (distill_row_kernel<T, TO, 4, 4><<<grid, 4 * kWave, 0, st>>>(a)));
            else if (held.waves == 4) XC_LAUNCH(K_DISTILL_GRAD, st, (distill_row_kernel<T, TO, 4, 16><<<grid, 4 * kWave, 0, st>>>(a)));
            else if (held.waves == 8) XC_LAUNCH(K_DISTILL_GRAD, st, (distill_row_kernel<T, TO, 8, 16><<<grid, 8 * kWave, 0, st>>>(a)));
            else if (held.pieces == 4) XC_LAUNCH(K_DISTILL_GRAD, st, (distill_row_kernel<T, TO, 16, 4><<<grid, 16 * kWave, 0, st>>>(a)));
            else XC_LAUNCH(K_DISTILL_GRAD, st, (distill_row_kernel<T, TO, 16, 16><<<grid, 16 * kWave, 0, st>>>(a)));
        }
        return;
    }
    const int64_t pieces = all.V / static_cast<int64_t>(16 / sizeof(T)), chunks = pieces > kDistillPieces ? (pieces + kDistillPieces - 1) / kDistillPieces : 1;
    int64_t rows = kSoftmaxGrid / (chunks > cut.segments ? chunks : cut.segments);
    if (rows < 1) rows = 1;
    for (int64_t b0 = 0; b0 < all.B; b0 += rows) {
        DistillArgs a = all;
        const int64_t nb = all.B - b0 < rows ? all.B - b0 : rows;
        a.B = nb;
        a.X = static_cast<const T*>(all.X) + b0 * all.ld;
        if (all.dX != nullptr) a.dX = static_cast<TO*>(all.dX) + b0 * all.ldd;
        a.labels += b0 * all.K;
        a.teacher += b0 * all.K;
        if (all.weight != nullptr) a.weight += b0;
        a.loss += b0;
        a.parts += b0 * cut.segments;
        a.terms += b0;
        const unsigned grid = static_cast<unsigned>(nb * cut.segments);
        constexpr int kSmall = small_block(sizeof(T)), kLarge = large_block(sizeof(T));
        if (cut.each == kSmall) XC_LAUNCH(K_DISTILL_SUMS, st, (distill_sums_kernel<T, kSmall><<<grid, kRowThreads, 0, st>>>(a)));
        else XC_LAUNCH(K_DISTILL_SUMS, st, (distill_sums_kernel<T, kLarge><<<grid, kRowThreads, 0, st>>>(a)));
        const unsigned chunk_grid = static_cast<unsigned>(nb * chunks);
        if (all.dX != nullptr && all.dX != all.X && chunk_grid <= kInlineGrid) {
            XC_LAUNCH(K_DISTILL_GRAD, st, (distill_grad_kernel<T, TO, true><<<chunk_grid, kDistillThreads, 0, st>>>(a, chunks)));
            continue;
        }
        XC_LAUNCH(K_DISTILL_TERMS, st, (distill_terms_kernel<T><<<static_cast<unsigned>((nb + kTermWaves - 1) / kTermWaves), kTermWaves * kWave, 0, st>>>(a)));
        if (all.dX != nullptr) XC_LAUNCH(K_DISTILL_GRAD, st, (distill_grad_kernel<T, TO, false><<<chunk_grid, kDistillThreads, 0, st>>>(a, chunks)));
    }
}

}  // namespace xc

extern "C" int xc_distill_workspace(int64_t B, int64_t V, xc_dtype t, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (!softmax_shape(B, V, V)) return XC_ESHAPE;
    *bytes = distill_bytes(B, V, t);
    return XC_OK;
}

extern "C" int xc_distill(const void* X, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature, const int32_t* labels, const float* teacher, int K,
                          int tail, const float* weight, float* loss, void* dX, int64_t ldd, xc_dtype out_t, void* ws, size_t ws_bytes, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (dX != nullptr && out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (!softmax_shape(B, V, ld) || (dX != nullptr && !softmax_shape(B, V, ldd)) || K < 1 || K > XC_MAX_TEACHER) return XC_ESHAPE;
    if (!softmax_temperature(temperature) || (tail != 0 && tail != 1)) return XC_EINVAL;
    if (!X || !labels || !teacher || !loss || !ws) return XC_EINVAL;
    for (const void* p : {X, static_cast<const void*>(labels), static_cast<const void*>(teacher), static_cast<const void*>(weight), static_cast<const void*>(loss),
                          static_cast<const void*>(dX), static_cast<const void*>(ws)})
        if (!aligned16(p)) return XC_EINVAL;
    const size_t need = distill_bytes(B, V, t);
    if (ws_bytes < need) return XC_EWORKSPACE;
    const size_t per = static_cast<size_t>(B) * 4;
    const Span x(X, rows_span(B, V, ld, t)), d(dX, dX != nullptr ? rows_span(B, V, ldd, out_t) : 0);
    const bool in_place = dX == X && t == out_t && ld == ldd;
    if ((!in_place && d.meets(x)) ||
        overlap({Span(loss, per), Span(ws, need)}, {x, d, Span(labels, per * K), Span(teacher, per * K), Span(weight, per)}) ||
        overlap({d}, {Span(labels, per * K), Span(teacher, per * K), Span(weight, per)}))
        return XC_EINVAL;
    const RowCut cut = cut_rows(B, V, t == XC_F32 ? 4 : 2);
    RowTerms* terms = static_cast<RowTerms*>(ws);
    const DistillArgs a{X, labels, teacher, weight, loss, dX, reinterpret_cast<float4*>(terms + B), terms, B, V, ld, ldd, cut.segments, cut.length,
                        temperature, softmax_scale(temperature), K, cut.blocks, tail != 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (t == XC_F32 && (dX == nullptr || out_t == XC_F32)) launch_distill<float, float>(a, cut, st);
    else if (t == XC_F32) launch_distill<float, bf16_t>(a, cut, st);
    else if (dX != nullptr && out_t == XC_F32) launch_distill<bf16_t, float>(a, cut, st);
    else launch_distill<bf16_t, bf16_t>(a, cut, st);
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
