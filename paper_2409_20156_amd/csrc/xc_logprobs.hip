// Log probabilities of given labels under the soft-max of all scores, its entropy and its top labels; and the gradient of the first two.
//   logp_v = (x_v - m) / T - log S,  S = sum exp((x_v - m) / T),  H = log S - sum exp((x_v - m) / T) (x_v - m) / T / S
//   dX_v = (sum of dlogp over v's places in the list - p_v (G + dH (logp_v + H))) / T,  G the sum of dlogp
#include "xc_softmax.h"

namespace xc {

constexpr int kTopKeys = 1024;           // candidates that a workgroup ranks at a time
constexpr int kJoinKeys = 2048;

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
    int n, k;
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

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
        const uint32_t t = __shfl_xor(v, off, kWave);
        v = t > v ? t : v;
    }
    return v;
}
__device__ __forceinline__ uint64_t wave_min_u64(uint64_t v) { return ~wave_max_u64(~v); }

constexpr uint32_t kLowest = 0x00800000u;        // ordered image of the lowest number above -inf

// A score (as its ordered image) that at least k of the 64 W largest scores of the threads reach, if as many are there, and that few
// others do: found by halving the range, by one wave.  At least k labels reach it, and no more than those of k or a few more threads.
template <int W>
__device__ __forceinline__ uint32_t reached_by(const float* largest, int k) {
    uint32_t o[W], lo = ~0u, hi = 0u;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        o[w] = float_to_ordered(largest[w * kWave + lane_id()] + 0.0f);
        lo = o[w] < lo ? o[w] : lo;
        hi = o[w] > hi ? o[w] : hi;
    }
    lo = ~wave_max_u32(~lo);
    hi = wave_max_u32(hi) + 1u;
    auto count = [&](uint32_t t) __attribute__((always_inline)) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) n += __popcll(__ballot(o[w] >= t));
        return n;
    };
    if (lo < kLowest) {
        lo = kLowest;
        if (count(lo) <= k) return lo;
    }
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        const int n = count(mid);
        if (n >= k) {
            lo = mid;
            if (n <= k + k / 4 + 3) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// A segment of a row by one workgroup: its sums, and its k best labels.
// The labels: each thread's largest score is known, and a score that k of the threads reach is reached by all k best labels and by few
// others (scores in no particular order: about a seventh more where k is a quarter of the threads).  These are put into LDS and ranked
// by counting.  Where many scores are equal there may be too many of them: then the k-th best is found by halving ranges over all elements.
template <typename T, int W, int C>
__global__ __launch_bounds__(W * kWave)
void logprobs_kernel(const LogprobArgs a) {
    constexpr int N = PiecedRow<T>::N, kThreads = W * kWave;
    __shared__ Sums sums[W];
    __shared__ float largest[kThreads];
    __shared__ uint64_t keys[kTopKeys];
    __shared__ uint32_t reach;
    __shared__ int found, counts[2];
    const int64_t b = blockIdx.x / static_cast<uint32_t>(a.segments), seg = blockIdx.x - b * a.segments;
    const PiecedRow<T> row(static_cast<const T*>(a.X) + b * a.ld, a.V);
    const int64_t first = seg * a.length, end = first + a.length < row.pieces ? first + a.length : row.pieces;
    uint4 v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int64_t at = first + i * kThreads + threadIdx.x;
        v[i] = at < end ? row.load(at) : Elem<T>::none();
    }
    const int64_t edge = seg == 0 && static_cast<int>(threadIdx.x) < row.edges ? row.edge(threadIdx.x) : -1;
    const float more = edge >= 0 ? Elem<T>::get(row.p + edge) : kNone;
    const Sums mine = thread_sums<true, C, T>(v, more, a.c);
    largest[threadIdx.x] = mine.m;
    if (threadIdx.x == 0) found = 0;
    const Sums s = block_sums<W>(mine, a.c, sums);
    const bool alone = a.segments == 1;
    if (alone) write_row<T>(a, b, s);
    else if (threadIdx.x == 0) a.parts[b * a.segments + seg] = make_float4(s.m, s.s, s.h, 0.0f);
    if (a.k == 0) return;

    if (threadIdx.x < kWave) {
        const uint32_t r = reached_by<W>(largest, a.k);
        if (threadIdx.x == 0) reach = r;
    }
    __syncthreads();
    // every element of the thread, with its label
    auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float x[N];
            Elem<T>::values(v[i], x);
            const int32_t id = static_cast<int32_t>(row.first(first + i * kThreads + threadIdx.x));
#pragma unroll
            for (int e = 0; e < N; ++e) f(x[e], id + e);
        }
        f(more, static_cast<int32_t>(edge));
    };
    auto take = [&](float x, int32_t id) __attribute__((always_inline)) {
        const int at = atomicAdd(&found, 1);
        if (at < kTopKeys) keys[at] = make_key(x + 0.0f, id);              // (-0 and 0 are equal)
    };
    const float least = ordered_to_float(reach);
    if (mine.m >= least) each([&](float x, int32_t id) __attribute__((always_inline)) { if (x >= least) take(x, id); });
    __syncthreads();
    if (found > kTopKeys) {                                  // uniform
        auto image = [](float x) __attribute__((always_inline)) { return x == x ? float_to_ordered(x + 0.0f) : 0u; };
        int turn = 0;
        auto count = [&](auto which) __attribute__((always_inline)) {      // of the workgroup's elements
            int n = 0;
            each([&](float x, int32_t id) __attribute__((always_inline)) { n += which(image(x), id) ? 1 : 0; });
#pragma unroll
            for (int off = kWave / 2; off > 0; off >>= 1) n += __shfl_xor(n, off, kWave);
            turn ^= 1;
            if (threadIdx.x == 0) counts[turn] = 0;
            __syncthreads();
            if (lane_id() == 0) atomicAdd(&counts[turn], n);
            __syncthreads();
            return counts[turn];
        };
        uint32_t lo = reach, hi = 0xff800001u;               // (behind infinity)
        while (hi - lo > 1u) {
            const uint32_t mid = lo + (hi - lo) / 2u;
            if (count([&](uint32_t o, int32_t) __attribute__((always_inline)) { return o >= mid; }) >= a.k) lo = mid;
            else hi = mid;
        }
        const int left = a.k - count([&](uint32_t o, int32_t) __attribute__((always_inline)) { return o > lo; });
        int64_t under = -1, last = a.V - 1;                  // of the labels that score lo, the `left` lowest: up to `last`
        while (last - under > 1) {
            const int64_t mid = under + (last - under) / 2;
            if (count([&](uint32_t o, int32_t id) __attribute__((always_inline)) { return o == lo && id <= mid; }) >= left) last = mid;
            else under = mid;
        }
        __syncthreads();
        if (threadIdx.x == 0) found = 0;
        __syncthreads();
        each([&](float x, int32_t id) __attribute__((always_inline)) {
            const uint32_t o = image(x);
            if (o > lo || (o == lo && id <= last)) take(x, id);
        });
        __syncthreads();
    }
    const int n = found;
    const Norm z = norm_of(s);
    uint64_t* out = a.keys + (b * a.segments + seg) * a.k;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t key = keys[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += keys[j] < key ? 1 : 0;
        if (rank < a.k) {
            if (alone) write_top(a, b, rank, key, z);
            else out[rank] = key;
        }
    }
    for (int i = n + threadIdx.x; i < a.k; i += kThreads) {
        if (alone) write_top(a, b, i, kKeySentinel, z);
        else out[i] = kKeySentinel;
    }
}

// The segments of a row joined, by a workgroup per row.  The best labels: of every segment the labels that are no worse than the worst of
// the segments' r-th ones, r = k / segments rounded up (k labels at least are no worse than that), ranked by counting.
constexpr int kJoinWaves = 4;
template <typename T>
__global__ __launch_bounds__(kJoinWaves * kWave)
void logprobs_join_kernel(const LogprobArgs a) {
    __shared__ Sums sums[kJoinWaves];
    __shared__ uint64_t keys[kJoinKeys], best[XC_MAX_TOP];
    __shared__ int found;
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
    const int64_t at_once = (kJoinKeys - a.k) / a.k;
    for (int64_t s0 = 0; s0 < a.segments; s0 += at_once) {
        const int g = static_cast<int>(a.segments - s0 < at_once ? a.segments - s0 : at_once);
        const uint64_t* in = a.keys + (b * a.segments + s0) * a.k;
        uint64_t bound = 0;
        for (int i = lane_id(); i < g; i += kWave) {
            const uint64_t x = in[static_cast<int64_t>(i) * a.k + (a.k + g - 1) / g - 1];
            bound = x > bound ? x : bound;
        }
        bound = wave_max_u64(bound);
        __syncthreads();                                     // (the round before has read its keys)
        for (int i = threadIdx.x; i < have; i += kThreads) keys[i] = best[i];
        if (threadIdx.x == 0) found = have;
        __syncthreads();
        for (int i = threadIdx.x; i < g * a.k; i += kThreads) {
            const uint64_t x = in[i];
            if (x <= bound && x != kKeySentinel) keys[atomicAdd(&found, 1)] = x;
        }
        __syncthreads();
        const int n = found;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t key = keys[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += keys[j] < key ? 1 : 0;
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
        v[i] = at < end ? row.load(at) : make_uint4(0, 0, 0, 0);
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
    const RowCut cut = cut_rows(B, V, t == XC_F32 ? 4 : 2);
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
        auto go = [&](auto kernel, int waves) { XC_LAUNCH(K_LOGPROBS, st, (kernel<<<grid, waves * kWave, 0, st>>>(a))); };
        if (cut.waves == 4) go(logprobs_kernel<T, 4, 2>, 4);
        else if (cut.each == 2) go(logprobs_kernel<T, 8, 2>, 8);
        else if (cut.each == 4) go(logprobs_kernel<T, 8, 4>, 8);
        else go(logprobs_kernel<T, 8, 8>, 8);
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
    const RowCut cut = cut_rows(B, V, t == XC_F32 ? 4 : 2);
    float4* parts = static_cast<float4*>(ws);
    const LogprobArgs a{X, labels, logp, entropy, norm, top, top_logp, parts, reinterpret_cast<uint64_t*>(parts + B * cut.segments), B, V, ld, cut.segments,
                        cut.length, temperature, softmax_scale(temperature), n, k};
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
