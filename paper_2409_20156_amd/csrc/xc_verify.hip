// The check of drafted labels against the classifier's probabilities, and the draw of the label behind the last one that
// stands.  Only the rows that decide are read: two values per draft, then one row of the target (and of the draft where one fell).
#include "xc_common.h"

namespace xc {

constexpr int kVerifyThreads = 256;
constexpr int kPiece = 512;              // elements of a wave's step: 8 neighbouring ones per lane
constexpr int kChunk = 4096;             // elements of a partial sum, whatever the launch

struct VerifyArgs {
    const int32_t* drafts;
    const void* target;
    const void* draft;                   // null: looked-up drafts
    const float* u;
    int32_t* tokens;
    int32_t* accepted;
    double* sums;                        // [B][n_chunks]
    int64_t V;
    int n, n_chunks;
};

template <typename T> __device__ __forceinline__ float prob(const T* p);
template <> __device__ __forceinline__ float prob<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float prob<bf16_t>(const bf16_t* p) { return bf16_bits_to_float(p->bits); }

enum Weights { kTarget, kDifference, kWithout };

// How far the drafts of sequence b stand; every wave finds out for itself.
struct Verdict { int a; bool fell; int32_t x; };
template <typename T>
__device__ __forceinline__ Verdict judge(const VerifyArgs& v, int64_t b) {
    const int lane = lane_id();
    for (int i0 = 0; i0 < v.n; i0 += kWave) {
        const int i = i0 + lane;
        const int32_t x = i < v.n ? v.drafts[b * v.n + i] : -1;
        const bool there = x >= 0 && x < v.V;
        bool stands = false;
        if (there) {
            // (the product of two fp32 numbers is exact in 64 bits)
            const double p = prob(static_cast<const T*>(v.target) + (b * (v.n + 1) + i) * v.V + x);
            const double q = v.draft != nullptr ? static_cast<double>(prob(static_cast<const T*>(v.draft) + (b * v.n + i) * v.V + x)) : 1.0;
            stands = static_cast<double>(v.u[b * (v.n + 1) + i]) * q < p;
        }
        const uint64_t down = __ballot(!stands);
        if (down != 0ull) {
            const int f = __ffsll(static_cast<long long>(down)) - 1;
            return Verdict{i0 + f, ((__ballot(there) >> f) & 1ull) != 0ull, __shfl(x, f, kWave)};
        }
    }
    return Verdict{v.n, false, -1};
}

// The weights of elements e .. e + 7 of a row.
template <typename T>
__device__ __forceinline__ void weights8(const T* p, const T* q, Weights kind, int32_t without, int64_t e, int64_t V, double (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = 0.0;
        if (e + i < V) {
            double x = prob(p + e + i);
            if (kind == kDifference) x -= static_cast<double>(prob(q + e + i));
            if (kind == kWithout && e + i == without) x = 0.0;
            w[i] = x > 0.0 && x < static_cast<double>(INFINITY) ? x : 0.0;
        }
    }
}
__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
    return s;
}
__device__ __forceinline__ double wave_incl_scan(double s) {
    const int lane = lane_id();
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double t = __shfl_up(s, off, kWave);
        if (lane >= off) s += t;
    }
    return s;
}

// Sum of chunk c, the same in all lanes: 8 pieces per lane, then the lanes.
template <typename T>
__device__ __forceinline__ double chunk_sum(const T* p, const T* q, Weights kind, int32_t without, int c, int64_t V) {
    double s = 0.0;
    for (int k = 0; k < kChunk; k += kPiece) {
        double w[8];
        weights8(p, q, kind, without, static_cast<int64_t>(c) * kChunk + k + lane_id() * 8, V, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += w[i];
    }
    return wave_sum(s);
}

// First element of chunk c at which the running sum, `before` ahead of the chunk, passes t; else the last one with a weight.
template <typename T>
__device__ __forceinline__ int32_t find_in_chunk(const T* p, const T* q, Weights kind, int32_t without, int c, int64_t V, double before, double t) {
    int32_t last = -1;
    for (int k = 0; k < kChunk; k += kPiece) {
        const int64_t e = static_cast<int64_t>(c) * kChunk + k + lane_id() * 8;
        double w[8], s = 0.0;
        weights8(p, q, kind, without, e, V, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += w[i];
        const double incl = wave_incl_scan(s);
        double run = before + (incl - s);
        int32_t here = -1, mine = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            run += w[i];
            if (w[i] > 0.0) {
                mine = static_cast<int32_t>(e + i);
                if (here < 0 && run > t) here = mine;
            }
        }
        // the first lane whose own sum passes t decides; its elements' running sum may stay below by a rounding: its last one then
        const uint64_t pass = __ballot(s > 0.0 && before + incl > t);
        if (pass != 0ull) return __shfl(here >= 0 ? here : mine, __ffsll(static_cast<long long>(pass)) - 1, kWave);
        const uint64_t some = __ballot(mine >= 0);
        if (some != 0ull) last = __shfl(mine, 63 - __clzll(static_cast<long long>(some)), kWave);
        before += __shfl(incl, kWave - 1, kWave);
    }
    return last;
}

// The label drawn, by one wave from the chunks' sums.  -1 if all weights are zero.
template <typename T>
__device__ __forceinline__ int32_t draw_label(const VerifyArgs& v, const double* sums, const T* p, const T* q, Weights kind, int32_t without, float u) {
    const int lane = lane_id();
    double total = 0.0;
    for (int c0 = 0; c0 < v.n_chunks; c0 += kWave) {
        const double s = c0 + lane < v.n_chunks ? sums[c0 + lane] : 0.0;
        total += __shfl(wave_incl_scan(s), kWave - 1, kWave);
    }
    if (!(total > 0.0)) return -1;
    const double t = static_cast<double>(u) * total;
    double before = 0.0, last_before = 0.0;
    int chunk = -1;
    for (int c0 = 0; c0 < v.n_chunks; c0 += kWave) {
        const double s = c0 + lane < v.n_chunks ? sums[c0 + lane] : 0.0;
        const double incl = wave_incl_scan(s);
        const uint64_t some = __ballot(s > 0.0), pass = __ballot(s > 0.0 && before + incl > t);
        const uint64_t take = pass != 0ull ? pass & (~pass + 1ull) : some;
        if (take != 0ull) {              // (no chunk passes: the last with a weight)
            const int f = 63 - __clzll(static_cast<long long>(take));
            chunk = c0 + f;
            last_before = before + __shfl(incl - s, f, kWave);
        }
        if (pass != 0ull) break;
        before += __shfl(incl, kWave - 1, kWave);
    }
    return find_in_chunk(p, q, kind, without, chunk, v.V, last_before, t);
}

template <typename T>
__global__ __launch_bounds__(kVerifyThreads)
void verify_kernel(const VerifyArgs v) {
    const int64_t b = blockIdx.x;
    const int wave = threadIdx.x >> 6;
    __shared__ int32_t drawn;
    const Verdict j = judge<T>(v, b);
    const T* p = static_cast<const T*>(v.target) + (b * (v.n + 1) + j.a) * v.V;
    const T* q = v.draft != nullptr ? static_cast<const T*>(v.draft) + (b * v.n + j.a) * v.V : nullptr;
    double* sums = v.sums + b * v.n_chunks;
    Weights kind = !j.fell ? kTarget : v.draft != nullptr ? kDifference : kWithout;
    for (;;) {
        for (int c = wave; c < v.n_chunks; c += kVerifyThreads / kWave) {
            const double s = chunk_sum(p, q, kind, j.x, c, v.V);
            if (lane_id() == 0) sums[c] = s;
        }
        __syncthreads();
        if (wave == 0) {
            const int32_t l = draw_label(v, sums, p, q, kind, j.x, v.u[b * (v.n + 1) + v.n]);
            if (lane_id() == 0) drawn = l;
        }
        __syncthreads();
        if (drawn >= 0 || kind == kTarget) break;
        kind = kTarget;                  // nothing is left of the target above the draft: the target itself
        __syncthreads();
    }
    for (int i = threadIdx.x; i <= v.n; i += kVerifyThreads)
        v.tokens[b * (v.n + 1) + i] = i < j.a ? v.drafts[b * v.n + i] : i == j.a ? drawn : -1;
    if (threadIdx.x == 0) v.accepted[b] = j.a;
}

static int verify_chunks(int64_t V) { return static_cast<int>((V + kChunk - 1) / kChunk); }

}  // namespace xc

extern "C" int xc_verify_workspace(int64_t B, int64_t V, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (B < 1 || B > 0x7fffffffLL || V < 1 || V > 0x7fffffffLL) return XC_ESHAPE;
    *bytes = static_cast<size_t>(B) * verify_chunks(V) * sizeof(double);
    return XC_OK;
}

extern "C" int xc_verify_drafts(const int32_t* drafts, int64_t B, int n, int64_t V, const void* target, const void* draft_probs,
                                xc_dtype t, const float* u, int32_t* tokens, int32_t* accepted, void* ws, size_t ws_bytes,
                                void* stream) {
    using namespace xc;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (B < 1 || B > 0x7fffffffLL || n < 0 || n > XC_MAX_DRAFTS || V < 1 || V > 0x7fffffffLL) return XC_ESHAPE;
    if ((!drafts && n > 0) || !target || !u || !tokens || !accepted || !ws) return XC_EINVAL;
    if (!aligned16(drafts) || !aligned16(target) || !aligned16(draft_probs) || !aligned16(u) || !aligned16(tokens) ||
        !aligned16(accepted) || !aligned16(ws))
        return XC_EINVAL;
    VerifyArgs v{drafts, target, draft_probs, u, tokens, accepted, static_cast<double*>(ws), V, n, verify_chunks(V)};
    if (ws_bytes < static_cast<size_t>(B) * v.n_chunks * sizeof(double)) return XC_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (t == XC_F32)
        XC_LAUNCH(K_VERIFY, st, (verify_kernel<float><<<static_cast<unsigned>(B), kVerifyThreads, 0, st>>>(v)));
    else
        XC_LAUNCH(K_VERIFY, st, (verify_kernel<bf16_t><<<static_cast<unsigned>(B), kVerifyThreads, 0, st>>>(v)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
