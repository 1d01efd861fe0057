// What the calls on a soft-max over all labels share (xc_logprobs.hip, xc_distill.hip): a row of scores in pieces of 16 aligned bytes,
// and its largest score m with the sums over 2^((x - m) c), c = log2(e) / temperature.
// A thread holds pieces of a row in registers, finds its own largest score, and sums relative to that; lanes, then waves, then the
// workgroups of a row are joined by rescaling.  Differences x - m are formed before they are scaled: x c alone overflows for scores
// near the type's lowest value, which masks are made of.
#pragma once

#include "xc_common.h"

namespace xc {

constexpr float kNone = -INFINITY;       // the score of a label that is not there
constexpr float kFloor = -1000.0f;       // 2^kFloor is 0 in fp32, kFloor * 0 is a number

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __forceinline__ void values(const uint4& v, float (&f)[4]) { __builtin_memcpy(f, &v, 16); }
};
template <> struct Elem<bf16_t> {
    static __device__ __forceinline__ float get(const bf16_t* p) { return bf16_bits_to_float(p->bits); }
    static __device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = static_cast<uint16_t>(float_to_bf16_bits(v)); }
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ void values(const uint4& v, float (&f)[8]) { unpack8(v, f); }
};

// N neighbouring elements at an address that may be any (nearest, ties to even)
typedef float softmax_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 softmax_bf16x2 __attribute__((ext_vector_type(2)));
template <int N> __device__ __forceinline__ void put_elements(float* p, const float (&v)[N]) { __builtin_memcpy(p, v, 4 * N); }
template <int N> __device__ __forceinline__ void put_elements(bf16_t* p, const float (&v)[N]) {
    softmax_bf16x2 h[N / 2];
#pragma unroll
    for (int e = 0; e < N / 2; ++e) h[e] = __builtin_convertvector(softmax_f32x2{v[2 * e], v[2 * e + 1]}, softmax_bf16x2);
    __builtin_memcpy(p, h, 2 * N);
}

// A row of V elements from any address on: whole pieces of 16 aligned bytes, and up to 2 N - 2 elements (edges) before and behind them.
template <typename T>
struct PiecedRow {
    static constexpr int N = 16 / static_cast<int>(sizeof(T));
    const T* p;
    int64_t V, pieces;
    int head, edges;
    __device__ __forceinline__ PiecedRow(const T* row, int64_t V_) : p(row), V(V_) {
        const int past = static_cast<int>(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (N - 1);
        head = past != 0 ? N - past : 0;
        if (head > V) head = static_cast<int>(V);
        pieces = (V - head) / N;
        edges = static_cast<int>(V - pieces * N);
    }
    __device__ __forceinline__ int64_t first(int64_t piece) const { return head + piece * N; }               // its first element
    __device__ __forceinline__ int64_t edge(int i) const { return i < head ? i : pieces * N + i; }
    __device__ __forceinline__ uint4 load(int64_t piece) const { return *reinterpret_cast<const uint4*>(p + first(piece)); }
};

// ---- lanes of a wave, in a fixed order
template <int CTRL, int ROWS>
__device__ __forceinline__ float lanes_from(float x, float none) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane_of(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), kWave - 1)); }
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, lanes_from<0x111, 0xf>(x, kNone));      // row_shr 1, 2, 4, 8
    x = fmaxf(x, lanes_from<0x112, 0xf>(x, kNone));
    x = fmaxf(x, lanes_from<0x114, 0xf>(x, kNone));
    x = fmaxf(x, lanes_from<0x118, 0xf>(x, kNone));
    x = fmaxf(x, lanes_from<0x142, 0xa>(x, kNone));      // row_bcast 15, 31
    x = fmaxf(x, lanes_from<0x143, 0xc>(x, kNone));
    return last_lane_of(x);
}
__device__ __forceinline__ float wave_sum(float x) {
    x += lanes_from<0x111, 0xf>(x, 0.0f);
    x += lanes_from<0x112, 0xf>(x, 0.0f);
    x += lanes_from<0x114, 0xf>(x, 0.0f);
    x += lanes_from<0x118, 0xf>(x, 0.0f);
    x += lanes_from<0x142, 0xa>(x, 0.0f);
    x += lanes_from<0x143, 0xc>(x, 0.0f);
    return last_lane_of(x);
}

// ---- sums
// s = sum of 2^((x - m) c), h = sum of that times (x - m) c; labels that are not there count as nothing in both.  Not a number in s: a
// score that is not a number, or an infinite one.
struct Sums { float m, s, h; };

__device__ __forceinline__ Sums joined(const Sums& a, float m, float c) {       // a's sums relative to m >= a.m
    const float shift = fmaxf((a.m - m) * c, kFloor), f = __builtin_amdgcn_exp2f(shift);
    return Sums{m, a.s * f, fmaf(shift, a.s, a.h) * f};
}

// Of the elements of a thread's C pieces and one more.
template <bool ENTROPY, int C, typename T>
__device__ __forceinline__ Sums thread_sums(const uint4 (&v)[C], float more, float c) {
    constexpr int N = PiecedRow<T>::N;
    float m = fmaxf(kNone, more);
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float f[N];
        Elem<T>::values(v[i], f);
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, f[e]);
    }
    const float base = m == kNone ? 0.0f : m;
    float s[4], h[4];
    {
        const float d = (more - base) * c, x = __builtin_amdgcn_exp2f(d);
        s[0] = x;
        h[0] = x * fmaxf(d, kFloor);
        s[1] = s[2] = s[3] = h[1] = h[2] = h[3] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float f[N];
        Elem<T>::values(v[i], f);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = (f[e] - base) * c, x = __builtin_amdgcn_exp2f(d);
            s[e & 3] += x;
            if constexpr (ENTROPY) h[e & 3] = fmaf(x, fmaxf(d, kFloor), h[e & 3]);
        }
    }
    return Sums{m, (s[0] + s[1]) + (s[2] + s[3]), (h[0] + h[1]) + (h[2] + h[3])};
}
__device__ __forceinline__ Sums wave_sums(const Sums& t, float c) {
    const float m = wave_max(t.m);
    const Sums j = joined(t, m, c);
    return Sums{m, wave_sum(j.s), wave_sum(j.h)};
}
// Of a workgroup of W waves, the same in all threads.  `shared` [W] is free again after the caller's next barrier.
template <int W>
__device__ __forceinline__ Sums block_sums(const Sums& t, float c, Sums* shared) {
    const Sums w = wave_sums(t, c);
    if (lane_id() == 0) shared[threadIdx.x >> 6] = w;
    __syncthreads();
    float m = kNone;
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, shared[i].m);
    Sums r{m, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const Sums j = joined(shared[i], m, c);
        r.s += j.s;
        r.h += j.h;
    }
    return r;
}

// How a call cuts its rows: workgroups of `waves` waves hold `each` pieces per thread; a row is `segments` workgroups' work.
struct RowCut { int waves, each; int64_t segments, length /* pieces of a segment */; };
inline RowCut cut_rows(int64_t B, int64_t V, size_t element) {
    const int64_t pieces = V / static_cast<int64_t>(16 / element);
    const RowCut kinds[4] = {{4, 2, 0, 0}, {8, 2, 0, 0}, {8, 4, 0, 0}, {8, 8, 0, 0}};
    RowCut r{};
    for (const RowCut& k : kinds) {
        r = k;
        const int64_t fit = 64 * k.waves * k.each;
        r.segments = pieces > fit ? (pieces + fit - 1) / fit : 1;
        if (r.segments == 1 || B * r.segments <= 1024) break;
    }
    r.length = r.segments > 1 ? (pieces + r.segments - 1) / r.segments : (pieces > 0 ? pieces : 1);
    return r;
}
constexpr int64_t kSoftmaxGrid = 1 << 24;        // workgroups of a launch at most

inline float softmax_scale(float temperature) { return static_cast<float>(1.4426950408889634 / static_cast<double>(temperature)); }
inline bool softmax_temperature(float t) { return t >= 1e-6f && t <= 1e6f; }
// Sizes of a matrix of rows that lie `ld` elements apart.
inline bool softmax_shape(int64_t B, int64_t V, int64_t ld) {
    return B >= 1 && B <= 0x7fffffffLL && V >= 1 && V <= 0x7fffffffLL && ld >= V && ld <= (1LL << 40) && static_cast<unsigned __int128>(B) * ld <= (1ull << 44);
}
inline unsigned __int128 rows_span(int64_t B, int64_t V, int64_t ld, xc_dtype t) {
    return (static_cast<unsigned __int128>(B - 1) * ld + V) * (t == XC_F32 ? 4 : 2);
}

}  // namespace xc
