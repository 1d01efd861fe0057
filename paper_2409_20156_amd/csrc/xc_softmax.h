// What the calls on a soft-max over all labels share (xc_logprobs.hip, xc_distill.hip): a row of scores in pieces of 16 aligned bytes,
// and its largest score m with the sums over 2^((x - m) c), c = log2(e) / temperature.
// A workgroup goes through its part of a row block by block, the next block's pieces under way; a thread holds a block's elements in
// registers and sums relative to a whole power of two near its own largest score; lanes, then waves, then the workgroups of a row are
// joined by rescaling.
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
    static __device__ __forceinline__ float value(const uint4& v, int e) { return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w); }
};
template <> struct Elem<bf16_t> {
    static __device__ __forceinline__ float get(const bf16_t* p) { return bf16_bits_to_float(p->bits); }
    static __device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = static_cast<uint16_t>(float_to_bf16_bits(v)); }
    static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ void values(const uint4& v, float (&f)[8]) { unpack8(v, f); }
    static __device__ __forceinline__ float value(const uint4& v, int e) {
        const uint32_t two = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __uint_as_float((e & 1) != 0 ? two & 0xffff0000u : two << 16);
    }
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
    // STREAM: with the non-temporal hint, for rows that a kernel reads once.  1024 x 131072 bf16: log probabilities and gradient 157 us
    // without, 140 with it, the loss against a teacher and its gradient 166 and 154.
    template <bool STREAM> __device__ __forceinline__ uint4 load(int64_t piece) const { return load16<STREAM>(p + first(piece)); }
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

// A block of a row in a thread's registers: C pieces, every `threads`-th of the block.
template <typename T, int C>
struct Block {
    static constexpr int N = PiecedRow<T>::N, E = C * N;
    uint4 v[C];
    template <bool STREAM> __device__ __forceinline__ void load(const PiecedRow<T>& row, int64_t first, int64_t end, int threads) {
        if (first + C * threads <= end) {                    // uniform: nothing to form for each piece but an offset
            const uint4* p = reinterpret_cast<const uint4*>(row.p + row.first(first));
#pragma unroll
            for (int i = 0; i < C; ++i) v[i] = load16<STREAM>(p + (static_cast<uint32_t>(threadIdx.x) + i * threads));
            return;
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int64_t at = first + i * threads + threadIdx.x;
            v[i] = at < end ? row.template load<STREAM>(at) : Elem<T>::none();
        }
    }
    __device__ __forceinline__ void values(float (&f)[E]) const {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float x[N];
            Elem<T>::values(v[i], x);
#pragma unroll
            for (int e = 0; e < N; ++e) f[i * N + e] = x[e];
        }
    }
};

// A thread's sums over its blocks.  Where |m c| is below 2^20, exponents are x c - k with a whole k near m c: one fused multiply-add with
// no rounding but its own, and rescaling by whole powers of two.  Beyond that (masks of the type's lowest value, say) x c may overflow:
// the difference x - m is formed first, in sums of their own.
struct Running {
    float m = kNone, k = -4194304.0f, s = 0.0f, h = 0.0f;
    Sums far{kNone, 0.0f, 0.0f};

    template <bool ENTROPY, int E>
    __device__ __forceinline__ void add(const float (&f)[E], float most /* the largest of f */, float c) {
        static_assert(E % 8 == 0, "");
        m = fmaxf(m, most);
        if (__builtin_expect(fabsf(most * c) < 1048576.0f, 1)) {
            const float kb = rintf(most * c);
            if (kb > k) {
                const float shift = k - kb, by = __builtin_amdgcn_exp2f(shift);
                h = fmaf(shift, s, h) * by;
                s *= by;
                k = kb;
            }
            float sum = 0.0f, weighted = 0.0f;
#pragma unroll
            for (int i = 0; i < E; i += 8) {
                float d[8], x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = fmaf(f[i + e], c, -k);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(d[e]);
                sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                if constexpr (ENTROPY) {                     // (0 times -infinity, of a label that is not there, is no number)
                    float w[2] = {x[0] * fmaxf(d[0], kFloor), x[4] * fmaxf(d[4], kFloor)};
#pragma unroll
                    for (int e = 1; e < 4; ++e) {
                        w[0] = fmaf(x[e], fmaxf(d[e], kFloor), w[0]);
                        w[1] = fmaf(x[4 + e], fmaxf(d[4 + e], kFloor), w[1]);
                    }
                    weighted += w[0] + w[1];
                }
            }
            s += sum;
            h += weighted;
        } else {
            const float base = most == kNone ? 0.0f : most;
            Sums t{most, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = (f[e] - base) * c, x = __builtin_amdgcn_exp2f(d);
                t.s += x;
                if constexpr (ENTROPY) t.h = fmaf(x, fmaxf(d, kFloor), t.h);
            }
            const float both = fmaxf(far.m, most);
            const Sums u = joined(far, both, c), w = joined(t, both, c);
            far = Sums{both, u.s + w.s, u.h + w.h};
        }
    }
    // One element by itself.
    __device__ __forceinline__ void add_one(float x, float c) {
        m = fmaxf(m, x);
        const float both = fmaxf(far.m, x);
        const Sums u = joined(far, both, c), w = joined(Sums{x, __builtin_amdgcn_exp2f(x == kNone ? kNone : x - x), 0.0f}, both, c);
        far = Sums{both, u.s + w.s, u.h + w.h};
    }
    // All of them relative to m.
    __device__ __forceinline__ Sums sums(float c) const {
        const float shift = s == 0.0f ? kFloor : fmaxf(fmaf(-m, c, k), kFloor), by = __builtin_amdgcn_exp2f(shift);      // (s = 0: no block's)
        const Sums u = joined(far, m, c);
        return Sums{m, fmaf(s, by, u.s), fmaf(fmaf(shift, s, h), by, u.h)};
    }
};
// The largest of N neighbouring elements of f.
template <int N, int E>
__device__ __forceinline__ float largest_of(const float (&f)[E], int first) {
    float m = kNone;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, f[first + e]);
    return m;
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

// How a call cuts its rows: a workgroup of kRowWaves waves goes through `blocks` blocks of kRowThreads * each pieces; a row is `segments`
// workgroups' work.
constexpr int kRowWaves = 4, kRowThreads = kRowWaves * kWave;
constexpr int small_block(size_t element) { return element == 4 ? 2 : 1; }        // pieces to a thread: 8 elements,
constexpr int large_block(size_t) { return 4; }                                  // 16 (fp32), 32
struct RowCut { int each, blocks; int64_t segments, length /* pieces of a segment */; };
// Segments: as many as give every compute unit several workgroups, of about 4096 elements at least (8 x 131072 fp32 with 20 top labels 13.8 us,
// of 2048 15.1; their number is rounded up, so that just beyond a multiple they are shorter: 4100 elements are two of 2052), and no more than the
// kernel that joins them has room for all top labels of (1 x 262144 bf16, 128 labels: 16 segments 25 us; 128 of them, joined in rounds by
// a thread to a key, 102 where 16 took 30).  It takes 128 segments at a time: with fewer than 16 top labels there may be more, in rounds.
constexpr int kJoinKeys = 2048;
inline RowCut cut_rows(int64_t B, int64_t V, size_t element, int k = 0) {
    const int64_t pieces = V / static_cast<int64_t>(16 / element);
    const int small = small_block(element), large = large_block(element);
    RowCut r{};
    const int64_t wanted = 1024;                                           // workgroups
    int64_t segments = B >= wanted / 2 ? 1 : wanted / B;
    const int64_t most = (pieces + 2 * kRowThreads * small - 1) / (2 * kRowThreads * small);
    if (segments > most) segments = most;
    if (k > 0 && segments > kJoinKeys / k) segments = kJoinKeys / k;
    if (pieces <= kRowThreads * large || segments < 1) segments = 1;
    r.length = pieces > 0 ? (pieces + segments - 1) / segments : 1;
    r.segments = pieces > 0 ? (pieces + r.length - 1) / r.length : 1;
    r.each = r.length <= kRowThreads * small ? small : large;
    r.blocks = static_cast<int>((r.length + kRowThreads * r.each - 1) / (kRowThreads * r.each));
    return r;
}
constexpr int64_t kSoftmaxGrid = 1 << 21;        // workgroups of a launch at most (of 1024 threads at most: a launch of 2^32 threads is refused)

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
