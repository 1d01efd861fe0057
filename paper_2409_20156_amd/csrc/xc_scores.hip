// Rows in 8 bits, and the scores of all labels from them: out = (<p, q> a) b with integers p, q and a scale per row on
// either side.  The integer sums are exact, so their order (and how the work is cut) cannot change a score.
#include "xc_mine.h"
#include "xc_scores_choice.h"

namespace xc {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ inline int quantized_pitch(int d) { return (d + 15) & ~15; }

// ---------------------------------------------------------------------------
// rows -> integers
// ---------------------------------------------------------------------------
// 127 x / m to the nearest integer, halves to even.  The fp32 product is off by less than 127 * 2^-23; where it comes near
// a half, 254 x is compared with (2 k + 1) m, both exact in 64 bits.
__device__ __forceinline__ int to_integer(float x, float m, float inv) {
    const float v = x * inv;
    float r = rintf(v);
    if (__builtin_expect(fabsf(fabsf(v - r) - 0.5f) < 1e-4f, 0)) {
        const float k = floorf(v);
        const double lhs = static_cast<double>(x) * 254.0, rhs = static_cast<double>(2.0f * k + 1.0f) * static_cast<double>(m);
        r = lhs > rhs ? k + 1.0f : lhs < rhs ? k : 2.0f * rintf(0.5f * k + 0.25f);
    }
    return static_cast<int>(r);
}
// What a row's largest magnitude m (as bits; all ones beyond infinity count as larger) makes of the row.
struct RowScale {
    float m, inv, up, scale;             // elements are multiplied by `up` first (2^100 for rows of tiny elements, whose inverse overflows)
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits) {
    RowScale r;
    const float m = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u, tiny = m < 7.888609052210118e-31f /* 2^-100 */;
    r.up = tiny ? 1.2676506002282294e30f : 1.0f;
    r.m = m * r.up;
    r.inv = finite && bits != 0u ? 127.0f / r.m : 0.0f;
    r.scale = finite ? m / 127.0f : __uint_as_float(0x7fc00000u);
    return r;
}

// 8 neighbouring elements of a row.
template <typename T> struct Eight;
template <> struct Eight<float> {
    uint4 v[2];
    __device__ __forceinline__ void zero() { v[0] = v[1] = make_uint4(0, 0, 0, 0); }
    template <bool STREAM> __device__ __forceinline__ void load(const unsigned char* row, int e, int d) {
        v[0] = load16<STREAM>(row + e * 4);
        if (e + 4 < d) v[1] = load16<STREAM>(row + e * 4 + 16);                          // (d is a multiple of 4)
    }
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t x[4] = {v[i].x & 0x7fffffffu, v[i].y & 0x7fffffffu, v[i].z & 0x7fffffffu, v[i].w & 0x7fffffffu};
#pragma unroll
            for (int e = 0; e < 4; ++e) m = x[e] > m ? x[e] : m;
        }
        return m;
    }
    __device__ __forceinline__ void values(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[4 * i] = __uint_as_float(v[i].x); f[4 * i + 1] = __uint_as_float(v[i].y);
            f[4 * i + 2] = __uint_as_float(v[i].z); f[4 * i + 3] = __uint_as_float(v[i].w);
        }
    }
};
template <> struct Eight<bf16_t> {
    uint4 v;
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    template <bool STREAM> __device__ __forceinline__ void load(const unsigned char* row, int e, int) { v = load16<STREAM>(row + e * 2); }
    __device__ __forceinline__ uint32_t largest() const {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        const uint32_t u[4] = {v.x & 0x7fff7fffu, v.y & 0x7fff7fffu, v.z & 0x7fff7fffu, v.w & 0x7fff7fffu};
        u16x2 x[4];
        __builtin_memcpy(x, u, 16);
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(x[0], x[1]), __builtin_elementwise_max(x[2], x[3]));
        return static_cast<uint32_t>(m.x > m.y ? m.x : m.y) << 16;
    }
    __device__ __forceinline__ void values(float (&f)[8]) const { unpack8(v, f); }
};

// 8 elements -> 8 integers.  Adding 1.5 * 2^23 leaves the nearest integer in the low bits; where any of the 8 comes near a
// half, all are decided exactly.
__device__ __forceinline__ uint2 to_integers(float (&f)[8], const RowScale& s) {
    constexpr float kMagic = 12582912.0f;
    if (s.up != 1.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= s.up;
    }
    uint32_t b[8];
    float off = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = fmaf(f[e], s.inv, kMagic);
        off = fmaxf(off, fabsf(fmaf(f[e], s.inv, kMagic - r)));
        b[e] = __float_as_uint(r);
    }
    if (__builtin_expect(off > 0.5f - 1e-4f, 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = static_cast<uint32_t>(to_integer(f[e], s.m, s.inv));
    }
    uint2 o;
    o.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
    o.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[7], b[6], 0x0c0c0400u), __builtin_amdgcn_perm(b[5], b[4], 0x0c0c0400u), 0x05040100u);
    return o;
}

// 2^lg lanes per row, which they hold in registers: C groups of 8 elements each, read once.  C = 0: rows of more than 4096
// elements, one wave per row, read twice.  Bound: memory, one read and half a write per bf16 element.  670000 x 768 bf16: 254 us,
// 6.1 TB/s; without the non-temporal hint, which rows beyond the last-level cache are loaded with, 276; a form that read rows twice,
// rounded by rint and stored bytes 501.  The 413 716 rows that a step on 670000 x 768 touched, by their list: 155 us, 6.2 TB/s.
constexpr int64_t kCachedBytes = 256ll << 20;
template <typename T, int C>
__global__ __launch_bounds__(256)
void quantize_kernel(const unsigned char* __restrict__ X, int64_t N, int d, const int32_t* __restrict__ ids, int64_t m,
                     const int32_t* __restrict__ count, int8_t* __restrict__ Q, int pitch, float* __restrict__ scale, int lg, bool stream) {
    const int lane = lane_id(), per = 1 << lg, sub = lane & (per - 1);
    const int64_t row_bytes = static_cast<int64_t>(d) * (sizeof(T) == 4 ? 4 : 2);
    int64_t rows = ids != nullptr ? m : N;
    if (ids != nullptr && count != nullptr) {
        const int64_t c = count[0];
        rows = c < rows ? c : rows;
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * 4 << (6 - lg);
    for (int64_t i = ((static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6)) << (6 - lg)) + (lane >> lg); i < rows; i += step) {
        const int64_t row = ids != nullptr ? ids[i] : i;
        if (row < 0 || row >= N) continue;               // (lanes of a row leave together)
        const unsigned char* src = X + row * row_bytes;
        int8_t* dst = Q + row * pitch;
        uint32_t big = 0;
        Eight<T> v[C > 0 ? C : 1];
        if constexpr (C > 0) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                v[c].zero();
                const int e = ((c << lg) + sub) * 8;
                if (e < d) {
                    if (stream) v[c].template load<true>(src, e, d);                   // uniform
                    else v[c].template load<false>(src, e, d);
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) { const uint32_t b = v[c].largest(); big = b > big ? b : big; }
        } else {
            for (int e = sub * 8; e < d; e += 8 << lg) {
                v[0].zero();
                v[0].template load<false>(src, e, d);
                const uint32_t b = v[0].largest();
                big = b > big ? b : big;
            }
        }
        for (int off = per >> 1; off > 0; off >>= 1) { const uint32_t o = __shfl_xor(big, off, kWave); big = o > big ? o : big; }
        const RowScale s = row_scale(big);
        auto put = [&](const Eight<T>& x, int e) __attribute__((always_inline)) {
            float f[8];
            x.values(f);
            const uint2 o = to_integers(f, s);
            *reinterpret_cast<uint2*>(dst + e) = s.inv == 0.0f ? make_uint2(0, 0) : o;
        };
        if constexpr (C > 0) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = ((c << lg) + sub) * 8;
                if (e < pitch) put(v[c], e);
            }
        } else {
            for (int e = sub * 8; e < pitch; e += 8 << lg) {
                v[0].zero();
                if (e < d) v[0].template load<false>(src, e, d);
                put(v[0], e);
            }
        }
        if (sub == 0) scale[row] = s.scale;
    }
}

template <typename T>
static void launch_quantize_kernel(const unsigned char* X, int64_t N, int d, const int32_t* ids, int64_t m, const int32_t* count,
                                   int8_t* Q, int pitch, float* scale, hipStream_t st) {
    const int64_t rows = ids != nullptr ? m : N;
    // lanes per row and groups of 8 per lane: as few lanes as hold the row, unless that leaves more of them idle
    const int groups = (pitch + 7) / 8;
    int lg = 6, C = 0, best = 1 << 30;
    for (int c : {1, 2, 3, 4, 6, 8}) {
        int g = 2;
        while (g < 6 && (c << g) < groups) ++g;
        if ((c << g) >= groups && (c << g) < best) { best = c << g; lg = g; C = c; }
    }
    const int64_t want = (rows + (4 << (6 - lg)) - 1) / (4 << (6 - lg));
    const unsigned grid = static_cast<unsigned>(want < 32768 ? want : 32768);
    const bool stream = rows * d * static_cast<int64_t>(sizeof(T) == 4 ? 4 : 2) > kCachedBytes;
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(X, N, d, ids, m, count, Q, pitch, scale, lg, stream); };
    switch (C) {
        case 1: go(quantize_kernel<T, 1>); break;
        case 2: go(quantize_kernel<T, 2>); break;
        case 3: go(quantize_kernel<T, 3>); break;
        case 4: go(quantize_kernel<T, 4>); break;
        case 6: go(quantize_kernel<T, 6>); break;
        case 8: go(quantize_kernel<T, 8>); break;
        default: go(quantize_kernel<T, 0>); break;
    }
}

static int launch_quantize(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count,
                           int8_t* Q, int pitch, float* scale, hipStream_t st) {
    const unsigned char* x = static_cast<const unsigned char*>(X);
    if (t == XC_F32) XC_LAUNCH(K_QUANTIZE, st, launch_quantize_kernel<float>(x, N, d, ids, m, count, Q, pitch, scale, st));
    else XC_LAUNCH(K_QUANTIZE, st, launch_quantize_kernel<bf16_t>(x, N, d, ids, m, count, Q, pitch, scale, st));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
// Tiles of BM queries x BN labels, K staged 128 bytes of each row at a time through a ring of R stages in LDS (direct
// global -> LDS loads).  WQ x WL waves, each with MQ x ML blocks of v_mfma_i32_16x16x64_i8.
// LDS rows are unpadded, their 16-byte chunks stored at chunk ^ swizzle(row) so that 16 lanes reading one chunk of 16 rows
// meet all banks.  Blocks of labels are interleaved, V at a time, so that a lane ends up with V neighbouring labels, 16
// bytes of scores where there are as many: label V j + v of a group of 16 V is column j of its block v.
// Accumulator i of a lane: query 4 (lane / 16) + i of its block, column lane % 16.
// A persistent workgroup takes its tiles one after the other with the loads running ahead into the next, so a tile's scores are
// stored while the next one's operands arrive; the waits count loads and stores, which retire in the order of their issue.
// Bound: few queries, the rows of Q (1 x 131072 x 768: 18.0 us in the kernel where they come from memory, 5.6 TB/s, 15.9 to 17.1
// where one call after the other reads the same 100 MB, part of which the last-level cache still holds; 64 x 670000 x 768, which
// also stores 86 MB: 121 us, 5.0 TB/s); many, what brings both operands through LDS and the clock that the chip's power limit
// allows (4096 x 100000 x 4096: 1.33 ms, 2.5 POP/s; the library's product of 8192^3 integers runs at 2.1); rows beyond 768 bytes to
// fp32, the stores of a 256 x 256 tile, which the loads of the next tile wait for (1440 x 164990 x 1472: 595 us, matrix pipe busy
// 27 % of the time, 905 MB read and 985 written).  256 x 256 tiles spill 14 registers; their reloads lie in the way of tiles that
// reach past the end.  Measured on 4096 x 131072 x 768 to bf16 (us): tiles of 128 x 256, one a workgroup, 813; epilogue on packed
// conversions and scales held ready 670; 256 x 256 602; persistent 570; stages brought in by half of the waves in turn, the others
// at their products already, 550; 16 x 16 products, whose lanes end up with 16 bytes of scores, 540.  Of that the stores took 140,
// the loads 100.
template <int WQ_, int WL_, int MQ_, int ML_, int R_, int G_, int RES_ = 0>
struct Tile {
    static constexpr int WQ = WQ_, WL = WL_, MQ = MQ_, ML = ML_, R = R_;
    static constexpr int G = G_;         // groups of waves that bring in the stages in turn
    static constexpr int RES = RES_;     // bytes of a query's row in LDS for good, brought to integers by the workgroup itself (0: staged like the labels)
    static constexpr int kWaves = WQ * WL, kThreads = 64 * kWaves, BM = 16 * WQ * MQ, BN = 16 * WL * ML;
    static constexpr int kStageRows = (RES > 0 ? 0 : BM) + BN, kStage = kStageRows * kStageBytes;
    static constexpr int kScaleLinesL = (BN + 63) / 64, kScaleLinesQ = RES > 0 ? 0 : (BM + 63) / 64;        // of 64 scales
    static constexpr int kScales = (kScaleLinesL + kScaleLinesQ) * 256;
    static constexpr int kLds = R * kStage + (R + 1) * kScales + (RES > 0 ? BM * (RES + 4) : 0);
    static constexpr int kPerCu = 160 * 1024 / kLds < 8 / kWaves ? 160 * 1024 / kLds : 8 / kWaves;           // workgroups of a compute unit
    static constexpr int kPerSimd = kPerCu * kWaves < 8 ? 1 : 2;
    // a wave's loads of a stage: 8 rows each
    static constexpr int kIssue = kWaves / G, kLoadsA = RES > 0 ? 0 : BM / 8 / kIssue, kLoadsB = BN / 8 / kIssue, kLoads = kLoadsA + kLoadsB;
    static_assert((RES > 0 || kLoadsA * 8 * kIssue == BM) && kLoadsB * 8 * kIssue == BN, "loads divide evenly among the waves");
};
__device__ __forceinline__ int row_swizzle(int row) { return (row >> 1) & 7; }

struct ScoresArgs {
    const unsigned char* Z;              // queries as they came, rows of d elements (tiles that bring them to integers themselves)
    int d;
    const int8_t* P;                     // queries in 8 bits, rows of ppitch bytes (zeros from column d on)
    const float* pscale;
    const int8_t* Q;
    const float* scale;
    void* out;
    int64_t B, L;
    int pitch, ppitch;                   // bytes of a row of Q, of P (whole stages)
    int tiles_m, tiles_n, group;         // tiles of queries that are taken together, label tile by label tile
};

// N neighbouring scores, all of them there
template <int N> __device__ __forceinline__ void store_labels(float* p, const float (&v)[N]) { __builtin_memcpy(p, v, 4 * N); }
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <int N> __device__ __forceinline__ void store_labels(bf16_t* p, const float (&v)[N]) {
    bf16x2 h[(N + 1) / 2];
#pragma unroll
    for (int e = 0; e < (N + 1) / 2; ++e) h[e] = __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1 < N ? 2 * e + 1 : 2 * e]}, bf16x2);      // nearest, ties to even
    __builtin_memcpy(p, h, 2 * N);
}
__device__ __forceinline__ void store_label(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_label(bf16_t* p, float v) {
    const __bf16 h = static_cast<__bf16>(v);
    __builtin_memcpy(p, &h, 2);
}

__device__ __forceinline__ void lds_dma4(const void* gptr, uint32_t lds_addr /* wave-uniform */) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(gptr), "s"(lds_addr) : "memory");
}
// Rows of whole lines that a call reads once: marked for early replacement.  In the kernel, from memory: 1 x 131072 x 768 20.1 ->
// 18.0 us, 32 x 131072 x 768 22.7 -> 20.8, 1 x 670000 x 768 91 -> 78, 64 x 670000 x 768 126 -> 117, 64 x 3 M x 256 228 -> 236;
// where one call after the other reads the same 100 MB, part of which the last-level cache holds, 1 query 16.4 -> 15.9, 32 queries
// 18.4 -> 19.8.  Not where two loads share a line, of which the second would find nothing left: 126 x 441376 x 776 185 us with the
// hint, 146 without; 32 x 600000 x 304 77 and 59.
template <bool STREAM>
__device__ __forceinline__ void load_labels(const void* sbase, uint32_t voff, uint32_t lds_addr) {
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" :: "v"(voff), "s"(sbase), "s"(lds_addr) : "memory");
    else
        lds_dma16_sbase<0>(sbase, voff, lds_addr);
}
__device__ __forceinline__ const void* uniform_ptr(const void* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const void*>(
        (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32)))) << 32) |
        static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a)))));
}

template <typename TO, typename T, bool STREAM, typename TZ = float>
__global__ __launch_bounds__(T::kThreads, T::kPerSimd)
void scores_kernel(const ScoresArgs a) {
    __shared__ __align__(1024) unsigned char smem[T::kLds];
    constexpr int V = T::ML < 16 / static_cast<int>(sizeof(TO)) ? T::ML : 16 / static_cast<int>(sizeof(TO));
    const int lane = lane_id(), quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wq = wave / T::WL, wl = wave % T::WL;
    const int wi = wave % T::kIssue, my_turn = wave / T::kIssue;      // stages n with n % G == my_turn are this wave's to bring in
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));

    // workgroup w runs on XCD w % 8: each XCD takes a contiguous part of the tiles, in an order that keeps a group of query
    // tiles in its L2 while the labels pass
    const uint32_t n_tiles = static_cast<uint32_t>(a.tiles_m) * static_cast<uint32_t>(a.tiles_n), per = (n_tiles + 7) / 8;
    const uint32_t t_begin = blockIdx.x % 8 * per, t_end = t_begin + per < n_tiles ? t_begin + per : n_tiles;
    const uint32_t t_first = t_begin + blockIdx.x / 8, t_step = gridDim.x / 8;
    if (t_first >= t_end) return;
    const int n_stages = (a.pitch + kStageBytes - 1) / kStageBytes;
    const int total = static_cast<int>((t_end - 1 - t_first) / t_step + 1) * n_stages;
    auto place = [&](uint32_t t, int64_t& q0, int64_t& l0) __attribute__((always_inline)) {
        const uint32_t in_groups = static_cast<uint32_t>(a.group) * static_cast<uint32_t>(a.tiles_n);
        const uint32_t g = t / in_groups, r = t - g * in_groups, m0 = g * a.group;
        const uint32_t gm = a.tiles_m - m0 < static_cast<uint32_t>(a.group) ? a.tiles_m - m0 : a.group;
        const uint32_t tn = r / gm;
        q0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(m0 + r - tn * gm)) * T::BM;
        l0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tn)) * T::BN;
    };

    // ---- loads.  A lane brings chunk (position ^ swizzle) of its row; its offsets from the tile's first row are the same for
    // every tile and stage.  Queries are padded to whole tiles and stages; a tile of labels or a stage that reaches past the end
    // takes another way.  The first stage of a tile has the scales of its labels and queries with it, 64 to a load, for one of
    // R + 1 tiles: with rows of one stage the loads are R tiles ahead.
    constexpr int kScaleLinesL = T::kScaleLinesL, kScaleLinesQ = T::kScaleLinesQ;
    // label of the tile in row r of the tile's labels in LDS
    auto label_of = [&](int r) __attribute__((always_inline)) { const int blk = r >> 4; return (blk / V) * 16 * V + (r & 15) * V + blk % V; };
    uint32_t off_a[T::kLoadsA > 0 ? T::kLoadsA : 1], off_b[T::kLoadsB];
#pragma unroll
    for (int i = 0; i < T::kLoadsA; ++i) {
        const int r = (wi * T::kLoadsA + i) * 8 + (lane >> 3);
        off_a[i] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.ppitch) + ((lane & 7) ^ row_swizzle(r)) * 16;
    }
#pragma unroll
    for (int i = 0; i < T::kLoadsB; ++i) {
        const int r = (wi * T::kLoadsB + i) * 8 + (lane >> 3);
        off_b[i] = static_cast<uint32_t>(label_of(r)) * static_cast<uint32_t>(a.pitch) + ((lane & 7) ^ row_swizzle(r)) * 16;
    }
    uint32_t ld_t = t_first;
    int ld_kb = 0, ld_slot = 0, ld_tile = 0, n_issued = 0;
    int64_t ld_q = 0, ld_l = 0;
    auto issue = [&]() __attribute__((always_inline)) {
        if (ld_kb == 0) place(ld_t, ld_q, ld_l);
        if (T::G == 1 || n_issued % T::G == my_turn) {
            const int64_t have = a.L - ld_l;                 // labels of the tile
            if (ld_kb == 0) {
                const uint32_t to = lds + T::R * T::kStage + ld_tile * T::kScales;
#pragma unroll
                for (int j = 0; j < kScaleLinesL + kScaleLinesQ; j += T::kIssue) {
                    const int i = j + wi, lab = i * 64 + lane;           // i: uniform
                    if (i < kScaleLinesL)
                        lds_dma4(a.scale + ld_l + (lab < have ? lab : have - 1), __builtin_amdgcn_readfirstlane(to + i * 256));
                    else if (i < kScaleLinesL + kScaleLinesQ)
                        lds_dma4(a.pscale + ld_q + (i - kScaleLinesL) * 64 + lane, __builtin_amdgcn_readfirstlane(to + i * 256));
                }
            }
            const uint32_t dst = __builtin_amdgcn_readfirstlane(lds + ld_slot * T::kStage);
            const void* from_a = uniform_ptr(a.P + ld_q * a.ppitch + ld_kb * kStageBytes);
#pragma unroll
            for (int i = 0; i < T::kLoadsA; ++i) lds_dma16_sbase<0>(from_a, off_a[i], dst + (wi * T::kLoadsA + i) * 1024);
            const int room = a.pitch - ld_kb * kStageBytes;        // bytes of the rows from here on
            const uint32_t dst_b = dst + (T::kStageRows - T::BN) * kStageBytes + wi * T::kLoadsB * 1024;
            const int8_t* from_b = a.Q + ld_l * a.pitch + ld_kb * kStageBytes;
            if (have >= T::BN && (room >= kStageBytes || have >= T::BN + 7)) {     // (what is read behind a row, at most 112 bytes, meets zeros of the queries)
                const void* from = uniform_ptr(from_b);
#pragma unroll
                for (int i = 0; i < T::kLoadsB; ++i) load_labels<STREAM>(from, off_b[i], dst_b + i * 1024);
            } else {                                         // rows past the end: the last one again; chunks behind a row: its first here (the query's are zero)
#pragma unroll 1
                for (int i = 0; i < T::kLoadsB; ++i) {
                    const int r = (wi * T::kLoadsB + i) * 8 + (lane >> 3), lab = label_of(r), at = ((lane & 7) ^ row_swizzle(r)) * 16;
                    lds_dma16(from_b + (lab < have ? lab : have - 1) * a.pitch + (at < room ? at : 0), __builtin_amdgcn_readfirstlane(dst_b + i * 1024));
                }
            }
        }
        if (ld_kb == 0 && ++ld_tile == T::R + 1) ld_tile = 0;
        if (++ld_kb == n_stages) { ld_kb = 0; ld_t += t_step; }
        if (++ld_slot == T::R) ld_slot = 0;
        ++n_issued;
    };

    // ---- products.  The operands of a k-step are read while the one before is multiplied: a block of labels right behind its
    // own products, blocks of queries into the other half of their registers.
    constexpr int kSteps = kStageBytes / 64;
    i32x4 acc[T::MQ][T::ML], fa[2][T::MQ], fb[T::ML];
    const int frag = (lane & 15) * kStageBytes + ((quarter ^ row_swizzle(lane & 15)) * 16);
    constexpr int kResAt = T::R * T::kStage + (T::R + 1) * T::kScales;     // resident queries: 128 bytes of every row, the next 128, ..; their scales
    auto read_a = [&](int slot, int kb, int kk, int x) __attribute__((always_inline)) {
        if constexpr (T::RES > 0)
            return *reinterpret_cast<const i32x4*>(smem + kResAt + kb * (T::BM * kStageBytes) + (wq * T::MQ + x) * 16 * kStageBytes + (frag ^ (kk * 64)));
        return *reinterpret_cast<const i32x4*>(smem + slot * T::kStage + (wq * T::MQ + x) * 16 * kStageBytes + (frag ^ (kk * 64)));
    };
    auto read_b = [&](int slot, int kk, int y) __attribute__((always_inline)) {
        return *reinterpret_cast<const i32x4*>(smem + slot * T::kStage + (T::kStageRows - T::BN + (wl * T::ML + y) * 16) * kStageBytes + (frag ^ (kk * 64)));
    };
    constexpr int kStores = 4 * T::MQ * (T::ML / V);         // of a whole tile
    int since_stores = T::R;                                 // stages published since a whole tile's scores were stored
    // the next stage is there for everyone, and the one before it has been read by everyone: its slot is filled again
    auto publish = [&](int g_next) __attribute__((always_inline)) {
        constexpr int kNewer = T::kLoads * ((T::R - 2) / T::G);
        if (T::G == 1 || g_next % T::G == my_turn) {
            if (n_issued - 1 - g_next < T::R - 2) wait_all_vmem();
            else if (since_stores < T::R - 1) wait_vmem_at_most<(kNewer + kStores < 63 ? kNewer + kStores : 63)>();
            else wait_vmem_at_most<kNewer>();
        }
        ++since_stores;
        lds_barrier();
        if (n_issued < total) issue();
    };

    if constexpr (T::RES > 0) {
        // The queries (one tile of them) to integers, before the wave's own loads of labels, which it would have to wait for as
        // well.  Rows past the end are zeros.
        constexpr int kGroups = (T::RES + 511) / 512, kRows = 4;                 // groups of 8 elements to a lane; rows under way at a time
        float* qs = reinterpret_cast<float*>(smem + kResAt + T::BM * T::RES);
        const int64_t row_bytes = static_cast<int64_t>(a.d) * (sizeof(TZ) == 4 ? 4 : 2);
        for (int i = threadIdx.x; i < a.ppitch / 16 * T::BM; i += T::kThreads)
            if ((i >> 3) % T::BM >= a.B) *reinterpret_cast<uint4*>(smem + kResAt + i * 16) = make_uint4(0, 0, 0, 0);
        for (int r0 = wave; r0 < a.B; r0 += kRows * T::kWaves) {
            Eight<TZ> v[kRows][kGroups];
            uint32_t big[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int c = 0; c < kGroups; ++c) {
                    const int r = r0 + i * T::kWaves, e = (c * kWave + lane) * 8;
                    v[i][c].zero();
                    if (r < a.B && e < a.d) v[i][c].template load<false>(a.Z + r * row_bytes, e, a.d);
                }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                big[i] = 0;
#pragma unroll
                for (int c = 0; c < kGroups; ++c) { const uint32_t b = v[i][c].largest(); big[i] = b > big[i] ? b : big[i]; }
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < kRows; ++i) { const uint32_t b = __shfl_xor(big[i], o, kWave); big[i] = b > big[i] ? b : big[i]; }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = r0 + i * T::kWaves;
                if (r >= a.B) break;                         // uniform
                const RowScale s = row_scale(big[i]);
#pragma unroll
                for (int c = 0; c < kGroups; ++c) {
                    const int e = (c * kWave + lane) * 8;
                    if (e < a.ppitch) {
                        float f[8];
                        v[i][c].values(f);
                        const uint2 o = to_integers(f, s);
                        *reinterpret_cast<uint2*>(smem + kResAt + (e >> 7) * (T::BM * kStageBytes) + r * kStageBytes + ((((e & 127) >> 4) ^ row_swizzle(r)) * 16) + (e & 15)) =
                            s.inv == 0.0f ? make_uint2(0, 0) : o;
                    }
                }
                if (lane == 0) qs[r] = s.scale;
            }
        }
    }
    for (int s = 0; s < T::R - 1 && s < total; ++s) issue();
    publish(0);
#pragma unroll
    for (int x = 0; x < T::MQ; ++x) fa[0][x] = read_a(0, 0, 0, x);
#pragma unroll
    for (int y = 0; y < T::ML; ++y) fb[y] = read_b(0, 0, y);
    int g = 0, slot = 0, tile = 0;
    for (uint32_t t = t_first; t < t_end; t += t_step) {
#pragma unroll
        for (int x = 0; x < T::MQ; ++x)
#pragma unroll
            for (int y = 0; y < T::ML; ++y) acc[x][y] = i32x4{0, 0, 0, 0};
        for (int kb = 0; kb < n_stages; ++kb) {
            const int slot_next = slot + 1 == T::R ? 0 : slot + 1;
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
                static_assert(kSteps % 2 == 0, "the halves of fa change places with every step");
                const int sel = kk & 1, kk_next = kk + 1 < kSteps ? kk + 1 : 0, from = kk + 1 < kSteps ? slot : slot_next;
                if (kk == kSteps - 1 && g + 1 < total) publish(g + 1);       // (behind the last stage: what is read is not used)
#pragma unroll
                for (int y = 0; y < T::ML; ++y) {
#pragma unroll
                    for (int x = y * T::MQ / T::ML; x < (y + 1) * T::MQ / T::ML; ++x) fa[sel ^ 1][x] = read_a(from, kk + 1 < kSteps ? kb : kb + 1 == n_stages ? 0 : kb + 1, kk_next, x);
#pragma unroll
                    for (int x = 0; x < T::MQ; ++x) acc[x][y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[sel][x], fb[y], acc[x][y], 0, 0, 0);
                    fb[y] = read_b(from, kk_next, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            ++g;
            slot = slot_next;
        }

        int64_t q0, l0;
        place(t, q0, l0);
        const float* scales = reinterpret_cast<const float*>(smem + T::R * T::kStage + tile * T::kScales);
        if (++tile == T::R + 1) tile = 0;
        const int lt = wl * 16 * T::ML + (lane & 15) * V, qt = wq * T::MQ * 16 + 4 * quarter;       // of the tile
        float sl[T::ML];
#pragma unroll
        for (int y = 0; y < T::ML; ++y) sl[y] = scales[lt + (y / V) * 16 * V + y % V];
        TO* out = static_cast<TO*>(a.out) + (q0 + qt) * a.L + l0 + lt;
        auto rows = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < T::MQ; ++x) {
                const float4 sq = *reinterpret_cast<const float4*>(
                    (T::RES > 0 ? reinterpret_cast<const float*>(smem + kResAt + T::BM * T::RES) : scales + kScaleLinesL * 64) + qt + x * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float s = i == 0 ? sq.x : i == 1 ? sq.y : i == 2 ? sq.z : sq.w;
#pragma unroll
                    for (int y0 = 0; y0 < T::ML; y0 += V) {
                        float v[V];
#pragma unroll
                        for (int y = 0; y < V; ++y) v[y] = (static_cast<float>(acc[x][y0 + y][i]) * s) * sl[y0 + y];
                        TO* p = out + (x * 16 + i) * a.L + y0 * 16;
                        if constexpr (decltype(whole)::value) {
                            store_labels(p, v);
                        } else if (q0 + qt + x * 16 + i < a.B) {
                            const int64_t left = a.L - l0 - lt - y0 * 16;
                            if (left >= V) {
                                store_labels(p, v);
                            } else {
#pragma unroll
                                for (int y = 0; y < V; ++y) if (y < left) store_label(p + y, v[y]);
                            }
                        }
                    }
                }
            }
        };
        if (q0 + T::BM <= a.B && l0 + T::BN <= a.L) {
            rows(std::true_type{});
            since_stores = 0;
        } else {
            rows(std::false_type{});
        }
    }
}

typedef Tile<4, 2, 4, 8, 2, 2> TileMany;            // 256 x 256
typedef Tile<2, 2, 4, 4, 2, 1> TileMid;             // 128 x 128
typedef Tile<2, 2, 2, 2, 4, 1> TileSmall;           // 64 x 64
typedef Tile<2, 2, 2, 1, 4, 1> TileLow;             // 64 x 32
typedef Tile<1, 4, 4, 2, 3, 1> TileSome;            // 64 x 128
typedef Tile<1, 4, 2, 2, 3, 1> TileFew;             // 32 x 128
typedef Tile<1, 1, 2, 2, 4, 1> TileNarrow;          // 32 x 32
typedef Tile<1, 1, 1, 1, 4, 1> TileThin;            // 16 x 16
typedef Tile<1, 4, 1, 2, 4, 1, 768> TileOnline;     // 16 x 128, queries of up to 768 bytes resident
template <typename T, int BM, int BN> constexpr bool tile_is() { return T::BM == BM && T::BN == BN; }
static_assert(tile_is<TileMany, 256, 256>() && tile_is<TileMid, 128, 128>() && tile_is<TileSmall, 64, 64>() && tile_is<TileLow, 64, 32>() &&
              tile_is<TileSome, 64, 128>() && tile_is<TileFew, 32, 128>() && tile_is<TileNarrow, 32, 32>() && tile_is<TileThin, 16, 16>() &&
              tile_is<TileOnline, kOnlineQueries, 128>() && TileOnline::RES == kOnlineBytes && kScoresUnits == kMineGrid && kScoresXcds == kXcds,
              "what choose_scores counts");
constexpr int kQueryPad = 128;                           // the queries in the workspace: rows of whole stages,
constexpr int kQueryTile = 256;                          // whole tiles of them of any kind

template <typename TO, typename T, typename TZ = float>
static void launch_scores(ScoresArgs a, hipStream_t st) {
    static_assert(kQueryTile % T::BM == 0, "the last tile of queries ends within the padded rows");
    a.tiles_m = static_cast<int>((a.B + T::BM - 1) / T::BM);
    a.tiles_n = static_cast<int>((a.L + T::BN - 1) / T::BN);
    // a group of query tiles takes half of an XCD's L2
    const int64_t fit = (2 << 20) / (static_cast<int64_t>(T::BM) * a.ppitch);
    a.group = static_cast<int>(fit < 1 ? 1 : fit < a.tiles_m ? fit : a.tiles_m);
    const int64_t per = (static_cast<int64_t>(a.tiles_m) * a.tiles_n + 7) / 8, most = kCusPerXcd * T::kPerCu;
    const unsigned grid = static_cast<unsigned>(8 * (per < most ? per : most));
    if (a.tiles_m == 1 && a.pitch % kStageBytes == 0) scores_kernel<TO, T, true, TZ><<<grid, T::kThreads, 0, st>>>(a);      // every line of Q is read once
    else scores_kernel<TO, T, false, TZ><<<grid, T::kThreads, 0, st>>>(a);
}

// ---- many queries, rows of up to 768 bytes: the labels stay where they are.  A wave holds 64 labels as operands in registers (NK
// k-steps of 64 bytes) and 512 labels of a workgroup meet the queries that stream through LDS, QS at a time.  Per product that is
// two thirds of the operand reads from LDS that a 256 x 256 tile takes, a quarter of the bytes brought into it, and a wave's scores are
// stored 16 queries at a time, while the other wave of its SIMD multiplies.
// Bound: the products at the clock that the chip's power limit allows, and the stores beside them.  4096 x 131072 x 768 to bf16,
// one output written again and again: 360 to 365 us under sustained load (2.3 POP/s), 407 while the clock settles, 321 to 345 in
// the first four calls; an output that no call has written before costs more (397 over 100 of them).  Counted: 1.8 GHz, the matrix
// pipe busy 64 % of the time in which compute units are, 127 MB read and 1075 written.  Without the stores 281, without the loads
// the same as with them; 846 x 570112 x 192, which the stores bound, 223 (4.3 TB/s).  Rows that begin within a line cost 5 to 20
// percent: 4096 x 131071 x 768 431, 846 x 569976 x 192 247; and did 45 when a workgroup took neighbouring tiles one after the
// other, whose shared lines left the cache half written (351).  Neither 16-byte stores (rows exchanged between neighbouring lanes:
// 379 against 368 us a call), nor rows put together in LDS and stored by whole lines (4096 x 131080 x 768 610 against 355), nor
// wave priorities made it faster.
template <int NK_>
struct Held {
    static constexpr int NK = NK_, QS = NK % 4 == 0 ? 32 : 64, kStage = QS * NK * 64;       // (the stage's loads divide evenly among 8 waves)
    static constexpr int kFit = 160 * 1024 / (kStage + 256), R = kFit < 6 ? kFit : 6;       // stages in LDS, at least 3
    static constexpr int kLoads = kStage / 1024 / 8, kStores = QS / 4;                      // of a wave and stage
    static constexpr int kLds = R * (kStage + 256);
    static_assert(kLoads * 8 * 1024 == kStage && R >= 3 && (kLoads + kStores) * (R - 3) < 64, "whole loads, and a count that the wait can hold");
};
constexpr int kHeldPieces = 4;                           // of the tiles behind the last whole round, to a workgroup

template <typename TO, int NK>
__global__ __launch_bounds__(512, 2)
void scores_held_kernel(const ScoresArgs a, int tiles, int stages, int rest_tiles, int rest_parts, int rest_parts_more) {
    typedef Held<NK> H;
    __shared__ __align__(1024) unsigned char smem[H::kLds];
    __shared__ int4 last[kHeldPieces + 1];
    const int lane = lane_id(), quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
    // Each XCD takes neighbouring tiles of labels, a workgroup one of every 32, so that the lines that two tiles share are written at
    // about the same time.  Of the last tiles, fewer than 32, a workgroup has parts of the queries: as many for each tile (`parts`), for
    // the same reason, or (0) an equal number of stages.
    const int xcd = blockIdx.x % 8, nth = blockIdx.x / 8;
    const int t_begin = static_cast<int>(static_cast<int64_t>(tiles) * xcd / 8) + nth;
    const int t_count = static_cast<int>(static_cast<int64_t>(tiles) * (xcd + 1) / 8) + nth - t_begin, rounds = t_count / kCusPerXcd;
    if (threadIdx.x == 0) {
        const int rest = t_count % kCusPerXcd, first = t_begin - nth + rounds * kCusPerXcd, parts = rest == rest_tiles ? rest_parts : rest_parts_more;
        int n = 0;
        if (parts > 0) {
            for (int i = nth; i < rest * parts; i += kCusPerXcd)
                last[n++] = make_int4(first + i % rest, static_cast<int>(static_cast<int64_t>(stages) * (i / rest) / parts),
                                      static_cast<int>(static_cast<int64_t>(stages) * (i / rest + 1) / parts), 0);
        } else {
            const int64_t all = static_cast<int64_t>(rest) * stages, u1 = all * (nth + 1) / kCusPerXcd;
            for (int64_t u = all * nth / kCusPerXcd; u < u1;) {
                const int t = static_cast<int>(u / stages), s = static_cast<int>(u - static_cast<int64_t>(t) * stages);
                const int e = stages - s < u1 - u ? stages : s + static_cast<int>(u1 - u);
                last[n++] = make_int4(first + t, s, e, 0);
                u += e - s;
            }
        }
        int sum = 0;
        for (int i = 0; i < n; ++i) sum += last[i].z - last[i].y;
        last[0].w = rounds * stages + sum;
    }
    __syncthreads();
    // the workgroup's n-th piece of work: a tile and stages of queries
    auto piece = [&](int n, int& tile, int& begin, int& end) __attribute__((always_inline)) {
        tile = t_begin + n * kCusPerXcd;
        begin = 0;
        end = stages;
        if (n >= rounds) {
            const int4 l = last[n - rounds];
            tile = __builtin_amdgcn_readfirstlane(l.x);
            begin = __builtin_amdgcn_readfirstlane(l.y);
            end = __builtin_amdgcn_readfirstlane(l.z);
        }
    };
    const int total = __builtin_amdgcn_readfirstlane(last[0].w);
    if (total == 0) return;
    int tile, ld_tile, st, st_end;
    piece(0, tile, st, st_end);

    uint32_t off[H::kLoads];
#pragma unroll
    for (int i = 0; i < H::kLoads; ++i) {
        const int n = wave * H::kLoads + i, row = n % (H::QS / 8) * 8 + (lane >> 3);
        off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(a.ppitch) + n / (H::QS / 8) * 128 + (((lane & 7) ^ row_swizzle(row)) * 16);
    }
    int n_piece = 0, ld_piece = 0;
    int ld_st = st, ld_end = st_end, ld_slot = 0, n_issued = 0;
    auto issue = [&]() __attribute__((always_inline)) {
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds + ld_slot * H::kStage);
        if (wave == 0) lds_dma4(a.pscale + static_cast<int64_t>(ld_st) * H::QS + lane, __builtin_amdgcn_readfirstlane(lds + H::R * H::kStage + ld_slot * 256));
        const void* from = uniform_ptr(a.P + static_cast<int64_t>(ld_st) * H::QS * a.ppitch);
#pragma unroll
        for (int i = 0; i < H::kLoads; ++i) lds_dma16_sbase<0>(from, off[i], dst + (wave * H::kLoads + i) * 1024);
        if (++ld_st == ld_end) {
            piece(++ld_piece, ld_tile, ld_st, ld_end);
        }
        if (++ld_slot == H::R) ld_slot = 0;
        ++n_issued;
    };
    int full = 0;                                            // stages in a row whose scores were all stored as whole blocks
    auto publish = [&](int g_next) __attribute__((always_inline)) {
        // (published while the stage before it still has a block to read: the slot of the one before that is filled)
        if (n_issued - 1 - g_next < H::R - 3) wait_all_vmem();
        else if (full >= H::R) wait_vmem_at_most<(H::kLoads + H::kStores) * (H::R - 3)>();
        else wait_vmem_at_most<H::kLoads*(H::R - 3)>();
        lds_barrier();
        if (n_issued < total && n_issued < g_next + H::R - 1) issue();
    };
    for (int s = 0; s < H::R - 1 && s < total; ++s) issue();

    i32x4 w[NK][4], fa[3];
    float sl[4];
    const int frag = (lane & 15) * 128 + ((quarter ^ row_swizzle(lane & 15)) * 16);
    auto read_a = [&](int slot, int qb, int k) __attribute__((always_inline)) {      // 16 queries, 64 bytes of each
        return *reinterpret_cast<const i32x4*>(smem + slot * H::kStage + (k >> 1) * (H::QS * 128) + qb * 2048 + (frag ^ ((k & 1) * 64)));
    };
    auto hold = [&](int64_t l0) __attribute__((always_inline)) {                     // the wave's labels: 4 neighbouring ones to a lane
        const int64_t l = l0 + wave * 64 + (lane & 15) * 4;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t row = l + y < a.L ? l + y : a.L - 1;
            sl[y] = a.scale[row];
            const int8_t* p = a.Q + row * a.pitch + quarter * 16;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                w[k][y] = i32x4{0, 0, 0, 0};
                if (k * 64 + quarter * 16 < a.pitch) w[k][y] = *reinterpret_cast<const i32x4*>(p + k * 64);
            }
        }
        // awaited here: the loop over the stages would wait for these (and for all loads and stores under way) every time round
        // (rows of 641 to 768 bytes leave wave 0 such a wait all the same: of its 256 registers the address of the queries' scales is
        // spilled, and issue() reloads it once a stage)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            asm volatile("" : "+v"(sl[y]));
#pragma unroll
            for (int k = 0; k < NK; ++k) asm volatile("" : "+v"(w[k][y]));
        }
    };
    hold(static_cast<int64_t>(tile) * kHeldLabels);
    publish(0);
    fa[0] = read_a(0, 0, 0);
    fa[1] = read_a(0, 0, 1);
    int slot = 0;
    constexpr int kBlocks = H::QS / 16;
    for (int g = 0; g < total; ++g) {
        const int64_t l0 = static_cast<int64_t>(tile) * kHeldLabels + wave * 64, l = l0 + (lane & 15) * 4;
        const int q0 = st * H::QS;
        const bool whole = static_cast<int64_t>(q0) + H::QS <= a.B && l0 + 64 <= a.L;
        const int slot_next = slot + 1 == H::R ? 0 : slot + 1;
        const float* sq = reinterpret_cast<const float*>(smem + H::R * H::kStage + slot * 256) + 4 * quarter;
        TO* out = static_cast<TO*>(a.out) + static_cast<int64_t>(q0 + 4 * quarter) * a.L + l;
#pragma unroll
        for (int qb = 0; qb < kBlocks; ++qb) {
            if (qb == kBlocks - 1 && g + 1 < total) publish(g + 1);
            i32x4 acc[4];
            const float4 s4 = *reinterpret_cast<const float4*>(sq + qb * 16);
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                constexpr int kDepth = 2;
                const int kn = k + kDepth < NK ? k + kDepth : k + kDepth - NK;
                const bool over = k + kDepth >= NK;
                const int n = qb * NK + k;                   // of the stage: NK * kBlocks is a multiple of 3 or fa is put right behind it
                fa[(n + kDepth) % 3] = !over ? read_a(slot, qb, kn) : qb + 1 < kBlocks ? read_a(slot, qb + 1, kn) : read_a(slot_next, 0, kn);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    acc[y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[n % 3], w[k][y], k == 0 ? i32x4{0, 0, 0, 0} : acc[y], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr ((NK * kBlocks) % 3 != 0) {
                if (qb == kBlocks - 1) {                     // the next stage starts at fa[0] again
                    const i32x4 f0 = fa[(NK * kBlocks) % 3], f1 = fa[(NK * kBlocks + 1) % 3];
                    fa[0] = f0;
                    fa[1] = f1;
                }
            }
            auto rows = [&](auto all) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float s = i == 0 ? s4.x : i == 1 ? s4.y : i == 2 ? s4.z : s4.w;
                    float v[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) v[y] = (static_cast<float>(acc[y][i]) * s) * sl[y];
                    TO* p = out + static_cast<int64_t>(qb * 16 + i) * a.L;
                    if constexpr (decltype(all)::value) {
                        store_labels(p, v);
                    } else if (q0 + qb * 16 + 4 * quarter + i < a.B) {
                        if (l + 4 <= a.L) {
                            store_labels(p, v);
                        } else {
#pragma unroll
                            for (int y = 0; y < 4; ++y) if (l + y < a.L) store_label(p + y, v[y]);
                        }
                    }
                }
            };
            if (whole) rows(std::true_type{});
            else rows(std::false_type{});
        }
        full = whole ? full + 1 : 0;
        slot = slot_next;
        if (++st == st_end) {
            piece(++n_piece, tile, st, st_end);
            full = 0;
            if (g + 1 < total) hold(static_cast<int64_t>(tile) * kHeldLabels);
        }
    }
}

template <typename TO, int NK>
static void launch_held(ScoresArgs a, hipStream_t st) {
    const int stages = static_cast<int>((a.B + Held<NK>::QS - 1) / Held<NK>::QS);
    const int tiles = static_cast<int>((a.L + kHeldLabels - 1) / kHeldLabels), rest = tiles / 8 % kCusPerXcd;      // of an XCD; some have one more
    // As few rounds of the parts as may be: to hold a tile's labels takes the time of about 5 stages (2809 x 106363 x 232 to fp32 391 ->
    // 285 us, 700 x 74141 x 640 89 -> 75).  Equal numbers of stages where rows of whole half lines leave next to nothing to share
    // (106368 labels to bf16: 143, in parts 160), and where the products take longer than the stores (700 x 74141 x 640 to bf16: 63 and 72).
    const bool equal = (sizeof(TO) == 2 && NK > 8) || ((reinterpret_cast<uintptr_t>(a.out) | static_cast<uintptr_t>(a.L) * sizeof(TO)) & 63) == 0;
    auto parts_of = [&](int rest) {
        int parts = 0, best = 0;
        for (int p = 1; !equal && p <= stages && rest * p <= kHeldPieces * kCusPerXcd; ++p) {
            const int cost = (rest * p + kCusPerXcd - 1) / kCusPerXcd * ((stages + p - 1) / p + 5);
            if (parts == 0 || cost < best) { best = cost; parts = p; }
            if (rest == 0) break;
        }
        return parts;
    };
    scores_held_kernel<TO, NK><<<kMineGrid, 512, 0, st>>>(a, tiles, stages, rest, parts_of(rest), parts_of((rest + 1) % kCusPerXcd));
}

template <typename TO>
static void run_held(const ScoresArgs& a, hipStream_t st) {
    switch (a.ppitch / 128) {
        case 1: launch_held<TO, 2>(a, st); break;
        case 2: launch_held<TO, 4>(a, st); break;
        case 3: launch_held<TO, 6>(a, st); break;
        case 4: launch_held<TO, 8>(a, st); break;
        case 5: launch_held<TO, 10>(a, st); break;
        default: launch_held<TO, 12>(a, st); break;
    }
}

template <typename TO>
static void run_scores(const ScoresArgs& a, ScoresKernel kernel, hipStream_t st) {
    switch (kernel) {
        case kScoresThin: launch_scores<TO, TileThin>(a, st); break;
        case kScoresNarrow: launch_scores<TO, TileNarrow>(a, st); break;
        case kScoresFew: launch_scores<TO, TileFew>(a, st); break;
        case kScoresLow: launch_scores<TO, TileLow>(a, st); break;
        case kScoresSmall: launch_scores<TO, TileSmall>(a, st); break;
        case kScoresSome: launch_scores<TO, TileSome>(a, st); break;
        case kScoresMid: launch_scores<TO, TileMid>(a, st); break;
        case kScoresMany: launch_scores<TO, TileMany>(a, st); break;
        default: run_held<TO>(a, st); break;
    }
}

template <typename TZ>
static void run_few(const ScoresArgs& a, xc_dtype out_t, hipStream_t st) {
    if (out_t == XC_F32) launch_scores<float, TileOnline, TZ>(a, st);
    else launch_scores<bf16_t, TileOnline, TZ>(a, st);
}

static size_t scores_bytes(int64_t B, int d) {
    return round_up(B, kQueryTile) * (4 + round_up(d, kQueryPad));
}

static bool row_ok(int d, xc_dtype t) {
    return d >= 1 && d <= XC_MAX_D_QUANTIZED && (static_cast<int64_t>(d) * (t == XC_F32 ? 4 : 2)) % 16 == 0;
}

}  // namespace xc

extern "C" int xc_quantize_rows(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count,
                                int8_t* Q, float* scale, void* stream) {
    using namespace xc;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (N < 1 || N > (1LL << 40) || !row_ok(d, t) || m < 0 || m > (1LL << 40)) return XC_ESHAPE;
    if (!X || !Q || !scale || !aligned16(X) || !aligned16(Q) || !aligned16(scale) || !aligned16(ids) || !aligned16(count)) return XC_EINVAL;
    if (ids == nullptr && count != nullptr) return XC_EINVAL;
    if (ids != nullptr && m == 0) return XC_OK;
    const unsigned __int128 rows = N;
    if (overlap({Span(Q, rows * quantized_pitch(d)), Span(scale, rows * 4)},
                {Span(X, rows * d * (t == XC_F32 ? 4 : 2)), Span(ids, static_cast<unsigned __int128>(m) * 4), Span(count, 4)}))
        return XC_EINVAL;
    return launch_quantize(X, N, d, t, ids, m, count, Q, quantized_pitch(d), scale, static_cast<hipStream_t>(stream));
}

extern "C" int xc_scores_workspace(int64_t B, int d, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (B < 1 || B > 0x7fffffffLL || d < 1 || d > XC_MAX_D_QUANTIZED) return XC_ESHAPE;
    *bytes = scores_bytes(B, d);
    return XC_OK;
}

extern "C" int xc_scores_quantized(const void* Z, int64_t B, int d, xc_dtype t, const int8_t* Q, const float* scale, int64_t L,
                                   xc_dtype out_t, void* out, void* ws, size_t ws_bytes, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (B < 1 || B > 0x7fffffffLL || L < 1 || L > 0x7fffffffLL || B > (1LL << 40) / L || !row_ok(d, t)) return XC_ESHAPE;
    if (!Z || !Q || !scale || !out || !ws) return XC_EINVAL;
    if (!aligned16(Z) || !aligned16(Q) || !aligned16(scale) || !aligned16(out) || !aligned16(ws)) return XC_EINVAL;
    if (ws_bytes < scores_bytes(B, d)) return XC_EWORKSPACE;
    const size_t queries = static_cast<size_t>(B), labels = static_cast<size_t>(L);
    if (overlap({Span(out, queries * labels * (out_t == XC_F32 ? 4 : 2)), Span(ws, scores_bytes(B, d))},
                {Span(Z, queries * d * (t == XC_F32 ? 4 : 2)), Span(Q, labels * quantized_pitch(d)), Span(scale, labels * 4)}))
        return XC_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* pscale = static_cast<float*>(ws);
    int8_t* P = static_cast<int8_t*>(ws) + round_up(B, kQueryTile) * 4;
    const int ppitch = static_cast<int>(round_up(d, kQueryPad));
    const ScoresArgs a{static_cast<const unsigned char*>(Z), d, P, pscale, Q, scale, out, B, L, quantized_pitch(d), ppitch, 0, 0, 0};
    const ScoresKernel kernel = choose_scores(B, L, ppitch, out_t == XC_F32 ? 4 : 2);
    if (kernel == kScoresOnline) {
        if (t == XC_F32) XC_LAUNCH(K_SCORES, st, run_few<float>(a, out_t, st));
        else XC_LAUNCH(K_SCORES, st, run_few<bf16_t>(a, out_t, st));
    } else {
        const int rc = launch_quantize(Z, B, d, t, nullptr, 0, nullptr, P, ppitch, pscale, st);
        if (rc != XC_OK) return rc;
        if (out_t == XC_F32) XC_LAUNCH(K_SCORES, st, run_scores<float>(a, kernel, st));
        else XC_LAUNCH(K_SCORES, st, run_scores<bf16_t>(a, kernel, st));
    }
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
