// Rows in 8 bits, and the scores of all labels from them: out = (<p, q> a) b with integers p, q and a scale per row on
// either side.  The integer sums are exact, so their order (and how the work is cut) cannot change a score.
#include "xc_mine.h"

namespace xc {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

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

template <typename T> struct Row;
template <> struct Row<float> {
    static constexpr int kPer = 4;       // elements of 16 bytes
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
};
template <> struct Row<bf16_t> {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) { unpack8(v, f); }
};

// One wave per row, which is read twice.
template <typename T>
__global__ __launch_bounds__(256)
void quantize_kernel(const unsigned char* __restrict__ X, int64_t N, int d, const int32_t* __restrict__ ids, int64_t m,
                     const int32_t* __restrict__ count, int8_t* __restrict__ Q, int pitch, float* __restrict__ scale) {
    constexpr int kPer = Row<T>::kPer;
    const int chunks = d / kPer, lane = lane_id();
    int64_t rows = ids != nullptr ? m : N;
    if (ids != nullptr && count != nullptr) {
        const int64_t c = count[0];
        rows = c < rows ? c : rows;
    }
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); i < rows; i += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = ids != nullptr ? ids[i] : i;
        if (row < 0 || row >= N) continue;
        const uint4* src = reinterpret_cast<const uint4*>(X) + row * chunks;
        uint32_t big = 0;
        for (int c = lane; c < chunks; c += kWave) {
            float f[kPer];
            Row<T>::unpack(src[c], f);
#pragma unroll
            for (int e = 0; e < kPer; ++e) { const uint32_t b = __float_as_uint(f[e]) & 0x7fffffffu; big = b > big ? b : big; }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) { const uint32_t o = __shfl_xor(big, off, kWave); big = o > big ? o : big; }
        const RowScale s = row_scale(big);
        int8_t* dst = Q + row * pitch;
        for (int c = lane; c * kPer < pitch; c += kWave) {
            float f[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) f[e] = 0.0f;
            if (c < chunks) Row<T>::unpack(src[c], f);
#pragma unroll
            for (int e = 0; e < kPer; ++e) dst[c * kPer + e] = s.inv == 0.0f ? 0 : static_cast<int8_t>(to_integer(f[e] * s.up, s.m, s.inv));
        }
        if (lane == 0) scale[row] = s.scale;
    }
}

static int launch_quantize(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count,
                           int8_t* Q, int pitch, float* scale, hipStream_t st) {
    const int64_t rows = ids != nullptr ? m : N;
    if (rows == 0) return XC_OK;
    const int64_t want = (rows + 3) / 4;
    const unsigned grid = static_cast<unsigned>(want < 16384 ? want : 16384);
    const unsigned char* x = static_cast<const unsigned char*>(X);
    if (t == XC_F32)
        XC_LAUNCH(K_QUANTIZE, st, (quantize_kernel<float><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, pitch, scale)));
    else
        XC_LAUNCH(K_QUANTIZE, st, (quantize_kernel<bf16_t><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, pitch, scale)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
// Tiles of BM queries x BN labels, K staged KB bytes of each row at a time through a ring of R stages in LDS (direct
// global -> LDS loads).  WQ x WL waves, each with MQ x ML blocks of v_mfma_i32_32x32x32_i8.
// LDS rows are unpadded, their 16-byte chunks stored at chunk ^ swizzle(row) so that 16 lanes reading one chunk of 16 rows
// meet all banks.  Block nt of a wave's labels holds every ML-th of them: label ML j + nt is column j of block nt, so that a
// lane ends up with ML neighbouring labels and stores them together.
// Accumulator i of a lane: query 8 (i / 4) + 4 (lane / 32) + i % 4 of its block, column lane % 32.
template <int WQ_, int WL_, int MQ_, int ML_, int KB_, int R_>
struct Tile {
    static constexpr int WQ = WQ_, WL = WL_, MQ = MQ_, ML = ML_, KB = KB_, R = R_;
    static constexpr int kWaves = WQ * WL, kThreads = 64 * kWaves, BM = 32 * WQ * MQ, BN = 32 * WL * ML;
    static constexpr int kStage = (BM + BN) * KB, kLds = R * kStage;
    static constexpr int kRowsPerLoad = 1024 / KB;       // rows that one load instruction of a wave brings in
    static constexpr int kLoadsA = BM / kRowsPerLoad / kWaves, kLoadsB = BN / kRowsPerLoad / kWaves, kLoads = kLoadsA + kLoadsB;
    static_assert(kLoadsA * kRowsPerLoad * kWaves == BM && kLoadsB * kRowsPerLoad * kWaves == BN, "loads divide evenly among the waves");
    static __device__ __forceinline__ int swizzle(int row) { return (row / (256 / KB)) & (KB / 16 - 1); }
};

struct ScoresArgs {
    const int8_t* P;                     // queries in 8 bits, rows of ppitch bytes (zeros from column d on)
    const float* pscale;
    const int8_t* Q;
    const float* scale;
    void* out;
    int64_t B, L;
    int pitch, ppitch;                   // bytes of a row of Q, of P (whole stages)
    int tiles_m, tiles_n, group;         // tiles of queries that are taken together, label tile by label tile
};

// N neighbouring scores; `left` of them exist
template <typename TO, int N>
__device__ __forceinline__ void store_labels(TO* p, const float (&v)[N], int64_t left) {
    if constexpr (sizeof(TO) == 4) {
        if (left >= N) { __builtin_memcpy(p, v, 4 * N); return; }
#pragma unroll
        for (int e = 0; e < N; ++e) if (e < left) reinterpret_cast<float*>(p)[e] = v[e];
    } else {
        uint16_t h[N];
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] = static_cast<uint16_t>(float_to_bf16_bits(v[e]));
        if (left >= N) { __builtin_memcpy(p, h, 2 * N); return; }
#pragma unroll
        for (int e = 0; e < N; ++e) if (e < left) p[e].bits = h[e];
    }
}

__device__ __forceinline__ const void* uniform_ptr(const void* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const void*>(
        (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32)))) << 32) |
        static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a)))));
}

template <typename TO, typename T>
__global__ __launch_bounds__(T::kThreads, 2)
void scores_kernel(const ScoresArgs a) {
    __shared__ __align__(1024) unsigned char smem[T::kLds];
    // workgroup w runs on XCD w % 8: each XCD takes a contiguous part of the tiles, in an order that keeps a group of query
    // tiles in its L2 while the labels pass
    const int64_t n_tiles = static_cast<int64_t>(a.tiles_m) * a.tiles_n, per = (n_tiles + 7) / 8;
    const int64_t t = static_cast<int64_t>(blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || t >= n_tiles) return;
    const int64_t in_groups = static_cast<int64_t>(a.group) * a.tiles_n;
    const int g = static_cast<int>(t / in_groups), m0 = g * a.group;
    const int gm = a.tiles_m - m0 < a.group ? a.tiles_m - m0 : a.group;
    const int64_t r = t - g * in_groups;
    const int tn = __builtin_amdgcn_readfirstlane(static_cast<int>(r / gm)), tm = __builtin_amdgcn_readfirstlane(m0 + static_cast<int>(r % gm));
    const int64_t q0 = static_cast<int64_t>(tm) * T::BM, l0 = static_cast<int64_t>(tn) * T::BN;

    const int lane = lane_id(), half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wq = wave / T::WL, wl = wave % T::WL;
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));

    // what a lane loads: chunk (position ^ swizzle) of its row, rows past the end repeat the last one
    constexpr int kPerRow = T::KB / 16;
    const int n_stages = (a.pitch + T::KB - 1) / T::KB;
    uint32_t off_a[T::kLoadsA], off_b[T::kLoadsB], last_b[T::kLoadsB];
    const int row_of = lane / kPerRow;
#pragma unroll
    for (int i = 0; i < T::kLoadsA; ++i) {
        const int rho = (wave * T::kLoadsA + i) * T::kRowsPerLoad + row_of;
        const int64_t left = a.B - 1 - q0;
        off_a[i] = static_cast<uint32_t>(rho < left ? rho : left) * static_cast<uint32_t>(a.ppitch) + (((lane % kPerRow) ^ T::swizzle(rho)) * 16);
    }
#pragma unroll
    for (int i = 0; i < T::kLoadsB; ++i) {
        const int rho = (wave * T::kLoadsB + i) * T::kRowsPerLoad + row_of;
        const int blk = rho >> 5, lab = (blk / T::ML) * 32 * T::ML + (rho & 31) * T::ML + blk % T::ML;
        const int64_t left = a.L - 1 - l0;
        const uint32_t row = static_cast<uint32_t>(lab < left ? lab : left) * static_cast<uint32_t>(a.pitch);
        const int chunk = (lane % kPerRow) ^ T::swizzle(rho);
        off_b[i] = row + chunk * 16;
        // the last stage may reach past the row: any chunk of it will do there, the query's are zero
        last_b[i] = (n_stages - 1) * T::KB + chunk * 16 < a.pitch ? off_b[i] : row;
    }
    const int8_t* base_a = a.P + q0 * a.ppitch;
    const int8_t* base_b = a.Q + l0 * a.pitch;
    auto issue = [&](int s) __attribute__((always_inline)) {
        const uint32_t dst = lds + (s % T::R) * T::kStage;
        const void* pa = uniform_ptr(base_a + s * T::KB);
        const void* pb = uniform_ptr(base_b + s * T::KB);
#pragma unroll
        for (int i = 0; i < T::kLoadsA; ++i)
            lds_dma16_sbase<0>(pa, off_a[i], __builtin_amdgcn_readfirstlane(dst + (wave * T::kLoadsA + i) * 1024));
#pragma unroll
        for (int i = 0; i < T::kLoadsB; ++i)
            lds_dma16_sbase<0>(pb, s == n_stages - 1 ? last_b[i] : off_b[i],
                               __builtin_amdgcn_readfirstlane(dst + T::BM * T::KB + (wave * T::kLoadsB + i) * 1024));
    };

    i32x16 acc[T::MQ][T::ML];
#pragma unroll
    for (int x = 0; x < T::MQ; ++x)
#pragma unroll
        for (int y = 0; y < T::ML; ++y) acc[x][y] = i32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const int frag = (lane & 31) * T::KB + ((half ^ T::swizzle(lane & 31)) * 16);

    for (int s = 0; s < T::R - 1 && s < n_stages; ++s) issue(s);
    for (int s = 0; s < n_stages; ++s) {
        if (s + T::R - 2 < n_stages) wait_vmem_at_most<T::kLoads * (T::R - 2)>();
        else wait_all_vmem();
        lds_barrier();                                   // everyone's part of stage s is there, and stage s - 1 is read
        if (s + T::R - 1 < n_stages) issue(s + T::R - 1);
        const unsigned char* sa = smem + (s % T::R) * T::kStage + wq * T::MQ * 32 * T::KB;
        const unsigned char* sb = smem + (s % T::R) * T::kStage + (T::BM + wl * T::ML * 32) * T::KB;
#pragma unroll
        for (int kk = 0; kk < T::KB / 32; ++kk) {
            i32x4 fa[T::MQ], fb[T::ML];
#pragma unroll
            for (int x = 0; x < T::MQ; ++x) fa[x] = *reinterpret_cast<const i32x4*>(sa + ((frag ^ (kk * 32)) + x * 32 * T::KB));
#pragma unroll
            for (int y = 0; y < T::ML; ++y) fb[y] = *reinterpret_cast<const i32x4*>(sb + ((frag ^ (kk * 32)) + y * 32 * T::KB));
#pragma unroll
            for (int x = 0; x < T::MQ; ++x)
#pragma unroll
                for (int y = 0; y < T::ML; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[x], fb[y], acc[x][y], 0, 0, 0);
        }
    }

    const int64_t l = l0 + wl * 32 * T::ML + (lane & 31) * T::ML, left = a.L - l;
    if (left <= 0) return;
    float sl[T::ML];
#pragma unroll
    for (int y = 0; y < T::ML; ++y) sl[y] = y < left ? a.scale[l + y] : 0.0f;
    TO* out = static_cast<TO*>(a.out);
#pragma unroll
    for (int x = 0; x < T::MQ; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t q = q0 + (wq * T::MQ + x) * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
            if (q < a.B) {
                const float sq = a.pscale[q];
                float v[T::ML];
#pragma unroll
                for (int y = 0; y < T::ML; ++y) v[y] = (static_cast<float>(acc[x][y][i]) * sq) * sl[y];
                store_labels(out + q * a.L + l, v, left);
            }
        }
}

typedef Tile<2, 2, 2, 4, 64, 3> TileMany;                // 128 x 256
typedef Tile<1, 4, 2, 1, 128, 3> TileSome;               // 64 x 128
typedef Tile<1, 4, 1, 1, 128, 4> TileFew;                // 32 x 128
constexpr int kQueryPad = 128;                           // rows of P are whole stages of any kind

template <typename TO, typename T>
static void launch_scores(ScoresArgs a, hipStream_t st) {
    a.tiles_m = static_cast<int>((a.B + T::BM - 1) / T::BM);
    a.tiles_n = static_cast<int>((a.L + T::BN - 1) / T::BN);
    // a group of query tiles takes half of an XCD's L2
    const int64_t fit = (2 << 20) / (static_cast<int64_t>(T::BM) * a.ppitch);
    a.group = static_cast<int>(fit < 1 ? 1 : fit < a.tiles_m ? fit : a.tiles_m);
    const int64_t per = (static_cast<int64_t>(a.tiles_m) * a.tiles_n + 7) / 8;
    scores_kernel<TO, T><<<static_cast<unsigned>(8 * per), T::kThreads, 0, st>>>(a);
}

static size_t scores_bytes(int64_t B, int d) {
    return round_up(static_cast<size_t>(B) * 4, 256) + static_cast<size_t>(B) * round_up(d, kQueryPad);
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
    if (B < 1 || B > 0x7fffffffLL || L < 1 || L > 0x7fffffffLL || !row_ok(d, t)) return XC_ESHAPE;
    if (!Z || !Q || !scale || !out || !ws) return XC_EINVAL;
    if (!aligned16(Z) || !aligned16(Q) || !aligned16(scale) || !aligned16(out) || !aligned16(ws)) return XC_EINVAL;
    if (ws_bytes < scores_bytes(B, d)) return XC_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* pscale = static_cast<float*>(ws);
    int8_t* P = static_cast<int8_t*>(ws) + round_up(static_cast<size_t>(B) * 4, 256);
    const int rc = launch_quantize(Z, B, d, t, nullptr, 0, nullptr, P, static_cast<int>(round_up(d, kQueryPad)), pscale, st);
    if (rc != XC_OK) return rc;
    const ScoresArgs a{P, pscale, Q, scale, out, B, L, quantized_pitch(d), static_cast<int>(round_up(d, kQueryPad)), 0, 0, 0};
    if (out_t == XC_F32)
        XC_LAUNCH(K_SCORES, st, B <= 32 ? (launch_scores<float, TileFew>(a, st)) : B <= 64 ? (launch_scores<float, TileSome>(a, st)) : (launch_scores<float, TileMany>(a, st)));
    else
        XC_LAUNCH(K_SCORES, st, B <= 32 ? (launch_scores<bf16_t, TileFew>(a, st)) : B <= 64 ? (launch_scores<bf16_t, TileSome>(a, st)) : (launch_scores<bf16_t, TileMany>(a, st)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
