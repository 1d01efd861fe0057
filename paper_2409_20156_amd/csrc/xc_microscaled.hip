// Rows in 4-bit floating point with shared scales, and the scores of all labels from them.
// 32 neighbouring elements of a row share a scale 2^(byte - 127); an element is a sign, two bits of exponent and one of mantissa: 0, 0.5, 1,
// 1.5, 2, 3, 4 or 6.  The largest magnitude of a block decides the scale: the power of two that brings it into [4, 8).  What lies beyond 6
// then is 6 (the format's published conversion, so that rows laid out elsewhere mean the same here).
#include "xc_common.h"

namespace xc {

typedef int mx_i32x4 __attribute__((ext_vector_type(4)));
typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMxRow = 128;              // elements that a row is padded to a multiple of: one product's worth
inline int64_t mx_pitch(int64_t d) { return (d + kMxRow - 1) / kMxRow * kMxRow; }

// ---------------------------------------------------------------------------
// rows -> 4 bits
// ---------------------------------------------------------------------------
// 8 neighbouring elements of a row
template <typename T> __device__ __forceinline__ void eight(const unsigned char* row, int e, int d, float (&f)[8]);
template <> __device__ __forceinline__ void eight<float>(const unsigned char* row, int e, int d, float (&f)[8]) {
    uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (e < d) v[0] = load16<false>(row + e * 4);
    if (e + 4 < d) v[1] = load16<false>(row + e * 4 + 16);                 // (d is a multiple of 4)
    __builtin_memcpy(f, v, 32);
}
template <> __device__ __forceinline__ void eight<bf16_t>(const unsigned char* row, int e, int d, float (&f)[8]) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (e < d) v = load16<false>(row + e * 2);
    unpack8(v, f);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {   // of four neighbouring lanes
    uint32_t o = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xB1, 0xf, 0xf, false);          // quad_perm 1 0 3 2
    x = o > x ? o : x;
    o = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4E, 0xf, 0xf, false);                   // quad_perm 2 3 0 1
    return o > x ? o : x;
}

// 16 lanes bring 128 elements of a row, four lanes to a block.
template <typename T>
__global__ __launch_bounds__(256)
void microscale_kernel(const unsigned char* __restrict__ X, int64_t N, int d, const int32_t* __restrict__ ids, int64_t m, const int32_t* __restrict__ count,
                       uint8_t* __restrict__ Q, uint8_t* __restrict__ scale, int units /* of 128 elements in a row */) {
    const int sub = threadIdx.x & 15;
    int64_t rows = ids != nullptr ? m : N;
    if (ids != nullptr && count != nullptr) {
        const int64_t c = count[0];
        rows = c < rows ? c : rows;
    }
    const int64_t total = rows * units, step = static_cast<int64_t>(gridDim.x) * 16;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4); u < total; u += step) {
        const int64_t i = u / units, row = ids != nullptr ? ids[i] : i;
        const int col = static_cast<int>(u - i * units);
        if (row < 0 || row >= N) continue;                   // (16 lanes leave together)
        float f[8];
        eight<T>(X + row * d * static_cast<int64_t>(sizeof(T)), col * kMxRow + sub * 8, d, f);
        uint32_t big = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = __float_as_uint(f[e]) & 0x7fffffffu;
            big = b > big ? b : big;
        }
        big = quad_max(big);
        const bool finite = big < 0x7f800000u;
        const uint32_t exponent = big >> 23, byte = exponent > 2u ? exponent - 2u : 0u;
        const float inv = __uint_as_float((254u - (finite ? byte : 0u)) << 23);
        uint32_t codes = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= inv;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], 1.0f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], 1.0f, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], 1.0f, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], 1.0f, 3);
        *reinterpret_cast<uint32_t*>(Q + (row * units + col) * (kMxRow / 2) + sub * 4) = finite ? codes : 0u;
        if ((sub & 3) == 0) scale[(row * units + col) * 4 + (sub >> 2)] = static_cast<uint8_t>(finite ? byte : 255u);
    }
}

static int launch_microscale(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count, uint8_t* Q, uint8_t* scale, hipStream_t st) {
    const int units = static_cast<int>(mx_pitch(d) / kMxRow);
    const int64_t rows = ids != nullptr ? m : N, want = (rows * units + 15) / 16;
    const unsigned grid = static_cast<unsigned>(want < 16384 ? want : 16384);
    const unsigned char* x = static_cast<const unsigned char*>(X);
    if (t == XC_F32) XC_LAUNCH(K_MICROSCALE, st, (microscale_kernel<float><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, scale, units)));
    else XC_LAUNCH(K_MICROSCALE, st, (microscale_kernel<bf16_t><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, scale, units)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
struct MicroArgs {
    const uint8_t *P, *pscale;           // queries in 4 bits
    const uint8_t *Q, *scale;
    void* out;
    int64_t B, L, tiles_m, tiles_n;
    int units;                           // of 128 elements in a row
};

// Blocks of 16 labels x 16 queries x 128 elements: lane l has the 32 elements of block l / 16 of row l % 16 of both operands; its
// accumulator i is label 4 (l / 16) + i, query l % 16.
__device__ __forceinline__ mx_f32x4 mx_product(const mx_i32x4& w, const mx_i32x4& z, const mx_f32x4& c, int ws, int zs) {
    const mx_i32x8 a = {w.x, w.y, w.z, w.w, 0, 0, 0, 0}, b = {z.x, z.y, z.z, z.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4 /* fp4 */, 4, 0, ws, 0, zs);
}
template <typename TO> __device__ __forceinline__ void put_scores(TO* p, const float* v, int n);
template <> __device__ __forceinline__ void put_scores<float>(float* p, const float* v, int n) {
    for (int e = 0; e < n; ++e) p[e] = v[e];
}
template <> __device__ __forceinline__ void put_scores<bf16_t>(bf16_t* p, const float* v, int n) {
    for (int e = 0; e < n; ++e) p[e].bits = static_cast<uint16_t>(float_to_bf16_bits(v[e]));
}

// A wave has 64 labels x 64 queries.
constexpr int kMxTile = 64;
template <typename TO>
__global__ __launch_bounds__(256)
void scores_micro_kernel(const MicroArgs a) {
    const int lane = lane_id(), r = lane & 15, quarter = lane >> 4;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t >= a.tiles_m * a.tiles_n) return;
    const int64_t l0 = t / a.tiles_m * kMxTile, q0 = t % a.tiles_m * kMxTile;
    const uint8_t *w[4], *z[4], *ws[4], *zs[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        int64_t row = l0 + y * 16 + r;
        row = row < a.L ? row : a.L - 1;
        w[y] = a.Q + row * a.units * 64 + quarter * 16;
        ws[y] = a.scale + row * a.units * 4 + quarter;
        row = q0 + y * 16 + r;
        row = row < a.B ? row : a.B - 1;
        z[y] = a.P + row * a.units * 64 + quarter * 16;
        zs[y] = a.pscale + row * a.units * 4 + quarter;
    }
    mx_f32x4 acc[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[x][y] = mx_f32x4{0, 0, 0, 0};
    for (int u = 0; u < a.units; ++u) {
        mx_i32x4 fw[4], fz[4];
        int sw[4], sz[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            fw[y] = *reinterpret_cast<const mx_i32x4*>(w[y] + u * 64);
            fz[y] = *reinterpret_cast<const mx_i32x4*>(z[y] + u * 64);
            sw[y] = ws[y][u * 4];
            sz[y] = zs[y][u * 4];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = mx_product(fw[y], fz[x], acc[x][y], sw[y], sz[x]);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int64_t q = q0 + x * 16 + r;
        if (q >= a.B) continue;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t l = l0 + y * 16 + quarter * 4;
            if (l >= a.L) continue;
            const float v[4] = {acc[x][y][0], acc[x][y][1], acc[x][y][2], acc[x][y][3]};
            put_scores<TO>(static_cast<TO*>(a.out) + q * a.L + l, v, static_cast<int>(a.L - l < 4 ? a.L - l : 4));
        }
    }
}

// ---- sizes
static bool micro_d(int d, xc_dtype t) { return d >= 1 && d <= XC_MAX_D_QUANTIZED && (static_cast<int64_t>(d) * (t == XC_F32 ? 4 : 2)) % 16 == 0; }
static size_t micro_bytes(int64_t B, int d) { return static_cast<size_t>(B) * (mx_pitch(d) / 2) + round_up(static_cast<size_t>(B) * (mx_pitch(d) / 32), 16); }

}  // namespace xc

extern "C" int xc_microscale_rows(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count, uint8_t* Q,
                                  uint8_t* scale, void* stream) {
    using namespace xc;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (N < 1 || N > 0x7fffffffLL || !micro_d(d, t) || m < 0) return XC_ESHAPE;
    if (!X || !Q || !scale || (count && !ids)) return XC_EINVAL;
    if (!aligned16(X) || !aligned16(ids) || !aligned16(count) || !aligned16(Q) || !aligned16(scale)) return XC_EINVAL;
    const unsigned __int128 n = N;
    if (overlap({Span(Q, n * (mx_pitch(d) / 2)), Span(scale, n * (mx_pitch(d) / 32))},
                {Span(X, n * d * (t == XC_F32 ? 4 : 2)), Span(ids, static_cast<unsigned __int128>(m) * 4), Span(count, 4)}))
        return XC_EINVAL;
    if (ids && m == 0) return XC_OK;
    return launch_microscale(X, N, d, t, ids, m, count, Q, scale, static_cast<hipStream_t>(stream));
}

extern "C" int xc_scores_microscaled_workspace(int64_t B, int d, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (B < 1 || B > 0x7fffffffLL || d < 1 || d > XC_MAX_D_QUANTIZED) return XC_ESHAPE;
    *bytes = micro_bytes(B, d);
    return XC_OK;
}

extern "C" int xc_scores_microscaled(const void* Z, int64_t B, int d, xc_dtype t, const uint8_t* Q, const uint8_t* scale, int64_t L, xc_dtype out_t,
                                     void* out, void* ws, size_t ws_bytes, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (B < 1 || B > 0x7fffffffLL || L < 1 || L > 0x7fffffffLL || !micro_d(d, t) || static_cast<unsigned __int128>(B) * L > (1ull << 40)) return XC_ESHAPE;
    if (!Z || !Q || !scale || !out || !ws) return XC_EINVAL;
    if (!aligned16(Z) || !aligned16(Q) || !aligned16(scale) || !aligned16(out) || !aligned16(ws)) return XC_EINVAL;
    const size_t need = micro_bytes(B, d);
    if (ws_bytes < need) return XC_EWORKSPACE;
    const unsigned __int128 b = B, l = L;
    if (overlap({Span(out, b * l * (out_t == XC_F32 ? 4 : 2)), Span(ws, need)},
                {Span(Z, b * d * (t == XC_F32 ? 4 : 2)), Span(Q, l * (mx_pitch(d) / 2)), Span(scale, l * (mx_pitch(d) / 32))}))
        return XC_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint8_t* P = static_cast<uint8_t*>(ws);
    uint8_t* pscale = P + B * (mx_pitch(d) / 2);
    const int rc = launch_microscale(Z, B, d, t, nullptr, 0, nullptr, P, pscale, st);
    if (rc != XC_OK) return rc;
    const MicroArgs a{P, pscale, Q, scale, out, B, L, (B + kMxTile - 1) / kMxTile, (L + kMxTile - 1) / kMxTile, static_cast<int>(mx_pitch(d) / kMxRow)};
    const unsigned grid = static_cast<unsigned>((a.tiles_m * a.tiles_n + 3) / 4);
    if (out_t == XC_F32) XC_LAUNCH(K_SCORES_MICRO, st, (scores_micro_kernel<float><<<grid, 256, 0, st>>>(a)));
    else XC_LAUNCH(K_SCORES_MICRO, st, (scores_micro_kernel<bf16_t><<<grid, 256, 0, st>>>(a)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
