// Rows in 8 bits, and the scores of all labels from them: out = (<p, q> a) b with integers p, q and a scale per row on
// either side.  The integer sums are exact, so their order (and how the work is cut) cannot change a score.
#include "xc_common.h"

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
                     const int32_t* __restrict__ count, int8_t* __restrict__ Q, float* __restrict__ scale) {
    constexpr int kPer = Row<T>::kPer;
    const int pitch = quantized_pitch(d), chunks = d / kPer, lane = lane_id();
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
                           int8_t* Q, float* scale, hipStream_t st) {
    const int64_t rows = ids != nullptr ? m : N;
    if (rows == 0) return XC_OK;
    const int64_t want = (rows + 3) / 4;
    const unsigned grid = static_cast<unsigned>(want < 16384 ? want : 16384);
    const unsigned char* x = static_cast<const unsigned char*>(X);
    if (t == XC_F32)
        XC_LAUNCH(K_QUANTIZE, st, (quantize_kernel<float><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, scale)));
    else
        XC_LAUNCH(K_QUANTIZE, st, (quantize_kernel<bf16_t><<<grid, 256, 0, st>>>(x, N, d, ids, m, count, Q, scale)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
// A wave multiplies 32 queries with 32 labels, operands straight from memory.  Accumulator i of a lane: label lane % 32,
// query 8 (i / 4) + 4 (lane / 32) + i % 4.
template <typename TO>
__global__ __launch_bounds__(256)
void scores_kernel(const int8_t* __restrict__ P, const float* __restrict__ pscale, int64_t B, const int8_t* __restrict__ Q,
                   const float* __restrict__ scale, int64_t L, int pitch, TO* __restrict__ out) {
    const int lane = lane_id(), half = lane >> 5;
    const int64_t l0 = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6)) * 32, q0 = static_cast<int64_t>(blockIdx.y) * 32;
    if (l0 >= L) return;
    const int64_t l = l0 + (lane & 31), q = q0 + (lane & 31);
    const int8_t* wr = Q + (l < L ? l : L - 1) * pitch + half * 16;
    const int8_t* zr = P + (q < B ? q : B - 1) * pitch + half * 16;
    i32x16 acc = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    for (int k = 0; k < pitch; k += 32) {
        i32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        if (k + half * 16 < pitch) {
            a = *reinterpret_cast<const i32x4*>(zr + k);
            b = *reinterpret_cast<const i32x4*>(wr + k);
        }
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
    if (l >= L) return;
    const float sl = scale[l];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t r = q0 + 8 * (i >> 2) + 4 * half + (i & 3);
        if (r < B) {
            const float v = (static_cast<float>(acc[i]) * pscale[r]) * sl;
            if constexpr (sizeof(TO) == 4) out[r * L + l] = v;
            else out[r * L + l].bits = static_cast<uint16_t>(float_to_bf16_bits(v));
        }
    }
}

static size_t scores_bytes(int64_t B, int d) {
    return round_up(static_cast<size_t>(B) * 4, 256) + static_cast<size_t>(B) * quantized_pitch(d);
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
    return launch_quantize(X, N, d, t, ids, m, count, Q, scale, static_cast<hipStream_t>(stream));
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
    const int rc = launch_quantize(Z, B, d, t, nullptr, 0, nullptr, P, pscale, st);
    if (rc != XC_OK) return rc;
    const int pitch = quantized_pitch(d);
    // (65535 blocks of queries to a launch)
    for (int64_t b0 = 0; b0 < B; b0 += 65535 * 32) {
        const int64_t nb = B - b0 < 65535 * 32 ? B - b0 : 65535 * 32;
        const dim3 grid(static_cast<unsigned>((L + 127) / 128), static_cast<unsigned>((nb + 31) / 32));
        if (out_t == XC_F32)
            XC_LAUNCH(K_SCORES, st, (scores_kernel<float><<<grid, 256, 0, st>>>(P + b0 * pitch, pscale + b0, nb, Q, scale, L, pitch,
                                                                                static_cast<float*>(out) + b0 * L)));
        else
            XC_LAUNCH(K_SCORES, st, (scores_kernel<bf16_t><<<grid, 256, 0, st>>>(P + b0 * pitch, pscale + b0, nb, Q, scale, L, pitch,
                                                                                 static_cast<bf16_t*>(out) + b0 * L)));
        XC_HIP_CHECK(hipGetLastError());
    }
    return XC_OK;
}
