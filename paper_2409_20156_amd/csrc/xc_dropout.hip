// Dropout from the samplers' counter-based generator: the mask is formed where it is used, forward and backward, and never
// stored.  A 64-bit word of the generator serves four neighbouring elements of a row with 16 bits each.
#include <cmath>

#include "xc_common.h"

namespace xc {

constexpr int kDropThreads = 256;
constexpr int64_t kDropMany = 1024;         // workgroups from which on a thread takes four units
constexpr int64_t kDropUnits = 1ll << 31;    // of a launch, at most
constexpr uint64_t kDropoutKey = 0x64726F706F757431ull;

// N neighbouring elements at any address, `have` of them there.
template <int N> struct Unit {
    static __device__ __forceinline__ void load(const float* p, int have, float (&f)[N]) {
        if (have >= N) __builtin_memcpy(f, p, 4 * N);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = i < have ? p[i] : 0.0f;
        }
    }
    static __device__ __forceinline__ void load(const bf16_t* p, int have, float (&f)[N]) {
        uint32_t v[N / 2];
        if (have >= N) __builtin_memcpy(v, p, 2 * N);
        else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                v[i] = (2 * i < have ? p[2 * i].bits : 0u) | ((2 * i + 1 < have ? p[2 * i + 1].bits : 0u) << 16);
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(float* p, int have, const float (&f)[N]) {
        if (have >= N) __builtin_memcpy(p, f, 4 * N);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) if (i < have) p[i] = f[i];
        }
    }
    static __device__ __forceinline__ void store(bf16_t* p, int have, const float (&f)[N]) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        bf16x2 h[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) h[i] = __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2);      // nearest, ties to even
        if (have >= N) __builtin_memcpy(p, h, 2 * N);
        else {
#pragma unroll
            for (int i = 0; i < N; ++i) if (i < have) { const __bf16 x = h[i / 2][i & 1]; __builtin_memcpy(p + i, &x, 2); }
        }
    }
};

struct DropArgs {
    int64_t d, n_units;
    uint64_t row0;
    uint32_t units;                      // of a row
    uint32_t magic;                      // ceil(2^32 / units) for units < 1024
    uint32_t least;
    float scale;
    uint64_t key;
};

// A thread has K units of N neighbouring elements (16 bytes of the wider type, N / 4 words of the generator).  The first of the
// generator's two rounds is the same for a row: a workgroup forms it once per row it meets.
// Bound: memory, with the generator's 64-bit products close behind (about 16 vector instructions an element).  65536 x 768: fp32 to
// bf16 57 us (302 MB, 5.3 TB/s), fp32 76, bf16 43 to 49; 10240 x 768 bf16 7.9.  A thread per word with both rounds of its own took 94
// and 13; rows of 763 take as long as those of 768, though their units lie at any address.
template <typename TI, typename TO, int N, int K>
__global__ __launch_bounds__(kDropThreads)
void dropout_kernel(const TI* X, TO* Y, const DropArgs a) {
    constexpr int kUnits = K * kDropThreads;
    __shared__ uint64_t rows[kUnits + 1];
    const int64_t u0 = static_cast<int64_t>(blockIdx.x) * kUnits;
    const int64_t r0 = u0 / a.units;
    const uint32_t c0 = static_cast<uint32_t>(u0 - r0 * a.units);            // of row r0
    const int64_t left = a.n_units - u0;
    const int here = left < kUnits ? static_cast<int>(left) : kUnits;
    // row and unit within it of the workgroup's i-th unit; c0 + i < 2^11, or below 2 units
    auto place = [&](int i, uint32_t& r, uint32_t& c) __attribute__((always_inline)) {
        const uint32_t x = c0 + static_cast<uint32_t>(i);
        r = a.units >= 1024u ? (x >= a.units ? 1u : 0u) : a.units > 1u ? __umulhi(x, a.magic) : x;
        c = x - r * a.units;
    };
    float f[K][N];
    uint32_t row[K], col[K];
    int have[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = k * kDropThreads + static_cast<int>(threadIdx.x);
        have[k] = 0;
        if (i < here) {
            place(i, row[k], col[k]);
            const int64_t c = static_cast<int64_t>(col[k]) * N, rest = a.d - c;
            have[k] = rest < N ? static_cast<int>(rest) : N;
            Unit<N>::load(X + (r0 + row[k]) * a.d + c, have[k], f[k]);
        }
    }
    uint32_t last_r, last_c;
    place(here - 1, last_r, last_c);
    for (uint32_t r = threadIdx.x; r <= last_r; r += kDropThreads)
        rows[r] = fmix64(a.key ^ (kQueryMul * (a.row0 + static_cast<uint64_t>(r0) + r + 1)));
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (have[k] == 0) continue;
        const uint64_t base = rows[row[k]];
        float y[N];
#pragma unroll
        for (int w = 0; w < N / 4; ++w) {
            const uint64_t word = fmix64(base + kDrawMul * (static_cast<uint64_t>(col[k]) * (N / 4) + w + 1));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[4 * w + e] = (static_cast<uint32_t>(word >> (16 * e)) & 0xffffu) >= a.least ? f[k][4 * w + e] * a.scale : 0.0f;
        }
        Unit<N>::store(Y + (r0 + row[k]) * a.d + static_cast<int64_t>(col[k]) * N, have[k], y);
    }
}

template <typename TI, typename TO>
static int launch(const void* X, void* Y, int64_t B, int64_t d, uint32_t least, uint64_t seed, int64_t row0, hipStream_t st) {
    constexpr int N = sizeof(TI) == 2 && sizeof(TO) == 2 ? 8 : 4;
    DropArgs a;
    a.d = d;
    a.units = static_cast<uint32_t>((d + N - 1) / N);
    a.magic = a.units > 1 ? static_cast<uint32_t>(((1ull << 32) + a.units - 1) / a.units) : 0u;
    a.least = least;
    a.scale = static_cast<float>(65536.0 / (65536 - static_cast<int>(least)));
    a.key = seed ^ kDropoutKey;
    const TI* x = static_cast<const TI*>(X);
    TO* y = static_cast<TO*>(Y);
    const int64_t most = kDropUnits / a.units;
    for (int64_t b0 = 0; b0 < B; b0 += most) {
        const int64_t nb = B - b0 < most ? B - b0 : most;
        a.n_units = nb * a.units;
        a.row0 = static_cast<uint64_t>(row0) + static_cast<uint64_t>(b0);
        // four units to a thread where that leaves every compute unit several workgroups
        if (a.n_units >= kDropMany * 4 * kDropThreads)
            XC_LAUNCH(K_DROPOUT, st, (dropout_kernel<TI, TO, N, 4><<<static_cast<unsigned>((a.n_units + 4 * kDropThreads - 1) / (4 * kDropThreads)), kDropThreads, 0, st>>>(x + b0 * d, y + b0 * d, a)));
        else
            XC_LAUNCH(K_DROPOUT, st, (dropout_kernel<TI, TO, N, 1><<<static_cast<unsigned>((a.n_units + kDropThreads - 1) / kDropThreads), kDropThreads, 0, st>>>(x + b0 * d, y + b0 * d, a)));
    }
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

}  // namespace xc

extern "C" int xc_dropout(const void* X, xc_dtype t, int64_t B, int64_t d, float rate, uint64_t seed, int64_t row0, void* Y,
                          xc_dtype out_t, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (B < 1 || d < 1 || d > 0x7fffffffLL || B > (1LL << 40) / d) return XC_ESHAPE;
    if (!(rate >= 0.0f) || !(rate < 1.0f) || row0 < 0) return XC_EINVAL;
    const double least = std::floor(static_cast<double>(rate) * 65536.0 + 0.5);
    if (least > 65535.0) return XC_EINVAL;
    if (!X || !Y || !aligned16(X) || !aligned16(Y) || (X == Y && t != out_t)) return XC_EINVAL;
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(X), y0 = reinterpret_cast<uintptr_t>(Y), n = static_cast<uintptr_t>(B) * static_cast<uintptr_t>(d);
    if (X != Y && x0 < y0 + n * (out_t == XC_F32 ? 4 : 2) && y0 < x0 + n * (t == XC_F32 ? 4 : 2)) return XC_EINVAL;      // they overlap
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t m = static_cast<uint32_t>(least);
    if (t == XC_F32)
        return out_t == XC_F32 ? launch<float, float>(X, Y, B, d, m, seed, row0, st) : launch<float, bf16_t>(X, Y, B, d, m, seed, row0, st);
    return out_t == XC_F32 ? launch<bf16_t, float>(X, Y, B, d, m, seed, row0, st) : launch<bf16_t, bf16_t>(X, Y, B, d, m, seed, row0, st);
}
