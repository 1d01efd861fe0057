// Dropout from the samplers' counter-based generator: the mask is formed where it is used, forward and backward, and never
// stored.  A 64-bit word of the generator serves four neighbouring elements of a row with 16 bits each.
#include <cmath>

#include "xc_common.h"

namespace xc {

constexpr int kDropThreads = 256;
constexpr uint64_t kDropoutKey = 0x64726F706F757431ull;

template <typename T> __device__ __forceinline__ float element(const T* p);
template <> __device__ __forceinline__ float element<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float element<bf16_t>(const bf16_t* p) { return bf16_bits_to_float(p->bits); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = static_cast<uint16_t>(float_to_bf16_bits(v)); }

// One thread per word.
template <typename TI, typename TO>
__global__ __launch_bounds__(kDropThreads)
void dropout_kernel(const TI* X, TO* Y, int64_t B, int64_t d, int64_t groups, uint32_t least, float scale, uint64_t key,
                    int64_t row0) {
    const int64_t n = B * groups, step = static_cast<int64_t>(gridDim.x) * kDropThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kDropThreads + threadIdx.x; i < n; i += step) {
        const int64_t row = i / groups, g = i % groups;
        const uint64_t word = fmix64(fmix64(key ^ (kQueryMul * static_cast<uint64_t>(row0 + row + 1))) +
                                     kDrawMul * static_cast<uint64_t>(g + 1));
        for (int e = 0; e < 4 && 4 * g + e < d; ++e) {
            const int64_t at = row * d + 4 * g + e;
            const float x = element(X + at);
            put(Y + at, (static_cast<uint32_t>(word >> (16 * e)) & 0xffffu) >= least ? x * scale : 0.0f);
        }
    }
}

template <typename TI, typename TO>
static int launch(const void* X, void* Y, int64_t B, int64_t d, uint32_t least, uint64_t seed, int64_t row0, hipStream_t st) {
    const int64_t groups = (d + 3) / 4, n = B * groups;
    const float scale = static_cast<float>(65536.0 / (65536 - static_cast<int>(least)));
    const int64_t want = (n + kDropThreads - 1) / kDropThreads;
    const unsigned grid = static_cast<unsigned>(want < 65536 ? want : 65536);
    XC_LAUNCH(K_DROPOUT, st, (dropout_kernel<TI, TO><<<grid, kDropThreads, 0, st>>>(
        static_cast<const TI*>(X), static_cast<TO*>(Y), B, d, groups, least, scale, seed ^ kDropoutKey, row0)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

}  // namespace xc

extern "C" int xc_dropout(const void* X, xc_dtype t, int64_t B, int64_t d, float rate, uint64_t seed, int64_t row0, void* Y,
                          xc_dtype out_t, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (B < 1 || d < 1 || d > 0x7fffffffLL || B > (1LL << 60) / d) return XC_ESHAPE;
    if (!(rate >= 0.0f) || !(rate < 1.0f) || row0 < 0) return XC_EINVAL;
    const double least = std::floor(static_cast<double>(rate) * 65536.0 + 0.5);
    if (least > 65535.0) return XC_EINVAL;
    if (!X || !Y || !aligned16(X) || !aligned16(Y) || (X == Y && t != out_t)) return XC_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t m = static_cast<uint32_t>(least);
    if (t == XC_F32)
        return out_t == XC_F32 ? launch<float, float>(X, Y, B, d, m, seed, row0, st) : launch<float, bf16_t>(X, Y, B, d, m, seed, row0, st);
    return out_t == XC_F32 ? launch<bf16_t, float>(X, Y, B, d, m, seed, row0, st) : launch<bf16_t, bf16_t>(X, Y, B, d, m, seed, row0, st);
}
