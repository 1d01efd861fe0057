// Rows in 4-bit floating point with shared scales, and the scores of all labels from them.
// 32 neighbouring elements of a row share a scale 2^(byte - 127); an element is a sign, two bits of exponent and one of mantissa: 0, 0.5, 1,
// 1.5, 2, 3, 4 or 6.  The largest magnitude of a block decides the scale: the power of two that brings it into [4, 8).  What lies beyond 6
// then is 6 (the format's published conversion, so that rows laid out elsewhere mean the same here).
#include "xc_microscaled_choice.h"
#include "xc_mine.h"

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

// Codes and scale byte of a lane's 8 elements; four lanes have a block.
struct MicroLane { uint32_t codes, byte, bytes; };       // bytes: of four blocks, in every 16th lane
__device__ __forceinline__ MicroLane to_micro(float (&f)[8]) {
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = __float_as_uint(f[e]) & 0x7fffffffu;
        big = b > big ? b : big;
    }
    big = quad_max(big);
    const bool finite = big < 0x7f800000u;
    const uint32_t exponent = big >> 23, byte = exponent > 2u ? exponent - 2u : 0u;
    const float inv = __uint_as_float((254u - (finite ? byte : 0u)) << 23);            // (a power of two: products are exact, or far below 0.25)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= inv;
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], 1.0f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], 1.0f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], 1.0f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], 1.0f, 3);
    const uint32_t b = finite ? byte : 255u;
    uint32_t all = b;
    all |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b), 0x104, 0xf, 0xf, false)) << 8;         // row_shl 4, 8, 12
    all |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b), 0x108, 0xf, 0xf, false)) << 16;
    all |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b), 0x10c, 0xf, 0xf, false)) << 24;
    return MicroLane{finite ? codes : 0u, b, all};
}

// Rows of 4 bits where they are kept: Q (64 bytes to 128 elements) and their scales row by row.
struct MicroRows {
    uint8_t *Q, *scale;
    int units;                           // of 128 elements in a row
    __device__ __forceinline__ void put(int64_t row, int u, int sub, const MicroLane& m) const {
        *reinterpret_cast<uint32_t*>(Q + (row * units + u) * 64 + sub * 4) = m.codes;
        if (sub == 0) *reinterpret_cast<uint32_t*>(scale + (row * units + u) * 4) = m.bytes;
    }
};
// Queries in the workspace: rows of `pitch` bytes (an even number of units), zeros behind the last element and the last query.  A row's
// scales are laid out as the products of labels held in registers ask for them: block 4 u + b of unit u at b * upad + u, so that a lane
// finds four units' in a word.  (Long rows are staged like the labels, and kept like them: MicroRows.)
struct MicroQueries {
    uint8_t *P, *scale;
    int units, pitch, upad;
    __device__ __forceinline__ void put(int64_t row, int u, int sub, const MicroLane& m) const {
        *reinterpret_cast<uint32_t*>(P + row * pitch + u * 64 + sub * 4) = m.codes;
        if ((sub & 3) == 0 && u < upad) scale[row * 4 * upad + (sub >> 2) * upad + u] = static_cast<uint8_t>(m.byte);
    }
};

// 16 lanes bring 128 elements of a row, U of these at a time.  Rows from N on (of the queries' padding) and units behind a row are zeros.
// Bound: memory.  670000 x 768 bf16: 240 us, 5.4 TB/s, what a copy reaches here; one at a time 252, four 237, with the non-temporal hint 240.
// Listed rows of as many: 100000 42.7 us (4.6 TB/s), 20000 10.1, 1000 7.7 (the caller's).
template <typename T, typename TO, int U>
__global__ __launch_bounds__(256)
void microscale_kernel(const unsigned char* __restrict__ X, int64_t N, int d, const int32_t* __restrict__ ids, int64_t m, const int32_t* __restrict__ count,
                       const TO out, int64_t n_rows, int units /* written of a row */) {
    const int sub = threadIdx.x & 15;
    int64_t rows = ids != nullptr ? m : n_rows;
    if (ids != nullptr && count != nullptr) {
        const int64_t c = count[0];
        rows = c < rows ? c : rows;
    }
    const int64_t total = rows * units, step = static_cast<int64_t>(gridDim.x) * (16 * U);
    const bool small = total <= 0xffffffffLL;                // uniform: divided in 32 bits
    for (int64_t u0 = static_cast<int64_t>(blockIdx.x) * (16 * U) + (threadIdx.x >> 4); u0 < total; u0 += step) {
        float f[U][8];
        int64_t row[U];
        int col[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t u = u0 + k * 16;
            row[k] = -1;
            if (u >= total) continue;
            const int64_t i = small ? static_cast<uint32_t>(u) / static_cast<uint32_t>(units) : u / units;
            col[k] = static_cast<int>(u - i * units);
            row[k] = ids != nullptr ? ids[i] : i;
            const bool there = row[k] >= 0 && row[k] < N;                  // (the same for 16 lanes)
            if (!there && ids != nullptr) { row[k] = -1; continue; }
            eight<T>(X + (there ? row[k] : 0) * d * static_cast<int64_t>(sizeof(T) == 4 ? 4 : 2), there ? col[k] * kMxRow + sub * 8 : d, d, f[k]);
        }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (row[k] >= 0) out.put(row[k], col[k], sub, to_micro(f[k]));
    }
}

constexpr int64_t kMxGrid = 1 << 20;
template <typename TO>
static int launch_microscale(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count, const TO& out, int64_t n_rows, int units,
                             hipStream_t st) {
    const int64_t rows = ids != nullptr ? m : n_rows, total = rows * units;
    const unsigned char* x = static_cast<const unsigned char*>(X);
    auto go = [&](auto kernel, int U) {
        const int64_t want = (total + 16 * U - 1) / (16 * U);
        kernel<<<static_cast<unsigned>(want < kMxGrid ? want : kMxGrid), 256, 0, st>>>(x, N, d, ids, m, count, out, n_rows, units);
    };
    const bool many = total > 256 * 16 * 8;
    if (t == XC_F32) XC_LAUNCH(K_MICROSCALE, st, (many ? go(microscale_kernel<float, TO, 2>, 2) : go(microscale_kernel<float, TO, 1>, 1)));
    else XC_LAUNCH(K_MICROSCALE, st, (many ? go(microscale_kernel<bf16_t, TO, 2>, 2) : go(microscale_kernel<bf16_t, TO, 1>, 1)));
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------
struct MicroArgs {
    const unsigned char* Z;              // queries as they came (the kernel that brings them to 4 bits itself)
    const uint8_t *P, *pscale;           // queries in 4 bits
    const uint8_t *Q, *scale;
    void* out;
    int64_t B, L;
    int d, units, ppitch, upad;          // units of 128 elements in a row of Q; the queries' rows, see MicroQueries
    bool stream;                         // scores beyond the last-level cache: stored with the non-temporal hint
};

// Blocks of 16 queries x 16 labels x 128 elements: lane l has the 32 elements of block l / 16 of row l % 16 of both operands; its
// accumulator i is query 4 (l / 16) + i, label l % 16 of the block.  A word of scale bytes holds four units', of which S is taken.
// In every kernel a score is the sum over its units in order, from 0: its bits do not depend on the kernel.
template <int S>
__device__ __forceinline__ mx_f32x4 mx_product(const mx_i32x4& z, const mx_i32x4& w, const mx_f32x4& c, int zs, int ws) {
    const mx_i32x8 a = {z.x, z.y, z.z, z.w, 0, 0, 0, 0}, b = {w.x, w.y, w.z, w.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4 /* fp4 */, 4, S, zs, S, ws);
}
__device__ __forceinline__ mx_f32x4 mx_product(int s /* known when compiled */, const mx_i32x4& z, const mx_i32x4& w, const mx_f32x4& c, int zs, int ws) {
    switch (s & 3) {
        case 0: return mx_product<0>(z, w, c, zs, ws);
        case 1: return mx_product<1>(z, w, c, zs, ws);
        case 2: return mx_product<2>(z, w, c, zs, ws);
        default: return mx_product<3>(z, w, c, zs, ws);
    }
}

// 4 neighbouring scores of a row, the first `have` of which are there.
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t mx_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void put_four(float* p, const float (&v)[4], bool stream) {
    mx_u32x4 u;
    __builtin_memcpy(&u, v, 16);
    if (stream) __builtin_nontemporal_store(u, reinterpret_cast<mx_u32x4*>(p));      // uniform
    else *reinterpret_cast<mx_u32x4*>(p) = u;
}
__device__ __forceinline__ void put_four(bf16_t* p, const float (&v)[4], bool stream) {
    const mx_bf16x2 h[2] = {__builtin_convertvector(mx_f32x2{v[0], v[1]}, mx_bf16x2), __builtin_convertvector(mx_f32x2{v[2], v[3]}, mx_bf16x2)};      // nearest, ties to even
    mx_u32x2 u;
    __builtin_memcpy(&u, h, 8);
    if (stream) __builtin_nontemporal_store(u, reinterpret_cast<mx_u32x2*>(p));
    else *reinterpret_cast<mx_u32x2*>(p) = u;
}
__device__ __forceinline__ void put_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_one(bf16_t* p, float v) {
    const __bf16 h = static_cast<__bf16>(v);
    __builtin_memcpy(p, &h, 2);
}
// (`whole` is the same for a wave: the stores one by one are left out where all labels of the wave are there)
template <typename TO> __device__ __forceinline__ void put_labels(TO* p, const float (&v)[4], bool whole, int64_t have) {
    if (whole) {
        put_four(p, v, false);
    } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) if (y < have) put_one(p + y, v[y]);
    }
}
__device__ __forceinline__ int mx_swizzle(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ const void* mx_uniform(const void* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const void*>(
        (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32)))) << 32) |
        static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a)))));
}

// ---- up to 16 queries: they stay in LDS (rows of up to 64 KU bytes), the labels pass, 64 to a wave at a time and two units of each to a
// step, through a ring of R steps in LDS that the wave fills and empties by itself.  Eight neighbouring lanes bring 128 bytes of a row, so
// that a load meets eight lines; straight into registers, where neighbouring lanes have different rows, it meets 64, and so do a row's
// scales: 1 x 131072 x 768 14.5 us, 1 x 670000 x 768 68, against 10.2 and 51 (5.3 TB/s).  Lane l has labels 4 (l % 16) .. + 3 of the 64, so
// that it stores neighbouring scores.  TZ: what the queries are brought to 4 bits from by every workgroup for itself (void: they are in the workspace).
// Bound: one read of Q.
constexpr int kFewSlot = 64 * 128 + 2 * 64 * 4;          // a step of 64 labels, their scales
constexpr int kFewLoads = 8 + 2;
template <int N> __device__ __forceinline__ void few_wait() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }
__device__ __forceinline__ void lds_dma4_sbase(const void* sbase /* wave-uniform */, uint32_t voff, uint32_t lds_addr /* wave-uniform */) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(voff), "s"(sbase), "s"(lds_addr) : "memory");
}
template <typename TO, typename TZ, int KU, int W, int R>
__global__ __launch_bounds__(W * kWave)
void scores_micro_few_kernel(const MicroArgs a) {
    constexpr int kRows = kMicroFewQueries, kUpad = (KU + 3) / 4 * 4;
    __shared__ __align__(1024) unsigned char ring[W][R][kFewSlot];
    __shared__ __align__(1024) unsigned char codes[kRows * KU * 64];       // 128 bytes of every row, the next 128, ..; chunks of 16 swizzled
    __shared__ __align__(16) unsigned char scales[kRows * 4 * kUpad];
    static_assert((R - 1) * kFewLoads < 64, "a count that the wait can hold");
    const int lane = lane_id(), r = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t groups = (a.L + 63) / 64;
    const uint32_t row_bytes = a.units * 64, row_scales = a.units * 4;
    // neighbouring groups to neighbouring waves, and a contiguous part of them to each XCD
    const int64_t per = (groups + kXcds - 1) / kXcds, g_begin = blockIdx.x % kXcds * per, g_end = g_begin + per < groups ? g_begin + per : groups;
    const int64_t g_step = static_cast<int64_t>(gridDim.x / kXcds) * W;
    int64_t g = g_begin + static_cast<int64_t>(blockIdx.x / kXcds) * W + wave, ahead_g = g;
    const int steps = (a.units + 1) / 2;
    const int64_t total = g < g_end ? ((g_end - 1 - g) / g_step + 1) * steps : 0;
    int ahead_step = 0, ahead_slot = 0;
    unsigned char* slots = &ring[wave][0][0];
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)slots));
    auto issue = [&]() __attribute__((always_inline)) {
        const int64_t l0 = ahead_g * 64, have = a.L - 1 - l0;
        const uint32_t last = have < 63 ? static_cast<uint32_t>(have) : 63u;           // rows past the end: the last one again
        const uint32_t mask = ahead_step * 2 + 1 < a.units ? 127u : 63u;                // (a single unit: it again)
        const void* q = mx_uniform(a.Q + l0 * row_bytes + ahead_step * 128);
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + ahead_slot * kFewSlot);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t row = i * 8 + (lane >> 3), chunk = (lane ^ (row >> 2)) & 7;
            lds_dma16_sbase<0>(q, (row < last ? row : last) * row_bytes + ((chunk * 16) & mask), to + i * 1024);
        }
        const void* s = mx_uniform(a.scale + l0 * row_scales + ahead_step * 8);
        const uint32_t at = (static_cast<uint32_t>(lane) < last ? lane : last) * row_scales;
        lds_dma4_sbase(s, at, to + 64 * 128);
        lds_dma4_sbase(s, at + (mask == 127u ? 4 : 0), to + 64 * 128 + 256);
        if (++ahead_step == steps) {
            ahead_step = 0;
            ahead_g += g_step;
        }
        if (++ahead_slot == R) ahead_slot = 0;
    };
    for (int i = 0; i < R && i < total; ++i) issue();

    // the queries; rows past the last one are zeros
    if constexpr (!std::is_void<TZ>::value) {
        const int rows = static_cast<int>(a.B), all = rows * a.units;
        if (rows < kRows) {
            for (int i = threadIdx.x; i < kRows * KU * 4; i += W * kWave)
                if ((i >> 3) % kRows >= rows) *reinterpret_cast<uint4*>(codes + i * 16) = make_uint4(0, 0, 0, 0);
            for (int i = rows * kUpad + static_cast<int>(threadIdx.x); i < kRows * kUpad; i += W * kWave) *reinterpret_cast<uint32_t*>(scales + i * 4) = 0;
        }
        constexpr int U = 4;                                 // of 128 elements, under way together
        const int sub = threadIdx.x & 15;
        for (int i0 = threadIdx.x >> 4; i0 < all; i0 += W * 4 * U) {
            float f[U][8];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * W * 4, row = i / a.units, u = i - row * a.units;
                if (i < all) eight<TZ>(a.Z + row * a.d * static_cast<int64_t>(sizeof(TZ) == 4 ? 4 : 2), u * kMxRow + sub * 8, a.d, f[k]);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * W * 4, row = i / a.units, u = i - row * a.units;
                if (i >= all) break;
                const MicroLane m = to_micro(f[k]);
                *reinterpret_cast<uint32_t*>(codes + (u >> 1) * (kRows * 128) + row * 128 + ((((u & 1) * 4 + (sub >> 2)) ^ mx_swizzle(row)) * 16) + (sub & 3) * 4) = m.codes;
                if ((sub & 3) == 0) scales[row * (4 * kUpad) + (sub >> 2) * kUpad + u] = static_cast<unsigned char>(m.byte);
            }
        }
    } else {
        const int chunks = a.ppitch / 16;
        for (int i = threadIdx.x; i < kRows * chunks; i += W * kWave) {
            const int row = i / chunks, c = i - row * chunks;
            *reinterpret_cast<uint4*>(codes + (c >> 3) * (kRows * 128) + row * 128 + (((c & 7) ^ mx_swizzle(row)) * 16)) =
                *reinterpret_cast<const uint4*>(a.P + row * a.ppitch + c * 16);
        }
        for (int i = threadIdx.x; i < kRows * a.upad; i += W * kWave) {    // words of 4 units
            const int row = i / a.upad, c = i - row * a.upad, b = c / (a.upad / 4), k = c - b * (a.upad / 4);
            *reinterpret_cast<uint32_t*>(scales + row * (4 * kUpad) + b * kUpad + k * 4) =
                *reinterpret_cast<const uint32_t*>(a.pscale + row * 4 * a.upad + b * a.upad + k * 4);
        }
    }
    __syncthreads();
    const int frag = r * 128 + ((quarter ^ mx_swizzle(r)) * 16);
    mx_f32x4 acc[4];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int y = 0; y < 4; ++y) acc[y] = mx_f32x4{0, 0, 0, 0};
    };
    clear();
    int step = 0, slot = 0;
    for (int64_t n = 0; n < total; ++n) {
        // (the waits count loads and stores, in the order of their issue: with stores among the younger ones they end a little later)
        if (total - 1 - n >= R - 1) few_wait<(R - 1) * kFewLoads>();
        else few_wait<0>();
        const unsigned char* from = slots + slot * kFewSlot;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int u = step * 2 + h;
            if (u >= a.units) break;                         // uniform
            mx_i32x4 w[4];
            int ws[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                w[y] = *reinterpret_cast<const mx_i32x4*>(from + (r * 4 + y) * 128 + (((h * 4 + quarter) ^ (r & 7)) * 16));
                ws[y] = from[64 * 128 + h * 256 + (r * 4 + y) * 4 + quarter];
            }
            const mx_i32x4 z = *reinterpret_cast<const mx_i32x4*>(codes + (u >> 1) * (kRows * 128) + (frag ^ ((u & 1) * 64)));
            const int zs = scales[r * (4 * kUpad) + quarter * kUpad + u];
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[y] = mx_product<0>(z, w[y], acc[y], zs, ws[y]);
        }
        if (n + R < total) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // (the slot has been read)
            issue();
        }
        if (++slot == R) slot = 0;
        if (++step == steps) {
            step = 0;
            const int64_t l = g * 64 + r * 4, have = a.L - l;
            const bool whole = g * 64 + 64 <= a.L;           // uniform
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t q = quarter * 4 + i;
                if (q >= a.B) continue;
                const float v[4] = {acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
                put_labels(static_cast<TO*>(a.out) + q * a.L + l, v, whole, have);
            }
            clear();
            g += g_step;
        }
    }
}

// ---- many queries, rows of up to 512 bytes (1024 elements): the labels stay where they are.  A wave holds 64 labels as operands in registers
// (NK units) and 512 labels of a workgroup meet the queries that stream through LDS, 64 at a time; a wave's scores are stored 16 queries at
// a time, while the other wave of its SIMD multiplies.
// Bound: stores and products that overlap in part.  4096 x 131072 x 768 to bf16 235 to 262 us (1.07 GB stored, 157 us of a fill; matrix pipe
// busy 47 % of the time); without the stores 163, with a sixth of the products 208: the stores as they are made here take more than a fill does,
// and the eight waves load, store and meet at a barrier in every stage, so that both waves of a SIMD tend to be in the same phase.  To fp32 400
// (2.15 GB, 316 us of a fill).
template <int NK_>
struct MicroHeld {
    static constexpr int NK = NK_, QS = kMicroHeldQueries, kUpad = NK <= 4 ? 4 : 8, kStage = QS * NK * 64, kScales = QS * 4 * kUpad;
    static constexpr int kTurn = 2048;                                                       // of a wave, to turn its labels in
    static constexpr int kFit = (160 * 1024 - 8 * kTurn - 1024) / (kStage + kScales), R = kFit < 6 ? kFit : 6;        // stages in LDS
    static constexpr int kLoads = kStage / 1024 / 8, kStores = QS / 4;                      // of a wave and stage
    static constexpr int kLds = R * (kStage + kScales) + 8 * kTurn;
    static_assert(kLoads * 8 * 1024 == kStage && R >= 3 && (kLoads + kStores) * (R - 3) < 64, "whole loads, and a count that the wait can hold");
};
constexpr int kMicroPieces = 4;                          // of the tiles behind the last whole round, to a workgroup

template <typename TO, int NK>
__global__ __launch_bounds__(512, 2)
void scores_micro_held_kernel(const MicroArgs a, int tiles, int stages) {
    typedef MicroHeld<NK> H;
    __shared__ __align__(1024) unsigned char smem[H::kLds];
    __shared__ int4 last[kMicroPieces + 1];
    const int lane = lane_id(), quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
    // Each XCD takes neighbouring tiles of labels, a workgroup one of every 32, so that the lines that two tiles share are written at
    // about the same time.  Of the last tiles, fewer than 32, a workgroup has an equal number of stages.
    const int xcd = blockIdx.x % kXcds, nth = blockIdx.x / kXcds;
    const int t_begin = static_cast<int>(static_cast<int64_t>(tiles) * xcd / kXcds) + nth;
    const int t_count = static_cast<int>(static_cast<int64_t>(tiles) * (xcd + 1) / kXcds) + nth - t_begin, rounds = t_count / kCusPerXcd;
    if (threadIdx.x == 0) {
        const int rest = t_count % kCusPerXcd, first = t_begin - nth + rounds * kCusPerXcd;
        const int64_t all = static_cast<int64_t>(rest) * stages, u1 = all * (nth + 1) / kCusPerXcd;
        int n = 0, sum = 0;
        for (int64_t u = all * nth / kCusPerXcd; u < u1;) {                // (less than a tile's stages: two tiles at most)
            const int t = static_cast<int>(u / stages), s = static_cast<int>(u - static_cast<int64_t>(t) * stages);
            const int e = stages - s < u1 - u ? stages : s + static_cast<int>(u1 - u);
            last[n++] = make_int4(first + t, s, e, 0);
            sum += e - s;
            u += e - s;
        }
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
        off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(NK * 64) + n / (H::QS / 8) * 128 + (((lane & 7) ^ mx_swizzle(row)) * 16);
    }
    int n_piece = 0, ld_piece = 0;
    int ld_st = st, ld_end = st_end, ld_slot = 0, n_issued = 0;
    auto issue = [&]() __attribute__((always_inline)) {
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds + ld_slot * H::kStage);
        if (wave < H::kScales / 1024)
            lds_dma16_sbase<0>(mx_uniform(a.pscale + static_cast<int64_t>(ld_st) * H::kScales + wave * 1024), lane * 16,
                               __builtin_amdgcn_readfirstlane(lds + H::R * H::kStage + ld_slot * H::kScales + wave * 1024));
        const void* from = mx_uniform(a.P + static_cast<int64_t>(ld_st) * H::kStage);
#pragma unroll
        for (int i = 0; i < H::kLoads; ++i) lds_dma16_sbase<0>(from, off[i], dst + (wave * H::kLoads + i) * 1024);
        if (++ld_st == ld_end) piece(++ld_piece, ld_tile, ld_st, ld_end);
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

    constexpr int kDepth = 3;                                // units whose queries are read ahead
    mx_i32x4 w[NK][4], fa[kDepth + 1];
    int sw[4][H::kUpad / 4];                                 // scale bytes of four units to a word
    const int frag = (lane & 15) * 128 + ((quarter ^ mx_swizzle(lane & 15)) * 16);
    auto read_a = [&](int slot, int qb, int k) __attribute__((always_inline)) {      // 16 queries, 64 bytes of each
        return *reinterpret_cast<const mx_i32x4*>(smem + slot * H::kStage + (k >> 1) * (H::QS * 128) + qb * 2048 + (frag ^ ((k & 1) * 64)));
    };
    struct Words { int v[H::kUpad / 4]; };
    auto read_s = [&](int slot, int qb) __attribute__((always_inline)) {             // their scales
        return *reinterpret_cast<const Words*>(smem + H::R * H::kStage + slot * H::kScales + (qb * 16 + (lane & 15)) * (4 * H::kUpad) + quarter * H::kUpad);
    };
    unsigned char* turn = smem + H::R * (H::kStage + H::kScales) + wave * H::kTurn;
    // The wave's labels: 4 neighbouring ones to a lane.  Four neighbouring lanes load 64 bytes of a row, so that a load meets 16 lines and
    // not 64, and are turned into the operands' order through LDS.
    auto hold = [&](int64_t l0) __attribute__((always_inline)) {
        const int64_t l = l0 + wave * 64;
        const int64_t past = a.L - 1 - l;                    // (a wave behind the last label: that one again)
        const int64_t row_bytes = a.units * 64, row_scales = a.units * 4;
        uint32_t words[NK];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t row = (lane >> 2) * 4 + y, at = l + (row < past ? row : past);
            const uint8_t* p = a.Q + at * row_bytes + (lane & 3) * 16;
#pragma unroll
            for (int k = 0; k < NK; ++k) w[k][y] = *reinterpret_cast<const mx_i32x4*>(p + (k < a.units ? k : a.units - 1) * 64);
        }
        {
            const uint8_t* p = a.scale + (l + (lane < past ? lane : past)) * row_scales;
#pragma unroll
            for (int k = 0; k < NK; ++k) words[k] = *reinterpret_cast<const uint32_t*>(p + (k < a.units ? k : a.units - 1) * 4);
        }
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                unsigned char* t = turn + (y & 1) * 1024;
                *reinterpret_cast<mx_i32x4*>(t + lane * 16) = w[k][y];
                w[k][y] = *reinterpret_cast<const mx_i32x4*>(t + ((lane & 15) * 4 + quarter) * 16);
                if (k >= a.units) w[k][y] = mx_i32x4{0, 0, 0, 0};          // uniform
            }
#pragma unroll
        for (int k = 0; k < NK; ++k) *reinterpret_cast<uint32_t*>(turn + k * 256 + lane * 4) = words[k];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
#pragma unroll
            for (int j = 0; j < H::kUpad / 4; ++j) sw[y][j] = 0;
#pragma unroll
            for (int k = 0; k < NK; ++k)
                if (k < a.units) sw[y][k >> 2] |= static_cast<int>(static_cast<uint32_t>(turn[k * 256 + ((lane & 15) * 4 + y) * 4 + quarter]) << ((k & 3) * 8));
        }
        // awaited here: the loop over the stages would wait for these (and for all loads and stores under way) every time round
#pragma unroll
        for (int y = 0; y < 4; ++y) {
#pragma unroll
            for (int j = 0; j < H::kUpad / 4; ++j) asm volatile("" : "+v"(sw[y][j]));
#pragma unroll
            for (int k = 0; k < NK; ++k) asm volatile("" : "+v"(w[k][y]));
        }
    };
    hold(static_cast<int64_t>(tile) * kMicroHeldLabels);
    publish(0);
#pragma unroll
    for (int n = 0; n < kDepth; ++n) fa[n] = read_a(0, n / NK, n % NK);
    Words zs = read_s(0, 0), zs_next = zs;
    int slot = 0;
    constexpr int kBlocks = H::QS / 16;
    static_assert(NK * kBlocks % (kDepth + 1) == 0 && kDepth <= NK * kBlocks, "a stage begins with the same registers");
    for (int g = 0; g < total; ++g) {
        const int64_t l0 = static_cast<int64_t>(tile) * kMicroHeldLabels + wave * 64, l = l0 + (lane & 15) * 4;
        const int64_t q0 = static_cast<int64_t>(st) * H::QS;
        const bool whole = q0 + H::QS <= a.B && l0 + 64 <= a.L;
        const int slot_next = slot + 1 == H::R ? 0 : slot + 1;
        TO* out = static_cast<TO*>(a.out) + (q0 + 4 * quarter) * a.L + l;
#pragma unroll
        for (int qb = 0; qb < kBlocks; ++qb) {
            if (qb == (NK * kBlocks - kDepth) / NK && g + 1 < total) publish(g + 1);       // (from here on the next stage is read)
            mx_f32x4 acc[4];
            zs_next = qb + 1 < kBlocks ? read_s(slot, qb + 1) : read_s(slot_next, 0);
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const int n = qb * NK + k, ahead = n + kDepth;             // of the stage's units
                fa[ahead % (kDepth + 1)] = ahead < NK * kBlocks ? read_a(slot, ahead / NK, ahead % NK) : read_a(slot_next, (ahead - NK * kBlocks) / NK, (ahead - NK * kBlocks) % NK);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    acc[y] = mx_product(k, fa[n % (kDepth + 1)], w[k][y], k == 0 ? mx_f32x4{0, 0, 0, 0} : acc[y], zs.v[k >> 2], sw[y][k >> 2]);
                __builtin_amdgcn_sched_barrier(0);
            }
            zs = zs_next;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v[4] = {acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
                TO* p = out + static_cast<int64_t>(qb * 16 + i) * a.L;
                if (whole) put_four(p, v, a.stream);         // uniform
                else if (q0 + qb * 16 + 4 * quarter + i < a.B) put_labels(p, v, l0 + 64 <= a.L, a.L - l);
            }
        }
        full = whole ? full + 1 : 0;
        slot = slot_next;
        if (++st == st_end) {
            piece(++n_piece, tile, st, st_end);
            full = 0;
            if (g + 1 < total) hold(static_cast<int64_t>(tile) * kMicroHeldLabels);
        }
    }
}

// ---- longer rows: tiles of 16 MQ WQ queries x 64 WL labels, two units of both to a stage, two stages in LDS, a wave with 16 MQ x 64.  A
// workgroup takes one tile after the other, the first stage of the next one under way while the last is multiplied and the scores are
// stored.  Rows of labels lie in the order of the products' blocks (block y, column j: label 4 j + y of 64), so that a lane stores
// neighbouring scores.  Consecutive workgroups of an XCD take the query tiles of one label tile.
// Bound: products and stores one after the other, since what a tile's second stage waits for is queued behind the stores before it.  1440 x
// 164990 to bf16: 281 us for rows of 1152 elements, 639 of 4096, which is 3.9 PFLOP/s for what lies between them (96 of the 128 bytes a cycle
// of LDS go to operands) and 140 us for the scores.
template <int WQ, int WL, int MQ>
struct MicroTile {
    static constexpr int kWaves = WQ * WL, BM = 16 * MQ * WQ, BN = 64 * WL, kRows = BM + BN, R = 2;
    static constexpr int kStage = kRows * (128 + 8), kParts = kRows / 64 * 2 /* of 64 scale words */, kScaleLoads = (kParts + kWaves - 1) / kWaves;
    static constexpr int kRowLoads = kRows / 8 / kWaves, kStores = 4 * MQ, kPerCu = 160 * 1024 / (R * kStage + 512);
    static_assert(kRowLoads * 8 * kWaves == kRows && BM % 64 == 0 && kPerCu >= 1 && kStores < 64, "whole loads, a count that the wait can hold");
};
template <typename TO, int WQ, int WL, int MQ>
__global__ __launch_bounds__(WQ * WL * kWave)
void scores_micro_tile_kernel(const MicroArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    typedef MicroTile<WQ, WL, MQ> T;
    __shared__ __align__(1024) unsigned char smem[T::R * T::kStage];
    const int lane = lane_id(), r = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wq = wave / WL, wl = wave % WL;
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
    const uint32_t n_tiles = tiles_m * tiles_n, per = (n_tiles + kXcds - 1) / kXcds;
    const uint32_t t_begin = blockIdx.x % kXcds * per, t_end = t_begin + per < n_tiles ? t_begin + per : n_tiles, t_step = gridDim.x / kXcds;
    uint32_t t = t_begin + blockIdx.x / kXcds;
    if (t >= t_end) return;                                  // uniform
    const uint32_t row_bytes = a.units * 64, row_scales = a.units * 4;
    const int steps = (a.units + 1) / 2;

    uint32_t at[T::kRowLoads], scale_at[T::kScaleLoads], ahead_t = t;
    const uint8_t *rows_q = nullptr, *rows_l = nullptr, *scale_q = nullptr, *scale_l = nullptr;
    int ahead = 0, ahead_slot = 0;
    auto issue = [&]() __attribute__((always_inline)) {
        if (ahead_t >= t_end) return;                        // uniform
        if (ahead == 0) {                                    // another tile
            const int64_t q0 = static_cast<int64_t>(ahead_t % tiles_m) * T::BM, l0 = static_cast<int64_t>(ahead_t / tiles_m) * T::BN;
            const uint32_t last_q = static_cast<uint32_t>(a.B - 1 - q0 < T::BM ? a.B - 1 - q0 : T::BM - 1);
            const uint32_t last_l = static_cast<uint32_t>(a.L - 1 - l0 < T::BN ? a.L - 1 - l0 : T::BN - 1);
            // row of the tile's queries or labels in place p of the stage, rows past the end: the last one again
            auto row_of = [&](uint32_t p) __attribute__((always_inline)) {
                if (p < T::BM) return p < last_q ? p : last_q;
                const uint32_t q = p - T::BM, l = (q & ~63u) + (q & 15) * 4 + ((q >> 4) & 3);
                return l < last_l ? l : last_l;
            };
#pragma unroll
            for (int i = 0; i < T::kRowLoads; ++i) at[i] = row_of((wave * T::kRowLoads + i) * 8 + (lane >> 3)) * row_bytes;
#pragma unroll
            for (int i = 0; i < T::kScaleLoads; ++i) scale_at[i] = row_of((wave + i * T::kWaves) % T::kParts / 2 * 64 + lane) * row_scales;
            rows_q = a.P + q0 * row_bytes;
            rows_l = a.Q + l0 * row_bytes;
            scale_q = a.pscale + q0 * row_scales;
            scale_l = a.scale + l0 * row_scales;
        }
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + ahead_slot * T::kStage), mask = ahead * 2 + 1 < a.units ? 127u : 63u;       // (a single unit: it again)
#pragma unroll
        for (int i = 0; i < T::kRowLoads; ++i) {
            const int n = wave * T::kRowLoads + i;           // (of one operand: a load's 8 rows)
            const uint32_t p = n * 8 + (lane >> 3), chunk = (lane ^ (p >> 1)) & 7;
            lds_dma16_sbase<0>(mx_uniform((n * 8 < T::BM ? rows_q : rows_l) + ahead * 128), at[i] + ((chunk * 16) & mask), to + n * 1024);
        }
#pragma unroll
        for (int i = 0; i < T::kScaleLoads; ++i) {
            const int n = (wave + i * T::kWaves) % T::kParts;          // (where they do not divide evenly, some twice)
            const uint32_t second = (n & 1) != 0 && mask == 127u ? 4 : 0;
            lds_dma4_sbase(mx_uniform((n / 2 * 64 < T::BM ? scale_q : scale_l) + ahead * 8), scale_at[i] + second,
                           __builtin_amdgcn_readfirstlane(to + T::kRows * 128 + n * 256));
        }
        if (++ahead == steps) {
            ahead = 0;
            ahead_t += t_step;
        }
        ahead_slot ^= 1;
    };
    issue();
    mx_f32x4 acc[MQ][4];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < MQ; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = mx_f32x4{0, 0, 0, 0};
    };
    clear();
    const int frag = r * 128 + ((quarter ^ mx_swizzle(r)) * 16);
    int slot = 0, step = 0;
    bool stored = false;                                     // a whole tile's scores, behind the loads that are waited for
    while (t < t_end) {
        if (stored) few_wait<T::kStores>();
        else few_wait<0>();
        stored = false;
        lds_barrier();                                       // the stage is there for everyone, the one before it has been read by everyone
        issue();
        const unsigned char* stage = smem + slot * T::kStage;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (step * 2 + h >= a.units) break;              // uniform
            mx_i32x4 w[4];
            int ws[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                w[y] = *reinterpret_cast<const mx_i32x4*>(stage + (T::BM + wl * 64 + y * 16) * 128 + (frag ^ (h * 64)));
                ws[y] = stage[T::kRows * 128 + ((T::BM / 64 + wl) * 2 + h) * 256 + (y * 16 + r) * 4 + quarter];
            }
#pragma unroll
            for (int x = 0; x < MQ; ++x) {
                const int row = (wq * MQ + x) * 16;
                const mx_i32x4 z = *reinterpret_cast<const mx_i32x4*>(stage + row * 128 + (frag ^ (h * 64)));
                const int zs = stage[T::kRows * 128 + (row / 64 * 2 + h) * 256 + (row % 64 + r) * 4 + quarter];
#pragma unroll
                for (int y = 0; y < 4; ++y) acc[x][y] = mx_product<0>(z, w[y], acc[x][y], zs, ws[y]);
            }
        }
        slot ^= 1;
        if (++step == steps) {
            step = 0;
            const int64_t q0 = static_cast<int64_t>(t % tiles_m) * T::BM + wq * MQ * 16, lw = static_cast<int64_t>(t / tiles_m) * T::BN + wl * 64;
            const int64_t l = lw + r * 4, have = a.L - l;
            const bool whole = lw + 64 <= a.L && q0 + MQ * 16 <= a.B;          // uniform
            TO* out = static_cast<TO*>(a.out) + (q0 + quarter * 4) * a.L + l;
#pragma unroll
            for (int x = 0; x < MQ; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v[4] = {acc[x][0][i], acc[x][1][i], acc[x][2][i], acc[x][3][i]};
                    TO* p = out + static_cast<int64_t>(x * 16 + i) * a.L;
                    if (whole) put_four(p, v, a.stream);     // uniform
                    else if (q0 + x * 16 + quarter * 4 + i < a.B) put_labels(p, v, lw + 64 <= a.L, have);
                }
            stored = whole;
            clear();
            t += t_step;
        }
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// (a row has 4 bytes of scales to a unit, read and written as a word: `scale` of a range of rows is aligned to as much, whichever its first row)
static bool micro_d(int d, xc_dtype t) { return d >= 1 && d <= XC_MAX_D_QUANTIZED && (static_cast<int64_t>(d) * (t == XC_F32 ? 4 : 2)) % 16 == 0; }

// The queries in the workspace: rows padded to whole pairs of units, their number to whole tiles of 64.
struct MicroSpace { int64_t rows; int units, pitch, upad; size_t bytes; };
static MicroSpace micro_space(int64_t B, int d) {
    MicroSpace s;
    s.rows = (B + 63) / 64 * 64;
    s.units = static_cast<int>(mx_pitch(d) / kMxRow);
    s.pitch = (s.units + 1) / 2 * 128;
    s.upad = (s.units + 3) / 4 * 4;
    s.bytes = static_cast<size_t>(s.rows) * (s.pitch + 4 * s.upad);
    return s;
}

constexpr int64_t kMxCachedBytes = 256ll << 20;

template <typename TO, typename TZ, int KU, int W, int R>
static void launch_few(const MicroArgs& a, hipStream_t st) {
    constexpr int kLds = W * R * kFewSlot + kMicroFewQueries * (KU * 64 + (KU + 3) / 4 * 16), kPerCu = 160 * 1024 / (kLds + 1024);
    static_assert(kPerCu >= 1, "");
    const int64_t groups = (a.L + 63) / 64, per = ((groups + kXcds - 1) / kXcds + W - 1) / W, most = kCusPerXcd * kPerCu;
    scores_micro_few_kernel<TO, TZ, KU, W, R><<<static_cast<unsigned>(kXcds * (per < most ? per : most)), W * kWave, 0, st>>>(a);
}
template <typename TO, int NK>
static void launch_micro_held(const MicroArgs& a, hipStream_t st) {
    scores_micro_held_kernel<TO, NK><<<kMineGrid, 512, 0, st>>>(a, static_cast<int>((a.L + kMicroHeldLabels - 1) / kMicroHeldLabels),
                                                                static_cast<int>((a.B + MicroHeld<NK>::QS - 1) / MicroHeld<NK>::QS));
}

template <typename TO, int WQ, int WL, int MQ>
static void launch_micro_tile(const MicroArgs& a, hipStream_t st) {
    typedef MicroTile<WQ, WL, MQ> T;
    // (launches of queries that leave the tiles countable)
    const int64_t tiles_n = (a.L + T::BN - 1) / T::BN, rows = ((1 << 24) / tiles_n > 1 ? (1 << 24) / tiles_n : 1) * T::BM;
    for (int64_t q0 = 0; q0 < a.B; q0 += rows) {
        MicroArgs p = a;
        p.B = a.B - q0 < rows ? a.B - q0 : rows;
        p.P += q0 * a.units * 64;
        p.pscale += q0 * a.units * 4;
        p.out = static_cast<TO*>(a.out) + q0 * a.L;
        const uint32_t tiles_m = static_cast<uint32_t>((p.B + T::BM - 1) / T::BM), per = (tiles_m * static_cast<uint32_t>(tiles_n) + kXcds - 1) / kXcds;
        const uint32_t most = kCusPerXcd * T::kPerCu;
        scores_micro_tile_kernel<TO, WQ, WL, MQ><<<kXcds * (per < most ? per : most), T::kWaves * kWave, 0, st>>>(p, tiles_m, static_cast<uint32_t>(tiles_n));
    }
}

typedef MicroTile<2, 2, 4> SmallTile;
typedef MicroTile<2, 4, 8> LargeTile;
static_assert(kMicroCus == kMineGrid && kMicroXcds == kXcds && SmallTile::BM == kMicroSmallSide && SmallTile::BN == kMicroSmallSide &&
              SmallTile::kPerCu == kMicroSmallPerCu && LargeTile::BM == kMicroLargeSide && LargeTile::BN == kMicroLargeSide &&
              LargeTile::kPerCu == kMicroLargePerCu, "what the choice counts with");

template <typename TO>
static int run_micro(MicroArgs a, const void* Z, xc_dtype t, const MicroSpace& space, hipStream_t st) {
    a.Z = static_cast<const unsigned char*>(Z);
    const MicroKernel kernel = choose_micro(a.B, a.L, a.units);
    if (kernel == kMicroOnline) {                            // one launch
        auto go = [&]() {
            if (a.units <= kMicroShortUnits) {
                if (t == XC_F32) launch_few<TO, float, kMicroShortUnits, 4, 2>(a, st);
                else launch_few<TO, bf16_t, kMicroShortUnits, 4, 2>(a, st);
            } else {
                if (t == XC_F32) launch_few<TO, float, kMicroFewUnits, 4, 3>(a, st);
                else launch_few<TO, bf16_t, kMicroFewUnits, 4, 3>(a, st);
            }
        };
        XC_LAUNCH(K_SCORES_MICRO, st, go());
        XC_HIP_CHECK(hipGetLastError());
        return XC_OK;
    }
    uint8_t *P = const_cast<uint8_t*>(a.P), *pscale = const_cast<uint8_t*>(a.pscale);
    const bool padded = kernel == kMicroHeld || kernel == kMicroFew;
    const int rc = padded ? launch_microscale(Z, a.B, a.d, t, nullptr, 0, nullptr, MicroQueries{P, pscale, space.units, space.pitch, space.upad}, space.rows, space.pitch / 64, st)
                          : launch_microscale(Z, a.B, a.d, t, nullptr, 0, nullptr, MicroRows{P, pscale, space.units}, a.B, space.units, st);
    if (rc != XC_OK) return rc;
    auto go = [&]() {
        if (kernel == kMicroHeld) {
            switch (space.pitch / 128) {
                case 1: launch_micro_held<TO, 2>(a, st); break;
                case 2: launch_micro_held<TO, 4>(a, st); break;
                case 3: launch_micro_held<TO, 6>(a, st); break;
                default: launch_micro_held<TO, 8>(a, st); break;
            }
        } else if (kernel == kMicroFew) {
            launch_few<TO, void, kMicroFewUnits, 4, 3>(a, st);         // (shorter rows of as many queries went the way above)
        } else if (kernel == kMicroSmall) {
            launch_micro_tile<TO, 2, 2, 4>(a, st);
        } else {
            launch_micro_tile<TO, 2, 4, 8>(a, st);
        }
    };
    XC_LAUNCH(K_SCORES_MICRO, st, go());
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}

}  // namespace xc

extern "C" int xc_microscale_rows(const void* X, int64_t N, int d, xc_dtype t, const int32_t* ids, int64_t m, const int32_t* count, uint8_t* Q,
                                  uint8_t* scale, void* stream) {
    using namespace xc;
    if (t != XC_F32 && t != XC_BF16) return XC_EDTYPE;
    if (N < 1 || N > 0x7fffffffLL || !micro_d(d, t) || m < 0) return XC_ESHAPE;
    if (!X || !Q || !scale || (count && !ids)) return XC_EINVAL;
    if (!aligned16(X) || !aligned16(ids) || !aligned16(count) || !aligned16(Q) || !aligned4(scale)) return XC_EINVAL;
    const unsigned __int128 n = N;
    if (overlap({Span(Q, n * (mx_pitch(d) / 2)), Span(scale, n * (mx_pitch(d) / 32))},
                {Span(X, n * d * (t == XC_F32 ? 4 : 2)), Span(ids, static_cast<unsigned __int128>(m) * 4), Span(count, 4)}))
        return XC_EINVAL;
    if (ids && m == 0) return XC_OK;
    const int units = static_cast<int>(mx_pitch(d) / kMxRow);
    return launch_microscale(X, N, d, t, ids, m, count, MicroRows{Q, scale, units}, N, units, static_cast<hipStream_t>(stream));
}

extern "C" int xc_scores_microscaled_workspace(int64_t B, int d, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (B < 1 || B > 0x7fffffffLL || d < 1 || d > XC_MAX_D_QUANTIZED) return XC_ESHAPE;
    *bytes = micro_space(B, d).bytes;
    return XC_OK;
}

extern "C" int xc_scores_microscaled(const void* Z, int64_t B, int d, xc_dtype t, const uint8_t* Q, const uint8_t* scale, int64_t L, xc_dtype out_t,
                                     void* out, void* ws, size_t ws_bytes, void* stream) {
    using namespace xc;
    if ((t != XC_F32 && t != XC_BF16) || (out_t != XC_F32 && out_t != XC_BF16)) return XC_EDTYPE;
    if (B < 1 || B > 0x7fffffffLL || L < 1 || L > 0x7fffffffLL || !micro_d(d, t) || static_cast<unsigned __int128>(B) * L > (1ull << 40)) return XC_ESHAPE;
    if (!Z || !Q || !scale || !out || !ws) return XC_EINVAL;
    if (!aligned16(Z) || !aligned16(Q) || !aligned4(scale) || !aligned16(out) || !aligned16(ws)) return XC_EINVAL;
    const MicroSpace space = micro_space(B, d);
    if (ws_bytes < space.bytes) return XC_EWORKSPACE;
    const unsigned __int128 b = B, l = L;
    if (overlap({Span(out, b * l * (out_t == XC_F32 ? 4 : 2)), Span(ws, space.bytes)},
                {Span(Z, b * d * (t == XC_F32 ? 4 : 2)), Span(Q, l * (mx_pitch(d) / 2)), Span(scale, l * (mx_pitch(d) / 32))}))
        return XC_EINVAL;
    uint8_t* P = static_cast<uint8_t*>(ws);
    const MicroArgs a{nullptr, P, P + space.rows * space.pitch, Q, scale, out, B, L, d, space.units, space.pitch, space.upad, B * L * (out_t == XC_F32 ? 4 : 2) > kMxCachedBytes};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return out_t == XC_F32 ? run_micro<float>(a, Z, t, space, st) : run_micro<bf16_t>(a, Z, t, space, st);
}
