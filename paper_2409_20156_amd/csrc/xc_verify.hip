// The check of drafted labels against the classifier's probabilities, and the draw of the label behind the last one that
// stands.  Only the rows that decide are read: two values per draft, then one row of the target (and of the draft where one fell).
// Sums are held in 64 bits: with V = 10^5 equal weights a running sum in fp32 would be off by whole labels.  The order of the sums
// depends on V alone (a wave's lanes by 8 neighbouring elements, pieces of a chunk one after the other, then the lanes, then the
// chunks), so a sequence's label depends neither on the others in the batch nor on the launch.
// Bound: few sequences, dependent memory accesses (draft -> its two probabilities -> the row -> the chunk again) and launches: 1 x 4 x
// 4096 fp32 5.0 us on the device, 8 x 5 x 131072 7.4 (two launches); a batch, the rows from memory: 256 x 4 x 131072 bf16, drafts that
// the target mostly takes, 23 us (110 MB, 4.8 TB/s), drafts that mostly fall 24 (127 MB read, 5.2 TB/s).  First form, 8 elements of a
// chunk at a time and all of it by one workgroup of 4 waves: 27, 140 and 181 us.
#include <type_traits>

#include "xc_common.h"

namespace xc {

constexpr int kPiece = 512;              // elements of a wave's step: 8 neighbouring ones per lane
constexpr int kPieces = 4;               // of a chunk, whose loads are under way together
constexpr int kChunk = kPieces * kPiece; // elements of a partial sum, formed by one wave whatever the launch
constexpr int kVerifyThreads = 256, kDrawWaves = kVerifyThreads / kWave;
constexpr int kOneChunks = 1024;         // of a sequence that one workgroup does alone
constexpr int64_t kManySequences = 192;  // that keep most compute units busy
constexpr int64_t kSumGrid = 2048;       // workgroups that fill the device
constexpr int64_t kSequences = 65535;    // of a launch

struct VerifyArgs {
    const int32_t* drafts;
    const void* target;
    const void* draft;                   // null: looked-up drafts
    const float* u;
    int32_t* tokens;
    int32_t* accepted;
    int4* verdicts;                      // [B]
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

// Elements e .. e + 7 of a row (zeros behind its end), whose address may be any.
template <typename T> struct Octet;
template <> struct Octet<float> {
    uint4 v[2];
    __device__ __forceinline__ void load(const float* p, int64_t e, int64_t V) {
        if (e + 8 <= V) {
            __builtin_memcpy(v, p + e, 32);
        } else {
            v[0] = v[1] = make_uint4(0, 0, 0, 0);
            if (e < V) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = e + i < V ? p[e + i] : 0.0f;
                __builtin_memcpy(v, f, 32);
            }
        }
    }
    __device__ __forceinline__ void values(float (&f)[8]) const { __builtin_memcpy(f, v, 32); }
};
template <> struct Octet<bf16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const bf16_t* p, int64_t e, int64_t V) {
        if (e + 8 <= V) {
            __builtin_memcpy(&v, p + e, 16);
        } else {
            v = make_uint4(0, 0, 0, 0);
            if (e < V) {
                uint32_t h[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] = e + i < V ? p[e + i].bits : 0u;
                v = make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
            }
        }
    }
    __device__ __forceinline__ void values(float (&f)[8]) const { unpack8(v, f); }
};

// ---- sums over a wave's lanes, in lane order (the neighbours' values come by DPP, not through LDS)
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lanes(double s) {     // 0 where there is no such lane
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(s));
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
__device__ __forceinline__ double wave_incl_scan(double s) {
    s += from_lanes<0x111, 0xf>(s);          // row_shr 1, 2, 4, 8
    s += from_lanes<0x112, 0xf>(s);
    s += from_lanes<0x114, 0xf>(s);
    s += from_lanes<0x118, 0xf>(s);
    s += from_lanes<0x142, 0xa>(s);          // row_bcast 15 into rows 1 and 3
    s += from_lanes<0x143, 0xc>(s);          // row_bcast 31 into rows 2 and 3
    return s;
}
__device__ __forceinline__ double of_lane(double s, int lane /* uniform */) {
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(s));
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(u), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(u >> 32), lane);
    return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
__device__ __forceinline__ int first_lane(uint64_t m) { return __ffsll(static_cast<long long>(m)) - 1; }
__device__ __forceinline__ int last_lane(uint64_t m) { return 63 - __clzll(static_cast<long long>(m)); }

// ---- a row's weights
template <typename T>
struct Row {
    const T *p, *q;
    Weights kind;
    int32_t without;
    int64_t V;
    // the lane's elements of piece k of chunk c: 8 from here on
    static __device__ __forceinline__ int64_t first(int c, int k) { return static_cast<int64_t>(c) * kChunk + k * kPiece + lane_id() * 8; }
    template <bool DIFF> __device__ __forceinline__ void load(int c, int k, Octet<T>& x, Octet<T>& y) const {
        x.load(p, first(c, k), V);
        if constexpr (DIFF) y.load(q, first(c, k), V);
    }
    template <bool DIFF> __device__ __forceinline__ void values(int c, int k, const Octet<T>& x, const Octet<T>& y, float (&f)[8], float (&g)[8]) const {
        x.values(f);
        if constexpr (DIFF) {
            y.values(g);
        } else {
            const int64_t at = kind == kWithout ? without - first(c, k) : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] = 0.0f;
                if (at == i) f[i] = 0.0f;
            }
        }
    }
    static __device__ __forceinline__ double weight(float x, float y) {
        const double w = static_cast<double>(x) - static_cast<double>(y);
        return w > 0.0 && w < static_cast<double>(INFINITY) ? w : 0.0;
    }
};

// Sum of a lane's 8 elements: pairs, then pairs of these.
__device__ __forceinline__ double sum8(const double (&w)[8]) {
    return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
}

// Sum of chunk c, the same in all lanes.
template <bool DIFF, typename T>
__device__ __forceinline__ double chunk_sum(const Row<T>& r, int c) {
    Octet<T> x[kPieces], y[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) r.template load<DIFF>(c, k, x[k], y[k]);
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        float f[8], g[8];
        double w[8];
        r.template values<DIFF>(c, k, x[k], y[k], f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = fmax(static_cast<double>(f[i]) - static_cast<double>(g[i]), 0.0);         // (no number: 0)
        s += sum8(w);
    }
    if (__builtin_expect(!(s < static_cast<double>(INFINITY)), 0)) {                   // an infinity among them counts as 0
        s = 0.0;
#pragma unroll 1
        for (int k = 0; k < kPieces; ++k) {
            float f[8], g[8];
            double w[8];
            r.template load<DIFF>(c, k, x[0], y[0]);
            r.template values<DIFF>(c, k, x[0], y[0], f, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = Row<T>::weight(f[i], g[i]);
            s += sum8(w);
        }
    }
    return of_lane(wave_incl_scan(s), kWave - 1);
}

// Sums of the chunks first, first + step, ..  The kind of weights is decided once: decided at every element it took 154 registers in place
// of 108 (1000 x 20000 fp32 41 us, now 32).  More waves hide the memory's latency better than a chunk loaded ahead (254 registers: 46 us).
template <typename T>
__device__ __forceinline__ void chunk_sums(const Row<T>& r, double* sums, int first, int step, int n_chunks) {
    auto go = [&](auto diff) __attribute__((always_inline)) {
        for (int c = first; c < n_chunks; c += step) {
            const double s = chunk_sum<decltype(diff)::value>(r, c);
            if (lane_id() == 0) sums[c] = s;
        }
    };
    if (r.kind == kDifference) go(std::true_type{});         // uniform
    else go(std::false_type{});
}

// ---- the label drawn, by a workgroup of W waves from the chunks' sums: -1 if all weights are zero.
template <int W> struct DrawShared { double group[W]; uint64_t pass[W], some[W]; double before[W]; int32_t label; };

template <typename T, int W>
__device__ __forceinline__ int32_t draw_label(const Row<T>& r, const double* sums, int n_chunks, float u, DrawShared<W>& sh) {
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    constexpr int kRound = W * kWave;
    // the chunk: 64 at a time to a wave
    double total = 0.0, incl = 0.0, s = 0.0;
    for (int c0 = 0; c0 < n_chunks; c0 += kRound) {
        const int c = c0 + static_cast<int>(threadIdx.x);
        s = c < n_chunks ? sums[c] : 0.0;
        incl = wave_incl_scan(s);
        if (lane == kWave - 1) sh.group[wave] = incl;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) total += sh.group[w];
        __syncthreads();
    }
    if (!(total > 0.0)) return -1;                           // uniform
    const double t = static_cast<double>(u) * total;
    double before = 0.0, chunk_before = 0.0;
    int chunk = 0;
    for (int c0 = 0; c0 < n_chunks; c0 += kRound) {
        if (n_chunks > kRound) {                             // (else these are the ones at hand)
            const int c = c0 + static_cast<int>(threadIdx.x);
            s = c < n_chunks ? sums[c] : 0.0;
            incl = wave_incl_scan(s);
            if (lane == kWave - 1) sh.group[wave] = incl;
            __syncthreads();
        }
        double mine = before;
        for (int w = 0; w < wave; ++w) mine += sh.group[w];
        const uint64_t some = __ballot(s > 0.0), pass = __ballot(s > 0.0 && mine + incl > t);
        const uint64_t take = pass != 0ull ? pass & (~pass + 1ull) : some;
        if (take != 0ull && lane == last_lane(take)) sh.before[wave] = mine + (incl - s);
        if (lane == 0) { sh.pass[wave] = pass; sh.some[wave] = some; }
        __syncthreads();
        int hit = -1, last = -1;                             // (no chunk passes: the last with a weight)
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (hit < 0 && sh.pass[w] != 0ull) hit = w;
            if (sh.some[w] != 0ull) last = w;
        }
        const int w = hit >= 0 ? hit : last;
        if (w >= 0) {
            chunk = c0 + w * kWave + (hit >= 0 ? first_lane(sh.pass[w]) : last_lane(sh.some[w]));
            chunk_before = sh.before[w];
        }
#pragma unroll
        for (int v = 0; v < W; ++v) before += sh.group[v];
        __syncthreads();
        if (hit >= 0) break;                                 // uniform
    }
    // the label: a piece of the chunk to each of the first waves.  The first lane whose own sum passes t decides; its elements'
    // running sum may stay below by a rounding: its last one then.  So may all lanes' sums: the last element with a weight.
    static_assert(kPieces <= W, "");
    double wt[8];
    s = 0.0;
    if (wave < kPieces) {
        Octet<T> x, y;
        float f[8], g[8];
        if (r.kind == kDifference) {                         // uniform
            r.template load<true>(chunk, wave, x, y);
            r.template values<true>(chunk, wave, x, y, f, g);
        } else {
            r.template load<false>(chunk, wave, x, y);
            r.template values<false>(chunk, wave, x, y, f, g);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) wt[i] = Row<T>::weight(f[i], g[i]);
        s = sum8(wt);
    }
    incl = wave_incl_scan(s);
    if (lane == kWave - 1) sh.group[wave] = incl;
    __syncthreads();
    before = chunk_before;
    for (int w = 0; w < wave && w < kPieces; ++w) before += sh.group[w];
    const uint64_t some = __ballot(s > 0.0), pass = __ballot(s > 0.0 && before + incl > t);
    if (lane == 0) { sh.pass[wave] = pass; sh.some[wave] = some; }
    __syncthreads();
    int hit = -1, last = -1;
#pragma unroll
    for (int w = 0; w < kPieces; ++w) {
        if (hit < 0 && sh.pass[w] != 0ull) hit = w;
        if (sh.some[w] != 0ull) last = w;
    }
    if (wave == (hit >= 0 ? hit : last) && lane == (hit >= 0 ? first_lane(pass) : last_lane(some))) {
        double run = before + (incl - s);
        int32_t here = -1, mine = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            run += wt[i];
            if (wt[i] > 0.0) {
                mine = static_cast<int32_t>(Row<T>::first(chunk, wave) + i);
                if (here < 0 && run > t) here = mine;
            }
        }
        sh.label = hit >= 0 && here >= 0 ? here : mine;
    }
    __syncthreads();
    return sh.label;
}

template <typename T>
__device__ __forceinline__ Row<T> deciding_row(const VerifyArgs& v, int64_t b, const Verdict& j) {
    Row<T> r;
    r.p = static_cast<const T*>(v.target) + (b * (v.n + 1) + j.a) * v.V;
    r.q = v.draft != nullptr && j.fell ? static_cast<const T*>(v.draft) + (b * v.n + j.a) * v.V : nullptr;
    r.kind = !j.fell ? kTarget : v.draft != nullptr ? kDifference : kWithout;
    r.without = j.x;
    r.V = v.V;
    return r;
}
__device__ __forceinline__ void write_tokens(const VerifyArgs& v, int64_t b, int a, int32_t drawn) {
    for (int i = threadIdx.x; i <= v.n; i += static_cast<int>(blockDim.x))
        v.tokens[b * (v.n + 1) + i] = i < a ? v.drafts[b * v.n + i] : i == a ? drawn : -1;
    if (threadIdx.x == 0) v.accepted[b] = a;
}

// One workgroup does a sequence with few chunks.
template <typename T, int W>
__global__ __launch_bounds__(W * kWave)
void verify_one_kernel(const VerifyArgs v) {
    const int64_t b = blockIdx.x;
    const int wave = threadIdx.x >> 6;
    __shared__ double sums[kOneChunks];
    __shared__ DrawShared<W> sh;
    const float u = v.u[b * (v.n + 1) + v.n];
    const Verdict j = judge<T>(v, b);
    Row<T> r = deciding_row<T>(v, b, j);
    int32_t drawn;
    for (;;) {
        chunk_sums(r, sums, wave, W, v.n_chunks);
        __syncthreads();
        drawn = draw_label<T, W>(r, sums, v.n_chunks, u, sh);
        if (drawn >= 0 || r.kind == kTarget) break;          // uniform
        r.kind = kTarget;                // nothing is left of the target above the draft: the target itself
        __syncthreads();
    }
    write_tokens(v, b, j.a, drawn);
}

// Longer rows: the partial sums by many workgroups, a chunk to a wave; then a workgroup per sequence.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads)
void verify_sums_kernel(const VerifyArgs v) {
    const int64_t b = blockIdx.y;
    const int c0 = blockIdx.x * kDrawWaves + (threadIdx.x >> 6), step = gridDim.x * kDrawWaves;
    if (c0 >= v.n_chunks) return;
    const Verdict j = judge<T>(v, b);
    const Row<T> r = deciding_row<T>(v, b, j);
    chunk_sums(r, v.sums + b * v.n_chunks, c0, step, v.n_chunks);
    if (c0 == 0 && lane_id() == 0) v.verdicts[b] = make_int4(j.a, j.fell ? 1 : 0, j.x, 0);
}
template <typename T>
__global__ __launch_bounds__(kVerifyThreads)
void verify_draw_kernel(const VerifyArgs v) {
    const int64_t b = blockIdx.x;
    __shared__ DrawShared<kDrawWaves> sh;
    double* sums = v.sums + b * v.n_chunks;
    const int4 w = v.verdicts[b];
    const float u = v.u[b * (v.n + 1) + v.n];
    const Verdict j{w.x, w.y != 0, w.z};
    Row<T> r = deciding_row<T>(v, b, j);
    int32_t drawn = draw_label<T, kDrawWaves>(r, sums, v.n_chunks, u, sh);
    if (drawn < 0 && r.kind != kTarget) {                    // as above; so rare that one workgroup adds the row up
        r.kind = kTarget;
        __syncthreads();
        chunk_sums(r, sums, threadIdx.x >> 6, kDrawWaves, v.n_chunks);
        __syncthreads();
        drawn = draw_label<T, kDrawWaves>(r, sums, v.n_chunks, u, sh);
    }
    write_tokens(v, b, j.a, drawn);
}

template <typename T>
static void launch_verify(const VerifyArgs& v, int64_t B, hipStream_t st) {
    // A workgroup per sequence saves a launch; many workgroups per sequence bring a long row in faster, where the sequences alone
    // leave compute units idle.  Device time, us, by 4 waves, by 8, by many: 1 x 8192 fp32 5.3, 5.9, 6.5; 1 x 32768 8.7, 7.8, 7.1 (a call of
    // which the caller takes 8 with one launch and 10.5 with two); 1 x 65536 12.9, 10.9, 7.1; 64 x 131072 27.9, 19.6, 17.0; 256 x
    // 131072 41.3, 39.7, 41.3, in bf16 29.9, 23.2, 26.2.
    const int alone = v.n_chunks <= 8 ? 4 : v.n_chunks <= 16 || (B >= kManySequences && v.n_chunks <= kOneChunks) ? 8 : 0;
    for (int64_t b0 = 0; b0 < B; b0 += kSequences) {
        VerifyArgs p = v;
        const int64_t nb = B - b0 < kSequences ? B - b0 : kSequences;
        p.drafts = v.drafts + b0 * v.n;
        p.target = static_cast<const T*>(v.target) + b0 * (v.n + 1) * v.V;
        if (v.draft != nullptr) p.draft = static_cast<const T*>(v.draft) + b0 * v.n * v.V;
        p.u += b0 * (v.n + 1);
        p.tokens += b0 * (v.n + 1);
        p.accepted += b0;
        p.verdicts += b0;
        p.sums += b0 * v.n_chunks;
        if (alone == 4) {
            XC_LAUNCH(K_VERIFY, st, (verify_one_kernel<T, 4><<<static_cast<unsigned>(nb), 4 * kWave, 0, st>>>(p)));
            continue;
        }
        if (alone == 8) {
            XC_LAUNCH(K_VERIFY, st, (verify_one_kernel<T, 8><<<static_cast<unsigned>(nb), 8 * kWave, 0, st>>>(p)));
            continue;
        }
        // as many chunks to a wave as leave the device full
        const int64_t wide = (v.n_chunks + kDrawWaves - 1) / kDrawWaves, most = kSumGrid / nb > 0 ? kSumGrid / nb : 1;
        const int64_t rounds = (wide + most - 1) / most, gx = (wide + rounds - 1) / rounds;
        XC_LAUNCH(K_VERIFY_SUMS, st, (verify_sums_kernel<T><<<dim3(static_cast<unsigned>(gx), static_cast<unsigned>(nb)), kVerifyThreads, 0, st>>>(p)));
        XC_LAUNCH(K_VERIFY, st, (verify_draw_kernel<T><<<static_cast<unsigned>(nb), kVerifyThreads, 0, st>>>(p)));
    }
}

static int verify_chunks(int64_t V) { return static_cast<int>((V + kChunk - 1) / kChunk); }

static size_t verify_bytes(int64_t B, int64_t V) {
    return static_cast<size_t>(B) * (sizeof(int4) + static_cast<size_t>(verify_chunks(V)) * sizeof(double));
}

}  // namespace xc

extern "C" int xc_verify_workspace(int64_t B, int64_t V, size_t* bytes) {
    using namespace xc;
    if (!bytes) return XC_EINVAL;
    if (B < 1 || B > 0x7fffffffLL || V < 1 || V > 0x7fffffffLL) return XC_ESHAPE;
    *bytes = verify_bytes(B, V);
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
    if (ws_bytes < verify_bytes(B, V)) return XC_EWORKSPACE;
    // (a workgroup writes a sequence's labels while others have yet to read theirs)
    const unsigned __int128 rows = static_cast<unsigned __int128>(B) * V * (t == XC_F32 ? 4 : 2);
    const size_t ids = static_cast<size_t>(B) * 4;
    if (overlap({Span(tokens, ids * (n + 1)), Span(accepted, ids), Span(ws, verify_bytes(B, V))},
                {Span(drafts, ids * n), Span(u, ids * (n + 1)), Span(target, rows * (n + 1)), Span(draft_probs, rows * n)}))
        return XC_EINVAL;
    int4* verdicts = static_cast<int4*>(ws);
    const VerifyArgs v{drafts, target, draft_probs, u, tokens, accepted, verdicts, reinterpret_cast<double*>(verdicts + B), V, n, verify_chunks(V)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (t == XC_F32) launch_verify<float>(v, B, st);
    else launch_verify<bf16_t>(v, B, st);
    XC_HIP_CHECK(hipGetLastError());
    return XC_OK;
}
