// Conversions between bf16 / fp32 rows and the block-scaled formats, and the root-mean-square norm, whose output comes in
// 8 bits as well.  All of it is bound by memory: every value is read once and written once, 16 bytes a lane.
//
// A block of 32 values is four lanes of eight: its largest magnitude is two exchanges inside a quad.  With m 2^k that
// magnitude (1 <= m < 2) and c 2^p the format's largest (1.5 * 2^2, 1.75 * 2^8), the block's scale is 2^(k - p), or twice
// that where m > c: the exponent field after adding (2 - c) 2^23 - 1 to the bits.  Dividing by it is exact, so each value
// is rounded once, by the hardware's conversion (to nearest, ties to even; never out of the format's range).
#include "mx_kernels.h"

namespace lora {
namespace {

typedef short i16x2_t __attribute__((ext_vector_type(2)));

// Eight consecutive values of a row as fp32.
__device__ __forceinline__ void load8(const __bf16 *p, float (&v)[8]) {
    const chunk_t c = load_chunk(p);
    const unsigned w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const chunk_t a = load_chunk(p), b = load_chunk(p + 4);
    v[0] = __uint_as_float(a.x), v[1] = __uint_as_float(a.y), v[2] = __uint_as_float(a.z), v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x), v[5] = __uint_as_float(b.y), v[6] = __uint_as_float(b.z), v[7] = __uint_as_float(b.w);
}

// The largest magnitude of the lane's quad, as bits (an unsigned maximum: infinities and NaN are the largest).
__device__ __forceinline__ unsigned quad_max(const float (&v)[8]) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    m = max(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
    return m;
}
// Scale byte of a block, from the bits of its largest magnitude.
template <int FMT>
__device__ __forceinline__ int scale_code(unsigned amax) {
    constexpr unsigned up = FMT == kMxE2M1 ? 0x3fffffu : 0x1fffffu;
    constexpr int p = FMT == kMxE2M1 ? 2 : 8;
    if (amax >= 0x7f800000u) return 255;
    return max((int)((amax + up) >> 23) - p, 0);
}
// 1 / scale; a NaN for 255, which every element of the block then becomes.
__device__ __forceinline__ float inverse_scale(int code) {
    return __uint_as_float(code == 255 ? 0x7fc00000u : code == 254 ? 0x00400000u : (unsigned)(254 - code) << 23);
}
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// The codes of eight values: 8 bytes, or 4 with the even one of two in the low half.
__device__ __forceinline__ uint2 codes_e4m3(const float (&v)[8], float inv) {
    return make_uint2(pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), pack_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
}
__device__ __forceinline__ unsigned codes_e2m1(const float (&v)[8], float inv) {
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0] * inv, v[1] * inv, 1.f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2] * inv, v[3] * inv, 1.f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4] * inv, v[5] * inv, 1.f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6] * inv, v[7] * inv, 1.f, 3);
}

constexpr int kMxWaves = 4;  // per workgroup

// A grid of `wgs` workgroups: a dimension of a launch holds fewer than 2^32 threads.
constexpr int64_t kGridX = 1 << 21;
dim3 grid_of(int64_t wgs) { return wgs <= kGridX ? dim3((unsigned)wgs) : dim3((unsigned)kGridX, (unsigned)((wgs + kGridX - 1) / kGridX)); }
__device__ __forceinline__ unsigned workgroup() { return blockIdx.y * (unsigned)kGridX + blockIdx.x; }

template <typename E, int FMT>
__global__ __launch_bounds__(kMxWaves * 64) void mx_quantize_kernel(MxConvertArgs p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned unit = workgroup() * kMxWaves + wave, urow = unit / (unsigned)p.strips;
    const int64_t row = urow;
    if (row >= p.rows) return;
    const int k0 = (int)(unit - urow * p.strips) * kMxStrip + lane * 8;
    const E *src = static_cast<const E *>(p.src) + row * p.lds;
    unsigned char *codes = static_cast<unsigned char *>(p.dst) + row * p.ldd;
    unsigned char *scales = p.scales + row * p.ldsc;
    float v[kMxPieces][8];
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) load8(src + min(k0 + i * 512, p.K - 8), v[i]);
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) {
        const int k = k0 + i * 512;
        const int s = scale_code<FMT>(quad_max(v[i]));  // (a quad is all inside the row or all behind it)
        const float inv = inverse_scale(s);
        if (k >= p.K) continue;
        if constexpr (FMT == kMxE4M3)
            *reinterpret_cast<uint2 *>(codes + k) = codes_e4m3(v[i], inv);
        else
            *reinterpret_cast<unsigned *>(codes + (k >> 1)) = codes_e2m1(v[i], inv);
        if ((lane & 3) == 0) scales[k >> 5] = (unsigned char)s;
    }
}

// A bf16 row as the sum of two e4m3 rows: the first is the row's quantization, the second that of what it leaves, with a scale
// 2^-4 of the first's (a remainder is at most half a step of the first, 2^-4 of 256 .. 448 there).  bf16 has 8 significant bits and each
// part holds 4, so the sum is the value itself where the second part's smallest step, 2^-13 of the first scale, is not above the
// value's own -- down to 2^-6 of that scale -- and off by at most half of that step, 2^-14 of the scale, below.  The block's largest
// value is above 224 scales: exact down to 2^-13 of it, off by less than 2^-21 of it below (2^-13.8 and 2^-21.8 where it is just above).
__global__ __launch_bounds__(kMxWaves * 64) void mx_split_kernel(MxSplitArgs p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned unit = workgroup() * kMxWaves + wave, urow = unit / (unsigned)p.strips;
    if (urow >= (unsigned)p.rows) return;
    const int k0 = (int)(unit - urow * p.strips) * kMxStrip + lane * 8;
    const __bf16 *src = static_cast<const __bf16 *>(p.X) + (int64_t)urow * p.ldx;
    unsigned char *codes = p.codes + (int64_t)urow * 2 * p.part_bytes, *scales = p.scales + (int64_t)urow * 2 * p.part_scales;
    float v[kMxPieces][8];
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) load8(src + min(k0 + i * 512, p.K - 8), v[i]);
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) {
        const int k = k0 + i * 512;
        const int s = scale_code<kMxE4M3>(quad_max(v[i])), s2 = s == 255 ? 255 : max(s - 4, 0);
        const float inv = inverse_scale(s), up = s == 255 ? 1.f : __uint_as_float((unsigned)(127 + s - s2) << 23);
        uint2 hi = codes_e4m3(v[i], inv), lo;
        float r[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned c = h ? hi.y : hi.x;
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.f, true);
            const float back[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
            for (int e = 0; e < 4; ++e) r[h * 4 + e] = v[i][h * 4 + e] * inv - back[e];
        }
        lo = codes_e4m3(r, up);
        if (k >= p.part_bytes) continue;
        if (k >= p.K) hi = lo = make_uint2(0u, 0u);
        *reinterpret_cast<uint2 *>(codes + k) = hi;
        *reinterpret_cast<uint2 *>(codes + p.part_bytes + k) = lo;
        if ((lane & 3) == 0) {
            scales[k >> 5] = (unsigned char)s;
            scales[p.part_scales + (k >> 5)] = (unsigned char)s2;
        }
    }
}

__device__ __forceinline__ void store_values(__bf16 *dst, const float (&v)[8]) { store8(dst, v); }
__device__ __forceinline__ void store_values(float *dst, const float (&v)[8]) { store8(dst, v); }

template <typename E, int FMT>
__global__ __launch_bounds__(kMxWaves * 64) void mx_dequantize_kernel(MxConvertArgs p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned unit = workgroup() * kMxWaves + wave, urow = unit / (unsigned)p.strips;
    const int64_t row = urow;
    if (row >= p.rows) return;
    const int k0 = (int)(unit - urow * p.strips) * kMxStrip + lane * 8;
    const unsigned char *codes = static_cast<const unsigned char *>(p.src) + row * p.lds;
    const unsigned char *scales = p.scales + row * p.ldsc;
    E *dst = static_cast<E *>(p.dst) + row * p.ldd;
    uint2 c[kMxPieces];
    unsigned s[kMxPieces];
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) {
        const int k = min(k0 + i * 512, p.K - 8);
        if constexpr (FMT == kMxE4M3)
            c[i] = *reinterpret_cast<const uint2 *>(codes + k);
        else
            c[i].x = *reinterpret_cast<const unsigned *>(codes + (k >> 1));
        s[i] = scales[k >> 5];
    }
#pragma unroll
    for (int i = 0; i < kMxPieces; ++i) {
        const int k = k0 + i * 512;
        // (the conversion takes the exponent field of its scale: 0 stands for 2^-127, 255 makes a NaN)
        const float sc = __uint_as_float(s[i] << 23);
        float v[8];
        if constexpr (FMT == kMxE4M3) {
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i].x, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i].x, sc, true);
            const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i].y, sc, false), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i].y, sc, true);
            v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
        } else {
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, sc, 1);
            const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, sc, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, sc, 3);
            v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
        }
        if (k < p.K) store_values(dst + k, v);
    }
}

// ---- root-mean-square norm -----------------------------------------------------------------------------------------
// TPR threads share a row, PCS pieces of 8 values each: the row stays in registers between its sum of squares and the
// outputs, so everything is read once.  A workgroup holds NT / TPR rows.
// Roundings: squares are exact in 64 bits and summed there, and the scale of a row is kept as two fp32 numbers, so that fp32's y is off by
// little more than its last product's half a step.  The narrower outputs are rounded from more bits than that (to_odd): from fp32's y one
// element in 2^21 would fall to the wrong side of a border between two 8-bit values.  The 64-bit sums hide
// behind the loads; rounding once costs 46.4 -> 47.1 us at 7500 rows of 4096, 14.9 -> 16.2 at 1500 of 5120.

// `y` with what is missing from it folded into its last bit ("round to odd"): a later rounding to at most 22 bits then gives what rounding
// y + rest once would give, because a border between such values has an even last bit, which only an exact y keeps.
// |rest| is at most half a step of y: towards zero if it points there, then the last bit set.  Nothing is folded in where rest is not a
// normal number: y is exact, not finite, or below 2^-102.
__device__ __forceinline__ float to_odd(float y, float rest) {
    const int bits = __float_as_int(y), back = (bits ^ __float_as_int(rest)) >> 31;
    return __builtin_amdgcn_classf(rest, 0x108) ? __int_as_float((bits + back) | 1) : y;
}

// What all lanes of the wave hold, in scalar registers.
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
__device__ __forceinline__ double uniform(double v) {
    const long long b = __double_as_longlong(v);
    return __hiloint2double(__builtin_amdgcn_readfirstlane((int)(b >> 32)), __builtin_amdgcn_readfirstlane((int)b));
}

template <typename E, int TPR, int PCS>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rms_norm_kernel(RmsNormArgs p) {
    constexpr int NT = TPR > 256 ? TPR : 256, RPW = NT / TPR, WPR = TPR / 64;
    __shared__ double part[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = (int64_t)workgroup() * RPW + (RPW > 1 ? wave / WPR : 0);
    const bool mine = row < p.rows;
    const int64_t rr = mine ? row : p.rows - 1;
    const int at = (RPW > 1 ? tid % TPR : tid) * 8;
    const E *x = static_cast<const E *>(p.X) + rr * p.ldx, *g = static_cast<const E *>(p.gamma);
    float v[PCS][8];
#pragma unroll
    for (int i = 0; i < PCS; ++i) load8(x + min(at + i * TPR * 8, p.K - 8), v[i]);
    if (p.R != nullptr) {
        const E *r = static_cast<const E *>(p.R) + rr * p.ldr;
        constexpr int AHEAD = PCS < 4 ? PCS : 4;  // (eight pieces of both do not fit the registers of 1024 threads)
#pragma unroll
        for (int j = 0; j < PCS; j += AHEAD) {
            float w[AHEAD][8];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) load8(r + min(at + (j + i) * TPR * 8, p.K - 8), w[i]);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[j + i][e] += w[i][e];
            if constexpr (AHEAD < PCS)
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(v[j + i][e])::"memory");
        }
    }
    // (whether any of the wave's lanes has a piece i; 1500 rows of 5120, where six of eight waves have no second one, 17.3 -> 16.2 us)
    const int first = (RPW > 1 ? wave % WPR : wave) * 512;
    auto any = [&](int i) { return i == 0 || first + i * TPR * 8 < p.K; };
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < PCS; ++i) {
        if (!any(i)) continue;
        double s[2] = {0.0, 0.0};
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e & 1] = __builtin_fma((double)v[i][e], (double)v[i][e], s[e & 1]);
        ss += at + i * TPR * 8 < p.K ? s[0] + s[1] : 0.0;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) ss += __shfl_xor(ss, d);
    if constexpr (WPR > 1) {
        if (lane == 0) part[wave] = ss;
        __syncthreads();
        ss = 0.0;
#pragma unroll
        for (int w = 0; w < WPR; ++w) ss += part[(RPW > 1 ? wave / WPR * WPR : 0) + w];
    }
    if (!mine) return;
    double scale = uniform(1.0 / __builtin_sqrt(ss / (double)p.K + (double)p.eps));  // (the row's, so the wave's: scalar registers)
    // (whatever is stored is stored behind the row's last load: H and Y may be X or R)
    if (p.H != nullptr) {
        E *h = static_cast<E *>(p.H) + row * p.ldh;
#pragma unroll
        for (int i = 0; i < PCS; ++i)
            if (at + i * TPR * 8 < p.K) store8(h + at + i * TPR * 8, v[i]);
    }
    // (rows below 2^-120 or above 2^100, whose scale or the second part of it is no normal number of fp32: a power of two goes from the scale
    // into the values, exactly where y is above 2^-100)
    if (scale > 0x1p120 || scale < 0x1p-100) {
        const float shift = scale > 1.0 ? 0x1p64f : 0x1p-32f;
        scale *= scale > 1.0 ? 0x1p-64 : 0x1p32;
#pragma unroll
        for (int i = 0; i < PCS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= shift;
    }
    const float hi = uniform((float)scale), lo = uniform(__builtin_isfinite(hi) ? (float)(scale - (double)hi) : 0.f);
#pragma unroll
    for (int i = 0; i < PCS; ++i) {
        if (!any(i)) continue;
        float w[8];
        load8(g + min(at + i * TPR * 8, p.K - 8), w);
        float y32[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = v[i][e] * hi;
            // (an infinity or NaN has no rest)
            const float rest = __builtin_isfinite(t) ? __builtin_fmaf(v[i][e], lo, __builtin_fmaf(v[i][e], hi, -t)) * w[e] : 0.f;
            y32[e] = __builtin_fmaf(t, w[e], rest);
            v[i][e] = to_odd(y32[e], __builtin_fmaf(t, w[e], -y32[e]) + rest);
        }
        if (sizeof(E) == 4 && p.Y != nullptr && at + i * TPR * 8 < p.K)  // (fp32's own rounding)
            store8(static_cast<E *>(p.Y) + row * p.ldy + at + i * TPR * 8, y32);
        if constexpr (TPR == 1024) asm volatile("" ::: "memory");  // one piece of gamma at a time: 128 registers are all there are
#pragma unroll
        for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(v[i][e]));  // (here, or its parts stay in registers until the codes are made)
    }
    if (sizeof(E) != 4 && p.Y != nullptr) {
        E *y = static_cast<E *>(p.Y) + row * p.ldy;
#pragma unroll
        for (int i = 0; i < PCS; ++i)
            if (at + i * TPR * 8 < p.K) store8(y + at + i * TPR * 8, v[i]);
    }
    if (p.codes != nullptr) {
        unsigned char *codes = p.codes + row * p.ldc, *scales = p.scales + row * p.ldsc;
#pragma unroll
        for (int i = 0; i < PCS; ++i) {
            if (!any(i)) continue;
            const int k = at + i * TPR * 8;
            const int s = scale_code<kMxE4M3>(quad_max(v[i]));
            const uint2 c = codes_e4m3(v[i], inverse_scale(s));
            if (k >= p.K) continue;
            *reinterpret_cast<uint2 *>(codes + k) = c;
            if ((lane & 3) == 0) scales[k >> 5] = (unsigned char)s;
        }
    }
}

template <typename E, int TPR, int PCS>
hipError_t launch_norm_t(const RmsNormArgs &a, hipStream_t stream, const KernelTimer *timer) {
    constexpr int NT = TPR > 256 ? TPR : 256, RPW = NT / TPR;
    const int64_t grid = (a.rows + RPW - 1) / RPW;
    return launch_kernel(rms_norm_kernel<E, TPR, PCS>, grid_of(grid), dim3(NT), 0, stream, timer, a);
}

// Threads per row by its length alone, so that a row's result does not depend on how many there are.  Measured in us with 64 / 256 / 512 / 1024
// threads (bf16 with residual, sum, normed rows and 8-bit rows): 7500 rows of 512 9.7 / 17.6 / 32 / 58; 1000 of 1024 4.2 / 4.9 / 6.2 / 9.9;
// 1 of 4096 5.1 / 2.7 / 2.6 / 3.2; 7500 of 4096 51 / 46 / 45 / 72 (one set of outputs, which the cache holds in part; 56 with three,
// 5.0 TB/s); 1500 of 5120 14.2 with 256, 14.4, 16.6; 391 of 11008 in fp32 17.0 with 256, 15.6, 15.1; 100 of 16384 7.6 with 256, 7.0,
// 6.8 (all without to_odd).
template <typename E>
hipError_t launch_norm_e(const RmsNormArgs &a, hipStream_t stream, const KernelTimer *timer) {
    const int pieces = a.K / 8;
    if (pieces <= 64) return launch_norm_t<E, 64, 1>(a, stream, timer);
    if (pieces <= 128) return launch_norm_t<E, 64, 2>(a, stream, timer);
    if (pieces <= 256) return launch_norm_t<E, 256, 1>(a, stream, timer);
    if (pieces <= 512) return launch_norm_t<E, 512, 1>(a, stream, timer);
    if (pieces <= 1024) return launch_norm_t<E, 512, 2>(a, stream, timer);
    if (pieces <= 2048) return launch_norm_t<E, 512, 4>(a, stream, timer);
    if (pieces <= 4096) return launch_norm_t<E, 1024, 4>(a, stream, timer);
    return launch_norm_t<E, 1024, 8>(a, stream, timer);
}

// A tensor without gaps between its rows, scales included, is one long row: blocks end where rows do.
template <typename F>
hipError_t launch_convert(const MxConvertArgs &a0, int format, int64_t ld_values, int64_t ld_codes, F launch) {
    MxConvertArgs a = a0;
    const int64_t code_bytes = format == kMxE2M1 ? a.K / 2 : a.K;
    if (ld_values == a.K && ld_codes == code_bytes && a.ldsc == a.K / kMxBlock && a.rows * a.K <= INT32_MAX - 2 * kMxStrip) {
        a.K = (int32_t)(a.rows * a.K);
        a.rows = 1;
    }
    a.strips = (a.K + kMxStrip - 1) / kMxStrip;
    const int64_t units = a.rows * a.strips;  // (fewer than 2^31: the caller has checked)
    if (units <= 0) return hipSuccess;
    return launch(a, grid_of((units + kMxWaves - 1) / kMxWaves));
}

}  // namespace

hipError_t launch_mx_quantize(const MxConvertArgs &a, int dtype, int format, hipStream_t stream, const KernelTimer *timer) {
    return launch_convert(a, format, a.lds, a.ldd, [&](const MxConvertArgs &b, dim3 grid) {
        const dim3 block(kMxWaves * 64);
        if (dtype == 1)
            return format == kMxE2M1 ? launch_kernel(mx_quantize_kernel<__bf16, kMxE2M1>, grid, block, 0, stream, timer, b)
                                     : launch_kernel(mx_quantize_kernel<__bf16, kMxE4M3>, grid, block, 0, stream, timer, b);
        return format == kMxE2M1 ? launch_kernel(mx_quantize_kernel<float, kMxE2M1>, grid, block, 0, stream, timer, b)
                                 : launch_kernel(mx_quantize_kernel<float, kMxE4M3>, grid, block, 0, stream, timer, b);
    });
}

hipError_t launch_mx_dequantize(const MxConvertArgs &a, int dtype, int format, hipStream_t stream, const KernelTimer *timer) {
    return launch_convert(a, format, a.ldd, a.lds, [&](const MxConvertArgs &b, dim3 grid) {
        const dim3 block(kMxWaves * 64);
        if (dtype == 1)
            return format == kMxE2M1 ? launch_kernel(mx_dequantize_kernel<__bf16, kMxE2M1>, grid, block, 0, stream, timer, b)
                                     : launch_kernel(mx_dequantize_kernel<__bf16, kMxE4M3>, grid, block, 0, stream, timer, b);
        return format == kMxE2M1 ? launch_kernel(mx_dequantize_kernel<float, kMxE2M1>, grid, block, 0, stream, timer, b)
                                 : launch_kernel(mx_dequantize_kernel<float, kMxE4M3>, grid, block, 0, stream, timer, b);
    });
}

hipError_t launch_mx_split(const MxSplitArgs &a0, hipStream_t stream, const KernelTimer *timer) {
    MxSplitArgs a = a0;
    a.strips = (a.part_bytes + kMxStrip - 1) / kMxStrip;
    const int64_t units = (int64_t)a.rows * a.strips;
    if (units <= 0) return hipSuccess;
    if (units > INT32_MAX || a.part_bytes % 512 || a.part_bytes < a.K || a.part_scales < a.part_bytes / kMxBlock) return hipErrorInvalidValue;
    return launch_kernel(mx_split_kernel, grid_of((units + kMxWaves - 1) / kMxWaves), dim3(kMxWaves * 64), 0, stream, timer, a);
}

hipError_t launch_rms_norm(const RmsNormArgs &a, int dtype, hipStream_t stream, const KernelTimer *timer) {
    if (a.rows <= 0) return hipSuccess;
    return dtype == 1 ? launch_norm_e<__bf16>(a, stream, timer) : launch_norm_e<float>(a, stream, timer);
}

}  // namespace lora
