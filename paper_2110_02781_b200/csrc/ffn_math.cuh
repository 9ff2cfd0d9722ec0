// Activations, their derivatives, 8-bit blocks and four-element accesses of the feed-forward kernels.
#pragma once
#include "ffn.h"

namespace ftp {
namespace ffn {

// exp and the division at float accuracy for float tensors; for bf16 tensors the hardware approximations, whose error
// (2^-21 relative) is far below the rounding of the result to 8 bits of mantissa.
__device__ __forceinline__ float rcp_fast(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float ex2_fast(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
constexpr float LOG2E = 1.4426950408889634f;
template <bool FAST> __device__ __forceinline__ float sigmoid_t(float z) {
    return FAST ? rcp_fast(1.f + ex2_fast(z * -LOG2E)) : 1.f / (1.f + expf(-z));
}

// For bf16 tensors: Phi(z) without a branch from e^(-z^2/2) and the rational approximation 7.1.26 of Abramowitz and Stegun,
// Handbook of Mathematical Functions (1964), of erfc: |error| <= 1.5e-7, a 1/26000 of bf16's half step at 1.  Relative to
// Phi(z) itself 0.36 % at z = -6 (half a step of bf16), 1 % at -8, 3 % at -12.  erff takes both sides of a branch in almost
// every warp and twice the instructions.  e: e^(-z^2/2), shared with the density.
__device__ __forceinline__ float phi_fast(float z, float e) {
    const float t = rcp_fast(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
    const float q = 0.5f * e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);   // Phi(-|z|)
    return z > 0.f ? 1.f - q : q;
}

// For float tensors: from erfc, whose error is relative; 0.5 + 0.5 erf cancels for negative z (4 % of the result at z = -5).
__device__ __forceinline__ float phi_exact(float z) { return 0.5f * erfcf(z * -0.70710678118654752f); }

// NaN passes through every branch.
template <bool FAST>
__device__ __forceinline__ float act_value(float z, int act) {
    switch (act) {
        case FTP_ACT_RELU: return z < 0.f ? 0.f : z;
        case FTP_ACT_RELU6: return z < 0.f ? 0.f : (z > 6.f ? 6.f : z);
        case FTP_ACT_GELU: return z * (FAST ? phi_fast(z, ex2_fast(z * z * (-0.5f * LOG2E))) : phi_exact(z));
        case FTP_ACT_SILU: return z * sigmoid_t<FAST>(z);
        default: return z;
    }
}
template <bool FAST>
__device__ __forceinline__ void act_both(float z, int act, float& v, float& d) {
    switch (act) {
        case FTP_ACT_RELU: v = z < 0.f ? 0.f : z; d = z > 0.f ? 1.f : (z <= 0.f ? 0.f : z); break;
        case FTP_ACT_RELU6: v = z < 0.f ? 0.f : (z > 6.f ? 6.f : z); d = z > 0.f && z < 6.f ? 1.f : (z == z ? 0.f : z); break;
        case FTP_ACT_GELU: {
            const float e = FAST ? ex2_fast(z * z * (-0.5f * LOG2E)) : expf(-0.5f * z * z), p = FAST ? phi_fast(z, e) : phi_exact(z);
            v = z * p;
            // for |z| beyond 14 the density is 0 in float; z * 0 at z = +-inf would be NaN
            d = p + (fabsf(z) > 14.f ? 0.f : z * e * 0.39894228040143268f);
            break;
        }
        case FTP_ACT_SILU: {
            const float s = sigmoid_t<FAST>(z);
            v = z * s;
            d = s + (s == 0.f || s == 1.f ? 0.f : v * (1.f - s));
            break;
        }
        default: v = z; d = 1.f;
    }
}

// ---- four consecutive elements ----
__device__ __forceinline__ float bf_lo(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(unsigned u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ unsigned bf_pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ void load4(const float* p, int valid, bool vec, float (&v)[4]) {
    if (vec && valid >= 4) { const float4 t = *reinterpret_cast<const float4*>(p); v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < valid ? p[i] : 0.f;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int valid, bool vec, float (&v)[4]) {
    if (vec && valid >= 4) { const uint2 t = *reinterpret_cast<const uint2*>(p); v[0] = bf_lo(t.x); v[1] = bf_hi(t.x); v[2] = bf_lo(t.y); v[3] = bf_hi(t.y); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < valid ? __bfloat162float(p[i]) : 0.f;
}
__device__ __forceinline__ void store4(float* p, int valid, bool vec, const float (&v)[4]) {
    if (vec && valid >= 4) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < valid) p[i] = v[i];
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, int valid, bool vec, const float (&v)[4]) {
    if (vec && valid >= 4) { *reinterpret_cast<uint2*>(p) = make_uint2(bf_pack(v[0], v[1]), bf_pack(v[2], v[3])); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < valid) p[i] = __float2bfloat16(v[i]);
}

// ---- 8-bit blocks ----
// Byte of the scale from the bits of the block's largest magnitude: exponent - 6 (so that the largest code is 64..127),
// at least that of 2^-126, 255 where the block holds a NaN or an infinity.
__device__ __forceinline__ unsigned img_exp(unsigned amax_bits) {
    const int be = (int)(amax_bits >> 23);
    return be == 255 ? 255u : (unsigned)max(be - 6, 1);
}
__device__ __forceinline__ float img_scale(unsigned e) { return e == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(e << 23); }
// 1 / scale = 2^(127 - byte): exact, a subnormal for byte 254 at most (bytes end at 248)
__device__ __forceinline__ float img_inv(unsigned e) { return e == 255u ? 0.f : __uint_as_float((254u - e) << 23); }
// Codes without a conversion instruction (a quarter of the rate of an addition): v * inv is exact, and adding 1.5 * 2^23
// rounds it to the nearest integer, ties to even, which then is the low byte of the sum's bits.
constexpr float IMG_MAGIC = 12582912.f;
__device__ __forceinline__ unsigned img_code(float v, float inv) {
    // a NaN (byte 255) becomes some code that no reader uses
    return __float_as_uint(fminf(fmaxf(v * inv, -127.f), 127.f) + IMG_MAGIC);
}
// low bytes of four words
__device__ __forceinline__ unsigned pack_codes(unsigned a, unsigned b, unsigned c, unsigned d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// the four codes of a word as floats: code + 128 under the exponent of 2^23, less 2^23 + 128
__device__ __forceinline__ void unpack_codes(unsigned q, float scale, float (&v)[4]) {
    const unsigned u = q ^ 0x80808080u;
    v[0] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)) - 8388736.f) * scale;
    v[1] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441)) - 8388736.f) * scale;
    v[2] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)) - 8388736.f) * scale;
    v[3] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443)) - 8388736.f) * scale;
}

// ---- consecutive elements of rows that start anywhere ----
// The bytes of a matrix, between which a whole 16-byte part may be read.
struct Span { const char *lo, *hi; };
template <typename T> Span span_of(const void* p, long long rows, long long cols, long long ld) {
    return Span{static_cast<const char*>(p), static_cast<const char*>(p) + ((rows - 1) * ld + cols) * (long long)sizeof(T)};
}
// W words from p on, as the aligned 16-byte parts that cover them, of which neighbouring threads read the same ones, and how
// far to shift them (element by element a copy of 4720 x 11570 bf16 ran at 2.4 TB/s).  `begin` has no branch in front of its
// loads, so that those of several rows are in flight together; where a part reaches out of the matrix, the `valid` elements
// are loaded one by one.  `end`: the words, zeros behind `valid`.
template <typename T, int W> struct Words {
    static constexpr int PER = 4 / (int)sizeof(T);
    unsigned w[W + 4], sh;
    __device__ __forceinline__ void begin(const T* p, int valid, const Span& all) {
        sh = (unsigned)(reinterpret_cast<uintptr_t>(p) & 15);
        const char* from = reinterpret_cast<const char*>(p) - sh;
        const bool ok = from >= all.lo && from + W * 4 + (sh ? 16 : 0) <= all.hi;
#pragma unroll
        for (int k = 0; k <= W / 4; ++k) {
            const uint4 t = ok && (k < W / 4 || sh) ? reinterpret_cast<const uint4*>(from)[k] : make_uint4(0u, 0u, 0u, 0u);
            w[4 * k] = t.x; w[4 * k + 1] = t.y; w[4 * k + 2] = t.z; w[4 * k + 3] = t.w;
        }
        if (!ok) {
            sh = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                w[i] = 0u;
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (i * PER + e < valid) w[i] |= bits_of(p[i * PER + e]) << (16 * e);
            }
        }
    }
    __device__ __forceinline__ void end(int valid, unsigned (&out)[W]) const {
        unsigned a[W + 2], b[W + 1];
#pragma unroll
        for (int i = 0; i < W + 2; ++i) a[i] = sh & 8 ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i < W + 1; ++i) b[i] = sh & 4 ? a[i + 1] : a[i];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const unsigned v = sh & 2 ? __funnelshift_r(b[i], b[i + 1], 16) : b[i];
            out[i] = i * PER >= valid ? 0u : PER == 2 && i * PER + 1 >= valid ? v & 0xffffu : v;
        }
    }
    static __device__ __forceinline__ unsigned bits_of(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ unsigned bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
};

}  // namespace ffn
}  // namespace ftp
