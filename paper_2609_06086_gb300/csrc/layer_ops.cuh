// Shared by the layer operators (ckpt.cu, qk.cu, wgrad.cu, norm*.cu, dropout.cu, attn*.cu):
// element types, 8-element vectors, and the arithmetic of an 8-bit checkpoint (poseidon.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cstring>

#include "common.cuh"

namespace pos {

// The library's scratch pool of the current device (eval.cu), and the one for a call's `bytes`:
// that one, which keeps its memory, or for many one that gives it back.
pos_status scratch_pool(cudaMemPool_t *out);
pos_status scratch_pool(cudaMemPool_t *out, int64_t bytes);

constexpr int kGroup = 32;             // columns that share a scale
constexpr int kScaleLo = 17;           // scale byte of e = -110
constexpr int kScaleNan = 255;
template <int F>                       // POS_CKPT_*
struct Fmt;
template <>
struct Fmt<POS_CKPT_INT8> {
    static constexpr int kScaleHi = 248;  // e = 121: 127 * 2^121 is finite in f32 and bf16
    // 127 = 1.984375 * 2^6: a larger mantissa carries into the exponent
    static constexpr uint32_t kCarry = 0x7fffffu - 0x7e0000u;
    static constexpr int kLead = 6;
    static constexpr float kTop = 127.f;
};
template <>
struct Fmt<POS_CKPT_E4M3> {
    static constexpr int kScaleHi = 246;  // e = 119: 448 * 2^119 is finite
    static constexpr uint32_t kCarry = 0x7fffffu - 0x600000u;  // 448 = 1.75 * 2^8
    static constexpr int kLead = 8;
    static constexpr float kTop = 448.f;
};

// Scale byte of a group from the bits of its largest |x| as f32 (whose order
// as whole numbers is that of the magnitudes, infinities and NaNs on top).
template <int F>
__device__ __forceinline__ int scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return kScaleNan;
    const int b = (int)((amax_bits + Fmt<F>::kCarry) >> 23) - Fmt<F>::kLead;
    return min(max(b, kScaleLo), Fmt<F>::kScaleHi);
}

// 2^e of a scale byte as f32, a NaN for kScaleNan.
__device__ __forceinline__ float scale_value(int byte) {
    return __uint_as_float(byte == kScaleNan ? 0x7fffffffu : (uint32_t)byte << 23);
}

// n / d for n < 2^31 by a multiplication (round-up method).
struct FastDiv {
    uint32_t d, mul, shift;
    explicit FastDiv(uint32_t v) : d(v), mul(0), shift(0) {
        while ((1ull << shift) < v) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - v)) / v + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const {
        return (__umulhi(n, mul) + n) >> shift;
    }
};

struct Vec8 {
    float v[8];
};

// Two f32 operations in one instruction.
struct F2 {
    float x, y;
};
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("{\n.reg .b64 a, b, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\n"
        "mul.rn.f32x2 r, a, b;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("{\n.reg .b64 a, b, c, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\n"
        "mov.b64 c, {%6, %7};\nfma.rn.f32x2 r, a, b, c;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ F2 both(float v) { return {v, v}; }

// Codes of 4 values under one scale byte below the largest.  x * 2^-e is exact
// (or an underflow far below half a code), so each code is rounded once: int8
// by adding 1.5 * 2^23, whose last bit is a whole number, e4m3 by the
// conversion.
template <int F>
__device__ __forceinline__ uint32_t encode4_inside(float x0, float x1, float x2, float x3,
                                                   int byte) {
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
    if constexpr (F == POS_CKPT_INT8) {
        const F2 u = fma2({x0, x1}, both(inv), both(12582912.f));
        const F2 v = fma2({x2, x3}, both(inv), both(12582912.f));
        return __byte_perm(__byte_perm(__float_as_uint(u.x), __float_as_uint(u.y), 0x0040),
                           __byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x0040),
                           0x5410);
    } else {
        const F2 u = mul2({x0, x1}, both(inv)), v = mul2({x2, x3}, both(inv));
        const uint32_t lo =
            __nv_cvt_float2_to_fp8x2(make_float2(u.x, u.y), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi =
            __nv_cvt_float2_to_fp8x2(make_float2(v.x, v.y), __NV_SATFINITE, __NV_E4M3);
        return lo | hi << 16;
    }
}
// The same under any scale byte: at the largest, values past the top code
// saturate; a group that is NaN has codes 0.
template <int F>
__device__ __forceinline__ uint32_t encode4(float x0, float x1, float x2, float x3, int byte) {
    if (byte >= Fmt<F>::kScaleHi) {
        if (byte == kScaleNan) return 0u;
        const float top = Fmt<F>::kTop * scale_value(byte);
        x0 = fminf(fmaxf(x0, -top), top), x1 = fminf(fmaxf(x1, -top), top);
        x2 = fminf(fmaxf(x2, -top), top), x3 = fminf(fmaxf(x3, -top), top);
    }
    return encode4_inside<F>(x0, x1, x2, x3, byte);
}
template <int F>
__device__ __forceinline__ uint2 encode8(const Vec8 &x, int byte) {
    return make_uint2(encode4<F>(x.v[0], x.v[1], x.v[2], x.v[3], byte),
                      encode4<F>(x.v[4], x.v[5], x.v[6], x.v[7], byte));
}

// The values of 8 codes: exact in f32.
template <int F>
__device__ __forceinline__ Vec8 decode8(uint2 c, float scale) {
    Vec8 x;
    const uint32_t w[2] = {c.x, c.y};
    if constexpr (F == POS_CKPT_INT8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the code + 128 in the last byte of 2^23
            const uint32_t u = __byte_perm(w[i / 4] ^ 0x80808080u, 0x4b000000u, 0x7440u | i % 4);
            x.v[i] = (__uint_as_float(u) - 8388736.f) * scale;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(
                (__nv_fp8x2_storage_t)(w[i / 2] >> (16 * (i % 2))), __NV_E4M3);
            const float2 f = __half22float2(__half2(h));
            x.v[2 * i] = f.x * scale;
            x.v[2 * i + 1] = f.y * scale;
        }
    }
    return x;
}

// ---------------------------------------------------------------------------
// Element types: 8 consecutive elements as raw words
// ---------------------------------------------------------------------------
template <typename T>
struct Raw8;  // 16 or 32 bytes
template <>
struct Raw8<__nv_bfloat16> {
    uint4 a;
};
template <>
struct Raw8<__half> {
    uint4 a;
};
template <>
struct Raw8<float> {
    uint4 a, b;
};

__device__ __forceinline__ void zero_raw(uint4 &a) { a = make_uint4(0, 0, 0, 0); }

// ALIGNED: p is 16-byte aligned and all 8 elements exist; otherwise `n` of
// them (any number, <= 0: none) are read one by one, the others are zeros.
template <bool ALIGNED, typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p, int n) {
    Raw8<T> r;
    if constexpr (ALIGNED) {
        if (n >= 8) {
            r.a = *reinterpret_cast<const uint4 *>(p);
            if constexpr (sizeof(T) == 4) r.b = *(reinterpret_cast<const uint4 *>(p) + 1);
            return r;
        }
    }
    zero_raw(r.a);
    if constexpr (sizeof(T) == 4) zero_raw(r.b);
    if constexpr (sizeof(T) == 4) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = i < n ? reinterpret_cast<const uint32_t *>(p)[i] : 0u;
        r.a = make_uint4(w[0], w[1], w[2], w[3]);
        r.b = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = i < n ? (uint32_t) reinterpret_cast<const uint16_t *>(p)[i] : 0u;
        r.a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16,
                         w[6] | w[7] << 16);
    }
    return r;
}

// 8 elements at p, which need not be 16-byte aligned, from the aligned words
// around them; those words lie inside the row, [p - before, p + left).
template <typename T>
__device__ __forceinline__ Raw8<T> load8_shifted(const T *p, int before, int left) {
    constexpr int kPer = 16 / sizeof(T);
    const int m = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % kPer);
    if (m == 0 && left >= 8) return load8<true>(p, 8);
    if (before < m || left < 8 - m + kPer) return load8<false>(p, left);
    constexpr int kWords = 4 * (8 / kPer + 1);
    uint32_t w[kWords];
    const uint4 *at = reinterpret_cast<const uint4 *>(p - m);
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
        const uint4 v = at[i];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
    // down by m elements: whole words by two choices, then half a word
    const int q = sizeof(T) == 2 ? m / 2 : m;
    if (q & 2) {
#pragma unroll
        for (int i = 0; i + 2 < kWords; ++i) w[i] = w[i + 2];
    }
    if (q & 1) {
#pragma unroll
        for (int i = 0; i + 1 < kWords; ++i) w[i] = w[i + 1];
    }
    if (sizeof(T) == 2 && (m & 1)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    Raw8<T> r;
    r.a = make_uint4(w[0], w[1], w[2], w[3]);
    if constexpr (sizeof(T) == 4) r.b = make_uint4(w[4], w[5], w[6], w[7]);
    return r;
}

template <bool ALIGNED, typename T>
__device__ __forceinline__ void store8(T *p, const Raw8<T> &r, int n) {
    if constexpr (ALIGNED) {
        if (n >= 8) {
            *reinterpret_cast<uint4 *>(p) = r.a;
            if constexpr (sizeof(T) == 4) *(reinterpret_cast<uint4 *>(p) + 1) = r.b;
            return;
        }
    }
    if constexpr (sizeof(T) == 4) {
        const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) reinterpret_cast<uint32_t *>(p)[i] = w[i];
    } else {
        const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    }
}

// 8 elements at p, which need not be 16-byte aligned, as aligned words: a lane takes the
// last elements of the lane before it and leaves its own last ones to the lane behind it.
// Called by all lanes of a warp; `left` elements exist from p on (any number), of which 8
// at most are this lane's.  has_prev, has_next: the lane before or behind holds the 8
// elements before or behind these, and calls with them.  What has no such lane is
// stored element by element.
template <typename T>
__device__ __forceinline__ void store8_shifted(T *p, const Raw8<T> &r, int left, bool has_prev,
                                               bool has_next) {
    constexpr int kPer = 16 / sizeof(T), kWords = 2 * sizeof(T);  // 32-bit words of 8 elements
    // (at least one lane is off the alignment in the cases that this is for)
    const int m = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % kPer);
    uint32_t w[2 * kWords];
    w[kWords] = r.a.x, w[kWords + 1] = r.a.y, w[kWords + 2] = r.a.z, w[kWords + 3] = r.a.w;
    if constexpr (sizeof(T) == 4)
        w[12] = r.b.x, w[13] = r.b.y, w[14] = r.b.z, w[15] = r.b.w;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = __shfl_up_sync(0xffffffffu, w[kWords + i], 1);
    if (m == 0) {
        store8<true>(p, r, left);
        return;
    }
    if (left + m > 0 && has_prev) {
        // the words from 8 - m elements of the lane before on: down by as many
        const int down = 8 - m, q = sizeof(T) == 2 ? down / 2 : down;
        uint32_t v[2 * kWords];
#pragma unroll
        for (int i = 0; i < 2 * kWords; ++i) v[i] = w[i];
        if (sizeof(T) == 4 && (q & 4)) {
#pragma unroll
            for (int i = 0; i + 4 < 2 * kWords; ++i) v[i] = v[i + 4];
        }
        if (q & 2) {
#pragma unroll
            for (int i = 0; i + 2 < 2 * kWords; ++i) v[i] = v[i + 2];
        }
        if (q & 1) {
#pragma unroll
            for (int i = 0; i + 1 < 2 * kWords; ++i) v[i] = v[i + 1];
        }
        if (sizeof(T) == 2 && (down & 1)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 16);
        }
        Raw8<T> o;
        o.a = make_uint4(v[0], v[1], v[2], v[3]);
        if constexpr (sizeof(T) == 4) o.b = make_uint4(v[4], v[5], v[6], v[7]);
        store8<true>(p - m, o, left + m);
    }
    if (!has_prev || !has_next) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >= left || (e < 8 - m ? has_prev : has_next)) continue;
            if constexpr (sizeof(T) == 4)
                reinterpret_cast<uint32_t *>(p)[e] = w[kWords + e];
            else
                reinterpret_cast<uint16_t *>(p)[e] = (uint16_t)(w[kWords + e / 2] >> (16 * (e % 2)));
        }
    }
}

template <typename T>
__device__ __forceinline__ Vec8 to_float(const Raw8<T> &r) {
    Vec8 x;
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
    if constexpr (std::is_same<T, float>::value) {
        const uint32_t u[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x.v[i] = __uint_as_float(w[i]);
            x.v[4 + i] = __uint_as_float(u[i]);
        }
    } else if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __half2 h;
            memcpy(&h, &w[i], 4);
            const float2 f = __half22float2(h);
            x.v[2 * i] = f.x;
            x.v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x.v[2 * i] = __uint_as_float(w[i] << 16);
            x.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    return x;
}

// Rounded to nearest even.  SAT: f16 saturates at its largest finite value
// (NaNs stay).
template <typename T, bool SAT = false>
__device__ __forceinline__ Raw8<T> from_float(const Vec8 &x) {
    Raw8<T> r;
    if constexpr (std::is_same<T, float>::value) {
        r.a = make_uint4(__float_as_uint(x.v[0]), __float_as_uint(x.v[1]), __float_as_uint(x.v[2]),
                         __float_as_uint(x.v[3]));
        r.b = make_uint4(__float_as_uint(x.v[4]), __float_as_uint(x.v[5]), __float_as_uint(x.v[6]),
                         __float_as_uint(x.v[7]));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __half>::value) {
                __half2 h = __floats2half2_rn(x.v[2 * i], x.v[2 * i + 1]);
                if constexpr (SAT) {
                    const __half2 top = __half2half2(__ushort_as_half(0x7bff));
                    h = __hmin2_nan(__hmax2_nan(h, __hneg2(top)), top);
                }
                memcpy(&w[i], &h, 4);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x.v[2 * i], x.v[2 * i + 1]);
                memcpy(&w[i], &h, 4);
            }
        }
        r.a = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}

// Bits of the largest |x| of 8 elements, in a form that max_bits() and
// shuffles combine and f32_bits() turns into the bits of an f32: two 16-bit
// magnitudes for the 16-bit types, whose bits order them too.
template <typename T>
__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) return max(a, b);
    else return __vmaxu2(a, b);
}
template <typename T>
__device__ __forceinline__ uint32_t amax_bits(const Raw8<T> &r) {
    constexpr uint32_t kAbs = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    uint32_t m = max_bits<T>(max_bits<T>(r.a.x & kAbs, r.a.y & kAbs),
                             max_bits<T>(r.a.z & kAbs, r.a.w & kAbs));
    if constexpr (sizeof(T) == 4)
        m = max(m, max(max(r.b.x & kAbs, r.b.y & kAbs), max(r.b.z & kAbs, r.b.w & kAbs)));
    return m;
}
template <typename T>
__device__ __forceinline__ uint32_t f32_bits(uint32_t m) {
    if constexpr (std::is_same<T, float>::value) return m;
    const uint32_t h = max(m & 0xffffu, m >> 16);
    if constexpr (std::is_same<T, __half>::value)
        return __float_as_uint(__half2float(__ushort_as_half((unsigned short)h)));
    return h << 16;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct CkptShape {
    int64_t groups, pitch, spitch;  // per row: groups, code bytes, scale bytes
};
inline CkptShape ckpt_shape(int64_t cols) {
    const int64_t g = (cols + kGroup - 1) / kGroup;
    return {g, g * kGroup, (g + 3) / 4 * 4};
}
// Sizes that a checkpoint can have (its byte count below 2^62).
inline bool ckpt_size_ok(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || cols > 0x7fffffffll - kGroup) return false;
    const CkptShape s = ckpt_shape(cols);
    return s.pitch == 0 || rows < (1ll << 62) / (s.pitch + s.spitch);
}
// Runs an entry point's work: no C++ exception leaves the library.
template <typename F>
pos_status guarded(F work) noexcept {
    try {
        return work();
    } catch (...) {  // only allocations of host memory throw here
        return POS_ENOMEM;
    }
}
// Whether two rows of a tensor share an element.
inline bool rows_overlap(int64_t tokens, int64_t heads, int64_t dim, int64_t token_stride,
                         int64_t head_stride) {
    if ((heads > 1 && head_stride < dim) || (tokens > 1 && token_stride < dim)) return true;
    if (heads <= 1 || tokens <= 1) return false;
    // one token's rows before the next token's, or one head's before the next head's
    if (token_stride >= (heads - 1) * head_stride + dim) return false;
    if ((head_stride - dim) / token_stride >= tokens - 1) return false;
    for (int64_t h = 1; h < heads; ++h) {  // against head 0 of the tokens beside it
        const int64_t at = h * head_stride, t = at / token_stride;
        if (t > 0 && t < tokens && at - t * token_stride < dim) return true;
        if (t + 1 < tokens && (t + 1) * token_stride - at < dim) return true;
    }
    return false;
}
inline bool dtype_ok(int32_t d) { return d == POS_BF16 || d == POS_F16 || d == POS_F32; }
inline bool format_ok(int32_t f) { return f == POS_CKPT_INT8 || f == POS_CKPT_E4M3; }
inline int dtype_size(int32_t d) { return d == POS_F32 ? 4 : 2; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace pos
