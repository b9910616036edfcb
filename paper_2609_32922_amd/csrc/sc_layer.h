// What the layer operators (fp8 quantiser and product, residual norms, rotary positions) share:
// element types, loads and stores of four elements at a time, sums and maxima over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/scgemm.h"

namespace scl {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_any __attribute__((aligned(1)));        // 16 bytes at any address
typedef u2 u2_any __attribute__((aligned(1)));
typedef uint32_t word_any __attribute__((aligned(1)));
typedef u4 u4_8 __attribute__((aligned(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr float E4M3_MAX = 448.0f, E5M2_MAX = 57344.0f;
constexpr int FP8_BLOCK = SC_FP8_BLOCK;

inline bool is_float_type(int t) { return t == SC_F32 || t == SC_BF16 || t == SC_F16; }
inline bool is_fp8_type(int t) { return t == SC_E4M3 || t == SC_E5M2; }
__host__ __device__ __forceinline__ int type_bytes(int t) { return t == SC_F32 ? 4 : t == SC_BF16 || t == SC_F16 ? 2 : 1; }
inline bool aligned_to(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

// Two floats to the nearest bf16 or fp16 values, ties to even, the first in the lower half
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 hf2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t to_pair(int type, float lo, float hi) {
    if (type == SC_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), bf2));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), hf2));
}
__device__ __forceinline__ float from_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float from_f16(uint32_t x) { return (float)__builtin_bit_cast(_Float16, (uint16_t)x); }

// Four elements as they lie in memory: all four words of a float32, two words of a 16-bit type.  The
// words are loaded first and turned into floats later, so that a row's loads are all in flight at once.  (VEC, here and below: four
// elements lie on their size, and there are four or none.  Otherwise four are moved at once wherever they lie, and what a row has
// behind its last four one by one.  18464 x 1023 bfloat16 to fp8 takes 18 us so, 34 with every element moved by itself, and 4097 x 1153
// gradients 39 and 52.)
struct Raw4 {
    u4 w;
};
template <bool VEC>
__device__ __forceinline__ Raw4 load_raw(int type, const void *p, int64_t at, int n) {
    Raw4 r;
    r.w = u4{0u, 0u, 0u, 0u};
    if (n <= 0) return r;
    if (type == SC_F32) {
        const uint32_t *q = static_cast<const uint32_t *>(p) + at;
        if (VEC) {
            r.w = *reinterpret_cast<const u4 *>(q);
        } else {
            if (n >= 4) r.w = *reinterpret_cast<const u4_any *>(q);
            else
                for (int j = 0; j < 3; ++j)
                    if (j < n) r.w[j] = q[j];
        }
    } else {
        const uint16_t *q = static_cast<const uint16_t *>(p) + at;
        if (VEC) {
            const u2 t = *reinterpret_cast<const u2 *>(q);
            r.w[0] = t[0];
            r.w[1] = t[1];
        } else {
            if (n >= 4) {
                const u2 t = *reinterpret_cast<const u2_any *>(q);
                r.w[0] = t[0];
                r.w[1] = t[1];
            } else {
                for (int j = 0; j < 3; ++j)
                    if (j < n) r.w[j >> 1] |= (uint32_t)q[j] << (16 * (j & 1));
            }
        }
    }
    return r;
}
__device__ __forceinline__ f4 to_floats(int type, const Raw4 &r) {
    f4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t h = (r.w[j >> 1] >> (16 * (j & 1))) & 0xffffu;
        v[j] = type == SC_F32 ? __uint_as_float(r.w[j]) : type == SC_BF16 ? from_bf16(h) : from_f16(h);
    }
    return v;
}
// (STREAM: past the caches)
template <bool VEC, bool STREAM = false>
__device__ __forceinline__ void store4(int type, void *p, int64_t at, f4 v, int n) {
    if (n <= 0) return;
    if (type == SC_F32) {
        float *q = static_cast<float *>(p) + at;
        if (VEC) {
            if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<f4 *>(q));
            else *reinterpret_cast<f4 *>(q) = v;
        } else {
            if (n >= 4) *reinterpret_cast<u4_any *>(q) = __builtin_bit_cast(u4, v);
            else
                for (int j = 0; j < 3; ++j)
                    if (j < n) q[j] = v[j];
        }
    } else {
        const u2 w = {to_pair(type, v[0], v[1]), to_pair(type, v[2], v[3])};
        uint16_t *q = static_cast<uint16_t *>(p) + at;
        if (VEC) {
            if (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<u2 *>(q));
            else *reinterpret_cast<u2 *>(q) = w;
        } else {
            if (n >= 4) *reinterpret_cast<u2_any *>(q) = w;
            else
                for (int j = 0; j < 3; ++j)
                    if (j < n) q[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// Over groups of W neighbouring lanes (W a power of two), every lane gets the result.  Within 16 lanes by the
// vector unit's own lane moves, beyond by the swaps of rows and halves: no trip through LDS.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int W, typename F>
__device__ __forceinline__ float lanes(float v, F f) {
    if (W >= 2) v = f(v, moved<0xb1>(v));       // quad_perm 1 0 3 2
    if (W >= 4) v = f(v, moved<0x4e>(v));       // quad_perm 2 3 0 1
    if (W >= 8) v = f(v, moved<0x141>(v));      // row_half_mirror
    if (W >= 16) v = f(v, moved<0x140>(v));     // row_mirror
    if (W >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if (W >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}
template <int W>
__device__ __forceinline__ float lanes_max(float v) {
    return lanes<W>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
    return lanes<W>(v, [](float a, float b) { return a + b; });
}

// Scale of an fp8 block with largest magnitude m, and its reciprocal.  The scale is at least the least
// normal float, so that its reciprocal is finite; a block of zeros has scale 0 and quantises to zeros.
struct Fp8Scale {
    float s, inv;
};
__device__ __forceinline__ Fp8Scale fp8_scale(float m, float top) {
    Fp8Scale r;
    r.s = m > 0.0f ? fmaxf(m / top, 1.1754943508222875e-38f) : 0.0f;
    r.inv = m > 0.0f ? 1.0f / r.s : 0.0f;
    return r;
}
// x * inv held within the type's range (the product may pass it by a rounding); NaN stays NaN
__device__ __forceinline__ float fp8_clamped(float x, float inv, float top) {
    const float y = x * inv;
    return y != y ? y : fminf(fmaxf(y, -top), top);
}
// four floats to four bytes, ties to even; E5: e5m2, else e4m3
template <bool E5>
__device__ __forceinline__ uint32_t to_fp8x4(float a, float b, float c, float d) {
    int w = 0;
    if (E5) {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}
__device__ __forceinline__ uint32_t quant_fp8x4(bool e5, f4 v, float inv) {
    const float top = e5 ? E5M2_MAX : E4M3_MAX;
    f4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fp8_clamped(v[j], inv, top);
    return e5 ? to_fp8x4<true>(y[0], y[1], y[2], y[3]) : to_fp8x4<false>(y[0], y[1], y[2], y[3]);
}
// int8 of a row with scale s (the quantiser's formula: rint(x / s), ties to even, s = 0 gives 0)
__device__ __forceinline__ uint32_t quant_int8x4(f4 v, float s) {
    uint32_t w = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = s > 0.0f ? fminf(fmaxf(rintf(v[j] / s), -127.0f), 127.0f) : 0.0f;
        w |= ((uint32_t)(int)q & 255u) << (8 * j);
    }
    return w;
}
template <bool VEC>
__device__ __forceinline__ void store_bytes4(void *p, int64_t at, uint32_t w, int n) {
    if (n <= 0) return;
    uint8_t *q = static_cast<uint8_t *>(p) + at;
    if (VEC) {
        *reinterpret_cast<uint32_t *>(q) = w;
    } else {
        if (n >= 4) *reinterpret_cast<word_any *>(q) = w;
        else
            for (int j = 0; j < 3; ++j)
                if (j < n) q[j] = (uint8_t)(w >> (8 * j));
    }
}

// Whether no two of the n0 x n1 x n2 runs of `unit` elements at strides s0, s1, s2 coincide, as a sufficient test: taken by
// growing stride, each stride passes what the smaller ones span
inline bool apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t unit) {
    int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (s[j] < s[i]) {
                const int64_t tn = n[i], ts = s[i];
                n[i] = n[j];
                s[i] = s[j];
                n[j] = tn;
                s[j] = ts;
            }
    __int128 span = unit;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (s[i] < span) return false;
        span += (__int128)(n[i] - 1) * s[i];
    }
    return true;
}
// the same of rows of `unit` elements in batch entries; nothing coincides where nothing is written
inline bool rows_apart(int64_t batch, int64_t stride, int64_t rows, int64_t ld, int64_t unit) {
    return rows == 0 || unit == 0 || apart(batch, stride, rows, ld, 1, 0, unit);
}

// A grid of `blocks` blocks for each of `batch` entries: a launch holds fewer than 2^32 threads along a
// dimension, so blocks go on in rows of 2^20; entries past the third dimension's are taken in turn.
inline dim3 grid_of(uint32_t blocks, int batch) {
    const uint32_t x = blocks < (1u << 20) ? blocks : 1u << 20;
    return dim3(x, (blocks + x - 1) / x, (unsigned)(batch < 32768 ? batch : 32768));
}
__device__ __forceinline__ uint32_t block_id() { return blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace scl
