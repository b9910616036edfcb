// Rotary positions with several axes.
#include <math.h>

#include "sc_layer.h"

namespace scl {

struct RopeArgs {
    sc_rope_desc d;
    const void *x;
    const int32_t *pos;
    const double *freq;
    const int32_t *axis;
    void *out;
    float *scale, *rowmax;
    int groups;              // threads of a head's row: each has four pairs, or eight elements that pass
    int turning;             // of these, those with pairs
    int each, hblocks;       // heads of a thread, and groups of them
};

// cosine and sine of four pairs of a token.  The turn n = pos freq / 2 pi is formed as an unevaluated sum of two float64
// (1 / 2 pi is one, and so is its product with freq), so that cutting it to [-1/2, 1/2] loses nothing at any position.
__device__ __forceinline__ void turns(const RopeArgs &a, int b, int64_t token, int p0, f4 &c, f4 &s) {
    constexpr double INV_HI = 0x1.45f306dc9c883p-3, INV_LO = -0x1.6b01ec5417056p-57;
    // (all loads before any use; what is not there is read where it does no harm and does not turn)
    int ax[4];
    double f[4];
    int32_t pos[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int p = min(p0 + j, a.d.pairs - 1);
        ax[j] = a.axis[p];
        f[j] = a.freq[p];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool there = (unsigned)ax[j] < (unsigned)a.d.axes;
        pos[j] = a.pos[(int64_t)b * a.d.stridePB + (int64_t)(there ? ax[j] : 0) * a.d.stridePA + token];
        if (!there) f[j] = 0.0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double x = (double)pos[j], step = f[j] * INV_HI, rest = fma(f[j], INV_HI, -step) + f[j] * INV_LO, whole = x * step;
        const double n = (whole - rint(whole)) + (fma(x, step, -whole) + x * rest);
        // (what rounding the half turns to float32 takes from the angle, up to pi 2^-25, is put back to first order: the square is
        // below 2^-46.  Beside a cosine or a sine near zero it would be many of its steps.)
        const double half_turns = 2.0 * n;
        const float near = (float)half_turns, rest_angle = (float)((half_turns - (double)near) * M_PI);
        float si, co;
        sincospif(near, &si, &co);
        c[j] = fmaf(-rest_angle, si, co);
        const float sine = fmaf(rest_angle, co, si);
        s[j] = a.d.inverse ? -sine : sine;
    }
}

// A head's eight elements of a thread, two quads, as they lie in memory.  R: words of a quad, 2 where the type has 16 bits, 4
// where it is float32.
template <int R, bool VEC, bool NEAR>
struct Eight {
    uint32_t w[2 * R];
    __device__ __forceinline__ void load(const void *p, int64_t at, int e0, int e1, int n0, int n1) {
        if (VEC && NEAR && R == 2 && n1 > 0) {      // the quads are neighbours: one 16-byte load
            const u4 x = *reinterpret_cast<const u4_8 *>(static_cast<const uint16_t *>(p) + at + e0);
#pragma unroll
            for (int j = 0; j < 2 * R; ++j) w[j] = x[j & 3];
            return;
        }
        const Raw4 a = load_raw<VEC>(R == 4 ? SC_F32 : SC_BF16, p, at + e0, n0), b = load_raw<VEC>(R == 4 ? SC_F32 : SC_BF16, p, at + e1, n1);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            w[j] = a.w[j];
            w[R + j] = b.w[j];
        }
    }
    __device__ __forceinline__ f4 quad(int type, int h) const {
        Raw4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[j] = w[h * R + (j < R ? j : 0)];
        return to_floats(R == 4 ? SC_F32 : type, r);
    }
};

// A thread has four pairs of a token (or eight elements that pass) and takes them through a.each heads with one set of cosines,
// HEADS of them at a time, the next ones' loads in flight.  Memory-bound (24960 x 24 x 128 in 16 bits: 61 us,
// 5.0 TB/s).  VEC: rows, pairs and halves on four elements.
// STREAM: stores that do not stay in the caches.
constexpr int HEADS = 4;
template <bool VEC, bool NEAR, int R, bool STREAM, bool INT8>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, uint32_t blocks, int shift) {
    const sc_rope_desc &d = a.d;
    if (block_id() >= blocks) return;
    const int G = 1 << shift, sub = threadIdx.x & (G - 1);
    const int64_t unit = ((int64_t)block_id() << (8 - shift)) + (threadIdx.x >> shift);
    const int64_t token = unit / a.hblocks;
    const int h0 = (int)(unit - token * a.hblocks) * a.each, h1 = min(h0 + a.each, d.heads);
    const bool live = token < d.tokens && sub < a.groups;
    const int P = d.pairs, p0 = 4 * sub, tail = 2 * P + 8 * (sub - a.turning);
    // the two quads of a thread: where they start and how many elements they have
    const bool turn = sub < a.turning;
    const int e0 = !turn ? tail : NEAR ? 2 * p0 : p0, e1 = !turn ? tail + 4 : NEAR ? 2 * p0 + 4 : P + p0;
    const int n0 = !live ? 0 : !turn ? min(d.D - e0, 4) : NEAR ? min(2 * P - e0, 4) : min(P - p0, 4);
    const int n1 = !live ? 0 : !turn ? min(d.D - e1, 4) : NEAR ? min(2 * P - e1, 4) : min(P - p0, 4);
    for (int b = blockIdx.z; b < d.batch; b += gridDim.z) {
        const int64_t from = (int64_t)b * d.strideXB + token * d.strideXT, to = (int64_t)b * d.strideOB + token * d.strideOT;
        Eight<R, VEC, NEAR> next[HEADS];
        const auto load = [&](int first) {
#pragma unroll
            for (int h = 0; h < HEADS; ++h)
                next[h].load(a.x, from + (int64_t)(first + h) * d.strideXH, e0, e1, first + h < h1 ? n0 : 0, first + h < h1 ? n1 : 0);
        };
        load(h0);
        f4 c = {1.0f, 1.0f, 1.0f, 1.0f}, s = {0.0f, 0.0f, 0.0f, 0.0f};
        if (live && turn) turns(a, b, token, p0, c, s);
        for (int first = h0; first < h1; first += HEADS) {
            Eight<R, VEC, NEAR> x[HEADS];
#pragma unroll
            for (int h = 0; h < HEADS; ++h) x[h] = next[h];
            load(first + HEADS);
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                const f4 u = x[h].quad(d.typeX, 0), v = x[h].quad(d.typeX, 1);
                f4 o0 = u, o1 = v;
                if (turn) {
                    if (NEAR) {
                        o0 = f4{u[0] * c[0] - u[1] * s[0], u[0] * s[0] + u[1] * c[0], u[2] * c[1] - u[3] * s[1], u[2] * s[1] + u[3] * c[1]};
                        o1 = f4{v[0] * c[2] - v[1] * s[2], v[0] * s[2] + v[1] * c[2], v[2] * c[3] - v[3] * s[3], v[2] * s[3] + v[3] * c[3]};
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            o0[j] = u[j] * c[j] - v[j] * s[j];
                            o1[j] = u[j] * s[j] + v[j] * c[j];
                        }
                    }
                }
                const int64_t at = to + (int64_t)(first + h) * d.strideOH;
                const int k0 = first + h < h1 ? n0 : 0, k1 = first + h < h1 ? n1 : 0;
                if (INT8) {
                    float m = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j < k0) m = fmaxf(m, fabsf(o0[j]));
                        if (j < k1) m = fmaxf(m, fabsf(o1[j]));
                    }
                    for (int o = G / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
                    const float sc = m / 127.0f;
                    if (live && sub == 0 && first + h < h1) {
                        const int64_t si = (int64_t)b * d.strideSB + token * d.strideST + (int64_t)(first + h) * d.strideSH;
                        a.scale[si] = sc;
                        if (a.rowmax) a.rowmax[si] = m;
                    }
                    store_bytes4<VEC>(a.out, at + e0, quant_int8x4(o0, sc), k0);
                    store_bytes4<VEC>(a.out, at + e1, quant_int8x4(o1, sc), k1);
                } else if (VEC && NEAR && d.typeO != SC_F32) {
                    if (k1 > 0) {
                        u4 w;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float lo = j < 2 ? o0[2 * (j & 1)] : o1[2 * (j & 1)], hi = j < 2 ? o0[2 * (j & 1) + 1] : o1[2 * (j & 1) + 1];
                            w[j] = to_pair(d.typeO, lo, hi);
                        }
                        u4_8 *q = reinterpret_cast<u4_8 *>(static_cast<uint16_t *>(a.out) + at + e0);
                        if (STREAM) __builtin_nontemporal_store(w, q);
                        else *q = w;
                    } else {
                        store4<VEC, STREAM>(d.typeO, a.out, at + e0, o0, k0);
                    }
                } else {
                    store4<VEC, STREAM>(d.typeO, a.out, at + e0, o0, k0);
                    store4<VEC, STREAM>(d.typeO, a.out, at + e1, o1, k1);
                }
            }
        }
    }
}

template <bool VEC, int R, bool STREAM, bool INT8>
static void launch_rope(const RopeArgs &a, bool near, dim3 grid, uint32_t blocks, int shift, hipStream_t st) {
    if (near) hipLaunchKernelGGL((k_rope<VEC, true, R, STREAM, INT8>), grid, dim3(256), 0, st, a, blocks, shift);
    else hipLaunchKernelGGL((k_rope<VEC, false, R, STREAM, INT8>), grid, dim3(256), 0, st, a, blocks, shift);
}
template <bool VEC, int R>
static void launch_rope(const RopeArgs &a, bool near, bool past, dim3 grid, uint32_t blocks, int shift, hipStream_t st) {
    if (a.d.typeO == SC_INT8) launch_rope<VEC, R, false, true>(a, near, grid, blocks, shift, st);
    else if (VEC && past) launch_rope<VEC, R, VEC, false>(a, near, grid, blocks, shift, st);
    else launch_rope<VEC, R, false, false>(a, near, grid, blocks, shift, st);
}

}  // namespace scl

using namespace scl;

extern "C" int sc_rope(const sc_rope_desc *desc, const void *x, const int32_t *pos, const double *freq, const int32_t *axis,
                       void *out, float *scale, float *rowmax, void *stream) {
    if (desc == nullptr) return SC_ERR_NULL;
    const sc_rope_desc &d = *desc;
    if (d.reserved[0] != 0 || d.reserved[1] != 0) return SC_ERR_RESERVED;
    if (d.batch < 0 || d.tokens < 0 || d.heads < 0 || d.D < 0 || d.D > SC_ROPE_D_LIMIT || d.pairs < 0 || 2 * (int64_t)d.pairs > d.D ||
        d.axes < 1 || d.axes > SC_ROPE_AXES_LIMIT || d.heads > 1 << 30)
        return SC_ERR_SHAPE;
    if (!is_float_type(d.typeX) || (!is_float_type(d.typeO) && d.typeO != SC_INT8)) return SC_ERR_TYPE;
    if ((d.pairing != SC_ROPE_HALVES && d.pairing != SC_ROPE_NEIGHBOURS) || (d.inverse != 0 && d.inverse != 1)) return SC_ERR_TYPE;
    const int64_t strides[] = {d.strideXB, d.strideXT, d.strideXH, d.strideOB, d.strideOT, d.strideOH,
                               d.strideSB, d.strideST, d.strideSH, d.stridePB, d.stridePA};
    for (int64_t s : strides)
        if (s < 0) return SC_ERR_STRIDE;
    if (d.batch == 0 || d.tokens == 0 || d.heads == 0 || (d.D == 0 && d.typeO != SC_INT8)) return SC_OK;
    if (!apart(d.batch, d.strideOB, d.tokens, d.strideOT, d.heads, d.strideOH, d.D)) return SC_ERR_STRIDE;
    if (d.typeO == SC_INT8 && !apart(d.batch, d.strideSB, d.tokens, d.strideST, d.heads, d.strideSH, 1)) return SC_ERR_STRIDE;
    if (d.D > 0 && (x == nullptr || out == nullptr)) return SC_ERR_NULL;
    if (d.pairs > 0 && (pos == nullptr || freq == nullptr || axis == nullptr)) return SC_ERR_NULL;
    if (d.typeO == SC_INT8 && scale == nullptr) return SC_ERR_NULL;
    if (d.typeO != SC_INT8 && rowmax != nullptr) return SC_ERR_TYPE;
    if (!aligned_to(x, type_bytes(d.typeX)) || !aligned_to(out, type_bytes(d.typeO)) || !aligned_to(pos, 4) || !aligned_to(freq, 8) ||
        !aligned_to(axis, 4) || !aligned_to(scale, 4) || !aligned_to(rowmax, 4))
        return SC_ERR_STRIDE;
    RopeArgs a{};
    a.d = d;
    a.x = x;
    a.pos = pos;
    a.freq = freq;
    a.axis = axis;
    a.out = out;
    a.scale = scale;
    a.rowmax = rowmax;
    a.turning = (d.pairs + 3) / 4;
    a.groups = a.turning + (d.D - 2 * d.pairs + 7) / 8;
    if (a.groups < 1) a.groups = 1;
    // (at most 33 groups, so a head's row lies in one wave, whose lanes take an int8 row's maximum)
    int shift = 0;
    while (1 << shift < a.groups) ++shift;
    // all heads by one thread, whose cosines are then computed once, where tokens are enough for every compute unit
    a.each = ((int64_t)d.tokens << shift) * (d.batch < 32768 ? d.batch : 32768) >= 256 * 512 ? (d.heads + HEADS - 1) / HEADS * HEADS : HEADS;
    a.hblocks = (int)(((int64_t)d.heads + a.each - 1) / a.each);
    const int64_t units = (int64_t)d.tokens * a.hblocks, blocks = (units + (256 >> shift) - 1) / (256 >> shift);
    if (blocks > INT32_MAX) return SC_ERR_SHAPE;
    const int64_t xb = 4 * type_bytes(d.typeX), ob = 4 * type_bytes(d.typeO);
    const bool vec = d.D % 4 == 0 && d.pairs % 4 == 0 && aligned_to(x, xb) && aligned_to(out, ob) &&
                     d.strideXB % 4 == 0 && d.strideXT % 4 == 0 && d.strideXH % 4 == 0 && d.strideOB % 4 == 0 &&
                     d.strideOT % 4 == 0 && d.strideOH % 4 == 0;
    const dim3 grid = grid_of((uint32_t)blocks, d.batch);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool near = d.pairing == SC_ROPE_NEIGHBOURS, wide = d.typeX == SC_F32;
    const uint32_t n = (uint32_t)blocks;
    // A result that the caches do not hold until it is read anyway (256 MB at most, half of them its source) is stored past them:
    // 24960 x 24 x 128 in 16 bits 74 -> 62 us.  One that they hold is not: 8192 x 8 x 256 in 32 bits takes 26 us either way, and
    // its reader finds it there.
    const bool stream_past = (int64_t)d.batch * d.tokens * d.heads * d.D * type_bytes(d.typeO) > (int64_t)128 << 20;
    if (vec && wide) launch_rope<true, 4>(a, near, stream_past, grid, n, shift, st);
    else if (vec) launch_rope<true, 2>(a, near, stream_past, grid, n, shift, st);
    else if (wide) launch_rope<false, 4>(a, near, stream_past, grid, n, shift, st);
    else launch_rope<false, 2>(a, near, stream_past, grid, n, shift, st);
    return hipGetLastError() == hipSuccess ? SC_OK : SC_ERR_HIP;
}
