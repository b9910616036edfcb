// Norms behind and before the branches of a transformer block with gate and residual, forward and backward.
#include <math.h>

#include "sc_layer.h"

namespace scl {

struct NormArgs {
    int batch, rows, D, post, pre, typeX, typeY, typeP, typeH;
    float eps_post, eps_pre, scale_res, off_post, off_pre;
    int64_t ldx, strideX, ldy, strideY, ldxo, strideXO, ldh, strideH, lds, strideS, lddxo, strideDXO, lddy, strideDY;
    int64_t s_post_w, s_post_b, s_gate, s_pre_w, s_pre_b;
    const void *x, *y, *post_w, *post_b, *gate, *pre_w, *pre_b;
    void *xo, *h;
    float *scale, *rowmax;
    // backward: x is the stored xo
    const void *dxo, *dh;
    void *dx, *dy;
    float *dpost_w, *dpost_b, *dgate, *dpre_w, *dpre_b;
    float *part;                 // [batch][chunks][NPART][D] partial sums
    int chunks;
};

// A block's threads: RPB rows side by side, W waves each; MOST waves where rows are shorter
template <int W, int MOST>
struct Waves {
    static constexpr int RPB = W >= MOST ? 1 : MOST / W, THREADS = 64 * W * RPB;
};

// Sums of N values over a row; every thread of the row gets them.  Rows of several waves meet in LDS, in one of two places
// by turns, so that one barrier is enough.
template <int W, int N, int RPB>
struct RowSums {
    static constexpr int SLOT = N * RPB * W;
    float *lds;
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N], int n) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < n) v[k] = lanes_sum<64>(v[k]);
        if (W > 1) {
            const int wave = threadIdx.x >> 6, first = wave / W * W;
            float *s = lds + turn * SLOT;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (k < n) s[wave * N + k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k >= n) continue;
                v[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) v[k] += s[(first + w) * N + k];
            }
        }
    }
};

// A row of a tensor for buffer instructions, whose bound drops what lies behind the row: loads of it give 0 and stores of it
// do nothing, so no lane branches.  The rows of a wave are the same in all of its lanes.  There is none where p is null.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer row_of(const void *p, int type, int b, int64_t stride, int64_t i, int64_t ld, int D, bool there = true) {
    const int es = type_bytes(type);
    return __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t *>(const_cast<void *>(p)) + (b * stride + i * ld) * es, 0,
                                             p != nullptr && there ? D * es : 0, 0x00020000);
}
// Its elements as they lie in memory, NV quads a thread: quad k of thread t is elements 4 (64 W k + t) .. + 3.  R: words of
// a quad, 2 where the type has 16 bits, 4 where it may be any.
template <int W, int NV, int R, bool VEC>
struct RawRow {
    uint32_t w[NV][R];
    __device__ __forceinline__ void load(int type, Buffer p, int t) {
        if (R == 4 && type == SC_F32) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = 16 * (64 * W * k + t);
                const u4 x = __builtin_amdgcn_raw_buffer_load_b128(p, at, 0, 0);
#pragma unroll
                for (int j = 0; j < R; ++j) w[k][j] = x[j];
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = 8 * (64 * W * k + t);
                const u2 x = __builtin_amdgcn_raw_buffer_load_b64(p, at, 0, 0);
                w[k][0] = x[0];
                w[k][1] = x[1];
            }
        }
    }
    // the same by address, with the lanes behind the row's end masked
    __device__ __forceinline__ void load(int type, const void *p, int64_t at, int t, int D) {
        if (R == 4 && type == SC_F32) {
            const uint32_t *q = static_cast<const uint32_t *>(p) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int d = 4 * (64 * W * k + t);
                if (VEC) {
                    u4 x = {0u, 0u, 0u, 0u};
                    if (d < D) x = *reinterpret_cast<const u4 *>(q + d);
#pragma unroll
                    for (int j = 0; j < R; ++j) w[k][j] = x[j];
                } else {
                    const Raw4 x = load_raw<false>(SC_F32, q, d, D - d);
#pragma unroll
                    for (int j = 0; j < R; ++j) w[k][j] = x.w[j];
                }
            }
        } else {
            const uint16_t *q = static_cast<const uint16_t *>(p) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int d = 4 * (64 * W * k + t);
                if (VEC) {
                    u2 x = {0u, 0u};
                    if (d < D) x = *reinterpret_cast<const u2 *>(q + d);
                    w[k][0] = x[0];
                    w[k][1] = x[1];
                } else {
                    const Raw4 x = load_raw<false>(SC_BF16, q, d, D - d);
                    w[k][0] = x.w[0];
                    w[k][1] = x.w[1];
                }
            }
        }
    }
    __device__ __forceinline__ void widen(int type, f4 (&v)[NV]) const {
        if (R == 4 && type == SC_F32) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][j] = __uint_as_float(w[k][j < R ? j : 0]);
        } else if (type == SC_BF16) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][j] = __uint_as_float(j & 1 ? w[k][j >> 1] & 0xffff0000u : w[k][j >> 1] << 16);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][j] = from_f16((w[k][j >> 1] >> (16 * (j & 1))) & 0xffffu);
        }
    }
};
// A parameter's row as it lies in memory, loaded ahead of its use
template <int W, int NV, int R, bool VEC>
struct Param {
    RawRow<W, NV, R, VEC> r;
    __device__ __forceinline__ void load(int type, const void *p, int64_t at, int t, int D) {
        if (p) r.load(type, p, at, t, D);
    }
    __device__ __forceinline__ void load_row(int type, const void *p, int b, int64_t stride, int t, int D) {
        if (!p) return;
        if (VEC) r.load(type, row_of(p, type, b, stride, 0, 0, D), t);
        else r.load(type, p, b * stride, t, D);
    }
    // plus `off`, or `none` where there is no parameter
    __device__ __forceinline__ void get(f4 (&v)[NV], int type, const void *p, float off, float none) const {
        if (p == nullptr) {
#pragma unroll
            for (int k = 0; k < NV; ++k) v[k] = f4{none, none, none, none};
            return;
        }
        r.widen(type, v);
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] += off;
    }
};
template <int W, int NV>
__device__ __forceinline__ void store_row(int type, Buffer p, int t, const f4 (&v)[NV]) {
    if (type == SC_F32) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = 16 * (64 * W * k + t);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, v[k]), p, at, 0, 0);
        }
    } else {
        u2 w[NV];
        if (type == SC_BF16) {
#pragma unroll
            for (int k = 0; k < NV; ++k) w[k] = u2{to_pair(SC_BF16, v[k][0], v[k][1]), to_pair(SC_BF16, v[k][2], v[k][3])};
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) w[k] = u2{to_pair(SC_F16, v[k][0], v[k][1]), to_pair(SC_F16, v[k][2], v[k][3])};
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = 8 * (64 * W * k + t);
            __builtin_amdgcn_raw_buffer_store_b64(w[k], p, at, 0, 0);
        }
    }
}
template <int W, int NV, bool VEC>
__device__ __forceinline__ void store_row(int type, void *p, int64_t at, int t, int D, const f4 (&v)[NV]) {
    if (type == SC_F32) {
#pragma unroll
        for (int k = 0; k < NV; ++k) store4<VEC>(SC_F32, p, at + 4 * (64 * W * k + t), v[k], D - 4 * (64 * W * k + t));
    } else if (type == SC_BF16) {
#pragma unroll
        for (int k = 0; k < NV; ++k) store4<VEC>(SC_BF16, p, at + 4 * (64 * W * k + t), v[k], D - 4 * (64 * W * k + t));
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) store4<VEC>(SC_F16, p, at + 4 * (64 * W * k + t), v[k], D - 4 * (64 * W * k + t));
    }
}
template <int NV>
__device__ __forceinline__ float sum(const f4 (&v)[NV]) {
    f4 s = v[0];
#pragma unroll
    for (int k = 1; k < NV; ++k) s += v[k];
    return (s[0] + s[1]) + (s[2] + s[3]);
}
template <int NV>
__device__ __forceinline__ float dot(const f4 (&u)[NV], const f4 (&v)[NV]) {
    f4 s = u[0] * v[0];
#pragma unroll
    for (int k = 1; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = fmaf(u[k][j], v[k][j], s[j]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}
// v - m where there are elements, 0 behind them
template <int W, int NV>
__device__ __forceinline__ void centre(f4 (&v)[NV], float m, int t, int D) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = 4 * (64 * W * k + t) + j < D ? v[k][j] - m : 0.0f;
}
__device__ __forceinline__ float inverse_deviation(float squares, float n_inv, float eps) { return rsqrtf(fmaf(squares, n_inv, eps)); }

// v normalised in place (elements past D become 0).  The mean is taken before the squares, which therefore lose
// nothing to it.
template <int W, int NV, typename Sums>
__device__ __forceinline__ void normalise(f4 (&v)[NV], int kind, float eps, float n_inv, int t, int D, Sums &sums) {
    if (kind == SC_NORM_LAYER) {
        float s[1] = {sum(v)};
        sums(s, 1);
        centre<W>(v, s[0] * n_inv, t, D);
    }
    float q[1] = {dot(v, v)};
    sums(q, 1);
    const float r = inverse_deviation(q[0], n_inv, eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] *= r;
}

// One row by W waves, held in registers from its loads to its stores: every operand is read once and every
// result written once.  Memory-bound (8192 x 1152, float32 stream, h in fp8: 32.4 us, 3.2 TB/s; 16384 x 1024 bfloat16: 26 us, 5.1 TB/s).
template <int W, int NV, int RX, int RY, bool VEC>
__global__ __launch_bounds__((Waves<W, 4>::THREADS)) void k_norm(NormArgs a) {
    constexpr int RPB = Waves<W, 4>::RPB;
    __shared__ float lds[2 * RPB * W];
    RowSums<W, 1, RPB> sums{lds};
    const int t = threadIdx.x % (64 * W), D = a.D;
    const float n_inv = 1.0f / (float)D;
    const int64_t row = (int64_t)block_id() * RPB + threadIdx.x / (64 * W);
    const bool live = row < a.rows;
    if (W == 1 && !live) return;          // (rows of several waves meet at barriers, so all of a block's stay)
    const int64_t i = min(row, (int64_t)a.rows - 1);
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        RawRow<W, NV, RX, VEC> rx;
        RawRow<W, NV, RY, VEC> ry;
        rx.load(a.typeX, a.x, (int64_t)b * a.strideX + i * a.ldx, t, D);
        if (a.y) ry.load(a.typeY, a.y, (int64_t)b * a.strideY + i * a.ldy, t, D);
        Param<W, NV, RY, VEC> gate, pre_w, pre_b;
        if (a.y) gate.load(a.typeP, a.gate, (int64_t)b * a.s_gate, t, D);
        pre_w.load(a.typeP, a.pre_w, (int64_t)b * a.s_pre_w, t, D);
        pre_b.load(a.typeP, a.pre_b, (int64_t)b * a.s_pre_b, t, D);
        f4 x[NV];
        rx.widen(a.typeX, x);
#pragma unroll
        for (int k = 0; k < NV; ++k) x[k] *= a.scale_res;
        if (a.y) {
            f4 u[NV], w[NV];
            ry.widen(a.typeY, u);
            if (a.post != SC_NORM_NONE) {
                Param<W, NV, RY, VEC> post_w, post_b;
                post_w.load(a.typeP, a.post_w, (int64_t)b * a.s_post_w, t, D);
                post_b.load(a.typeP, a.post_b, (int64_t)b * a.s_post_b, t, D);
                normalise<W>(u, a.post, a.eps_post, n_inv, t, D, sums);
                f4 c[NV];
                post_w.get(w, a.typeP, a.post_w, a.off_post, 1.0f);
                post_b.get(c, a.typeP, a.post_b, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < NV; ++k) u[k] = u[k] * w[k] + c[k];
            }
            gate.get(w, a.typeP, a.gate, 0.0f, 1.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k) x[k] += u[k] * w[k];
        }
        if (a.xo && live) store_row<W, NV, VEC>(a.typeX, a.xo, (int64_t)b * a.strideXO + i * a.ldxo, t, D, x);
        if (a.h == nullptr) continue;
        if (a.pre != SC_NORM_NONE) {
            normalise<W>(x, a.pre, a.eps_pre, n_inv, t, D, sums);
            f4 w[NV], c[NV];
            pre_w.get(w, a.typeP, a.pre_w, a.off_pre, 1.0f);
            pre_b.get(c, a.typeP, a.pre_b, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k) x[k] = x[k] * w[k] + c[k];
        }
        const int64_t ho = (int64_t)b * a.strideH + i * a.ldh;
        if (a.typeH == SC_INT8) {
            float m = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = 4 * (64 * W * k + t) + j < D ? fmaxf(m, fabsf(x[k][j])) : m;
            m = lanes_max<64>(m);
            if (W > 1) {
                __shared__ float most[RPB * W];
                const int wave = threadIdx.x >> 6, first = wave / W * W;
                __syncthreads();
                if ((threadIdx.x & 63) == 0) most[wave] = m;
                __syncthreads();
                for (int w = 0; w < W; ++w) m = fmaxf(m, most[first + w]);
            }
            if (!live) continue;
            const float s = m / 127.0f;
            if (t == 0) {
                a.scale[(int64_t)b * a.strideS + i] = s;
                if (a.rowmax) a.rowmax[(int64_t)b * a.strideS + i] = m;
            }
#pragma unroll
            for (int k = 0; k < NV; ++k)
                store_bytes4<VEC>(a.h, ho + 4 * (64 * W * k + t), quant_int8x4(x[k], s), D - 4 * (64 * W * k + t));
        } else if (a.typeH == SC_E4M3 || a.typeH == SC_E5M2) {
            // a block of 128 is the quads of 32 neighbouring lanes
            if (!live) continue;
            const bool e5 = a.typeH == SC_E5M2;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int d = 4 * (64 * W * k + t);
                float m = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) m = d + j < D ? fmaxf(m, fabsf(x[k][j])) : m;
                m = lanes_max<32>(m);
                const Fp8Scale s = fp8_scale(m, e5 ? E5M2_MAX : E4M3_MAX);
                if ((t & 31) == 0 && d < D) a.scale[(int64_t)b * a.strideS + i * a.lds + (d >> 7)] = s.s;
                store_bytes4<VEC>(a.h, ho + d, quant_fp8x4(e5, x[k], s.inv), D - d);
            }
        } else if (live) {
            store_row<W, NV, VEC>(a.typeH, a.h, ho, t, D, x);
        }
    }
}

// ----------------------------------------------------------------------------
// backward
// ----------------------------------------------------------------------------
enum { P_PRE_W, P_PRE_B, P_GATE, P_POST_W, P_POST_B, NPART };

// A block takes a run of a batch entry's rows, RPB side by side, and sums its rows' shares of the parameters' gradients in
// registers; the blocks' sums go to memory and k_norm_sums adds them in a fixed order.  The next row is loaded while one is
// worked on.  With n the normalised row, r = 1 / deviation and d the gradient behind the norm times its weight, the
// gradient before it is r (d - n mean(d n)), LayerNorm also - mean(d); both means and the deviation come from one round of
// sums.  POST: a norm behind the branch.  Bound by memory and the rows' barriers (8192 x 1152, float32 stream: 53.6 us with the sums,
// 3.2 TB/s; 4099 x 4096 bfloat16 with POST: 57.7, 3.5 TB/s; 16384 x 1024 bfloat16: 41, 4.9 TB/s).
// A block's waves: eight, a block to a compute unit; rows of 1025 to 2048 elements two blocks of four, which wait for fewer
// waves at their barriers (8192 x 1152, float32 stream: 56.7 -> 53.5 us; 4096 x 2048 52.3 -> 49.6).  Shorter ones do not gain
// what the additional partial sums cost (16384 x 1024: 41.4 -> 42.4).
template <int W, int NV> constexpr int BACK_WAVES = W <= 4 && W * NV > 4 ? 4 : 8;
template <int W, int NV, int RX, int RY, bool VEC, bool POST>
__global__ __launch_bounds__((Waves<W, BACK_WAVES<W, NV>>::THREADS), W <= 8 ? 2 : 4) void k_norm_back(NormArgs a) {
    constexpr int RPB = Waves<W, BACK_WAVES<W, NV>>::RPB, NP = POST ? 5 : 3, NS = 4;
    __shared__ float lds[2 * NS * RPB * W];
    __shared__ f4 join[RPB > 1 ? RPB : 1][RPB > 1 ? NP * NV : 1][64 * W];
    RowSums<W, NS, RPB> sums{lds};
    const int t = threadIdx.x % (64 * W), side = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W)), D = a.D;
    const int64_t chunk = block_id();
    if (chunk >= a.chunks) return;
    const int64_t i0 = chunk * a.rows / a.chunks, i1 = (chunk + 1) * a.rows / a.chunks;
    const float n_inv = 1.0f / (float)D;
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        f4 acc[NP][NV];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int k = 0; k < NV; ++k) acc[p][k] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        RawRow<W, NV, RX, VEC> rx, rg;
        RawRow<W, NV, RY, VEC> ry, rh;
        // (a row that is not there is one of zeros)
        const auto fetch = [&](int64_t i) {
            const bool live = i < i1;
            const auto get = [&](auto &r, int type, const void *p, int64_t stride, int64_t ld) {
                if (VEC) r.load(type, row_of(p, type, b, stride, i, ld, D, live), t);
                else r.load(type, p, b * stride + i * ld, t, p != nullptr && live ? D : 0);
            };
            get(rx, a.typeX, a.x, a.strideXO, a.ldxo);
            get(rh, a.typeH, a.dh, a.strideH, a.ldh);
            get(ry, a.typeY, a.y, a.strideY, a.ldy);
            get(rg, a.typeX, a.dxo, a.strideDXO, a.lddxo);
        };
        const auto put_row = [&](int type, void *p, int64_t stride, int64_t i, int64_t ld, const f4 (&v)[NV]) {
            if (VEC) store_row<W, NV>(type, row_of(p, type, b, stride, i, ld, D, i < i1), t, v);
            else store_row<W, NV, false>(type, p, b * stride + i * ld, t, i < i1 ? D : 0, v);
        };
        fetch(i0 + side);
        // (the parameters are the same for all of the rows)
        Param<W, NV, RY, VEC> pre_w, gate, post_w, post_b;
        pre_w.load_row(a.typeP, a.pre_w, b, a.s_pre_w, t, D);
        if (a.y || a.dy) gate.load_row(a.typeP, a.gate, b, a.s_gate, t, D);
        if (POST) {
            post_w.load_row(a.typeP, a.post_w, b, a.s_post_w, t, D);
            post_b.load_row(a.typeP, a.post_b, b, a.s_post_b, t, D);
        }
        for (int64_t first = i0; first < i1; first += RPB) {
            const int64_t i = first + side;
            const bool live = i < i1;               // (a row behind the last takes part in barriers and counts nothing)
            if (W == 1 && !live) break;
            f4 n[NV], g[NV], e[NV], m[NV];
            rx.widen(a.typeX, n);
            rh.widen(a.typeH, g);
            ry.widen(a.typeY, m);
            rg.widen(a.typeX, e);
            fetch(i + RPB);
            const bool pre = a.pre != SC_NORM_NONE && a.dh, pre_mean = pre && a.pre == SC_NORM_LAYER,
                       post_mean = POST && a.post == SC_NORM_LAYER;
            if (pre_mean || post_mean) {
                float s[NS] = {pre ? sum(n) : 0.0f, POST ? sum(m) : 0.0f, 0.0f, 0.0f};
                sums(s, 2);
                if (pre_mean) centre<W>(n, s[0] * n_inv, t, D);
                if (post_mean) centre<W>(m, s[1] * n_inv, t, D);
            }
            float r_post = 1.0f;
            if (pre || POST) {
                f4 d[NV];
                float s[NS] = {0.0f, 0.0f, 0.0f, POST ? dot(m, m) : 0.0f};
                if (pre) {
                    pre_w.get(d, a.typeP, a.pre_w, a.off_pre, 1.0f);
#pragma unroll
                    for (int k = 0; k < NV; ++k) d[k] *= g[k];
                    s[0] = dot(n, n);
                    s[1] = dot(d, n);
                    s[2] = sum(d);
                }
                sums(s, NS);
                if (POST) r_post = inverse_deviation(s[3], n_inv, a.eps_post);
                if (pre) {
                    const float r = inverse_deviation(s[0], n_inv, a.eps_pre), dn = s[1] * r * n_inv,
                                dm = pre_mean ? s[2] * n_inv : 0.0f;
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float nr = n[k][j] * r;
                            acc[P_PRE_W][k][j] = fmaf(g[k][j], nr, acc[P_PRE_W][k][j]);
                            acc[P_PRE_B][k][j] += g[k][j];
                            g[k][j] = fmaf(r, d[k][j] - dm - nr * dn, e[k][j]);
                        }
                }
            }
            if (!pre)
#pragma unroll
                for (int k = 0; k < NV; ++k) g[k] += e[k];
            if (a.dx) {
#pragma unroll
                for (int k = 0; k < NV; ++k) e[k] = a.scale_res * g[k];
                put_row(a.typeX, a.dx, a.strideX, i, a.ldx, e);
            }
            if (a.y == nullptr && a.dy == nullptr) continue;
            gate.get(e, a.typeP, a.gate, 0.0f, 1.0f);
            if (POST) {
                f4 pw[NV], c[NV];
                post_w.get(pw, a.typeP, a.post_w, a.off_post, 1.0f);
                post_b.get(c, a.typeP, a.post_b, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int left = D - 4 * (64 * W * k + t);       // (elements of the row from this quad on)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float nr = m[k][j] * r_post, du = g[k][j] * e[k][j];
                        m[k][j] = nr;
                        acc[P_GATE][k][j] = fmaf(g[k][j], fmaf(nr, pw[k][j], c[k][j]), acc[P_GATE][k][j]);
                        acc[NP - 2][k][j] = fmaf(du, nr, acc[NP - 2][k][j]);
                        acc[NP - 1][k][j] += du;
                        // (behind the row a LayerNorm's gradient above is - r mean(d), not 0, and must not enter the sums below)
                        g[k][j] = (VEC ? left > 0 : j < left) ? du * pw[k][j] : 0.0f;
                    }
                }
                if (a.dy) {
                    float s[NS] = {dot(g, m), sum(g), 0.0f, 0.0f};
                    sums(s, 2);
                    const float dn = s[0] * n_inv, dm = post_mean ? s[1] * n_inv : 0.0f;
#pragma unroll
                    for (int k = 0; k < NV; ++k) g[k] = r_post * (g[k] - dm - m[k] * dn);
                }
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[P_GATE][k][j] = fmaf(g[k][j], m[k][j], acc[P_GATE][k][j]);
                        g[k][j] *= e[k][j];
                    }
            }
            if (a.dy) put_row(a.typeY, a.dy, a.strideDY, i, a.lddy, g);
        }
        if (a.part == nullptr) continue;
        // The rows side by side join their sums in LDS, each side the ones of every RPB-th quad
        float *part = a.part + ((int64_t)b * a.chunks + chunk) * NPART * D;
        const auto put = [&](int p, int k, f4 v) {
            const bool wanted = p == P_PRE_W ? a.dpre_w != nullptr : p == P_PRE_B ? a.dpre_b != nullptr : p == P_GATE ? a.dgate != nullptr
                              : p == P_POST_W ? a.dpost_w != nullptr : a.dpost_b != nullptr;
            const int d = 4 * (64 * W * k + t);
            if (wanted) store4<VEC>(SC_F32, part, (int64_t)p * D + d, v, D - d);
        };
        if (RPB == 1) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int k = 0; k < NV; ++k) put(p, k, acc[p][k]);
        } else {
            __syncthreads();                        // (the last batch entry's have been read)
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int k = 0; k < NV; ++k) join[side][p * NV + k][t] = acc[p][k];
            __syncthreads();
            for (int x = side; x < NP * NV; x += RPB) {
                f4 v = join[0][x][t];
#pragma unroll
                for (int o = 1; o < RPB; ++o) v += join[o][x][t];
                put(x / NV, x % NV, v);
            }
        }
    }
}

// Sums over the chunks, and over the batch where a parameter is shared: COLS columns by GROUPS groups of chunks, whose
// sums are joined in order (4 us for the sums of 8192 x 1152)
template <int COLS, int GROUPS>
__global__ __launch_bounds__(COLS * GROUPS) void k_norm_sums(NormArgs a) {
    __shared__ float join[GROUPS][COLS];
    const int c = threadIdx.x % COLS, grp = threadIdx.x / COLS, d = blockIdx.x * COLS + c, p = blockIdx.y;
    float *out = p == P_PRE_W ? a.dpre_w : p == P_PRE_B ? a.dpre_b : p == P_GATE ? a.dgate : p == P_POST_W ? a.dpost_w : a.dpost_b;
    const int64_t stride = p == P_PRE_W ? a.s_pre_w : p == P_PRE_B ? a.s_pre_b : p == P_GATE ? a.s_gate : p == P_POST_W ? a.s_post_w : a.s_post_b;
    if (out == nullptr) return;
    const int64_t entries = stride == 0 ? 1 : a.batch, n = stride == 0 ? (int64_t)a.batch * a.chunks : a.chunks;
    for (int64_t b = blockIdx.z; b < entries; b += gridDim.z) {
        const float *q = a.part + ((int64_t)b * a.chunks * NPART + p) * a.D + d;
        float s = 0.0f;
        if (d < a.D)
#pragma unroll 8
            for (int64_t k = grp; k < n; k += GROUPS) s += q[k * NPART * a.D];
        __syncthreads();
        join[grp][c] = s;
        __syncthreads();
        if (grp == 0 && d < a.D) {
            s = 0.0f;
            for (int k = 0; k < GROUPS; ++k) s += join[k][c];
            out[b * a.D + d] = s;      // (b = 0 where shared)
        }
    }
}

// ----------------------------------------------------------------------------
// host
// ----------------------------------------------------------------------------
enum { ODD, ANY_ANY, ANY_16, ALL_16 };     // rows that do not lie on four elements; else types of the residual stream, and of the rest

template <int W, int NV, int RX, int RY, bool VEC>
static void launch_forward(const NormArgs &a, hipStream_t st) {
    const uint32_t blocks = (uint32_t)(((int64_t)a.rows + Waves<W, 4>::RPB - 1) / Waves<W, 4>::RPB);
    hipLaunchKernelGGL((k_norm<W, NV, RX, RY, VEC>), grid_of(blocks, a.batch), dim3(Waves<W, 4>::THREADS), 0, st, a);
}
template <int W, int NV, int RX, int RY, bool VEC>
static void launch_backward(const NormArgs &a, hipStream_t st) {
    const dim3 grid = grid_of((uint32_t)a.chunks, a.batch), block(Waves<W, BACK_WAVES<W, NV>>::THREADS);
    if (a.post != SC_NORM_NONE) hipLaunchKernelGGL((k_norm_back<W, NV, RX, RY, VEC, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_norm_back<W, NV, RX, RY, VEC, false>), grid, block, 0, st, a);
}
template <int W, int NV>
static void forward_of(const NormArgs &a, int types, hipStream_t st) {
    if (types == ALL_16) launch_forward<W, NV, 2, 2, true>(a, st);
    else if (types == ANY_16) launch_forward<W, NV, 4, 2, true>(a, st);
    else if (types == ANY_ANY) launch_forward<W, NV, 4, 4, true>(a, st);
    else launch_forward<W, NV, 4, 4, false>(a, st);
}
template <int W, int NV>
static void backward_of(const NormArgs &a, int types, hipStream_t st) {
    if (types == ALL_16) launch_backward<W, NV, 2, 2, true>(a, st);
    else if (types == ANY_16) launch_backward<W, NV, 4, 2, true>(a, st);
    else if (types == ANY_ANY) launch_backward<W, NV, 4, 4, true>(a, st);
    else launch_backward<W, NV, 4, 4, false>(a, st);
}
// The fewest waves that hold a row in two quads a thread (three just below a power of two's half); gradients of more than 4096
// elements in four, since sixteen waves have 128 registers each (1024 x 8192 with both norms: 197 us, and 72 by eight).
// Scratch, in bytes a lane as the compiler reports it: none where everything but x has 16 bits and x too, up to 8192 elements forward,
// and from 1537 to 4096 backward (to 8192 without a norm behind the branch).  Elsewhere it is 12 (float32 x) or 60 (float32 parameters,
// rows off four elements) forward, where the words of a row are filled in one of two ways by the type at run time; 0 to 364 backward
// up to 1536 elements, 0 to 128 up to 4096.  Registers spill in gradients of 1025 to 1536 elements with a norm behind the branch and
// a float32 operand or rows off four elements (11 to 182), of 4097 to 8192 with such a norm (140 to 428) or such an operand or rows (21 to 173),
// and in both directions past 8192.
static hipError_t launch_rows(const NormArgs &a, bool back, bool vec, hipStream_t st) {
    const bool x16 = a.typeX != SC_F32, rest16 = (a.y == nullptr || a.typeY != SC_F32) && a.typeP != SC_F32 && (!back || a.dh == nullptr || a.typeH != SC_F32);
    const int types = !vec ? ODD : x16 && rest16 ? ALL_16 : rest16 ? ANY_16 : ANY_ANY, D = a.D;
    if (back) {
        if (D <= 512) backward_of<1, 2>(a, types, st);
        else if (D <= 1024) backward_of<2, 2>(a, types, st);
        else if (D <= 1536) backward_of<2, 3>(a, types, st);
        else if (D <= 2048) backward_of<4, 2>(a, types, st);
        else if (D <= 4096) backward_of<8, 2>(a, types, st);
        else if (D <= 8192) backward_of<8, 4>(a, types, st);
        else backward_of<16, 4>(a, types, st);
    } else {
        if (D <= 512) forward_of<1, 2>(a, types, st);
        else if (D <= 768) forward_of<1, 3>(a, types, st);
        else if (D <= 1024) forward_of<2, 2>(a, types, st);
        else if (D <= 1536) forward_of<2, 3>(a, types, st);
        else if (D <= 2048) forward_of<4, 2>(a, types, st);
        else if (D <= 4096) forward_of<8, 2>(a, types, st);
        else if (D <= 8192) forward_of<16, 2>(a, types, st);
        else forward_of<16, 4>(a, types, st);
    }
    return hipGetLastError();
}

// Runs of rows whose sums go to memory: as many as there are blocks of eight waves, or of four (BACK_WAVES), at a time
static int chunks_of(const sc_norm_desc &d) {
    const int all = d.D > 1024 && d.D <= 2048 ? 512 : 256, want = d.batch < 1 ? 1 : d.batch < all ? (all + d.batch - 1) / d.batch : 1;
    return d.rows < want ? d.rows : want;
}

static int check_norm(const sc_norm_desc *d) {
    if (d == nullptr) return SC_ERR_NULL;
    if (d->reserved != 0) return SC_ERR_RESERVED;
    if (d->batch < 0 || d->rows < 0 || d->D < 0 || d->D > SC_NORM_D_LIMIT) return SC_ERR_SHAPE;
    if (d->post < SC_NORM_NONE || d->post > SC_NORM_LAYER || d->pre < SC_NORM_NONE || d->pre > SC_NORM_LAYER) return SC_ERR_TYPE;
    if (!is_float_type(d->typeX) || !is_float_type(d->typeY) || !is_float_type(d->typeP)) return SC_ERR_TYPE;
    if (d->typeH < SC_F32 || d->typeH > SC_INT8) return SC_ERR_TYPE;
    if (!(d->eps_post > 0.0f) || !(d->eps_pre > 0.0f)) return SC_ERR_SHAPE;
    const int64_t D = d->D, strides[] = {d->strideX, d->strideY, d->strideXO, d->strideH, d->strideS, d->lds, d->lddxo, d->strideDXO, d->lddy, d->strideDY,
                                         d->stride_post_w, d->stride_post_b, d->stride_gate, d->stride_pre_w, d->stride_pre_b};
    for (int64_t s : strides)
        if (s < 0) return SC_ERR_STRIDE;
    if (d->ldx < D || d->ldy < D || d->ldxo < D || d->ldh < D) return SC_ERR_STRIDE;
    if (is_fp8_type(d->typeH) && d->lds < (D + FP8_BLOCK - 1) / FP8_BLOCK) return SC_ERR_STRIDE;
    return SC_OK;
}
// rows of something written must not lie on top of each other
static bool entries_apart(const sc_norm_desc &d, int64_t ld, int64_t stride) {
    return rows_apart(d.batch, stride, d.rows, ld, d.D);
}
static bool quads(const void *p, int type, int64_t ld, int64_t stride) {
    const int64_t b = type_bytes(type);
    return p == nullptr || (aligned_to(p, 4 * b) && ld % 4 == 0 && stride % 4 == 0);
}
static NormArgs norm_args(const sc_norm_desc &d) {
    NormArgs a{};
    a.batch = d.batch;
    a.rows = d.rows;
    a.D = d.D;
    a.post = d.post;
    a.pre = d.pre;
    a.typeX = d.typeX;
    a.typeY = d.typeY;
    a.typeP = d.typeP;
    a.typeH = d.typeH;
    a.eps_post = d.eps_post;
    a.eps_pre = d.eps_pre;
    a.scale_res = d.scale_res;
    a.off_post = d.off_post;
    a.off_pre = d.off_pre;
    a.ldx = d.ldx;
    a.strideX = d.strideX;
    a.ldy = d.ldy;
    a.strideY = d.strideY;
    a.ldxo = d.ldxo;
    a.strideXO = d.strideXO;
    a.ldh = d.ldh;
    a.strideH = d.strideH;
    a.lds = d.lds;
    a.strideS = d.strideS;
    a.lddxo = d.lddxo;
    a.strideDXO = d.strideDXO;
    a.lddy = d.lddy;
    a.strideDY = d.strideDY;
    a.s_post_w = d.stride_post_w;
    a.s_post_b = d.stride_post_b;
    a.s_gate = d.stride_gate;
    a.s_pre_w = d.stride_pre_w;
    a.s_pre_b = d.stride_pre_b;
    return a;
}
static bool params_aligned(const sc_norm_desc &d, const void *const (&p)[5]) {
    for (const void *q : p)
        if (!aligned_to(q, type_bytes(d.typeP))) return false;
    return true;
}
static bool params_quads(const sc_norm_desc &d, const void *const (&p)[5]) {
    const int64_t s[5] = {d.stride_post_w, d.stride_post_b, d.stride_gate, d.stride_pre_w, d.stride_pre_b};
    for (int k = 0; k < 5; ++k)
        if (!quads(p[k], d.typeP, 0, s[k])) return false;
    return true;
}

}  // namespace scl

using namespace scl;

extern "C" {

int sc_residual_norm(const sc_norm_desc *desc, const void *x, const void *y, const void *post_w, const void *post_b,
                     const void *gate, const void *pre_w, const void *pre_b, void *xo, void *h, float *scale,
                     float *rowmax, void *stream) {
    const int rc = check_norm(desc);
    if (rc != SC_OK) return rc;
    const sc_norm_desc &d = *desc;
    if ((xo != nullptr && !entries_apart(d, d.ldxo, d.strideXO)) || (h != nullptr && !entries_apart(d, d.ldh, d.strideH)))
        return SC_ERR_STRIDE;
    const bool quantised = !is_float_type(d.typeH);
    const int64_t srow = is_fp8_type(d.typeH) ? d.lds : 1, slen = is_fp8_type(d.typeH) ? (d.D + FP8_BLOCK - 1) / FP8_BLOCK : 1;
    if (h != nullptr && quantised && !rows_apart(d.batch, d.strideS, d.rows, srow, slen)) return SC_ERR_STRIDE;
    if (d.batch == 0 || d.rows == 0 || (d.D == 0 && d.typeH != SC_INT8)) return SC_OK;
    if (xo == nullptr && h == nullptr) return SC_OK;
    if (d.D > 0 && x == nullptr) return SC_ERR_NULL;
    if (h != nullptr && quantised && scale == nullptr) return SC_ERR_NULL;
    if (rowmax != nullptr && h != nullptr && d.typeH != SC_INT8) return SC_ERR_TYPE;
    // (parameters of a norm that is not there are refused, not passed over)
    if ((d.post == SC_NORM_NONE || y == nullptr) && (post_w != nullptr || post_b != nullptr)) return SC_ERR_TYPE;
    if (y == nullptr && (gate != nullptr || d.post != SC_NORM_NONE)) return SC_ERR_TYPE;
    if (d.pre == SC_NORM_NONE && (pre_w != nullptr || pre_b != nullptr)) return SC_ERR_TYPE;
    const void *const params[5] = {post_w, post_b, gate, pre_w, pre_b};
    if (!aligned_to(x, type_bytes(d.typeX)) || !aligned_to(y, type_bytes(d.typeY)) || !aligned_to(xo, type_bytes(d.typeX)) ||
        !aligned_to(h, type_bytes(d.typeH)) || !aligned_to(scale, 4) || !aligned_to(rowmax, 4) || !params_aligned(d, params))
        return SC_ERR_STRIDE;
    NormArgs a = norm_args(d);
    a.x = x;
    a.y = y;
    a.post_w = post_w;
    a.post_b = post_b;
    a.gate = gate;
    a.pre_w = pre_w;
    a.pre_b = pre_b;
    a.xo = xo;
    a.h = h;
    a.scale = scale;
    a.rowmax = rowmax;
    // four elements at a time where every row starts on four
    const bool vec = d.D % 4 == 0 && quads(x, d.typeX, d.ldx, d.strideX) && quads(y, d.typeY, d.ldy, d.strideY) &&
                     quads(xo, d.typeX, d.ldxo, d.strideXO) && quads(h, d.typeH, d.ldh, d.strideH) && params_quads(d, params);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return launch_rows(a, false, vec, st) == hipSuccess ? SC_OK : SC_ERR_HIP;
}

int sc_residual_norm_backward_workspace_size(const sc_norm_desc *desc, size_t *bytes) {
    if (bytes == nullptr) return SC_ERR_NULL;
    const int rc = check_norm(desc);
    if (rc != SC_OK) return rc;
    if (!is_float_type(desc->typeH)) return SC_ERR_TYPE;
    *bytes = (size_t)desc->batch * chunks_of(*desc) * NPART * desc->D * sizeof(float);
    return SC_OK;
}

int sc_residual_norm_backward(const sc_norm_desc *desc, const void *xo, const void *y, const void *post_w,
                              const void *post_b, const void *gate, const void *pre_w, const void *dxo, const void *dh,
                              void *dx, void *dy, float *dpost_w, float *dpost_b, float *dgate, float *dpre_w,
                              float *dpre_b, void *workspace, size_t workspace_bytes, void *stream) {
    size_t need = 0;
    const int rc = sc_residual_norm_backward_workspace_size(desc, &need);
    if (rc != SC_OK) return rc;
    const sc_norm_desc &d = *desc;
    const int64_t D = d.D;
    if ((dxo != nullptr && d.lddxo < D) || (dy != nullptr && d.lddy < D)) return SC_ERR_STRIDE;
    if ((dx != nullptr && !entries_apart(d, d.ldx, d.strideX)) || (dy != nullptr && !entries_apart(d, d.lddy, d.strideDY)))
        return SC_ERR_STRIDE;
    const float *const sums[5] = {dpost_w, dpost_b, dgate, dpre_w, dpre_b};
    bool any = false;
    for (const float *s : sums) any = any || s != nullptr;
    if (d.D == 0 || (!any && dx == nullptr && dy == nullptr)) return SC_OK;
    if (d.pre == SC_NORM_NONE && (pre_w != nullptr || dpre_w != nullptr || dpre_b != nullptr)) return SC_ERR_TYPE;
    if (d.post == SC_NORM_NONE && (post_w != nullptr || post_b != nullptr || dpost_w != nullptr || dpost_b != nullptr)) return SC_ERR_TYPE;
    const bool rows = d.batch > 0 && d.rows > 0;
    if (rows && d.pre != SC_NORM_NONE && xo == nullptr) return SC_ERR_NULL;
    if (rows && y == nullptr && (dgate != nullptr || (d.post != SC_NORM_NONE && (dy != nullptr || dpost_w != nullptr || dpost_b != nullptr))))
        return SC_ERR_NULL;
    if (rows && any && (workspace == nullptr || workspace_bytes < need || !aligned_to(workspace, 256))) return SC_ERR_WORKSPACE;
    const void *const params[5] = {post_w, post_b, gate, pre_w, nullptr};
    if (!aligned_to(xo, type_bytes(d.typeX)) || !aligned_to(dxo, type_bytes(d.typeX)) || !aligned_to(dx, type_bytes(d.typeX)) ||
        !aligned_to(y, type_bytes(d.typeY)) || !aligned_to(dy, type_bytes(d.typeY)) || !aligned_to(dh, type_bytes(d.typeH)) ||
        !params_aligned(d, params))
        return SC_ERR_STRIDE;
    for (const float *s : sums)
        if (!aligned_to(s, 4)) return SC_ERR_STRIDE;
    NormArgs a = norm_args(d);
    a.x = xo;
    a.y = dy != nullptr || dgate != nullptr || dpost_w != nullptr || dpost_b != nullptr ? y : nullptr;
    a.post_w = post_w;
    a.post_b = post_b;
    a.gate = gate;
    a.pre_w = pre_w;
    a.dxo = dxo;
    a.dh = dh;
    a.dx = dx;
    a.dy = dy;
    a.dpost_w = dpost_w;
    a.dpost_b = dpost_b;
    a.dgate = dgate;
    a.dpre_w = dpre_w;
    a.dpre_b = dpre_b;
    a.part = any ? static_cast<float *>(workspace) : nullptr;
    a.chunks = chunks_of(d);
    const bool vec = d.D % 4 == 0 && quads(xo, d.typeX, d.ldxo, d.strideXO) && quads(y, d.typeY, d.ldy, d.strideY) &&
                     quads(dxo, d.typeX, d.lddxo, d.strideDXO) && quads(dh, d.typeH, d.ldh, d.strideH) &&
                     quads(dx, d.typeX, d.ldx, d.strideX) && quads(dy, d.typeY, d.lddy, d.strideDY) && params_quads(d, params);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (rows && launch_rows(a, true, vec, st) != hipSuccess) return SC_ERR_HIP;
    // (without rows the sums are zeros)
    if (any) {
        const unsigned entries = d.batch < 1 ? 1 : d.batch < 32768 ? d.batch : 32768;
        // (few chunks and many entries: a thread a column; else 32 groups)
        if (a.chunks <= 32 && d.batch >= 8 && a.s_gate && a.s_pre_w)
            hipLaunchKernelGGL((k_norm_sums<64, 4>), dim3((unsigned)((d.D + 63) / 64), NPART, entries), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((k_norm_sums<32, 32>), dim3((unsigned)((d.D + 31) / 32), NPART, entries), dim3(1024), 0, st, a);
        if (hipGetLastError() != hipSuccess) return SC_ERR_HIP;
    }
    return SC_OK;
}

}  // extern "C"
