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
    int chunks, chunk_rows;
};

// Sums of N values over a row, which W waves share; every thread gets them
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *lds) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<64>(v[k]);
    if (W > 1) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) lds[k * W + wave] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0f;
            for (int w = 0; w < W; ++w) v[k] += lds[k * W + w];
        }
    }
}
template <int W>
__device__ __forceinline__ float row_max(float v, float *lds) {
    v = lanes_max<64>(v);
    if (W > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int w = 0; w < W; ++w) v = fmaxf(v, lds[w]);
    }
    return v;
}

// A row of D elements by W waves, NV quads a thread: element 4 (64 W k + t) + j is thread t's
template <int W, int NV>
struct Row {
    f4 v[NV];
};
template <int W, int NV, bool VEC>
__device__ __forceinline__ void load_row(Raw4 (&r)[NV], int type, const void *p, int64_t at, int t, int D) {
    if (type == SC_F32) {
#pragma unroll
        for (int k = 0; k < NV; ++k) r[k] = load_raw<VEC>(SC_F32, p, at + 4 * (64 * W * k + t), D - 4 * (64 * W * k + t));
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) r[k] = load_raw<VEC>(SC_BF16, p, at + 4 * (64 * W * k + t), D - 4 * (64 * W * k + t));
    }
}
template <int NV>
__device__ __forceinline__ void widen(f4 (&v)[NV], int type, const Raw4 (&r)[NV]) {
    if (type == SC_F32) {
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = to_floats(SC_F32, r[k]);
    } else if (type == SC_BF16) {
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = to_floats(SC_BF16, r[k]);
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = to_floats(SC_F16, r[k]);
    }
}
template <int W, int NV, bool VEC>
__device__ __forceinline__ void load_param(f4 (&v)[NV], int type, const void *p, int64_t at, int t, int D, float off, float none) {
    if (p == nullptr) {
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = f4{none, none, none, none};
        return;
    }
    Raw4 r[NV];
    load_row<W, NV, VEC>(r, type, p, at, t, D);
    widen(v, type, r);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] += off;
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

// v normalised in place (elements past D become 0); returns 1 / deviation.  The mean is taken before the squares,
// which therefore lose nothing to it.
template <int W, int NV>
__device__ __forceinline__ float normalise(f4 (&v)[NV], int kind, float eps, int t, int D, float *lds) {
    if (kind == SC_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k) s[0] += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
        row_sums<W, 1>(s, lds);
        const float mean = s[0] / (float)D;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k][j] = 4 * (64 * W * k + t) + j < D ? v[k][j] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) q[0] += (v[k][0] * v[k][0] + v[k][1] * v[k][1]) + (v[k][2] * v[k][2] + v[k][3] * v[k][3]);
    row_sums<W, 1>(q, lds);
    const float r = 1.0f / sqrtf(q[0] / (float)D + eps);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] *= r;
    return r;
}

// One row by W waves, held in registers from its loads to its stores: every operand is read once and every
// result written once.  Memory-bound.
template <int W, int NV, bool VEC>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(NormArgs a) {
    constexpr int RPB = W == 1 ? 4 : 1;           // rows of a block
    __shared__ float lds[W];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t i = (int64_t)block_id() * RPB + (W == 1 ? threadIdx.x >> 6 : 0);
    if (i >= a.rows) return;
    const int D = a.D;
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        Raw4 rx[NV], ry[NV];
        load_row<W, NV, VEC>(rx, a.typeX, a.x, (int64_t)b * a.strideX + i * a.ldx, t, D);
        if (a.y) load_row<W, NV, VEC>(ry, a.typeY, a.y, (int64_t)b * a.strideY + i * a.ldy, t, D);
        f4 x[NV];
        widen(x, a.typeX, rx);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[k][j] *= a.scale_res;
        if (a.y) {
            f4 u[NV], w[NV];
            widen(u, a.typeY, ry);
            if (a.post != SC_NORM_NONE) {
                normalise<W, NV>(u, a.post, a.eps_post, t, D, lds);
                f4 c[NV];
                load_param<W, NV, VEC>(w, a.typeP, a.post_w, (int64_t)b * a.s_post_w, t, D, a.off_post, 1.0f);
                load_param<W, NV, VEC>(c, a.typeP, a.post_b, (int64_t)b * a.s_post_b, t, D, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[k][j] = u[k][j] * w[k][j] + c[k][j];
            }
            load_param<W, NV, VEC>(w, a.typeP, a.gate, (int64_t)b * a.s_gate, t, D, 0.0f, 1.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[k][j] += u[k][j] * w[k][j];
        }
        if (a.xo) store_row<W, NV, VEC>(a.typeX, a.xo, (int64_t)b * a.strideXO + i * a.ldxo, t, D, x);
        if (a.h == nullptr) continue;
        if (a.pre != SC_NORM_NONE) {
            normalise<W, NV>(x, a.pre, a.eps_pre, t, D, lds);
            f4 w[NV], c[NV];
            load_param<W, NV, VEC>(w, a.typeP, a.pre_w, (int64_t)b * a.s_pre_w, t, D, a.off_pre, 1.0f);
            load_param<W, NV, VEC>(c, a.typeP, a.pre_b, (int64_t)b * a.s_pre_b, t, D, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[k][j] = x[k][j] * w[k][j] + c[k][j];
        }
        const int64_t ho = (int64_t)b * a.strideH + i * a.ldh;
        if (a.typeH == SC_INT8) {
            float m = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = 4 * (64 * W * k + t) + j < D ? fmaxf(m, fabsf(x[k][j])) : m;
            m = row_max<W>(m, lds);
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
        } else {
            store_row<W, NV, VEC>(a.typeH, a.h, ho, t, D, x);
        }
    }
}

// ----------------------------------------------------------------------------
// backward
// ----------------------------------------------------------------------------
enum { P_PRE_W, P_PRE_B, P_GATE, P_POST_W, P_POST_B, NPART };

// The gradient before a norm, in place of the one behind it (d, already times the weight): with n the normalised
// row and r = 1 / deviation, r (d - n mean(d n)), LayerNorm also - mean(d)
template <int W, int NV>
__device__ __forceinline__ void norm_back(f4 (&d)[NV], const f4 (&n)[NV], float r, int kind, int D, float *lds) {
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[0] += d[k][j] * n[k][j];
            s[1] += d[k][j];
        }
    row_sums<W, 2>(s, lds);
    const float dn = s[0] / (float)D, dm = kind == SC_NORM_LAYER ? s[1] / (float)D : 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) d[k][j] = r * (d[k][j] - dm - n[k][j] * dn);
}

template <int NV>
__device__ __forceinline__ void zero(f4 (&v)[NV]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = f4{0.0f, 0.0f, 0.0f, 0.0f};
}

// A block takes chunk_rows rows of a batch entry, RPB at a time, and sums its rows' shares of the parameters'
// gradients in registers; the blocks' sums go to memory and k_norm_sums adds them in a fixed order.  POST: a norm
// behind the branch.
template <int W, int NV, bool VEC, bool POST>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm_back(NormArgs a) {
    constexpr int RPB = W == 1 ? 4 : 1, NP = POST ? 5 : 3;
    __shared__ float lds[2 * W];
    __shared__ f4 join[W == 1 ? 3 * 64 : 1];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x, grp = W == 1 ? threadIdx.x >> 6 : 0;
    const int64_t chunk = block_id();
    if (chunk >= a.chunks) return;
    const int D = a.D;
    const int64_t i1 = min((chunk + 1) * a.chunk_rows, (int64_t)a.rows);
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        f4 sum[NP][NV];
#pragma unroll
        for (int p = 0; p < NP; ++p) zero(sum[p]);
        for (int64_t i = chunk * a.chunk_rows + grp; i < i1; i += RPB) {
            Raw4 rx[NV], ry[NV], rg[NV], rh[NV];
            if (a.x) load_row<W, NV, VEC>(rx, a.typeX, a.x, (int64_t)b * a.strideXO + i * a.ldxo, t, D);
            if (a.y) load_row<W, NV, VEC>(ry, a.typeY, a.y, (int64_t)b * a.strideY + i * a.ldy, t, D);
            if (a.dxo) load_row<W, NV, VEC>(rg, a.typeX, a.dxo, (int64_t)b * a.strideDXO + i * a.lddxo, t, D);
            if (a.dh) load_row<W, NV, VEC>(rh, a.typeH, a.dh, (int64_t)b * a.strideH + i * a.ldh, t, D);
            f4 g[NV];
            if (a.dh) {
                f4 n[NV], w[NV];
                widen(g, a.typeH, rh);
                if (a.pre != SC_NORM_NONE) {
                    widen(n, a.typeX, rx);
                    const float r = normalise<W, NV>(n, a.pre, a.eps_pre, t, D, lds);
                    load_param<W, NV, VEC>(w, a.typeP, a.pre_w, (int64_t)b * a.s_pre_w, t, D, a.off_pre, 1.0f);
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sum[P_PRE_W][k][j] += g[k][j] * n[k][j];
                            sum[P_PRE_B][k][j] += g[k][j];
                            g[k][j] *= w[k][j];
                        }
                    norm_back<W, NV>(g, n, r, a.pre, D, lds);
                }
            } else {
                zero(g);
            }
            if (a.dxo) {
                f4 e[NV];
                widen(e, a.typeX, rg);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[k][j] += e[k][j];
            }
            if (a.dx) {
                f4 e[NV];
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[k][j] = a.scale_res * g[k][j];
                store_row<W, NV, VEC>(a.typeX, a.dx, (int64_t)b * a.strideX + i * a.ldx, t, D, e);
            }
            if (a.y == nullptr && a.dy == nullptr) continue;
            f4 w[NV], n[NV];
            load_param<W, NV, VEC>(w, a.typeP, a.gate, (int64_t)b * a.s_gate, t, D, 0.0f, 1.0f);
            if (a.y) widen(n, a.typeY, ry);
            else zero(n);
            if (POST) {
                f4 pw[NV], c[NV];
                const float r = normalise<W, NV>(n, a.post, a.eps_post, t, D, lds);
                load_param<W, NV, VEC>(pw, a.typeP, a.post_w, (int64_t)b * a.s_post_w, t, D, a.off_post, 1.0f);
                load_param<W, NV, VEC>(c, a.typeP, a.post_b, (int64_t)b * a.s_post_b, t, D, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sum[P_GATE][k][j] += g[k][j] * (n[k][j] * pw[k][j] + c[k][j]);
                        const float du = g[k][j] * w[k][j];
                        sum[NP - 2][k][j] += du * n[k][j];
                        sum[NP - 1][k][j] += du;
                        g[k][j] = du * pw[k][j];
                    }
                if (a.dy) norm_back<W, NV>(g, n, r, a.post, D, lds);
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sum[P_GATE][k][j] += g[k][j] * n[k][j];
                        g[k][j] *= w[k][j];
                    }
            }
            if (a.dy) store_row<W, NV, VEC>(a.typeY, a.dy, (int64_t)b * a.strideDY + i * a.lddy, t, D, g);
        }
        if (a.part == nullptr) continue;
        float *part = a.part + ((int64_t)b * a.chunks + chunk) * NPART * D;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const bool wanted = p == P_PRE_W ? a.dpre_w != nullptr : p == P_PRE_B ? a.dpre_b != nullptr : p == P_GATE ? a.dgate != nullptr
                              : p == P_POST_W ? a.dpost_w != nullptr : a.dpost_b != nullptr;
            if (!wanted) continue;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (W == 1) {
                    __syncthreads();
                    if (grp > 0) join[(grp - 1) * 64 + t] = sum[p][k];
                    __syncthreads();
                    if (grp > 0) continue;
#pragma unroll
                    for (int o = 0; o < 3; ++o)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum[p][k][j] += join[o * 64 + t][j];
                }
                const int d = 4 * (64 * W * k + t);
                store4<VEC>(SC_F32, part, (int64_t)p * D + d, sum[p][k], D - d);
            }
        }
    }
}

// Sums over the chunks, and over the batch where a parameter is shared: 64 columns by 16 groups of chunks, whose
// sums are joined in order
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs a) {
    __shared__ float join[16][64];
    const int c = threadIdx.x & 63, grp = threadIdx.x >> 6, d = blockIdx.x * 64 + c, p = blockIdx.y;
    float *out = p == P_PRE_W ? a.dpre_w : p == P_PRE_B ? a.dpre_b : p == P_GATE ? a.dgate : p == P_POST_W ? a.dpost_w : a.dpost_b;
    const int64_t stride = p == P_PRE_W ? a.s_pre_w : p == P_PRE_B ? a.s_pre_b : p == P_GATE ? a.s_gate : p == P_POST_W ? a.s_post_w : a.s_post_b;
    if (out == nullptr) return;
    const int64_t entries = stride == 0 ? 1 : a.batch, n = stride == 0 ? (int64_t)a.batch * a.chunks : a.chunks;
    for (int64_t b = blockIdx.z; b < entries; b += gridDim.z) {
        const float *q = a.part + ((int64_t)b * a.chunks * NPART + p) * a.D + d;
        float s = 0.0f;
        if (d < a.D)
            for (int64_t k = grp; k < n; k += 16) s += q[k * NPART * a.D];
        __syncthreads();
        join[grp][c] = s;
        __syncthreads();
        if (grp == 0 && d < a.D) {
            s = 0.0f;
            for (int k = 0; k < 16; ++k) s += join[k][c];
            out[b * a.D + d] = s;      // (b = 0 where shared)
        }
    }
}

// ----------------------------------------------------------------------------
// host
// ----------------------------------------------------------------------------
template <int W, int NV>
static void launch_norm(const NormArgs &a, bool vec, hipStream_t st) {
    const dim3 grid = grid_of((uint32_t)(((int64_t)a.rows + (W == 1 ? 3 : 0)) / (W == 1 ? 4 : 1)), a.batch), block(W == 1 ? 256 : 64 * W);
    constexpr int SCALAR_W = W == 1 ? 1 : 16, SCALAR_NV = W == 1 ? 5 : 4;     // (shape_of without vec)
    if (vec) hipLaunchKernelGGL((k_norm<W, NV, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_norm<SCALAR_W, SCALAR_NV, false>), grid, block, 0, st, a);
}
template <int W, int NV>
static void launch_back(const NormArgs &a, bool vec, hipStream_t st) {
    const dim3 grid = grid_of((uint32_t)a.chunks, a.batch), block(W == 1 ? 256 : 64 * W);
    constexpr int SCALAR_W = W == 1 ? 1 : 16, SCALAR_NV = W == 1 ? 5 : 4;
    if (a.post != SC_NORM_NONE) {
        if (vec) hipLaunchKernelGGL((k_norm_back<W, NV, true, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_norm_back<SCALAR_W, SCALAR_NV, false, true>), grid, block, 0, st, a);
    } else {
        if (vec) hipLaunchKernelGGL((k_norm_back<W, NV, true, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_norm_back<SCALAR_W, SCALAR_NV, false, false>), grid, block, 0, st, a);
    }
}

struct Shape {
    int W, NV;
};
// The fewest waves that hold a row in five quads a thread (four from 1280 elements on), and the fewest quads.  Rows
// that are read element by element (an odd length or alignment) have two sizes only.
static Shape shape_of(int D, bool vec) {
    if (!vec) return D <= 1280 ? Shape{1, 5} : Shape{16, 4};
    if (D <= 1280) return {1, D <= 256 ? 1 : (D + 255) / 256};
    if (D <= 2048) return {2, 4};
    if (D <= 4096) return {4, D <= 3 * 1024 ? 3 : 4};
    return {16, D <= 8192 ? 2 : 4};
}

// rows of a chunk: about four blocks for each compute unit, and at least four rows in each
static void chunks_of(const sc_norm_desc &d, int *chunks, int *chunk_rows) {
    const int64_t want = 1024 / (d.batch > 0 ? d.batch : 1) + 1;
    int64_t rows = ((int64_t)d.rows + want - 1) / want;
    rows = (rows + 3) / 4 * 4;
    if (rows < 4) rows = 4;
    *chunk_rows = (int)rows;
    *chunks = (int)(((int64_t)d.rows + rows - 1) / rows);
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
// entries of something written must not lie on top of each other
static bool entries_apart(const sc_norm_desc &d, int64_t ld, int64_t stride) {
    return d.batch <= 1 || d.rows == 0 || d.D == 0 || stride >= (int64_t)(d.rows - 1) * ld + d.D;
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

#define SCL_BY_SHAPE(LAUNCH, s, ...)                          \
    do {                                                      \
        if ((s).W == 1) {                                     \
            switch ((s).NV) {                                 \
                case 1: LAUNCH<1, 1>(__VA_ARGS__); break;     \
                case 2: LAUNCH<1, 2>(__VA_ARGS__); break;     \
                case 3: LAUNCH<1, 3>(__VA_ARGS__); break;     \
                case 4: LAUNCH<1, 4>(__VA_ARGS__); break;     \
                default: LAUNCH<1, 5>(__VA_ARGS__); break;    \
            }                                                 \
        } else if ((s).W == 2) {                              \
            LAUNCH<2, 4>(__VA_ARGS__);                        \
        } else if ((s).W == 4) {                              \
            if ((s).NV == 3) LAUNCH<4, 3>(__VA_ARGS__);       \
            else LAUNCH<4, 4>(__VA_ARGS__);                   \
        } else {                                              \
            if ((s).NV == 2) LAUNCH<16, 2>(__VA_ARGS__);      \
            else LAUNCH<16, 4>(__VA_ARGS__);                  \
        }                                                     \
    } while (0)

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
    if (h != nullptr && quantised && d.batch > 1 && d.rows > 0 && d.strideS < (int64_t)(d.rows - 1) * srow + slen) return SC_ERR_STRIDE;
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
    SCL_BY_SHAPE(launch_norm, shape_of(d.D, vec), a, vec, st);
    return hipGetLastError() == hipSuccess ? SC_OK : SC_ERR_HIP;
}

int sc_residual_norm_backward_workspace_size(const sc_norm_desc *desc, size_t *bytes) {
    if (bytes == nullptr) return SC_ERR_NULL;
    const int rc = check_norm(desc);
    if (rc != SC_OK) return rc;
    if (!is_float_type(desc->typeH)) return SC_ERR_TYPE;
    int chunks, chunk_rows;
    chunks_of(*desc, &chunks, &chunk_rows);
    *bytes = (size_t)desc->batch * chunks * NPART * desc->D * sizeof(float);
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
    chunks_of(d, &a.chunks, &a.chunk_rows);
    const bool vec = d.D % 4 == 0 && quads(xo, d.typeX, d.ldxo, d.strideXO) && quads(y, d.typeY, d.ldy, d.strideY) &&
                     quads(dxo, d.typeX, d.lddxo, d.strideDXO) && quads(dh, d.typeH, d.ldh, d.strideH) &&
                     quads(dx, d.typeX, d.ldx, d.strideX) && quads(dy, d.typeY, d.lddy, d.strideDY) && params_quads(d, params);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (rows) {
        SCL_BY_SHAPE(launch_back, shape_of(d.D, vec), a, vec, st);
        if (hipGetLastError() != hipSuccess) return SC_ERR_HIP;
    }
    // (without rows the sums are zeros)
    if (any) {
        hipLaunchKernelGGL(k_norm_sums, dim3((unsigned)((d.D + 63) / 64), NPART, (unsigned)(d.batch < 1 ? 1 : d.batch < 32768 ? d.batch : 32768)),
                           dim3(1024), 0, st, a);
        if (hipGetLastError() != hipSuccess) return SC_ERR_HIP;
    }
    return SC_OK;
}

}  // extern "C"
