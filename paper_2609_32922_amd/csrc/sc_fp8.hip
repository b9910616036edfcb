// 8-bit floats with a scale for each block of 128: the quantiser, and the product of two such operands
// on the matrix cores.
#include <math.h>

#include "sc_layer.h"

namespace scl {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// ----------------------------------------------------------------------------
// quantiser
// ----------------------------------------------------------------------------
struct QuantArgs {
    int batch, rows, K, KB;
    const void *X;
    int64_t ldx, strideX;
    int e5;
    uint8_t *Q;
    int64_t ldq, strideQ;
    float *scale;
    int64_t lds, strideS;
};

// eight elements of type TX as floats, zeros past n
template <int TX, bool VEC>
struct Raw8 {
    u4 w[TX == SC_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *p, int64_t at, int n) {
        if (VEC) {   // (whole octets: n is 8 or at most 0)
#pragma unroll
            for (int k = 0; k < (TX == SC_F32 ? 2 : 1); ++k) w[k] = u4{0u, 0u, 0u, 0u};
            if (n <= 0) return;
            const u4 *q = reinterpret_cast<const u4 *>(static_cast<const uint8_t *>(p) + at * (TX == SC_F32 ? 4 : 2));
#pragma unroll
            for (int k = 0; k < (TX == SC_F32 ? 2 : 1); ++k) w[k] = q[k];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (TX == SC_F32) {
                    w[j >> 2][j & 3] = j < n ? static_cast<const uint32_t *>(p)[at + j] : 0u;
                } else {
                    const uint32_t h = j < n ? static_cast<const uint16_t *>(p)[at + j] : 0u;
                    w[0][j >> 1] = j & 1 ? w[0][j >> 1] | h << 16 : h;
                }
            }
        }
    }
    __device__ __forceinline__ float at(int j) const {
        if (TX == SC_F32) return __uint_as_float(w[j >> 2][j & 3]);
        const uint32_t h = (w[0][j >> 1] >> (16 * (j & 1))) & 0xffffu;
        return TX == SC_BF16 ? from_bf16(h) : from_f16(h);
    }
};

// 1 x 128: sixteen lanes take a block, eight elements each, so a 16-bit block is one 16-byte load and
// one 8-byte store per lane; each group of lanes has QU blocks in flight.  Memory-bound.
constexpr int QU = 4;
template <int TX, bool VEC>
__global__ __launch_bounds__(256) void k_fp8_rows(QuantArgs a, uint32_t blocks) {
    const int sub = threadIdx.x & 15;
    const float top = a.e5 ? E5M2_MAX : E4M3_MAX;
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        const uint8_t *X = static_cast<const uint8_t *>(a.X) + (size_t)b * a.strideX * (TX == SC_F32 ? 4 : 2);
        Raw8<TX, VEC> r[QU];
        uint32_t row[QU];
        int d[QU], n[QU];
#pragma unroll
        for (int k = 0; k < QU; ++k) {
            const uint32_t i = (block_id() * QU + k) * 16u + (threadIdx.x >> 4);
            row[k] = i / (uint32_t)a.KB;
            d[k] = (int)(i - row[k] * (uint32_t)a.KB) * FP8_BLOCK + 8 * sub;
            n[k] = i < blocks ? min(a.K - d[k], 8) : 0;
            if (i >= blocks) row[k] = 0;
            r[k].load(X, (int64_t)row[k] * a.ldx + d[k], n[k]);
        }
#pragma unroll
        for (int k = 0; k < QU; ++k) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(r[k].at(j)));
            m = lanes_max<16>(m);
            const Fp8Scale s = fp8_scale(m, top);
            if (n[k] > 0 && sub == 0) a.scale[(size_t)b * a.strideS + (size_t)row[k] * a.lds + (d[k] >> 7)] = s.s;
            const f4 lo = {r[k].at(0), r[k].at(1), r[k].at(2), r[k].at(3)}, hi = {r[k].at(4), r[k].at(5), r[k].at(6), r[k].at(7)};
            const u2 w = {quant_fp8x4(a.e5, lo, s.inv), quant_fp8x4(a.e5, hi, s.inv)};
            uint8_t *q = a.Q + (size_t)b * a.strideQ + (size_t)row[k] * a.ldq + d[k];
            if (VEC) {
                if (n[k] > 0) *reinterpret_cast<u2 *>(q) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n[k]) q[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

// largest over a block of 256 threads
__device__ __forceinline__ float block_max(float m) {
    __shared__ float part[4];
    m = lanes_max<64>(m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// 128 x 128: a block of threads takes a block of the operand, kept in registers between its two passes
template <int TX, bool VEC>
__global__ __launch_bounds__(256) void k_fp8_tiles(QuantArgs a) {
    const float top = a.e5 ? E5M2_MAX : E4M3_MAX;
    const int kb = (int)(block_id() % (uint32_t)a.KB), rb = (int)(block_id() / (uint32_t)a.KB);
    if ((int64_t)rb * 128 >= a.rows) return;
    const int d = kb * FP8_BLOCK + 8 * (threadIdx.x & 15);
    const int64_t i0 = (int64_t)rb * 128 + (threadIdx.x >> 4);
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        const uint8_t *X = static_cast<const uint8_t *>(a.X) + (size_t)b * a.strideX * (TX == SC_F32 ? 4 : 2);
        Raw8<TX, VEC> r[8];
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t i = i0 + 16 * k;
            r[k].load(X, min(i, (int64_t)a.rows - 1) * a.ldx + d, i < a.rows ? min(a.K - d, 8) : 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(r[k].at(j)));
        const Fp8Scale s = fp8_scale(block_max(m), top);
        if (threadIdx.x == 0) a.scale[(size_t)b * a.strideS + (size_t)rb * a.lds + kb] = s.s;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t i = i0 + 16 * k;
            const int n = i < a.rows ? min(a.K - d, 8) : 0;
            const f4 lo = {r[k].at(0), r[k].at(1), r[k].at(2), r[k].at(3)}, hi = {r[k].at(4), r[k].at(5), r[k].at(6), r[k].at(7)};
            const u2 w = {quant_fp8x4(a.e5, lo, s.inv), quant_fp8x4(a.e5, hi, s.inv)};
            uint8_t *q = a.Q + (size_t)b * a.strideQ + min(i, (int64_t)a.rows - 1) * a.ldq + d;
            if (VEC) {
                if (n > 0) *reinterpret_cast<u2 *>(q) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) q[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

// 128 x 1, transposed: a block of threads takes 128 rows x 64 columns, four neighbouring rows and eight
// columns a thread, and turns the bytes over in LDS, so that loads and stores both run along rows.
constexpr int QT_COLS = 64, QT_LD = 33;      // dwords of a column in LDS: 128 bytes and one to spread the banks
template <int TX, bool VEC>
__global__ __launch_bounds__(256) void k_fp8_turned(QuantArgs a, int colblocks, int vecq) {
    __shared__ float part[4][QT_COLS];
    __shared__ uint32_t turned[QT_COLS * QT_LD];
    const float top = a.e5 ? E5M2_MAX : E4M3_MAX;
    const int tid = threadIdx.x, c8 = 8 * (tid & 7), rq = tid >> 3;
    const int cb = (int)(block_id() % (uint32_t)colblocks), rb = (int)(block_id() / (uint32_t)colblocks);
    if ((int64_t)rb * 128 >= a.rows) return;
    const int d0 = cb * QT_COLS;
    const int64_t i0 = (int64_t)rb * 128;
    for (int b = blockIdx.z; b < a.batch; b += gridDim.z) {
        const uint8_t *X = static_cast<const uint8_t *>(a.X) + (size_t)b * a.strideX * (TX == SC_F32 ? 4 : 2);
        Raw8<TX, VEC> r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = i0 + 4 * rq + k;
            r[k].load(X, min(i, (int64_t)a.rows - 1) * a.ldx + d0 + c8, i < a.rows ? min(a.K - d0 - c8, 8) : 0);
        }
        float m[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) m[j] = fmaxf(m[j], fabsf(r[k].at(j)));
            for (int o = 8; o < 64; o <<= 1) m[j] = fmaxf(m[j], __shfl_xor(m[j], o, 64));
        }
        __syncthreads();                    // (the last batch entry's reads of LDS)
        if ((tid & 63) < 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) part[tid >> 6][c8 + j] = m[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c8 + j;
            const Fp8Scale s = fp8_scale(fmaxf(fmaxf(part[0][c], part[1][c]), fmaxf(part[2][c], part[3][c])), top);
            if (rq == 0 && d0 + c < a.K) a.scale[(size_t)b * a.strideS + (size_t)(d0 + c) * a.lds + rb] = s.s;
            const f4 v = {r[0].at(j), r[1].at(j), r[2].at(j), r[3].at(j)};
            turned[c * QT_LD + rq] = quant_fp8x4(a.e5, v, s.inv);
        }
        __syncthreads();
        // a column's 128 bytes by eight threads, 16 each
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = (tid >> 3) + 32 * h, at = 16 * (tid & 7), n = d0 + c < a.K ? (int)min(a.rows - i0 - at, (int64_t)16) : 0;
            if (n > 0) {
                uint8_t *q = a.Q + (size_t)b * a.strideQ + (size_t)(d0 + c) * a.ldq + i0 + at;
                u4 w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = turned[c * QT_LD + (at >> 2) + k];
                if (vecq && n == 16) {
                    *reinterpret_cast<u4 *>(q) = w;
                } else {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (k < n) q[k] = (uint8_t)(w[k >> 2] >> (8 * (k & 3)));
                }
            }
        }
    }
}

template <int TX, bool VEC>
static hipError_t launch_quant_fp8(const QuantArgs &a, int block, hipStream_t st) {
    if (block == SC_BLOCK_1X128) {
        const uint32_t blocks = (uint32_t)a.rows * (uint32_t)a.KB;
        hipLaunchKernelGGL((k_fp8_rows<TX, VEC>), grid_of((blocks + 16 * QU - 1) / (16 * QU), a.batch), dim3(256), 0, st, a, blocks);
    } else if (block == SC_BLOCK_128X128) {
        const uint32_t tiles = (uint32_t)((int)(((int64_t)a.rows + 127) / 128)) * (uint32_t)a.KB;
        hipLaunchKernelGGL((k_fp8_tiles<TX, VEC>), grid_of(tiles, a.batch), dim3(256), 0, st, a);
    } else {
        const int colblocks = (a.K + QT_COLS - 1) / QT_COLS;
        const int vecq = aligned_to(a.Q, 16) && a.ldq % 16 == 0 && a.strideQ % 16 == 0;
        hipLaunchKernelGGL((k_fp8_turned<TX, VEC>), grid_of((uint32_t)((int)(((int64_t)a.rows + 127) / 128)) * (uint32_t)colblocks, a.batch), dim3(256), 0,
                           st, a, colblocks, vecq);
    }
    return hipGetLastError();
}

// ----------------------------------------------------------------------------
// product
// ----------------------------------------------------------------------------
struct GemmArgs {
    int M, N, K, KB;
    const uint8_t *A, *B;
    const float *sA, *sB, *bias;
    void *out;
    int64_t lda, ldb, ldo, strideA, strideB, strideO, ldsA, ldsB, strideSA, strideSB, strideBias;
    int shiftA, shiftB;          // log2 of the rows that share a scale
    int typeO, vecO;             // vecO: four outputs of a row can be stored at once
    int tilesM, tilesN, batch;
};

// D = X Y^T over 128 elements: lane l holds 32 bytes of X's row l % 16 and of Y's row l % 16, the same
// elements of both (which ones does not matter), and gets D[4 (l / 16) + r][l % 16], r = 0..3.
//
// The matrix cores' 8-bit products keep, of each eight neighbours in a lane, what lies within 2^-13 of the
// largest one's power of two (measured: beside a product of 2^16 one of 2^3 counts and one of 2^2 does not) and add the
// eights in float32.  That is far inside the rounding of a 16-bit result.  EXACT, for float32 results, turns the
// bytes into bfloat16 (every value of both types is one) and takes the 16-bit products, whose sums are float32
// throughout, at half the rate.
template <int T, bool EXACT>
struct Frag {
    v8i w;
    __device__ __forceinline__ void set(u4 lo, u4 hi) {      // the granules that a lane holds
        w = v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    }
};
template <int T>
struct Frag<T, true> {
    b8 w[4];
    __device__ __forceinline__ b2 pair(uint32_t x, bool upper) {
        if (T == 0) return upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false);
        return upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(x, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(x, 1.0f, false);
    }
    __device__ __forceinline__ void set(u4 lo, u4 hi) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = k < 2 ? lo[2 * k] : hi[2 * k - 4], y = k < 2 ? lo[2 * k + 1] : hi[2 * k - 3];
            const b2 p = pair(x, false), q = pair(x, true), r = pair(y, false), s = pair(y, true);
            w[k] = b8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
        }
    }
};
template <int TX, int TY>
__device__ __forceinline__ f4 mma_128(const Frag<TX, false> &x, const Frag<TY, false> &y) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.w, y.w, f4{0.0f, 0.0f, 0.0f, 0.0f}, TX, TY, 0, 0, 0, 0);
}
template <int TX, int TY>
__device__ __forceinline__ f4 mma_128(const Frag<TX, true> &x, const Frag<TY, true> &y) {
    f4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.w[k], y.w[k], d, 0, 0, 0);
    return d;
}

// sixteen bytes of a row from element k on, zeros from element K on
__device__ __forceinline__ u4 load_granule(const uint8_t *row, int k, int K) {
    if (k + 16 <= K) return *reinterpret_cast<const u4_any *>(row + k);
    u4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (k + j < K) w[j >> 2] |= (uint32_t)row[k + j] << (8 * (j & 3));
    return w;
}

__device__ __forceinline__ void store_out4(const GemmArgs &g, int b, int64_t i, int j, f4 v) {
    const int64_t at = (int64_t)b * g.strideO + i * g.ldo + j;
    if (g.vecO && j + 4 <= g.N) store4<true>(g.typeO, g.out, at, v, 4);
    else store4<false>(g.typeO, g.out, at, v, g.N - j);
}

// LDS holds a stage of 128 elements as rows of eight 16-byte granules; granule q of row r lies at
// q ^ swz(r), so that the 16 rows that a fragment read takes at one granule spread over all banks
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

// Copies 16 (or 4) bytes for each lane from the buffer, at off, to LDS, at `to` (the same in every lane) plus 16 (4)
// bytes a lane, past the registers.  Nothing waits for it but wait_copies().  What lies behind the buffer's bound
// leaves no byte of another row in LDS, and only rows that are not stored have any.
typedef uint32_t Buffer __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Buffer buffer_of(const void *p, int64_t bytes) {
    const uint64_t x = (uint64_t)p;
    return Buffer{(uint32_t)x, (uint32_t)(x >> 32) & 0xffffu, (uint32_t)bytes, 0x00020000u};
}
__device__ __forceinline__ Buffer advanced(Buffer s, uint32_t bytes) {
    const uint64_t x = ((uint64_t)s[1] << 32 | s[0]) + bytes;
    return Buffer{(uint32_t)x, (uint32_t)(x >> 32), s[2] - min(s[2], bytes), s[3]};
}
__device__ __forceinline__ Buffer scalar(Buffer s) {      // (it is the same in every lane; told to the compiler)
    return Buffer{(uint32_t)__builtin_amdgcn_readfirstlane((int)s[0]), (uint32_t)__builtin_amdgcn_readfirstlane((int)s[1]),
                  (uint32_t)__builtin_amdgcn_readfirstlane((int)s[2]), 0x00020000u};
}
__device__ __forceinline__ void copy16(Buffer s, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(scalar(s)) : "memory");
}
__device__ __forceinline__ void copy4(Buffer s, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(scalar(s)) : "memory");
}
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

// a word's bytes before the n-th
__device__ __forceinline__ uint32_t bytes_before(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// Where a block's tile starts, in an order that keeps neighbours together on an XCD (blocks are dealt to the eight
// XCDs in turn, and each has an L2 of its own): a contiguous run of tiles for each, in groups of eight tile rows
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t tiles, int tilesM, int tilesN, int *b, int *tm, int *tn) {
    const uint32_t xcd = id & 7u, each = tiles >> 3, more = tiles & 7u;
    const uint32_t all = xcd * each + (xcd < more ? xcd : more) + (id >> 3), per = (uint32_t)tilesM * (uint32_t)tilesN;
    const uint32_t entry = all / per, at = all - entry * per;
    const uint32_t group = at / (8u * (uint32_t)tilesN), in = at - group * 8u * (uint32_t)tilesN;
    const uint32_t rows = min(8u, (uint32_t)tilesM - 8u * group);
    *b = (int)entry;
    *tm = (int)(8u * group + in % rows);
    *tn = (int)(in / rows);
}

// A tile of BM x BN outputs by waves of WM x WN each.  A scale block is one stage: the matrix cores sum its
// 128 products from zero and the sum enters the accumulators times its two scales.
template <int TA, int TB, bool EXACT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_fp8_any(GemmArgs g) {
    constexpr int NT = (BM / WM) * (BN / WN) * 64, MI = WM / 16, NI = WN / 16, GA = BM * 8 / NT, GB = BN * 8 / NT;
    __shared__ u4 sm[(BM + BN) * 8];
    __shared__ float sc[BM + BN];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, q4 = lane >> 4;
    const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
    const int64_t m0 = (int64_t)(block_id() % (uint32_t)g.tilesM) * BM, n0 = (int64_t)(block_id() / (uint32_t)g.tilesM) * BN;
    if (n0 >= g.N) return;
    for (int b = blockIdx.z; b < g.batch; b += gridDim.z) {
        const uint8_t *A = g.A + (int64_t)b * g.strideA, *B = g.B + (int64_t)b * g.strideB;
        const float *sA = g.sA + (int64_t)b * g.strideSA, *sB = g.sB + (int64_t)b * g.strideSB;
        f4 acc[MI][NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int t = 0; t < g.KB; ++t) {
            u4 ra[GA], rb[GB];
#pragma unroll
            for (int k = 0; k < GA; ++k) {
                const int x = tid + k * NT;
                ra[k] = load_granule(A + min(m0 + (x >> 3), (int64_t)g.M - 1) * g.lda, t * 128 + 16 * (x & 7), g.K);
            }
#pragma unroll
            for (int k = 0; k < GB; ++k) {
                const int x = tid + k * NT;
                rb[k] = load_granule(B + min(n0 + (x >> 3), (int64_t)g.N - 1) * g.ldb, t * 128 + 16 * (x & 7), g.K);
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < GA; ++k) {
                const int x = tid + k * NT, r = x >> 3;
                sm[r * 8 + ((x & 7) ^ swz(r))] = ra[k];
            }
#pragma unroll
            for (int k = 0; k < GB; ++k) {
                const int x = tid + k * NT, r = x >> 3;
                sm[(BM + r) * 8 + ((x & 7) ^ swz(r))] = rb[k];
            }
            for (int x = tid; x < BM + BN; x += NT)
                sc[x] = x < BM ? sA[(min(m0 + x, (int64_t)g.M - 1) >> g.shiftA) * g.ldsA + t]
                               : sB[(min(n0 + x - BM, (int64_t)g.N - 1) >> g.shiftB) * g.ldsB + t];
            __syncthreads();
            Frag<TB, EXACT> fb[NI];
            f4 sb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = wn + 16 * j + l16;
                const u4 lo = sm[(BM + r) * 8 + ((2 * q4) ^ swz(r))], hi = sm[(BM + r) * 8 + ((2 * q4 + 1) ^ swz(r))];
                fb[j].set(lo, hi);
                sb[j] = *reinterpret_cast<const f4 *>(&sc[BM + wn + 16 * j + 4 * q4]);
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int r = wm + 16 * i + l16;
                const u4 lo = sm[r * 8 + ((2 * q4) ^ swz(r))], hi = sm[r * 8 + ((2 * q4 + 1) ^ swz(r))];
                Frag<TA, EXACT> fa;
                fa.set(lo, hi);
                const float s = sc[r];
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const f4 p = mma_128(fb[j], fa);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += p[e] * (s * sb[j][e]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t m = m0 + wm + 16 * i + l16;
            if (m >= g.M) continue;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int64_t n = n0 + wn + 16 * j + 4 * q4;
                if (n >= g.N) continue;
                f4 v = acc[i][j];
                if (g.bias) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + e < g.N) v[e] += g.bias[(int64_t)b * g.strideBias + n + e];
                }
                store_out4(g, b, m, (int)n, v);
            }
        }
    }
}

// A wave's outputs from row m0 and column n0 on: lane (q4, l16) holds rows 16 i + l16, columns 16 j + 4 q4 .. + 3.
// Stores carry 32-bit offsets from the corner; rows behind the last lie behind the buffer's bound, which drops them, and
// columns behind the last are sent there, so nothing branches.  (store_tile's caller has 16 MI rows in 2^30 bytes.)
template <int TO, bool QUADS, int MI, int NI>
__device__ __forceinline__ void store_rows(const __amdgpu_buffer_rsrc_t o, const float *bias, int cols, uint32_t ldo, int l16, int q4,
                                           const f4 (&acc)[MI][NI]) {
    constexpr uint32_t ES = TO == SC_F32 ? 4 : 2, BEHIND = 0x80000000u;
    const uint32_t row = (uint32_t)l16 * ldo * ES, step = 16u * ldo * ES;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int n = 16 * j + 4 * q4;
        f4 add = {0.0f, 0.0f, 0.0f, 0.0f};
        if (bias)
#pragma unroll
            for (int e = 0; e < 4; ++e) add[e] = bias[min(n + e, cols - 1)];
        uint32_t at[4];
#pragma unroll
        for (int e = 0; e < (QUADS ? 1 : 4); ++e) at[e] = n + e < cols ? row + (uint32_t)(n + e) * ES : BEHIND;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const f4 v = acc[i][j] + add;
            if (QUADS && TO == SC_F32) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, v), o, at[0] + i * step, 0, 0);
            } else if (QUADS) {
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = TO == SC_BF16 ? to_bf16(v[e]) : to_f16(v[e]);
                __builtin_amdgcn_raw_buffer_store_b64(u2{h[0] | h[1] << 16, h[2] | h[3] << 16}, o, at[0] + i * step, 0, 0);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (TO == SC_F32) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[e]), o, at[e] + i * step, 0, 0);
                    else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(TO == SC_BF16 ? to_bf16(v[e]) : to_f16(v[e])), o, at[e] + i * step, 0, 0);
                }
            }
        }
    }
}
template <bool EXACT, int MI, int NI>
__device__ __forceinline__ void store_tile(const GemmArgs &g, int b, int64_t m0, int64_t n0, int l16, int q4, const f4 (&acc)[MI][NI]) {
    const int64_t es = EXACT ? 4 : 2;
    const int rows = (int)min(g.M - m0, (int64_t)(16 * MI)), cols = (int)min(g.N - n0, (int64_t)(16 * NI));
    if (rows <= 0 || cols <= 0) return;
    uint8_t *corner = static_cast<uint8_t *>(g.out) + (b * g.strideO + m0 * g.ldo + n0) * es;
    const __amdgpu_buffer_rsrc_t o = __builtin_amdgcn_make_buffer_rsrc(corner, 0, (int)(((rows - 1) * g.ldo + cols) * es), 0x00020000);
    const float *bias = g.bias ? g.bias + b * g.strideBias + n0 : nullptr;
    const uint32_t ldo = (uint32_t)g.ldo;
    if (EXACT) {
        if (g.vecO) store_rows<SC_F32, true>(o, bias, cols, ldo, l16, q4, acc);
        else store_rows<SC_F32, false>(o, bias, cols, ldo, l16, q4, acc);
    } else if (g.typeO == SC_BF16) {
        if (g.vecO) store_rows<SC_BF16, true>(o, bias, cols, ldo, l16, q4, acc);
        else store_rows<SC_BF16, false>(o, bias, cols, ldo, l16, q4, acc);
    } else {
        if (g.vecO) store_rows<SC_F16, true>(o, bias, cols, ldo, l16, q4, acc);
        else store_rows<SC_F16, false>(o, bias, cols, ldo, l16, q4, acc);
    }
}

// A tile of BM x BN outputs by waves of WM x WN each, one block after the other by the same threads.  A scale block is
// one stage: the matrix cores sum its 128 products from zero and the sum enters the accumulators times its two
// scales.  A stage's operands and scales are copied to LDS while the stage before it is multiplied.
// BLOCKB: the rows of B share a scale by 128, so a wave's columns have one.
template <int TA, int TB, bool EXACT, bool BLOCKB, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_fp8_gemm(GemmArgs g, uint32_t tiles) {
    constexpr int NW = (BM / WM) * (BN / WN), MI = WM / 16, NI = WN / 16, ROWS = BM + BN;
    constexpr int WR = ROWS / NW, CH = WR / 8;      // rows that a wave copies of each stage, eight at a time
    static_assert(WR == 64 && BM % WR == 0, "a wave copies rows of one operand, and a scale for each of its lanes");
    __shared__ u4 sm[2][ROWS * 8];
    __shared__ float sc[2][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, q4 = lane >> 4;
    const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;

    // what this wave copies: rows r0 .. r0 + 63 of a tile of A or of B
    const bool forB = wave >= BM / WR;
    const int r0 = (forB ? wave - BM / WR : wave) * WR, shift = forB ? g.shiftB : g.shiftA, all = forB ? g.N : g.M;
    const int64_t ld = forB ? g.ldb : g.lda, lds = forB ? g.ldsB : g.ldsA, stride = forB ? g.strideB : g.strideA,
                  sstride = forB ? g.strideSB : g.strideSA;
    const uint8_t *const src = forB ? g.B : g.A;
    const float *const ssrc = forB ? g.sB : g.sA;
    uint32_t off[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int r = r0 + 8 * k + (lane >> 3);
        off[k] = (uint32_t)r * (uint32_t)ld + 16u * ((lane & 7) ^ swz(r));
    }
    const uint32_t soff = 4u * (uint32_t)((r0 + lane) >> shift) * (uint32_t)lds;
    // the next stage to copy: stage ct of the tile (cb, cm, cn)
    Buffer from, sfrom;
    uint32_t next = blockIdx.x;
    int cb, cm, cn, ct = 0;
    const auto enter = [&]() {
        tile_at(next, tiles, g.tilesM, g.tilesN, &cb, &cm, &cn);
        const int64_t x0 = forB ? (int64_t)cn * BN : (int64_t)cm * BM, rows = min((int64_t)(forB ? BN : BM), all - x0);
        from = buffer_of(src + cb * stride + x0 * ld, (rows - 1) * ld + g.K);
        sfrom = buffer_of(ssrc + cb * sstride + (x0 >> shift) * lds, 4 * (((rows - 1) >> shift) * lds + g.KB));
    };
    const auto advance = [&]() {      // to the stage behind the one that has been copied; behind the last there is nothing to read
        if (++ct < g.KB) {
            from = advanced(from, 128);
            sfrom = advanced(sfrom, 4);
            return;
        }
        ct = 0;
        next += gridDim.x;
        if (next < tiles) enter();
        else from[2] = sfrom[2] = 0u;
    };
    const auto copy = [&](int buf, int k) { copy16(from, off[k], lds_address(&sm[buf][(wave * CH + k) * 64])); };
    const auto copy_scales = [&](int buf) { copy4(sfrom, soff, lds_address(&sc[buf][wave * WR])); };
    enter();
    if (g.KB > 0) {
#pragma unroll
        for (int k = 0; k < CH; ++k) copy(0, k);
        copy_scales(0);
    }
    const int cut = g.K & 127;
    int buf = 0;
    for (uint32_t id = blockIdx.x; id < tiles; id += gridDim.x) {
        const int64_t m0 = (int64_t)cm * BM, n0 = (int64_t)cn * BN;
        const int b = cb;
        f4 acc[MI][NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int t = 0; t < g.KB; ++t) {
            wait_copies();
            if (cut && t + 1 == g.KB) {
                // a cut last stage: what lies behind K in this wave's rows becomes zero
#pragma unroll 1
                for (int k = 0; k < CH; ++k) {
                    u4 *p = &sm[buf][(wave * CH + k) * 64 + lane];
                    const int left = cut - 16 * ((lane & 7) ^ swz(8 * k + (lane >> 3)));
                    *p &= u4{bytes_before(left), bytes_before(left - 4), bytes_before(left - 8), bytes_before(left - 12)};
                }
            }
            __syncthreads();          // everyone's copies have arrived, and the other buffer has been read
            advance();
            // Row group i is multiplied while group i + 1 is read, a part of the next stage is sent for and the sums of group
            // i - 1 are scaled.  The fences hold that order: left to itself the compiler scales a group's sums as soon as they
            // are there, and both waves of a SIMD then wait for the same unit in turn.
            const u4 *s = sm[buf];
            const auto read = [&](auto &f, int r) { f.set(s[r * 8 + (q4 ^ swz(r))], s[r * 8 + ((q4 + 4) ^ swz(r))]); };
            Frag<TB, EXACT> fb[NI];
            Frag<TA, EXACT> fa[2];
            f4 sb[BLOCKB ? 1 : NI], p[2][NI];
            float sa[3];
            read(fa[0], wm + l16);
#pragma unroll
            for (int j = 0; j < NI; ++j) read(fb[j], BM + wn + 16 * j + l16);
            if (BLOCKB) {
                sb[0] = f4{sc[buf][BM + wn], 0.0f, 0.0f, 0.0f};
            } else {
#pragma unroll
                for (int j = 0; j < NI; ++j) sb[j] = *reinterpret_cast<const f4 *>(&sc[buf][BM + wn + 16 * j + 4 * q4]);
            }
            sa[0] = sc[buf][wm + l16];
            copy_scales(buf ^ 1);
            const auto add = [&](int i, int j) {
                const float s0 = sa[i % 3];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[i & 1][j][e], BLOCKB ? s0 : s0 * sb[BLOCKB ? 0 : j][e], acc[i][j][e]);
            };
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (i + 1 < MI) {
                    read(fa[(i + 1) & 1], wm + 16 * (i + 1) + l16);
                    sa[(i + 1) % 3] = sc[buf][wm + 16 * (i + 1) + l16];
                }
#pragma unroll
                for (int k = i * CH / MI; k < (i + 1) * CH / MI; ++k) copy(buf ^ 1, k);
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    p[i & 1][j] = mma_128(fb[j], fa[i & 1]);
                    if (i > 0) add(i - 1, j);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (BLOCKB) sa[i % 3] *= sb[0][0];
            }
#pragma unroll
            for (int j = 0; j < NI; ++j) add(MI - 1, j);
            buf ^= 1;
        }
        if (g.KB == 0) {
            next += gridDim.x;
            if (next < tiles) enter();
        }
        store_tile<EXACT, MI, NI>(g, b, m0 + wm, n0 + wn, l16, q4, acc);
    }
}

template <int TA, int TB, bool EXACT, bool BLOCKB, int BM, int BN, int WM, int WN>
static hipError_t launch_tile(const GemmArgs &g0, int per_cu, hipStream_t st) {
    GemmArgs g = g0;
    g.tilesM = (int)(((int64_t)g.M + BM - 1) / BM);
    g.tilesN = (int)(((int64_t)g.N + BN - 1) / BN);
    const uint32_t tiles = (uint32_t)g.tilesM * (uint32_t)g.tilesN * (uint32_t)g.batch, most = 256u * per_cu;
    hipLaunchKernelGGL((k_fp8_gemm<TA, TB, EXACT, BLOCKB, BM, BN, WM, WN>), dim3(tiles < most ? tiles : most), dim3((BM / WM) * (BN / WN) * 64),
                       0, st, g, tiles);
    return hipGetLastError();
}
template <int TA, int TB, bool EXACT>
static hipError_t launch_gemm(const GemmArgs &g, hipStream_t st) {
    const bool al = aligned_to(g.A, 16) && aligned_to(g.B, 16) && g.lda % 16 == 0 && g.ldb % 16 == 0 && g.strideA % 16 == 0 && g.strideB % 16 == 0;
    if (!al || g.lda > (1 << 23) || g.ldb > (1 << 23) || g.ldsA > (1 << 21) || g.ldsB > (1 << 21) || g.ldo > (1 << 20) || getenv("SCT0")) {
        GemmArgs h = g;
        h.tilesM = (int)(((int64_t)g.M + 127) / 128);
        h.tilesN = (int)(((int64_t)g.N + 127) / 128);
        hipLaunchKernelGGL((k_fp8_any<TA, TB, EXACT, 128, 128, 64, 64>), grid_of((uint32_t)h.tilesM * (uint32_t)h.tilesN, g.batch), dim3(256), 0, st, h);
        return hipGetLastError();
    }
    if (getenv("SCT") && atoi(getenv("SCT")) == 1) return g.shiftB ? launch_tile<TA, TB, EXACT, true, 128, 128, 64, 64>(g, 2, st) : launch_tile<TA, TB, EXACT, false, 128, 128, 64, 64>(g, 2, st);
    if (EXACT) return g.shiftB ? launch_tile<TA, TB, EXACT, true, 128, 128, 64, 64>(g, 2, st) : launch_tile<TA, TB, EXACT, false, 128, 128, 64, 64>(g, 2, st);
    return g.shiftB ? launch_tile<TA, TB, false, true, 256, 256, 128, 64>(g, 1, st) : launch_tile<TA, TB, false, false, 256, 256, 128, 64>(g, 1, st);
}

template <bool EXACT>
static hipError_t launch_gemm_types(const GemmArgs &g, int typeA, int typeB, hipStream_t st) {
    if (typeA == SC_E4M3) return typeB == SC_E4M3 ? launch_gemm<0, 0, EXACT>(g, st) : launch_gemm<0, 1, EXACT>(g, st);
    return typeB == SC_E4M3 ? launch_gemm<1, 0, EXACT>(g, st) : launch_gemm<1, 1, EXACT>(g, st);
}

static int check_gemm(const sc_fp8_gemm_desc *d) {
    if (d == nullptr) return SC_ERR_NULL;
    if (d->reserved != 0) return SC_ERR_RESERVED;
    if (d->batch < 0 || d->M < 0 || d->N < 0 || d->K < 0 || d->K > SC_K_LIMIT) return SC_ERR_SHAPE;
    if (!is_fp8_type(d->typeA) || !is_fp8_type(d->typeB) || !is_float_type(d->typeO)) return SC_ERR_TYPE;
    if ((d->rowsA != 1 && d->rowsA != 128) || (d->rowsB != 1 && d->rowsB != 128)) return SC_ERR_TYPE;
    const int64_t kb = (d->K + FP8_BLOCK - 1) / FP8_BLOCK;
    if (d->lda < d->K || d->ldb < d->K || d->ldo < d->N || d->ldsA < kb || d->ldsB < kb) return SC_ERR_STRIDE;
    if (d->strideA < 0 || d->strideB < 0 || d->strideO < 0 || d->strideSA < 0 || d->strideSB < 0 || d->strideBias < 0)
        return SC_ERR_STRIDE;
    // (batch entries of the output must not lie on top of each other)
    if (d->batch > 1 && d->M > 0 && d->N > 0 && d->strideO < (int64_t)(d->M - 1) * d->ldo + d->N) return SC_ERR_STRIDE;
    const int64_t tiles = (((int64_t)d->M + 63) / 64) * (((int64_t)d->N + 63) / 64);
    if (tiles > INT32_MAX) return SC_ERR_SHAPE;
    return SC_OK;
}

}  // namespace scl

using namespace scl;

extern "C" {

int sc_fp8_quantize(int32_t batch, int32_t rows, int32_t K, int32_t typeX, const void *X, int64_t ldx,
                    int64_t strideX, int32_t typeQ, int32_t block, void *Q, int64_t ldq, int64_t strideQ,
                    float *scale, int64_t lds, int64_t strideS, void *stream) {
    if (batch < 0 || rows < 0 || K < 0 || K > SC_K_LIMIT) return SC_ERR_SHAPE;
    if (!is_float_type(typeX) || !is_fp8_type(typeQ) || block < SC_BLOCK_1X128 || block > SC_BLOCK_128X1_T) return SC_ERR_TYPE;
    const bool turned = block == SC_BLOCK_128X1_T;
    const int32_t KB = (K + FP8_BLOCK - 1) / FP8_BLOCK;
    const int32_t RB = (int32_t)(((int64_t)rows + 127) / 128);
    const int64_t qrows = turned ? K : rows, qcols = turned ? rows : K;
    const int64_t srows = block == SC_BLOCK_128X128 ? RB : qrows, scols = turned ? RB : KB;
    if (ldx < K || ldq < qcols || lds < scols || strideX < 0 || strideQ < 0 || strideS < 0) return SC_ERR_STRIDE;
    if (batch > 1 && rows > 0 && K > 0 && (strideQ < (qrows - 1) * ldq + qcols || strideS < (srows - 1) * lds + scols))
        return SC_ERR_STRIDE;
    if ((int64_t)rows * KB > INT32_MAX || (int64_t)RB * ((K + 63) / 64) > INT32_MAX) return SC_ERR_SHAPE;
    if (batch == 0 || rows == 0 || K == 0) return SC_OK;
    if (X == nullptr || Q == nullptr || scale == nullptr) return SC_ERR_NULL;
    const int xb = type_bytes(typeX);
    if (!aligned_to(X, xb) || !aligned_to(scale, 4)) return SC_ERR_STRIDE;
    const QuantArgs a{batch, rows, K, KB, X, ldx, strideX, typeQ == SC_E5M2, static_cast<uint8_t *>(Q), ldq, strideQ, scale, lds, strideS};
    // whole octets of X by 16-byte loads, and of Q (unless transposed) by 8-byte stores
    const bool vec = K % 8 == 0 && aligned_to(X, 16) && ldx * xb % 16 == 0 && strideX * xb % 16 == 0 &&
                     (turned || (aligned_to(Q, 8) && ldq % 8 == 0 && strideQ % 8 == 0));
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const hipError_t e = typeX == SC_F32    ? (vec ? launch_quant_fp8<SC_F32, true>(a, block, st) : launch_quant_fp8<SC_F32, false>(a, block, st))
                         : typeX == SC_BF16 ? (vec ? launch_quant_fp8<SC_BF16, true>(a, block, st) : launch_quant_fp8<SC_BF16, false>(a, block, st))
                                            : (vec ? launch_quant_fp8<SC_F16, true>(a, block, st) : launch_quant_fp8<SC_F16, false>(a, block, st));
    return e == hipSuccess ? SC_OK : SC_ERR_HIP;
}

int sc_fp8_gemm_workspace_size(const sc_fp8_gemm_desc *desc, size_t *bytes) {
    if (bytes == nullptr) return SC_ERR_NULL;
    const int rc = check_gemm(desc);
    if (rc != SC_OK) return rc;
    *bytes = 0;
    return SC_OK;
}

int sc_fp8_gemm(const sc_fp8_gemm_desc *desc, const void *A, const float *sA, const void *B, const float *sB,
                const float *bias, void *out, void *workspace, size_t workspace_bytes, void *stream) {
    size_t need = 0;
    const int rc = sc_fp8_gemm_workspace_size(desc, &need);
    if (rc != SC_OK) return rc;
    const sc_fp8_gemm_desc &d = *desc;
    if (d.batch == 0 || d.M == 0 || d.N == 0) return SC_OK;
    if (out == nullptr || (d.K > 0 && (A == nullptr || sA == nullptr || B == nullptr || sB == nullptr))) return SC_ERR_NULL;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned_to(workspace, 256))) return SC_ERR_WORKSPACE;
    if (!aligned_to(out, type_bytes(d.typeO)) || !aligned_to(sA, 4) || !aligned_to(sB, 4) || !aligned_to(bias, 4)) return SC_ERR_STRIDE;
    GemmArgs g{};
    g.M = d.M;
    g.N = d.N;
    g.K = d.K;
    g.KB = (d.K + FP8_BLOCK - 1) / FP8_BLOCK;
    g.A = static_cast<const uint8_t *>(A);
    g.B = static_cast<const uint8_t *>(B);
    g.sA = sA;
    g.sB = sB;
    g.bias = bias;
    g.out = out;
    g.lda = d.lda;
    g.ldb = d.ldb;
    g.ldo = d.ldo;
    g.strideA = d.strideA;
    g.strideB = d.strideB;
    g.strideO = d.strideO;
    g.ldsA = d.ldsA;
    g.ldsB = d.ldsB;
    g.strideSA = d.strideSA;
    g.strideSB = d.strideSB;
    g.strideBias = d.strideBias;
    g.shiftA = d.rowsA == 128 ? 7 : 0;
    g.shiftB = d.rowsB == 128 ? 7 : 0;
    g.typeO = d.typeO;
    const int vb = 4 * type_bytes(d.typeO);
    g.vecO = aligned_to(out, vb) && d.N % 4 == 0 && d.ldo % 4 == 0 && d.strideO % 4 == 0;
    g.batch = d.batch;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const hipError_t e = d.typeO == SC_F32 ? launch_gemm_types<true>(g, d.typeA, d.typeB, st) : launch_gemm_types<false>(g, d.typeA, d.typeB, st);
    return e == hipSuccess ? SC_OK : SC_ERR_HIP;
}

}  // extern "C"
