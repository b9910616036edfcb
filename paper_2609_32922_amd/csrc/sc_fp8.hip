// 8-bit floats with a scale for each block of 128: the quantiser, and the product of two such operands
// on the matrix cores.
#include <math.h>

#include "sc_layer.h"

namespace scl {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

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
        } else if (n >= 8) {
            const u4_any *q = reinterpret_cast<const u4_any *>(static_cast<const uint8_t *>(p) + at * (TX == SC_F32 ? 4 : 2));
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
// one 8-byte store per lane; each group of lanes has QU blocks in flight.  Memory-bound (18464 x 1024 bfloat16: 12.8 us,
// 4.5 TB/s).
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
            } else if (n[k] >= 8) {
                *reinterpret_cast<u2_any *>(q) = w;
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

// 128 x 128: a block of threads takes a block of the operand, kept in registers between its two passes.  Memory-bound (18464 x 1024
// bfloat16: 12.3 us, 4.6 TB/s).
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
            } else if (n >= 8) {
                *reinterpret_cast<u2_any *>(q) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) q[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

// 128 x 1, transposed: a block of threads takes 128 rows x 64 columns, four neighbouring rows and eight
// columns a thread, and turns the bytes over in LDS, so that loads and stores both run along rows (4096 x 4608 bfloat16:
// 15.3 us, 3.7 TB/s).
constexpr int QT_COLS = 64, QT_LD = 33;      // dwords of a column in LDS: 128 bytes and one to spread the banks
template <int TX, bool VEC>
__global__ __launch_bounds__(256) void k_fp8_turned(QuantArgs a, int colblocks) {
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
                if (n == 16) {
                    *reinterpret_cast<u4_any *>(q) = w;
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
        hipLaunchKernelGGL((k_fp8_turned<TX, VEC>), grid_of((uint32_t)((int)(((int64_t)a.rows + 127) / 128)) * (uint32_t)colblocks, a.batch), dim3(256), 0,
                           st, a, colblocks);
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
    int typeO, whole;            // whole: output rows of whole 16-byte stores, at 32-bit offsets in a tile
    int tilesM, tilesN, batch;
    int parts;                   // blocks that share a tile's stages
    float *part;                 // their sums [parts][batch][M][N], where there is more than one
};

// D = X Y^T over 128 elements: lane l holds 32 bytes of X's row l % 16 and of Y's row l % 16, the same
// elements of both (which ones does not matter), and gets D[4 (l / 16) + r][l % 16], r = 0..3.
//
// The matrix cores' 8-bit products keep, of each eight neighbours in a lane, what lies within 2^-13 of the
// largest one's power of two (measured: beside a product of 2^16 one of 2^3 counts and one of 2^2 does not) and add the
// eights in float32.  Seven of eight products may lose up to 2^-13 of the largest each: at most 8.5e-4 of the sum of
// magnitudes, which is less than a quarter of a bfloat16's half step (3.9e-3) of a result as large as that sum, but more than a
// float16's (4.9e-4), and more than a rounding of any type where large products cancel.  bfloat16 results of more than
// 16 rows take them: operands of random signs up to K = 2^20 come out as near as their rounding lets them (error over the rounding's own 1.000).
// EXACT, for the others, turns the bytes into float16 (every value of both types is one) and takes the
// 16-bit products, whose sums are float32 throughout, at half the rate.
template <int T, bool EXACT>
struct Frag {
    v8i w;
    __device__ __forceinline__ void set(u4 lo, u4 hi) {      // the granules that a lane holds
        w = v8i{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    }
};
template <int T>
struct Frag<T, true> {
    h8 w[4];
    // e5m2 is float16's upper byte; e4m3 is converted, two at a time
    static __device__ __forceinline__ h2 pair(uint32_t x, bool upper) {
        if (T == 1) return __builtin_bit_cast(h2, __builtin_amdgcn_perm(x, 0u, upper ? 0x070c060cu : 0x050c040cu));
        return upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false);
    }
    __device__ __forceinline__ void set(u4 lo, u4 hi) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = k < 2 ? lo[2 * k] : hi[2 * k - 4], y = k < 2 ? lo[2 * k + 1] : hi[2 * k - 3];
            const h2 p = pair(x, false), q = pair(x, true), r = pair(y, false), s = pair(y, true);
            w[k] = h8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
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
    for (int k = 0; k < 4; ++k) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.w[k], y.w[k], d, 0, 0, 0);
    return d;
}

// sixteen bytes of a row from element k on, zeros from element K on
__device__ __forceinline__ u4 load_granule(const uint8_t *row, int k, int K) {
    if (k + 16 <= K) return *reinterpret_cast<const u4_any *>(row + k);
    u4 w = {0u, 0u, 0u, 0u};
    if (k >= K) return w;
    if (K >= 16) {
        // the row's last sixteen, moved down over those that lie before k
        const u4 x = *reinterpret_cast<const u4_any *>(row + K - 16);
        const uint64_t lo = (uint64_t)x[1] << 32 | x[0], hi = (uint64_t)x[3] << 32 | x[2];
        const int s = 8 * (k + 16 - K);              // 8 .. 120 bits
        const uint64_t l = s >= 64 ? hi >> (s - 64) : lo >> s | hi << (64 - s), h = s >= 64 ? 0u : hi >> s;
        return u4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
    }
#pragma unroll
    for (int j = 0; j < 15; ++j)                     // (k is 0)
        if (j < K) w[j >> 2] |= (uint32_t)row[j] << (8 * (j & 3));
    return w;
}

// LDS holds a stage of 128 elements as rows of eight 16-byte granules; granule q of row r lies at
// q ^ swz(r), so that the 16 rows that a fragment read takes at one granule spread over all banks
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }
// The rows of B go to the matrix cores in an order that gives a lane neighbouring columns: row 4 q + e of fragment j is
// row 16 q + 4 j + e of 64, so its sums over the four fragments are 16 columns in a row.  Their granules' places:
__device__ __forceinline__ int fragment_row(int l16, int j) { return 16 * (l16 >> 2) + 4 * j + (l16 & 3); }
__device__ __forceinline__ int swz_b(int r) { return ((r >> 1) & 1) | ((r >> 3) & 6); }

// Copies 16 (or 4) bytes for each lane from the buffer, at off, to LDS, at `to` (the same in every lane) plus 16 (4)
// bytes a lane, past the registers.  Nothing waits for it but wait_copies().  A dword that does not lie whole before the
// buffer's bound is not loaded (measured: of a last row of 201 bytes under a bound of 201 the last byte was 0; 204 of 204 arrived),
// so bounds are whole dwords.
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
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(scalar(s)) : "memory", "m0");
}
__device__ __forceinline__ void copy4(Buffer s, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(scalar(s)) : "memory", "m0");
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

// A wave's outputs from row m0 and column n0 on: lane (q4, l16) holds rows 16 i + l16 and, in fragment j, columns 16 j + 4 q4 .. + 3;
// RUN: 16 q4 + 4 j .. + 3 (fragment_row), so that two fragments' 16-bit outputs are stored together.
// WHOLE: rows of whole 16-byte stores.  Stores then carry 32-bit offsets from the corner; rows behind the last lie
// behind the buffer's bound, which drops them, and columns behind the last are sent there, so nothing branches
// (16 MI rows lie in 2^30 bytes).  Otherwise stores go by address, of any alignment, and a run that is cut by the row's end goes
// element by element.
template <int TO, bool WHOLE, bool RUN, int MI, int NI>
__device__ __forceinline__ void store_rows(uint8_t *corner, const float *bias, int rows, int cols, int64_t ldo, int l16, int q4,
                                           const f4 (&acc)[MI][NI]) {
    constexpr int ES = TO == SC_F32 ? 4 : 2, STEP = RUN && TO != SC_F32 ? 2 : 1;   // fragments that are stored together
    constexpr uint32_t BEHIND = 0x80000000u;
    const __amdgpu_buffer_rsrc_t o = __builtin_amdgcn_make_buffer_rsrc(corner, 0, (int)(((rows - 1) * ldo + cols) * ES), 0x00020000);
#pragma unroll
    for (int j = 0; j < NI; j += STEP) {
        const int n = RUN ? 16 * q4 + 4 * j : 16 * j + 4 * q4;
        f4 add[STEP];
#pragma unroll
        for (int h = 0; h < STEP; ++h) {
            add[h] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            if (bias)
#pragma unroll
                for (int e = 0; e < 4; ++e) add[h][e] = bias[min(n + 4 * h + e, cols - 1)];
        }
        const uint32_t at = n < cols ? (l16 * (uint32_t)ldo + n) * ES : BEHIND;
        uint8_t *p = corner + (l16 * ldo + n) * ES;
#pragma unroll
        for (int i = 0; i < MI; ++i, p += 16 * ldo * ES) {
            if (!WHOLE) __builtin_amdgcn_sched_barrier(0);       // (one row's addresses at a time)
            uint32_t w[TO == SC_F32 ? 4 : 2 * STEP];
#pragma unroll
            for (int h = 0; h < STEP; ++h) {
                const f4 v = acc[i][j + h] + add[h];
                if (TO == SC_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[TO == SC_F32 ? e : 0] = __float_as_uint(v[e]);
                } else {
                    w[2 * h] = to_pair(TO, v[0], v[1]);
                    w[2 * h + 1] = to_pair(TO, v[2], v[3]);
                }
            }
            constexpr int WORDS = TO == SC_F32 ? 4 : 2 * STEP;
            if (WHOLE) {
                const uint32_t to = at + (uint32_t)i * 16u * (uint32_t)ldo * ES;
                if (WORDS == 4) __builtin_amdgcn_raw_buffer_store_b128(u4{w[0], w[1], w[WORDS - 2], w[WORDS - 1]}, o, to, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b64(u2{w[0], w[1]}, o, to, 0, 0);
            } else if (16 * i + l16 < rows && n < cols) {
                if (n + 4 * STEP <= cols) {
                    if (WORDS == 4) *reinterpret_cast<u4_any *>(p) = u4{w[0], w[1], w[WORDS - 2], w[WORDS - 1]};
                    else *reinterpret_cast<u2_any *>(p) = u2{w[0], w[1]};
                } else {
#pragma unroll
                    for (int e = 0; e < 4 * STEP; ++e) {
                        if (n + e >= cols) continue;
                        if (TO == SC_F32) reinterpret_cast<uint32_t *>(p)[e] = w[e & 3];
                        else reinterpret_cast<uint16_t *>(p)[e] = (uint16_t)(w[(e >> 1) % WORDS] >> (16 * (e & 1)));
                    }
                }
            }
        }
    }
}
// (BF, REST: results are bfloat16; float32 and float16)
template <bool BF, bool REST, bool RUN, int MI, int NI>
__device__ __forceinline__ void store_tile(const GemmArgs &g, int b, int64_t m0, int64_t n0, int l16, int q4, const f4 (&acc)[MI][NI]) {
    const int rows = (int)min(g.M - m0, (int64_t)(16 * MI)), cols = (int)min(g.N - n0, (int64_t)(16 * NI));
    if (rows <= 0 || cols <= 0) return;
    uint8_t *corner = static_cast<uint8_t *>(g.out) + (b * g.strideO + m0 * g.ldo + n0) * (REST && g.typeO == SC_F32 ? 4 : 2);
    const float *bias = g.bias ? g.bias + b * g.strideBias + n0 : nullptr;
    if (BF && (!REST || g.typeO == SC_BF16)) {
        if (g.whole) store_rows<SC_BF16, true, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
        else store_rows<SC_BF16, false, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
    } else if (g.typeO == SC_F32) {
        if (g.whole) store_rows<SC_F32, true, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
        else store_rows<SC_F32, false, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
    } else {
        if (g.whole) store_rows<SC_F16, true, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
        else store_rows<SC_F16, false, RUN>(corner, bias, rows, cols, g.ldo, l16, q4, acc);
    }
}

// A tile of BM x BN outputs by waves of WM x WN each, one block after the other by the same threads.  A scale block is
// one stage: the matrix cores sum its 128 products from zero and the sum enters the accumulators times its two
// scales.  A stage's operands and scales are copied to LDS while the stage before it is multiplied.
// BLOCKB: the rows of B share a scale by 128, so a wave's columns have one.
// Bound by LDS reads and the scaling of the sums between matrix instructions (18464 x 4096 x 1024 to bfloat16: 101 us, 1534 TFLOP/s);
// EXACT by the conversions (4608 x 1152 x 4096: 68 us, 643 TFLOP/s).
template <int TA, int TB, bool EXACT, bool BLOCKB, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64, 2) void k_fp8_gemm(GemmArgs g, uint32_t tiles) {
    constexpr int NW = (BM / WM) * (BN / WN), MI = WM / 16, NI = WN / 16, ROWS = BM + BN;
    constexpr int WR = ROWS / NW, CH = WR / 8;      // rows that a wave copies of each stage, eight at a time
    constexpr bool ALONE = BM == 256;               // a block to a compute unit
    constexpr int EARLY = ALONE ? 4 : 1;            // a stage is sent for during the first 1 / EARLY of the row groups
    static_assert(NI == 4 && WR == 64 && BM % WR == 0, "a wave copies rows of one operand, and a scale for each of its lanes");
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
        off[k] = (uint32_t)r * (uint32_t)ld + 16u * ((lane & 7) ^ (forB ? swz_b(r) : swz(r)));
    }
    const uint32_t soff = 4u * (uint32_t)((r0 + lane) >> shift) * (uint32_t)lds;
    // the next stage to copy: stage ct of the tile (cb, cm, cn)
    Buffer from, sfrom;
    uint32_t next = blockIdx.x;
    int cb, cm, cn, ct = 0;
    const auto enter = [&]() {
        tile_at(next, tiles, g.tilesM, g.tilesN, &cb, &cm, &cn);
        const int64_t x0 = forB ? (int64_t)cn * BN : (int64_t)cm * BM, rows = min((int64_t)(forB ? BN : BM), all - x0);
        // (up to the end of the dword that holds the last row's last byte; what it holds behind K becomes zero below)
        from = buffer_of(src + cb * stride + x0 * ld, (rows - 1) * ld + (g.K + 3) / 4 * 4);
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
    // Where some blocks have a tile less than others, those start a part of a tile later (two sleeps, 7 us; the shortest
    // tile takes that): else the whole chip stores its outputs at the same time, and multiplies nothing meanwhile
    // (18464 x 4096 x 1024: 124 us at once, 113 with one sleep, 101 with two, 101 with three).
    if (const uint32_t more = tiles % gridDim.x; ALONE && tiles > gridDim.x && more != 0 && blockIdx.x >= more) {
        __builtin_amdgcn_s_sleep(127);
        __builtin_amdgcn_s_sleep(127);
    }
    enter();
#pragma unroll
    for (int k = 0; k < CH; ++k) copy(0, k);
    copy_scales(0);
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
                    const int r = r0 + 8 * k + (lane >> 3), left = cut - 16 * ((lane & 7) ^ (forB ? swz_b(r) : swz(r)));
                    *p &= u4{bytes_before(left), bytes_before(left - 4), bytes_before(left - 8), bytes_before(left - 12)};
                }
            }
            __syncthreads();          // everyone's copies have arrived, and the other buffer has been read
            advance();
            // Row group i is multiplied while group i + 1 is read, a part of the next stage is sent for and the sums of group
            // i - 1 are scaled.  The fences hold that order (one a row group where two blocks share a compute unit and fill each
            // other's gaps): left to itself the compiler would draw the reads together, into more registers than there are.
            const u4 *s = sm[buf];
            Frag<TB, EXACT> fb[NI];
            Frag<TA, EXACT> fa[2];
            f4 sb[BLOCKB ? 1 : NI], p[2][NI];
            float sa[3];
            const auto read = [&](auto &f, int r, int z) { f.set(s[r * 8 + (q4 ^ z)], s[r * 8 + ((q4 + 4) ^ z)]); };
            const auto read_a = [&](int i) { read(fa[i & 1], wm + 16 * i + l16, swz(l16)); };
            read_a(0);
#pragma unroll
            for (int j = 0; j < NI; ++j) read(fb[j], BM + wn + fragment_row(l16, j), swz_b(fragment_row(l16, j)));
            if (BLOCKB) {
                sb[0] = f4{sc[buf][BM + wn], 0.0f, 0.0f, 0.0f};
            } else {
#pragma unroll
                for (int j = 0; j < NI; ++j) sb[j] = *reinterpret_cast<const f4 *>(&sc[buf][BM + wn + 16 * q4 + 4 * j]);
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
                    read_a(i + 1);
                    sa[(i + 1) % 3] = sc[buf][wm + 16 * (i + 1) + l16];
                }
#pragma unroll
                for (int k = i * CH / MI * EARLY; k < (i + 1) * CH / MI * EARLY; ++k)
                    if (k < CH) copy(buf ^ 1, k);
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    p[i & 1][j] = mma_128(fb[j], fa[i & 1]);
                    if (ALONE && i > 0) add(i - 1, j);
                    if (ALONE) __builtin_amdgcn_sched_barrier(0);
                }
                if (BLOCKB) sa[i % 3] *= sb[0][0];
                if (!ALONE) {
#pragma unroll
                    for (int j = 0; j < NI; ++j) add(i, j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (ALONE)
#pragma unroll
                for (int j = 0; j < NI; ++j) add(MI - 1, j);
            buf ^= 1;
        }
        store_tile<!EXACT, EXACT, true>(g, b, m0 + wm, n0 + wn, l16, q4, acc);
    }
}

// Up to 16 rows: a block has 16 MI x 16 NI outputs, and its eight waves deal the
// blocks of 128 among themselves.  A wave takes its fragments from memory as they lie (a row's 128 bytes by four lanes, 64 of
// them at a time), the next block's while one is multiplied; the eight sums are joined in LDS in order.  Results of every type
// take the 16-bit products (Frag): latency bounds it, and the conversions hide behind it but for a little (in a graph 1 x 4608 x 1152
// 7.2 us, 6.9 by 8-bit products; 16 x 16384 x 4096 29.9 and 29.0; 16 x 65536 x 2048 69.1 and 66.5, 1.9 TB/s).
constexpr int DW = 8;
template <int TA, int TB, int MI, int NI>
__global__ __launch_bounds__(64 * DW) void k_fp8_direct(GemmArgs g, uint32_t tiles) {
    __shared__ f4 join[DW][MI * NI][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q4 = lane >> 4;
    if (block_id() >= tiles) return;
    const int64_t m0 = (int64_t)(block_id() % (uint32_t)g.tilesM) * (16 * MI), n0 = (int64_t)(block_id() / (uint32_t)g.tilesM) * (16 * NI);
    for (int b = blockIdx.z; b < g.batch; b += gridDim.z) {
        const uint8_t *A = g.A + b * g.strideA, *B = g.B + b * g.strideB;
        const float *sA = g.sA + b * g.strideSA, *sB = g.sB + b * g.strideSB;
        // (rows behind the last read the last one; their outputs are not stored)
        uint32_t ra[MI], rb[NI], sb[NI];
#pragma unroll
        for (int i = 0; i < MI; ++i) ra[i] = (uint32_t)min(m0 + 16 * i + l16, (int64_t)g.M - 1);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            rb[j] = (uint32_t)min(n0 + 16 * j + l16, (int64_t)g.N - 1);
            sb[j] = (uint32_t)min(n0 + 16 * j + 4 * q4, (int64_t)g.N - 1);
        }
        f4 acc[MI][NI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        struct Block {
            u4 a[MI][2], b[NI][2];
            float sa[MI];
            f4 sb[NI];
        };
        const auto fetch = [&](Block &f, int t) {
            const int k = 128 * t + 16 * q4;
            if (128 * t + 128 <= g.K) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) f.a[i][h] = *reinterpret_cast<const u4_any *>(A + ra[i] * g.lda + k + 64 * h);
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) f.b[j][h] = *reinterpret_cast<const u4_any *>(B + rb[j] * g.ldb + k + 64 * h);
            } else {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) f.a[i][h] = load_granule(A + ra[i] * g.lda, k + 64 * h, g.K);
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) f.b[j][h] = load_granule(B + rb[j] * g.ldb, k + 64 * h, g.K);
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) f.sa[i] = sA[(ra[i] >> g.shiftA) * g.ldsA + t];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if (g.shiftB) {
                    const float s = sB[(sb[j] >> 7) * g.ldsB + t];
                    f.sb[j] = f4{s, s, s, s};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) f.sb[j][e] = sB[min(sb[j] + e, (uint32_t)g.N - 1u) * g.ldsB + t];
                }
            }
        };
        const auto multiply = [&](const Block &f) {
            Frag<TB, true> fb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) fb[j].set(f.b[j][0], f.b[j][1]);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                Frag<TA, true> fa;
                fa.set(f.a[i][0], f.a[i][1]);
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const f4 p = mma_128(fb[j], fa);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], f.sa[i] * f.sb[j][e], acc[i][j][e]);
                }
            }
        };
        Block now, then;
        if (wave < g.KB) fetch(now, wave);
        for (int t = wave; t < g.KB; t += DW) {
            if (t + DW < g.KB) fetch(then, t + DW);
            multiply(now);
            now = then;
        }
        __syncthreads();                 // (the last batch entry's sums have been read)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) join[wave][i * NI + j][lane] = acc[i][j];
        __syncthreads();
        for (int x = wave; x < MI * NI; x += DW) {
            f4 v[1][1] = {{join[0][x][lane]}};
#pragma unroll
            for (int w = 1; w < DW; ++w) v[0][0] += join[w][x][lane];
            store_tile<true, true, false>(g, b, m0 + 16 * (x / NI), n0 + 16 * (x % NI), l16, q4, v);
        }
    }
}

// Too few tiles for every compute unit, or operands off 16 bytes: a block has 64 x 64 outputs, and KG groups of four waves
// take every KG-th block of 128 each, through registers (which take any alignment) into two stages of LDS of their own, the
// next block's loads in flight while one is multiplied; the groups' sums are joined in LDS in order.  Where tiles are few and K is
// long, g.parts blocks share a tile's stages and k_fp8_join adds their sums.  Bound by latency, about 0.8 us a stage
// (577 x 1000 x 1031 to float32: 10.4 us).
template <int TA, int TB, bool EXACT, int KG>
__global__ __launch_bounds__(256 * KG) void k_fp8_parts(GemmArgs g, uint32_t tiles) {
    constexpr int T = 64, G = 2 * T * 8 / 256;       // granules a thread
    __shared__ u4 sm[KG][2][2 * T * 8];
    __shared__ float sc[KG][2][2 * T];
    const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255, lane = tid & 63, wave = tid >> 6,
              l16 = lane & 15, q4 = lane >> 4, wm = 32 * (wave & 1), wn = 32 * (wave >> 1);
    uint32_t tile = block_id(), part = 0;
    int t0 = 0, t1 = g.KB;
    if (g.parts > 1) {
        part = tile / tiles;
        tile -= part * tiles;
        t0 = (int)(part * (uint32_t)g.KB / (uint32_t)g.parts);
        t1 = (int)((part + 1) * (uint32_t)g.KB / (uint32_t)g.parts);
    }
    if (tile >= tiles || part >= (uint32_t)g.parts) return;
    const int64_t m0 = (int64_t)(tile % (uint32_t)g.tilesM) * T, n0 = (int64_t)(tile / (uint32_t)g.tilesM) * T;
    for (int b = blockIdx.z; b < g.batch; b += gridDim.z) {
        const uint8_t *row[G];
#pragma unroll
        for (int k = 0; k < G; ++k) {
            const int r = (k * 256 + tid) >> 3;      // (rows behind the last read the last one; their outputs are not stored)
            row[k] = k < G / 2 ? g.A + b * g.strideA + min(m0 + r, (int64_t)g.M - 1) * g.lda
                               : g.B + b * g.strideB + min(n0 + r - T, (int64_t)g.N - 1) * g.ldb;
        }
        const float *scale = tid < T ? g.sA + b * g.strideSA + (min(m0 + tid, (int64_t)g.M - 1) >> g.shiftA) * g.ldsA
                                     : g.sB + b * g.strideSB + (min(n0 + (tid & (T - 1)), (int64_t)g.N - 1) >> g.shiftB) * g.ldsB;
        f4 acc[2][2] = {};
        u4 r[G];
        float s = 0.0f;
        const auto load = [&](int t) {
#pragma unroll
            for (int k = 0; k < G; ++k) r[k] = load_granule(row[k], 128 * t + 16 * (tid & 7), g.K);
            if (tid < 2 * T) s = scale[t];
        };
        const auto put = [&](int buf) {
#pragma unroll
            for (int k = 0; k < G; ++k) {
                const int x = (k * 256 + tid) >> 3;
                sm[grp][buf][x * 8 + ((tid & 7) ^ swz(x))] = r[k];
            }
            if (tid < 2 * T) sc[grp][buf][tid] = s;
        };
        __syncthreads();                             // (the last batch entry's sums have been read)
        if (t0 + grp < t1) {
            load(t0 + grp);
            put(0);
        }
        int buf = 0;
        for (int t = t0 + grp; t - grp < t1; t += KG, buf ^= 1) {
            __syncthreads();
            const bool more = t + KG < t1;
            if (more) load(t + KG);
            if (t < t1) {
                const u4 *p = sm[grp][buf];
                const auto read = [&](auto &f, int x) { f.set(p[x * 8 + (q4 ^ swz(x))], p[x * 8 + ((q4 + 4) ^ swz(x))]); };
                Frag<TB, EXACT> fb[2];
                f4 sb[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    read(fb[j], T + wn + 16 * j + l16);
                    sb[j] = *reinterpret_cast<const f4 *>(&sc[grp][buf][T + wn + 16 * j + 4 * q4]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    Frag<TA, EXACT> fa;
                    read(fa, wm + 16 * i + l16);
                    const float sa = sc[grp][buf][wm + 16 * i + l16];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f4 d = mma_128(fb[j], fa);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(d[e], sa * sb[j][e], acc[i][j][e]);
                    }
                }
            }
            if (more) put(buf ^ 1);
        }
        if (KG > 1) {
            f4 *join = reinterpret_cast<f4 *>(sm);   // [KG - 1][4][256]
            __syncthreads();
            if (grp > 0)
#pragma unroll
                for (int x = 0; x < 4; ++x) join[((grp - 1) * 4 + x) * 256 + tid] = acc[x >> 1][x & 1];
            __syncthreads();
            if (grp > 0) continue;
#pragma unroll
            for (int w = 0; w < KG - 1; ++w)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[x >> 1][x & 1] += join[(w * 4 + x) * 256 + tid];
        }
        if (g.parts == 1) {
            store_tile<!EXACT, EXACT, false>(g, b, m0 + wm, n0 + wn, l16, q4, acc);
        } else if (m0 + wm < g.M && n0 + wn < g.N) {
            const int rows = (int)min(g.M - m0 - wm, (int64_t)32), cols = (int)min(g.N - n0 - wn, (int64_t)32);
            float *corner = g.part + (((int64_t)part * g.batch + b) * g.M + m0 + wm) * g.N + n0 + wn;
            store_rows<SC_F32, false, false>(reinterpret_cast<uint8_t *>(corner), nullptr, rows, cols, g.N, l16, q4, acc);
        }
    }
}
// The parts' sums added in order, and the bias: four columns a thread.  Memory-bound.
__global__ __launch_bounds__(256) void k_fp8_join(GemmArgs g) {
    const int quads = (g.N + 3) / 4;
    const int64_t at = (int64_t)block_id() * 256 + threadIdx.x, row = at / quads, entry = (int64_t)g.batch * g.M;
    if (row >= entry) return;
    const int n = 4 * (int)(at - row * quads), left = g.N - n;
    const int64_t b = row / g.M, i = row - b * g.M;
    f4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = 0; k < g.parts; ++k) s += to_floats(SC_F32, load_raw<false>(SC_F32, g.part, (k * entry + row) * g.N + n, left));
    if (g.bias) s += to_floats(SC_F32, load_raw<false>(SC_F32, g.bias, b * g.strideBias + n, left));
    store4<false>(g.typeO, g.out, b * g.strideO + i * g.ldo + n, s, left);
}

template <int TA, int TB, bool EXACT, bool BLOCKB, int BM, int BN, int WM, int WN>
static void launch_tile(GemmArgs g, int per_cu, hipStream_t st) {
    g.tilesM = (int)(((int64_t)g.M + BM - 1) / BM);
    g.tilesN = (int)(((int64_t)g.N + BN - 1) / BN);
    const uint32_t tiles = (uint32_t)g.tilesM * (uint32_t)g.tilesN * (uint32_t)g.batch, most = 256u * per_cu;
    hipLaunchKernelGGL((k_fp8_gemm<TA, TB, EXACT, BLOCKB, BM, BN, WM, WN>), dim3(tiles < most ? tiles : most), dim3((BM / WM) * (BN / WN) * 64),
                       0, st, g, tiles);
}
template <int TA, int TB, int MI, int NI>
static void launch_direct(GemmArgs g, hipStream_t st) {
    g.tilesM = (int)(((int64_t)g.M + 16 * MI - 1) / (16 * MI));
    g.tilesN = (int)(((int64_t)g.N + 16 * NI - 1) / (16 * NI));
    const uint32_t tiles = (uint32_t)g.tilesM * (uint32_t)g.tilesN;
    hipLaunchKernelGGL((k_fp8_direct<TA, TB, MI, NI>), grid_of(tiles, g.batch), dim3(64 * DW), 0, st, g, tiles);
}
template <int TA, int TB, bool EXACT, int KG>
static void launch_parts(GemmArgs g, hipStream_t st) {
    g.tilesM = (int)(((int64_t)g.M + 63) / 64);
    g.tilesN = (int)(((int64_t)g.N + 63) / 64);
    const uint32_t tiles = (uint32_t)g.tilesM * (uint32_t)g.tilesN;
    hipLaunchKernelGGL((k_fp8_parts<TA, TB, EXACT, KG>), grid_of(tiles * (uint32_t)g.parts, g.batch), dim3(256 * KG), 0, st, g, tiles);
    if (g.parts > 1) {
        const int64_t quads = (int64_t)g.batch * g.M * ((g.N + 3) / 4);
        hipLaunchKernelGGL(k_fp8_join, grid_of((uint32_t)((quads + 255) / 256), 1), dim3(256), 0, st, g);
    }
}
// An operand whose rows do not start on 16 bytes, laid out anew: rows of whole blocks of 128, zeros behind K.  Memory-bound,
// and worth it where many tiles read every row (4608 x 1152 x 4099 to bfloat16: 54 us with it; 39 for 4096, whose rows lie as they
// should).
__global__ __launch_bounds__(256) void k_fp8_lay(const uint8_t *src, int64_t ld, int64_t stride, int rows, int K, int KB, int batch,
                                                 uint8_t *dst) {
    const int64_t each = (int64_t)rows * KB * 8, all = each * batch, at = (int64_t)block_id() * 256 + threadIdx.x;
    if (at >= all) return;
    const int64_t b = at / each, in = at - b * each, row = in / (KB * 8);
    const int q = (int)(in - row * (KB * 8));
    reinterpret_cast<u4 *>(dst)[at] = load_granule(src + b * stride + row * ld, 16 * q, K);
}

// How a product is done.  Tiles of 128 x 128 (two blocks to a compute unit) or, for bfloat16 results, 256 x 256 (one) where there
// are enough for half of the compute units; their rows have to start 16 bytes apart, or are laid out so first.  Few tiles, or an address off 16:
// 64 x 64 by groups of waves (so too K = 0, a product of the bias alone).  Up to 16 rows: without LDS.
enum { DIRECT, PARTS, TILES };
static int64_t tiles_of(const GemmArgs &g, int side) { return ((int64_t)g.M + side - 1) / side * (((int64_t)g.N + side - 1) / side) * g.batch; }
static bool rows_aligned(int64_t ld, int64_t stride, int batch) { return ld % 16 == 0 && (batch == 1 || stride % 16 == 0); }
static int way_of(const GemmArgs &g) {
    if (g.M <= 16) return DIRECT;
    if (g.KB == 0) return PARTS;
    const int64_t tiles = tiles_of(g, 128);
    // (copies to LDS and a tile's scales have 32-bit offsets)
    return tiles < 128 || tiles > INT32_MAX / 4 || g.ldsA > 1 << 21 || g.ldsB > 1 << 21 ? PARTS : TILES;
}
static size_t laid_bytes(int rows, int KB, int64_t stride, int batch) {
    return (size_t)rows * KB * 128 * (stride == 0 ? 1 : batch);
}
// Blocks that share a tile's stages: one for each compute unit, three stages or more to each of a block's two groups, if that takes
// ten stages from every group; fewer cost less than the second launch (100 x 1152 x 4608 to bfloat16: 17.4 us alone, 11.6 in six parts;
// 64 x 256 x 8192 27.3 and 11.3; 256 x 2048 x 8192 30.6 and 22.9; but 17 x 1024 x 2048 9.7 and 11.2 in two).
static int parts_of(const GemmArgs &g) {
    const int64_t tiles = tiles_of(g, 64);
    if (way_of(g) != PARTS || tiles > 128) return 1;
    const int parts = (int)(256 / tiles < g.KB / 6 ? 256 / tiles : g.KB / 6);
    return parts > 1 && g.KB * (parts - 1) >= 20 * parts ? parts : 1;
}
static size_t part_bytes(const GemmArgs &g) {
    const int parts = parts_of(g);
    return parts == 1 ? 0 : (size_t)parts * g.batch * g.M * g.N * sizeof(float);
}
// bytes that the operands take that have to be laid out, A's first
static void lay_sizes(const GemmArgs &g, size_t *a, size_t *b) {
    const bool tiles = way_of(g) == TILES;
    *a = tiles && (!rows_aligned(g.lda, g.strideA, g.batch) || g.lda > 1 << 22) ? laid_bytes(g.M, g.KB, g.strideA, g.batch) : 0;
    *b = tiles && (!rows_aligned(g.ldb, g.strideB, g.batch) || g.ldb > 1 << 22) ? laid_bytes(g.N, g.KB, g.strideB, g.batch) : 0;
    *a = (*a + 255) / 256 * 256;
}
static hipError_t lay(const uint8_t **p, int64_t *ld, int64_t *stride, int rows, const GemmArgs &g, uint8_t *dst, hipStream_t st) {
    const int batch = *stride == 0 ? 1 : g.batch;
    const int64_t granules = (int64_t)rows * g.KB * 8 * batch;
    hipLaunchKernelGGL(k_fp8_lay, grid_of((uint32_t)((granules + 255) / 256), 1), dim3(256), 0, st, *p, *ld, *stride, rows, g.K, g.KB, batch, dst);
    *p = dst;
    *ld = (int64_t)g.KB * 128;
    *stride = *stride == 0 ? 0 : (int64_t)rows * g.KB * 128;
    return hipGetLastError();
}

template <int TA, int TB, bool EXACT>
static hipError_t launch_gemm(const GemmArgs &g, hipStream_t st) {
    const bool tiled = way_of(g) == TILES && aligned_to(g.A, 16) && aligned_to(g.B, 16) && rows_aligned(g.lda, g.strideA, g.batch) &&
                       rows_aligned(g.ldb, g.strideB, g.batch);
    if (way_of(g) == DIRECT) {
        launch_direct<TA, TB, 1, 1>(g, st);
    } else if (!tiled) {
        // one group of waves where there are tiles for all anyway (577 x 4096 x 1024: 16.9 us, 20.5 with two), else two
        // (256 x 4096 x 4096: 23.1 us, 24.2 with one; 577 x 1024 x 4096: 17.9, 23.0)
        if (tiles_of(g, 64) > 512) launch_parts<TA, TB, EXACT, 1>(g, st);
        else launch_parts<TA, TB, EXACT, 2>(g, st);
    } else {
        // Microseconds by what was measured: a stage of a round of tiles and what a round costs besides (8192 x 8192 x 8192 takes
        // 532 us in 256 x 256 tiles and 716 in 128 x 128; 8192 x 4096 x 4096 151 and 189; 18464 x 4096 x 1024 104 and 118; 4096 x 4608 x 1152
        // is the faster in 128 x 128, 40 against 51).  With a scale for each row of B both cost more, the 256 x 256 tiles spill 15 registers,
        // and the order is the same: 647 and 816, 179 and 214, 116 and 123.
        const double big = (double)((tiles_of(g, 256) + 255) / 256) * (2.0 * g.KB + 5.6),
                     small = (double)((tiles_of(g, 128) + 511) / 512) * (1.225 * g.KB + 1.2);
        if (EXACT || small < big) {
            if (g.shiftB) launch_tile<TA, TB, EXACT, true, 128, 128, 64, 64>(g, 2, st);
            else launch_tile<TA, TB, EXACT, false, 128, 128, 64, 64>(g, 2, st);
        } else {
            if (g.shiftB) launch_tile<TA, TB, false, true, 256, 256, 128, 64>(g, 1, st);
            else launch_tile<TA, TB, false, false, 256, 256, 128, 64>(g, 1, st);
        }
    }
    return hipGetLastError();
}
template <bool EXACT>
static hipError_t launch_gemm_types(const GemmArgs &g, int typeA, int typeB, hipStream_t st) {
    if (typeA == SC_E4M3) return typeB == SC_E4M3 ? launch_gemm<0, 0, EXACT>(g, st) : launch_gemm<0, 1, EXACT>(g, st);
    return typeB == SC_E4M3 ? launch_gemm<1, 0, EXACT>(g, st) : launch_gemm<1, 1, EXACT>(g, st);
}

static GemmArgs gemm_args(const sc_fp8_gemm_desc &d) {
    GemmArgs g{};
    g.M = d.M;
    g.N = d.N;
    g.K = d.K;
    g.KB = (d.K + FP8_BLOCK - 1) / FP8_BLOCK;
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
    g.batch = d.batch;
    g.parts = 1;
    return g;
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
    if (!rows_apart(d->batch, d->strideO, d->M, d->ldo, d->N)) return SC_ERR_STRIDE;
    const int64_t tiles = (((int64_t)d->M + 63) / 64) * (((int64_t)d->N + 31) / 32);
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
    if (rows > 0 && K > 0 && (!rows_apart(batch, strideQ, qrows, ldq, qcols) || !rows_apart(batch, strideS, srows, lds, scols)))
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
    if (desc->batch == 0 || desc->M == 0 || desc->N == 0) return SC_OK;
    size_t a, b;
    const GemmArgs g = gemm_args(*desc);
    lay_sizes(g, &a, &b);
    *bytes = a + b + part_bytes(g);        // (never both)
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
    GemmArgs g = gemm_args(d);
    g.A = static_cast<const uint8_t *>(A);
    g.B = static_cast<const uint8_t *>(B);
    g.sA = sA;
    g.sB = sB;
    g.bias = bias;
    g.out = out;
    const int eb = type_bytes(d.typeO), run = 16 / eb;       // outputs of a 16-byte store
    g.whole = aligned_to(out, 16) && d.N % run == 0 && d.ldo % run == 0 && (d.batch == 1 || d.strideO % run == 0) && d.ldo <= 1 << 20;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    size_t la, lb;
    lay_sizes(g, &la, &lb);
    // (an operand that starts off 16 bytes, which its strides do not say, keeps both from the tiles that the other is laid out for)
    if ((la == 0 && !aligned_to(A, 16)) || (lb == 0 && !aligned_to(B, 16))) la = lb = 0;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (la > 0 && lay(&g.A, &g.lda, &g.strideA, g.M, g, ws, st) != hipSuccess) return SC_ERR_HIP;
    if (lb > 0 && lay(&g.B, &g.ldb, &g.strideB, g.N, g, ws + la, st) != hipSuccess) return SC_ERR_HIP;
    g.parts = parts_of(g);
    if (g.parts > 1) g.part = static_cast<float *>(workspace);
    if (la > 0 && lb > 0) g.K = g.KB * 128;         // (both operands have zeros there now)
    const hipError_t e = d.typeO == SC_BF16 ? launch_gemm_types<false>(g, d.typeA, d.typeB, st) : launch_gemm_types<true>(g, d.typeA, d.typeB, st);
    return e == hipSuccess ? SC_OK : SC_ERR_HIP;
}

}  // extern "C"
