// Kernels of include/tuna_moe.h in 4 bits for gfx950: rows and columns as e2m1 with a power of two for each 32 of them, read back, and multiplied.
// Times in these comments are averages over a kernel trace.
#pragma once
#include "moe_common.h"

namespace moe {

typedef float v2f __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------------------ quantisation

// The magnitude of a value as bits, whose order is that of the magnitudes: infinity above all finite ones, NaN above infinity.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// The scale byte of a block whose largest magnitude has these bits.  With a = f 2^e, 1 <= f < 2: a / 6 = f / 1.5 * 2^(e - 2), so the power of two that
// is not below is 2^(e - 2) for f <= 1.5 and 2^(e - 1) above, which a carry out of the fraction says.
__device__ __forceinline__ unsigned scale4_of(unsigned peak) {
    const int s = (int)((peak + 0x3fffffu) >> 23) - 2;
    return peak >= 0x7f800000u ? 255u : peak == 0u ? 127u : (unsigned)(s < 1 ? 1 : s);
}
__device__ __forceinline__ float power_of(unsigned s) { return __uint_as_float(s << 23); }        // 0 and 255 too, as the conversions read them

// Eight values as e2m1, the first in the lowest bits; to nearest, ties to even, by the conversion itself.  A block that is not finite: zeros.
__device__ __forceinline__ unsigned pack8(const float (&v)[8], unsigned s) {
    const float p = power_of(s);
    unsigned q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], p, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], p, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], p, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], p, 3);
    return s == 255u ? 0u : q;
}

// Up to eight packed values; what is behind the row's end is zero already.
template <bool WIDE> __device__ __forceinline__ void store_packed(uint8_t* d, unsigned q, int64_t left) {
    if (WIDE && left >= 8) {
        *(unsigned*)d = q;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (2 * i < left) d[i] = (uint8_t)(q >> (8 * i));
}

// Four lanes per block of 32 values, eight each; U blocks in turn, whose loads are under way together.
template <class T, int ACT, bool WIDE, int U>
__global__ __launch_bounds__(256) void k_fp4_quantise(const T* x, int64_t ldx, unsigned total, int64_t cols, const int32_t* slots, int copies, int64_t out_rows,
                                                      uint8_t* q, int64_t ldq, uint8_t* scales, int64_t ld_scales) {
    const unsigned nb = (unsigned)((cols + kBlock4 - 1) / kBlock4), at0 = blockIdx.x * (64 * U) + (threadIdx.x >> 2);
    float v[U][8], up[U][8];
    unsigned row[U], block[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = at0 + u * 64 < total ? at0 + u * 64 : total - 1;
        row[u] = at / nb;
        block[u] = at - row[u] * nb;
        const int64_t c = (int64_t)block[u] * kBlock4 + (threadIdx.x & 3) * 8;
        const T* p = x + row[u] * ldx + c;
        load8<WIDE>(p, cols - c, v[u]);
        if (ACT == TUNA_ACT_SWIGLU) load8<WIDE>(p + cols, cols - c, up[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (at0 + u * 64 >= total) break;                         // (four lanes together)
        const int64_t r = row[u], b = block[u], c = b * kBlock4 + (threadIdx.x & 3) * 8, left = cols - c;
        if (ACT == TUNA_ACT_SWIGLU) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = i < left ? gate_of(v[u][i]).silu * up[u][i] : 0.f;
        }
        unsigned peak = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) peak = larger(peak, magnitude(v[u][i]));
        peak = larger(peak, (unsigned)__shfl_xor((int)peak, 1));
        peak = larger(peak, (unsigned)__shfl_xor((int)peak, 2));
        const unsigned s = scale4_of(peak), o = pack8(v[u], s);
        for (int j = 0; j < copies; ++j) {
            int64_t to = r;
            if (slots) {
                to = slots[r * copies + j];
                if (to < 0 || to >= out_rows) continue;
            }
            store_packed<WIDE>(q + to * ldq + c / 2, o, left);
            if ((threadIdx.x & 3) == 0) scales[to * ld_scales + b] = (uint8_t)s;
        }
    }
}

// A tile of 128 rows by 128 columns: a thread has 8 x 8 of them, a wave's four rows of threads have 32 rows, one block of each column.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_fp4_quantise_columns(const T* x, int64_t ldx, int64_t rows, int64_t cols, const int32_t* group_rows, int groups,
                                                              uint8_t* q, int64_t ldq, uint8_t* scales, int64_t ld_scales) {
    __shared__ __align__(16) unsigned tile[kBlock][20];           // a column's 64 bytes, and its four scales behind them
    const Place pl = find_tile(group_rows, groups, rows, kBlock, blockIdx.x);
    if (pl.group < 0) return;
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.y * kBlock + cx * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = pl.first + ry * 8 + i;
        if (r < pl.end && c < cols) load8<WIDE>(x + r * ldx + c, cols - c, v[i]);
        else for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float col[8];
        unsigned peak = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            col[i] = v[i][j];
            peak = larger(peak, magnitude(col[i]));
        }
        peak = larger(peak, (unsigned)__shfl_xor((int)peak, 16));
        peak = larger(peak, (unsigned)__shfl_xor((int)peak, 32));
        const unsigned s = scale4_of(peak);
        tile[cx * 8 + j][ry] = pack8(col, s);
        if ((ry & 3) == 0) ((uint8_t*)&tile[cx * 8 + j][16])[ry >> 2] = (uint8_t)s;
    }
    __syncthreads();
    const bool wide = (((uintptr_t)q | (uintptr_t)ldq) & 15) == 0;
    for (int i = threadIdx.x; i < kBlock * 4; i += 256) {
        const int row = i >> 2, ch = i & 3;
        const int64_t to = (int64_t)blockIdx.y * kBlock + row;
        if (to >= cols) continue;
        uint8_t* d = q + to * ldq + pl.block * 64 + ch * 16;
        const v4u val = *(const v4u*)&tile[row][ch * 4];
        if (wide) *(v4u*)d = val;
        else for (int b = 0; b < 16; ++b) d[b] = (uint8_t)(val[b >> 2] >> (8 * (b & 3)));
        scales[to * ld_scales + pl.block * 4 + ch] = ((const uint8_t*)&tile[row][16])[ch];
    }
}

// Eight packed values times their scale; exact.
__device__ __forceinline__ void unpack8(unsigned q, float p, float (&v)[8]) {
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, p, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, p, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, p, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, p, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}

// A thread per eight values, U times in turn.
template <class T, bool WIDE, int U>
__global__ __launch_bounds__(256) void k_fp4_dequantise(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t ld_scales, unsigned total, int64_t cols,
                                                        T* x, int64_t ldx) {
    const unsigned nb = (unsigned)((cols + kBlock4 - 1) / kBlock4), at0 = blockIdx.x * (64 * U) + (threadIdx.x >> 2);
    unsigned packed[U], scale[U], row[U], block[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = at0 + u * 64 < total ? at0 + u * 64 : total - 1;
        row[u] = at / nb;
        block[u] = at - row[u] * nb;
        const int64_t c = (int64_t)block[u] * kBlock4 + (threadIdx.x & 3) * 8, left = cols - c;
        const uint8_t* p = q + row[u] * ldq + c / 2;
        packed[u] = 0;
        if (WIDE && left >= 8) packed[u] = *(const unsigned*)p;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (2 * i < left) packed[u] |= (unsigned)p[i] << (8 * i);
        }
        scale[u] = scales[row[u] * ld_scales + block[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = (int64_t)block[u] * kBlock4 + (threadIdx.x & 3) * 8;
        if (at0 + u * 64 >= total || c >= cols) continue;
        float v[8];
        unpack8(packed[u], power_of(scale[u]), v);
        store8<WIDE>(x + row[u] * ldx + c, cols - c, v);
    }
}

// ------------------------------------------------------------------------------------------------ products in 4 bits

// Operands of a product out[i, j] = sum over k of a[i, k] * b[j, k].  Rows a are the activations (or dy transposed), rows b the weights
// (or x transposed).  Distances of values are in bytes.
struct Product4 {
    const uint8_t* a; int64_t lda; const uint8_t* as; int64_t ld_as;
    const uint8_t* b; int64_t ldb; int64_t b_group; const uint8_t* bs; int64_t ld_bs; int64_t bs_group;
    const int32_t* group_rows; int groups;
    void* out; int64_t ldo; int64_t out_group;
    int64_t m, n, k;                   // rows a, rows b, length (by columns: rows of all groups)
};

// 16 x 16 x 128: `b` gives the rows of the result, `a` its columns, so that a lane holds four neighbours of one row of `out`.  Lane (r, g) holds block
// number g of four of row r, sixteen bytes, and its scale in byte STEP of sb or sa.  The products are exact and added in 32 bits: measured, off by less than
// 2^-23 of the sum of their magnitudes, whatever the scales.
template <int STEP> __device__ __forceinline__ v4f mma4(const v4u& b, const v4u& a, v4f c, unsigned sb, unsigned sa) {
    const v8i wb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3]}, wa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, c, 4, 4, STEP, (int)sb, STEP, (int)sa);
}

// The simple form: a tile of 64 x 64, four waves of 16 rows each, 128 of the length at a time through the LDS; any alignment.
// COLS: the reduction is over the groups' rows (gradient of the weights).
template <bool COLS, bool WIDE, class OUT>
__global__ __launch_bounds__(256) void k_fp4_product64(Product4 P) {
    __shared__ __align__(16) uint8_t la[64][64 + 16], lb[64][64 + 16];
    __shared__ uint8_t sa[64][4], sb[64][4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int64_t i0, i_end, j0 = (int64_t)blockIdx.y * 64, kb0 = 0, kb1, length = P.k;
    int group;
    if (COLS) {
        group = blockIdx.z;
        i0 = (int64_t)blockIdx.x * 64;
        i_end = i0 + 64 < P.m ? i0 + 64 : P.m;
        int64_t count;
        group_blocks(P.group_rows, P.groups, group, P.k, kb0, count);
        kb1 = kb0 + count;
        length = kb1 * kBlock;
    } else {
        const Place pl = find_tile(P.group_rows, P.groups, P.m, 64, blockIdx.x);
        if (pl.group < 0) return;
        group = pl.group; i0 = pl.first; i_end = pl.end;
        kb1 = blocks_of(P.k);
    }
    const uint8_t* b = P.b + (COLS ? 0 : group * P.b_group);
    const uint8_t* bs = P.bs + (COLS ? 0 : group * P.bs_group);
    const int64_t blocks = (length + kBlock4 - 1) / kBlock4;
    v4f acc[4] = {};
    for (int64_t kb = kb0; kb < kb1; ++kb) {
        __syncthreads();
        for (int c = tid; c < 512; c += 256) {                    // 64 rows of a, then 64 of b, in blocks of 32 values
            const int r = (c >> 2) & 63, ch = c & 3;
            const int64_t blk = kb * 4 + ch, left = length - blk * kBlock4;
            if (c < 256) {
                const int64_t row = i0 + r < i_end ? i0 + r : i_end - 1;
                *(v4u*)&la[r][ch * 16] = chunk32<WIDE>(P.a + row * P.lda + blk * 16, left);
                sa[r][ch] = blk < blocks ? P.as[row * P.ld_as + blk] : (uint8_t)127;
            } else {
                const int64_t row = j0 + r < P.n ? j0 + r : P.n - 1;
                *(v4u*)&lb[r][ch * 16] = chunk32<WIDE>(b + row * P.ldb + blk * 16, left);
                sb[r][ch] = blk < blocks ? bs[row * P.ld_bs + blk] : (uint8_t)127;
            }
        }
        __syncthreads();
        const int r = lane & 15, g = lane >> 4;
        const v4u fa = *(const v4u*)&la[w * 16 + r][g * 16];
        const unsigned ka = sa[w * 16 + r][g];
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[s] = mma4<0>(*(const v4u*)&lb[s * 16 + r][g * 16], fa, acc[s], sb[s * 16 + r][g], ka);
    }
    const int64_t row = i0 + w * 16 + (lane & 15);
    if (row >= i_end) return;
    OUT* out = (OUT*)P.out + (COLS ? group * P.out_group : 0) + row * P.ldo;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t j = j0 + s * 16 + (lane >> 4) * 4;
        if (j < P.n) store_four(out + j, acc[s], (int)(P.n - j < 4 ? P.n - j : 4));
    }
}

}  // namespace moe
