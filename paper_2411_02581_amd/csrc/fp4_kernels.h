// Kernels of include/tuna_moe.h in 4 bits for gfx950: rows and columns as e2m1 with a power of two for each 32 of them, read back, and multiplied.
// Times in these comments are averages over a kernel trace.
#pragma once
#include "moe_common.h"

namespace moe {

typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));

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

// Two lanes per block of 32 values, sixteen each; U blocks in turn, whose loads are under way together, and the first slots with them.  Bound by memory:
// 16384 x 4096 in bf16 to two records each, 205 MB, 49 us (4.2 TB/s); gated, 20011 x 1792, 162 MB, 43 us.
template <class T, int ACT, bool WIDE, int U>
__global__ __launch_bounds__(256) void k_fp4_quantise(const T* x, int64_t ldx, unsigned total, int64_t cols, const int32_t* slots, int copies, int64_t out_rows,
                                                      uint8_t* q, int64_t ldq, uint8_t* scales, int64_t ld_scales) {
    constexpr int FIRST = 2;
    const unsigned nb = (unsigned)((cols + kBlock4 - 1) / kBlock4), at0 = blockIdx.x * (128 * U) + (threadIdx.x >> 1);
    const int mine = (threadIdx.x & 1) * 16;
    float v[U][2][8], up[U][2][8];
    unsigned row[U], block[U];
    int to_first[U][FIRST];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = at0 + u * 128 < total ? at0 + u * 128 : total - 1;
        row[u] = at / nb;
        block[u] = at - row[u] * nb;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t c = (int64_t)block[u] * kBlock4 + mine + h * 8;
            const T* p = x + row[u] * ldx + c;
            load8<WIDE>(p, cols - c, v[u][h]);
            if (ACT == TUNA_ACT_SWIGLU) load8<WIDE>(p + cols, cols - c, up[u][h]);
        }
        if (slots) {
#pragma unroll
            for (int j = 0; j < FIRST; ++j) to_first[u][j] = slots[(int64_t)row[u] * copies + (j < copies ? j : 0)];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (at0 + u * 128 >= total) break;                        // (two lanes together)
        const int64_t r = row[u], b = block[u], c = b * kBlock4 + mine, left = cols - c;
        unsigned peak = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (ACT == TUNA_ACT_SWIGLU) v[u][h][i] = h * 8 + i < left ? gate_of(v[u][h][i]).silu * up[u][h][i] : 0.f;
                peak = larger(peak, magnitude(v[u][h][i]));
            }
        peak = larger(peak, dpp<0xb1>(peak, peak));               // the other lane of the two
        const unsigned s = scale4_of(peak);
        const v2u o = {pack8(v[u][0], s), pack8(v[u][1], s)};
        auto put = [&](int64_t to) {
            uint8_t* d = q + to * ldq + c / 2;
            if (WIDE && left >= 16) {
                *(v2u*)d = o;
            } else {
                store_packed<WIDE>(d, o[0], left);
                store_packed<WIDE>(d + 4, o[1], left - 8);
            }
            if (mine == 0) scales[to * ld_scales + b] = (uint8_t)s;
        };
        if (!slots) {
            put(r);
            continue;
        }
        for (int j = 0; j < copies; ++j) {
            const int64_t to = j == 0 ? to_first[u][0] : j < FIRST ? to_first[u][1] : slots[r * copies + j];
            if (to >= 0 && to < out_rows) put(to);
        }
    }
}

// A tile of 128 rows by 128 columns: a thread has 8 x 8 of them, a wave's four rows of threads have 32 rows, one block of each column.  The packed columns go
// through the LDS, so that a store is 16 bytes of a column and not one.  Bound by memory: 10007 x 2816 in bf16, 71 MB, 19 us (3.7 TB/s).
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_fp4_quantise_columns(const T* x, int64_t ldx, int64_t rows, int64_t cols, const int32_t* group_rows, int groups,
                                                              uint8_t* q, int64_t ldq, uint8_t* scales, int64_t ld_scales) {
    __shared__ __align__(16) unsigned tile[kBlock][20];           // a column's 64 bytes, its sixteens moved on by column / 16 places; its four scales behind them
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
        tile[cx * 8 + j][(ry + (cx >> 1) * 4) & 15] = pack8(col, s);
        if ((ry & 3) == 0) ((uint8_t*)&tile[cx * 8 + j][16])[ry >> 2] = (uint8_t)s;
    }
    __syncthreads();
    const bool wide = (((uintptr_t)q | (uintptr_t)ldq) & 15) == 0;
    for (int i = threadIdx.x; i < kBlock * 4; i += 256) {
        const int row = i >> 2, ch = i & 3;
        const int64_t to = (int64_t)blockIdx.y * kBlock + row;
        if (to >= cols) continue;
        uint8_t* d = q + to * ldq + pl.block * 64 + ch * 16;
        const v4u val = *(const v4u*)&tile[row][((ch + (row >> 4)) & 3) * 4];
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

// A thread per eight values, U times in turn.  Bound by memory: 32668 x 4096 to bf16, 339 MB, 54 us (6.3 TB/s, most of it written).
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

// 32 x 32 x 64, lane (r, g) with block number g of two of row r: a lane holds four times four neighbours of one row of `out`.
template <int STEP> __device__ __forceinline__ v16f mma4_32(const v4u& b, const v4u& a, v16f c, unsigned sb, unsigned sa) {
    const v8i wb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3]}, wa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3]};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wb, wa, c, 4, 4, STEP, (int)sb, STEP, (int)sa);
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

// At most N of the wave's loads and M of its reads of the LDS are still under way, and all waves of the workgroup are here.
template <int N, int M> __device__ __forceinline__ void left_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" ::"n"(N), "n"(M) : "memory");
}

// The large form: a tile of BM x BN, four waves, stages of 128 of the length through four parts of the LDS.  While a stage is multiplied, the next
// one's rows go from the LDS to registers, the one behind it is on its way and the one after that is asked for: a load has from one to two stages' time to arrive
// (in the largest tile 1.1 to 2.2 us, a stage being 1.8 thousand cycles at 1.6 GHz), and between stages there is one barrier.  A row of a stage is 64 bytes; its sixteen number c lies at place c xor
// (row / 4 mod 4), so that the lanes that the LDS serves together meet every bank once.  The scales come in sixteens, for four stages (512 of the
// length, from multiples of 512); a lane collects its blocks' bytes of two stages in one register, of which a product takes byte STEP.
// The waves: WM x WN, 32 MT by 32 NT each; a stage is two steps of 64, in which lane (r, g) has block number 2 g + step of row r.
// 16384 x 8192 x 8192 0.56 to 0.61 ms (3.6 to 3.9 PFLOP/s): eight rounds of 64 stages of 1.8 thousand cycles, 1.0 of them matrix instructions, while the clock
// falls to some 1.6 GHz.  Short lengths pay the first loads and the stores of every tile: 20011 rows of 32 groups, 3584 x 2048, 154 us, six rounds of 52 thousand
// cycles, of which 16 stages would be 29.  128 x 128, two workgroups a compute unit: one's stages run beside the other's first loads and stores, at twice the reads of
// the LDS for a product (16384 x 4096 x 1024 64 to 70 us against 87, x 2048 109 against 103).  Rows of scales start on 16 bytes, for their loads are as wide; others
// go to the simple form.  The instances of 128 x 256 by columns keep 32 bytes a lane in scratch, none other does.  Tiles of 128 rows at
// the ends of groups, and tiles dealt to the XCDs in runs of 32, changed the groups' times by less than one machine differs from itself, and cost the dense ones 2 to 4 %.
template <bool COLS, class OUT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(256, BM + BN <= 256 ? 2 : 1) void k_fp4_product(Product4 P, int m_tiles, int n_tiles) {
    constexpr int W = 4, MT = BM / (32 * WM), NT = BN / (32 * WN), LA = BM / 16 / W, LB = BN / 16 / W, LS = ((BM + BN) / 64 + W - 1) / W, PART = (BM + BN) * 64;
    static_assert(WM * WN == W && LA * 16 * W == BM && LB * 16 * W == BN && BM % 64 == 0 && BN % 64 == 0 && MT % 2 == 0 && (NT == 4 || (NT == 2 && MT == 2)), "");
    __shared__ __align__(1024) uint8_t tile[4][PART];
    __shared__ __align__(1024) uint8_t scale[2][(BM + BN) * 16];
    __shared__ __align__(1024) uint8_t nowhere[W][1024];          // where loads go that ask for no stage
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WN, wn = w % WN;
    int group = 0, id;
    if (COLS) {                                                   // every XCD has an eighth of each group, for groups are of any length
        const unsigned share = (m_tiles * n_tiles + 7) / 8, at = blockIdx.x / 8;
        group = at / share;
        id = blockIdx.x % 8 * share + at % share;
        if (id >= m_tiles * n_tiles) return;
    } else {
        m_tiles = __builtin_amdgcn_readfirstlane(count_tiles(P.group_rows, P.groups, P.m, BM));
        id = xcd_run(blockIdx.x, (unsigned)m_tiles * n_tiles);
        if (id < 0) return;
    }
    // runs of four rows of tiles, column after column
    const int run = id / (4 * n_tiles), in_run = id - run * 4 * n_tiles, height = m_tiles - run * 4 < 4 ? m_tiles - run * 4 : 4;
    const int ti = run * 4 + in_run % height, tj = in_run / height;
    int64_t i0, i_end, first = 0, last;
    const int64_t j0 = (int64_t)tj * BN;
    if (COLS) {
        i0 = (int64_t)ti * BM;
        i_end = i0 + BM < P.m ? i0 + BM : P.m;
        int64_t count;
        group_blocks(P.group_rows, P.groups, group, P.k, first, count);
        last = first + count;
    } else {
        const Place pl = find_tile(P.group_rows, P.groups, P.m, BM, ti);
        if (pl.group < 0) return;
        group = pl.group; i0 = pl.first; i_end = pl.end;
        last = blocks_of(P.k);
    }
    i0 = (int64_t)__builtin_amdgcn_readfirstlane((int)i0);
    i_end = (int64_t)__builtin_amdgcn_readfirstlane((int)i_end);
    group = __builtin_amdgcn_readfirstlane(group);
    int s0 = __builtin_amdgcn_readfirstlane((int)first);
    asm("" : "+s"(s0));                                           // (a first stage that the compiler knows makes it peel the loop, and spill)
    const int s1 = __builtin_amdgcn_readfirstlane((int)last);
    const int whole = COLS ? s1 : (int)(P.k / kBlock);            // stages before this one are whole
    const int rows_a = (int)(i_end - i0), rows_b = (int)(P.n - j0 < BN ? P.n - j0 : BN);
    const uint8_t* a = scalar(P.a + i0 * P.lda);
    const uint8_t* b = scalar(P.b + (COLS ? 0 : group * P.b_group) + j0 * P.ldb);
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&tile[0][0];
    const unsigned lds_scale = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&scale[0][0];
    // this lane's sixteens of a stage: LA of a's rows, then LB of b's
    const int chunk = (lane & 3) ^ (lane >> 4);
    unsigned at[LA + LB];
#pragma unroll
    for (int j = 0; j < LA + LB; ++j) {
        const bool of_a = j < LA;
        const int r = (of_a ? w * LA + j : w * LB + j - LA) * 16 + (lane >> 2), most = of_a ? rows_a : rows_b;
        at[j] = (unsigned)((r < most ? r : most - 1) * (of_a ? P.lda : P.ldb)) + chunk * 16;
    }
    // and its rows of scales
    const uint8_t* at_s[LS];
#pragma unroll
    for (int j = 0; j < LS; ++j) {
        const int r = (w * LS + j) * 64 + lane;
        if (r >= BM + BN) at_s[j] = P.as;                         // (no row: not asked for)
        else if (r < BM) at_s[j] = P.as + (i0 + (r < rows_a ? r : rows_a - 1)) * P.ld_as;
        else at_s[j] = P.bs + (COLS ? 0 : group * P.bs_group) + (j0 + (r - BM < rows_b ? r - BM : rows_b - 1)) * P.ld_bs;
    }
    auto place = [&](int j) { return j < LA ? (w * LA + j) * 1024 : BM * 64 + (w * LB + j - LA) * 1024; };
    // sixteens number j of whole stage s; behind the whole stages the last one's, to nowhere, so that every stage is as many loads
    const unsigned away = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&nowhere[w][0];
    auto ask = [&](int s, int part, int j) {
        const bool there = s < whole;
        dma16((j < LA ? a : b) + (int64_t)(there ? s : whole - 1) * 64, at[j], there ? lds + part * PART + place(j) : away);
    };
    // a stage that ends inside: zeros behind the end, through registers; a sixteen that ends inside is read up to the row's end, from as many bytes ahead
    auto fill = [&](int s, int part) {
        const int left = (int)(P.k - (int64_t)s * kBlock) - chunk * 32, ahead = left >= 32 ? 0 : 16 - (left + 1) / 2;
#pragma unroll 1
        for (int j = 0; j < LA + LB; ++j) {
            const int to = place(j), row = (j < LA ? to : to - BM * 64) / 64 + (lane >> 2), most = j < LA ? rows_a : rows_b;
            unsigned __int128 v = 0;
            if (left > 0) {
                __builtin_memcpy(&v, (j < LA ? P.a + i0 * P.lda : P.b + group * P.b_group + j0 * P.ldb) + (row < most ? row : most - 1) * (j < LA ? P.lda : P.ldb) +
                                 (int64_t)s * 64 + chunk * 16 - ahead, 16);
                v >>= 8 * ahead;
                if (left < 32) v &= ((unsigned __int128)1 << (4 * left)) - 1;
            }
            __builtin_memcpy(&tile[part][to + lane * 16], &v, 16);
        }
    };
    auto ask_scales = [&](int t) {
        if (t * 4 >= s1) return;
        // sixteen scales that all exist, of four stages, or what there is
        const int64_t there = (COLS ? (int64_t)s1 * 4 : (P.k + kBlock4 - 1) / kBlock4) - (int64_t)t * 16;
        if (there >= 16) {
#pragma unroll
            for (int j = 0; j < LS; ++j)
                if ((w * LS + j) * 64 < BM + BN) dma16(at_s[j] + (int64_t)t * 16, lds_scale + (t & 1) * (BM + BN) * 16 + (w * LS + j) * 1024);
        } else {
#pragma unroll
            for (int j = 0; j < LS; ++j) {
                if ((w * LS + j) * 64 >= BM + BN) break;
                v4u v = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
#pragma unroll 1
                for (int i = 0; i < there; ++i) {
                    const unsigned one = ((unsigned)at_s[j][(int64_t)t * 16 + i] ^ 0x7fu) << (8 * (i & 3));
                    if (i < 4) v[0] ^= one; else if (i < 8) v[1] ^= one; else if (i < 12) v[2] ^= one; else v[3] ^= one;
                }
                *(v4u*)&scale[t & 1][(w * LS + j) * 1024 + lane * 16] = v;
            }
        }
    };
    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
    const int r = lane & 31, g = lane >> 5, mine = r * 64 + (2 * g ^ ((r >> 2) & 3)) * 16;
    constexpr int G = 2 * MT, L = LA + LB;                        // groups of NT products, and loads, of a stage
    // reads that a stage does behind its last one of its own rows (they come back in order): those of the next stage's rows
    constexpr int LATE = G == 8 ? 5 : NT == 4 ? 6 : 4;
    v4u fa[4], fb[2][NT];
    unsigned sa[MT][2], sb[NT][2];
    auto read_a = [&](int part, int i, int h) { return *(const v4u*)&tile[part][(wm * MT + i) * 2048 + (mine ^ h * 16)]; };
    auto read_b = [&](int part, int j, int h) { return *(const v4u*)&tile[part][BM * 64 + (wn * NT + j) * 2048 + (mine ^ h * 16)]; };
    const unsigned two = 0x05040100u + g * 0x02020202u;           // bytes 2 g and 2 g + 1 of two words
    auto read_scale = [&](int t, int row) { return *(const v4u*)&scale[t & 1][row * 16]; };
    auto spread = [&](const v4u& v, unsigned (&to)[2]) {
        to[0] = __builtin_amdgcn_perm(v[1], v[0], two);
        to[1] = __builtin_amdgcn_perm(v[3], v[2], two);
    };
    const int row_a = wm * MT * 32 + r, row_b = BM + wn * NT * 32 + r;
    if (s0 < s1) {
        const int t0 = s0 / 4;
        ask_scales(t0);
        ask_scales(t0 + 1);
#pragma unroll 1
        for (int s = s0; s < s0 + 3; ++s) {
            if (s >= whole && s < s1) fill(s, s & 3);
#pragma unroll
            for (int j = 0; j < L; ++j) ask(s, s & 3, j);
        }
        left_and_barrier<2 * L, 0>();
        fa[0] = read_a(s0 & 3, 0, 0);
        fa[1] = read_a(s0 & 3, 1, 0);
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[0][j] = read_b(s0 & 3, j, 0);
#pragma unroll
        for (int i = 0; i < MT; ++i) spread(read_scale(t0, row_a + i * 32), sa[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) spread(read_scale(t0, row_b + j * 32), sb[j]);
        // Stage s = 4 t + U.  False: there is no such stage.
        auto stage = [&](int t, auto number) {
            constexpr int U = number.value;
            const int s = 4 * t + U;
            if (s < s0) return true;
            if (s >= s1) return false;
            left_and_barrier<L, LATE>();
            if (U == 0 && t > t0) ask_scales(t + 1);
            if (s + 3 >= whole && s + 3 < s1) fill(s + 3, (U + 3) & 3);
            v4u raw[MT + NT];
            // Between two products one read of the LDS or one load: a product takes 32 cycles, in whose shadow the others are issued.
            auto group = [&](auto which) {
                constexpr int q = which.value, h = q / MT, i = q % MT, ahead = q + 2, J0 = i * NT / MT, J1 = (i + 1) * NT / MT;
                auto between = [&](auto slot) {
                    constexpr int n = slot.value;                 // 0: a's rows of two groups ahead; then b's of the next step, this group's loads, and scales
                    if constexpr (n == 0) {
                        fa[ahead & 3] = ahead < G ? read_a(U, ahead % MT, ahead / MT) : read_a((U + 1) & 3, ahead - G, 0);
                    } else if constexpr (n <= J1 - J0) {
                        fb[h ^ 1][J0 + n - 1] = h == 0 ? read_b(U, J0 + n - 1, 1) : read_b((U + 1) & 3, J0 + n - 1, 0);
                    }
                    if constexpr (n == (J1 - J0 + 1 < NT ? J1 - J0 + 1 : NT - 1)) {
#pragma unroll
                        for (int j = q * L / G; j < (q + 1) * L / G; ++j) ask(s + 3, (U + 3) & 3, j);
                    }
                    if constexpr (U == 3 && n == NT - 1) {
                        if constexpr (h == 0) raw[i] = read_scale(t + 1, row_a + i * 32);
                        else
#pragma unroll
                            for (int j = J0; j < J1; ++j) raw[MT + j] = read_scale(t + 1, row_b + j * 32);
                    }
                };
                auto product = [&](auto jj) {
                    constexpr int j = jj.value;
                    acc[i][j] = mma4_32<(U & 1) * 2 + h>(fb[h][j], fa[q & 3], acc[i][j], sb[j][U / 2], sa[i][U / 2]);
                    __builtin_amdgcn_sched_barrier(0);
                    between(Int<j>{});
                    __builtin_amdgcn_sched_barrier(0);
                };
                product(Int<0>{});
                product(Int<1>{});
                if constexpr (NT == 4) {
                    product(Int<2>{});
                    product(Int<3>{});
                }
            };
            group(Int<0>{});
            group(Int<1>{});
            group(Int<2>{});
            group(Int<3>{});
            if constexpr (G == 8) {
                group(Int<4>{});
                group(Int<5>{});
                group(Int<6>{});
                group(Int<7>{});
            }
            if (U == 3) {
#pragma unroll
                for (int i = 0; i < MT; ++i) spread(raw[i], sa[i]);
#pragma unroll
                for (int j = 0; j < NT; ++j) spread(raw[MT + j], sb[j]);
            }
            return true;
        };
        static_assert(G == 4 || G == 8, "");
        for (int t = t0; stage(t, Int<0>{}) && stage(t, Int<1>{}) && stage(t, Int<2>{}) && stage(t, Int<3>{}); ++t) {}
    }
    // The result goes through the LDS, a wave's own part of it, so that a store takes whole pieces of 256 or 512 bytes of a row: a lane's four neighbours
    // alone are 8 or 16 bytes of 32 rows (16384 x 8192 columns in bf16 then took 125 us beside the products).  A row's sixteen number c lies at place c xor
    // the row's number.
    constexpr int SZ = (int)sizeof(OUT), CH = NT * 32 * SZ / 16, IP = SZ == 2 ? MT : MT / 2, REGION = IP * 32 * CH * 16;
    static_assert(W * REGION <= 4 * PART, "");
    left_and_barrier<0, 0>();
    uint8_t* own = &tile[0][0] + w * REGION;
    OUT* out = (OUT*)P.out + (COLS ? group * P.out_group : 0);
    const bool wide = (((uintptr_t)P.out | (uintptr_t)(P.ldo * SZ) | (uintptr_t)(COLS ? P.out_group * SZ : 0)) & 15) == 0;
#pragma unroll
    for (int i1 = 0; i1 < MT; i1 += IP) {
#pragma unroll
        for (int i = 0; i < IP; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v16f& c = acc[i1 + i][j];
                    uint8_t* row = own + (i * 32 + r) * CH * 16;
                    if constexpr (SZ == 2)
                        *(v2u*)(row + ((j * 4 + q) ^ (r & (CH - 1))) * 16 + g * 8) = v2u{(unsigned)to_bf16(c[q * 4]) | (unsigned)to_bf16(c[q * 4 + 1]) << 16,
                                                                                  (unsigned)to_bf16(c[q * 4 + 2]) | (unsigned)to_bf16(c[q * 4 + 3]) << 16};
                    else
                        *(v4f*)(row + ((j * 8 + q * 2 + g) ^ (r & (CH - 1))) * 16) = v4f{c[q * 4], c[q * 4 + 1], c[q * 4 + 2], c[q * 4 + 3]};
                }
        wave_lds_done();
#pragma unroll 4
        for (int k = 0; k < IP * 32 * CH / 64; ++k) {
            const int at_row = k * (64 / CH) + lane / CH, c = lane % CH;
            const v4u v = *(const v4u*)(own + at_row * CH * 16 + (c ^ (at_row & (CH - 1))) * 16);
            const int64_t row = i0 + (wm * MT + i1) * 32 + at_row, col = j0 + wn * NT * 32 + c * (16 / SZ);
            if (row >= i_end || col >= P.n) continue;
            OUT* to = out + row * P.ldo + col;
            if (wide && P.n - col >= 16 / SZ) {
                *(v4u*)to = v;
            } else {
#pragma unroll
                for (int e = 0; e < 16 / SZ; ++e)
                    if (col + e < P.n) {
                        if constexpr (SZ == 2) ((unsigned short*)to)[e] = (unsigned short)(v[e >> 1] >> (16 * (e & 1)));
                        else ((unsigned*)to)[e] = v[e];
                    }
            }
        }
        wave_lds_done();
    }
}

// The form for few rows, which reads the weights once and little else: a workgroup has 16 NT rows of b and 16 MT rows of a, its W waves share the length
// in units of 256, and the waves' sums are added up in their order.  Rows of b go through the LDS, a wave's own part of it, in whole pieces of 128 bytes
// (sixteen number i of a row at place i xor (row / 2 mod 8)): the product's lanes, sixteen rows side by side, would ask for every sixteen bytes by
// themselves.  A row's scales of a unit are two words in the lane of its number, read by those that need them.  These loads hang on the lane, and the compiler does
// not count the rows' loads into the LDS: it waits for more than it has to, and of the AHEAD units the one just asked for is often the only one under way.
// 40 x 4096 x 2880 5.1 us, most of it the way there and back; 96 rows of 16 groups, 2816 x 2048, 49 MB, 13 us (3.7 TB/s).  Loads of scales by all lanes, so that none
// hangs on a condition: 6.0 and 14.4 us.
template <class OUT, int MT, int NT, int W>
__global__ __launch_bounds__(W * 64) void k_fp4_product_thin(Product4 P) {
    constexpr int T = MT * NT, AHEAD = T > 4 ? 2 : 3, RING = AHEAD * NT * 2048;
    __shared__ __align__(1024) uint8_t shared[W * (RING > T * 1024 ? RING : T * 1024)];      // the waves' rings, and then their sums
    v4f(*sums)[T][64] = (v4f(*)[T][64])shared;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Place pl = find_tile(P.group_rows, P.groups, P.m, 16 * MT, blockIdx.y);
    if (pl.group < 0) return;
    const int group = __builtin_amdgcn_readfirstlane(pl.group);
    const int64_t i0 = pl.first, i_end = pl.end, j0 = (int64_t)blockIdx.x * (16 * NT);
    const int r = lane & 15, g = lane >> 4;
    auto row_a = [&](int n) { return i0 + n < i_end ? i0 + n : i_end - 1; };
    auto row_b = [&](int n) { return j0 + n < P.n ? j0 + n : P.n - 1; };
    const uint8_t *first_b = P.b + group * P.b_group, *first_bs = P.bs + group * P.bs_group;
    v4f acc[MT][NT];
#pragma unroll
    for (int s = 0; s < MT; ++s)
#pragma unroll
        for (int q = 0; q < NT; ++q) acc[s][q] = v4f{0.f, 0.f, 0.f, 0.f};
    // units of two whole blocks; the last may have one (the other half is then that one again, and not used); the rest of the length is less than a block
    const int whole = (int)(P.k / kBlock), units = ((whole + 1) / 2 - w + W - 1) / W;
    {
        struct Ahead { v2u kb, ka; v4u a[MT][2]; };
        const uint8_t* base = scalar(first_b + j0 * P.ldb);
        unsigned off[2 * NT];                                     // eight rows of 128 bytes a load
#pragma unroll
        for (int j = 0; j < 2 * NT; ++j)
            off[j] = (unsigned)((row_b(j * 8 + (lane >> 3)) - j0) * P.ldb);
        const int chunk = (lane & 7) ^ (lane >> 4);               // of the first eight rows; of the next it is 4 further or nearer
        const uint8_t *at_sb = first_bs + row_b(lane % (16 * NT)) * P.ld_bs, *at_sa = P.as + row_a(lane % (16 * MT)) * P.ld_as;
        const uint8_t* at_a[MT];
#pragma unroll
        for (int s = 0; s < MT; ++s) at_a[s] = P.a + row_a(s * 16 + r) * P.lda + g * 16;
        uint8_t* ring = shared + w * RING;
        const unsigned slots = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;
        const int place = r * 128 + (g ^ (r >> 1)) * 16;
        auto fetch = [&](Ahead& t, int u) {
            const int64_t at = (int64_t)(u * W + w) * kBlock;     // in bytes
            const int two = 2 * (u * W + w) + 1 < whole ? 1 : 0;
            const unsigned in = (chunk & (two ? 7 : 3)) * 16;
            const unsigned to = slots + (unsigned)u % AHEAD * (NT * 2048);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // what is read of this part of the LDS has been read
#pragma unroll
            for (int j = 0; j < 2 * NT; ++j) dma16(base + at, off[j] + (two && (j & 1) ? in ^ 64u : in), to + j * 1024);
            t.kb = t.ka = v2u{0u, 0u};
            auto words = [&](v2u& k, const uint8_t* p) {
                if (two) __builtin_memcpy(&k, p, 8);
                else __builtin_memcpy(&k, p, 4);
            };
            if (NT == 4 || lane < 16 * NT) words(t.kb, at_sb + at / 16);      // behind the rows of b: a wait for it is a wait for them
            if (MT == 4 || lane < 16 * MT) words(t.ka, at_sa + at / 16);
#pragma unroll
            for (int s = 0; s < MT; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) t.a[s][h] = *(const v4u*)(at_a[s] + at + h * two * 64);
        };
        Ahead st[AHEAD];
        pipeline<AHEAD, false>(st, 0, units, fetch, [&](const Ahead& t, int u) {
            asm volatile("" ::"v"(t.kb) : "memory");
            const uint8_t* from = ring + (unsigned)u % AHEAD * (NT * 2048);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h && 2 * (u * W + w) + 1 >= whole) break;
                v4u b[NT];
                unsigned sb[NT], sa[MT];
#pragma unroll
                for (int q = 0; q < NT; ++q) {
                    b[q] = *(const v4u*)(from + q * 2048 + (place ^ h * 64));
                    sb[q] = (unsigned)__shfl((int)t.kb[h], q * 16 + r) >> (8 * g);
                }
#pragma unroll
                for (int s = 0; s < MT; ++s) sa[s] = (unsigned)__shfl((int)t.ka[h], s * 16 + r) >> (8 * g);
#pragma unroll
                for (int s = 0; s < MT; ++s)
#pragma unroll
                    for (int q = 0; q < NT; ++q) acc[s][q] = mma4<0>(b[q], t.a[s][h], acc[s][q], sb[q], sa[s]);
            }
        });
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // nothing is on its way to the LDS when it is used again
    }
    if (whole * (int64_t)kBlock < P.k && (whole + 1) / 2 % W == w) {
        const int64_t blk = (int64_t)whole * 4 + g, left = P.k - blk * kBlock4;
        auto row = [&](const uint8_t* p) { return chunk32<true>(p + blk * 16, left); };
        auto one = [&](const uint8_t* p) { return left > 0 ? (unsigned)p[blk] : 127u; };
        v4u b[NT];
        unsigned sb[NT];
#pragma unroll
        for (int q = 0; q < NT; ++q) { b[q] = row(first_b + row_b(q * 16 + r) * P.ldb); sb[q] = one(first_bs + row_b(q * 16 + r) * P.ld_bs); }
#pragma unroll
        for (int s = 0; s < MT; ++s) {
            const v4u a = row(P.a + row_a(s * 16 + r) * P.lda);
            const unsigned sa = one(P.as + row_a(s * 16 + r) * P.ld_as);
#pragma unroll
            for (int q = 0; q < NT; ++q) acc[s][q] = mma4<0>(b[q], a, acc[s][q], sb[q], sa);
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < MT; ++s)
#pragma unroll
        for (int q = 0; q < NT; ++q) sums[w][s * NT + q][lane] = acc[s][q];
    __syncthreads();
    for (int t = w; t < T; t += W) {
        v4f v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < W; ++q) v += sums[q][t][lane];
        const int64_t row = i0 + t / NT * 16 + r, col = j0 + t % NT * 16 + g * 4;
        if (row < i_end && col < P.n) store_four((OUT*)P.out + row * P.ldo + col, v, (int)(P.n - col < 4 ? P.n - col : 4));
    }
}

}  // namespace moe
