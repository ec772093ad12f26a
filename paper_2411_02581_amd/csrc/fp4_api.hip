// C entry points of include/tuna_moe.h in 4 bits: checks of the arguments and the choice of kernels.  No state is kept between calls.
#include "fp4_kernels.h"
#include "moe_host.h"

using namespace moe;

namespace {

// Blocks of 32 that all rows have are counted in 31 bits.
bool blocks_fit(int64_t rows, int64_t cols) { return rows <= kMaxRows && cols <= kMaxRows && rows * ceil_div(cols, kBlock4) <= kMaxRows; }

// For every two (or four) lanes two (or four) blocks in turn, or one where there would be too few workgroups for the device.
template <int LANES, class F> void in_turn(int64_t blocks, F f) {
    constexpr int EACH = 256 / LANES;
    if (blocks > 256 * 1024) f(Int<LANES>{}, dim3((unsigned)ceil_div(blocks, 256)));
    else f(Int<1>{}, dim3((unsigned)ceil_div(blocks, EACH)));
}

}  // namespace

extern "C" {

int tuna_fp4_quantize(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols, int act,
                      const int32_t* slots, int copies, int64_t out_rows,
                      void* q, int64_t ldq, void* scales, int64_t ld_scales, void* stream) {
    if (rows < 0 || cols < 0 || out_rows < 0 || !is_float(type) || (act != TUNA_ACT_NONE && act != TUNA_ACT_SWIGLU)) return TUNA_ERR_ARG;
    if (copies < 1 || copies > TUNA_MOE_MAX_K || (!slots && (copies != 1 || out_rows < rows)) || (slots && !on(slots, 4))) return TUNA_ERR_ARG;
    if (rows == 0 || cols == 0) return TUNA_OK;
    if (!blocks_fit(rows, cols) || out_rows > kMaxRows) return TUNA_ERR_TOO_LARGE;
    const int64_t width = act == TUNA_ACT_SWIGLU ? 2 * cols : cols, nb = ceil_div(cols, kBlock4);
    if (!rows_ok(x, size_of(type), ldx, width)) return TUNA_ERR_ARG;
    if (out_rows > 0 && (!rows_ok(q, 1, ldq, ceil_div(cols, 2)) || !rows_ok(scales, 1, ld_scales, nb))) return TUNA_ERR_ARG;
    if (out_rows == 0) return TUNA_OK;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(x, size_of(type), ldx) && on(q, 8) && ldq % 8 == 0 && (act == TUNA_ACT_NONE || (cols * size_of(type)) % 16 == 0);
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(act == TUNA_ACT_SWIGLU, [&](auto a) {
            with_bool(wide, [&](auto wd) {
                in_turn<2>(rows * nb, [&](auto u, dim3 grid) {
                    LAUNCH((k_fp4_quantise<T, a.value, wd.value != 0, u.value>), grid, 256, (const T*)x, ldx, (unsigned)(rows * nb), cols, slots, copies, out_rows,
                           (uint8_t*)q, ldq, (uint8_t*)scales, ld_scales);
                });
            });
        });
    });
    return launched();
}

int tuna_fp4_quantize_columns(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols,
                              const int32_t* group_rows, int groups, void* q, int64_t ldq, void* scales, int64_t ld_scales,
                              void* stream) {
    if (rows < 0 || cols < 0 || groups < 1 || groups > TUNA_MOE_MAX_EXPERTS || (!group_rows && groups != 1) || (group_rows && !on(group_rows, 4)) || !is_float(type))
        return TUNA_ERR_ARG;
    if (rows > kMaxRows || cols > kMaxRows) return TUNA_ERR_TOO_LARGE;
    if (rows == 0 || cols == 0) return TUNA_OK;
    const int64_t nb = ceil_div(rows, kBlock) + groups - 1;
    if (!rows_ok(x, size_of(type), ldx, cols) || !rows_ok(q, 1, ldq, nb * (kBlock / 2)) || !rows_ok(scales, 1, ld_scales, nb * (kBlock / kBlock4))) return TUNA_ERR_ARG;
    const int64_t across = ceil_div(cols, kBlock);
    if (across > kMaxGridY || !grid_fits(nb, 256)) return TUNA_ERR_TOO_LARGE;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(rows_wide(x, size_of(type), ldx), [&](auto wd) {
            LAUNCH((k_fp4_quantise_columns<T, wd.value != 0>), dim3((unsigned)nb, (unsigned)across), 256, (const T*)x, ldx, rows, cols, group_rows, groups,
                   (uint8_t*)q, ldq, (uint8_t*)scales, ld_scales);
        });
    });
    return launched();
}

int tuna_fp4_dequantize(const void* q, int64_t ldq, const void* scales, int64_t ld_scales, int64_t rows, int64_t cols,
                        void* x, int type, int64_t ldx, void* stream) {
    if (rows < 0 || cols < 0 || !is_float(type)) return TUNA_ERR_ARG;
    if (rows == 0 || cols == 0) return TUNA_OK;
    if (!blocks_fit(rows, cols)) return TUNA_ERR_TOO_LARGE;
    const int64_t nb = ceil_div(cols, kBlock4);
    if (!rows_ok(q, 1, ldq, ceil_div(cols, 2)) || !rows_ok(scales, 1, ld_scales, nb) || !rows_ok(x, size_of(type), ldx, cols)) return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(x, size_of(type), ldx) && on(q, 4) && ldq % 4 == 0;
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(wide, [&](auto wd) {
            in_turn<4>(rows * nb, [&](auto u, dim3 grid) {
                LAUNCH((k_fp4_dequantise<T, wd.value != 0, u.value>), grid, 256, (const uint8_t*)q, ldq, (const uint8_t*)scales, ld_scales, (unsigned)(rows * nb), cols,
                       (T*)x, ldx);
            });
        });
    });
    return launched();
}

}  // extern "C"

namespace {

// The operands of a product that may be loaded by sixteens of bytes, and scales by fours: rows start on them.
bool product_wide(const Product4& P) {
    return on(P.a, 16) && on(P.b, 16) && P.lda % 16 == 0 && P.ldb % 16 == 0 && P.b_group % 16 == 0 && on(P.as, 4) && on(P.bs, 4) && P.ld_as % 4 == 0 &&
           P.ld_bs % 4 == 0 && P.bs_group % 4 == 0;
}

template <int BM, int BN, int WM, int WN, bool COLS, class OUT> void launch_tiles(const Product4& P, void* stream) {
    const int64_t nt = ceil_div(P.n, BN), mt = COLS ? ceil_div(P.m, BM) : ceil_div(P.m, BM) + P.groups - 1;
    const int64_t grid = COLS ? ceil_div(mt * nt, 8) * 8 * P.groups : ceil_div(mt * nt, 8) * 8;
    LAUNCH((k_fp4_product<COLS, OUT, BM, BN, WM, WN>), dim3((unsigned)grid), 256, P, (int)mt, (int)nt);
}

// Tiles of the large form: rows of scales start on 16 bytes, as wide as their loads (where they do not, the simple form: 20011 rows of 32 groups, 2048 x 1792,
// 195 us for 77; dx by columns, 10007 rows of 8, 2816 x 2048, 154 for 64), offsets inside a tile are 32 bits, and there is a whole stage of 128.
bool product_large(const Product4& P, bool cols) {
    const int64_t nt = ceil_div(P.n, 128), mt = ceil_div(P.m, 128) + (cols ? 0 : P.groups - 1);
    return product_wide(P) && on(P.as, 16) && on(P.bs, 16) && P.ld_as % 16 == 0 && P.ld_bs % 16 == 0 && P.bs_group % 16 == 0 && P.lda < (1 << 22) && P.ldb < (1 << 22) &&
           grid_fits((mt * nt + 8) * (cols ? P.groups : 1), 256) && P.n > 64 && (cols || P.k >= kBlock);
}

// Whether tiles of 256 x 256 fill the device: with fewer than a tile for each compute unit, or groups that are mostly shorter than one, tiles of 128 x 256
// are faster.  256 x 256 / 128 x 256, us a call, 4096 x 4096 weights: 512 rows 28 / 20, 1024 rows 30 / 22, 2048 rows 33 / 28, 4096 rows 43 / 51; 64 groups,
// 3584 x 4096: 4096 rows 156 / 136, 8192 rows 172 / 149, 16384 rows 212 / 257; by columns, 2048 x 2048 of 2048 rows 21 / 15, 16 groups of it 63 / 73.
bool product_fills(const Product4& P, bool cols) {
    return ceil_div(P.m, 256) * ceil_div(P.n, 256) * (cols ? P.groups : 1) >= 256 && (cols || P.m >= 192 * (int64_t)P.groups);
}

// Whether tiles of 128 x 128, of which a compute unit has two, are faster: one's first loads and stores are hidden behind the other's stages, which pays for lengths of
// up to eight stages, and where there is at most one of them for each compute unit.  This form / the larger ones, us a call, bf16, on two machines: 16384 x 4096 x 1024 64 to 70 / 87, x 2048
// 109 / 103; 32 groups, 20011 x 2048 x 768 54 / 61, x 1792 88 / 78; 1024 x 4096 x 4096 16.8 / 20.7, 2048 rows 30 / 27; by columns, 2048 x 2048 of 2048 rows 12 / 16,
// 16 groups of 1024 96 to 99 / 114, 8 groups of 1250, 2816 x 2048, 79 / 75.
bool product_short(const Product4& P, bool cols) {
    const int64_t length = cols ? P.k / P.groups : P.k;
    return length <= 1024 || ceil_div(P.m, 128) * ceil_div(P.n, 128) * (cols ? P.groups : 1) <= 256;
}

// Few rows: tiles for which the waves of a workgroup share the length.  Which of them, and whether: the tiles of one group are at most a round of workgroups.
// 4096 x 4096, us a call, this form / tiles of 128 x 256: 1 row 6.4 / 19, 64 rows 8.4 / 19, 128 rows 9.5 / 19, 256 rows 11.4 / 19, 512 rows 22 / 19.
// Groups, rows by 16 and columns by 32 / by 32 and 64 / tiles of 128 x 256: 16 of 2816 x 2048, 96 rows 12.5 / 14.4 / 15.9, 256 rows 13.8 / 14.7 / 16.1, 512 rows
// 19 / 14.9 / 16.7, 1024 rows 32 / 25 / 17; 64 of 3584 x 4096, 512 rows 89 / 94 / 121, 1024 rows 107 / 102 / 127, 2048 rows 157 / 114 / 127.  The host has the mean alone, for the
// bounds are the device's: one group with half of the rows, 64 of 3584 x 4096, 768 rows 106 / 102 / 118, 1024 117 / 108 / 119, 2048 171 / 134 / 128; 128 of 2816 x 4096,
// 768 rows 147 / 145 / 177, 2048 189 / 168 / 185, 4096 270 / 210 / 209; 16 of 2816 x 2048, 256 rows 15.6 / 15.3 / 17.0: at worst 15 % beside the best.
template <class F> bool product_thin(const Product4& P, F rows) {
    if (!product_wide(P) || P.ldb >= (1 << 24) || ceil_div(P.m, 16) + P.groups > kMaxGridY || ceil_div(P.n, 16) > kMaxRows / 512) return false;
    if (P.groups > 1) {
        if (P.m <= 16 * (int64_t)P.groups) rows(Int<1>{}, Int<2>{}, Int<4>{});
        else if (P.m <= 32 * (int64_t)P.groups) rows(Int<2>{}, Int<4>{}, Int<4>{});
        else return false;
        return true;
    }
    if (P.m <= 16) rows(Int<1>{}, Int<1>{}, Int<8>{});
    else if (P.m <= 32) rows(Int<2>{}, Int<1>{}, Int<8>{});
    else if (P.m <= 48) rows(Int<3>{}, Int<1>{}, Int<8>{});
    else if (P.m <= 64) rows(Int<4>{}, Int<1>{}, Int<8>{});
    else if (ceil_div(P.m, 64) * ceil_div(P.n, 32) <= 256) rows(Int<4>{}, Int<2>{}, Int<8>{});
    else if (ceil_div(P.m, 64) * ceil_div(P.n, 64) <= 256) rows(Int<4>{}, Int<4>{}, Int<8>{});
    else return false;
    return true;
}

int launch_product(const Product4& P, bool cols, int out_type, void* stream) {
    bool done = false;
    with_type(out_type, [&](auto* o) {
        using O = Pointee<decltype(o)>;
        done = !cols && product_thin(P, [&](auto mt, auto nt, auto w) {
            const dim3 grid((unsigned)ceil_div(P.n, 16 * nt.value), (unsigned)(ceil_div(P.m, 16 * mt.value) + P.groups - 1));
            LAUNCH((k_fp4_product_thin<O, mt.value, nt.value, w.value>), grid, w.value * 64, P);
        });
        if (done || !product_large(P, cols)) return;
        done = true;
        with_bool(cols, [&](auto cl) {
            if (product_short(P, cols)) launch_tiles<128, 128, 2, 2, cl.value != 0, O>(P, stream);
            else if (product_fills(P, cols)) launch_tiles<256, 256, 2, 2, cl.value != 0, O>(P, stream);
            else launch_tiles<128, 256, 2, 2, cl.value != 0, O>(P, stream);
        });
    });
    if (done) return launched();
    const int64_t nt = ceil_div(P.n, 64), mt = cols ? ceil_div(P.m, 64) : ceil_div(P.m, 64) + P.groups - 1;
    if (!grid_fits(mt, 256)) return TUNA_ERR_TOO_LARGE;
    const dim3 grid((unsigned)mt, (unsigned)nt, cols ? P.groups : 1);
    with_type(out_type, [&](auto* o) {
        using O = Pointee<decltype(o)>;
        with_bool(cols, [&](auto cl) {
            with_bool(product_wide(P), [&](auto wd) { LAUNCH((k_fp4_product64<cl.value != 0, wd.value != 0, O>), grid, 256, P); });
        });
    });
    return launched();
}

bool product_args(const int32_t* group_rows, int groups, int64_t m, int64_t n, int64_t k, int out_type) {
    return m >= 0 && n >= 0 && k >= 0 && groups >= 1 && groups <= TUNA_MOE_MAX_EXPERTS && (group_rows || groups == 1) && on(group_rows, 4) && is_float(out_type);
}

}  // namespace

extern "C" {

int tuna_fp4_matmul(const void* x, int64_t ldx, const void* xs, int64_t ld_xs,
                    const void* w, int64_t ldw, int64_t w_group, const void* ws, int64_t ld_ws, int64_t ws_group,
                    const int32_t* group_rows, int groups, void* y, int y_type, int64_t ldy,
                    int64_t m, int64_t n, int64_t k, void* stream) {
    if (!product_args(group_rows, groups, m, n, k, y_type)) return TUNA_ERR_ARG;
    if (m > kMaxRows || ceil_div(n, 64) > kMaxGridY || k > kMaxRows) return TUNA_ERR_TOO_LARGE;
    if (m == 0 || n == 0) return TUNA_OK;
    const int64_t half = ceil_div(k, 2), nk = ceil_div(k, kBlock4);
    if (!rows_ok(y, size_of(y_type), ldy, n)) return TUNA_ERR_ARG;
    if (k > 0 && (!rows_ok(x, 1, ldx, half) || !rows_ok(w, 1, ldw, half) || !rows_ok(xs, 1, ld_xs, nk) || !rows_ok(ws, 1, ld_ws, nk))) return TUNA_ERR_ARG;
    if (groups > 1 && (w_group < 0 || ws_group < 0)) return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    Product4 P = {(const uint8_t*)x, ldx, (const uint8_t*)xs, ld_xs, (const uint8_t*)w, ldw, groups > 1 ? w_group : 0, (const uint8_t*)ws, ld_ws,
                  groups > 1 ? ws_group : 0, group_rows, groups, y, ldy, 0, m, n, k};
    return launch_product(P, false, y_type, stream);
}

int tuna_fp4_matmul_grad_w(const void* dyt, int64_t ld_dyt, const void* dyt_scales, int64_t ld_dyt_scales,
                           const void* xt, int64_t ld_xt, const void* xt_scales, int64_t ld_xt_scales,
                           const int32_t* group_rows, int groups, void* dw, int dw_type, int64_t ld_dw, int64_t dw_group,
                           int64_t m, int64_t n, int64_t k, void* stream) {
    if (!product_args(group_rows, groups, m, n, k, dw_type)) return TUNA_ERR_ARG;
    if (m > kMaxRows || n > kMaxRows || ceil_div(k, 64) > kMaxGridY) return TUNA_ERR_TOO_LARGE;
    if (n == 0 || k == 0) return TUNA_OK;
    const int64_t nb = m > 0 ? ceil_div(m, kBlock) + groups - 1 : 0, half = nb * (kBlock / 2), ns = nb * (kBlock / kBlock4);
    if (!rows_ok(dw, size_of(dw_type), ld_dw, k) || (groups > 1 && dw_group < (n - 1) * ld_dw + k)) return TUNA_ERR_ARG;
    if (m > 0 && (!rows_ok(dyt, 1, ld_dyt, half) || !rows_ok(xt, 1, ld_xt, half) || !rows_ok(dyt_scales, 1, ld_dyt_scales, ns) || !rows_ok(xt_scales, 1, ld_xt_scales, ns)))
        return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    Product4 P = {(const uint8_t*)dyt, ld_dyt, (const uint8_t*)dyt_scales, ld_dyt_scales, (const uint8_t*)xt, ld_xt, 0, (const uint8_t*)xt_scales, ld_xt_scales, 0,
                  group_rows, groups, dw, ld_dw, dw_group, n, k, m};
    return launch_product(P, true, dw_type, stream);
}

}  // extern "C"
