// C entry points of include/tuna_moe.h: checks of the arguments and the choice of kernels.  No state is kept between calls.
#include "moe_kernels.h"
#include "moe_host.h"

using namespace moe;

namespace {

struct RouteSizes {
    int64_t shard; int shards;
    size_t counts, before, totals, places, bytes;     // offsets
};

// The shards of the count: the ranks' with a plan, else of 64 tokens and more, at most as many as a workgroup scans.
RouteSizes route_sizes(int64_t n, int experts, int k, bool plan) {
    RouteSizes r;
    if (plan) {
        r.shards = experts;
        r.shard = n > 0 ? ceil_div(n, experts) : 1;
    } else {
        r.shard = ceil_div(ceil_div(n > 0 ? n : 1, TUNA_MOE_MAX_EXPERTS), 64) * 64;
        r.shards = (int)(n > 0 ? ceil_div(n, r.shard) : 1);
    }
    // room for as many shards as any batch of up to this size has, so that its workspace is enough for them: 65536 tokens are 1024 shards, 65537 are 513
    const int64_t batches = n > 0 ? ceil_div(n, 64) : 1;
    const int64_t most = plan ? r.shards : batches < TUNA_MOE_MAX_EXPERTS ? batches : TUNA_MOE_MAX_EXPERTS;
    size_t at = 0;
    r.counts = at; at += align16((size_t)most * experts * 4);
    r.before = at; at += align16((size_t)most * experts * 4);
    r.totals = at; at += align16((size_t)experts * 4);
    r.places = at; at += align16((size_t)n * k * 4);
    r.bytes = at;
    return r;
}

// What a call takes: pairs are counted in 31 bits, and a wave has a token.
bool route_fits(int64_t n, int k) { return n <= kMaxRows / k && grid_fits(ceil_div(n, 4), 256); }

bool route_args(int64_t n, int experts, int k) {
    return n >= 0 && experts >= 1 && experts <= TUNA_MOE_MAX_EXPERTS && k >= 1 && k <= TUNA_MOE_MAX_K && k <= experts;
}

}  // namespace

extern "C" {

int tuna_moe_route_workspace(int64_t n_tokens, int n_experts, int k, int with_plan, size_t* bytes) {
    if (!bytes || !route_args(n_tokens, n_experts, k)) return TUNA_ERR_ARG;
    if (!route_fits(n_tokens, k)) return TUNA_ERR_TOO_LARGE;
    *bytes = route_sizes(n_tokens, n_experts, k, with_plan != 0).bytes;
    return TUNA_OK;
}

int tuna_moe_route(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, int k, int flags,
                   int32_t* experts, float* weights, int32_t* slots, int32_t* expert_rows,
                   int64_t row_bytes, int32_t* sendcounts, int64_t* sdispls, int32_t* recvcounts, int64_t* rdispls,
                   void* workspace, size_t workspace_bytes, void* stream) {
    if (!route_args(n_tokens, n_experts, k) || !is_float(type) || (flags & ~TUNA_ROUTE_RENORM)) return TUNA_ERR_ARG;
    if (!expert_rows || !on(expert_rows, 4)) return TUNA_ERR_ARG;
    if (n_tokens > 0 && (!rows_ok(logits, size_of(type), ld, n_experts) || !experts || !weights || !slots || !on(experts, 4) || !on(weights, 4) || !on(slots, 4)))
        return TUNA_ERR_ARG;
    const bool plan = sendcounts || sdispls || recvcounts || rdispls;
    if (plan && (!sendcounts || !sdispls || !recvcounts || !rdispls || row_bytes < 1 || !on(sendcounts, 4) || !on(sdispls, 8) || !on(recvcounts, 4) ||
                 !on(rdispls, 8)))
        return TUNA_ERR_ARG;
    if (!route_fits(n_tokens, k)) return TUNA_ERR_TOO_LARGE;
    const RouteSizes r = route_sizes(n_tokens, n_experts, k, plan);
    // a token has an expert once, so a block of the all-to-all is at most a shard long
    if (plan && row_bytes > kMaxRows / r.shard) return TUNA_ERR_TOO_LARGE;
    if (!workspace || !on(workspace, 16)) return TUNA_ERR_ARG;
    if (workspace_bytes < r.bytes) return TUNA_ERR_WORKSPACE_TOO_SMALL;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    char* ws = (char*)workspace;
    int32_t *counts = (int32_t*)(ws + r.counts), *before = (int32_t*)(ws + r.before), *totals = (int32_t*)(ws + r.totals), *places = (int32_t*)(ws + r.places);
    const int renorm = flags & TUNA_ROUTE_RENORM ? 1 : 0;
    // a wave holds a token's logits in registers, as many as there may be of them
    auto held = [&](auto f) {
        if (n_experts <= 64) f(Int<1>{});
        else if (n_experts <= 128) f(Int<2>{});
        else if (n_experts <= 256) f(Int<4>{});
        else if (n_experts <= 512) f(Int<8>{});
        else f(Int<16>{});
    };
    // Up to 64 tokens without a plan: one workgroup, one launch in place of four.  A call, this way / the other: 1 token of 64 experts, k = 4, 8 / 15 us,
    // 64 tokens 8 / 16; 64 tokens of 256 experts, k = 8, 16 / 17.  Of 1024 experts, k = 16, one workgroup is enough for some 20 tokens: 16 tokens 18 / 22,
    // 32 tokens 32 / 22, 64 tokens 61 / 24.
    const bool small = !plan && n_tokens > 0 && n_tokens <= 64;
    if (n_tokens > 0)
        with_type(type, [&](auto* t) {
            using T = Pointee<decltype(t)>;
            held([&](auto per) {
                if (small) LAUNCH((k_route_small<T, per.value>), dim3(1), 1024, (const T*)logits, ld, (int)n_tokens, n_experts, k, renorm, experts, weights, slots,
                                  expert_rows);
                else LAUNCH((k_route_choose<T, per.value>), dim3((unsigned)ceil_div(n_tokens, 4)), 256, (const T*)logits, ld, n_tokens, n_experts, k, renorm,
                            experts, weights);
            });
        });
    // every kernel reads what those before it have written: none is launched behind one that was not
    int e = launched();
    if (small || e != TUNA_OK) return e;
    LAUNCH(k_route_count, dim3(r.shards), 256, experts, n_tokens, n_experts, k, r.shard, counts, places);
    if ((e = launched()) != TUNA_OK) return e;
    LAUNCH(k_route_columns, dim3(n_experts), 256, counts, r.shards, n_experts, before, totals);
    if ((e = launched()) != TUNA_OK) return e;
    LAUNCH(k_route_place, dim3(r.shards), 256, experts, counts, before, totals, n_tokens, n_experts, k, r.shard, r.shards, places, slots, expert_rows,
           row_bytes, sendcounts, sdispls, recvcounts, rdispls);
    return launched();
}

int tuna_moe_route_grad(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, int k, int flags,
                        const int32_t* experts, const float* weights, const float* dweights,
                        void* dlogits, int64_t ld_dlogits, void* stream) {
    if (!route_args(n_tokens, n_experts, k) || !is_float(type) || (flags & ~TUNA_ROUTE_RENORM)) return TUNA_ERR_ARG;
    if (!route_fits(n_tokens, k)) return TUNA_ERR_TOO_LARGE;
    if (n_tokens == 0) return TUNA_OK;
    if (!rows_ok(logits, size_of(type), ld, n_experts) || !rows_ok(dlogits, size_of(type), ld_dlogits, n_experts) || !experts || !weights || !dweights ||
        !on(experts, 4) || !on(weights, 4) || !on(dweights, 4))
        return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        auto go = [&](auto n) {
            LAUNCH((k_route_grad<T, n.value>), dim3((unsigned)ceil_div(n_tokens, 4)), 256, (const T*)logits, ld, n_tokens, n_experts, k,
                   flags & TUNA_ROUTE_RENORM ? 1 : 0, experts, weights, dweights, (T*)dlogits, ld_dlogits);
        };
        const bool wide = rows_wide(logits, sizeof(T), ld) && rows_wide(dlogits, sizeof(T), ld_dlogits);
        // Four logits a lane / eight, 65536 tokens, k = 8: in 32 bits 256 experts 28 / 36 us, 384 46 / 41, 512 50 / 50, 768 74 / 79, 1024 101 / 104; in
        // bf16 24 / 33, 36 / 34, 40 / 37, 57 / 60, 71 / 62.  Renormalised four are faster throughout: 1024 experts 63 / 72 and 40 / 44.
        if (wide && n_experts <= 256 && n_experts % 4 == 0) go(Int<4>{});
        else if (wide && n_experts % 8 == 0) go(Int<8>{});
        else go(Int<1>{});
    });
    return launched();
}

int tuna_fp8_quantize(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols, int act,
                      const int32_t* slots, int copies, int64_t out_rows,
                      void* q, int64_t ldq, void* scales, int64_t ld_scales, int scale_type, void* stream) {
    if (rows < 0 || cols < 0 || out_rows < 0 || !is_float(type) || !is_scale(scale_type) || (act != TUNA_ACT_NONE && act != TUNA_ACT_SWIGLU)) return TUNA_ERR_ARG;
    if (copies < 1 || copies > TUNA_MOE_MAX_K || (!slots && (copies != 1 || out_rows < rows)) || (slots && !on(slots, 4))) return TUNA_ERR_ARG;
    if (rows == 0 || cols == 0) return TUNA_OK;
    const int64_t width = act == TUNA_ACT_SWIGLU ? 2 * cols : cols, nb = ceil_div(cols, kBlock);
    if (cols > kMaxRows || rows > kMaxRows || out_rows > kMaxRows || rows * nb > kMaxRows || !grid_fits(ceil_div(rows * nb, 32), 256)) return TUNA_ERR_TOO_LARGE;
    if (!rows_ok(x, size_of(type), ldx, width)) return TUNA_ERR_ARG;
    if (out_rows > 0 && (!rows_ok(q, 1, ldq, cols) || !rows_ok(scales, scale_size(scale_type), ld_scales, nb))) return TUNA_ERR_ARG;
    if (out_rows == 0) return TUNA_OK;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(x, size_of(type), ldx) && on(q, 8) && ldq % 8 == 0 && (act == TUNA_ACT_NONE || (cols * size_of(type)) % 16 == 0);
    const dim3 grid((unsigned)ceil_div(rows * nb, 32));
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(scale_type == TUNA_SCALE_E8, [&](auto kind) {
            with_bool(act == TUNA_ACT_SWIGLU, [&](auto a) {
                with_bool(wide, [&](auto wd) {
                    LAUNCH((k_quantise<T, kind.value, a.value, wd.value != 0>), grid, 256, (const T*)x, ldx, (unsigned)(rows * nb), cols, slots, copies, out_rows, (uint8_t*)q, ldq,
                           scales, ld_scales);
                });
            });
        });
    });
    return launched();
}

int tuna_fp8_quantize_columns(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols,
                              const int32_t* group_rows, int groups, void* q, int64_t ldq, void* scales, int64_t ld_scales,
                              int scale_type, void* stream) {
    if (rows < 0 || cols < 0 || groups < 1 || groups > TUNA_MOE_MAX_EXPERTS || (!group_rows && groups != 1) || (group_rows && !on(group_rows, 4)) ||
        !is_float(type) || !is_scale(scale_type))
        return TUNA_ERR_ARG;
    if (rows > kMaxRows || cols > kMaxRows) return TUNA_ERR_TOO_LARGE;
    if (rows == 0 || cols == 0) return TUNA_OK;
    const int64_t nb = ceil_div(rows, kBlock) + groups - 1;
    if (!rows_ok(x, size_of(type), ldx, cols) || !rows_ok(q, 1, ldq, nb * kBlock) || !rows_ok(scales, scale_size(scale_type), ld_scales, nb)) return TUNA_ERR_ARG;
    const int64_t across = ceil_div(cols, kBlock);
    if (across > kMaxGridY || !grid_fits(nb, 256)) return TUNA_ERR_TOO_LARGE;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(scale_type == TUNA_SCALE_E8, [&](auto kind) {
            with_bool(rows_wide(x, size_of(type), ldx), [&](auto wd) {
                LAUNCH((k_quantise_columns<T, kind.value, wd.value != 0>), dim3((unsigned)nb, (unsigned)across), 256, (const T*)x, ldx, rows, cols, group_rows,
                       groups, (uint8_t*)q, ldq, scales, ld_scales);
            });
        });
    });
    return launched();
}

int tuna_moe_swiglu_grad(const void* x, int type, int64_t ldx, const void* dh, int64_t ld_dh, int64_t rows, int64_t cols,
                         void* dx, int64_t ld_dx, void* stream) {
    if (rows < 0 || cols < 0 || !is_float(type)) return TUNA_ERR_ARG;
    if (rows == 0 || cols == 0) return TUNA_OK;
    if (rows > kMaxRows || cols > kMaxRows || !eights_fit(rows, cols)) return TUNA_ERR_TOO_LARGE;
    const int sz = size_of(type);
    if (!rows_ok(x, sz, ldx, 2 * cols) || !rows_ok(dh, sz, ld_dh, cols) || !rows_ok(dx, sz, ld_dx, 2 * cols)) return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(x, sz, ldx) && rows_wide(dh, sz, ld_dh) && rows_wide(dx, sz, ld_dx) && (cols * sz) % 16 == 0;
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        with_bool(wide, [&](auto wd) {
            LAUNCH((k_swiglu_grad<T, wd.value != 0>), eights_grid(rows, cols), 256, (const T*)x, ldx, (const T*)dh, ld_dh, rows,
                   cols, (T*)dx, ld_dx);
        });
    });
    return launched();
}

}  // extern "C"

namespace {

// The operands of a product that may be loaded by sixteens: rows of whole sixteens that start on 16 bytes.
bool product_wide(const Product& P, bool cols) {
    return on(P.a, 16) && on(P.b, 16) && P.lda % 16 == 0 && P.ldb % 16 == 0 && P.b_group % 16 == 0 && (cols || P.k % 16 == 0);
}

template <int BM, int BN, int WM, int WN, int KIND, bool COLS, class OUT> void launch_tiles(const Product& P, void* stream) {
    const int64_t nt = ceil_div(P.n, BN), mt = COLS ? ceil_div(P.m, BM) : ceil_div(P.m, BM) + P.groups - 1;
    const int64_t grid = COLS ? ceil_div(mt * nt, 8) * 8 * P.groups : ceil_div(mt * nt, 8) * 8;
    LAUNCH((k_product<KIND, COLS, OUT, BM, BN, WM, WN>), dim3((unsigned)grid), WM * WN * 64, P, (int)mt, (int)nt);
}

// Tiles of the large form: offsets inside a tile are 32 bits, tiles of 128 x 128 have 256 threads.  Up to 64 columns go to the simple form, which is the
// slower one here too: 2048 rows of 4096, 64 columns 49 us, in tiles of 128 x 128 23.
bool product_large(const Product& P, bool cols) {
    const int64_t nt = ceil_div(P.n, 128), mt = ceil_div(P.m, 128) + (cols ? 0 : P.groups - 1);
    return product_wide(P, cols) && P.lda < (1 << 22) && P.ldb < (1 << 22) && P.ld_as < (1 << 20) && P.ld_bs < (1 << 20) && grid_fits((mt * nt + 8) * (cols ? P.groups : 1), 256) && P.n > 64;
}

// Whether tiles of 256 x 256 fill the device: with fewer than a tile for each compute unit, or groups that are mostly shorter than one, tiles of
// 128 x 128 are faster.  Of 4096 x 4096 weights, a power of two as the scale, 256 x 256 / 128 x 128: 1024 rows 55 / 29 us, 2048 rows 58 / 37,
// 4096 rows 63 / 72; 64 groups, 3584 x 4096: 8192 rows 282 / 305, 16384 rows 375 / 427.
bool product_fills(const Product& P, bool cols) {
    const int64_t tiles = ceil_div(P.m, 256) * ceil_div(P.n, 256) * (cols ? P.groups : 1);
    const int64_t most = cols ? (tiles / P.groups + 8) * P.groups : (ceil_div(P.m, 256) + P.groups - 1) * ceil_div(P.n, 256) + 8;
    return tiles >= 256 && (cols || P.m / P.groups >= 128) && grid_fits(most, 512);
}

// Few rows: each workgroup reads 16 rows of the weights.  4096 x 4096, this form / tiles of 128 x 128: 8 rows 9 / 27 us, 64 rows 16 / 28; 32 groups:
// 64 rows 98 / 111, 256 rows 142 / 129, 2048 rows 568 / 139, for every 16 rows read a group's weights again.
bool product_thin(const Product& P, bool cols) {
    return !cols && product_wide(P, cols) && P.m <= (P.groups == 1 ? 64 : 2 * (int64_t)P.groups) && ceil_div(P.m, 16) + P.groups <= kMaxGridY && ceil_div(P.n, 16) <= kMaxRows / 512;
}

int launch_product(const Product& P, int kind, bool cols, int out_type, void* stream) {
    if (product_thin(P, cols)) {
        with_type(out_type, [&](auto* o) {
            using O = Pointee<decltype(o)>;
            with_bool(kind == TUNA_SCALE_E8, [&](auto sk) {
                auto rows = [&](auto mt) {
                    const dim3 grid((unsigned)ceil_div(P.n, 16), (unsigned)(ceil_div(P.m, 16 * mt.value) + P.groups - 1));
                    LAUNCH((k_product_thin<sk.value, O, mt.value>), grid, kThinWaves * 64, P);
                };
                const int64_t each = P.groups == 1 ? P.m : 16;
                if (each <= 16) rows(Int<1>{});
                else if (each <= 32) rows(Int<2>{});
                else rows(Int<4>{});
            });
        });
        return launched();
    }
    if (product_large(P, cols)) {
        with_type(out_type, [&](auto* o) {
            using O = Pointee<decltype(o)>;
            with_bool(kind == TUNA_SCALE_E8, [&](auto sk) {
                with_bool(cols, [&](auto cl) {
                    // with 32-bit outputs the widening has no room in the registers of the larger tile: 4096^3 152 us in 128 x 128, 194 in 256 x 256
                    if constexpr (sizeof(O) == 2)
                        if (product_fills(P, cols)) return launch_tiles<256, 256, 2, 4, sk.value, cl.value != 0, O>(P, stream);
                    launch_tiles<128, 128, 2, 2, sk.value, cl.value != 0, O>(P, stream);
                });
            });
        });
        return launched();
    }
    const int64_t nt = ceil_div(P.n, 64), mt = cols ? ceil_div(P.m, 64) : ceil_div(P.m, 64) + P.groups - 1;
    if (!grid_fits(mt, 256)) return TUNA_ERR_TOO_LARGE;
    const dim3 grid((unsigned)mt, (unsigned)nt, cols ? P.groups : 1);
    with_type(out_type, [&](auto* o) {
        using O = Pointee<decltype(o)>;
        with_bool(kind == TUNA_SCALE_E8, [&](auto sk) {
            with_bool(cols, [&](auto cl) {
                with_bool(product_wide(P, cols), [&](auto wd) {
                    LAUNCH((k_product64<sk.value, cl.value != 0, wd.value != 0, O>), grid, 256, P);
                });
            });
        });
    });
    return launched();
}

bool product_args(const int32_t* group_rows, int groups, int64_t m, int64_t n, int64_t k, int scale_type, int out_type) {
    return m >= 0 && n >= 0 && k >= 0 && groups >= 1 && groups <= TUNA_MOE_MAX_EXPERTS && (group_rows || groups == 1) && on(group_rows, 4) &&
           is_scale(scale_type) && is_float(out_type);
}

}  // namespace

extern "C" {

int tuna_fp8_matmul(const void* x, int64_t ldx, const void* xs, int64_t ld_xs,
                    const void* w, int64_t ldw, int64_t w_group, const void* ws, int64_t ld_ws, int64_t ws_group, int scale_type,
                    const int32_t* group_rows, int groups, void* y, int y_type, int64_t ldy,
                    int64_t m, int64_t n, int64_t k, void* stream) {
    if (!product_args(group_rows, groups, m, n, k, scale_type, y_type)) return TUNA_ERR_ARG;
    if (m > kMaxRows || ceil_div(n, 64) > kMaxGridY || k > kMaxRows) return TUNA_ERR_TOO_LARGE;
    if (m == 0 || n == 0) return TUNA_OK;
    const int64_t nk = ceil_div(k, kBlock);
    const int ss = scale_size(scale_type);
    if (!rows_ok(y, size_of(y_type), ldy, n)) return TUNA_ERR_ARG;
    if (k > 0 && (!rows_ok(x, 1, ldx, k) || !rows_ok(w, 1, ldw, k) || !rows_ok(xs, ss, ld_xs, nk) || !rows_ok(ws, ss, ld_ws, nk))) return TUNA_ERR_ARG;
    if (groups > 1 && (w_group < 0 || ws_group < 0)) return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    Product P = {(const uint8_t*)x, ldx, xs, ld_xs, (const uint8_t*)w, ldw, groups > 1 ? w_group : 0, ws, ld_ws, groups > 1 ? ws_group : 0,
                 group_rows, groups, y, ldy, 0, m, n, k};
    return launch_product(P, scale_type, false, y_type, stream);
}

int tuna_fp8_matmul_grad_w(const void* dyt, int64_t ld_dyt, const void* dyt_scales, int64_t ld_dyt_scales,
                           const void* xt, int64_t ld_xt, const void* xt_scales, int64_t ld_xt_scales, int scale_type,
                           const int32_t* group_rows, int groups, void* dw, int dw_type, int64_t ld_dw, int64_t dw_group,
                           int64_t m, int64_t n, int64_t k, void* stream) {
    if (!product_args(group_rows, groups, m, n, k, scale_type, dw_type)) return TUNA_ERR_ARG;
    if (m > kMaxRows || n > kMaxRows || ceil_div(k, 64) > kMaxGridY) return TUNA_ERR_TOO_LARGE;
    if (n == 0 || k == 0) return TUNA_OK;
    const int64_t nb = m > 0 ? ceil_div(m, kBlock) + groups - 1 : 0;
    const int ss = scale_size(scale_type);
    if (!rows_ok(dw, size_of(dw_type), ld_dw, k) || (groups > 1 && dw_group < (n - 1) * ld_dw + k)) return TUNA_ERR_ARG;
    if (m > 0 && (!rows_ok(dyt, 1, ld_dyt, nb * kBlock) || !rows_ok(xt, 1, ld_xt, nb * kBlock) || !rows_ok(dyt_scales, ss, ld_dyt_scales, nb) ||
                  !rows_ok(xt_scales, ss, ld_xt_scales, nb)))
        return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    Product P = {(const uint8_t*)dyt, ld_dyt, dyt_scales, ld_dyt_scales, (const uint8_t*)xt, ld_xt, 0, xt_scales, ld_xt_scales, 0,
                 group_rows, groups, dw, ld_dw, dw_group, n, k, m};
    return launch_product(P, scale_type, true, dw_type, stream);
}

int tuna_moe_combine(const void* y, int y_type, int64_t ldy, int64_t y_rows, const int32_t* slots, const float* weights,
                     int64_t n_tokens, int k, int64_t cols, void* out, int out_type, int64_t ld_out, void* stream) {
    if (n_tokens < 0 || y_rows < 0 || cols < 0 || k < 1 || k > TUNA_MOE_MAX_K || !is_float(y_type) || !is_float(out_type)) return TUNA_ERR_ARG;
    if (n_tokens == 0 || cols == 0) return TUNA_OK;
    if (n_tokens > kMaxRows / k || y_rows > kMaxRows || cols > kMaxRows || !eights_fit(n_tokens, cols)) return TUNA_ERR_TOO_LARGE;
    if ((y_rows > 0 && !rows_ok(y, size_of(y_type), ldy, cols)) || !slots || !weights || !on(slots, 4) || !on(weights, 4) ||
        !rows_ok(out, size_of(out_type), ld_out, cols))
        return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(y, size_of(y_type), ldy) && rows_wide(out, size_of(out_type), ld_out);
    with_type(y_type, [&](auto* a) {
        using Y = Pointee<decltype(a)>;
        with_type(out_type, [&](auto* b) {
            using O = Pointee<decltype(b)>;
            with_bool(wide, [&](auto wd) {
                LAUNCH((k_combine<Y, O, wd.value != 0>), eights_grid(n_tokens, cols), 256, (const Y*)y, ldy, y_rows, slots,
                       weights, n_tokens, k, cols, (O*)out, ld_out);
            });
        });
    });
    return launched();
}

int tuna_moe_combine_grad(const void* dout, int out_type, int64_t ld_dout, const void* y, int y_type, int64_t ldy, int64_t y_rows,
                          const int32_t* slots, const float* weights, int64_t n_tokens, int k, int64_t cols,
                          void* dy, int64_t ld_dy, float* dweights, void* stream) {
    if (n_tokens < 0 || y_rows < 0 || cols < 0 || k < 1 || k > TUNA_MOE_MAX_K || !is_float(y_type) || !is_float(out_type)) return TUNA_ERR_ARG;
    if (n_tokens == 0) return TUNA_OK;
    if (n_tokens > kMaxRows / k || !grid_fits(n_tokens, 256) || y_rows > kMaxRows || cols > kMaxRows) return TUNA_ERR_TOO_LARGE;
    if (!slots || !weights || !dweights || !on(slots, 4) || !on(weights, 4) || !on(dweights, 4)) return TUNA_ERR_ARG;
    if (cols > 0 && !rows_ok(dout, size_of(out_type), ld_dout, cols)) return TUNA_ERR_ARG;
    if (cols > 0 && y_rows > 0 && (!rows_ok(y, size_of(y_type), ldy, cols) || !rows_ok(dy, size_of(y_type), ld_dy, cols))) return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    const bool wide = rows_wide(y, size_of(y_type), ldy) && rows_wide(dy, size_of(y_type), ld_dy) && rows_wide(dout, size_of(out_type), ld_dout);
    with_type(y_type, [&](auto* a) {
        using Y = Pointee<decltype(a)>;
        with_type(out_type, [&](auto* b) {
            using O = Pointee<decltype(b)>;
            with_bool(wide, [&](auto wd) {
                LAUNCH((k_combine_grad<O, Y, wd.value != 0>), dim3((unsigned)n_tokens), 256, (const O*)dout, ld_dout, (const Y*)y, ldy, y_rows, slots, weights, k,
                       cols, (Y*)dy, ld_dy, dweights);
            });
        });
    });
    return launched();
}

int tuna_moe_few_workspace(int64_t n_tokens, int64_t hidden, int64_t inner, int n_experts, int k, size_t* bytes) {
    if (!bytes || !route_args(n_tokens, n_experts, k) || n_tokens > TUNA_MOE_FEW_TOKENS || hidden < 0 || inner < 0) return TUNA_ERR_ARG;
    if (hidden > kMaxRows || inner > kMaxRows) return TUNA_ERR_TOO_LARGE;
    const size_t pairs = (size_t)n_tokens * k;
    *bytes = 2 * align16(pairs * 4) + 2 * pairs * (size_t)ceil_div(inner, 8) * 16 + 16;
    return TUNA_OK;
}

int tuna_moe_few(const void* x, int64_t ldx, int64_t n_tokens, int64_t hidden, const void* logits, int logits_type, int64_t ld_logits,
                 int n_experts, int k, int flags, const void* w1, const void* s1, const void* w2, const void* s2, int64_t inner,
                 int weight_type, int scale_type, void* out, int out_type, int64_t ld_out,
                 void* workspace, size_t workspace_bytes, void* stream) {
    size_t need;
    const int rw = tuna_moe_few_workspace(n_tokens, hidden, inner, n_experts, k, &need);
    if (rw != TUNA_OK) return rw;
    if ((flags & ~TUNA_ROUTE_RENORM) || !is_float(logits_type) || !is_float(out_type) || (weight_type != TUNA_F8 && weight_type != TUNA_BF16 && weight_type != TUNA_F4))
        return TUNA_ERR_ARG;
    if (n_tokens == 0 || hidden == 0) return TUNA_OK;
    const size_t pairs = (size_t)n_tokens * k;
    if (inner < 1 || !rows_ok(x, 2, ldx, hidden) || !rows_ok(logits, size_of(logits_type), ld_logits, n_experts) || !rows_ok(out, size_of(out_type), ld_out, hidden))
        return TUNA_ERR_ARG;
    const int wsz = size_of(weight_type);
    if (!w1 || !w2 || !on(w1, wsz) || !on(w2, wsz)) return TUNA_ERR_ARG;
    const bool scaled = weight_type != TUNA_BF16;
    if (weight_type == TUNA_F4 && scale_type != TUNA_SCALE_E8) return TUNA_ERR_ARG;
    if (scaled && (!is_scale(scale_type) || !s1 || !s2 || !on(s1, scale_size(scale_type)) || !on(s2, scale_size(scale_type)))) return TUNA_ERR_ARG;
    if (!scaled && (s1 || s2)) return TUNA_ERR_ARG;
    if (ldx > (1 << 24) || (int64_t)pairs * (inner + 8) > (1 << 30) || ceil_div(inner, 16) > kMaxRows / 256 || ceil_div(hidden, 16) > kMaxRows / 256) return TUNA_ERR_TOO_LARGE;
    if (!workspace || !on(workspace, 16)) return TUNA_ERR_ARG;
    if (workspace_bytes < need) return TUNA_ERR_WORKSPACE_TOO_SMALL;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    char* at = (char*)workspace;
    Few F;
    F.x = (const unsigned short*)x; F.ldx = ldx; F.tokens = (int)n_tokens; F.hidden = hidden;
    F.logits = logits; F.ld_logits = ld_logits; F.experts = n_experts; F.k = k; F.renorm = flags & TUNA_ROUTE_RENORM ? 1 : 0;
    F.w1 = w1; F.s1 = s1; F.w2 = w2; F.s2 = s2; F.inner = inner; F.out = out; F.ld_out = ld_out;
    F.ld_h = ceil_div(inner, 8) * 8;
    F.chosen = (int32_t*)at; at += align16(pairs * 4);
    F.share = (float*)at; at += align16(pairs * 4);
    F.hi = (unsigned short*)at; at += pairs * F.ld_h * 2;
    F.lo = (unsigned short*)at;
    const int64_t row1 = weight_type == TUNA_F4 ? ceil_div(hidden, 2) : hidden * wsz, row2 = weight_type == TUNA_F4 ? ceil_div(inner, 2) : inner * wsz;
    const bool wide = rows_wide(x, 2, ldx) && on(w1, 16) && on(w2, 16) && row1 % 16 == 0 && row2 % 16 == 0 &&
                      row1 <= ((int64_t)1 << 31) / inner && row2 <= ((int64_t)1 << 31) / hidden;       // a lane's offset in an expert's half is 32 bits
    // One token: its k experts' rows alone; else all experts', most of which may have nothing to do.  Few pairs: the waves of a workgroup share
    // 16 columns, so that there are workgroups enough for the device; many: each wave has 16, and fewer workgroups look for their tokens.
    // Calls, shared / each 16: 8-bit weights, k = 4 of 64 experts, 1024 x 2048: 3 tokens 45 / 52 us, 4 54 / 56, 8 97 / 80, 12 120 / 95, 16 135 / 100;
    // bf16: 4 tokens 76 / 88, 8 123 / 126, 16 169 / 155.  k = 8 of 128, 1536 x 4096: 2 tokens 130 / 114, 5 245 / 216, 24 640 / 530, 40 755 / 580.
    // k = 2 of 8, 1536 x 4096: 16 tokens 59 / 72.  4-bit weights: k = 4 of 64, 1024 x 2048: 2 tokens 23.5 / 23.2, 8 43 / 41, 12 55 / 48, 16 61 / 53, 64 131 / 114; k = 8
    // of 128, 1408 x 4096: 2 tokens 59 / 51, 5 105 / 98, 24 259 / 229, 48 364 / 321; k = 2 of 8, 1536 x 4096: 16 tokens 34 / 46; k = 8 of 8, 1024 x 2048: 4 tokens
    // 21 / 26, 16 41 / 46, 64 125 / 149.  What counts is how many experts have a token times their columns: the limit here is the pairs'.
    const bool one = n_tokens == 1, split = one || (int64_t)pairs * ceil_div(inner, 64) < 1024;
    // Up to 8 pairs an expert 16 tokens at a time, else 32 (fewer waves have room).  16 / 32, 8-bit weights, 64 tokens, 1024 x 2048: k = 2 of 8 experts
    // 82 / 69 us, k = 2 of 16 65 / 65, k = 4 of 16 104 / 91, k = 4 of 32 109 / 109, k = 4 of 64 184 / 177; 16 tokens, k = 4 of 64, 101 / 126;
    // k = 8 of 128, 1536 x 4096: 24 tokens 530 / 597, 40 tokens 584 / 667, 64 tokens 644 / 718.  4-bit weights, 64 tokens, 1024 x 2048: k = 2 of 8 62 / 61, k = 2 of
    // 16 56 / 58, k = 4 of 16 85 / 84, k = 4 of 32 84 / 84, k = 4 of 64 114 / 114, k = 8 of 8 149 / 145 (8 bits 166); k = 8 of 128, 1408 x 4096: 24 tokens 229 / 263,
    // 48 321 / 356, 64 361 / 400.
    const dim3 g1((unsigned)ceil_div(inner, split ? 16 : 16 * kFewFirst), (unsigned)(one ? k : n_experts)), g2((unsigned)ceil_div(hidden, 16));
    const size_t sums = (size_t)kFewSecond * n_tokens * 16 * 4;
    int e = TUNA_OK;
    with_bool(wide, [&](auto wd) {
        auto both = [&](auto* wp, auto kind) {
            using W = Pointee<decltype(wp)>;
            with_type(logits_type, [&](auto* l) {
                using L = Pointee<decltype(l)>;
                if (one) LAUNCH((k_few_first<L, W, kind.value, wd.value != 0, 1, true, true>), g1, 256, F);
                else if (split) LAUNCH((k_few_first<L, W, kind.value, wd.value != 0, 1, true, false>), g1, 256, F);
                else if (pairs <= (size_t)n_experts * 8) LAUNCH((k_few_first<L, W, kind.value, wd.value != 0, 1, false, false>), g1, 256, F);
                else LAUNCH((k_few_first<L, W, kind.value, wd.value != 0, 2, false, false>), g1, 256, F);
            });
            if ((e = launched()) != TUNA_OK) return;              // the second kernel reads what the first has written
            with_type(out_type, [&](auto* o) {
                using O = Pointee<decltype(o)>;
                if (one) hipLaunchKernelGGL((k_few_second<W, kind.value, wd.value != 0, O, true>), g2, dim3(kFewSecond * 64), sums, (hipStream_t)stream, F);
                else hipLaunchKernelGGL((k_few_second<W, kind.value, wd.value != 0, O, false>), g2, dim3(kFewSecond * 64), sums, (hipStream_t)stream, F);
            });
        };
        if (weight_type == TUNA_BF16) both((unsigned short*)nullptr, Int<-1>{});
        else if (weight_type == TUNA_F4) both((Four*)nullptr, Int<TUNA_SCALE_E8>{});
        else if (scale_type == TUNA_SCALE_E8) both((uint8_t*)nullptr, Int<TUNA_SCALE_E8>{});
        else both((uint8_t*)nullptr, Int<TUNA_SCALE_F32>{});
    });
    return e != TUNA_OK ? e : launched();
}

}  // extern "C"
