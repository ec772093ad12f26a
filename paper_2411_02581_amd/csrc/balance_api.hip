// C entry points of the balance loss of include/tuna_moe.h: checks of the arguments and the choice of kernels.  No state is kept between calls.
#include "balance_kernels.h"
#include "moe_host.h"

using namespace moe;

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 28;

struct BalanceSizes {
    int64_t tiles; int tile;
    size_t counts, live, bytes;                       // offsets; the shares' sums come first
};

BalanceSizes balance_sizes(int64_t n, int experts, int groups) {
    BalanceSizes b;
    // a workgroup for each compute unit, of 16 tokens (a wave has one) to 128: 4096 tokens of 1024 experts 36 us a call in tiles of 128, 19 of 16
    const int64_t waves = ceil_div(n, 16 * 256);
    b.tile = 16 * (int)(waves < 1 ? 1 : waves > kBalanceTile / 16 ? kBalanceTile / 16 : waves);
    b.tiles = ceil_div(n, b.tile) + groups - 1;
    // room for the tiles of any batch of up to this size: at most 512, or those of the largest
    const int64_t few = ceil_div(n, 16), many = ceil_div(n, kBalanceTile) > 512 ? ceil_div(n, kBalanceTile) : 512, most = (few < many ? few : many) + groups - 1;
    size_t at = align16((size_t)most * experts * 4);
    b.counts = at; at += align16((size_t)most * experts * 4);
    b.live = at; at += align16((size_t)most * 4);
    b.bytes = at;
    return b;
}

bool balance_args(int64_t n, int experts, int groups) {
    return n >= 0 && experts >= 1 && experts <= TUNA_MOE_MAX_EXPERTS && groups >= 1 && groups <= TUNA_MOE_MAX_EXPERTS;
}

// A wave holds a token's logits in registers, as many as there may be of them.
template <class F> void held(int experts, F f) {
    if (experts <= 64) f(Int<1>{});
    else if (experts <= 128) f(Int<2>{});
    else if (experts <= 256) f(Int<4>{});
    else if (experts <= 512) f(Int<8>{});
    else f(Int<16>{});
}

}  // namespace

extern "C" {

int tuna_moe_balance_workspace(int64_t n_tokens, int n_experts, int groups, size_t* bytes) {
    if (!bytes || !balance_args(n_tokens, n_experts, groups)) return TUNA_ERR_ARG;
    if (n_tokens > kMostTokens) return TUNA_ERR_TOO_LARGE;
    *bytes = balance_sizes(n_tokens, n_experts, groups).bytes;
    return TUNA_OK;
}

int tuna_moe_balance(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, const int32_t* experts, int k,
                     const int32_t* group_rows, int groups, int32_t* counts, int32_t* tokens, float* shares, float* loss,
                     void* workspace, size_t workspace_bytes, void* stream) {
    if (!balance_args(n_tokens, n_experts, groups) || k < 1 || k > TUNA_MOE_MAX_K || !is_float(type)) return TUNA_ERR_ARG;
    if ((!group_rows && groups != 1) || !on(group_rows, 4) || !counts || !tokens || !shares || !loss || !on(counts, 4) || !on(tokens, 4) || !on(shares, 4) || !on(loss, 4))
        return TUNA_ERR_ARG;
    if (n_tokens > 0 && (!rows_ok(logits, size_of(type), ld, n_experts) || !experts || !on(experts, 4))) return TUNA_ERR_ARG;
    if (n_tokens > kMostTokens || n_tokens > kMaxRows / k) return TUNA_ERR_TOO_LARGE;
    const BalanceSizes s = balance_sizes(n_tokens, n_experts, groups);
    if (!workspace || !on(workspace, 16)) return TUNA_ERR_ARG;
    if (workspace_bytes < s.bytes) return TUNA_ERR_WORKSPACE_TOO_SMALL;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    char* ws = (char*)workspace;
    const Balance B = {logits, ld, n_tokens, n_experts, experts, k, group_rows, groups, s.tile, counts, tokens, shares, loss,
                       (float*)ws, (int32_t*)(ws + s.counts), (int32_t*)(ws + s.live)};
    // Up to a tile of one sequence: one workgroup and one launch for everything.
    const bool all = groups == 1 && !group_rows && n_tokens > 0 && n_tokens <= kBalanceTile;
    if (n_tokens > 0) {
        with_type(type, [&](auto* t) {
            using T = Pointee<decltype(t)>;
            held(n_experts, [&](auto per) {
                if (all) LAUNCH((k_balance_part<T, per.value, true>), dim3(1), 1024, B);
                else LAUNCH((k_balance_part<T, per.value, false>), dim3((unsigned)s.tiles), 1024, B);
            });
        });
        // the next kernel reads what this one has written: it is not launched behind one that was not
        const int e = launched();
        if (all || e != TUNA_OK) return e;
    }
    // Sequences of many tiles: sixteen waves for every 64 experts, and the loss in a launch of its own.
    if (s.tiles <= 32 * (int64_t)groups) {
        held(n_experts, [&](auto per) { LAUNCH((k_balance_join<per.value, true>), dim3(groups), 1024, B); });
        return launched();
    }
    LAUNCH((k_balance_join<1, false>), dim3(groups, (unsigned)ceil_div(n_experts, 64)), 1024, B);
    const int e = launched();
    if (e != TUNA_OK) return e;
    LAUNCH(k_balance_loss, dim3(groups), 1024, B);
    return launched();
}

int tuna_moe_balance_grad(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts,
                          const int32_t* group_rows, int groups, const int32_t* counts, const int32_t* tokens, const float* dloss,
                          int flags, void* dlogits, int64_t ld_dlogits, void* stream) {
    if (!balance_args(n_tokens, n_experts, groups) || !is_float(type) || (flags & ~TUNA_BALANCE_ADD) || (!group_rows && groups != 1) || !on(group_rows, 4)) return TUNA_ERR_ARG;
    if (n_tokens > kMostTokens) return TUNA_ERR_TOO_LARGE;
    if (n_tokens == 0) return TUNA_OK;
    if (!rows_ok(logits, size_of(type), ld, n_experts) || !rows_ok(dlogits, size_of(type), ld_dlogits, n_experts) || !counts || !tokens || !dloss || !on(counts, 4) ||
        !on(tokens, 4) || !on(dloss, 4))
        return TUNA_ERR_ARG;
    const int rc = tuna_host::ensure_device();
    if (rc != TUNA_OK) return rc;
    Balance B = {};
    B.logits = logits; B.ld = ld; B.tokens = n_tokens; B.experts = n_experts; B.group_rows = group_rows; B.groups = groups;
    B.counts = (int32_t*)counts; B.live = (int32_t*)tokens;
    // tiles of all sequences, and of the tokens before and behind them: each of these is at most a tile more than its length has
    const int64_t tiles = ceil_div(n_tokens, kBalanceGradTile) + groups - 1 + (group_rows ? 2 : 0);
    with_type(type, [&](auto* t) {
        using T = Pointee<decltype(t)>;
        held(n_experts, [&](auto per) {
            with_bool(flags & TUNA_BALANCE_ADD, [&](auto add) {
                LAUNCH((k_balance_grad<T, per.value, add.value != 0>), dim3((unsigned)tiles), 256, B, dloss, (T*)dlogits, ld_dlogits);
            });
        });
    });
    return launched();
}

}  // extern "C"
