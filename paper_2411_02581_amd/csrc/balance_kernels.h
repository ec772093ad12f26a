// Kernels of the balance loss of include/tuna_moe.h for gfx950.  Times in these comments are averages over a kernel trace.
#pragma once
#include "moe_common.h"

namespace moe {

constexpr int kBalanceTile = 128;      // the most tokens of a sequence that a workgroup adds up
constexpr int kBalanceGradTile = 32;   // and of which it makes the gradient

struct Balance {
    const void* logits; int64_t ld, tokens; int experts;
    const int32_t* chosen; int k;
    const int32_t* group_rows; int groups, tile;                  // tile: tokens of a workgroup
    int32_t* counts; int32_t* live; float* shares; float* loss;
    // workspace: what each tile has of every expert, [tiles, experts] each, and its tokens with an eligible expert
    float* part; int32_t* part_count; int32_t* part_live;
};

// A token's logits in a wave: lane i holds the experts i, i + 64, ...; one that is NaN or does not exist is -inf.
template <class T, int PER> __device__ __forceinline__ void load_logits(const T* row, int n_experts, int lane, float (&v)[PER]) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        v[i] = e < n_experts ? load1(row + e) : -__builtin_inff();
    }
}

// Their softmax in their place; false where no logit is eligible (all shares are 0 then).
template <int PER> __device__ __forceinline__ bool shares_of(float (&v)[PER]) {
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = v[i] == v[i] ? v[i] : -__builtin_inff();
        most = fmaxf(most, v[i]);
    }
    const unsigned top = wave_max(logit_key(most));
    most = key_logit(top);
    float sum = 0.f;
    if (most == __builtin_inff()) {                               // they share the whole equally
#pragma unroll
        for (int i = 0; i < PER; ++i) { v[i] = v[i] == most ? 1.f : 0.f; sum += v[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) { v[i] = top ? exp_32(v[i] - most) : 0.f; sum += v[i]; }
    }
    sum = wave_total(sum);
    const float r = __builtin_amdgcn_rcpf(sum), inverse = top ? __builtin_fmaf(__builtin_fmaf(-sum, r, 1.f), r, r) : 0.f;      // to a unit of the last place
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] *= inverse;
    return top != 0;
}

// A workgroup's sums of every expert's 64 bits and counts: the loss.
__device__ __forceinline__ void balance_loss(const Balance& B, int64_t g, double both, double all, double (&part)[2][16]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int d = 32; d; d >>= 1) { both += __shfl_xor(both, d); all += __shfl_xor(all, d); }
    if (lane == 0) { part[0][w] = both; part[1][w] = all; }
    __syncthreads();
    if (threadIdx.x) return;
    both = all = 0;
    for (int q = 0; q < 16; ++q) { both += part[0][q]; all += part[1][q]; }
    B.loss[g] = all > 0 ? (float)(B.experts * both / all) : 0.f;
}

// One workgroup per tile of a sequence: sixteen waves add up their tokens' shares, the logits of up to four under way together, then the waves' sums are
// added in their order.  ALL: the tile is the whole batch, one sequence, and the sums are the results.  65536 x 256 in 32 bits, 37 sequences: 67 MB, 24 us (2.8 TB/s:
// a wave's sums and largest logits take as long as its loads); 24 x 64 in one launch 4.8 us.
template <class T, int PER, bool ALL>
__global__ __launch_bounds__(1024) void k_balance_part(Balance B) {
    constexpr int U = PER <= 4 ? 4 : PER == 8 ? 2 : 1;
    __shared__ float sums[16][PER * 64];
    __shared__ int count[PER * 64];
    __shared__ int live[16];
    __shared__ double terms[2][16];
    Place pl = {0, 0, B.tokens, 0};
    if (!ALL) pl = find_tile(B.group_rows, B.groups, B.tokens, B.tile, blockIdx.x);
    if (pl.group < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < PER * 64) count[tid] = 0;
    __syncthreads();
    float sum[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) sum[i] = 0.f;
    int mine = 0;
    for (int64_t t0 = pl.first + w; t0 < pl.end; t0 += 16 * U) {
        float p[U][PER];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + u * 16 < pl.end) load_logits<T, PER>((const T*)B.logits + (t0 + u * 16) * B.ld, B.experts, lane, p[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + u * 16 >= pl.end) break;
            mine += shares_of<PER>(p[u]);
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[i] += p[u][i];
        }
    }
    for (int64_t i = pl.first * B.k + tid; i < pl.end * B.k; i += 1024) {
        const int e = B.chosen[i];
        if (e >= 0 && e < B.experts) atomicAdd(&count[e], 1);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) sums[w][i * 64 + lane] = sum[i];
    if (lane == 0) live[w] = mine;
    __syncthreads();
    int n = 0;
    for (int q = 0; q < 16; ++q) n += live[q];
    float s = 0.f;                                                // a thread per expert there can be
    if (tid < B.experts) for (int q = 0; q < 16; ++q) s += sums[q][tid];
    if (ALL) {
        const double share = n > 0 ? (double)s / n : 0.;
        const int c = tid < B.experts ? count[tid] : 0;
        if (tid < B.experts) {
            B.counts[tid] = c;
            B.shares[tid] = (float)share;
        }
        if (tid == 0) B.live[0] = n;
        balance_loss(B, 0, c * share, c, terms);
        return;
    }
    const int64_t at = (int64_t)blockIdx.x * B.experts;
    if (tid < B.experts) {
        B.part[at + tid] = s;
        B.part_count[at + tid] = count[tid];
    }
    if (tid == 0) B.part_live[blockIdx.x] = n;
}

// A workgroup per sequence: its sixteen waves are C columns of 64 experts and 16 / C runs of its tiles; sums in 64 bits.  WHOLE: that is all experts, and the
// loss follows; else blockIdx.y counts the columns, and k_balance_loss makes it.
template <int C, bool WHOLE>
__global__ __launch_bounds__(1024) void k_balance_join(Balance B) {
    constexpr int R = 16 / C;
    __shared__ double sums[R][C * 64];
    __shared__ int counts[R][C * 64], live[R];
    __shared__ double terms[2][16];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), run = w / C, g = blockIdx.x, col = (w % C) * 64 + lane, e0 = blockIdx.y * (C * 64), e = e0 + col;
    int64_t first, tiles;
    group_blocks(B.group_rows, B.groups, g, B.tokens, first, tiles, B.tile);
    double s = 0;
    int c = 0, n = 0;
    const int there = e < B.experts ? e : B.experts - 1;          // (the others' sums are nobody's)
#pragma unroll 8
    for (int64_t i = first + run; i < first + tiles; i += R) {
        s += (double)B.part[i * B.experts + there];
        c += B.part_count[i * B.experts + there];
        n += B.part_live[i];
    }
    sums[run][col] = s;
    counts[run][col] = c;
    if (lane == 0) live[run] = n;                                 // (the columns' waves have the same)
    __syncthreads();
    s = 0;
    c = n = 0;
    for (int q = 0; q < R; ++q) n += live[q];
    if (tid < C * 64 && e0 + tid < B.experts) {                   // a thread per expert
        for (int q = 0; q < R; ++q) { s += sums[q][tid]; c += counts[q][tid]; }
        s = n > 0 ? s / n : 0.;
        B.counts[(int64_t)g * B.experts + e0 + tid] = c;
        B.shares[(int64_t)g * B.experts + e0 + tid] = (float)s;
    }
    if (tid == 0 && blockIdx.y == 0) B.live[g] = n;
    if (WHOLE) balance_loss(B, g, c * s, c, terms);
}

// A workgroup per sequence, from its counts and shares.
__global__ __launch_bounds__(1024) void k_balance_loss(Balance B) {
    __shared__ double terms[2][16];
    const int64_t at = (int64_t)blockIdx.x * B.experts + threadIdx.x;
    const bool there = (int)threadIdx.x < B.experts;
    const double c = there ? B.counts[at] : 0, s = there ? B.shares[at] : 0.f;
    balance_loss(B, blockIdx.x, c * s, c, terms);
}

// Every wave has the fractions f_e = counts_e / C of its tile's sequence in registers: dl_i = dloss E / N p_i (f_i - sum over e of f_e p_e).  The tiles behind the
// sequences' are the tokens outside every sequence: those before the first bound, then those behind the last.  Bound by memory: 65536 x 256 in 32 bits, 134 MB, 27 us
// (5.1 TB/s).
template <class T, int PER, bool ADD>
__global__ __launch_bounds__(256) void k_balance_grad(Balance B, const float* dloss, T* dlogits, int64_t ld_d) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place pl = find_tile(B.group_rows, B.groups, B.tokens, kBalanceGradTile, blockIdx.x);
    if (pl.group < 0) {
        if (ADD || !B.group_rows) return;
        int last = 0;
        for (int g = lane; g <= B.groups; g += 64) { const int b = bound_at(B.group_rows, g, B.tokens); last = b > last ? b : last; }
        last = (int)wave_max((unsigned)last);
        const int before = bound_at(B.group_rows, 0, B.tokens);
        int64_t at = (int64_t)blockIdx.x - count_tiles(B.group_rows, B.groups, B.tokens, kBalanceGradTile);
        const int64_t tiles = ((int64_t)before + kBalanceGradTile - 1) / kBalanceGradTile;
        pl.first = at < tiles ? at * kBalanceGradTile : last + (at - tiles) * kBalanceGradTile;
        pl.end = at < tiles ? before : B.tokens;
        if (pl.first + kBalanceGradTile < pl.end) pl.end = pl.first + kBalanceGradTile;
        for (int64_t t = pl.first + w; t < pl.end; t += 4)
            for (int e = lane; e < B.experts; e += 64) store1(dlogits + t * ld_d + e, 0.f);
        return;
    }
    float f[PER];
    int all = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane, c = e < B.experts ? B.counts[(int64_t)pl.group * B.experts + e] : 0;
        all += c;
        f[i] = (float)c;
    }
    for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d);
    const int n = B.live[pl.group];
    const float slope = all > 0 && n > 0 ? dloss[pl.group] * ((float)B.experts / (float)n) : 0.f, inverse = all > 0 ? 1.f / (float)all : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) f[i] *= inverse;
    constexpr int U = PER <= 4 ? 4 : PER == 8 ? 2 : 1;            // tokens whose logits are under way together
    for (int64_t t0 = pl.first + w; t0 < pl.end; t0 += 4 * U) {
        float p[U][PER], before[U][PER];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t t = t0 + u * 4;
            if (t >= pl.end) break;
            load_logits<T, PER>((const T*)B.logits + t * B.ld, B.experts, lane, p[u]);
            if (ADD) load_logits<T, PER>(dlogits + t * ld_d, B.experts, lane, before[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t t = t0 + u * 4;
            if (t >= pl.end) break;
            shares_of<PER>(p[u]);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) dot += p[u][i] * f[i];
            dot = wave_total(dot);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * 64 + lane;
                const float d = slope * p[u][i] * (f[i] - dot);
                if (e < B.experts) store1(dlogits + t * ld_d + e, ADD ? before[u][i] + d : d);
            }
        }
    }
}

}  // namespace moe
