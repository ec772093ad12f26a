// Kernels of the balance loss of include/tuna_moe.h for gfx950.  Times in these comments are averages over a kernel trace.
#pragma once
#include "moe_common.h"

namespace moe {

constexpr int kBalanceTile = 256;      // tokens of a sequence that a workgroup adds up
constexpr int kBalanceGradTile = 32;   // and of which it makes the gradient

struct Balance {
    const void* logits; int64_t ld, tokens; int experts;
    const int32_t* chosen; int k;
    const int32_t* group_rows; int groups;
    int32_t* counts; int32_t* live; float* shares; float* loss;
    // workspace: what each tile has of every expert, [tiles, experts] each, and its tokens with an eligible expert; C and the loss's sum of 64 experts
    float* part; int32_t* part_count; int32_t* part_live; double* terms;
};

// A token's softmax by a wave: lane i holds the experts i, i + 64, ...; false where no logit is eligible (all shares are 0 then).
template <class T, int PER> __device__ __forceinline__ bool shares_of(const T* row, int n_experts, int lane, float (&p)[PER]) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        p[i] = e < n_experts ? load1(row + e) : -__builtin_inff();
        const unsigned key = logit_key(p[i]);
        top = key > top ? key : top;
    }
    top = wave_max(top);
    const float most = key_logit(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p[i] = top ? exp_share(p[i], most) : 0.f;
        sum += p[i];
    }
    sum = wave_total(sum);
    const float inverse = top ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) p[i] *= inverse;
    return top != 0;
}

// One workgroup per tile of a sequence: sixteen waves add up their tokens' shares, then the waves' sums are added in their order.
template <class T, int PER>
__global__ __launch_bounds__(1024) void k_balance_part(Balance B) {
    __shared__ float sums[16][PER * 64];
    __shared__ int count[PER * 64];
    __shared__ int live[16];
    const Place pl = find_tile(B.group_rows, B.groups, B.tokens, kBalanceTile, blockIdx.x);
    if (pl.group < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < PER * 64) count[tid] = 0;
    __syncthreads();
    float sum[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) sum[i] = 0.f;
    int mine = 0;
    for (int64_t t = pl.first + w; t < pl.end; t += 16) {
        float p[PER];
        mine += shares_of<T, PER>((const T*)B.logits + t * B.ld, B.experts, lane, p);
#pragma unroll
        for (int i = 0; i < PER; ++i) sum[i] += p[i];
    }
    for (int64_t i = pl.first * B.k + tid; i < pl.end * B.k; i += 1024) {
        const int e = B.chosen[i];
        if (e >= 0 && e < B.experts) atomicAdd(&count[e], 1);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) sums[w][i * 64 + lane] = sum[i];
    if (lane == 0) live[w] = mine;
    __syncthreads();
    const int64_t at = (int64_t)blockIdx.x * B.experts;
    for (int e = tid; e < B.experts; e += 1024) {
        float s = 0.f;
        for (int q = 0; q < 16; ++q) s += sums[q][e];
        B.part[at + e] = s;
        B.part_count[at + e] = count[e];
    }
    if (tid == 0) {
        int n = 0;
        for (int q = 0; q < 16; ++q) n += live[q];
        B.part_live[blockIdx.x] = n;
    }
}

// A workgroup per sequence and 64 experts: four waves share its tiles, in 64 bits.
__global__ __launch_bounds__(256) void k_balance_join(Balance B) {
    __shared__ double sums[4][64];
    __shared__ int counts[4][64], live[4];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = blockIdx.x, e = blockIdx.y * 64 + lane;
    int64_t first, tiles;
    group_blocks(B.group_rows, B.groups, g, B.tokens, first, tiles, kBalanceTile);
    double s = 0;
    int c = 0, n = 0;
    for (int64_t i = first + w; i < first + tiles; i += 4) {
        if (e < B.experts) {
            s += (double)B.part[i * B.experts + e];
            c += B.part_count[i * B.experts + e];
        }
        n += B.part_live[i];
    }
    sums[w][lane] = s;
    counts[w][lane] = c;
    if (lane == 0) live[w] = n;
    __syncthreads();
    if (w) return;
    for (int q = 1; q < 4; ++q) { s += sums[q][lane]; c += counts[q][lane]; n += live[q]; }
    s = n > 0 ? s / n : 0.;
    if (e < B.experts) {
        B.counts[(int64_t)g * B.experts + e] = c;
        B.shares[(int64_t)g * B.experts + e] = (float)s;
    }
    double both = c * s, all = c;
    for (int d = 32; d; d >>= 1) { both += __shfl_xor(both, d); all += __shfl_xor(all, d); }
    if (lane == 0) {
        double* to = B.terms + ((int64_t)g * gridDim.y + blockIdx.y) * 2;
        to[0] = both;
        to[1] = all;
        if (blockIdx.y == 0) B.live[g] = n;
    }
}

// A thread per sequence.
__global__ __launch_bounds__(256) void k_balance_loss(Balance B, int parts) {
    const int g = blockIdx.x * 256 + threadIdx.x;
    if (g >= B.groups) return;
    double both = 0, all = 0;
    for (int i = 0; i < parts; ++i) {
        both += B.terms[((int64_t)g * parts + i) * 2];
        all += B.terms[((int64_t)g * parts + i) * 2 + 1];
    }
    B.loss[g] = all > 0 ? (float)(B.experts * both / all) : 0.f;
}

// Every wave has the fractions f_e = counts_e / C of its tile's sequence in registers: dl_i = dloss E / N p_i (f_i - sum over e of f_e p_e).  The tiles behind the
// sequences' are the tokens outside every sequence: those before the first bound, then those behind the last.
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
    for (int64_t t = pl.first + w; t < pl.end; t += 4) {
        float p[PER];
        shares_of<T, PER>((const T*)B.logits + t * B.ld, B.experts, lane, p);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) dot += p[i] * f[i];
        dot = wave_total(dot);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = i * 64 + lane;
            if (e >= B.experts) continue;
            T* to = dlogits + t * ld_d + e;
            store1(to, (ADD ? load1(to) : 0.f) + slope * p[i] * (f[i] - dot));
        }
    }
}

}  // namespace moe
