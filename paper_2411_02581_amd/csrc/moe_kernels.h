// Kernels of include/tuna_moe.h for gfx950: routing, 8-bit quantisation, products with a scale for each block of 128, the sum
// over a token's experts, and the whole layer for a few tokens.  Times in these comments are averages over a kernel trace; where one is given in brackets
// it is the least of the trace.
#pragma once
#include "moe_common.h"

namespace moe {

// ------------------------------------------------------------------------------------------------ routing
//
// One wave per token: lane i holds the logits i, i + 64, ...; k rounds take the largest key each.  The largest of the wave and where it is
// are scalars: a round is some thirty vector instructions, a ballot for each register and scalar work beside it.  65536 x 256 in 32 bits, k = 8:
// 51 us, bound by these instructions (the logits alone take 15 us to read).
// Lane j < k receives choice number j (-1: none) and its weight.
template <class T, int PER>
__device__ __forceinline__ void choose(const T* row, int n_experts, int k, int renorm, int lane, int& chosen, float& weight) {
    float v[PER];
    unsigned key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * 64 + lane;
        v[i] = load1(row + (e < n_experts ? e : n_experts - 1));
        key[i] = e < n_experts ? logit_key(v[i]) : 0u;
    }
    unsigned first = 0;                                           // the largest key of all
    int best = 0;                                                 // lane j: the key of choice number j
    chosen = -1;
    for (int j = 0; j < k; ++j) {
        unsigned m = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) m = key[i] > m ? key[i] : m;
        m = wave_max(m);
        if (m == 0) break;
        int e = -1;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {                      // the lowest index that has it
            const unsigned long long b = __ballot(key[i] == m);
            e = b ? i * 64 + __ffsll((long long)b) - 1 : e;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = i * 64 + lane == e ? 0u : key[i];
        first = j == 0 ? m : first;
        chosen = lane == j ? e : chosen;
        best = lane == j ? (int)m : best;
    }
    const float top = key_logit(first);
    const float mine = chosen < 0 ? 0.f : exp_share(key_logit((unsigned)best), top);
    float total = mine;
    if (!renorm) {
        total = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) total += i * 64 + lane < n_experts ? exp_share(v[i], top) : 0.f;
    }
    total = wave_total(total);
    weight = chosen < 0 ? 0.f : mine / total;
}

template <class T, int PER>
__global__ __launch_bounds__(256) void k_route_choose(const T* logits, int64_t ld, int64_t n_tokens, int n_experts, int k, int renorm,
                                                      int32_t* experts, float* weights) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= n_tokens) return;
    int e;
    float weight;
    choose<T, PER>(logits + t * ld, n_experts, k, renorm, lane, e, weight);
    if (lane < k) {
        experts[t * k + lane] = e;
        weights[t * k + lane] = weight;
    }
}

// Everything for up to 64 tokens without a plan, in one workgroup: sixteen waves choose, then every expert has a word with a bit per token.
// One launch in place of four: 24 tokens of 64 experts 4.6 us in place of 10.1, and less on the host.
template <class T, int PER>
__global__ __launch_bounds__(1024) void k_route_small(const T* logits, int64_t ld, int n_tokens, int n_experts, int k, int renorm, int32_t* experts,
                                                      float* weights, int32_t* slots, int32_t* expert_rows) {
    __shared__ unsigned long long word[TUNA_MOE_MAX_EXPERTS];
    __shared__ int first[TUNA_MOE_MAX_EXPERTS + 1];
    __shared__ int part[16];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    word[tid] = 0;                                                // a thread per expert there can be
    __syncthreads();
    int mine[4];                                                  // lane j: the choice number j of the wave's tokens w, w + 16, ...
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + w;
        mine[i] = -1;
        if (t >= n_tokens) break;
        float weight;
        choose<T, PER>(logits + t * ld, n_experts, k, renorm, lane, mine[i], weight);
        if (lane < k) {
            experts[t * k + lane] = mine[i];
            weights[t * k + lane] = weight;
            if (mine[i] >= 0) atomicOr(&word[mine[i]], 1ull << t);
        }
    }
    __syncthreads();
    const int count = __popcll(word[tid]), inc = wave_scan(count, lane);
    if (lane == 63) part[w] = inc;
    __syncthreads();
    int at = inc - count;
    for (int i = 0; i < w; ++i) at += part[i];
    first[tid] = at;
    if (tid < n_experts) expert_rows[tid] = at;
    if (tid == n_experts - 1) expert_rows[n_experts] = at + count;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + w;
        if (t >= n_tokens) break;
        if (lane < k) slots[t * k + lane] = mine[i] < 0 ? -1 : first[mine[i]] + __popcll(word[mine[i]] & ((1ull << t) - 1));
    }
}

// (65536 x 8 pairs of 256 experts: 7.6 us for the count, 4.9 for the columns, 11.2 for the places with the plan's 1.5 MB.)
// One workgroup per shard of tokens: how many of its pairs every expert has, and each pair's place among them.  A batch is
// 64 tokens: a bit per token in a word per expert, so the order of the atomics does not matter.
__global__ __launch_bounds__(256) void k_route_count(const int32_t* experts, int64_t n_tokens, int n_experts, int k, int64_t shard,
                                                     int32_t* counts, int32_t* places) {
    __shared__ unsigned long long word[TUNA_MOE_MAX_EXPERTS];
    __shared__ int base[TUNA_MOE_MAX_EXPERTS];
    const int64_t first = (int64_t)blockIdx.x * shard;
    const int64_t last = first + shard < n_tokens ? first + shard : n_tokens;
    for (int e = threadIdx.x; e < n_experts; e += 256) { word[e] = 0; base[e] = 0; }
    __syncthreads();
    for (int64_t t0 = first; t0 < last; t0 += 64) {
        const int n = (int)(last - t0 < 64 ? last - t0 : 64) * k;
        for (int i = threadIdx.x; i < n; i += 256) {
            const int e = experts[t0 * k + i];
            if (e >= 0) atomicOr(&word[e], 1ull << (i / k));
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += 256) {
            const int e = experts[t0 * k + i];
            if (e >= 0) places[t0 * k + i] = base[e] + __popcll(word[e] & ((1ull << (i / k)) - 1));
        }
        __syncthreads();
        for (int e = threadIdx.x; e < n_experts; e += 256) { base[e] += __popcll(word[e]); word[e] = 0; }
        __syncthreads();
    }
    for (int e = threadIdx.x; e < n_experts; e += 256) counts[(int64_t)blockIdx.x * n_experts + e] = base[e];
}

// Exclusive prefix of a[0 .. n) in LDS by a workgroup of 256 threads, n <= 1024; a[n] receives the sum.
__device__ __forceinline__ void scan_lds(int* a, int n, int* tmp) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int v[4], s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = tid * 4 + i < n ? a[tid * 4 + i] : 0; s += v[i]; }
    const int inc = wave_scan(s, lane);
    if (lane == 63) tmp[w] = inc;
    __syncthreads();
    int off = inc - s;
    for (int i = 0; i < w; ++i) off += tmp[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (tid * 4 + i < n) a[tid * 4 + i] = off;
        off += v[i];
    }
    if (tid == 255) a[n] = off;
    __syncthreads();
}

// One workgroup per expert: its column of the shards' counts becomes a prefix, and its sum.
__global__ __launch_bounds__(256) void k_route_columns(const int32_t* counts, int shards, int n_experts, int32_t* before, int32_t* totals) {
    __shared__ int col[TUNA_MOE_MAX_EXPERTS + 1];
    __shared__ int tmp[4];
    const int e = blockIdx.x;
    for (int i = threadIdx.x; i < shards; i += 256) col[i] = counts[(int64_t)i * n_experts + e];
    __syncthreads();
    scan_lds(col, shards, tmp);
    for (int i = threadIdx.x; i < shards; i += 256) before[(int64_t)i * n_experts + e] = col[i];
    if (threadIdx.x == 0) totals[e] = col[shards];
}

// One workgroup per shard i: the slots of its pairs, row i of the send side and row i of the receive side of the plan.
__global__ __launch_bounds__(256) void k_route_place(const int32_t* experts, const int32_t* counts, const int32_t* before, const int32_t* totals,
                                                     int64_t n_tokens, int n_experts, int k, int64_t shard, int shards, const int32_t* places,
                                                     int32_t* slots, int32_t* expert_rows, int64_t row_bytes,
                                                     int32_t* sendcounts, int64_t* sdispls, int32_t* recvcounts, int64_t* rdispls) {
    __shared__ int row[TUNA_MOE_MAX_EXPERTS + 1];
    __shared__ int mine[TUNA_MOE_MAX_EXPERTS + 1];
    __shared__ int tmp[4];
    __shared__ int first_row;
    const int i = blockIdx.x;
    const bool plan = sendcounts != nullptr;
    for (int e = threadIdx.x; e < n_experts; e += 256) {
        row[e] = totals[e];
        mine[e] = plan ? counts[(int64_t)i * n_experts + e] : 0;
    }
    __syncthreads();
    scan_lds(row, n_experts, tmp);                                // row[e]: the first row of expert e
    if (i == 0) for (int e = threadIdx.x; e <= n_experts; e += 256) expert_rows[e] = row[e];
    if (plan) {
        // the pairs of the shards before this one: what they have of every expert
        int s = 0;
        for (int e = threadIdx.x; e < n_experts; e += 256) s += before[(int64_t)i * n_experts + e];
        if (threadIdx.x == 0) first_row = 0;
        __syncthreads();
        atomicAdd(&first_row, s);
        __syncthreads();
        scan_lds(mine, n_experts, tmp);
        for (int e = threadIdx.x; e < n_experts; e += 256) {
            const int64_t at = (int64_t)i * n_experts + e;
            sendcounts[at] = (int32_t)((mine[e + 1] - mine[e]) * row_bytes);
            sdispls[at] = (int64_t)(first_row + mine[e]) * row_bytes;
            // as expert i, from shard e
            recvcounts[at] = (int32_t)(counts[(int64_t)e * n_experts + i] * row_bytes);
            rdispls[at] = (int64_t)(row[i] + before[(int64_t)e * n_experts + i]) * row_bytes;
        }
    }
    const int64_t first = (int64_t)i * shard * k;
    const int64_t last = ((int64_t)(i + 1) * shard < n_tokens ? (int64_t)(i + 1) * shard : n_tokens) * k;
    for (int64_t p = first + threadIdx.x; p < last; p += 256) {
        const int e = experts[p];
        slots[p] = e < 0 ? -1 : places[p] + (plan ? first_row + mine[e] : row[e] + before[(int64_t)i * n_experts + e]);
    }
}

// N neighbours of a row in one load or store, N = 4 or 8; rows start on 16 bytes and N divides what is left of them.
template <int N> __device__ __forceinline__ void load_n(const float* p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const v4f a = *(const v4f*)(p + i);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[i + q] = a[q];
    }
}
template <int N> __device__ __forceinline__ void load_n(const unsigned short* p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const v2u a = *(const v2u*)(p + i);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[i + q] = bf16_bits((unsigned short)(a[q >> 1] >> 16 * (q & 1)));
    }
}
template <int N> __device__ __forceinline__ void store_n(float* p, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *(v4f*)(p + i) = v4f{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
template <int N> __device__ __forceinline__ void store_n(unsigned short* p, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
        *(v2u*)(p + i) = v2u{(unsigned)to_bf16(v[i]) | (unsigned)to_bf16(v[i + 1]) << 16, (unsigned)to_bf16(v[i + 2]) | (unsigned)to_bf16(v[i + 3]) << 16};
}

// A workgroup of four waves, one token each.  p_i = weight of the first choice * exp(l_i - its logit): no sum has to be formed again.  N > 1:
// a lane has N neighbours (four up to 256 experts, so that all lanes have some, else eight).  65536 x 256 in 32 bits: 26 us, 5.2 TB/s.
template <class T, int N>
__global__ __launch_bounds__(256) void k_route_grad(const T* logits, int64_t ld, int64_t n_tokens, int n_experts, int k, int renorm,
                                                    const int32_t* experts, const float* weights, const float* dweights, T* dlogits, int64_t ld_d) {
    __shared__ __align__(16) float g[4][TUNA_MOE_MAX_EXPERTS];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = (int64_t)blockIdx.x * 4 + w;
    if (t >= n_tokens) return;
    const T* row = logits + t * ld;
    const int e = lane < k ? experts[t * k + lane] : -1;
    const float wt = lane < k ? weights[t * k + lane] : 0.f, d = lane < k ? dweights[t * k + lane] : 0.f;
    constexpr int M = N > 1 ? N : 4;
    float l[M] = {};
    if (N > 1 && !renorm && lane * M < n_experts) load_n<M>(row + lane * M, l);
    if (N > 1) {
        for (int i = lane * 4; i < n_experts; i += 256) *(v4f*)&g[w][i] = v4f{0.f, 0.f, 0.f, 0.f};
    } else {
        for (int i = lane; i < n_experts; i += 64) g[w][i] = 0.f;
    }
    wave_lds_done();
    const bool there = e >= 0 && e < n_experts;
    const float sum = wave_total(there ? wt * d : 0.f);
    if (there) g[w][e] = renorm ? wt * (d - sum) : d;
    const int e0 = __builtin_amdgcn_readfirstlane(there ? e : -1);
    const float w0 = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wt)));
    const float top = e0 < 0 ? 0.f : load1(row + e0);
    wave_lds_done();
    auto slope = [&](float logit, float v) { return renorm ? v : e0 < 0 ? 0.f : w0 * exp_share(logit, top) * (v - sum); };
    if (N > 1) {
        for (int at = lane * M; at < n_experts; at += 64 * M) {
            if (at >= 64 * M && !renorm) load_n<M>(row + at, l);
            float o[M];
#pragma unroll
            for (int i = 0; i < M; ++i) o[i] = slope(l[i], g[w][at + i]);
            store_n<M>(dlogits + t * ld_d + at, o);
        }
    } else {
        for (int i = lane; i < n_experts; i += 64) store1(dlogits + t * ld_d + i, slope(renorm ? 0.f : load1(row + i), g[w][i]));
    }
}

// ------------------------------------------------------------------------------------------------ quantisation

struct Scale { float value; unsigned stored; float inverse; };   // inverse: what scaled() multiplies by, 0: it divides

// The scale of a block whose largest finite magnitude is `peak`.
template <int KIND> __device__ __forceinline__ Scale scale_of(float peak) {
    Scale s;
    float v = __fdiv_rn(peak, 448.f);
    v = v < 0x1p-126f ? 0x1p-126f : v;
    v = peak == 0.f ? 1.f : v;
    if (KIND == TUNA_SCALE_E8) {
        s.stored = (__float_as_uint(v) + 0x7fffffu) >> 23;        // the exponent of the next power of two
        s.value = __uint_as_float(s.stored << 23);
        s.inverse = __uint_as_float((254u - s.stored) << 23);     // a normal number: the largest scale is below 2^120
    } else {
        s.stored = __float_as_uint(v);
        s.value = v;
        s.inverse = v < 0x1p-90f ? 0.f : __fdiv_rn(1.f, v);
    }
    return s;
}

// v / scale, rounded once.  A power of two: a product.  Else the product with the rounded inverse and one correction by what it leaves,
// which gives the rounded quotient (Markstein) as long as that remainder does not underflow: below 2^-90 it divides.
template <int KIND> __device__ __forceinline__ float scaled(float v, const Scale& s) {
    if (KIND == TUNA_SCALE_E8) return v * s.inverse;
    if (s.inverse == 0.f) return __fdiv_rn(v, s.value);
    const float q = v * s.inverse;
    return copysignf(__builtin_fmaf(__builtin_fmaf(-q, s.value, v), s.inverse, q), v);      // (the sums lose the sign of -0)
}

// Four values as e4m3, the first in the lowest byte.
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
    return (unsigned)p;
}

template <int KIND> __device__ __forceinline__ v2u quantise8(const float (&v)[8], const Scale& s) {
    float u[8];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] = scaled<KIND>(v[i], s);
        odd |= !(fabsf(v[i]) < __builtin_inff());
    }
    v2u q = {pack4(u[0], u[1], u[2], u[3]), pack4(u[4], u[5], u[6], u[7])};
    if (odd) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(v[i]) < __builtin_inff())) q[i >> 2] |= 0x7fu << (8 * (i & 3));
    }
    return q;
}

__device__ __forceinline__ float max16(float v) {                 // over 16 neighbouring lanes
#pragma unroll
    for (int d = 8; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Sixteen lanes per block of 128 values, eight each; two blocks in turn, whose loads are under way together.  Bound by memory: 16384 x 4096 of
// bf16 to four records each 92 us (88), 4.4 TB/s; 20011 x 1792 gated 54 us (52), 3.3 TB/s.
template <class T, int KIND, int ACT, bool WIDE>
__global__ __launch_bounds__(256) void k_quantise(const T* x, int64_t ldx, unsigned total, int64_t cols, const int32_t* slots, int copies, int64_t out_rows,
                                                  uint8_t* q, int64_t ldq, void* scales, int64_t ld_scales) {
    const unsigned nb = (unsigned)blocks_of(cols), at0 = blockIdx.x * 32 + (threadIdx.x >> 4);
    float v[2][8], up[2][8];
    unsigned row[2], block[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const unsigned at = at0 + u * 16 < total ? at0 + u * 16 : total - 1;
        row[u] = at / nb;
        block[u] = at - row[u] * nb;
        const int64_t c = (int64_t)block[u] * kBlock + (threadIdx.x & 15) * 8;
        const T* p = x + row[u] * ldx + c;
        load8<WIDE>(p, cols - c, v[u]);
        if (ACT == TUNA_ACT_SWIGLU) load8<WIDE>(p + cols, cols - c, up[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (at0 + u * 16 >= total) break;                         // (sixteen lanes together)
        const int64_t r = row[u], b = block[u], c = b * kBlock + (threadIdx.x & 15) * 8, left = cols - c;
        if (ACT == TUNA_ACT_SWIGLU) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = i < left ? gate_of(v[u][i]).silu * up[u][i] : 0.f;
        }
        float peak = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) peak = fmaxf(peak, finite_abs(v[u][i]));
        const Scale s = scale_of<KIND>(max16(peak));
        const v2u o = quantise8<KIND>(v[u], s);
        for (int j = 0; j < copies; ++j) {
            int64_t to = r;
            if (slots) {
                to = slots[r * copies + j];
                if (to < 0 || to >= out_rows) continue;
            }
            uint8_t* d = q + to * ldq + c;
            if (WIDE && left >= 8) {
                *(v2u*)d = o;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (i < left) d[i] = (uint8_t)(o[i >> 2] >> (8 * (i & 3)));
            }
            if ((threadIdx.x & 15) == 0) {
                if (KIND == TUNA_SCALE_E8) ((uint8_t*)scales)[to * ld_scales + b] = (uint8_t)s.stored;
                else ((unsigned*)scales)[to * ld_scales + b] = s.stored;
            }
        }
    }
}

// Bound by memory and the two passes through the LDS: 12005 x 2048 and x 2736 of bf16 26 and 36 us, 2.9 TB/s.
// A tile of 128 rows by 128 columns: thread (16 column chunks of 8) x (16 row chunks of 8).
template <class T, int KIND, bool WIDE>
__global__ __launch_bounds__(256) void k_quantise_columns(const T* x, int64_t ldx, int64_t rows, int64_t cols, const int32_t* group_rows, int groups,
                                                          uint8_t* q, int64_t ldq, void* scales, int64_t ld_scales) {
    __shared__ float peaks[16][kBlock];
    __shared__ Scale column[kBlock];
    __shared__ __align__(16) uint8_t tile[kBlock][kBlock + 16];
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
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) p = fmaxf(p, finite_abs(v[i][j]));
        peaks[ry][cx * 8 + j] = p;
    }
    __syncthreads();
    if (threadIdx.x < kBlock) {                                   // a thread per column: its largest, its scale
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) p = fmaxf(p, peaks[i][threadIdx.x]);
        const Scale s = scale_of<KIND>(p);
        column[threadIdx.x] = s;
        const int64_t to = (int64_t)blockIdx.y * kBlock + threadIdx.x;
        if (to < cols) {
            if (KIND == TUNA_SCALE_E8) ((uint8_t*)scales)[to * ld_scales + pl.block] = (uint8_t)s.stored;
            else ((unsigned*)scales)[to * ld_scales + pl.block] = s.stored;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float col[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) col[i] = v[i][j];
        *(v2u*)&tile[cx * 8 + j][ry * 8] = quantise8<KIND>(col, column[cx * 8 + j]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBlock * 8; i += 256) {
        const int row = i >> 3, ch = i & 7;
        const int64_t to = (int64_t)blockIdx.y * kBlock + row;
        if (to >= cols) continue;
        uint8_t* d = q + to * ldq + pl.block * kBlock + ch * 16;
        const v4u val = *(const v4u*)&tile[row][ch * 16];
        if ((((uintptr_t)q | (uintptr_t)ldq) & 15) == 0) *(v4u*)d = val;
        else for (int b = 0; b < 16; ++b) d[b] = (uint8_t)(val[b >> 2] >> (8 * (b & 3)));
    }
}

// Bound by memory: 20011 x 2 x 1792 of bf16 58 us (56), 6.2 TB/s with what is still in the caches.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_swiglu_grad(const T* x, int64_t ldx, const T* dh, int64_t ld_dh, int64_t rows, int64_t cols, T* dx, int64_t ld_dx) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, left = cols - c, r = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (left <= 0 || r >= rows) return;
    float g[8], u[8], d[8];
    load8<WIDE>(x + r * ldx + c, left, g);
    load8<WIDE>(x + r * ldx + cols + c, left, u);
    load8<WIDE>(dh + r * ld_dh + c, left, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Gate t = gate_of(g[i]);
        const float s = t.sigmoid, act = t.silu;
        const float dg = d[i] * u[i] * s * (1.f + g[i] * (1.f - s));
        u[i] = d[i] * act;
        g[i] = dg;
    }
    store8<WIDE>(dx + r * ld_dx + c, left, g);
    store8<WIDE>(dx + r * ld_dx + cols + c, left, u);
}

// ------------------------------------------------------------------------------------------------ products in 8 bits

// Operands of a product out[i, j] = sum over k of a[i, k] * b[j, k].  Rows a are the activations (or dy transposed), rows b the weights
// (or x transposed).
struct Product {
    const uint8_t* a; int64_t lda; const void* as; int64_t ld_as;
    const uint8_t* b; int64_t ldb; int64_t b_group; const void* bs; int64_t ld_bs; int64_t bs_group;
    const int32_t* group_rows; int groups;
    void* out; int64_t ldo; int64_t out_group;
    int64_t m, n, k;                   // rows a, rows b, length (by columns: rows of all groups)
};

// A stored scale as the matrix core wants it (E8) or as its value.
template <int KIND> __device__ __forceinline__ unsigned scale_at(const void* s, int64_t i) {
    return KIND == TUNA_SCALE_E8 ? (unsigned)((const uint8_t*)s)[i] : ((const unsigned*)s)[i];
}

template <int KIND> __device__ __forceinline__ float scale_float(unsigned v) {
    if (KIND != TUNA_SCALE_E8) return __uint_as_float(v);
    return v == 0 ? 0x1p-127f : v == 255 ? __builtin_nanf("") : __uint_as_float(v << 23);
}

// Eight e4m3 values as bf16, which holds every one of them exactly.
__device__ __forceinline__ v8b widen8(unsigned a, unsigned b) {
    const v2b p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const v2b r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return v8b{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// 16 x 16 x 128 in bf16, exact products and 32-bit sums: the operands' 32 bytes a lane, eight at a time.
__device__ __forceinline__ v4f mma_wide(v8i b, v8i a, v4f c) {
#pragma unroll
    for (int h = 0; h < 4; ++h)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8((unsigned)b[2 * h], (unsigned)b[2 * h + 1]), widen8((unsigned)a[2 * h], (unsigned)a[2 * h + 1]), c, 0, 0, 0);
    return c;
}

// 16 x 16 x 128: `b` gives the rows of the result, `a` its columns, so that a lane holds four neighbours of one row of `out`.
template <int KIND> __device__ __forceinline__ v4f mma(v8i b, v8i a, v4f c, unsigned sb, unsigned sa) {
    if (KIND == TUNA_SCALE_E8) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, 0, (int)sb, 0, (int)sa);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, 0, 127, 0, 127);
}

// Which matrix cores: the 8-bit ones add eight neighbouring products at a time, each cut at 2^-13 of the largest one's power of two: at most 2^-10 of
// the sum of the magnitudes (measured: 1.5e-5 of a result of normally distributed values).  A result that is rounded to bf16 (2^-9) does not show
// that unless large products cancel in it, and is rounded to the other neighbour in some two places of a thousand; one that stays in 32 bits would show it always, so its
// operands are widened to bf16, whose cores keep products and sums in 32 bits, at half the rate.
//
// The simple form: a tile of 64 x 64, four waves of 16 rows each, one block of 128 at a time through the LDS; any alignment.
// COLS: the reduction is over the groups' rows (gradient of the weights), every row of both sides has scales of its own.
template <int KIND, bool COLS, bool WIDE, class OUT>
__global__ __launch_bounds__(256) void k_product64(Product P) {
    __shared__ __align__(16) uint8_t la[64][kBlock + 16], lb[64][kBlock + 16];
    __shared__ unsigned sa[64], sb[64];
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
    const int64_t bs0 = COLS ? 0 : group * P.bs_group;
    v4f acc[4] = {};
    for (int64_t kb = kb0; kb < kb1; ++kb) {
        __syncthreads();
        for (int c = tid; c < 1024; c += 256) {
            const int r = (c >> 3) & 63, ch = c & 7;
            const int64_t at = kb * kBlock + ch * 16;
            if (c < 512) {
                const int64_t row = i0 + r < i_end ? i0 + r : i_end - 1;
                *(v4u*)&la[r][ch * 16] = chunk16<WIDE>(P.a + row * P.lda + at, length - at);
            } else {
                const int64_t row = j0 + r < P.n ? j0 + r : P.n - 1;
                *(v4u*)&lb[r][ch * 16] = chunk16<WIDE>(b + row * P.ldb + at, length - at);
            }
        }
        if (tid < 64) {
            const int64_t row = i0 + tid < i_end ? i0 + tid : i_end - 1;
            sa[tid] = scale_at<KIND>(P.as, row * P.ld_as + kb);
        } else if (tid < 128) {
            const int64_t row = j0 + tid - 64 < P.n ? j0 + tid - 64 : P.n - 1;
            sb[tid - 64] = scale_at<KIND>(P.bs, bs0 + (COLS ? row : row / kBlock) * P.ld_bs + kb);
        }
        __syncthreads();
        const int r = lane & 15, part = (lane >> 4) * 32;
        v8i fa;
        __builtin_memcpy(&fa, &la[w * 16 + r][part], 32);
        const unsigned ka = sa[w * 16 + r];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v8i fb;
            __builtin_memcpy(&fb, &lb[s * 16 + r][part], 32);
            if (KIND == TUNA_SCALE_E8 && sizeof(OUT) == 2) {
                acc[s] = mma<KIND>(fb, fa, acc[s], sb[s * 16 + r], ka);
            } else {
                const v4f zero = {0.f, 0.f, 0.f, 0.f};
                const v4f p = sizeof(OUT) == 2 ? mma<KIND>(fb, fa, zero, 0, 0) : mma_wide(fb, fa, zero);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[s][i] += p[i] * (scale_float<KIND>(ka) * scale_float<KIND>(sb[s * 16 + (lane >> 4) * 4 + i]));
            }
        }
    }
    const int64_t row = i0 + w * 16 + (lane & 15);
    if (row >= i_end) return;
    OUT* out = (OUT*)P.out + (COLS ? group * P.out_group : 0) + row * P.ldo;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t j = j0 + s * 16 + (lane >> 4) * 4 + i;
            if (j < P.n) store1(out + j, acc[s][i]);
        }
}

// The large form: a tile of BM x BN, WM x WN waves, blocks of 128 in turn through two halves of the LDS: while one is multiplied the next
// one is on its way.  A row's sixteens lie in the LDS at their place xor (row / 2 mod 8), and a lane reads numbers part and part + 4: the
// sixteen lanes that the LDS serves together then meet every bank once; the lanes load them in that order.
// No conflicts are counted.  256 x 256, 16384 x 8192 x 8192: 919 to 959 us by machine, 2.3 to 2.4 PFLOP/s, the matrix cores at work 51 % of the
// time: between two blocks all waves wait for the barrier and then for the same LDS.  64 groups of 256 rows, 3584 x 4096: 378 to 396 us, of which
// the weights alone take 235 to read.  128 x 128 by columns, 8 groups of 12005 x 2736 x 2048: to 32 bits 200 us (193), 0.7 PFLOP/s,
// bound by the widening and scaling (278 us with scales as powers of two, which are made into 32-bit values here one by one); to bf16 133 us, 101 with powers
// of two.  Four waves of 128 x 128 in place of eight of 128 x 64 took 995 us for the first.
template <int KIND, bool COLS, class OUT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_product(Product P, int m_tiles, int n_tiles) {
    constexpr int W = WM * WN, MT = BM / (16 * WM), NT = BN / (16 * WN), LA = BM / 8 / W, LB = BN / 8 / W;
    constexpr bool CORE8 = sizeof(OUT) == 2;
    static_assert(LA * 8 * W == BM && LB * 8 * W == BN && (BM + BN) / 64 <= W, "");
    __shared__ __align__(1024) uint8_t tile[2][(BM + BN) * kBlock];
    __shared__ __align__(16) unsigned scale[2][BM + BN];
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
    int64_t i0, i_end, kb0 = 0, kb1;
    const int64_t j0 = (int64_t)tj * BN;
    if (COLS) {
        i0 = (int64_t)ti * BM;
        i_end = i0 + BM < P.m ? i0 + BM : P.m;
        int64_t count;
        group_blocks(P.group_rows, P.groups, group, P.k, kb0, count);
        kb1 = kb0 + count;
    } else {
        const Place pl = find_tile(P.group_rows, P.groups, P.m, BM, ti);
        if (pl.group < 0) return;
        group = pl.group; i0 = pl.first; i_end = pl.end;
        kb1 = blocks_of(P.k);
    }
    i0 = (int64_t)__builtin_amdgcn_readfirstlane((int)i0);
    i_end = (int64_t)__builtin_amdgcn_readfirstlane((int)i_end);
    group = __builtin_amdgcn_readfirstlane(group);
    kb0 = __builtin_amdgcn_readfirstlane((int)kb0);
    kb1 = __builtin_amdgcn_readfirstlane((int)kb1);
    const uint8_t* a = P.a + i0 * P.lda;
    const uint8_t* b = P.b + (COLS ? 0 : group * P.b_group) + j0 * P.ldb;
    const int rows_a = (int)(i_end - i0), rows_b = (int)(P.n - j0 < BN ? P.n - j0 : BN);
    const int sixteen = ((lane & 7) ^ (lane >> 4)) * 16;          // of the rows of even loads; of odd ones it is 64 further or nearer
    static_assert(LA % 2 == 0 && LB % 2 == 0, "");
    unsigned at_a[LA], at_b[LB];
#pragma unroll
    for (int j = 0; j < LA; ++j) {
        const int r = (w * LA + j) * 8 + (lane >> 3);
        at_a[j] = (unsigned)((r < rows_a ? r : rows_a - 1) * P.lda) + (sixteen ^ (j & 1) * 64);
    }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
        const int r = (w * LB + j) * 8 + (lane >> 3);
        at_b[j] = (unsigned)((r < rows_b ? r : rows_b - 1) * P.ldb) + (sixteen ^ (j & 1) * 64);
    }
    const uint8_t* at_s = nullptr;                                // this lane's row of scales
    constexpr int SS = KIND == TUNA_SCALE_E8 ? 1 : 4;
    if (w < BM / 64) {
        const int r = w * 64 + lane;
        at_s = (const uint8_t*)P.as + (i0 + (r < rows_a ? r : rows_a - 1)) * P.ld_as * SS;
    } else if (w < (BM + BN) / 64) {
        const int r = w * 64 + lane - BM;
        const int64_t row = j0 + (r < rows_b ? r : rows_b - 1);
        at_s = (const uint8_t*)P.bs + ((COLS ? 0 : group * P.bs_group) + (COLS ? row : row / kBlock) * P.ld_bs) * SS;
    }
    auto issue = [&](int64_t kb, int half) {
        const int left = (int)(P.k - kb * kBlock < kBlock ? P.k - kb * kBlock : kBlock);
        const uint8_t *ga = a + kb * kBlock, *gb = b + kb * kBlock;
        uint8_t *la = tile[half] + w * LA * 1024, *lb = tile[half] + BM * kBlock + w * LB * 1024;
        if (COLS || left == kBlock) {
#pragma unroll
            for (int j = 0; j < LA; ++j) to_lds<16>(ga + at_a[j], la + j * 1024);
#pragma unroll
            for (int j = 0; j < LB; ++j) to_lds<16>(gb + at_b[j], lb + j * 1024);
        } else {                                                  // the row ends inside the block: zeros behind it
            const v4u zero = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < LA; ++j) {
                if ((sixteen ^ (j & 1) * 64) < left) to_lds<16>(ga + at_a[j], la + j * 1024);
                else *(v4u*)(la + j * 1024 + lane * 16) = zero;
            }
#pragma unroll
            for (int j = 0; j < LB; ++j) {
                if ((sixteen ^ (j & 1) * 64) < left) to_lds<16>(gb + at_b[j], lb + j * 1024);
                else *(v4u*)(lb + j * 1024 + lane * 16) = zero;
            }
        }
        if (w < (BM + BN) / 64) to_lds<SS>(at_s + kb * SS, &scale[half][w * 64]);
    };
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    if (kb0 < kb1) issue(kb0, 0);
    const int r = lane & 15, c0 = ((lane >> 4) ^ (r >> 1)) * 16, c1 = c0 ^ 64;
    int half = 0;
    for (int64_t kb = kb0; kb < kb1; ++kb, half ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const uint8_t *ta = tile[half] + (wm * MT * 16 + r) * kBlock, *tb = tile[half] + (BM + wn * NT * 16 + r) * kBlock;
        const unsigned *sa = scale[half] + wm * MT * 16, *sb = scale[half] + BM + wn * NT * 16;
        auto fragment = [&](const uint8_t* t) {
            const v4u x = *(const v4u*)(t + c0), y = *(const v4u*)(t + c1);
            return v8i{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
        };
        // the next 16 rows of a are read while these are multiplied
        v8i fb[NT], fa[2];
        unsigned ka[2], kbs[NT];
        v4f kbv[NT];
        float one = 1.f;
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = fragment(tb + j * 16 * kBlock);
        fa[0] = fragment(ta);
        ka[0] = sa[r];
        if (CORE8 && KIND == TUNA_SCALE_E8) {
#pragma unroll
            for (int j = 0; j < NT; ++j) kbs[j] = sb[j * 16 + r];
        } else if (COLS) {                                        // by columns every row of b has a scale of its own, else these rows share one
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) kbv[j][q] = scale_float<KIND>(sb[j * 16 + (lane >> 4) * 4 + q]);
        } else {
            one = scale_float<KIND>(sb[0]);
        }
        if (kb + 1 < kb1) issue(kb + 1, half ^ 1);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (i + 1 < MT) {
                fa[(i + 1) & 1] = fragment(ta + (i + 1) * 16 * kBlock);
                ka[(i + 1) & 1] = sa[(i + 1) * 16 + r];
            }
            if (CORE8 && KIND == TUNA_SCALE_E8) {
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mma<KIND>(fb[j], fa[i & 1], acc[i][j], kbs[j], ka[i & 1]);
            } else {
                const float k = scale_float<KIND>(ka[i & 1]) * one;
                const v4f zero = {0.f, 0.f, 0.f, 0.f};
                v4f p[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) p[j] = CORE8 ? mma<TUNA_SCALE_F32>(fb[j], fa[i & 1], zero, 0, 0) : mma_wide(fb[j], fa[i & 1], zero);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j][q] += COLS ? p[j][q] * kbv[j][q] * k : p[j][q] * k;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    OUT* out = (OUT*)P.out + (COLS ? group * P.out_group : 0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t row = i0 + (wm * MT + i) * 16 + r;
        if (row >= i_end) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t col = j0 + (wn * NT + j) * 16 + (lane >> 4) * 4;
            if (col >= P.n) continue;
            store_four(out + row * P.ldo + col, acc[i][j], (int)(P.n - col < 4 ? P.n - col : 4));
        }
    }
}

// The form for few rows, which reads the weights once and little else: a workgroup has 16 rows of b and 16 MT rows of a, its waves share the
// blocks of the length, operands go from memory to registers, and the waves' sums are added up in their order.  40 x 4096 x 2048: 8.4 us (8.1), of which
// the 8 MB of weights need 2: bound by the way of one load after the start of a kernel, and the launch.
constexpr int kThinWaves = 8;

template <int KIND, class OUT, int MT>
__global__ __launch_bounds__(kThinWaves * 64) void k_product_thin(Product P) {
    constexpr bool CORE8 = sizeof(OUT) == 2;
    __shared__ v4f sums[kThinWaves][MT][64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Place pl = find_tile(P.group_rows, P.groups, P.m, 16 * MT, blockIdx.y);
    if (pl.group < 0) return;
    const int group = __builtin_amdgcn_readfirstlane(pl.group);
    const int64_t i0 = pl.first, i_end = pl.end, j0 = (int64_t)blockIdx.x * 16;
    const int r = lane & 15, part = lane >> 4;
    const int64_t rb = j0 + r < P.n ? j0 + r : P.n - 1;
    const uint8_t* b = P.b + group * P.b_group + rb * P.ldb;
    const int64_t bs = group * P.bs_group + rb / kBlock * P.ld_bs;
    const uint8_t* a[MT];
    int64_t as[MT];
#pragma unroll
    for (int s = 0; s < MT; ++s) {
        const int64_t ra = i0 + s * 16 + r < i_end ? i0 + s * 16 + r : i_end - 1;
        a[s] = P.a + ra * P.lda;
        as[s] = ra * P.ld_as;
    }
    v4f acc[MT];
#pragma unroll
    for (int s = 0; s < MT; ++s) acc[s] = v4f{0.f, 0.f, 0.f, 0.f};
    struct Ahead { v8i b, a[MT]; unsigned sb, sa[MT]; };
    // a lane's 32 bytes of a block: sixteen in each half, so that a load takes 64 bytes of a row in a piece
    auto both = [&](const v4u& x, const v4u& y) { return v8i{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]}; };
    auto fetch = [&](Ahead& t, int64_t kb, auto full) {
        const int64_t at = kb * kBlock + part * 16, left = P.k - at;
        auto row = [&](const uint8_t* p) {
            if (full.value) return both(*(const v4u*)(p + at), *(const v4u*)(p + at + 64));
            return both(chunk16<true>(p + at, left), chunk16<true>(p + at + 64, left - 64));
        };
        t.b = row(b);
        t.sb = scale_at<KIND>(P.bs, bs + kb);
#pragma unroll
        for (int s = 0; s < MT; ++s) {
            t.a[s] = row(a[s]);
            t.sa[s] = scale_at<KIND>(P.as, as[s] + kb);
        }
    };
    auto use = [&](const Ahead& t) {
#pragma unroll
        for (int s = 0; s < MT; ++s) {
            if (CORE8 && KIND == TUNA_SCALE_E8) {
                acc[s] = mma<KIND>(t.b, t.a[s], acc[s], t.sb, t.sa[s]);
            } else {
                // the 16 rows of b lie in one block of 128 and share their scale
                const v4f zero = {0.f, 0.f, 0.f, 0.f};
                acc[s] += (CORE8 ? mma<TUNA_SCALE_F32>(t.b, t.a[s], zero, 0, 0) : mma_wide(t.b, t.a[s], zero)) *
                          (scale_float<KIND>(t.sa[s]) * scale_float<KIND>(t.sb));
            }
        }
    };
    const int whole = (int)(P.k / kBlock), units = (whole - w + kThinWaves - 1) / kThinWaves;
    Ahead st[3];
    pipeline<3, false>(st, 0, units, [&](Ahead& t, int u) { fetch(t, u * kThinWaves + w, Int<1>{}); }, [&](const Ahead& t, int) { use(t); });
    if (whole * (int64_t)kBlock < P.k && whole % kThinWaves == w) {
        fetch(st[0], whole, Int<0>{});
        use(st[0]);
    }
#pragma unroll
    for (int s = 0; s < MT; ++s) sums[w][s][lane] = acc[s];
    __syncthreads();
    if (w >= MT) return;
    v4f v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < kThinWaves; ++q) v += sums[q][w][lane];
    const int64_t row = i0 + w * 16 + r, col = j0 + part * 4;
    if (row < i_end && col < P.n) store_four((OUT*)P.out + row * P.ldo + col, v, (int)(P.n - col < 4 ? P.n - col : 4));
}

// ------------------------------------------------------------------------------------------------ the sum over a token's experts

// Bound by memory: 16384 tokens, k = 8, 4096 columns of bf16 260 us, 4.6 TB/s.
template <class Y, class O, bool WIDE>
__global__ __launch_bounds__(256) void k_combine(const Y* y, int64_t ldy, int64_t y_rows, const int32_t* slots, const float* weights, int64_t n_tokens, int k,
                                                 int64_t cols, O* out, int64_t ld_out) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, left = cols - c, t = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (left <= 0 || t >= n_tokens) return;
    float s[8] = {};
    for (int j = 0; j < k; ++j) {
        const int64_t r = slots[t * k + j];
        if (r < 0 || r >= y_rows) continue;
        const float w = weights[t * k + j];
        float v[8];
        load8<WIDE>(y + r * ldy + c, left, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += w * v[i];
    }
    store8<WIDE>(out + t * ld_out + c, left, s);
}

// One workgroup per token: a row of dout is read once, k rows of y and dy beside it.  The same sizes: 443 us (438), 5.2 TB/s.
template <class O, class Y, bool WIDE>
__global__ __launch_bounds__(256) void k_combine_grad(const O* dout, int64_t ld_dout, const Y* y, int64_t ldy, int64_t y_rows, const int32_t* slots,
                                                      const float* weights, int k, int64_t cols, Y* dy, int64_t ld_dy, float* dweights) {
    __shared__ float part[4][TUNA_MOE_MAX_K];
    const int64_t t = blockIdx.x;
    float dot[TUNA_MOE_MAX_K];
#pragma unroll
    for (int j = 0; j < TUNA_MOE_MAX_K; ++j) dot[j] = 0.f;
    for (int64_t c = threadIdx.x * 8; c < cols; c += 256 * 8) {
        float d[8];
        load8<WIDE>(dout + t * ld_dout + c, cols - c, d);
#pragma unroll
        for (int j = 0; j < TUNA_MOE_MAX_K; ++j) {
            if (j >= k) break;
            const int64_t r = slots[t * k + j];
            if (r < 0 || r >= y_rows) continue;
            const float w = weights[t * k + j];
            float v[8];
            load8<WIDE>(y + r * ldy + c, cols - c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) { dot[j] += d[i] * v[i]; v[i] = w * d[i]; }
            store8<WIDE>(dy + r * ld_dy + c, cols - c, v);
        }
    }
#pragma unroll
    for (int j = 0; j < TUNA_MOE_MAX_K; ++j) {
        if (j >= k) break;
        const float s = wave_sum(dot[j]);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][j] = s;
    }
    __syncthreads();
    if (threadIdx.x < k) dweights[t * k + threadIdx.x] = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
}

// ------------------------------------------------------------------------------------------------ the layer for a few tokens

struct Few {
    const unsigned short* x; int64_t ldx; int tokens; int64_t hidden;
    const void* logits; int64_t ld_logits; int experts, k, renorm;
    const void* w1; const void* s1; const void* w2; const void* s2; int64_t inner;
    void* out; int64_t ld_out;
    // workspace: the chosen experts and their shares of the softmax, [tokens * k]; the activations as two bf16 parts, [tokens * k, ld_h]
    int32_t* chosen; float* share; unsigned short* hi; unsigned short* lo; int64_t ld_h;
};

// The parts of 128 neighbours of a row that one of four lanes holds, as they lie in memory, and eight of them at a time as bf16, which holds
// every e4m3 exactly.  at(h, part): where the eight number h of lane `part` start.  Every load takes 64 bytes of a row in a piece.  whole(): all of it
// is inside the row, so that the loads hang on no condition; the address is a wave's base and a lane's 32-bit offset in bytes.
// row(n): the elements of a row of n values; kUnit: those of a block of 128.  A lane's scales of row r of `rows` of expert e: scales(...) says where the
// first is, the next block's is kScales behind.  kAhead1, kAhead2: blocks that a wave
// of the first kernel has in registers or on their way, weights and tokens, and of the second, weights and activations.  4-bit values take theirs where they are widened (INSIDE: bf16 holds the products), others in 32 bits.
struct Four { uint8_t two; };           // two 4-bit values
template <class W> struct Part;
template <class W> struct PartBase {
    static constexpr int kUnit = kBlock, kScales = 1, kAhead1 = 3, kAhead2 = 4;
    static constexpr bool INSIDE = false;
    static __device__ __forceinline__ int64_t row(int64_t n) { return n; }
    static __device__ __forceinline__ int64_t scales(int64_t e, int64_t rows, int64_t r, int64_t cols, int) { return (e * blocks_of(rows) + r / kBlock) * blocks_of(cols); }
    static __device__ __forceinline__ int64_t last(int64_t at, int64_t, int, int64_t) { return at; }
};
template <> struct Part<Four> {
    static constexpr int kUnit = kBlock / 2, kScales = kBlock / kBlock4, kAhead1 = 2, kAhead2 = 4;
    static constexpr bool INSIDE = true;
    v4u v;
    static __device__ __forceinline__ int at(int h, int part) { return part * 32 + h * 8; }
    static __device__ __forceinline__ int64_t row(int64_t n) { return (n + 1) / 2; }
    static __device__ __forceinline__ int64_t scales(int64_t e, int64_t rows, int64_t r, int64_t cols, int part) { return (e * rows + r) * ((cols + kBlock4 - 1) / kBlock4) + part; }
    // in the last block of a row: the row's last scale for the parts behind its end, whose values are zeros
    static __device__ __forceinline__ int64_t last(int64_t at, int64_t b, int part, int64_t cols) {
        const int64_t over = b * kScales + part - ((cols + kBlock4 - 1) / kBlock4 - 1);
        return over > 0 ? at - over : at;
    }
    template <bool WIDE> __device__ __forceinline__ void load(const Four* p, int part, int64_t left) { v = chunk32<WIDE>((const uint8_t*)p + part * 16, left - part * 32); }
    __device__ __forceinline__ v8b eight(int h, float k) const {
        const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[h], k, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[h], k, 1);
        const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[h], k, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[h], k, 3);
        return v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
};
template <> struct Part<uint8_t> : PartBase<uint8_t> {
    v4u v[2];
    static __device__ __forceinline__ int at(int h, int part) { return (h >> 1) * 64 + part * 16 + (h & 1) * 8; }
    __device__ __forceinline__ void whole(const uint8_t* base, unsigned off) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = *(const v4u*)(base + i * 64 + (size_t)off);
    }
    template <bool WIDE> __device__ __forceinline__ void load(const uint8_t* p, int part, int64_t left) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = chunk16<WIDE>(p + i * 64 + part * 16, left - (i * 64 + part * 16));
    }
    __device__ __forceinline__ v8b eight(int h, float) const { return widen8(v[h >> 1][(h & 1) * 2], v[h >> 1][(h & 1) * 2 + 1]); }
};
template <> struct Part<unsigned short> : PartBase<unsigned short> {
    v4u v[4];
    static __device__ __forceinline__ int at(int h, int part) { return h * 32 + part * 8; }
    __device__ __forceinline__ void whole(const unsigned short* base, unsigned off) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *(const v4u*)((const uint8_t*)base + i * 64 + (size_t)off);
    }
    template <bool WIDE> __device__ __forceinline__ void load(const unsigned short* p, int part, int64_t left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = bits8<WIDE>(p + at(i, part), left - at(i, part));
    }
    __device__ __forceinline__ v8b eight(int h, float) const {
        v8b r;
        __builtin_memcpy(&r, &v[h], 16);
        return r;
    }
};
__device__ __forceinline__ v8b as_bf16(const v4u& a) {
    v8b r;
    __builtin_memcpy(&r, &a, 16);
    return r;
}

// Lane (c, part) of sixteen c holds step c / (16 / P) of the place c mod (16 / P): the places' four steps, each in the lanes of its place.  What the lanes behind
// them then hold makes rows of a product that nobody reads.
template <int SHIFT> __device__ __forceinline__ v8b lanes_down(const v8b& a) {
    v4u v;
    __builtin_memcpy(&v, &a, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v[i], 0x100 + SHIFT, 0xf, 0xf, true);
    return as_bf16(v);
}
template <int P> __device__ __forceinline__ void later_steps(const v8b (&from)[4 / P], v8b (&to)[4]) {
    if constexpr (P == 4) { to[0] = from[0]; to[1] = lanes_down<4>(from[0]); to[2] = lanes_down<8>(from[0]); to[3] = lanes_down<12>(from[0]); }
    else if constexpr (P == 2) { to[0] = from[0]; to[1] = lanes_down<8>(from[0]); to[2] = from[1]; to[3] = lanes_down<8>(from[1]); }
    else { to[0] = from[0]; to[1] = from[1]; to[2] = from[2]; to[3] = from[3]; }
}

template <int KIND> __device__ __forceinline__ float scale_value(const void* s, int64_t i) {
    if (KIND < 0) return 1.f;
    return scale_float<KIND>(scale_at<KIND>(s, i));
}

constexpr int kFewFirst = 4;           // waves of a workgroup of the first kernel: they share the length of the sums
constexpr int kFewSecond = 8;         // and of the second: they share the experts

// First kernel: a workgroup makes 16 activations, or 64, of one expert (as many rows of the gate half and of the up half) for all tokens that
// chose it, 16 MT of them at a time.  Bound by reading the weights: 40 tokens, k = 8 of 128 experts, 1536 x 4096: 1.49 GB in 367 us (357), 4.1 TB/s; one
// token, k = 4, 1024 x 2048: 17 MB in 10 us, the way from logits to weights to sums and the launch.  ONE: there is one token, and blockIdx.y counts its chosen experts; else blockIdx.y is the expert, and its tokens
// are found without a sort: it is among the k first of a token when fewer than k eligible logits come before its own.  Three waves a SIMD leave 168
// registers, which suit 8-bit weights with one token or 16 columns a wave; shared columns of several tokens keep 33 to 43 registers in scratch, bf16
// weights 14 to 111.
template <class L, class W, int KIND, bool WIDE, int MT, bool SPLIT, bool ONE>
__global__ __launch_bounds__(256, MT == 1 ? 3 : 2) void k_few_first(Few F) {
    __shared__ int rank_of[TUNA_MOE_FEW_TOKENS];                  // how many come before this expert, or -1: not chosen
    __shared__ int list[TUNA_MOE_FEW_TOKENS];
    __shared__ float sums[SPLIT ? kFewFirst : 1][2][256];
    __shared__ __align__(1024) uint8_t ring[kFewFirst][WIDE && Part<W>::INSIDE ? Part<W>::kAhead1 : 1][2][2048];
    const int tid = threadIdx.x, lane = tid & 63;
    const bool first = blockIdx.x == 0;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int e = blockIdx.y, n;
    auto share_in = [&](const L* row, float own) {                // of the softmax over all eligible experts
        float top = -__builtin_inff(), sum = 0.f;
        for (int i = lane; i < F.experts; i += 64) { const float l = load1(row + i); if (logit_key(l)) top = fmaxf(top, l); }
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        for (int i = lane; i < F.experts; i += 64) sum += exp_share(load1(row + i), top);
        return exp_share(own, top) / wave_sum(sum);
    };
    if (ONE) {
        const L* row = (const L*)F.logits;
        constexpr int PER = TUNA_MOE_MAX_EXPERTS / 64;
        unsigned key[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = i * 64 + lane < F.experts ? logit_key(load1(row + i * 64 + lane)) : 0u;
        e = -1;
        for (int j = 0; j <= (int)blockIdx.y; ++j) {
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) m = key[i] > m ? key[i] : m;
#pragma unroll
            for (int d = 32; d; d >>= 1) { const unsigned o = __shfl_xor(m, d); m = o > m ? o : m; }
            e = -1;
            if (m == 0) break;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const unsigned long long b = __ballot(e < 0 && key[i] == m);
                if (b) {
                    const int l = __ffsll((long long)b) - 1;
                    e = i * 64 + l;
                    if (lane == l) key[i] = 0;
                }
            }
        }
        e = __builtin_amdgcn_readfirstlane(e);
        n = e < 0 ? 0 : 1;
        if (first && w == 0) {
            const float s = n ? share_in(row, load1(row + e)) : 0.f;
            if (lane == 0) { F.chosen[blockIdx.y] = e; F.share[blockIdx.y] = s; }
        }
        if (n == 0) return;
        if (tid == 0) { list[0] = 0; rank_of[0] = blockIdx.y; }
    } else {
        constexpr int TOGETHER = 4;                               // tokens whose logits are under way together
        for (int t0 = w * TOGETHER; t0 < F.tokens; t0 += kFewFirst * TOGETHER) {
            float own[TOGETHER];
            int before[TOGETHER] = {}, eligible[TOGETHER] = {};
            const L* row[TOGETHER];
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) {
                const int t = t0 + q < F.tokens ? t0 + q : F.tokens - 1;
                row[q] = (const L*)F.logits + t * F.ld_logits;
                own[q] = load1(row[q] + e);
            }
            for (int i0 = 0; i0 < F.experts; i0 += 64) {
                const int i = i0 + lane, at = i < F.experts ? i : F.experts - 1;
                float l[TOGETHER];
#pragma unroll
                for (int q = 0; q < TOGETHER; ++q) l[q] = load1(row[q] + at);
#pragma unroll
                for (int q = 0; q < TOGETHER; ++q) {
                    const unsigned key = logit_key(own[q]), o = i < F.experts ? logit_key(l[q]) : 0u;
                    before[q] += __popcll(__ballot(o > key || (o == key && i < e)));
                    eligible[q] += __popcll(__ballot(o != 0));
                }
            }
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) {
                const int t = t0 + q;
                if (t >= F.tokens) break;
                const bool in = logit_key(own[q]) != 0 && before[q] < F.k;
                if (lane == 0) rank_of[t] = in ? before[q] : -1;
                // a token with fewer than k eligible experts: its last places are empty
                if (first && e == 0 && lane < F.k && lane >= eligible[q]) F.chosen[t * F.k + lane] = -1;
            }
        }
        __syncthreads();
        if (first) {
#pragma unroll 1
            for (int t = w; t < F.tokens; t += kFewFirst)
                if (rank_of[t] >= 0) {
                    const L* row = (const L*)F.logits + t * F.ld_logits;
                    const float s = share_in(row, load1(row + e));
                    if (lane == 0) {
                        F.chosen[t * F.k + rank_of[t]] = e;
                        F.share[t * F.k + rank_of[t]] = s;
                    }
                }
        }
        const bool in = lane < F.tokens && rank_of[lane] >= 0;
        const unsigned long long b = __ballot(in);
        n = __popcll(b);
        if (w == 0 && in) list[__popcll(b & ((1ull << lane) - 1))] = lane;
        if (n == 0) return;
    }
    __syncthreads();
    // SPLIT: the waves share the length of one 16 columns' sums; else each wave has 16 columns of its own
    const int64_t f0 = SPLIT ? (int64_t)blockIdx.x * 16 : ((int64_t)blockIdx.x * kFewFirst + w) * 16;
    const int c = lane & 15, part = lane >> 4;
    const int64_t col = f0 + c < F.inner ? f0 + c : F.inner - 1;
    using Wp = Part<W>;
    const int64_t row_w = Wp::row(F.hidden), at_w = col * row_w, nb = blocks_of(F.hidden);
    const W* wg = (const W*)F.w1 + (int64_t)e * 2 * F.inner * row_w;
    const W* wu = wg + F.inner * row_w;
    const int64_t sg = Wp::scales(e, 2 * F.inner, col, F.hidden, part), su = Wp::scales(e, 2 * F.inner, F.inner + col, F.hidden, part);
    const unsigned off_w = (unsigned)(at_w * sizeof(W)) + part * 16;
    // whole blocks in a pipeline; what is behind them (all, for rows that do not start on 16 bytes) one block at a time
    const int pairs = WIDE ? (int)(F.hidden / (2 * kBlock)) : 0, whole = WIDE && Wp::INSIDE ? 2 * pairs : WIDE ? (int)(F.hidden / kBlock) : 0;
    for (int t0 = 0; t0 < n; t0 += MT * 16) {                     // more than 16 MT tokens of one expert read its weights again
        v4f gate[MT], up[MT];
        unsigned at_x[MT];
#pragma unroll
        for (int s = 0; s < MT; ++s) {
            gate[s] = up[s] = v4f{0.f, 0.f, 0.f, 0.f};
            const int i = t0 + s * 16 + c;
            at_x[s] = i < n ? (unsigned)(list[i] * F.ldx) : ~0u;
        }
        // the tokens' parts of one block
        auto load_x = [&](v8b (&a)[MT][4], int64_t at, auto full) {
#pragma unroll
            for (int s = 0; s < MT; ++s) {
#pragma unroll
                for (int h = 0; h < 4; ++h) a[s][h] = v8b{};
                if (at_x[s] != ~0u) {                             // places without a token are zeros, and cost no loads
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int k = Part<W>::at(h, 0);
                        const unsigned lane_at = at_x[s] + Part<W>::at(0, part);
                        if (full.value) a[s][h] = as_bf16(*(const v4u*)((const uint8_t*)(F.x + at + k) + (size_t)(lane_at * 2)));
                        else a[s][h] = as_bf16(bits8<WIDE>(F.x + at + k + lane_at, F.hidden - at - k - Part<W>::at(0, part)));
                    }
                }
            }
        };
        auto multiply = [&](const v8b (&a)[MT][4], const Part<W>& pg, const Part<W>& pu, float kg, float ku) {
            v4f g[MT], u[MT];
#pragma unroll
            for (int s = 0; s < MT; ++s) {
                g[s] = Wp::INSIDE ? gate[s] : v4f{0.f, 0.f, 0.f, 0.f};
                u[s] = Wp::INSIDE ? up[s] : v4f{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const v8b bg = pg.eight(h, kg), bu = pu.eight(h, ku);
#pragma unroll
                for (int s = 0; s < MT; ++s) {
                    g[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s][h], bg, g[s], 0, 0, 0);
                    u[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s][h], bu, u[s], 0, 0, 0);
                }
            }
#pragma unroll
            for (int s = 0; s < MT; ++s) {
                if (Wp::INSIDE) { gate[s] = g[s]; up[s] = u[s]; }
                else { gate[s] += g[s] * kg; up[s] += u[s] * ku; }
            }
        };
        constexpr int stride = SPLIT ? kFewFirst : 1, skip = SPLIT;
        if constexpr (WIDE && Wp::INSIDE) {
            // The weights go through the LDS, a wave's own part of it: its lanes load whole pieces of rows, where the product's lanes, sixteen rows side by side,
            // would ask for every sixteen bytes by themselves; two blocks at a time, so that a piece is 128 bytes.  The scales of gate rows and up rows are two words in the lanes 0 to 31.  A wait for the
            // scales, which are asked for behind the weights, is a wait for these.  Up to 4 (8) tokens: the lanes of places without one load the
            // tokens' later steps, P = 4 (2) steps in one load.  48 tokens, k = 8 of 128 experts, 1408 x 4096, first kernel: 316 us without all this,
            // 250 with the weights through the LDS, 194 so (0.78 GB, 4.0 TB/s; a stage more ahead, without a condition on any load, gives the same while the
            // compiler sets the waits: it waits for all loads, those of the next unit too).
            auto stream = [&](auto packed) {
                constexpr int P = packed.value;
                struct Ahead { v2u k; v8b a[MT][2][4 / P]; };
                Ahead st[Wp::kAhead1];
                const int units = (pairs - skip * w + stride - 1) / stride;
                const unsigned slots = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&ring[w][0][0][0];
                unsigned off[2];                                  // eight rows of 128 bytes a load; sixteen number i of a row lies at place i xor (row / 2 mod 8)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t mine = f0 + j * 8 + (lane >> 3) < F.inner ? f0 + j * 8 + (lane >> 3) : F.inner - 1;
                    off[j] = (unsigned)(mine * row_w) + ((lane & 7) ^ (lane >> 4) ^ j * 4) * 16;
                }
                const uint8_t* scale_row = (const uint8_t*)F.s1 + (lane & 16 ? su : sg) - part;      // of this lane's column
                const int place = c * 128 + (part ^ (c >> 1)) * 16;
                unsigned x_at[MT];                                // this lane's token, and its first value of a block
#pragma unroll
                for (int s = 0; s < MT; ++s) {
                    const int i = t0 + s * 16 + c % (16 / P);
                    x_at[s] = i < n ? (unsigned)(list[i] * F.ldx) + part * 32 + c / (16 / P) * 8 : ~0u;
                }
                auto fetch = [&](Ahead& t, int unit) {
                    const int64_t b = 2 * (unit * stride + skip * w);
                    const unsigned to = slots + (unsigned)unit % Wp::kAhead1 * 4096;
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // what is read of this part of the LDS has been read
                    const uint8_t *from_g = scalar((const uint8_t*)(wg + b * Wp::kUnit)), *from_u = scalar((const uint8_t*)(wu + b * Wp::kUnit));
                    dma16(from_g, off[0], to);
                    dma16(from_g, off[1], to + 1024);
                    dma16(from_u, off[0], to + 2048);
                    dma16(from_u, off[1], to + 3 * 1024);
                    t.k = v2u{0u, 0u};
                    if (lane < 32) __builtin_memcpy(&t.k, scale_row + b * Wp::kScales, 8);
#pragma unroll
                    for (int s = 0; s < MT; ++s) {
#pragma unroll
                        for (int q = 0; q < 8 / P; ++q) t.a[s][q / (4 / P)][q % (4 / P)] = v8b{};
                        if (x_at[s] != ~0u) {
#pragma unroll
                            for (int q = 0; q < 8 / P; ++q)
                                t.a[s][q / (4 / P)][q % (4 / P)] =
                                    as_bf16(*(const v4u*)((const uint8_t*)(F.x + b * kBlock + q / (4 / P) * kBlock + q % (4 / P) * P * 8) + (size_t)(x_at[s] * 2)));
                        }
                    }
                };
                pipeline<Wp::kAhead1, !SPLIT>(st, 0, units, fetch, [&](const Ahead& t, int unit) {
                    asm volatile("" ::"v"(t.k) : "memory");
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint8_t* from = ring[w][(unsigned)unit % Wp::kAhead1][0] + (place ^ half * 64);
                        Part<W> g, u;
                        g.v = *(const v4u*)from;
                        u.v = *(const v4u*)(from + 2048);
                        const unsigned kg = (unsigned)__shfl((int)t.k[half], c) >> (part * 8) & 255u, ku = (unsigned)__shfl((int)t.k[half], 16 + c) >> (part * 8) & 255u;
                        v8b a[MT][4];
#pragma unroll
                        for (int s = 0; s < MT; ++s) later_steps<P>(t.a[s][half], a[s]);
                        multiply(a, g, u, scale_float<TUNA_SCALE_E8>(kg), scale_float<TUNA_SCALE_E8>(ku));
                    }
                });
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to the LDS when it is used again, or given back
            };
            if (ONE || (MT == 1 && n - t0 <= 4)) stream(Int<4>{});
            else if (MT == 1 && n - t0 <= 8) stream(Int<2>{});
            else stream(Int<1>{});
        } else if constexpr (WIDE) {
            struct Ahead { Part<W> g, u; float kg, ku; v8b a[MT][4]; };
            Ahead st[Wp::kAhead1];
            const int units = (whole - skip * w + stride - 1) / stride;
            auto fetch = [&](Ahead& t, int unit) {
                const int64_t b = unit * stride + skip * w;
                t.g.whole(wg + b * Wp::kUnit, off_w);
                t.u.whole(wu + b * Wp::kUnit, off_w);
                t.kg = scale_value<KIND>(F.s1, sg + b * Wp::kScales);
                t.ku = scale_value<KIND>(F.s1, su + b * Wp::kScales);
                load_x(t.a, b * kBlock, Int<1>{});
            };
            pipeline<Wp::kAhead1, !SPLIT>(st, 0, units, fetch, [&](const Ahead& t, int) { multiply(t.a, t.g, t.u, t.kg, t.ku); });
        }
        for (int64_t b = whole + skip * w; b < nb; b += stride) {
            Part<W> g, u;
            const int64_t at = b * kBlock;
            g.template load<WIDE>(wg + b * Wp::kUnit + at_w, part, F.hidden - at);
            u.template load<WIDE>(wu + b * Wp::kUnit + at_w, part, F.hidden - at);
            v8b a[MT][4];
            load_x(a, at, Int<0>{});
            multiply(a, g, u, scale_value<KIND>(F.s1, Wp::last(sg + b * Wp::kScales, b, part, F.hidden)),
                     scale_value<KIND>(F.s1, Wp::last(su + b * Wp::kScales, b, part, F.hidden)));
        }
        auto keep = [&](int i, int64_t f, float x, float y) {     // activation f of token number i of the list
            if (i >= n || f >= F.inner) return;
            const int t = list[i];
            const float v = gate_of(x).silu * y;
            const bool finite = fabsf(v) < __builtin_inff();
            unsigned short hi = to_bf16(v);
            if (finite && (hi & 0x7fff) == 0x7f80) --hi;          // above bf16's largest value: that one, and the rest in the second part
            const int64_t to = (int64_t)(t * F.k + rank_of[t]) * F.ld_h + f;
            F.hi[to] = hi;
            F.lo[to] = finite ? to_bf16(v - bf16_bits(hi)) : (unsigned short)0;
        };
#pragma unroll
        for (int s = 0; s < MT; ++s) {
            if (t0 + s * 16 >= n) break;
            if (SPLIT) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sums[w][0][(part * 4 + i) * 16 + c] = gate[s][i];
                    sums[w][1][(part * 4 + i) * 16 + c] = up[s][i];
                }
                __syncthreads();
                float x = 0.f, y = 0.f;
                for (int q = 0; q < kFewFirst; ++q) { x += sums[q][0][tid]; y += sums[q][1][tid]; }
                keep(t0 + s * 16 + (tid >> 4), f0 + (tid & 15), x, y);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) keep(t0 + s * 16 + part * 4 + i, f0 + c, gate[s][i], up[s][i]);
            }
        }
    }
}

// Second kernel: a workgroup per 16 columns of the result, for all tokens and chosen experts.  A task is a chosen expert with up to 16 of its
// pairs (more of them read its weights again), with up to four where 4-bit weights go through the LDS; 0.74 GB in 210 us, 3.5 TB/s, and 8.4 MB in 7 us for the sizes above; 4-bit weights, 48 tokens, 1408 x 4096:
// 0.39 GB in 146 us (2.7 TB/s: once in four units all loads are waited for).  The tasks' steps are one sequence, of which every wave has a run; a wave's sums are its own,
// and at the end they are added up in the waves' order.
template <class W, int KIND, bool WIDE, class OUT, bool ONE>
__global__ __launch_bounds__(kFewSecond * 64) void k_few_second(Few F) {
    extern __shared__ float shared[];                             // [kFewSecond][tokens][16] sums
    constexpr bool RING = WIDE && Part<W>::INSIDE;
    constexpr int TASK = RING ? 4 : 16;                           // pairs of a task
    __shared__ __align__(1024) uint8_t ring[kFewSecond][RING ? Part<W>::kAhead2 : 1][RING ? 2048 : 16];
    constexpr int PAIRS = TUNA_MOE_FEW_TOKENS * TUNA_MOE_MAX_K;
    __shared__ int pair_of[PAIRS];                                // pairs by expert
    __shared__ float weight[PAIRS];
    __shared__ int first_of[TUNA_MOE_MAX_EXPERTS];
    __shared__ unsigned long long tokens_of[TUNA_MOE_MAX_EXPERTS];        // a bit per token: the order of the atomics does not matter
    __shared__ int task_expert[PAIRS], task_first[PAIRS], task_count[PAIRS];
    __shared__ int n_tasks;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int np = F.tokens * F.k;
    float* sums = shared + w * F.tokens * 16;
    for (int i = lane; i < F.tokens * 16; i += 64) sums[i] = 0.f;
    if (ONE) {                                                    // a task is a pair, in order; the pairs without an expert are the last
        if (w == 0) {
            const int e = lane < np ? F.chosen[lane] : -1;
            float s = e < 0 ? 0.f : F.share[lane];
            if (F.renorm) s /= wave_sum(s);
            if (lane < np) { pair_of[lane] = lane; weight[lane] = s; task_expert[lane] = e; task_first[lane] = lane; task_count[lane] = 1; }
            const int there = __popcll(__ballot(e >= 0));
            if (lane == 0) n_tasks = there;
        }
        __syncthreads();
    } else {
        for (int i = tid; i < F.experts; i += kFewSecond * 64) tokens_of[i] = 0;
        __syncthreads();
        for (int i = tid; i < np; i += kFewSecond * 64) {
            const int e = F.chosen[i];
            if (e >= 0) atomicOr(&tokens_of[e], 1ull << (i / F.k));
            float s = e < 0 ? 0.f : F.share[i];
            if (F.renorm && e >= 0) {
                const int t0 = i / F.k * F.k;
                float total = 0.f;
                for (int j = t0; j < t0 + F.k; ++j) if (F.chosen[j] >= 0) total += F.share[j];
                s /= total;
            }
            weight[i] = s;
        }
        __syncthreads();
        if (w == 0) {                                                 // the tasks in order of their experts
            int tasks = 0, pairs = 0;
            for (int e0 = 0; e0 < F.experts; e0 += 64) {
                const int cnt = e0 + lane < F.experts ? __popcll(tokens_of[e0 + lane]) : 0;
                const int inc = wave_scan(cnt, lane), parts = (cnt + TASK - 1) / TASK, inc_parts = wave_scan(parts, lane);
                if (cnt > 0) {
                    first_of[e0 + lane] = pairs + inc - cnt;
                    for (int i = 0; i < parts; ++i) {
                        const int at = tasks + inc_parts - parts + i;
                        task_expert[at] = e0 + lane;
                        task_first[at] = pairs + inc - cnt + i * TASK;
                        task_count[at] = cnt - i * TASK < TASK ? cnt - i * TASK : TASK;
                    }
                }
                tasks += __shfl(inc_parts, 63);
                pairs += __shfl(inc, 63);
            }
            if (lane == 0) n_tasks = tasks;
        }
        __syncthreads();
        // an expert's pairs in order of their tokens: where a task begins and a wave's run of steps ends may change a sum's last place
        for (int i = tid; i < np; i += kFewSecond * 64) {
            const int e = F.chosen[i];
            if (e >= 0) pair_of[first_of[e] + __popcll(tokens_of[e] & ((1ull << (i / F.k)) - 1))] = i;
        }
        __syncthreads();
    }
    const int64_t c0 = (int64_t)blockIdx.x * 16;
    const int c = lane & 15, part = lane >> 4;
    const int64_t col = c0 + c < F.hidden ? c0 + c : F.hidden - 1;
    using Wp = Part<W>;
    const int64_t nb = blocks_of(F.inner), row_w = Wp::row(F.inner);
    // whole blocks of all tasks in a pipeline; what is behind them (all, for rows that do not start on 16 bytes) one block at a time
    const int per = WIDE ? (int)(F.inner / kBlock) : 0;
    const int units = RING ? (per + 1) / 2 : per;                // of a task
    const int64_t total = (int64_t)n_tasks * units;
    const int lo = (int)(total * w / kFewSecond), hi = (int)(total * (w + 1) / kFewSecond);
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    // one block of a task's activations, in two parts
    struct Act { v8b x[4], z[4]; };
    auto load_h = [&](Act& a, int task, int64_t at, auto full) {
#pragma unroll
        for (int h = 0; h < 4; ++h) a.x[h] = a.z[h] = v8b{};
        if (c < task_count[task]) {                               // places without a pair are zeros, and cost no loads
            const unsigned lane_at = (unsigned)(pair_of[task_first[task] + c] * F.ld_h) + Part<W>::at(0, part);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int k = Part<W>::at(h, 0);
                if (full.value) {
                    a.x[h] = as_bf16(*(const v4u*)((const uint8_t*)(F.hi + at + k) + (size_t)(lane_at * 2)));
                    a.z[h] = as_bf16(*(const v4u*)((const uint8_t*)(F.lo + at + k) + (size_t)(lane_at * 2)));
                } else {
                    const int64_t left = F.inner - at - k - Part<W>::at(0, part);
                    a.x[h] = as_bf16(bits8<true>(F.hi + at + k + lane_at, left));
                    a.z[h] = as_bf16(bits8<true>(F.lo + at + k + lane_at, left));
                }
            }
        }
    };
    auto multiply = [&](const Act& a, const Part<W>& v, float scale) {
        v4f y = Wp::INSIDE ? acc : v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const v8b bw = v.eight(h, scale);
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x[h], bw, y, 0, 0, 0);
            y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.z[h], bw, y, 0, 0, 0);
        }
        if (Wp::INSIDE) acc = y;
        else acc += y * scale;
    };
    auto keep = [&](int task) {                                   // to the tokens' sums
        const int n = task_count[task], p0 = task_first[task];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = part * 4 + i;
            if (r < n) {
                const int p = pair_of[p0 + r];
                sums[p / F.k * 16 + c] += weight[p] * acc[i];
            }
        }
        acc = v4f{0.f, 0.f, 0.f, 0.f};
        wave_lds_done();
    };
    struct Cursor { int task, block; };                           // a place in the sequence
    if constexpr (RING) {
        // As in the first kernel: weights through the LDS, two blocks at a time (one where a task's last has none beside it: the other half is then that one again,
        // and not used), scales as a word in the lanes 0 to 15 and one in 16 to 31.  A task is up to four pairs, so that one load of each part of
        // the activations brings all steps of a block; more pairs of an expert are its next task, whose weights are then near.
        struct Ahead { unsigned k; v8b x[2][1], z[2][1]; };
        const unsigned slots = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&ring[w][0][0];
        const int64_t each = Wp::scales(1, F.hidden, 0, F.inner, 0);
        unsigned off[2];
        const int chunk = (lane & 7) ^ (lane >> 4);               // of the first eight rows; of the second it is 4 further or nearer
#pragma unroll
        for (int j = 0; j < 2; ++j) off[j] = (unsigned)((c0 + j * 8 + (lane >> 3) < F.hidden ? c0 + j * 8 + (lane >> 3) : F.hidden - 1) * row_w);
        const uint8_t* scale_row = (const uint8_t*)F.s2 + Wp::scales(0, F.hidden, col, F.inner, 0);
        const int place = c * 128 + (part ^ (c >> 1)) * 16;
        auto step = [&](Cursor& q) { if (++q.block == units) { q.block = 0; ++q.task; } };
        Cursor now = {units ? lo / units : 0, units ? lo % units : 0}, far = now;
        auto fetch = [&](Ahead& t, int unit) {
            const int e = __builtin_amdgcn_readfirstlane(task_expert[far.task]);
            const int two = far.block * 2 + 1 < per ? 1 : 0;      // there is a second block
            const unsigned to = slots + (unsigned)unit % Wp::kAhead2 * 2048, in = (chunk & (two ? 7 : 3)) * 16;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // what is read of this part of the LDS has been read
            const uint8_t* from = scalar((const uint8_t*)((const W*)F.w2 + (int64_t)e * F.hidden * row_w + far.block * (2 * Wp::kUnit)));
            dma16(from, off[0] + in, to);
            dma16(from, off[1] + (two ? in ^ 64u : in), to + 1024);
            t.k = 0;
            if (lane < 32) __builtin_memcpy(&t.k, scale_row + e * each + (far.block * 2 + (lane >> 4) * two) * Wp::kScales, 4);
#pragma unroll
            for (int half = 0; half < 2; ++half) t.x[half][0] = t.z[half][0] = v8b{};
            if ((c & 3) < task_count[far.task]) {
                const unsigned at = ((unsigned)(pair_of[task_first[far.task] + (c & 3)] * F.ld_h) + part * 32 + (c >> 2) * 8) * 2;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int64_t b = (far.block * 2 + half * two) * kBlock;
                    t.x[half][0] = as_bf16(*(const v4u*)((const uint8_t*)(F.hi + b) + (size_t)at));
                    t.z[half][0] = as_bf16(*(const v4u*)((const uint8_t*)(F.lo + b) + (size_t)at));
                }
            }
            step(far);
        };
        Ahead st[Wp::kAhead2];
        pipeline<Wp::kAhead2, false>(st, lo, hi, fetch, [&](const Ahead& t, int unit) {
            asm volatile("" ::"v"(t.k) : "memory");
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (half && now.block * 2 + 1 >= per) break;
                Part<W> v;
                v.v = *(const v4u*)(ring[w][(unsigned)unit % Wp::kAhead2] + (place ^ half * 64));
                const unsigned k = (unsigned)__shfl((int)t.k, half * 16 + c) >> (part * 8) & 255u;
                Act a;
                later_steps<4>(t.x[half], a.x);
                later_steps<4>(t.z[half], a.z);
                multiply(a, v, scale_float<TUNA_SCALE_E8>(k));
            }
            if (unit + 1 == hi || now.block + 1 == units) keep(now.task);
            step(now);
        });
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // nothing is on its way to the LDS when it is given back
    } else if constexpr (WIDE) {
        struct Ahead { Part<W> v; float k; Act a; };
        const int64_t at_s = Wp::scales(0, F.hidden, col, F.inner, part), each = Wp::scales(1, F.hidden, 0, F.inner, 0);
        const unsigned off_w = (unsigned)(col * row_w * sizeof(W)) + part * 16;
        auto step = [&](Cursor& q) { if (++q.block == per) { q.block = 0; ++q.task; } };
        Cursor now = {per ? lo / per : 0, per ? lo % per : 0}, far = now;
        auto fetch = [&](Ahead& t, int) {
            const int e = __builtin_amdgcn_readfirstlane(task_expert[far.task]);
            t.v.whole((const W*)F.w2 + (int64_t)e * F.hidden * row_w + far.block * Wp::kUnit, off_w);
            t.k = scale_value<KIND>(F.s2, e * each + far.block * Wp::kScales + at_s);
            load_h(t.a, far.task, far.block * kBlock, Int<1>{});
            step(far);
        };
        Ahead st[Wp::kAhead2];
        pipeline<Wp::kAhead2, false>(st, lo, hi, fetch, [&](const Ahead& t, int u) {
            multiply(t.a, t.v, t.k);
            if (u + 1 == hi || now.block + 1 == per) keep(now.task);      // the wave's last of this task
            step(now);
        });
    }
    if (per < nb) {
        for (int task = w; task < n_tasks; task += kFewSecond) {
            const int e = __builtin_amdgcn_readfirstlane(task_expert[task]);
            for (int64_t b = per; b < nb; ++b) {
                Part<W> v;
                v.template load<WIDE>((const W*)F.w2 + ((int64_t)e * F.hidden + col) * row_w + b * Wp::kUnit, part, F.inner - b * kBlock);
                Act a;
                load_h(a, task, b * kBlock, Int<0>{});
                multiply(a, v, scale_value<KIND>(F.s2, Wp::last(Wp::scales(e, F.hidden, col, F.inner, part) + b * Wp::kScales, b, part, F.inner)));
            }
            keep(task);
        }
    }
    __syncthreads();
    for (int i = tid; i < F.tokens * 16; i += kFewSecond * 64) {
        float s = 0.f;
        for (int q = 0; q < kFewSecond; ++q) s += shared[q * F.tokens * 16 + i];
        if (c0 + (i & 15) < F.hidden) store1((OUT*)F.out + (i >> 4) * F.ld_out + c0 + (i & 15), s);
    }
}

}  // namespace moe
