// What the kernels of include/tuna_moe.h share: values in memory and in registers, moves between lanes, shares of a softmax, groups of rows, loads ahead of
// their use.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "tuna_moe.h"

namespace moe {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));

constexpr int kBlock = 128;            // values that share a scale
constexpr int kBlock4 = 32;            // and in 4 bits
template <int V> struct Int { static constexpr int value = V; };
constexpr int kLanes = 64;

__device__ __forceinline__ int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// ------------------------------------------------------------------------------------------------ values

__device__ __forceinline__ float bf16_bits(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ unsigned short to_bf16(float v) {      // to nearest, ties to even; NaN stays NaN
    const __bf16 h = (__bf16)v;
    unsigned short b;
    __builtin_memcpy(&b, &h, 2);
    return b;
}

template <class T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<unsigned short>(const unsigned short* p) { return bf16_bits(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(unsigned short* p, float v) { *p = to_bf16(v); }

// Eight neighbours, of which `left` are inside the row (the others read as 0 and are not stored).  WIDE: the address is on 16 bytes.
template <bool WIDE> __device__ __forceinline__ void load8(const float* p, int64_t left, float (&v)[8]) {
    if (WIDE && left >= 8) {
        const v4f a = *(const v4f*)p, b = *(const v4f*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
}
template <bool WIDE> __device__ __forceinline__ void load8(const unsigned short* p, int64_t left, float (&v)[8]) {
    if (WIDE && left >= 8) {
        const v4u a = *(const v4u*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_bits(p[i]) : 0.f;
}
template <bool WIDE> __device__ __forceinline__ void store8(float* p, int64_t left, const float (&v)[8]) {
    if (WIDE && left >= 8) {
        *(v4f*)p = v4f{v[0], v[1], v[2], v[3]};
        *(v4f*)(p + 4) = v4f{v[4], v[5], v[6], v[7]};
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = v[i];
}
template <bool WIDE> __device__ __forceinline__ void store8(unsigned short* p, int64_t left, const float (&v)[8]) {
    if (WIDE && left >= 8) {
        v4u a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = (unsigned)to_bf16(v[2 * i]) | (unsigned)to_bf16(v[2 * i + 1]) << 16;
        *(v4u*)p = a;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = to_bf16(v[i]);
}

// Eight 16-bit values of which `left` exist, as they lie; zeros behind them.
template <bool WIDE> __device__ __forceinline__ v4u bits8(const unsigned short* p, int64_t left) {
    v4u a = {0u, 0u, 0u, 0u};
    if (WIDE && left >= 8) return *(const v4u*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) a[i >> 1] |= (unsigned)p[i] << (16 * (i & 1));
    return a;
}

// Sixteen 8-bit values of which `left` exist; zeros behind them.  WIDE: on 16 bytes, and rows of whole sixteens.
template <bool WIDE> __device__ __forceinline__ v4u chunk16(const uint8_t* p, int64_t left) {
    v4u a = {0u, 0u, 0u, 0u};
    if (left <= 0) return a;
    if (WIDE) return *(const v4u*)p;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < left) a[i >> 2] |= (unsigned)p[i] << (8 * (i & 3));
    return a;
}

// Thirty-two 4-bit values of which `left` exist; zeros behind them.  WIDE: on 16 bytes.
template <bool WIDE> __device__ __forceinline__ v4u chunk32(const uint8_t* p, int64_t left) {
    if (WIDE && left >= 32) return *(const v4u*)p;
    v4u a = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (2 * i < left) a[i >> 2] |= (2 * i + 1 < left ? (unsigned)p[i] : (unsigned)p[i] & 15u) << (8 * (i & 3));
    return a;
}

// ------------------------------------------------------------------------------------------------ moves between lanes

// What a wave's lanes have written to the LDS is there for its other lanes.
__device__ __forceinline__ void wave_lds_done() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ int wave_scan(int v, int lane) {       // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// The largest, and the sum, of a wave's 64 values, as scalars: shifts within rows of 16 lanes, then from row to row.
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned old, unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ unsigned wave_max_scan(unsigned v) {   // inclusive, in vector registers
    auto more = [&](unsigned o) { v = o > v ? o : v; };
    more(dpp<0x111>(v, v));
    more(dpp<0x112>(v, v));
    more(dpp<0x114>(v, v));
    more(dpp<0x118>(v, v));
    more(dpp<0x142>(v, v));
    more(dpp<0x143>(v, v));
    return v;
}
__device__ __forceinline__ unsigned wave_max(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)wave_max_scan(v), 63); }
__device__ __forceinline__ float wave_total(float v) {
    auto more = [&](unsigned o) { v += __uint_as_float(o); };
    more(dpp<0x111>(0u, __float_as_uint(v)));
    more(dpp<0x112>(0u, __float_as_uint(v)));
    more(dpp<0x114>(0u, __float_as_uint(v)));
    more(dpp<0x118>(0u, __float_as_uint(v)));
    more((unsigned)__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
    more((unsigned)__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// exp(x) for x <= 88 within two units of the last place: 2^(x log2 e), with what the product rounds away put back.
__device__ __forceinline__ float exp_32(float x) {
    constexpr float kLog2e = 1.44269504088896341f, kRest = 1.9259629911266175e-08f, kLn2 = 0.693147180559945309f;
    const float t = x * kLog2e;
    const float rest = __builtin_fmaf(x, kRest, __builtin_fmaf(x, kLog2e, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return t > -150.f ? __builtin_fmaf(e, rest * kLn2, e) : 0.f;
}

// ------------------------------------------------------------------------------------------------ shares and gates

// A logit as a key whose order is the logits' (ties by index come from the index below it); 0 = not eligible.
__device__ __forceinline__ unsigned logit_key(float v) {
    v += 0.0f;                                                    // -0 and +0 are equal
    const unsigned b = __float_as_uint(v);
    if (v != v || b == 0xff800000u) return 0u;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float key_logit(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// exp(l - top) for eligible logits; where the largest is +inf, only those at +inf have a share.
__device__ __forceinline__ float exp_share(float l, float top) {
    if (logit_key(l) == 0u) return 0.f;
    if (top == __builtin_inff()) return l == top ? 1.f : 0.f;
    return exp_32(l - top);
}

__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a < __builtin_inff() ? a : 0.f;                        // NaN too
}

// The sigmoid of g and silu(g) = g sigmoid(g).  1 / (1 + exp(-g)) is one approximate reciprocal and a step of Newton's, exact to a unit of the last
// place.  Below -87, where exp(-g) would leave the range, the sigmoid is exp(g) (the 1 is far below its last place), taken as exp(g + 44) exp(-44):
// the sum is exact, and the product with exp(-44) comes last, so that it alone goes below the normal numbers, down to 0.  A sigmoid that
// stopped at some small value would leave a large negative gate something of itself.
struct Gate { float sigmoid, silu; };
__device__ __forceinline__ Gate gate_of(float g) {
    const bool low = g < -87.f;
    const float e = exp_32(low ? g + 44.f : -g), d = 1.f + e;
    const float r = __builtin_amdgcn_rcpf(d);
    Gate t;
    t.sigmoid = low ? e : __builtin_fmaf(__builtin_fmaf(-d, r, 1.f), r, r);
    t.silu = g * t.sigmoid;
    if (low) { t.sigmoid *= 7.78113224e-20f; t.silu *= 7.78113224e-20f; }
    return t;
}

// ------------------------------------------------------------------------------------------------ groups of rows

// Where a block of 128 rows of the columns' form lies: block `want` of all groups' blocks.
struct Place { int group; int64_t first, end, block; };           // rows first .. end - 1; block: its number among all

// The groups g0 .. g0 + 63 of `groups`, one a lane: rows a .. b - 1 of [0, m).  A bound counts as the largest of all up to it, so that groups never
// overlap, and their blocks of n rows are at most ceil(m / n) + groups - 1 whatever the bounds are: what the host has checked room for.  low: the
// largest bound before g0's groups, then before the next 64's.
__device__ __forceinline__ int bound_at(const int32_t* group_rows, int i, int64_t m) {
    const int v = group_rows[i];
    return v < 0 ? 0 : v > m ? (int)m : v;
}
__device__ __forceinline__ void group_bounds(const int32_t* group_rows, int groups, int g0, int64_t m, int& low, int& a, int& b) {
    const int lane = threadIdx.x & 63, g = g0 + lane;
    const int top = (int)wave_max_scan(g < groups ? (unsigned)bound_at(group_rows, g + 1, m) : 0u), before = __shfl_up(top, 1);
    b = top > low ? top : low;
    a = lane > 0 && before > low ? before : low;
    low = __builtin_amdgcn_readlane(b, 63);
}

// The group and the part of it that tile number `want` is, tiles of `size` rows counted group after group; group -1: there is none.
__device__ __forceinline__ Place find_tile(const int32_t* group_rows, int groups, int64_t m, int size, int64_t want) {
    const int lane = threadIdx.x & 63;
    if (!group_rows) {
        Place p = {want * size < m ? 0 : -1, want * size, want * size + size < m ? want * size + size : m, want};
        return p;
    }
    int64_t done = 0;
    int low = bound_at(group_rows, 0, m);
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int a, b;
        group_bounds(group_rows, groups, g0, m, low, a, b);
        const int n = (int)(((int64_t)b - a + size - 1) / size);
        const int inc = wave_scan(n, lane);
        const unsigned long long hit = __ballot(done + inc > want);
        if (hit) {
            const int l = __ffsll((long long)hit) - 1;
            const int64_t before = done + __shfl(inc, l) - __shfl(n, l);
            const int64_t first = (int64_t)__shfl(a, l) + (want - before) * size;
            const int64_t end = (int64_t)__shfl(b, l);
            Place p = {g0 + l, first, first + size < end ? first + size : end, want};
            return p;
        }
        done += __shfl(inc, 63);
    }
    Place p = {-1, 0, 0, 0};
    return p;
}

// The first block of `size` rows of a group (128: in the columns' form), and how many it has.
__device__ __forceinline__ void group_blocks(const int32_t* group_rows, int groups, int g, int64_t m, int64_t& first, int64_t& count, int size = kBlock) {
    const int lane = threadIdx.x & 63;
    if (!group_rows) { first = 0; count = (m + size - 1) / size; return; }
    int64_t done = 0;
    int low = bound_at(group_rows, 0, m);
    for (int g0 = 0; g0 <= g; g0 += 64) {
        int a, b;
        group_bounds(group_rows, groups, g0, m, low, a, b);
        const int n = (int)(((int64_t)b - a + size - 1) / size);
        const int inc = wave_scan(n, lane);
        const int l = g - g0 < 63 ? g - g0 : 63;
        count = __shfl(n, l);
        done += __shfl(inc, l);
    }
    first = done - count;
}

// Workgroups go to the eight XCDs in turn: each XCD gets a run of neighbouring tiles, whose operands meet in its L2.  The tile of workgroup `id`
// among `total`, or -1 (there may be more workgroups than tiles).
__device__ __forceinline__ int xcd_run(unsigned id, unsigned total) {
    const unsigned per = total / 8, more = total % 8, x = id % 8, at = id / 8;
    return at < per + (x < more ? 1 : 0) ? (int)(x * per + (x < more ? x : more) + at) : -1;
}

// How many tiles of `size` rows the groups have.
__device__ __forceinline__ int count_tiles(const int32_t* group_rows, int groups, int64_t m, int size) {
    if (!group_rows) return (int)((m + size - 1) / size);
    int n = 0, low = bound_at(group_rows, 0, m);
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int a, b;
        group_bounds(group_rows, groups, g0, m, low, a, b);
        n += (int)(((int64_t)b - a + size - 1) / size);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    return n;
}

// ------------------------------------------------------------------------------------------------ loads and stores

// Units lo .. hi - 1: each is fetched AHEAD - 1 units before it is used.  In the loop no load hangs on a condition, so that a wait for one unit's
// leaves the later ones' under way, as long as none does in `fetch`.  (Those of the 4-bit forms do, and load into the LDS besides, which the compiler does not
// count: it then waits for all loads once a unit, or once in AHEAD units, the last asked for included.)  MANY: the loop runs to the end, where it fetches the last unit again; else the end is a loop of its own,
// which costs registers and spares short runs those loads (one token: both kernels 23.1 us with them, 18.2 without).
template <int AHEAD, bool MANY, class S, class FETCH, class USE> __device__ __forceinline__ void pipeline(S (&st)[AHEAD], int lo, int hi, FETCH fetch, USE use) {
    if (MANY && lo >= hi) return;
#pragma unroll
    for (int d = 0; d < AHEAD - 1; ++d) if (MANY || lo + d < hi) fetch(st[d], lo + d < hi ? lo + d : hi - 1);
    int v = lo;
    for (; MANY ? v < hi : v + 2 * AHEAD - 2 < hi; v += AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int next = v + d + AHEAD - 1;
            fetch(st[(d + AHEAD - 1) % AHEAD], !MANY || next < hi ? next : hi - 1);
            __builtin_amdgcn_sched_barrier(0);
            if (!MANY || v + d < hi) use(st[d], v + d);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (!MANY)
        for (; v < hi; v += AHEAD) {
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) {
                if (v + d + AHEAD - 1 < hi) fetch(st[(d + AHEAD - 1) % AHEAD], v + d + AHEAD - 1);
                if (v + d < hi) use(st[d], v + d);
            }
        }
}

// Sixteen bytes a lane (or a scale a lane, as a word) from memory straight into the LDS, lane after lane behind `to`.
template <int BYTES> __device__ __forceinline__ void to_lds(const void* from, void* to) {
    const auto* g = (const __attribute__((address_space(1))) void*)from;
    auto* l = (__attribute__((address_space(3))) void*)to;
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds(g, l, 16, 0, 0);
    else if constexpr (BYTES == 4) __builtin_amdgcn_global_load_lds(g, l, 4, 0, 0);
    else __builtin_amdgcn_global_load_lds(g, l, 1, 0, 0);
}

// Sixteen bytes a lane from memory straight into the LDS, lane after lane behind `to`, which a wave has in common: from a base that it has in common and a
// lane's offset, or from a lane's address.  Nothing but the counter of loads says when they are there: whoever reads the LDS waits for it.
__device__ __forceinline__ void dma16(const uint8_t* base, unsigned off, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma16(const uint8_t* from, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
// An address that a wave has in common, as one of its scalars.
__device__ __forceinline__ const uint8_t* scalar(const uint8_t* p) {
    const uint64_t v = (uint64_t)p;
    const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)v), high = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
    return (const uint8_t*)((uint64_t)high << 32 | low);
}

// Up to four neighbours of a row of the result, in one store where all exist and lie on their size.
template <class OUT> __device__ __forceinline__ void store_four(OUT* o, const v4f& v, int n) {
    if (n == 4 && ((uintptr_t)o & (4 * sizeof(OUT) - 1)) == 0) {
        if constexpr (sizeof(OUT) == 2) *(v2u*)o = v2u{(unsigned)to_bf16(v[0]) | (unsigned)to_bf16(v[1]) << 16, (unsigned)to_bf16(v[2]) | (unsigned)to_bf16(v[3]) << 16};
        else *(v4f*)o = v;
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) if (q < n) store1(o + q, v[q]);
}

}  // namespace moe
