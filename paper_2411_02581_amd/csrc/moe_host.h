// What the C entry points of include/tuna_moe.h share: checks of arguments, limits of a launch, types and flags carried into templates.
#pragma once
#include "moe_common.h"
#include <cstdint>
#include <type_traits>

namespace tuna_host {
// tuna_api.hip: the device of the library's first call, and the code of a HIP call that failed
__attribute__((visibility("hidden"))) int ensure_device();
__attribute__((visibility("hidden"))) void note_hip_error(int code);
}

using namespace moe;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int64_t kMaxGridY = 65535;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align16(size_t v) { return (v + 15) / 16 * 16; }
inline bool on(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline int size_of(int type) { return type == TUNA_F32 ? 4 : type == TUNA_BF16 ? 2 : 1; }
inline bool is_float(int type) { return type == TUNA_F32 || type == TUNA_BF16; }
inline bool is_scale(int type) { return type == TUNA_SCALE_F32 || type == TUNA_SCALE_E8; }
inline int scale_size(int type) { return type == TUNA_SCALE_F32 ? 4 : 1; }

// An array of rows whose elements are aligned; and whether every row starts on 16 bytes.
inline bool rows_ok(const void* p, int size, int64_t ld, int64_t cols) { return p && on(p, size) && ld >= cols; }
inline bool rows_wide(const void* p, int size, int64_t ld) { return on(p, 16) && (ld * size) % 16 == 0; }

// A grid dimension has at most 2^32 - 1 threads.
inline bool grid_fits(int64_t blocks, int threads) { return blocks <= 0xffffffffll / threads; }

// A thread for eight neighbours, a row (y and z) at a time.
inline bool eights_fit(int64_t rows, int64_t cols) { return ceil_div(rows, 32768) <= kMaxGridY && ceil_div(cols, 2048) <= kMaxRows / 256; }
inline dim3 eights_grid(int64_t rows, int64_t cols) {
    return dim3((unsigned)ceil_div(cols, 2048), (unsigned)(rows < 32768 ? rows : 32768), (unsigned)ceil_div(rows, 32768));
}

inline int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return TUNA_OK;
    tuna_host::note_hip_error((int)e);
    return TUNA_ERR_HIP;
}

#define LAUNCH(kernel, grid, threads, ...) hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, (hipStream_t)stream, __VA_ARGS__)

// Calls f with a null pointer of the type that `type` names, to carry it into a template.
template <class F> inline void with_type(int type, F f) {
    if (type == TUNA_F32) f((float*)nullptr); else f((unsigned short*)nullptr);
}
template <class F> inline void with_bool(bool b, F f) { if (b) f(Int<1>{}); else f(Int<0>{}); }
template <class T> using Pointee = typename std::remove_pointer<T>::type;

}  // namespace
