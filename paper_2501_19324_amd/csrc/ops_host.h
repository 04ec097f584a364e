// What the operators' entry points share on the host: errors, launches, and whether arrays that a kernel would race on share memory.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "rsd_ops.h"

namespace __attribute__((visibility("hidden"))) rsd_ops_host {

inline thread_local char op_error[256] = "";


inline int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(op_error, sizeof(op_error), fmt, ap);
    va_end(ap);
    return code;
}
// The launches of a call, by the status that each returns: the runtime's last error may be one that the caller has not read yet, and stays.
class Launches {
    hipStream_t st_;
    hipError_t first_ = hipSuccess;
public:
    explicit Launches(void* stream) : st_(static_cast<hipStream_t>(stream)) {}
    template <typename... P> void run(void (*kernel)(P...), dim3 grid, unsigned threads, size_t lds, std::common_type_t<P>... args) {
        if (first_ != hipSuccess) return;
        void* at[] = {&args...};
        first_ = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, lds, st_);
    }
    int done(const char* what) {
        if (first_ == hipSuccess) return RSD_OK;
        (void)hipGetLastError();                            // reported here
        return fail(RSD_EHIP, "%s: %s", what, hipGetErrorString(first_));
    }
};
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool is_type(int32_t t) { return t == RSD_F32 || t == RSD_BF16; }
inline size_t size_of(int32_t t) { return t == RSD_F32 ? 4 : 2; }
inline uint64_t up256(uint64_t n) { return (n + 255) & ~255ull; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kMostBlocks = 1ll << 22;      // blocks of at most 512 threads: a launch counts threads in 32 bits per dimension

// Pieces of `len` elements at i s0 + j s1, i < n0, j < n1: whether two of them share an element.  Mostly one stride passes the other's pieces, which is seen
// at once; else every distance in the shorter dimension is set against the nearest ones in the other.
inline bool pieces_overlap(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t len) {
    typedef __int128 wide;
    if (n0 > n1) std::swap(n0, n1), std::swap(s0, s1);
    const wide a = s0 < 0 ? -(wide)s0 : s0, b = s1 < 0 ? -(wide)s1 : s1;      // distances count in both directions
    if (n0 == 1) return n1 > 1 && b < len;
    if (a < len || b < len) return true;
    if (b >= (n0 - 1) * a + len || a >= (n1 - 1) * b + len) return false;
    for (wide i = 1; i < n0; ++i) {
        const wide j = i * a / b;
        if ((j < n1 && i * a - j * b < len) || (j + 1 < n1 && (j + 1) * b - i * a < len)) return true;
    }
    return false;
}

// Two arrays of one type, pieces at i s0 + j s1 of each (i < n0, j < n1), of `len` elements
struct Pieces { const void* at; int64_t s0, s1, len; };
// Whether they share an element.  Views of one buffer (heads of q beside those of out) mostly have the same s0; where that differs, arrays that lie between
// each other's ends count as sharing.
inline bool share_memory(Pieces p, Pieces q, int64_t n0, int64_t n1, size_t size) {
    typedef __int128 wide;
    if (n0 == 1) p.s0 = q.s0 = 0;
    if (n1 == 1) p.s1 = q.s1 = 0;
    const wide d = ((wide)reinterpret_cast<uintptr_t>(q.at) - (wide)reinterpret_cast<uintptr_t>(p.at)) / (int64_t)size;
    auto low = [&](const Pieces& x) { return std::min<wide>(0, (wide)(n0 - 1) * x.s0) + std::min<wide>(0, (wide)(n1 - 1) * x.s1); };
    auto high = [&](const Pieces& x) { return std::max<wide>(0, (wide)(n0 - 1) * x.s0) + std::max<wide>(0, (wide)(n1 - 1) * x.s1) + x.len; };
    if (d + low(q) >= high(p) || d + high(q) <= low(p)) return false;
    if (p.s0 != q.s0) return true;
    const wide s0 = p.s0 < 0 ? -(wide)p.s0 : p.s0;         // distances in i count in both directions
    auto floor_div = [](wide a, wide b) { return a / b - (a % b < 0); };
    if (s0 > 0 && p.s1 >= 0 && q.s1 >= 0) {                 // side by side in every row of the buffer
        const wide from = d - floor_div(d, s0) * s0;
        if (from >= (n1 - 1) * (wide)p.s1 + p.len && from + (n1 - 1) * (wide)q.s1 + q.len <= s0) return false;
    }
    // q's piece starts `c` behind p's, and a multiple of s0: somewhere between -q.len and p.len?
    auto meet = [&](wide c) {
        return s0 == 0 ? c > -q.len && c < p.len : std::max<wide>(-floor_div(q.len - 1 + c, s0), 1 - n0) <= std::min<wide>(floor_div(p.len - 1 - c, s0), n0 - 1);
    };
    for (int64_t j = 0; j < n1; ++j)
        for (int64_t i = 0; i < n1; ++i) {
            if (p.s1 == q.s1 && i > 0 && j > 0) break;      // (only their distance counts)
            if (meet(d + (wide)j * q.s1 - (wide)i * p.s1)) return true;
        }
    return false;
}

}  // namespace rsd_ops_host
using namespace rsd_ops_host;
