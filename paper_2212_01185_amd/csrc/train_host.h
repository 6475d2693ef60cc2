// What the host side of the training operators shares: launches, checks of arguments, chunks of ragged groups of rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "pcc.h"

namespace pcc_train {

// The status of a launch.  An error that another call left is not this one's: it is taken away before.
template <class F>
int launch(F&& f) {
    (void)hipGetLastError();
    f();
    return hipGetLastError() == hipSuccess ? PCC_OK : PCC_E_HIP;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() { if (prev >= 0) (void)hipSetDevice(prev); }
};

constexpr size_t kMaxLd = (size_t)1 << 22;
constexpr size_t kMaxRows = (size_t)1 << 40;

// A launch has fewer than 2^32 threads (some grids are rounded up to a multiple of eight workgroups).
inline bool launchable(uint64_t blocks, int threads) { return blocks < ((uint64_t)1 << 32) / threads - 8; }

inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline size_t size_of(int type) { return type == PCC_FP32 ? 4 : 2; }

// `count` rows of `length` bytes, `pitch` apart; what is one piece is one row.
struct Span {
    const void* p;
    size_t count, pitch, length;
};
inline Span piece(const void* p, size_t bytes) { return {p, 1, bytes, bytes}; }
// Whether they share bytes.  Rows at one distance may lie beside each other (columns of one buffer).
inline bool overlap(const Span& a, const Span& b) {
    if (!a.p || !b.p || !a.count || !b.count || !a.length || !b.length) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    if (a0 + (a.count - 1) * a.pitch + a.length <= b0 || b0 + (b.count - 1) * b.pitch + b.length <= a0) return false;
    if (a.pitch != b.pitch || a.count == 1 || b.count == 1) return true;
    const size_t apart = a0 <= b0 ? (b0 - a0) % a.pitch : (a.pitch - (a0 - b0) % a.pitch) % a.pitch;    // of b's row from a's in front of it
    return apart < a.length || a.pitch - apart < b.length;
}
inline bool overlap(const Span& a, std::initializer_list<Span> others) {
    return std::any_of(others.begin(), others.end(), [&](const Span& b) { return overlap(a, b); });
}
inline bool ld_ok(size_t ld, int features) { return ld >= (size_t)features && ld <= kMaxLd; }

// More LDS than 64 KB, a kernel's static variables among it, has to be asked for; per device and kernel, and cheap enough to do at every launch.
// No kernel that comes here has more than this of static ones (the norm's forward pass of 1024 lanes has 384 bytes).
constexpr size_t kStaticLds = 1024;
template <class K>
bool allow_lds(K kernel, size_t bytes) {
    return bytes <= 64 * 1024 - kStaticLds || hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
}

// Chunks of mult * 2^log2 rows: about rows / want rows, in steps of 1/4 to 1/8 of a power of two, and a multiple of `unit` (a power of two).  The
// number of chunks (with one more for each group's part) is at most `want`, if there are not too many groups for that.
inline void chunk_rows(int64_t all, int groups, uint64_t want, int unit_log2, int& log2, uint32_t& mult) {
    const uint64_t whole = want > 2 * (uint64_t)groups ? want - groups : std::max<uint64_t>(want, 1) / 2 + 1;
    const uint64_t rows = std::max<uint64_t>(((uint64_t)all + whole - 1) / whole, 1);
    log2 = unit_log2;
    while (log2 < 24 && ((uint64_t)8 << log2) < rows) ++log2;     // rows of a chunk are counted in 32 bits
    mult = (uint32_t)std::min<uint64_t>((rows + ((uint64_t)1 << log2) - 1) >> log2, 8);
}
inline uint64_t chunk_count(int64_t rows, int groups, int log2, uint32_t mult) { return (uint64_t)rows / ((uint64_t)mult << log2) + groups; }
// Chunks that can be in groups of more than one: such a group of n has more than (n - 1) chunks' rows, n/2 at least.
inline size_t shared_chunks(size_t rows, int groups, size_t chunk) {
    return rows <= chunk ? 0 : std::min(rows / chunk + groups, 2 * (rows / chunk));
}

}  // namespace pcc_train
