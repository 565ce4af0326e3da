// Host checks of row-strided tensors and the chip's size, shared by entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "gdn_resume.h"

namespace gdn {

// `rows` rows of `width` bytes, `pitch` bytes apart.
struct Rows {
    uintptr_t at;
    int64_t rows, pitch, width;
    Rows(const void* p, int64_t n, int64_t pitch_, int64_t width_) : at(reinterpret_cast<uintptr_t>(p)), rows(p ? n : 0), pitch(pitch_), width(width_) {}
    uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};

// Whether two tensors share a byte.  Columns of one wider buffer (rows of equal pitch) are told apart exactly; rows
// of different pitches whose spans meet count as sharing.
inline bool share_bytes(const Rows& a, const Rows& b) {
    if (a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
    if (a.end() <= b.at || b.end() <= a.at) return false;
    if (a.rows == 1 || b.rows == 1 || a.pitch != b.pitch) {
        // one row against many: its span may lie in the gap between two rows of the other
        const Rows &one = a.rows == 1 ? a : b, &many = a.rows == 1 ? b : a;
        if (one.rows != 1 || many.rows == 1 || one.at < many.at) return true;
        const int64_t off = (int64_t)((one.at - many.at) % (uintptr_t)many.pitch);
        return off < many.width || off + one.width > many.pitch;
    }
    const uintptr_t lo = a.at < b.at ? a.at : b.at, hi = a.at < b.at ? b.at : a.at;
    const int64_t lo_width = a.at < b.at ? a.width : b.width, hi_width = a.at < b.at ? b.width : a.width;
    const int64_t off = (int64_t)((hi - lo) % (uintptr_t)a.pitch);
    return off < lo_width || off + hi_width > a.pitch;
}

// The same rows, element for element: an output over an input that each thread reads before it writes.
inline bool same_rows(const Rows& a, const Rows& b) {
    return a.at == b.at && a.width == b.width && a.rows == b.rows && (a.pitch == b.pitch || a.rows <= 1);
}

// Compute units of the chip (256 where that cannot be asked).
inline int chip_cus() {
    static const int n = [] {
        int dev = 0, cus = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
            (void)hipGetLastError();
            return 256;
        }
        return cus;
    }();
    return n;
}

// Lets a kernel have more than 64 KiB of LDS, once for each device that it is launched on; `done`: the kernel's own.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

inline bool dtype_known(int32_t t) { return t == GDN_F32 || t == GDN_BF16; }
inline int dtype_bytes(int32_t t) { return t == GDN_F32 ? 4 : 2; }
inline bool off_align(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

}  // namespace gdn
