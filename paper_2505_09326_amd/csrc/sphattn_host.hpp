// What the host side of the entry points around the attention shares: ranges of memory, alignment, workspaces, launches.
#pragma once
#include "../../include/sphattn.h"

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <atomic>

namespace {

constexpr int kCus = 256;

// A range of bytes that a call reads or writes.
struct Range { const void* at; size_t bytes; };

bool meet(const Range& a, const Range& b)
{
    if (!a.at || !b.at || !a.bytes || !b.bytes) return false;
    const uintptr_t a0 = (uintptr_t)a.at, b0 = (uintptr_t)b.at;
    return a0 <= b0 ? b0 - a0 < a.bytes : a0 - b0 < b.bytes;
}

// Each written range against everything else.
template <int W, int R>
bool any_meet(const Range (&written)[W], const Range (&read)[R])
{
    for (int i = 0; i < W; ++i) {
        for (int j = i + 1; j < W; ++j)
            if (meet(written[i], written[j])) return true;
        for (int j = 0; j < R; ++j)
            if (meet(written[i], read[j])) return true;
    }
    return false;
}

bool off(const void* p, size_t alignment) { return ((uintptr_t)p & (alignment - 1)) != 0; }

int element_bytes(int dtype)
{
    return dtype == SPHATTN_F32 ? 4 : dtype == SPHATTN_BF16 || dtype == SPHATTN_F16 ? 2 : 0;
}

int launched() { return hipGetLastError() == hipSuccess ? SPHATTN_OK : SPHATTN_ERR_LAUNCH; }

// A kernel with more than 64 KB of LDS needs its limit raised once per device.  `done` is the kernel's own: kernels of one type
// share whatever a template over the type keeps.
template <typename Kern>
bool raise_lds_limit(Kern kern, int lds_bytes, std::atomic<uint64_t>& done)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
        (void)hipGetLastError();
        return false;
    }
    const uint64_t bit = 1ull << dev;
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    done.fetch_or(bit, std::memory_order_release);
    return true;
}

// Pieces of a workspace, each on a 256-byte line.
class Carve {
public:
    explicit Carve(void* base) : base_((unsigned char*)base) {}
    template <typename T> T* take(size_t count)
    {
        T* p = base_ ? (T*)((uintptr_t)base_ + used_) : nullptr;
        used_ += (count * sizeof(T) + 255) / 256 * 256;
        return p;
    }
    size_t used() const { return used_; }
private:
    unsigned char* base_;
    size_t used_ = 0;
};

}  // namespace
