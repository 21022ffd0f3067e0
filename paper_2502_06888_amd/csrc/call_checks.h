// What the host code of the calls without a context shares: the error text of a thread, checks of pointers, the device of a call.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>

#include "../../include/moe.h"

namespace kcall {

struct CallError {
    char text[256];
    __attribute__((format(printf, 3, 4))) moe_status fail(moe_status s, const char* fmt, ...) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(text, sizeof text, fmt, ap);
        va_end(ap);
        return s;
    }
};

#define TRY(expr)                          \
    do {                                   \
        const moe_status s_ = (expr);      \
        if (s_ != MOE_OK) return s_;       \
    } while (0)

// Device of the tensors of a call: the first one sets it, the others have to be there too.
struct Where {
    CallError* error;
    int device = -1;
    moe_status on(const void* p, const char* name, unsigned align) {
        if (!p) return error->fail(MOE_ERR_INVALID_ARG, "%s is null", name);
        if (((uintptr_t)p & (align - 1)) != 0) return error->fail(MOE_ERR_INVALID_ARG, "%s is not aligned to %u bytes", name, align);
        hipPointerAttribute_t at;
        if (hipPointerGetAttributes(&at, p) != hipSuccess) {
            (void)hipGetLastError();
            return error->fail(MOE_ERR_INVALID_ARG, "%s is not device memory", name);
        }
        if (at.type != hipMemoryTypeDevice) return error->fail(MOE_ERR_INVALID_ARG, "%s is not device memory", name);
        if (device >= 0 && at.device != device) return error->fail(MOE_ERR_INVALID_ARG, "%s is on device %d, other tensors on %d", name, at.device, device);
        device = at.device;
        return MOE_OK;
    }
};

// The tensors' device for the time of the launches, where it is not the current one.
class OnDevice {
public:
    explicit OnDevice(int device) {
        if (hipGetDevice(&before_) != hipSuccess) before_ = device;
        if (before_ != device) failed_ = hipSetDevice(device) != hipSuccess;
        moved_ = before_ != device && !failed_;
    }
    ~OnDevice() {
        if (moved_) (void)hipSetDevice(before_);
    }
    bool failed() const { return failed_; }

private:
    int before_ = 0;
    bool moved_ = false, failed_ = false;
};

// Whether two of rows x heads pieces of `width` elements, at these strides, share an element.
inline bool pieces_overlap(int64_t rows, int64_t heads, int64_t row, int64_t head, int64_t width) {
    if ((heads > 1 && head < width) || (rows > 1 && row < width)) return true;
    if (rows <= 1 || heads <= 1) return false;
    typedef __int128 wide;  // any stride times any number of rows
    if (row >= (wide)(heads - 1) * head + width || head >= (wide)(rows - 1) * row + width) return false;  // one inside the other
    // `down` rows on and `back` heads back there is another piece, |down * row - back * head| away
    for (int64_t back = 1; back < heads; ++back) {
        const wide to = (wide)back * head;
        const int64_t down = (int64_t)(to / row);
        if (down >= 1 && down < rows && to - (wide)down * row < width) return true;
        if (down + 1 < rows && (wide)(down + 1) * row - to < width) return true;
    }
    return false;
}

}  // namespace kcall
