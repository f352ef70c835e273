// What the libraries that answer with a model share: element types, moves within a wave, lists of columns, and the
// host's checks and launches.  Everything is private to the source that includes it.
#ifndef ALS_COMMON_H
#define ALS_COMMON_H

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "als_serve.h"

namespace {

constexpr int kWave = 64;

struct F16 { uint16_t bits; };
struct BF16 { uint16_t bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(F16 v) {
    return (float)__builtin_bit_cast(_Float16, v.bits);
}
__device__ __forceinline__ float to_float(BF16 v) {
    return __builtin_bit_cast(float, (uint32_t)v.bits << 16);
}
// A score that fmaxf may meet: of a signalling NaN it may make NaN, and lose the other operand; a quiet one it leaves out.
// (f16 scores are quiet from their conversion on.)
__device__ __forceinline__ float quiet(float v) { return __builtin_canonicalizef(v); }
// The nearest value of the type, ties to even.
__device__ __forceinline__ void from_float(float v, float* out) { *out = v; }
__device__ __forceinline__ void from_float(float v, F16* out) {
    *out = F16{__builtin_bit_cast(uint16_t, (_Float16)v)};
}
__device__ __forceinline__ void from_float(float v, BF16* out) {
    *out = BF16{__builtin_bit_cast(uint16_t, (__bf16)v)};
}

// Larger scores have larger keys; -0 has +0's.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) {
    const uint32_t b = key & 0x80000000u ? key ^ 0x80000000u : ~key;
    return __builtin_bit_cast(float, b);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp32(uint32_t v) {
    return __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, dpp32<0x111, 0xF>(v));
    v = max(v, dpp32<0x112, 0xF>(v));
    v = max(v, dpp32<0x114, 0xF>(v));
    v = max(v, dpp32<0x118, 0xF>(v));
    v = max(v, dpp32<0x142, 0xA>(v));
    v = max(v, dpp32<0x143, 0xC>(v));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float wave_max(float v) {      // NaN-free
    const uint32_t least = __builtin_bit_cast(uint32_t, -INFINITY);
#define ALS_STEP(CTRL, ROWS)                                                                                        \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(                                             \
                     (int)least, (int)__builtin_bit_cast(uint32_t, v), CTRL, ROWS, 0xF, false)))
    ALS_STEP(0x111, 0xF);
    ALS_STEP(0x112, 0xF);
    ALS_STEP(0x114, 0xF);
    ALS_STEP(0x118, 0xF);
    ALS_STEP(0x142, 0xA);
    ALS_STEP(0x143, 0xC);
#undef ALS_STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

__device__ __forceinline__ float limit_of(const float* each, float all, int64_t r) { return each ? each[r] : all; }

// A row's CSR row of columns to leave out.
struct Rated {
    const int64_t* ptr;
    const int32_t* idx;
    const int32_t* users;
    int64_t of;
    // false: the row's user does not exist
    __device__ __forceinline__ bool row(int64_t r, const int32_t** list, int64_t* count) const {
        *list = nullptr;
        *count = 0;
        if (!ptr) return true;
        const int64_t u = users ? (int64_t)users[r] : r;
        if (u < 0 || u >= of) return false;
        const int64_t first = ptr[u];
        *list = idx + first;
        *count = ptr[u + 1] - first;
        return true;
    }
};

// ---------------------------------------------------------------------------------- host --

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

size_t type_bytes(int dtype) { return dtype == ALS_F32 ? 4 : 2; }

// Bytes from the first element of a strided matrix to past its last.
uint64_t span_of(int64_t rows, int64_t cols, int64_t ld, size_t bytes) {
    return rows <= 0 || cols <= 0 ? 0 : ((uint64_t)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * bytes;
}

bool overlap(const void* a, uint64_t an, const void* b, uint64_t bn) {
    if (!a || !b || an == 0 || bn == 0) return false;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + bn && y < x + an;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        ok = (prev == dev) || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// What a device is: asked for once per device and process.
constexpr int kMaxDevices = 64;
struct DeviceInfo {
    std::mutex mu;
    bool known = false;
    int cus = 0;
};
DeviceInfo g_device[kMaxDevices];

int query_device(int device, int* cus) {
    int count = 0;
    if (hipGetDeviceCount(&count) != hipSuccess || device < 0 || device >= count || device >= kMaxDevices)
        return ALS_ERR_DEVICE;
    DeviceInfo& d = g_device[device];
    std::lock_guard<std::mutex> lock(d.mu);
    if (!d.known) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, device) != hipSuccess) return ALS_ERR_DEVICE;
        if (strncmp(prop.gcnArchName, "gfx950", 6) != 0) return ALS_ERR_DEVICE;
        d.cus = prop.multiProcessorCount;
        d.known = true;
    }
    *cus = d.cus;
    return ALS_OK;
}

// Lets a kernel use all of a CU's LDS; once per kernel and device.
template <typename Kernel>
void whole_lds(Kernel kernel, int device, std::atomic<uint64_t>* done) {
    if (done->load(std::memory_order_acquire) >> device & 1) return;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess)
        done->fetch_or(1ull << device, std::memory_order_release);
}

// A launch counts its threads in 32 bits: one of 2^32 or more fails or, worse, runs only what is left of the count and
// reports nothing.  fn(first, count) for parts of `total` rows, `most` at a time.
constexpr int64_t kMaxThreads = UINT32_MAX;
template <typename Fn>
void in_parts(int64_t total, int64_t most, Fn fn) {
    for (int64_t first = 0; first < total; first += most) fn(first, total - first < most ? total - first : most);
}

}  // namespace

#endif  // ALS_COMMON_H
