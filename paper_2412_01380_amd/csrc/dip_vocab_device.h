// What the kernels over rows of a vocabulary share (verification, sampling): loads of a row that starts anywhere, sums and
// running sums in fp64.
#ifndef DIP_VOCAB_DEVICE_H_
#define DIP_VOCAB_DEVICE_H_

#include "dip_decode_internal.h"

namespace dip {

constexpr int kPer = 16;                  // entries of a thread at a time: in flight together

template <typename E>
__device__ __forceinline__ float entry_at(const char* row, int x);
template <>
__device__ __forceinline__ float entry_at<float>(const char* row, int x) { return ((const float*)row)[x]; }
template <>
__device__ __forceinline__ float entry_at<uint16_t>(const char* row, int x) {
    return __uint_as_float((uint32_t)((const uint16_t*)row)[x] << 16);
}
// kPer entries of a row from x on, widened (exactly); zeros from `end` on.  Rows of an odd vocabulary start
// anywhere: 16-byte loads that ask for no more than E's alignment.
template <typename E>
__device__ __forceinline__ void load_entries(const char* row, int x, int end, float (&f)[kPer]) {
    constexpr int N = 16 / sizeof(E);
    struct __attribute__((packed, aligned(sizeof(E)))) Any { uint32_t w[4]; };
    if (x + kPer <= end) {
#pragma unroll
        for (int y = 0; y < kPer / N; ++y) {
            const Any r = *(const Any*)(row + (size_t)(x + y * N) * sizeof(E));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(E) == 4) {
                    f[y * N + i] = __uint_as_float(r.w[i]);
                } else {
                    f[y * N + 2 * i] = __uint_as_float(r.w[i] << 16);
                    f[y * N + 2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) f[i] = x + i < end ? entry_at<E>(row, x + i) : 0.f;
    }
}

// inclusive running sums over a wavefront: data-parallel moves within rows of 16 lanes, then the rows' sums by scalar
template <int CTRL>
__device__ __forceinline__ double moved(double x) {
    const uint64_t b = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double of_lane(double x, int lane) {
    const uint64_t b = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __longlong_as_double(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double in_rows(double x) {
    x += moved<0x111>(x);                             // row_shr 1, 2, 4, 8
    x += moved<0x112>(x);
    x += moved<0x114>(x);
    return x + moved<0x118>(x);
}
__device__ __forceinline__ double running(double x) {
    x = in_rows(x);
    const double a = of_lane(x, 15), b = of_lane(x, 31), c = of_lane(x, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row == 0 ? 0.0 : row == 1 ? a : row == 2 ? a + b : a + b + c);
}
__device__ __forceinline__ int running(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    const int a = __builtin_amdgcn_readlane(x, 15), b = __builtin_amdgcn_readlane(x, 31), c = __builtin_amdgcn_readlane(x, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row > 0 ? a : 0) + (row > 1 ? b : 0) + (row > 2 ? c : 0);
}
__device__ __forceinline__ uint32_t running(uint32_t x) { return (uint32_t)running((int)x); }
__device__ __forceinline__ double wave_sum(double x) {
    x = in_rows(x);
    return of_lane(x, 15) + of_lane(x, 31) + of_lane(x, 47) + of_lane(x, 63);
}
// sum over the workgroup, in thread 0
__device__ __forceinline__ double block_sum(double x, double* waves) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += waves[w];
    return s;
}

__device__ __forceinline__ void put(double* to, double x) { __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double get(const double* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

}  // namespace dip

#endif  // DIP_VOCAB_DEVICE_H_
