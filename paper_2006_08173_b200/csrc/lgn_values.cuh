// Runs of consecutive values of a matrix row in registers, shared by the quantisers.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_launch.h"

namespace lgn {

// Pattern of |x| if x is finite, else 0.
__device__ __forceinline__ uint32_t finite_abs(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float max_nan(float a, float b) {                          // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// N consecutive values of a row as they lie in memory: N words of fp32, N/2 of two bf16 each.  A value costs
// about six instructions per copy written, so bf16 stays packed for maxima and scaling.
template <int DT, int N> struct Values {
    static constexpr int kWords = DT == LGN_F32 ? N : N / 2;
    uint32_t w[kWords];

    // of which the first `valid` exist (others read as 0)
    template <bool VEC>
    __device__ __forceinline__ void load(const char *p, int valid) {
        if (VEC && valid >= N) {
            #pragma unroll
            for (int k = 0; k < kWords; k += 4)
                asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]) : "l"(p + 4 * k) : "memory");
            return;
        }
        #pragma unroll
        for (int k = 0; k < kWords; ++k) {
            w[k] = 0u;
            if constexpr (DT == LGN_F32) {
                if (k < valid) w[k] = ldro_u32(p + 4 * k);
            } else {
                if (2 * k < valid) w[k] = ldro_u16(p + 4 * k);
                if (2 * k + 1 < valid) w[k] |= ldro_u16(p + 4 * k + 2) << 16;
            }
        }
    }
    __device__ __forceinline__ float at(int k) const {
        if constexpr (DT == LGN_F32) return __uint_as_float(w[k]);
        else return k & 1 ? bf_hi(w[k >> 1]) : bf_lo(w[k >> 1]);
    }
    // fp32 pattern of the largest magnitude: at least 0x7f800000 if any value is not finite
    __device__ __forceinline__ uint32_t max_abs() const {
        if constexpr (DT == LGN_F32) {
            float m = fabsf(__uint_as_float(w[0]));
            #pragma unroll
            for (int k = 1; k < kWords; ++k) m = max_nan(m, fabsf(__uint_as_float(w[k])));
            return __float_as_uint(m) & 0x7fffffffu;
        } else {
            uint32_t m = w[0] & 0x7fff7fffu;
            #pragma unroll
            for (int k = 1; k < kWords; ++k) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
            return max(m << 16, m & 0xffff0000u);
        }
    }
    __device__ __forceinline__ uint32_t max_abs_finite() const {
        uint32_t a = 0;
        #pragma unroll
        for (int k = 0; k < N; ++k) a = max(a, finite_abs(at(k)));
        return a;
    }
};

}  // namespace lgn
