// The two 16-bit types of the serving operators: DT 1 f16, 2 bf16, as in
// ecasq_dtype.  Values travel as their bit patterns.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ecasq {

template <int DT>
__device__ __forceinline__ float from16(uint32_t h) {
    if (DT == 2) return __uint_as_float(h << 16);
    const uint16_t b = (uint16_t)h;
    return (float)__builtin_bit_cast(_Float16, b);
}

// Round to nearest, ties to even.
template <int DT>
__device__ __forceinline__ uint16_t to16(float f) {
    if (DT == 2) return __builtin_bit_cast(uint16_t, (__bf16)f);
    return __builtin_bit_cast(uint16_t, (_Float16)f);
}

// A double rounded once: through the float between it and zero whose last bit
// is set where the value is not a float (the float's 24 bits are two more than
// the 16-bit types need for that).
template <int DT>
__device__ __forceinline__ uint16_t to16(double q) {
    float f = (float)q;
    if (f == f && (double)f != q) {
        uint32_t b = __float_as_uint(f);
        if (__builtin_fabs((double)f) > __builtin_fabs(q)) b--;
        f = __uint_as_float(b | 1u);
    }
    return to16<DT>(f);
}

template <int DT>
constexpr uint16_t kNan16 = DT == 2 ? 0x7FC0u : 0x7E00u;

}  // namespace ecasq
