// lpv_attention.h -- device helpers shared by the attention kernels (gfx950 only).
#pragma once

#include "lpv_device.h"

namespace lpv {

typedef short att_v4s __attribute__((ext_vector_type(4)));
typedef unsigned int att_u4 __attribute__((ext_vector_type(4)));

__device__ inline uint2 att_tr_read(uint32_t addr)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) att_v4s*)(uintptr_t)addr));
}

// c + the two 16-bit values packed in p (one dot product with (1, 1): the
// products are exact, the sum is float32)
template <int DT> __device__ inline float att_add2(uint32_t p, float c)
{
    if (DT == 2)  // bf16
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p),
                                               __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, p), __builtin_bit_cast(f16x2, 0x3c003c00u),
                                  c, false);
}

__device__ inline uint4 att_read16(uint32_t addr)
{
    return __builtin_bit_cast(uint4, *(const __attribute__((address_space(3))) att_u4*)(uintptr_t)addr);
}

// The same as an operand (read as the vector that it is: taken apart and put together, the
// load may become four).
template <typename F> __device__ inline F att_frag(uint32_t addr)
{
    return *(const __attribute__((address_space(3))) F*)(uintptr_t)addr;
}

}  // namespace lpv
