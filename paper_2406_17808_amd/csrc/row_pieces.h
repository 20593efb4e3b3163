// Rows in 16-byte pieces, as 32-bit numbers.
#pragma once

#include "mfma_util.h"
#include "paged.h"

namespace ckv {

// Eight consecutive elements at a 16-byte aligned place.
__device__ inline void load8(const bf16_t* p, float (&x)[8])
{
    const u32x4_t v = *(const u32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = f32_from_bits(v[i] << 16);
        x[2 * i + 1] = f32_from_bits(v[i] & 0xFFFF0000u);
    }
}
__device__ inline void load8(const float* p, float (&x)[8])
{
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ inline void store8(bf16_t* p, const float (&x)[8])
{
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
    *(u32x4_t*)p = v;
}
__device__ inline void store8(float* p, const float (&x)[8])
{
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

}  // namespace ckv
