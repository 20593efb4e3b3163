// The rotation table, and the RMS norm of queries and keys per head with the rotation in the same pass.
#include "row_pieces.h"

namespace ckv {

// ------------------------------------------------------------------ rotation table
size_t rope_pair_table_bytes(int64_t n_positions, int head_dim)
{
    return (size_t)(256 + (n_positions + 255) / 256) * (size_t)(head_dim / 2) * sizeof(double2);
}

__global__ void rope_pair_table_kernel(double2* __restrict__ rope, int64_t entries, int half, double base)
{
    const int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (x >= entries) return;
    const int64_t row = x / half;
    const int i = (int)(x - row * half);
    const double p = row < 256 ? (double)row : 256.0 * (double)(row - 256);
    double s, c;
    sincos(p * pow(base, -(double)i / (double)half), &s, &c);
    rope[x] = make_double2(c, s);
}

void launch_rope_pair_table(double2* rope, int64_t n_positions, int head_dim, double base, hipStream_t s)
{
    const int half = head_dim / 2;
    const int64_t n = (256 + (n_positions + 255) / 256) * half;
    hipLaunchKernelGGL(rope_pair_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, rope, n, half, base);
}

// ------------------------------------------------------------------ norm and rotation
// The cosine and sine of a token's pair in 32 bits; NaN where the position is outside the table.
__device__ inline float2 cos_sin(const NormRope& a, int token, int i)
{
    const int p = a.positions[token];
    if (p < 0 || p >= a.rope_positions) return make_float2(f32_from_bits(0x7FC00000u), f32_from_bits(0x7FC00000u));
    const double2 cs = rope_entry(a.rope, a.d / 2, (uint32_t)p, i);
    return make_float2((float)cs.x, (float)cs.y);
}

__device__ inline void store_rounded(float* p, float x) { *p = x; }
__device__ inline void store_rounded(bf16_t* p, float x) { *p = (bf16_t)cvt_pk_bf16(x, x); }

// Any even head size, any strides: a wave per row, which makes its cosines and sines itself (4096 tokens of 40 heads, bf16: d 120 59 us, d 128 off the 16-byte grid 62; the form
// below, d 128: 18).
template <typename T> __global__ __launch_bounds__(256) void norm_rope_any_kernel(NormRope a)
{
    const int lane = threadIdx.x & 63, heads = a.Hq + a.Hk, half = a.d / 2;
    const int64_t rows = (int64_t)a.n_tokens * heads;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        const int t = (int)(row / heads), h = (int)(row - (int64_t)t * heads);
        const bool is_q = h < a.Hq;
        const T* x = is_q ? (const T*)a.q + t * a.q_stride + (int64_t)h * a.d : (const T*)a.k + t * a.k_stride + (int64_t)(h - a.Hq) * a.d;
        T* y = is_q ? (T*)a.q_out + t * a.q_out_stride + (int64_t)h * a.d : (T*)a.k_out + t * a.k_out_stride + (int64_t)(h - a.Hq) * a.d;
        const T* w = (const T*)(is_q ? a.q_weight : a.k_weight);
        float lo[2], hi[2], sum = 0.f;      // pairs lane and lane + 64
        for (int j = 0; j < 2; ++j) {
            const int i = lane + 64 * j;
            lo[j] = i < half ? Elem<T>::load(x + i) : 0.f;
            hi[j] = i < half ? Elem<T>::load(x + half + i) : 0.f;
            sum += lo[j] * lo[j] + hi[j] * hi[j];
        }
        if (a.norm) {
            for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
            const float r = 1.f / sqrtf(sum / (float)a.d + a.eps);
            for (int j = 0; j < 2; ++j) {
                const int i = lane + 64 * j;
                if (i >= half) continue;
                lo[j] *= r * (w ? Elem<T>::load(w + i) : 1.f);
                hi[j] *= r * (w ? Elem<T>::load(w + half + i) : 1.f);
            }
        }
        for (int j = 0; j < 2; ++j) {
            const int i = lane + 64 * j;
            if (i >= half) continue;
            const float2 cs = a.positions ? cos_sin(a, t, i) : make_float2(1.f, 0.f);
            store_rounded(y + i, a.positions ? rot_lo(lo[j], hi[j], cs.x, cs.y) : lo[j]);
            store_rounded(y + half + i, a.positions ? rot_hi(lo[j], hi[j], cs.x, cs.y) : hi[j]);
        }
    }
}

// Bound by memory: 4096 tokens of 32 + 8 heads, d 128, bf16 (84 MB) take 18.0 us in a row of calls, 4.66 TB/s; a large copy reaches 4.74.  One token takes the device 3.3 us and
// the caller 10.  (As above: 62 us.)
// Rows of whole 16-byte pieces, TPR threads a row (the first d / 16 of them work), each with 8 channels of the lower half and their partners of
// the upper half: the rotation needs no exchange.  A workgroup has all rows of `per` tokens (or, with more than 1024 / TPR rows a token, goes over
// them), whose cosines and sines are made once, in LDS, while the rows are on their way.
template <typename T, int TPR> __global__ __launch_bounds__(1024) void norm_rope_kernel(NormRope a, int per)
{
    extern __shared__ float2 cs[];      // [per][d / 2]
    const int half = a.d / 2, heads = a.Hq + a.Hk, t0 = blockIdx.x * per, tokens = min(per, a.n_tokens - t0);
    const int j = threadIdx.x % TPR, work = tokens * heads;
    const bool on = j < a.d / 16;
    int row = threadIdx.x / TPR;
    float lo[8], hi[8];
    const T* w = nullptr;
    T* y = nullptr;
    int t = 0;
    auto load = [&]() {
        t = row / heads;
        const int h = row - t * heads;
        const bool is_q = h < a.Hq;
        const int64_t at = t0 + t;
        const T* x = is_q ? (const T*)a.q + at * a.q_stride + h * a.d : (const T*)a.k + at * a.k_stride + (h - a.Hq) * a.d;
        y = is_q ? (T*)a.q_out + at * a.q_out_stride + h * a.d : (T*)a.k_out + at * a.k_out_stride + (h - a.Hq) * a.d;
        w = (const T*)(is_q ? a.q_weight : a.k_weight);
        load8(x + 8 * j, lo);
        load8(x + half + 8 * j, hi);
    };
    if (row < work && on) load();
    if (a.positions) {
        for (int i = threadIdx.x; i < tokens * half; i += blockDim.x) cs[i] = cos_sin(a, t0 + i / half, i % half);
        __syncthreads();
    }
    while (row < work) {
        if (a.norm) {
            float sum = 0.f;
            if (on)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += lo[e] * lo[e] + hi[e] * hi[e];
#pragma unroll
            for (int o = 1; o < TPR; o <<= 1) sum += __shfl_xor(sum, o);
            const float r = 1.f / sqrtf(sum / (float)a.d + a.eps);
            float wl[8], wh[8];
            if (w && on) {
                load8(w + 8 * j, wl);
                load8(w + half + 8 * j, wh);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo[e] *= w ? r * wl[e] : r;
                hi[e] *= w ? r * wh[e] : r;
            }
        }
        if (on) {
            if (a.positions)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 c = cs[t * half + 8 * j + e];
                    const float x = lo[e], z = hi[e];
                    lo[e] = rot_lo(x, z, c.x, c.y);
                    hi[e] = rot_hi(x, z, c.x, c.y);
                }
            store8(y + 8 * j, lo);
            store8(y + half + 8 * j, hi);
        }
        row += blockDim.x / TPR;
        if (row < work && on) load();
    }
}

template <typename T> static void launch_norm_rope_typed(const NormRope& a, hipStream_t s)
{
    const int heads = a.Hq + a.Hk;
    if (!a.vectors) {
        const int64_t blocks = ((int64_t)a.n_tokens * heads + 3) / 4;
        hipLaunchKernelGGL((norm_rope_any_kernel<T>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, a);
        return;
    }
    int tpr = 1;
    while (tpr < a.d / 16) tpr *= 2;
    // as many tokens as make 256 threads; a token with more than 1024 threads' rows is gone over in rounds
    const int each = heads * tpr, per = each >= 256 ? 1 : 256 / each, threads = (each * per + 63) / 64 * 64;
    const dim3 grid((a.n_tokens + per - 1) / per), block(threads > 1024 ? 1024 : threads);
    const size_t lds = (size_t)per * (a.d / 2) * sizeof(float2);
    switch (tpr) {
    case 1: hipLaunchKernelGGL((norm_rope_kernel<T, 1>), grid, block, lds, s, a, per); break;
    case 2: hipLaunchKernelGGL((norm_rope_kernel<T, 2>), grid, block, lds, s, a, per); break;
    case 4: hipLaunchKernelGGL((norm_rope_kernel<T, 4>), grid, block, lds, s, a, per); break;
    case 8: hipLaunchKernelGGL((norm_rope_kernel<T, 8>), grid, block, lds, s, a, per); break;
    default: hipLaunchKernelGGL((norm_rope_kernel<T, 16>), grid, block, lds, s, a, per); break;
    }
}

void launch_norm_rope(const NormRope& a, int dtype, hipStream_t s)
{
    if (dtype == CASCADE_BF16) launch_norm_rope_typed<bf16_t>(a, s);
    else launch_norm_rope_typed<float>(a, s);
}

}  // namespace ckv
