// The rotation table, and the RMS norm of queries and keys per head with the rotation in the same pass.
#include "mfma_util.h"
#include "paged.h"

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

// A wave per row, any even head size, any strides.
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

void launch_norm_rope(const NormRope& a, int dtype, hipStream_t s)
{
    const int64_t rows = (int64_t)a.n_tokens * (a.Hq + a.Hk);
    const dim3 grid((unsigned)(rows / 4 + 1 < 65536 ? rows / 4 + 1 : 65536));
    if (dtype == CASCADE_BF16) hipLaunchKernelGGL((norm_rope_any_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((norm_rope_any_kernel<float>), grid, dim3(256), 0, s, a);
}

}  // namespace ckv
