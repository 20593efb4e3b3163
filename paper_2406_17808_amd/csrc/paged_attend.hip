// Attention over the paged cache in 4 bits.
#include "mfma_util.h"
#include "paged.h"

namespace ckv {

// A wave per query row: 32 keys at a time, two lanes a key for the logits, then a lane per channel (two at D = 128).
template <typename T, int D> __global__ __launch_bounds__(64) void attend_row_kernel(PagedGeom g, PagedBatch b, const T* __restrict__ q, int64_t q_stride, T* __restrict__ out)
{
    __shared__ float qs[D], ps[32];
    const int lane = threadIdx.x, t = blockIdx.x, h = blockIdx.y, hk = h / g.G;
    const int s = seq_of_row(b, t);
    const SeqView v = seq_view(b, s);
    const int i = t - v.first, p = v.len + i;
    if (i < 0 || i >= v.n) return;
    for (int c = lane; c < D; c += 64) qs[c] = Elem<T>::load(q + t * q_stride + h * D + c) * g.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    const int from = g.window > 0 && p - g.window + 1 > 0 ? p - g.window + 1 : 0;
    for (int k0 = from & ~31; k0 <= p; k0 += 32) {
        const int64_t at = paged_group(g, b, s, k0);
        if (at < 0) continue;
        const uint8_t* group = g.pages + (at + (int64_t)hk * g.groups) * g.group_bytes;
        const int r = lane & 31;
        float x = 0.f;
        for (int blk = lane >> 5; blk < D / 32; blk += 2) {
            float part = 0.f;
            for (int c = 0; c < 32; ++c) part += qs[32 * blk + c] * fp4_value(group[k_code_byte(32 * blk + c, r)] >> (4 * (c & 1)));
            x += part * k_scale(group[k_exp_byte(D, blk, r)]);
        }
        x += __shfl_xor(x, 32);
        const bool seen = k0 + r >= from && k0 + r <= p && k0 + r < b.max_length;
        float top = seen ? x : -INFINITY;
        for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
        const float mn = fmaxf(m, top), shrink = mn == -INFINITY ? 1.f : expf(m - mn);
        const float e = seen ? expf(x - mn) : 0.f;
        float sum = e;
        for (int w = 16; w; w >>= 1) sum += __shfl_xor(sum, w);
        l = l * shrink + sum;
        m = mn;
        __syncthreads();
        if (lane < 32) ps[r] = seen ? e * bf16_to_f32(*(const bf16_t*)(group + v_scale_byte(D, r))) : 0.f;
        __syncthreads();
        for (int y = 0; y < D / 64; ++y) {
            const int c = lane + 64 * y;
            float acc = o[y] * shrink;
            for (int k = 0; k < 32; ++k) acc += ps[k] * fp4_value(group[v_code_byte(D, c >> 5, c & 15, k)] >> (4 * ((c >> 4) & 1)));
            o[y] = acc;
        }
    }
    for (int y = 0; y < D / 64; ++y) Elem<T>::store(out + ((int64_t)t * g.Hq + h) * D + lane + 64 * y, l == 0.f ? 0.f : o[y] / l);
}

size_t paged_scratch_bytes(const PagedGeom&) { return 256; }

void launch_paged_attend(const PagedGeom& g, const PagedBatch& b, const void* q, int64_t q_stride, void* out, void*, int dtype, hipStream_t s)
{
    const dim3 grid(b.n_tokens, g.Hq), block(64);
    with_paged_form(dtype, g.d, [&](auto f) {
        typedef typename decltype(f)::Elt T;
        hipLaunchKernelGGL((attend_row_kernel<T, decltype(f)::d>), grid, block, 0, s, g, b, (const T*)q, q_stride, (T*)out);
    });
}

}  // namespace ckv
